"""Cases of the attention-side operators: norms and rotation of queries and keys (with the backward pass), appending
to a paged cache, and attention of a batch that shares a prefix.

``run`` computes a case in plain form (elementary torch operations in 32 bits, one rounding at the end) or, where
``own`` is true, through the library's entry points; ``exact`` gives the same outputs from the definitions in 64 bits.

Heads follow the linear layers they sit between: queries, keys and values are column ranges of one stacked projection
[tokens x (Hq + 2 Hkv) D], so every operator sees rows with a pitch.  32 query and 32 key heads of 128 and 40 of each are
the 7B and 13B shapes of this repository's workloads; 32 with 8 and heads of 64 are the grouped and the small form.
"""
import math

import torch

own = False

BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


# ---------------------------------------------------------------------------------------------
# cases

def listed():
    return [
        # training: the norms and the rotation before attention, one short packed sequence
        dict(name="norm_rope.m509", op="norm_rope", M=509, Hq=32, Hkv=32, D=128, R=128, inter=False, norm=True),
        # training: a micro-batch of 8 sequences of 2048 tokens with grouped heads
        dict(name="norm_rope.m16384", op="norm_rope", M=16384, Hq=32, Hkv=8, D=128, R=128, inter=False, norm=True),
        # training: the gradient of the same for one sequence of the 13B shape, an odd number of tokens
        dict(name="norm_rope_bwd.m2047", op="norm_rope_bwd", M=2047, Hq=40, Hkv=40, D=128, R=128, inter=False, norm=True),
        # training: the gradient for the micro-batch, heads of 64 with half of them rotated, pairs interleaved
        dict(name="norm_rope_bwd.m16384", op="norm_rope_bwd", M=16384, Hq=32, Hkv=8, D=64, R=32, inter=True, norm=True),
        # serving, latency: one token of one sequence appended, 7B heads, rotation only
        dict(name="append.m1", op="append", M=1, Hq=32, Hkv=32, D=128, R=128, inter=False, norm=False, page=16),
        # serving: a decode step of 64 sequences, grouped heads with norms
        dict(name="append.m64", op="append", M=64, Hq=32, Hkv=8, D=128, R=128, inter=False, norm=True, page=32),
        # serving: the prompt of a 13B-shaped model written to the cache, an odd number of tokens
        dict(name="append.m8191", op="append", M=8191, Hq=40, Hkv=40, D=128, R=128, inter=False, norm=False, page=16),
        # serving, latency: one sequence just after its prompt
        dict(name="attn.b1.p128", op="attn", B=1, T=1, Hq=32, Hkv=32, D=128, P=128, lo=64, hi=64, page=16, lse=False),
        # serving: batch 16 behind a system prompt, 7B heads, up to 1024 tokens generated
        dict(name="attn.b16.p2048", op="attn", B=16, T=1, Hq=32, Hkv=32, D=128, P=2048, lo=1, hi=1024, page=16, lse=False),
        # serving: five drafted tokens per sequence to be scored at once, grouped heads, odd lengths
        dict(name="attn.b16.t5.p4093", op="attn", B=16, T=5, Hq=32, Hkv=8, D=128, P=4093, lo=5, hi=777, page=32, lse=True),
        # serving: 13B heads behind a few-shot prompt
        dict(name="attn.b32.p8192", op="attn", B=32, T=1, Hq=40, Hkv=40, D=128, P=8192, lo=17, hi=513, page=16, lse=False),
        # serving: many sequences over one long document, grouped heads
        dict(name="attn.b64.p32768", op="attn", B=64, T=1, Hq=32, Hkv=8, D=128, P=32768, lo=33, hi=2048, page=64, lse=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rope", "norm_rope_bwd", "append", "attn", "attn", "attn"])
    D = rng.choice([64, 128, 128])
    Hq, Hkv = rng.choice([(32, 32), (32, 8), (40, 40), (16, 2), (24, 8), (8, 1)])
    if op != "attn":
        R = rng.choice([D, D, D // 2])
        case = dict(op=op, M=_log(rng, 1, 8191 if op == "append" else 16384), Hq=Hq, Hkv=Hkv, D=D, R=R,
                    inter=rng.random() < 0.3, norm=op == "norm_rope_bwd" or rng.random() < 0.6)
        if op == "append":
            case["page"] = rng.choice([16, 32, 64, 128])
        while case["M"] * (Hq + Hkv) * D > 16384 * 40 * 128:
            case["M"] = case["M"] * 3 // 4
        return case
    case = dict(op="attn", B=_log(rng, 1, 128), T=rng.choice([1, 1, 1, 2, 4, 7]), Hq=Hq, Hkv=Hkv, D=D,
                P=rng.choice([0, 1, 1, 1]) * _log(rng, 1, 32768), hi=_log(rng, 8, 4096), page=rng.choice([16, 32, 64, 128]),
                lse=rng.random() < 0.3)
    case["lo"] = rng.randint(0, case["hi"])
    top = work(listed()[-1])
    while True:
        w = work(case)
        if w["bytes"] <= 0.9 * top["bytes"] and w["flops"] <= 0.9 * top["flops"] and case["B"] * case["hi"] * Hkv * D <= 64 * 2048 * 8 * 128:
            return case
        case["B"], case["hi"], case["P"] = max(1, case["B"] * 3 // 4), max(8, case["hi"] * 7 // 8), case["P"] * 7 // 8
        case["lo"] = min(case["lo"], case["hi"])


def _lens(c):
    """The sequences' own lengths, spread evenly between lo and hi; which sequence has which is the seed's."""
    return [c["lo"] + (c["hi"] - c["lo"]) * (i + 1) // c["B"] for i in range(c["B"])]


def work(c):
    if c["op"] != "attn":
        q, k = c["M"] * c["Hq"] * c["D"] * 2, c["M"] * c["Hkv"] * c["D"] * 2
        table = c["M"] * (c["R"] * 4 + 4)
        if c["op"] == "norm_rope":
            return {"bytes": 2 * (q + k) + table, "flops": 5 * (q + k)}
        if c["op"] == "norm_rope_bwd":
            return {"bytes": 3 * (q + k) + table, "flops": 8 * (q + k)}
        return {"bytes": 2 * (q + 2 * k) + table + c["M"] * 8, "flops": 5 * (q + k)}
    keys, pairs = c["P"] + sum(_lens(c)), 0
    for n in _lens(c):
        for t in range(c["T"]):
            pairs += c["P"] + max(0, n - (c["T"] - 1 - t))
    rows = c["B"] * c["T"] * c["Hq"]
    return {"bytes": keys * c["Hkv"] * c["D"] * 4 + rows * c["D"] * 4 + rows * 4 * c["lse"] + keys // c["page"] * 4,
            "flops": 4 * pairs * c["Hq"] * c["D"]}


# ---------------------------------------------------------------------------------------------
# what a program has in hand

def _rope_table(n, R, dev):
    """Cosines, then sines, of every position: the usual frequencies 10000^(-2 i / R)."""
    freq = 10000.0 ** (-torch.arange(0, R, 2, dtype=F64, device=dev) / R)
    angle = torch.arange(n, dtype=F64, device=dev)[:, None] * freq[None, :]
    return torch.cat((angle.cos(), angle.sin()), dim=1).to(F32)


def _split(x, Hq, Hkv, D):
    """Column ranges of a stacked projection as heads: q [M, Hq, D], k and v [M, Hkv, D], all with the stack's pitch."""
    return (x[:, : Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D : (Hq + Hkv) * D].unflatten(1, (Hkv, D)),
            x[:, (Hq + Hkv) * D :].unflatten(1, (Hkv, D)))


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    randn = lambda *s, dtype=BF16: torch.randn(*s, generator=g, device=dev, dtype=F32).to(dtype)  # noqa: E731
    s = dict(case=c, Hq=c["Hq"], Hkv=c["Hkv"], D=c["D"])
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["op"] != "attn":
        M = c["M"]
        s["qkv"] = randn(M, (Hq + 2 * Hkv) * D) * (1.0 + 0.5 * torch.rand(M, 1, generator=g, device=dev)).to(BF16)
        s["q"], s["k"], s["v"] = _split(s["qkv"], Hq, Hkv, D)
        s["wq"], s["wk"] = (1 + 0.2 * randn(D, dtype=F32)).to(BF16), (1 + 0.2 * randn(D, dtype=F32)).to(BF16)
        if not c["norm"]:
            s["wq"] = s["wk"] = None
        s["cos_sin"] = _rope_table(4096, c["R"], dev)
        if c["op"] == "append" and M <= 128:      # a decode step: every sequence at a place of its own
            s["pos"] = torch.randint(0, 4096, (M,), generator=g, device=dev, dtype=I32)
        else:                                     # sequences packed one after the other
            s["pos"] = (torch.arange(M, device=dev) % 2048).to(I32)
        s["qo"], s["ko"] = torch.empty(M, Hq, D, dtype=BF16, device=dev), torch.empty(M, Hkv, D, dtype=BF16, device=dev)
        if c["op"] == "norm_rope_bwd":
            s["gqo"], s["gko"] = randn(M, Hq, D), randn(M, Hkv, D)
            s["gq"], s["gk"] = torch.empty_like(s["qo"]), torch.empty_like(s["ko"])
            s["gwq"], s["gwk"] = torch.empty(D, dtype=F32, device=dev), torch.empty(D, dtype=F32, device=dev)
        if c["op"] == "append":
            pages = (M + c["page"] - 1) // c["page"] + 3 if M > 128 else M + 3
            s["kc"], s["vc"] = randn(pages, Hkv, c["page"], D), randn(pages, Hkv, c["page"], D)
            if M > 128:                           # a prompt fills whole pages, in any order
                order = torch.randperm(pages, generator=g, device=dev)
                at = torch.arange(M, device=dev)
                s["slots"] = order[at // c["page"]] * c["page"] + at % c["page"]
            else:                                 # a decode step: one slot in a page of each sequence
                s["slots"] = (torch.randperm(pages, generator=g, device=dev)[:M] * c["page"]
                              + torch.randint(0, c["page"], (M,), generator=g, device=dev))
    else:
        B, T, P, page = c["B"], c["T"], c["P"], c["page"]
        lens = torch.tensor(_lens(c), dtype=I32, device=dev)[torch.randperm(B, generator=g, device=dev)]
        width = max(1, (c["hi"] + page - 1) // page)
        used = (P + page - 1) // page
        pool = used + int(((lens + page - 1) // page).sum()) + 2
        s["kc"], s["vc"] = randn(pool, Hkv, page, D), randn(pool, Hkv, page, D)
        order = torch.randperm(pool, generator=g, device=dev).to(I32)
        s["prefix_pages"] = order[:used].clone()
        count = (lens + page - 1) // page
        first = used + torch.cumsum(count, 0) - count
        at = torch.arange(width, device=dev)[None, :]
        table = order[(first[:, None] + at).clamp(max=pool - 1).long()]
        s["table"] = torch.where(at < count[:, None], table, torch.full_like(table, -1)).contiguous()
        s["lens"] = lens
        s["q"] = _split(1.5 * randn(B * T, (Hq + 2 * Hkv) * D), Hq, Hkv, D)[0]
        s["o"] = torch.empty(B * T, Hq, D, dtype=BF16, device=dev)
        s["lse"] = torch.empty(B * T, Hq, dtype=F32, device=dev) if c["lse"] else None
    if own:
        from paper_2509_23410_b200 import binding as L
        s["L"] = L
        if "cos_sin" in s:
            s["rope"] = L.patch_rope(s["cos_sin"], interleaved=c["inter"])
        if "kc" in s:
            s["cache"] = L.patch_kv_cache(s["kc"], s["vc"])
        if c["op"] == "norm_rope_bwd":
            n = L.patch_qk_norm_rope_backward_workspace_size(c["M"], Hq, Hkv, D)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=dev)
            L.patch_workspace_init(s["ws"])
        if c["op"] == "attn":
            n = L.patch_prefix_attention_workspace_size(s["cache"], c["B"], c["T"], Hq)
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=dev)
            L.patch_workspace_init(s["ws"])
    return s


# ---------------------------------------------------------------------------------------------
# one pass

EPS = 1e-6


def run(s):
    c = s["case"]
    return (_run_own if own else _run_plain)(s, c)


def _run_own(s, c):
    L = s["L"]
    if c["op"] == "norm_rope":
        L.patch_qk_norm_rope(s["q"], s["k"], s["rope"], s["pos"], wq=s["wq"], wk=s["wk"], eps=EPS, Q_out=s["qo"], K_out=s["ko"])
        return {"q": s["qo"], "k": s["ko"]}
    if c["op"] == "norm_rope_bwd":
        L.patch_qk_norm_rope_backward(s["gqo"], s["gko"], s["rope"], s["pos"], Q=s["q"], K=s["k"], wq=s["wq"], wk=s["wk"],
                                      eps=EPS, gQ=s["gq"], gK=s["gk"], gwq=s["gwq"], gwk=s["gwk"], workspace=s["ws"])
        return {"gq": s["gq"], "gk": s["gk"], "gwq": s["gwq"], "gwk": s["gwk"]}
    if c["op"] == "append":
        L.patch_kv_append(s["cache"], s["k"], s["v"], s["slots"], rope=s["rope"], positions=s["pos"], wk=s["wk"], eps=EPS,
                          Q=s["q"], wq=s["wq"], Q_out=s["qo"])
        return {"q": s["qo"], "kc": s["kc"], "vc": s["vc"]}
    L.patch_prefix_attention(s["cache"], s["q"], s["prefix_pages"], c["P"], s["table"], s["lens"], O=s["o"], lse=s["lse"],
                             workspace=s["ws"])
    return {"o": s["o"], "lse": s["lse"]} if c["lse"] else {"o": s["o"]}


def _cos_sin(s, c, f):
    t = s["cos_sin"].to(f)[s["pos"].long()]
    return t[:, None, : c["R"] // 2], t[:, None, c["R"] // 2 :]


def _turn(x, cos, sin, R, inter):
    """The pairs (i, i + R/2), or (2i, 2i + 1), of the first R elements of each head turned by the position's angles."""
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if inter else (x[..., : R // 2], x[..., R // 2 : R])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., R:]), -1)


def _norm_turn(x, w, s, c):
    y = x.to(F32)
    if w is not None:
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w.to(F32)
    return _turn(y, *_cos_sin(s, c, F32), c["R"], c["inter"])


def _norm_turn_bwd(gy, x, w, s, c):
    cos, sin = _cos_sin(s, c, F32)
    g = _turn(gy.to(F32), cos, -sin, c["R"], c["inter"])
    x = x.to(F32)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    xh, gn = x * r, g * w.to(F32)
    return (r * (gn - xh * (gn * xh).mean(-1, keepdim=True))).to(BF16), (g * xh).sum((0, 1))


def _run_plain(s, c):
    if c["op"] == "norm_rope":
        return {"q": _norm_turn(s["q"], s["wq"], s, c).to(BF16), "k": _norm_turn(s["k"], s["wk"], s, c).to(BF16)}
    if c["op"] == "norm_rope_bwd":
        gq, gwq = _norm_turn_bwd(s["gqo"], s["q"], s["wq"], s, c)
        gk, gwk = _norm_turn_bwd(s["gko"], s["k"], s["wk"], s, c)
        return {"gq": gq, "gk": gk, "gwq": gwq, "gwk": gwk}
    if c["op"] == "append":
        page, at = s["slots"] // c["page"], s["slots"] % c["page"]
        s["kc"][page, :, at] = _norm_turn(s["k"], s["wk"], s, c).to(BF16)
        s["vc"][page, :, at] = s["v"]
        return {"q": _norm_turn(s["q"], s["wq"], s, c).to(BF16), "kc": s["kc"], "vc": s["vc"]}
    # attention: the batch's rows against the prefix as one product per key head, against their own pages as another
    B, T, P, Hq, Hkv, D = c["B"], c["T"], c["P"], s["Hq"], s["Hkv"], s["D"]
    G, dev = Hq // Hkv, s["q"].device
    q = s["q"].to(F32).view(B, T, Hkv, G, D) * (D ** -0.5)
    qp = q.permute(2, 0, 1, 3, 4).reshape(Hkv, B * T * G, D)
    kp, vp = (x[s["prefix_pages"].long()].transpose(0, 1).flatten(1, 2)[:, :P].to(F32) for x in (s["kc"], s["vc"]))
    sp = (qp @ kp.transpose(1, 2)).view(Hkv, B, T, G, P).permute(1, 0, 2, 3, 4)                   # [B, Hkv, T, G, P]
    pages = s["table"].clamp(min=0).long()
    ks, vs = (x[pages].transpose(1, 2).flatten(2, 3).to(F32) for x in (s["kc"], s["vc"]))
    n = ks.shape[2]
    ss = (q.transpose(1, 2).reshape(B, Hkv, T * G, D) @ ks.transpose(2, 3)).view(B, Hkv, T, G, n)
    sees = s["lens"].long()[:, None] - (T - 1 - torch.arange(T, device=dev))[None, :]             # [B, T]
    ss = torch.where(torch.arange(n, device=dev) < sees[:, None, :, None, None], ss, torch.full_like(ss, -torch.inf))
    m = ss.amax(-1, keepdim=True)
    if P:
        m = torch.maximum(m, sp.amax(-1, keepdim=True))
    m0 = torch.where(m > -torch.inf, m, torch.zeros_like(m))
    ep, es = torch.exp(sp - m0), torch.exp(ss - m0)
    den = ep.sum(-1, keepdim=True) + es.sum(-1, keepdim=True)
    o = (es.view(B, Hkv, T * G, n) @ vs).view(B, Hkv, T, G, D)
    o = o + (ep.permute(1, 0, 2, 3, 4).reshape(Hkv, B * T * G, P) @ vp).view(Hkv, B, T, G, D).transpose(0, 1)
    o = torch.where(den > 0, o / den, torch.zeros_like(o))
    out = {"o": o.transpose(1, 2).reshape(B * T, Hq, D).to(BF16)}
    if c["lse"]:
        out["lse"] = (m0 + torch.log(den)).squeeze(-1).transpose(1, 2).reshape(B * T, Hq)
    return out


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_rotation(s, c):
    """The R x R rotation of every token, as matrices [M, D, D]."""
    M, D, R = c["M"], c["D"], c["R"]
    t = s["cos_sin"].to(F64)[s["pos"].long()]
    cos, sin = t[:, : R // 2], t[:, R // 2 :]
    i = torch.arange(R // 2, device=t.device)
    a, b = (2 * i, 2 * i + 1) if c["inter"] else (i, i + R // 2)
    m = torch.zeros(M, D, D, dtype=F64, device=t.device)
    rest = torch.arange(R, D, device=t.device)
    m[:, a, a], m[:, b, b], m[:, a, b], m[:, b, a] = cos, cos, -sin, sin
    m[:, rest, rest] = 1.0
    return m


def _exact_heads(s, c, rot, x, w):
    y = x.to(F64)
    if w is not None:
        y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["D"] + EPS) * w.to(F64)
    return torch.einsum("mij,mhj->mhi", rot, y)


def _exact_heads_bwd(s, c, rot, gy, x, w):
    D = c["D"]
    g = torch.einsum("mij,mhi->mhj", rot, gy.to(F64))
    x = x.to(F64)
    n = torch.sqrt((x * x).sum(-1, keepdim=True) / D + EPS)
    gw = g * w.to(F64)
    return gw / n - x * (gw * x).sum(-1, keepdim=True) / (D * n ** 3), torch.einsum("mhd,mhd->d", g, x / n)


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"] != "attn":
        # in blocks of tokens: a rotation is a D x D matrix for each
        parts = []
        for lo in range(0, c["M"], 2048):
            hi = min(c["M"], lo + 2048)
            b = dict(c, M=hi - lo)
            t = dict(s, pos=s["pos"][lo:hi])
            rot = _exact_rotation(t, b)
            if c["op"] == "norm_rope_bwd":
                parts.append(_exact_heads_bwd(t, b, rot, s["gqo"][lo:hi], s["q"][lo:hi], s["wq"])
                             + _exact_heads_bwd(t, b, rot, s["gko"][lo:hi], s["k"][lo:hi], s["wk"]))
            else:
                parts.append((_exact_heads(t, b, rot, s["q"][lo:hi], s["wq"]), _exact_heads(t, b, rot, s["k"][lo:hi], s["wk"])))
        if c["op"] == "norm_rope_bwd":
            gq, gwq, gk, gwk = zip(*parts)
            return {"gq": torch.cat(gq), "gk": torch.cat(gk), "gwq": sum(gwq), "gwk": sum(gwk)}
        q, k = (torch.cat(x) for x in zip(*parts))
        if c["op"] == "norm_rope":
            return {"q": q, "k": k}
        kc, vc = s["kc"].to(F64), s["vc"].to(F64)
        for h in range(c["Hkv"]):
            kc[s["slots"] // c["page"], h, s["slots"] % c["page"]] = k[:, h]
            vc[s["slots"] // c["page"], h, s["slots"] % c["page"]] = s["v"][:, h].to(F64)
        return {"q": q, "kc": kc, "vc": vc}
    # attention: every sequence by itself over its keys written out in a row
    B, T, P, Hq, Hkv, D = c["B"], c["T"], c["P"], c["Hq"], c["Hkv"], c["D"]
    o = torch.zeros(B * T, Hq, D, dtype=F64, device="cuda")
    lse = torch.full((B * T, Hq), -torch.inf, dtype=F64, device="cuda")
    lens = s["lens"].tolist()
    for b in range(B):
        used = (lens[b] + c["page"] - 1) // c["page"]
        own_pages = s["table"][b, :used].long()
        k, v = (torch.cat((x[s["prefix_pages"].long()].permute(1, 0, 2, 3).flatten(1, 2)[:, :P],
                           x[own_pages].permute(1, 0, 2, 3).flatten(1, 2)[:, : lens[b]]), 1).to(F64)
                for x in (s["kc"], s["vc"]))
        for t in range(T):
            n = P + max(0, lens[b] - (T - 1 - t))
            if n == 0:
                continue
            q = s["q"][b * T + t].to(F64).view(Hkv, Hq // Hkv, D)
            z = torch.einsum("hgd,hnd->hgn", q, k[:, :n]) / math.sqrt(D)
            top = z.amax(-1, keepdim=True)
            e = (z - top).exp()
            den = e.sum(-1, keepdim=True)
            o[b * T + t] = (torch.einsum("hgn,hnd->hgd", e, v[:, :n]) / den).reshape(Hq, D)
            lse[b * T + t] = (top + den.log()).reshape(Hq)
    return {"o": o, "lse": lse} if c["lse"] else {"o": o}
