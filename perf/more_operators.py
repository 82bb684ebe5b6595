"""Cases of the operators between the masked weights and the loss of a training step: attention within packed sequences (with its
backward pass), log probabilities of given tokens with entropy and top alternatives (with their gradient), and distillation from a
teacher's top logits (loss and gradient).

``run`` computes a case in plain form (elementary torch operations in 32 bits, one rounding at the end) or, where
``own`` is true, through the library's entry points; ``exact`` gives the same outputs from the definitions in 64 bits.

Queries, keys and values are column ranges of one stacked projection [tokens x (Hq + 2 Hkv) D], as the linear layers leave them.
Logits have a pitch that is a multiple of eight; vocabularies are generic: 32000, 50257, 128256 and 151936 tokens.
"""
import math

import torch

own = False

BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


# ---------------------------------------------------------------------------------------------
# cases

def listed():
    return [
        # serving, latency: the alternatives of one token
        dict(name="logp.m1.v128256", op="logp", M=1, V=128256, f32=False, k=20, entropy=False, tokens=True, temp=1.0),
        # serving: a decode batch with entropy and a few alternatives at a temperature
        dict(name="logp.m61.v151936", op="logp", M=61, V=151936, f32=False, k=8, entropy=True, tokens=True, temp=0.7),
        # evaluation: log probabilities of a text under the masked model (perplexity)
        dict(name="logp.m8192.v32000", op="logp", M=8192, V=32000, f32=False, k=0, entropy=False, tokens=True, temp=1.0),
        # distillation, teacher's side: the top 64 of every position, logits in 32 bits
        dict(name="logp.m4095.v128256", op="logp", M=4095, V=128256, f32=True, k=64, entropy=False, tokens=False, temp=2.0),
        # training: gradient of log probabilities and entropy, an odd vocabulary
        dict(name="logp_bwd.m4096.v50257", op="logp_bwd", M=4096, V=50257, f32=False, entropy=True, temp=1.0),
        # distillation of a short packed sequence, logits in 32 bits, renormalised teacher
        dict(name="distill.m509.v32000", op="distill", M=509, V=32000, f32=True, K=32, rest=False, temp=1.0),
        # distillation of a micro-batch: loss (the cross entropy) and gradient, the teacher's remaining mass as one more class
        dict(name="distill.m8192.v128256", op="distill", M=8192, V=128256, f32=False, K=64, rest=True, temp=2.0),
        # training or scoring, latency: a few short sequences
        dict(name="attn.m300.b7", op="attn", M=300, tail=0, B=7, skew=1.0, Hq=32, Hkv=32, D=128),
        # a long prompt with grouped heads, an odd number of tokens
        dict(name="attn.m8191.b1", op="attn", M=8191, tail=0, B=1, skew=0.0, Hq=32, Hkv=8, D=128),
        # training: a micro-batch of ragged sequences, 13B heads
        dict(name="attn.m16384.b23", op="attn", M=16384, tail=0, B=23, skew=0.7, Hq=40, Hkv=40, D=128),
        # training: the gradient for ragged sequences in a padded buffer, grouped heads of 64
        dict(name="attn_bwd.m4001.b9", op="attn_bwd", M=4001, tail=95, B=9, skew=1.0, Hq=32, Hkv=8, D=64),
        # training: the gradient for a micro-batch of four sequences of 2048, 7B heads
        dict(name="attn_bwd.m8192.b4", op="attn_bwd", M=8192, tail=0, B=4, skew=0.0, Hq=32, Hkv=32, D=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logp", "logp", "logp_bwd", "distill", "distill", "attn", "attn", "attn_bwd", "attn_bwd"])
    if op.startswith("attn"):
        Hq, Hkv = rng.choice([(32, 32), (32, 8), (40, 40), (16, 2), (24, 8), (8, 1)])
        c = dict(op=op, M=_log(rng, 1, 16384), tail=rng.choice([0, 0, 1, 130]), B=1, skew=rng.choice([0.0, 0.5, 1.0, 2.0]), Hq=Hq, Hkv=Hkv,
                 D=rng.choice([64, 128, 128]))
        c["B"] = _log(rng, 1, min(64, c["M"]))
        most = max(work(x)["flops"] for x in listed() if x["op"] == op)
        while work(c)["flops"] > 0.9 * most:
            c["M"] = c["M"] * 7 // 8
        return c
    c = dict(op=op, M=_log(rng, 1, 8192), V=rng.choice([32000, 32001, 50257, 128256, 151936, _log(rng, 300, 160000)]), f32=rng.random() < 0.3,
             temp=rng.choice([1.0, 1.0, 0.7, 2.0]))
    if op == "distill":
        c["K"], c["rest"] = min(c["V"], _log(rng, 1, 128)), rng.random() < 0.5
    else:
        c["entropy"] = rng.random() < 0.5
    if op == "logp":
        c["k"] = min(c["V"], rng.choice([0, 1, _log(rng, 1, 128)]))
        c["tokens"] = c["k"] == 0 or rng.random() < 0.6
    while c["M"] * c["V"] * (2 if c["f32"] else 1) > 0.9 * 8192 * 128256:
        c["M"] = c["M"] * 7 // 8
    return c


def _lens(c):
    """Lengths of the sequences, growing with the power `skew` of their number; which sequence has which is the seed's."""
    w, at = [(i + 1.0) ** c["skew"] for i in range(c["B"])], [0]
    for i in range(c["B"]):
        at.append(c["M"] if i == c["B"] - 1 else int(c["M"] * sum(w[: i + 1]) / sum(w)))
    return [b - a for a, b in zip(at, at[1:])]


def work(c):
    if c["op"].startswith("attn"):
        pairs = c["Hq"] * sum(n * (n + 1) // 2 for n in _lens(c))
        q, kv, lse = c["M"] * c["Hq"] * c["D"] * 2, c["M"] * c["Hkv"] * c["D"] * 4, c["M"] * c["Hq"] * 4
        if c["op"] == "attn":
            return {"bytes": 2 * q + kv + lse, "flops": 4 * c["D"] * pairs}
        return {"bytes": 4 * q + 2 * kv + lse, "flops": 10 * c["D"] * pairs}
    z = c["M"] * c["V"] * (4 if c["f32"] else 2)
    if c["op"] == "logp":
        return {"bytes": z + c["M"] * (8 * c["k"] + 4 * c["entropy"] + 12 * c["tokens"]), "flops": 4 * c["M"] * c["V"]}
    if c["op"] == "logp_bwd":
        return {"bytes": 2 * z + c["M"] * 24, "flops": 6 * c["M"] * c["V"]}
    return {"bytes": 2 * z + c["M"] * (8 * c["K"] + 8), "flops": 7 * c["M"] * c["V"]}


# ---------------------------------------------------------------------------------------------
# what a program has in hand

def _split(x, Hq, Hkv, D):
    """Column ranges of a stacked projection as heads: q [M, Hq, D], k and v [M, Hkv, D], all with the stack's pitch."""
    return (x[:, : Hq * D].unflatten(1, (Hq, D)), x[:, Hq * D : (Hq + Hkv) * D].unflatten(1, (Hkv, D)),
            x[:, (Hq + Hkv) * D :].unflatten(1, (Hkv, D)))


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    randn = lambda *s, dtype=BF16: torch.randn(*s, generator=g, device=dev, dtype=F32).to(dtype)  # noqa: E731
    s = dict(case=c)
    if c["op"].startswith("attn"):
        Hq, Hkv, D, rows = c["Hq"], c["Hkv"], c["D"], c["M"] + c["tail"]
        order = torch.randperm(c["B"], generator=g, device=dev).tolist()
        lens = [_lens(c)[i] for i in order]
        s["bounds"] = [sum(lens[:i]) for i in range(len(lens) + 1)]
        s["starts"] = torch.tensor(s["bounds"], dtype=I32, device=dev)
        s["q"], s["k"], s["v"] = _split(1.3 * randn(rows, (Hq + 2 * Hkv) * D), Hq, Hkv, D)
        s["o"], s["lse"] = torch.zeros(rows, Hq, D, dtype=BF16, device=dev), torch.zeros(rows, Hq, dtype=F32, device=dev)
        if c["op"] == "attn_bwd":                 # what the forward call left
            s["go"] = randn(rows, Hq, D)
            o, lse = _attention(s, c)
            s["o"][: c["M"]], s["lse"][: c["M"]] = o[: c["M"]], lse[: c["M"]]
            s["gqkv"] = torch.zeros(rows, (Hq + 2 * Hkv) * D, dtype=BF16, device=dev)
            s["gq"], s["gk"], s["gv"] = _split(s["gqkv"], Hq, Hkv, D)
    else:
        M, V, ld, dtype = c["M"], c["V"], (c["V"] + 7) // 8 * 8, F32 if c["f32"] else BF16
        z = torch.randn(M, ld, generator=g, device=dev, dtype=dtype).mul_(2.5)
        s["tokens"] = torch.randint(0, V, (M,), generator=g, device=dev)
        z[torch.arange(M, device=dev), s["tokens"]] += (8 * torch.rand(M, generator=g, device=dev)).to(dtype)   # most tokens are likely ones
        s["tokens"][::17] = -1                    # positions that do not count: a sequence's first token, a user's turn
        s["z"], f = z[:, :V], dict(dtype=F32, device=dev)
        if c["op"] != "logp":
            s["gz"] = torch.zeros(M, ld, dtype=dtype, device=dev)[:, :V]
        if c["op"] == "logp":
            k = c["k"]
            s["tokens"] = s["tokens"] if c["tokens"] else None
            s["logp"], s["entropy"] = torch.empty(M, **f) if c["tokens"] else None, torch.empty(M, **f) if c["entropy"] else None
            s["ids"], s["top"] = (torch.empty(M, k, dtype=I32, device=dev), torch.empty(M, k, **f)) if k else (None, None)
        elif c["op"] == "logp_bwd":
            s["glogp"] = randn(M, dtype=F32)
            s["gent"] = 0.1 * randn(M, dtype=F32) if c["entropy"] else None
            _, s["h"], s["lse"] = _logprobs(s["z"], None, c["temp"])     # what the forward call left
        else:                                     # the teacher's list, made in blocks of tokens
            s["ids"], s["t"] = torch.empty(M, c["K"], dtype=I32, device=dev), torch.empty(M, c["K"], **f)
            for lo in range(0, M, 512):
                x = (0.8 * s["z"][lo : lo + 512].to(F32) + randn(min(512, M - lo), V, dtype=F32)) / c["temp"]
                top, at = x.topk(c["K"], -1)
                s["ids"][lo : lo + 512], s["t"][lo : lo + 512] = at.to(I32), top - x.logsumexp(-1, keepdim=True)
            s["gloss"] = (torch.rand(M, generator=g, device=dev) < 0.9).to(F32) / M
            s["loss"] = torch.empty(M, **f)
    if own:
        from paper_2509_23410_b200 import binding as L
        s["L"] = L
        if c["op"] == "attn_bwd":
            n = L.patch_sequence_attention_backward_workspace_size(c["M"] + c["tail"], c["B"], c["Hq"], c["Hkv"], c["D"])
            s["ws"] = torch.empty(n, dtype=torch.uint8, device=dev)
    return s


# ---------------------------------------------------------------------------------------------
# one pass

def run(s):
    c = s["case"]
    return (_run_own if own else _run_plain)(s, c)


def _run_own(s, c):
    L = s["L"]
    if c["op"] == "attn":
        L.patch_sequence_attention(s["q"], s["k"], s["v"], s["starts"], O=s["o"], lse=s["lse"])
        return {"o": s["o"], "lse": s["lse"]}
    if c["op"] == "attn_bwd":
        L.patch_sequence_attention_backward(s["go"], s["q"], s["k"], s["v"], s["o"], s["lse"], s["starts"], gQ=s["gq"], gK=s["gk"],
                                            gV=s["gv"], workspace=s["ws"])
        return {"gqkv": s["gqkv"]}
    if c["op"] == "logp":
        L.patch_token_logprobs(s["z"], s["tokens"], k=c["k"], temperature=c["temp"], logp=s["logp"], entropy=s["entropy"],
                               top_ids=s["ids"], top_logp=s["top"])
        return {"logp": s["logp"], "entropy": s["entropy"], "ids": s["ids"], "top": s["top"]}
    if c["op"] == "logp_bwd":
        L.patch_token_logprobs_backward(s["z"], s["tokens"], s["lse"], s["glogp"], entropy=s["h"] if c["entropy"] else None,
                                        gentropy=s["gent"], temperature=c["temp"], gZ=s["gz"])
        return {"gz": s["gz"]}
    L.patch_distill_loss(s["z"], s["ids"], s["t"], temperature=c["temp"], rest=c["rest"], loss=s["loss"], gloss=s["gloss"], gZ=s["gz"])
    return {"loss": s["loss"], "gz": s["gz"]}


def _logprobs(z, tokens, temp):
    """Log probabilities of the tokens, entropies and ln sum exp of rows of logits."""
    x = z.to(F32) / temp
    m = x.amax(-1, keepdim=True)
    x = x - m
    e = torch.exp(x)
    total = e.sum(-1, keepdim=True)
    ln = torch.log(total)
    entropy = (ln - (e * x).sum(-1, keepdim=True) / total).squeeze(-1)
    logp = None
    if tokens is not None:
        logp = (x.gather(1, tokens.clamp(min=0)[:, None]) - ln).squeeze(-1)
        logp = torch.where(tokens >= 0, logp, torch.zeros_like(logp))
    return logp, entropy, (m + ln).squeeze(-1)


def _attention(s, c):
    """The padded batch's rows are zeros behind the last sequence."""
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    q, k, v = s["q"].to(F32), s["k"].to(F32), s["v"].to(F32)
    o, lse = torch.zeros_like(s["o"]), torch.zeros_like(s["lse"])
    for a, b in zip(s["bounds"], s["bounds"][1:]):
        n = b - a
        if n == 0:
            continue
        x = (q[a:b].view(n, Hkv, Hq // Hkv, D).permute(1, 2, 0, 3) * D ** -0.5) @ k[a:b].permute(1, 2, 0)[:, None]      # [Hkv, G, n, n]
        x += torch.full((n, n), -torch.inf, device=x.device).triu(1)
        m = x.amax(-1, keepdim=True)
        e = torch.exp(x - m)
        total = e.sum(-1, keepdim=True)
        o[a:b] = (e @ v[a:b].transpose(0, 1)[:, None] / total).permute(2, 0, 1, 3).reshape(n, Hq, D).to(BF16)
        lse[a:b] = (m + torch.log(total)).squeeze(-1).permute(2, 0, 1).reshape(n, Hq)
    return o, lse


def _attention_backward(s, c):
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    G = Hq // Hkv
    gqkv = torch.zeros_like(s["gqkv"])
    gq, gk, gv = _split(gqkv, Hq, Hkv, D)
    heads = lambda x, a, b: x[a:b].to(F32).view(b - a, Hkv, x.shape[1] // Hkv, D).permute(1, 2, 0, 3)  # noqa: E731
    for a, b in zip(s["bounds"], s["bounds"][1:]):
        n = b - a
        if n == 0:
            continue
        q, k, v, o, go = (heads(s[x], a, b) for x in ("q", "k", "v", "o", "go"))
        lse = s["lse"][a:b].view(n, Hkv, G).permute(1, 2, 0)[..., None]
        delta = (o * go).sum(-1, keepdim=True)
        x = (q * D ** -0.5) @ k.transpose(2, 3)
        x += torch.full((n, n), -torch.inf, device=x.device).triu(1)
        p = torch.exp(x - lse)
        gv[a:b] = (p.transpose(2, 3) @ go).sum(1).permute(1, 0, 2).to(BF16)
        gs = p * (go @ v.transpose(2, 3) - delta) * D ** -0.5
        gq[a:b] = (gs @ k).permute(2, 0, 1, 3).reshape(n, Hq, D).to(BF16)
        gk[a:b] = (gs.transpose(2, 3) @ q).sum(1).permute(1, 0, 2).to(BF16)
    return gqkv


def _run_plain(s, c):
    if c["op"] == "attn":
        o, lse = _attention(s, c)
        return {"o": o, "lse": lse}
    if c["op"] == "attn_bwd":
        return {"gqkv": _attention_backward(s, c)}
    z, temp = s["z"], c["temp"]
    if c["op"] == "logp":
        logp, entropy, lse = _logprobs(z, s["tokens"], temp)
        ids = top = None
        if c["k"]:                                # value and index as one number: equal values by the lower index
            bits = (z.to(F32) + 0.0).view(I32)
            order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).to(I64) * (1 << 32) + ((1 << 31) - torch.arange(c["V"], device=z.device))
            ids = (1 << 31) - (order.topk(c["k"], -1).values & 0xFFFFFFFF)
            top = z.gather(1, ids).to(F32) / temp - lse[:, None]
            ids = ids.to(I32)
        return {"logp": logp, "entropy": entropy if c["entropy"] else None, "ids": ids, "top": top}
    row = torch.arange(c["M"], device=z.device)
    if c["op"] == "logp_bwd":
        x = z.to(F32) / temp - s["lse"][:, None]
        p, tokens = torch.exp(x), s["tokens"]
        glogp = torch.where(tokens >= 0, s["glogp"], torch.zeros_like(s["glogp"]))
        g = -p * glogp[:, None]
        if c["entropy"]:
            g -= s["gent"][:, None] * p * (x + s["h"][:, None])
        g[row, tokens.clamp(min=0)] += glogp
        return {"gz": (g / temp).to(z.dtype)}
    ids, t = s["ids"].long(), s["t"]
    x = z.to(F32) / temp
    x = x - x.amax(-1, keepdim=True)
    e = torch.exp(x)
    total = e.sum(-1, keepdim=True)
    logp = x.gather(1, ids) - torch.log(total)
    q = torch.exp(t.to(F64))
    if c["rest"]:
        q_rest = (1.0 - q.sum(-1, keepdim=True)).clamp(min=0).to(F32)
    else:
        q = q / q.sum(-1, keepdim=True)
    q = q.to(F32)
    loss = -(q * logp).sum(-1)
    g = e / total
    if c["rest"]:
        p_listed = g.gather(1, ids)
        g_rest = g.scatter(1, ids, 0.0)
        p_rest = g_rest.sum(-1, keepdim=True)
        loss = loss - torch.where(q_rest > 0, q_rest * torch.log(p_rest), torch.zeros_like(q_rest)).squeeze(-1)
        g = g_rest * (1.0 - q_rest / p_rest)
        g.scatter_(1, ids, p_listed)
    g.scatter_add_(1, ids, -q)
    return {"loss": loss, "gz": (g * (s["gloss"] / temp)[:, None]).to(z.dtype)}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _exact_attention(s, c):
    """One query head of one sequence at a time, the row of scores written out."""
    Hq, G, D = c["Hq"], c["Hq"] // c["Hkv"], c["D"]
    rows = c["M"] + c["tail"]
    o, lse = torch.zeros(rows, Hq, D, dtype=F64, device="cuda"), torch.zeros(rows, Hq, dtype=F64, device="cuda")
    grads = [torch.zeros(rows, h, D, dtype=F64, device="cuda") for h in (Hq, c["Hkv"], c["Hkv"])]
    for a, b in zip(s["bounds"], s["bounds"][1:]):
        if a == b:
            continue
        i = torch.arange(b - a, device="cuda")
        sees = i[:, None] >= i[None, :]
        for h in range(Hq):
            q, k, v = s["q"][a:b, h].to(F64), s["k"][a:b, h // G].to(F64), s["v"][a:b, h // G].to(F64)
            z = torch.where(sees, torch.mm(q, k.t()) / math.sqrt(D), -math.inf)
            if c["op"] == "attn":
                lse[a:b, h] = torch.logsumexp(z, -1)
                o[a:b, h] = torch.mm(torch.exp(z - lse[a:b, h, None]), v)
                continue
            p = torch.exp(z - s["lse"][a:b, h, None].to(F64))
            go = s["go"][a:b, h].to(F64)
            gz = p * (torch.mm(go, v.t()) - torch.mv(go * s["o"][a:b, h].to(F64), torch.ones(D, dtype=F64, device="cuda"))[:, None]) / math.sqrt(D)
            grads[0][a:b, h] = torch.mm(gz, k)
            grads[1][a:b, h // G] += torch.mm(gz.t(), q)
            grads[2][a:b, h // G] += torch.mm(p.t(), go)
    if c["op"] == "attn":
        return {"o": o, "lse": lse}
    return {"gqkv": torch.cat([g.flatten(1) for g in grads], 1)}


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["op"].startswith("attn"):
        return _exact_attention(s, c)
    out = []
    for lo in range(0, c["M"], 256):
        at = slice(lo, lo + 256)
        z = s["z"][at].to(F64)
        lnp = torch.log_softmax(z / c["temp"], -1)
        p = lnp.exp()
        if c["op"] == "logp":
            r = {"logp": None, "entropy": -(p * lnp).sum(-1) if c["entropy"] else None, "ids": None, "top": None}
            if c["tokens"]:
                tok = s["tokens"][at]
                r["logp"] = torch.stack([lnp[i, t] if t >= 0 else lnp.new_zeros(()) for i, t in enumerate(tok.tolist())])
            if c["k"]:
                order = torch.sort(z, stable=True, dim=-1, descending=True).indices[:, : c["k"]]
                r["ids"], r["top"] = order.to(I32), lnp.gather(1, order)
        elif c["op"] == "logp_bwd":
            lnp = z / c["temp"] - s["lse"][at, None].to(F64)      # the statistics are inputs here
            p = lnp.exp()
            tok = s["tokens"][at]
            hot = torch.zeros_like(p)
            hot[tok >= 0, tok[tok >= 0]] = 1.0
            g = s["glogp"][at].to(F64)[:, None] * (hot - p) * (tok >= 0)[:, None]
            if c["entropy"]:
                g = g - s["gent"][at].to(F64)[:, None] * p * (lnp + s["h"][at].to(F64)[:, None])
            r = {"gz": g / c["temp"]}
        else:
            ids, q = s["ids"][at].long(), s["t"][at].to(F64).exp()
            if not c["rest"]:
                q = q / q.sum(-1, keepdim=True)
            target = torch.zeros_like(p).scatter_add_(1, ids, q)
            inside = torch.zeros_like(p).scatter_(1, ids, 1.0)
            loss = -(q * lnp.gather(1, ids)).sum(-1)
            g = p - target
            if c["rest"]:
                q_rest = (1.0 - q.sum(-1)).clamp(min=0)
                p_rest = (p * (1.0 - inside)).sum(-1)
                loss = loss - torch.where(q_rest > 0, q_rest * p_rest.log(), 0.0)
                g = g - (q_rest / p_rest)[:, None] * p * (1.0 - inside)
            r = {"loss": loss, "gz": g * s["gloss"][at].to(F64)[:, None] / c["temp"]}
        out.append(r)
    return {k: torch.cat([r[k] for r in out]) if out[0][k] is not None else None for k in out[0]}
