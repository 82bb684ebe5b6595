"""Thin ctypes binding over the C ABI declared in ``include/patch.h``.

Argument marshalling only: every step of the path (mask selection, packing, the matmul, its
split-K reduction and the bf16 epilogue) runs in the CUDA library.  There is no CPU fallback:
if ``libpatch_b200.so`` is missing this module raises on first use.  The calls between the linear layers (a few
microseconds of kernel) hand their tensors to the CPython module ``_marshal``, which calls the same C entry points.

Tensors are torch CUDA tensors used purely as device buffers (``data_ptr()``); weights,
activations and results are ``torch.bfloat16``; packed blobs and workspaces are ``torch.uint8``.
"""
from __future__ import annotations

import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpatch_b200.so")

TILE_DENSE, TILE_SPARSE_2_4, TILE_DENSE_Q4, TILE_SPARSE_2_4_Q4 = 0, 1, 2, 3
VARIANT_AUTO, VARIANT_GEMV, VARIANT_MMA, VARIANT_PAIR = 0, 1, 2, 3
WEIGHTS_STATIC = 0x100   # OR into `variant`: the packed weight is not produced by the preceding kernel
INPUT_STATIC = 0x200     # OR into `variant`: X is not produced by the preceding kernel
OUTPUT_STATIC = 0x400    # OR into `variant` (with the other two): nothing in the overlap window reads or writes Y
OK = 0
ERR_NULL, ERR_SHAPE, ERR_TILE, ERR_FLAG, ERR_ALIGN = -1, -2, -3, -4, -5
ERR_SIZE, ERR_FORMAT, ERR_ARCH, ERR_CUDA, ERR_TIMEOUT = -6, -7, -8, -9, -10

EXPORTS = ["patch_packed_size", "patch_pack", "patch_unpack", "patch_gemm_workspace_size",
           "patch_workspace_init", "patch_gemm", "patch_gemm_ex", "patch_gemm_gated", "patch_gemm_gated_workspace_size", "patch_gemm_host", "patch_gemm_host_batch", "patch_gemm_host_batch_pipelined",
           "patch_gemm_noalloc",
           "patch_hard_mask", "patch_pack_patterns", "patch_pack_dev", "patch_read_layout", "patch_soft_mask_workspace_size", "patch_soft_mask",
           "patch_mask_regularizers", "patch_mask_regularizer_coefficients", "patch_soft_mask_backward",
           "patch_qk_norm_rope", "patch_qk_norm_rope_backward_workspace_size", "patch_qk_norm_rope_backward",
           "patch_kv_append", "patch_prefix_attention_workspace_size", "patch_prefix_attention",
           "patch_sequence_attention", "patch_sequence_attention_backward_workspace_size", "patch_sequence_attention_backward",
           "patch_token_logprobs", "patch_token_logprobs_backward", "patch_distill_loss", "patch_distill_loss_backward",
           "patch_strerror", "patch_version"]
MASK_NO_NOISE = 1
LOGITS_BF16, LOGITS_F32 = 0, 1
DISTILL_REST = 1


class Layout(ctypes.Structure):
    """Mirror of ``patch_layout_t``."""
    _fields_ = [("magic", ctypes.c_uint32), ("version", ctypes.c_uint32),
                ("N", ctypes.c_int64), ("K", ctypes.c_int64),
                ("tile_n", ctypes.c_int32), ("tile_k", ctypes.c_int32),
                ("n_dense", ctypes.c_int64), ("n_sparse", ctypes.c_int64),
                ("table_off", ctypes.c_uint64), ("payload_off", ctypes.c_uint64),
                ("payload_bytes", ctypes.c_uint64), ("total_bytes", ctypes.c_uint64),
                ("n_dense_q4", ctypes.c_int64), ("n_sparse_q4", ctypes.c_int64)]


class Rope(ctypes.Structure):
    """Mirror of ``patch_rope_t``; keeps its table alive."""
    _fields_ = [("cos_sin_dev", ctypes.c_void_p), ("max_positions", ctypes.c_int64), ("rotary_dim", ctypes.c_int32),
                ("interleaved", ctypes.c_int32)]


class KVCache(ctypes.Structure):
    """Mirror of ``patch_kv_cache_t``; keeps its page buffers alive."""
    _fields_ = [("k_dev", ctypes.c_void_p), ("v_dev", ctypes.c_void_p), ("num_pages", ctypes.c_int64),
                ("page_stride", ctypes.c_int64), ("page_size", ctypes.c_int32), ("Hkv", ctypes.c_int32),
                ("D", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class PatchError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {strerror(status)} (status {status})")


_lib = None


def load(path: str) -> ctypes.CDLL:
    """Load a build of the library from ``path`` and declare its argument types (``lib()`` is the product build;
    the tests also load the fault-injection build this way)."""
    if True:
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: run `python -m paper_2509_23410_b200.build` "
                               "(there is no CPU fallback)")
        L = ctypes.CDLL(path)
        vp, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
        L.patch_packed_size.argtypes = [i64, i64, ctypes.c_int, ctypes.c_int, vp, ctypes.POINTER(Layout)]
        L.patch_pack.argtypes = [vp, i64, vp, ctypes.POINTER(Layout), vp, sz, vp]
        L.patch_unpack.argtypes = [ctypes.POINTER(Layout), vp, vp, i64, vp]
        L.patch_gemm_workspace_size.argtypes = [ctypes.POINTER(Layout), i64, ctypes.POINTER(sz)]
        L.patch_workspace_init.argtypes = [vp, sz, vp]
        L.patch_gemm.argtypes = [vp, i64, i64, ctypes.POINTER(Layout), vp, vp, i64, vp, sz, vp, vp]
        L.patch_gemm_ex.argtypes = L.patch_gemm.argtypes + [ctypes.c_int]
        L.patch_gemm_gated.argtypes = [vp, i64, i64, ctypes.POINTER(Layout), vp, vp, i64, vp, sz, vp, vp, ctypes.c_int]
        L.patch_gemm_gated_workspace_size.argtypes = [ctypes.POINTER(Layout), i64, ctypes.POINTER(sz)]
        L.patch_gemm_host.argtypes = [vp, i64, ctypes.POINTER(Layout), vp, vp, vp, vp, vp, sz, vp]
        L.patch_gemm_noalloc.argtypes = [vp, i64, i64, ctypes.POINTER(Layout), vp, vp, i64, vp]
        L.patch_gemm_host_batch.argtypes = [vp, ctypes.c_int, ctypes.c_int, vp]
        L.patch_gemm_host_batch_pipelined.argtypes = [vp, ctypes.c_int, ctypes.c_int, ctypes.c_int, vp, vp, vp]
        L.patch_hard_mask.argtypes = [vp, vp, i64, i64, ctypes.c_int, ctypes.c_int, vp, vp, vp]
        L.patch_pack_patterns.argtypes = [vp, i64, vp, vp, ctypes.POINTER(Layout), vp, sz, vp, vp]
        L.patch_soft_mask_workspace_size.argtypes = [i64, i64, ctypes.c_int, ctypes.c_int, ctypes.POINTER(sz)]
        L.patch_soft_mask.argtypes = [vp, i64, vp, vp, i64, i64, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                      ctypes.c_float, ctypes.c_uint64, ctypes.c_int, vp, i64, vp, i64, vp, vp, sz, vp]
        L.patch_mask_regularizers.argtypes = [vp, ctypes.c_int, ctypes.c_double, ctypes.c_double, ctypes.c_double,
                                              ctypes.POINTER(ctypes.c_double)]
        L.patch_mask_regularizer_coefficients.argtypes = [vp, ctypes.c_int, ctypes.c_double, ctypes.c_double,
                                                          ctypes.c_double, ctypes.POINTER(ctypes.c_double),
                                                          ctypes.POINTER(ctypes.c_double)]
        L.patch_soft_mask_backward.argtypes = [vp, i64, vp, vp, i64, i64, ctypes.c_int, ctypes.c_int, ctypes.c_float,
                                               ctypes.c_float, ctypes.c_uint64, ctypes.c_int, vp, i64, ctypes.c_double,
                                               ctypes.c_double, vp, vp, vp]
        L.patch_pack_dev.argtypes = [vp, i64, vp, vp, i64, i64, ctypes.c_int, ctypes.c_int, vp, sz, vp, vp]
        L.patch_read_layout.argtypes = [vp, ctypes.POINTER(Layout), vp]
        i32, f32, rp, cp = ctypes.c_int, ctypes.c_float, ctypes.POINTER(Rope), ctypes.POINTER(KVCache)
        L.patch_qk_norm_rope.argtypes = [vp, i64, i32, vp, i64, i32, i64, i32, vp, vp, f32, rp, vp, vp, i64, vp, i64, vp, vp]
        L.patch_qk_norm_rope_backward_workspace_size.argtypes = [i64, i32, i32, i32, ctypes.POINTER(sz)]
        L.patch_qk_norm_rope_backward.argtypes = [vp, i64, vp, i64, vp, i64, i32, vp, i64, i32, i64, i32, vp, vp, f32, rp, vp,
                                                  vp, i64, vp, i64, vp, vp, vp, sz, vp, vp]
        L.patch_kv_append.argtypes = [cp, vp, i64, vp, i64, vp, i64, vp, f32, rp, vp, vp, i64, i32, vp, vp, i64, vp, vp]
        L.patch_prefix_attention_workspace_size.argtypes = [cp, i64, i32, i32, ctypes.POINTER(sz)]
        L.patch_prefix_attention.argtypes = [cp, vp, i64, i64, i32, i32, vp, i64, vp, i64, vp, f32, vp, i64, vp, vp, sz, vp, vp]
        L.patch_sequence_attention.argtypes = [vp, i64, vp, i64, vp, i64, i64, i32, i32, i32, vp, i64, f32, vp, i64, vp, vp, vp]
        L.patch_sequence_attention_backward_workspace_size.argtypes = [i64, i64, i32, i32, i32, ctypes.POINTER(sz)]
        L.patch_sequence_attention_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i32, i32, i32, vp, i64, f32, vp, i64, vp, i64,
                                                        vp, i64, vp, sz, vp, vp]
        L.patch_token_logprobs.argtypes = [vp, i64, i32, i64, i64, vp, i32, f32, vp, vp, vp, vp, vp, vp, vp]
        L.patch_token_logprobs_backward.argtypes = [vp, i64, i32, i64, i64, vp, f32, vp, vp, vp, vp, vp, i64, vp, vp]
        L.patch_distill_loss.argtypes = [vp, i64, i32, i64, i64, vp, vp, i32, f32, i32, vp, vp, vp, vp, i64, vp, vp]
        L.patch_distill_loss_backward.argtypes = [vp, i64, i32, i64, i64, vp, vp, i32, f32, i32, vp, vp, vp, i64, vp, vp]
        L.patch_strerror.argtypes = [ctypes.c_int]
        L.patch_strerror.restype = ctypes.c_char_p
        for name in EXPORTS:
            if name != "patch_strerror":
                getattr(L, name).restype = ctypes.c_int
        # addresses for the calls that do not go through ctypes (see csrc/marshal.cpp)
        for name in ("patch_qk_norm_rope", "patch_qk_norm_rope_backward", "patch_kv_append", "patch_prefix_attention",
                     "patch_sequence_attention", "patch_sequence_attention_backward",
                     "patch_token_logprobs", "patch_token_logprobs_backward", "patch_distill_loss", "patch_distill_loss_backward"):
            setattr(L, "at_" + name, ctypes.cast(getattr(L, name), vp).value)
    return L


def lib() -> ctypes.CDLL:
    """The product build of the CUDA library; fails loudly if it has not been built."""
    global _lib
    if _lib is None:
        _lib = load(LIB_PATH)
    return _lib


def strerror(status: int) -> str:
    return lib().patch_strerror(status).decode()


def _check(status: int, where: str):
    if status != OK:
        raise PatchError(status, where)


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _empty(stream, shape, dtype, device):
    """Memory for a call that runs on ``stream``, from that stream's share of torch's allocator.  From the current stream's it could be in use
    there still, and be given away there when the last reference goes (a workspace's: on return), while the kernels run on ``stream``."""
    torch = _torch
    if torch is None:
        import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if not isinstance(stream, torch.cuda.Stream):             # any object with a handle will do for the launch
        stream = torch.cuda.ExternalStream(stream.cuda_stream, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _flags_buf(flags):
    import numpy as np
    f = np.ascontiguousarray(flags, dtype=np.uint8).reshape(-1)
    return f, ctypes.c_void_p(f.ctypes.data)


def patch_packed_size(N: int, K: int, flags, tile_n: int = 128, tile_k: int = 128) -> Layout:
    L = Layout()
    f, fp = _flags_buf(flags)
    _check(lib().patch_packed_size(N, K, tile_n, tile_k, fp, ctypes.byref(L)), "patch_packed_size")
    return L


def patch_pack(W, flags, layout: Layout | None = None, out=None, stream=None):
    """Pack a bf16 CUDA weight [N x K]; returns (packed uint8 tensor, layout)."""
    import torch
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    N, K = W.shape
    if layout is None:
        layout = patch_packed_size(N, K, flags)
    if out is None:
        out = _empty(stream, layout.total_bytes, torch.uint8, W.device)
    f, fp = _flags_buf(flags)
    _check(lib().patch_pack(_ptr(W), W.stride(0), fp, ctypes.byref(layout), _ptr(out), out.numel(),
                            _stream(stream)), "patch_pack")
    return out, layout


def patch_unpack(layout: Layout, packed, out=None, stream=None):
    import torch
    if out is None:
        out = _empty(stream, (layout.N, layout.K), torch.bfloat16, packed.device)
    _check(lib().patch_unpack(ctypes.byref(layout), _ptr(packed), _ptr(out), out.stride(0), _stream(stream)),
           "patch_unpack")
    return out


def patch_gemm_workspace_size(layout: Layout, M: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_gemm_workspace_size(ctypes.byref(layout), M, ctypes.byref(n)), "patch_gemm_workspace_size")
    return int(n.value)


def patch_workspace_init(workspace, stream=None):
    if workspace is not None and workspace.numel():
        _check(lib().patch_workspace_init(_ptr(workspace), workspace.numel(), _stream(stream)), "patch_workspace_init")


def patch_gemm(X, layout: Layout, packed, Y=None, workspace=None, status=None, stream=None,
               variant: int = VARIANT_AUTO):
    """Y = X @ What^T.  X bf16 [M x K] (row stride >= K), returns Y bf16 [M x N]."""
    import torch
    assert X.is_cuda and X.dtype == torch.bfloat16 and X.dim() == 2 and (X.shape[0] == 0 or X.stride(1) == 1)
    M = X.shape[0]
    if Y is None:
        Y = _empty(stream, (M, layout.N), torch.bfloat16, X.device)
    ws_bytes = workspace.numel() if workspace is not None else 0
    _check(lib().patch_gemm_ex(_ptr(X), X.stride(0) if M else layout.K, M, ctypes.byref(layout), _ptr(packed),
                               _ptr(Y), Y.stride(0) if M else layout.N, _ptr(workspace), ws_bytes,
                               _ptr(status), _stream(stream), variant), "patch_gemm")
    return Y


def interleave_row_blocks(A, B_, block: int = 128):
    """Stack two [N x ...] arrays (torch or numpy) so that 128-row blocks alternate: A block 0, B block 0,
    A block 1, ...  With ``block=1`` the same for per-tile flag arrays.  Data movement only."""
    n = A.shape[0]
    assert A.shape == B_.shape and n % block == 0
    tail = tuple(A.shape[1:])
    if hasattr(A, "cpu"):
        import torch
        return torch.stack((A.reshape(n // block, block, *tail), B_.reshape(n // block, block, *tail)), dim=1).reshape(2 * n, *tail)
    import numpy as np
    return np.stack((A.reshape(n // block, block, *tail), B_.reshape(n // block, block, *tail)), axis=1).reshape(2 * n, *tail)


def patch_gemm_gated_workspace_size(layout: Layout, M: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_gemm_gated_workspace_size(ctypes.byref(layout), M, ctypes.byref(n)), "patch_gemm_gated_workspace_size")
    return int(n.value)


def patch_gemm_gated(X, layout: Layout, packed, Y=None, workspace=None, status=None, stream=None, flags: int = 0):
    """Y [M x N/2] = silu(X Wgate^T) * (X Wup^T) for a packed weight with interleaved gate/up row-blocks."""
    import torch
    M = X.shape[0]
    if Y is None:
        Y = _empty(stream, (M, layout.N // 2), torch.bfloat16, X.device)
    ws_bytes = workspace.numel() if workspace is not None else 0
    _check(lib().patch_gemm_gated(_ptr(X), X.stride(0) if M else layout.K, M, ctypes.byref(layout), _ptr(packed),
                                  _ptr(Y), Y.stride(0) if M else layout.N // 2, _ptr(workspace), ws_bytes,
                                  _ptr(status), _stream(stream), flags),
           "patch_gemm_gated")
    return Y


def patch_gemm_host(X_host, layout: Layout, packed, Y_host, X_stage, Y_stage, workspace=None, stream=None):
    """End-to-end call with host (pinned) X and Y; synchronises the stream."""
    M = X_host.shape[0]
    ws_bytes = workspace.numel() if workspace is not None else 0
    _check(lib().patch_gemm_host(_ptr(X_host), M, ctypes.byref(layout), _ptr(packed), _ptr(Y_host),
                                 _ptr(X_stage), _ptr(Y_stage), _ptr(workspace), ws_bytes, _stream(stream)),
           "patch_gemm_host")
    return Y_host


class HostJob(ctypes.Structure):
    """Mirror of ``patch_host_job_t``."""
    _fields_ = [("X_host", ctypes.c_void_p), ("M", ctypes.c_int64), ("layout", ctypes.POINTER(Layout)),
                ("packed_dev", ctypes.c_void_p), ("Y_host", ctypes.c_void_p), ("X_stage_dev", ctypes.c_void_p),
                ("Y_stage_dev", ctypes.c_void_p), ("workspace_dev", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t)]


def make_host_batch(jobs):
    """Marshal a list of dicts (Xh, layout, packed, Yh, X, Y, ws) once; the arrays must outlive the result."""
    arr = (HostJob * len(jobs))()
    for a, j in zip(arr, jobs):
        a.X_host, a.M, a.layout = j["Xh"].data_ptr(), j["Xh"].shape[0], ctypes.pointer(j["layout"])
        a.packed_dev, a.Y_host = j["packed"].data_ptr(), j["Yh"].data_ptr()
        a.X_stage_dev, a.Y_stage_dev = j["X"].data_ptr(), j["Y"].data_ptr()
        ws = j.get("ws")
        a.workspace_dev, a.workspace_bytes = (ws.data_ptr(), ws.numel()) if ws is not None else (None, 0)
    return arr


def patch_gemm_host_batch(batch, weights_static: bool = False, stream=None):
    """One step of GEMMs with host X / Y: all copies in, all launches, all copies out, one synchronisation."""
    _check(lib().patch_gemm_host_batch(batch, len(batch), 1 if weights_static else 0, _stream(stream)),
           "patch_gemm_host_batch")


def patch_gemm_host_batch_pipelined(batch, copy_in_stream, copy_out_stream, n_chunks: int = 4,
                                    weights_static: bool = False, stream=None):
    """The same step with copies in, GEMMs and copies out overlapped over ``n_chunks`` runs of jobs (three streams)."""
    _check(lib().patch_gemm_host_batch_pipelined(batch, len(batch), 1 if weights_static else 0, int(n_chunks),
                                                 _stream(stream), _stream(copy_in_stream), _stream(copy_out_stream)),
           "patch_gemm_host_batch_pipelined")


def patch_gemm_noalloc(X, layout: Layout, packed, Y, stream=None):
    """Y = X @ What^T for callers that may not allocate: the library's own fixed scratch array is used.

    The caller passes every buffer, Y included; nothing is allocated here either.  M <= 16.
    """
    M = X.shape[0]
    _check(lib().patch_gemm_noalloc(_ptr(X), X.stride(0) if M else layout.K, M, ctypes.byref(layout), _ptr(packed),
                                    _ptr(Y), Y.stride(0) if M else layout.N, _stream(stream)), "patch_gemm_noalloc")
    return Y


def patch_version() -> int:
    return int(lib().patch_version())


# ---------------------------------------------------------------------------------------------
# Mask learning: hard masks from logits, packing with a given 2:4 mask, soft-mask forward.


def patch_hard_mask(P_tile, P24, N: int, K: int, flags_out=None, patterns_out=None, stream=None):
    """Tile flags (uint8 [N/128 * K/128]) and candidate index per group (uint8 [N * K/4]) from the logits."""
    import torch
    assert P_tile.is_cuda and P_tile.dtype == torch.float32 and P_tile.is_contiguous()
    assert P24.is_cuda and P24.dtype == torch.float32 and P24.is_contiguous() and tuple(P24.shape) == (6, N * K // 4)
    if flags_out is None:
        flags_out = _empty(stream, (N // 128) * (K // 128), torch.uint8, P24.device)
    if patterns_out is None:
        patterns_out = _empty(stream, N * K // 4, torch.uint8, P24.device)
    _check(lib().patch_hard_mask(_ptr(P_tile), _ptr(P24), N, K, 128, 128, _ptr(flags_out), _ptr(patterns_out),
                                 _stream(stream)), "patch_hard_mask")
    return flags_out, patterns_out


def patch_pack_patterns(W, flags, patterns, layout: Layout | None = None, out=None, status=None, stream=None):
    """patch_pack with the 2:4 mask given as candidate indices (uint8 CUDA tensor [N * K/4])."""
    import torch
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    assert patterns.is_cuda and patterns.dtype == torch.uint8 and patterns.is_contiguous()
    N, K = W.shape
    assert patterns.numel() == N * K // 4
    if layout is None:
        layout = patch_packed_size(N, K, flags)
    if out is None:
        out = _empty(stream, layout.total_bytes, torch.uint8, W.device)
    f, fp = _flags_buf(flags)
    _check(lib().patch_pack_patterns(_ptr(W), W.stride(0), fp, _ptr(patterns), ctypes.byref(layout), _ptr(out),
                                     out.numel(), _ptr(status), _stream(stream)), "patch_pack_patterns")
    return out, layout


def patch_soft_mask_workspace_size(N: int, K: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_soft_mask_workspace_size(N, K, 128, 128, ctypes.byref(n)), "patch_soft_mask_workspace_size")
    return int(n.value)


def patch_soft_mask(W, P_tile, P24, tau: float, kappa: float, seed: int = 0, flags: int = 0, Wt=None, Mt=None,
                    sums=None, workspace=None, stream=None):
    """Soft-mask forward of one matrix: returns (Wt bf16 [N x K], sums float64 CUDA tensor [4]);
    pass a float32 ``Mt`` [N x K] to also get the soft mask itself."""
    import torch
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    N, K = W.shape
    assert P_tile.is_cuda and P_tile.dtype == torch.float32 and P_tile.is_contiguous()
    assert P24.is_cuda and P24.dtype == torch.float32 and P24.is_contiguous() and tuple(P24.shape) == (6, N * K // 4)
    if Wt is None:
        Wt = _empty(stream, (N, K), torch.bfloat16, W.device)
    if sums is None:
        sums = _empty(stream, 4, torch.float64, W.device)
    if workspace is None:
        workspace = _empty(stream, patch_soft_mask_workspace_size(N, K), torch.uint8, W.device)
    assert Mt is None or (Mt.is_cuda and Mt.dtype == torch.float32 and Mt.stride(1) == 1)
    _check(lib().patch_soft_mask(_ptr(W), W.stride(0), _ptr(P_tile), _ptr(P24), N, K, 128, 128, float(tau),
                                 float(kappa), int(seed) & 0xFFFFFFFFFFFFFFFF, int(flags), _ptr(Wt), Wt.stride(0),
                                 _ptr(Mt), Mt.stride(0) if Mt is not None else 0, _ptr(sums), _ptr(workspace),
                                 workspace.numel(), _stream(stream)), "patch_soft_mask")
    return Wt, sums


def patch_mask_regularizers(sums, rho: float, lambda1: float, lambda2: float) -> float:
    """The two regularisers of Eq. 5 from per-matrix sums (host array-like [n x 4])."""
    import numpy as np
    a = np.ascontiguousarray(sums, dtype=np.float64).reshape(-1, 4)
    out = ctypes.c_double(0.0)
    _check(lib().patch_mask_regularizers(ctypes.c_void_p(a.ctypes.data), int(a.shape[0]), float(rho), float(lambda1),
                                         float(lambda2), ctypes.byref(out)), "patch_mask_regularizers")
    return float(out.value)


def patch_mask_regularizer_coefficients(sums, rho: float, lambda1: float, lambda2: float):
    """(c1, c2) of the regularisers' gradient from per-matrix sums (host array-like [n x 4])."""
    import numpy as np
    a = np.ascontiguousarray(sums, dtype=np.float64).reshape(-1, 4)
    c1, c2 = ctypes.c_double(0.0), ctypes.c_double(0.0)
    _check(lib().patch_mask_regularizer_coefficients(ctypes.c_void_p(a.ctypes.data), int(a.shape[0]), float(rho),
                                                     float(lambda1), float(lambda2), ctypes.byref(c1), ctypes.byref(c2)),
           "patch_mask_regularizer_coefficients")
    return float(c1.value), float(c2.value)


def patch_soft_mask_backward(W, P_tile, P24, tau: float, kappa: float, Gw, c1: float, c2: float, seed: int = 0,
                             flags: int = 0, gP_tile=None, gP24=None, stream=None):
    """Gradient of the soft-mask objective w.r.t. the logits: returns (gP_tile float32, gP24 float32 [6 x G])."""
    import torch
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    assert Gw.is_cuda and Gw.dtype == torch.bfloat16 and Gw.shape == W.shape and Gw.stride(1) == 1
    N, K = W.shape
    assert P_tile.is_cuda and P_tile.dtype == torch.float32 and P_tile.is_contiguous()
    assert P24.is_cuda and P24.dtype == torch.float32 and P24.is_contiguous() and tuple(P24.shape) == (6, N * K // 4)
    if gP_tile is None:
        gP_tile = _empty(stream, P_tile.shape, torch.float32, P_tile.device)
    if gP24 is None:
        gP24 = _empty(stream, P24.shape, torch.float32, P24.device)
    _check(lib().patch_soft_mask_backward(_ptr(W), W.stride(0), _ptr(P_tile), _ptr(P24), N, K, 128, 128, float(tau),
                                          float(kappa), int(seed) & 0xFFFFFFFFFFFFFFFF, int(flags), _ptr(Gw), Gw.stride(0),
                                          float(c1), float(c2), _ptr(gP_tile), _ptr(gP24), _stream(stream)),
           "patch_soft_mask_backward")
    return gP_tile, gP24


def patch_pack_dev(W, flags_dev, patterns=None, out=None, status=None, stream=None):
    """Pack with the tile flags in device memory (uint8 CUDA tensor); returns the packed uint8 tensor.
    ``out`` defaults to a buffer that fits any flags; get the layout with ``patch_read_layout``."""
    import torch
    assert W.is_cuda and W.dtype == torch.bfloat16 and W.dim() == 2 and W.stride(1) == 1
    assert flags_dev.is_cuda and flags_dev.dtype == torch.uint8 and flags_dev.is_contiguous()
    N, K = W.shape
    T = (N // 128) * (K // 128)
    assert flags_dev.numel() == T
    if out is None:
        out = _empty(stream, (256 + 16 * T + 1023) // 1024 * 1024 + T * 32768, torch.uint8, W.device)
    _check(lib().patch_pack_dev(_ptr(W), W.stride(0), _ptr(flags_dev), _ptr(patterns), N, K, 128, 128, _ptr(out),
                                out.numel(), _ptr(status), _stream(stream)), "patch_pack_dev")
    return out


def patch_read_layout(packed, stream=None) -> Layout:
    L = Layout()
    _check(lib().patch_read_layout(_ptr(packed), ctypes.byref(L), _stream(stream)), "patch_read_layout")
    return L


# ---------------------------------------------------------------------------------------------
# Between the linear layers: norms and rotation of queries and keys, the paged cache, attention behind a shared prefix.
#
# These calls take a few microseconds on the GPU for a decode step's handful of tokens, so what the host does for each of them
# counts: the tensors are checked and taken apart by a CPython module (csrc/marshal.cpp), which calls the library by address.

_torch = _bf16 = _raw_stream = _marshal = None


def _use_torch():
    global _torch, _bf16, _raw_stream, _marshal
    import torch
    try:
        from . import _marshal as m
    except ImportError as e:
        raise RuntimeError("_marshal.so is missing or was built for another torch: run `python -m paper_2509_23410_b200.build`") from e
    if m.built != f"for torch {torch.__version__}":
        raise RuntimeError(f"_marshal.so was built {m.built}, this is {torch.__version__}: run `python -m paper_2509_23410_b200.build`")
    _torch, _bf16, _marshal = torch, torch.bfloat16, m
    # the current stream's handle without a Stream object around it (five times quicker); device index -> handle
    _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


def _stream_of(x, stream):
    return _raw_stream(x.get_device()) if stream is None else stream.cuda_stream


def patch_rope(cos_sin, interleaved: bool = False) -> Rope:
    """Rotation by a table float32 [max_positions, rotary_dim]: a position's cosines, then its sines."""
    _use_torch()
    assert cos_sin.is_cuda and cos_sin.dtype is _torch.float32 and cos_sin.dim() == 2 and cos_sin.is_contiguous()
    r = Rope(cos_sin.data_ptr(), cos_sin.shape[0], cos_sin.shape[1], 1 if interleaved else 0)
    r.table, r.at = cos_sin, ctypes.addressof(r)
    return r


def patch_kv_cache(k, v) -> KVCache:
    """Paged cache over bf16 page buffers [num_pages, Hkv, page_size, D]; the two may be views of one buffer."""
    _use_torch()
    assert k.is_cuda and v.is_cuda and k.dtype is _bf16 and v.dtype is _bf16 and k.dim() == 4
    assert k.shape == v.shape and k.stride() == v.stride(), "keys and values have the same shape and strides"
    pages, H, page, D = k.shape
    assert k.stride()[1:] == (page * D, D, 1), "a page holds [Hkv, page_size, D] without gaps"
    c = KVCache(k.data_ptr(), v.data_ptr(), pages, k.stride(0) if pages > 1 else H * page * D, page, H, D, 0)
    c.buffers, c.at = (k, v), ctypes.addressof(c)
    return c


def patch_qk_norm_rope(Q, K, rope: Rope | None, positions, wq=None, wk=None, eps: float = 1e-6, Q_out=None, K_out=None,
                       status=None, stream=None):
    """Norms of queries [M, Hq, D] and keys [M, Hkv, D] (either may be None) and the rotation: returns (Q_out, K_out)."""
    if _torch is None:
        _use_torch()
    if Q_out is None and Q is not None:
        Q_out = _empty(stream, Q.shape, _bf16, Q.device)
    if K_out is None and K is not None:
        K_out = _empty(stream, K.shape, _bf16, K.device)
    rc = _marshal.qk_norm_rope((_lib or lib()).at_patch_qk_norm_rope, Q, K, wq, wk, eps, rope.at if rope is not None else None, positions,
                               Q_out, K_out, status, _stream_of(Q if Q is not None else K, stream))
    if rc:
        _check(rc, "patch_qk_norm_rope")
    return Q_out, K_out


def patch_qk_norm_rope_backward_workspace_size(M: int, Hq: int, Hkv: int, D: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_qk_norm_rope_backward_workspace_size(M, Hq, Hkv, D, ctypes.byref(n)),
           "patch_qk_norm_rope_backward_workspace_size")
    return int(n.value)


def patch_qk_norm_rope_backward(gQ_out, gK_out, rope: Rope | None, positions, Q=None, K=None, wq=None, wk=None, eps: float = 1e-6,
                                gQ=None, gK=None, gwq=None, gwk=None, workspace=None, status=None, stream=None):
    """Gradient of ``patch_qk_norm_rope``: returns (gQ, gK, gwq, gwk); the inputs Q, K are needed where a weight is given."""
    if _torch is None:
        _use_torch()
    some = gQ_out if gQ_out is not None else gK_out
    if gQ is None and gQ_out is not None:
        gQ = _empty(stream, gQ_out.shape, _bf16, some.device)
    if gK is None and gK_out is not None:
        gK = _empty(stream, gK_out.shape, _bf16, some.device)
    if gwq is None and wq is not None:
        gwq = _empty(stream, some.shape[2], _torch.float32, some.device)
    if gwk is None and wk is not None:
        gwk = _empty(stream, some.shape[2], _torch.float32, some.device)
    if workspace is None and (wq is not None or wk is not None):
        n = patch_qk_norm_rope_backward_workspace_size(some.shape[0], gQ_out.shape[1] if gQ_out is not None else 0,
                                                       gK_out.shape[1] if gK_out is not None else 0, some.shape[2])
        workspace = _empty(stream, n, _torch.uint8, some.device)
    rc = _marshal.qk_norm_rope_backward((_lib or lib()).at_patch_qk_norm_rope_backward, gQ_out, gK_out, Q if wq is not None else None,
                                        K if wk is not None else None, wq, wk, eps, rope.at if rope is not None else None, positions, gQ, gK,
                                        gwq, gwk, workspace, status, _stream_of(some, stream))
    if rc:
        _check(rc, "patch_qk_norm_rope_backward")
    return gQ, gK, gwq, gwk


def patch_kv_append(cache: KVCache, K, V, slots, rope: Rope | None = None, positions=None, wk=None, eps: float = 1e-6, Q=None,
                    wq=None, Q_out=None, status=None, stream=None):
    """Keys (normed and rotated) and values [M, Hkv, D] into the cache's slots (int64 [M]; negative: not stored); with Q
    [M, Hq, D] also the queries, normed and rotated: returns Q_out (None without Q)."""
    if Q_out is None and Q is not None:
        Q_out = _empty(stream, Q.shape, _bf16, Q.device)
    rc = _marshal.kv_append((_lib or lib()).at_patch_kv_append, cache.at, K, V, slots, wk, eps, rope.at if rope is not None else None,
                            positions, Q, wq, Q_out, status, _stream_of(K, stream))
    if rc:
        _check(rc, "patch_kv_append")
    return Q_out


def patch_prefix_attention_workspace_size(cache: KVCache, B: int, T: int, Hq: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_prefix_attention_workspace_size(cache, B, T, Hq, ctypes.byref(n)), "patch_prefix_attention_workspace_size")
    return int(n.value)


def patch_prefix_attention(cache: KVCache, Q, prefix_pages, prefix_len: int, page_table, suffix_lens, scale: float | None = None,
                           O=None, lse=None, workspace=None, status=None, stream=None):
    """Attention of Q [B T, Hq, D] over the shared prefix (int32 ``prefix_pages``, ``prefix_len`` keys) and each sequence's own
    keys (int32 ``page_table`` [B, n], int32 ``suffix_lens`` [B]): returns O; ``lse`` float32 [B T, Hq] is written if given.
    ``scale`` defaults to 1 / sqrt(D)."""
    if O is None:
        O = _empty(stream, Q.shape, _bf16, Q.device)
    if workspace is None:
        B = page_table.shape[0]
        workspace = _empty(stream, patch_prefix_attention_workspace_size(cache, B, Q.shape[0] // B if B else 1, Q.shape[1]), _torch.uint8, Q.device)
    rc = _marshal.prefix_attention((_lib or lib()).at_patch_prefix_attention, cache.at, Q, prefix_pages, prefix_len, page_table, suffix_lens,
                                   scale, O, lse, workspace, status, _stream_of(Q, stream))
    if rc:
        _check(rc, "patch_prefix_attention")
    return O


def patch_sequence_attention(Q, K, V, starts, scale: float | None = None, O=None, lse=None, status=None, stream=None):
    """Causal attention within packed sequences: Q [M, Hq, D], K and V [M, Hkv, D], sequence b in rows starts[b] .. starts[b + 1] - 1 (int32
    [B + 1]): returns O; ``lse`` float32 [M, Hq] is written if given.  ``scale`` defaults to 1 / sqrt(D).  Rows outside the sequences are
    not written (where O is made here: they hold whatever the memory did)."""
    if _torch is None:
        _use_torch()
    assert Q.is_cuda, "heads are on the GPU"
    if O is None:
        O = _empty(stream, Q.shape, _bf16, Q.device)
    rc = _marshal.sequence_attention((_lib or lib()).at_patch_sequence_attention, Q, K, V, starts, scale, O, lse, status, _stream_of(Q, stream))
    if rc:
        _check(rc, "patch_sequence_attention")
    return O


def patch_sequence_attention_backward_workspace_size(M: int, B: int, Hq: int, Hkv: int, D: int) -> int:
    n = ctypes.c_size_t(0)
    _check(lib().patch_sequence_attention_backward_workspace_size(M, B, Hq, Hkv, D, ctypes.byref(n)), "patch_sequence_attention_backward_workspace_size")
    return int(n.value)


def patch_sequence_attention_backward(gO, Q, K, V, O, lse, starts, scale: float | None = None, gQ=None, gK=None, gV=None, workspace=None, status=None,
                                      stream=None):
    """Gradient of ``patch_sequence_attention`` from its inputs and results: returns (gQ, gK, gV).  Rows outside the sequences are not written."""
    if _torch is None:
        _use_torch()
    assert Q.is_cuda and Q.dim() == 3 and K.dim() == 3, "heads are CUDA tensors [rows, heads, D]"
    if gQ is None:
        gQ = _empty(stream, Q.shape, _bf16, Q.device)
    if gK is None:
        gK = _empty(stream, K.shape, _bf16, Q.device)
    if gV is None:
        gV = _empty(stream, V.shape, _bf16, Q.device)
    if workspace is None:
        n = patch_sequence_attention_backward_workspace_size(Q.shape[0], max(0, starts.shape[0] - 1), Q.shape[1], K.shape[1], Q.shape[2])
        workspace = _empty(stream, n, _torch.uint8, Q.device)
    rc = _marshal.sequence_attention_backward((_lib or lib()).at_patch_sequence_attention_backward, gO, Q, K, V, O, lse, starts, scale, gQ, gK, gV, workspace,
                                              status, _stream_of(Q, stream))
    if rc:
        _check(rc, "patch_sequence_attention_backward")
    return gQ, gK, gV


# ---------------------------------------------------------------------------------------------
# From logits to a loss: log probabilities of tokens, entropy, alternatives; distillation from a teacher's list.
#
# Logits are bf16 or float32 [M, V] with contiguous rows, any pitch that is a multiple of eight elements.  The calls run on the tensors'
# device, whichever is the current one.

def _rows_like(Z, stream):
    """Memory for a gradient of Z [M, V]: rows of a pitch that the library takes."""
    M, V = Z.shape
    return _empty(stream, (M, (V + 7) // 8 * 8), Z.dtype, Z.device)[:, :V]


def patch_token_logprobs(Z, tokens=None, k: int = 0, temperature: float = 1.0, logp=None, entropy=None, lse=None, top_ids=None,
                         top_logp=None, status=None, stream=None):
    """Log probabilities of ``tokens`` (int64 [M]; negative: the row does not count, 0) under softmax(Z / temperature), and the ``k`` most
    likely alternatives of every row: returns (logp, entropy, lse, top_ids, top_logp).  ``logp`` is None without tokens, ``top_ids`` (int32) and
    ``top_logp`` [M, k] without k; ``entropy`` and ``lse`` (float32 [M]) are written if given, made if True."""
    if _torch is None:
        _use_torch()
    assert Z.is_cuda and Z.dim() == 2, "logits are CUDA tensors [rows, columns]"
    M = Z.shape[0]
    if logp is None and tokens is not None:
        logp = _empty(stream, M, _torch.float32, Z.device)
    if entropy is True:
        entropy = _empty(stream, M, _torch.float32, Z.device)
    if lse is True:
        lse = _empty(stream, M, _torch.float32, Z.device)
    if k > 0 and top_ids is None:
        top_ids = _empty(stream, (M, k), _torch.int32, Z.device)
    if k > 0 and top_logp is None:
        top_logp = _empty(stream, (M, k), _torch.float32, Z.device)
    rc = _marshal.token_logprobs((_lib or lib()).at_patch_token_logprobs, Z, tokens, k, temperature, logp, entropy, lse, top_ids, top_logp, status,
                                 _stream_of(Z, stream))
    if rc:
        _check(rc, "patch_token_logprobs")
    return logp, entropy, lse, top_ids, top_logp


def patch_token_logprobs_backward(Z, tokens, lse, glogp=None, entropy=None, gentropy=None, temperature: float = 1.0, gZ=None, status=None,
                                  stream=None):
    """Gradient of sum(glogp * logp) + sum(gentropy * entropy) with respect to the logits, from the forward call's ``lse`` (and
    ``entropy``): returns gZ (which may be Z itself)."""
    if _torch is None:
        _use_torch()
    assert Z.is_cuda and Z.dim() == 2, "logits are CUDA tensors [rows, columns]"
    if gZ is None:
        gZ = _rows_like(Z, stream)
    rc = _marshal.token_logprobs_backward((_lib or lib()).at_patch_token_logprobs_backward, Z, tokens, temperature, lse, glogp, entropy, gentropy, gZ,
                                          status, _stream_of(Z, stream))
    if rc:
        _check(rc, "patch_token_logprobs_backward")
    return gZ


def patch_distill_loss(Z, top_ids, top_logp, temperature: float = 1.0, rest: bool = False, loss=None, stats=None, gloss=None, gZ=None, status=None,
                       stream=None):
    """Cross entropy of the rows of Z [M, V] with a teacher's list (int32 ``top_ids`` and float32 ``top_logp`` [M, K], at the same
    temperature), renormalised or, with ``rest``, with what the list leaves as one more class: returns loss float32 [M].  ``gZ`` takes the gradient of
    sum(gloss * loss) if given (it may be Z itself); ``stats`` float32 [M, 2] what ``patch_distill_loss_backward`` reads."""
    if _torch is None:
        _use_torch()
    assert Z.is_cuda and Z.dim() == 2, "logits are CUDA tensors [rows, columns]"
    if loss is None:
        loss = _empty(stream, Z.shape[0], _torch.float32, Z.device)
    rc = _marshal.distill_loss((_lib or lib()).at_patch_distill_loss, Z, top_ids, top_logp, temperature, DISTILL_REST if rest else 0, loss, stats, gloss,
                               gZ, status, _stream_of(Z, stream))
    if rc:
        _check(rc, "patch_distill_loss")
    return loss


def patch_distill_loss_backward(Z, top_ids, top_logp, stats, gloss=None, temperature: float = 1.0, rest: bool = False, gZ=None, status=None,
                                stream=None):
    """Gradient of sum(gloss * loss) with respect to the logits from the forward call's ``stats``: returns gZ (not Z itself)."""
    if _torch is None:
        _use_torch()
    assert Z.is_cuda and Z.dim() == 2, "logits are CUDA tensors [rows, columns]"
    if gZ is None:
        gZ = _rows_like(Z, stream)
    rc = _marshal.distill_loss_backward((_lib or lib()).at_patch_distill_loss_backward, Z, top_ids, top_logp, temperature, DISTILL_REST if rest else 0,
                                        stats, gloss, gZ, status, _stream_of(Z, stream))
    if rc:
        _check(rc, "patch_distill_loss_backward")
    return gZ
