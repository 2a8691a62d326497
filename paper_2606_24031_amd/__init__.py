"""W4A8 (Q4_0 weight x Q8_0 activation) MoE hot path for AMD MI355X (gfx950).

A thin ctypes binding over ``libw4a8.so``: every function marshals torch
tensors (device memory and the current HIP stream) into the C ABI declared in
``include/w4a8.h`` and raises on a non-zero status.  All arithmetic runs in the
HIP kernels; there is no CPU or PyTorch fallback -- if the library is missing
or the device is not gfx950 the calls raise.
"""
from __future__ import annotations

import ctypes
import os

try:
    import torch
except (ImportError, OSError):        # (its libraries may not load) building needs none
    torch = None

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libw4a8.so")

OK, ENULL, ESHAPE, ERANGE, EWORKSPACE, EALIGN, EHIP, EDEVICE, EALIAS, ESCRATCH = \
    0, -1, -2, -3, -4, -5, -6, -7, -8, -9
NOALLOC_SCRATCH_BYTES = 8 << 20
Q4_0_BLOCK_BYTES = 18
Q8_0_BLOCK_BYTES = 34
Q4_SYM_BLOCK_BYTES = 20
Q8_F32_BLOCK_BYTES = 36
WS_XQ, WS_H, WS_HQ, WS_PERM, WS_COUNT, WS_SYNC, WS_SYNC_END, WS_XN = 0, 1, 2, 3, 4, 5, 6, 7
WS_NFIELDS = 8
KV_PAGE = 64
KV_FORMATS = {"q4_0": 0, "q4_sym": 1}
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
ROPE_KINDS = {"none": 0, "linear": 1, "parts": 2}
Q8_ROW_PAD = 128
CONV_ACTS = {"none": 0, "silu": 1}

EXPORTS = ("w4a8_strerror", "q8_0_quantize", "q4_0_quantize", "q4q8_gemv",
           "moe_w4a8_workspace_size", "moe_w4a8_workspace_init",
           "moe_w4a8_workspace_layout", "moe_w4a8_forward", "moe_w4a8_layer",
           "rmsnorm_residual", "moe_router_topk", "moe_w4a8_layer_routed",
           "q4_sym_quantize", "q8_f32_quantize", "q4sym_q8f32_gemv",
           "w4a8_decode_wait_bound", "moe_w4a8_forward_noalloc", "q4q8_gemm_workspace_size",
           "q4q8_gemm", "moe_sym_workspace_size", "moe_sym_workspace_layout", "moe_sym_forward",
           "gdn_workspace_size", "gdn_chunked_scan", "rope_frequencies", "rope_rotate",
           "kv_q4_tile_bytes", "kv_q4_append", "kv_q4_read", "attn_q4_workspace_size",
           "attn_q4_forward", "token_logprobs_workspace_size", "token_logprobs",
           "q8_row_bytes", "q8_row_quantize", "q8q8_gemm", "short_conv", "ssm_workspace_size",
           "ssm_scan")

_lib = None


class _RopeArgs(ctypes.Structure):     # w4a8_rope
    _fields_ = [("inv_freq", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("n_rot", ctypes.c_int64), ("layout", ctypes.c_int32), ("mscale", ctypes.c_float)]


class _KvArgs(ctypes.Structure):       # w4a8_kv
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p),
                ("page_table", ctypes.c_void_p), ("kv_len", ctypes.c_void_p),
                ("cu_rows", ctypes.c_void_p), ("n_pages", ctypes.c_int64),
                ("max_pages", ctypes.c_int64), ("B", ctypes.c_int64), ("NKV", ctypes.c_int64),
                ("D", ctypes.c_int64), ("format", ctypes.c_int32)]


class _SeqArgs(ctypes.Structure):      # w4a8_seqs
    _fields_ = [("cu_rows", ctypes.c_void_p), ("src", ctypes.c_void_p), ("dst", ctypes.c_void_p),
                ("n_slots", ctypes.c_int64), ("B", ctypes.c_int64)]


class _SsmArgs(ctypes.Structure):      # w4a8_ssm
    _fields_ = [(n, ctypes.c_void_p) for n in ("x", "dt", "b", "c", "z", "A", "D", "dt_bias")] + \
               [(n, ctypes.c_int64) for n in ("x_stride", "dt_stride", "b_stride", "c_stride", "z_stride",
                                              "NH", "NG", "N", "P")] + [("softplus", ctypes.c_int32)]


class W4A8Error(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


def lib() -> ctypes.CDLL:
    """Load libw4a8.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                           "`python -m paper_2606_24031_amd.build`")
    L = ctypes.CDLL(LIB_PATH)
    P, I64, SZ = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    L.w4a8_strerror.argtypes = [ctypes.c_int]
    L.w4a8_strerror.restype = ctypes.c_char_p
    for name in ("q8_0_quantize", "q4_0_quantize", "q4_sym_quantize", "q8_f32_quantize"):
        getattr(L, name).argtypes = [P, P, I64, I64, P]
        getattr(L, name).restype = ctypes.c_int
    L.q4q8_gemv.argtypes = [P, P, P, I64, I64, P]
    L.q4q8_gemv.restype = ctypes.c_int
    L.q4sym_q8f32_gemv.argtypes = [P, P, P, I64, I64, P]
    L.q4sym_q8f32_gemv.restype = ctypes.c_int
    L.moe_w4a8_workspace_size.argtypes = [I64, I64, I64, I64, I64]
    L.moe_w4a8_workspace_size.restype = SZ
    L.moe_w4a8_workspace_init.argtypes = [P, SZ, P]
    L.moe_w4a8_workspace_init.restype = ctypes.c_int
    L.moe_w4a8_workspace_layout.argtypes = [I64, I64, I64, I64, I64, P]
    L.moe_w4a8_workspace_layout.restype = ctypes.c_int
    L.moe_w4a8_forward.argtypes = [P, P, P, P, P, P, P, P, I64, I64, I64, I64, I64, P, SZ, P]
    L.moe_w4a8_forward.restype = ctypes.c_int
    L.moe_w4a8_layer.argtypes = [P, P, P, ctypes.c_float, P, P, P, P, P, P, P, P,
                                 I64, I64, I64, I64, I64, P, SZ, P]
    L.moe_w4a8_layer.restype = ctypes.c_int
    L.rmsnorm_residual.argtypes = [P, P, P, P, P, I64, I64, ctypes.c_float, P]
    L.rmsnorm_residual.restype = ctypes.c_int
    L.moe_router_topk.argtypes = [P, P, P, I64, I64, I64, P]
    L.moe_router_topk.restype = ctypes.c_int
    L.moe_w4a8_layer_routed.argtypes = [P, P, P, ctypes.c_float, P, P, P, P, P, P, P, P, P, P,
                                        I64, I64, I64, I64, I64, P, SZ, P]
    L.moe_w4a8_layer_routed.restype = ctypes.c_int
    L.w4a8_decode_wait_bound.argtypes = [I64]
    L.w4a8_decode_wait_bound.restype = ctypes.c_int
    L.moe_w4a8_forward_noalloc.argtypes = [P, P, P, P, P, P, P, P, I64, I64, I64, I64, I64, P]
    L.moe_w4a8_forward_noalloc.restype = ctypes.c_int
    L.q4q8_gemm_workspace_size.argtypes = [I64, I64]
    L.q4q8_gemm_workspace_size.restype = SZ
    L.q4q8_gemm.argtypes = [P, P, P, I64, I64, I64, P, SZ, P]
    L.q4q8_gemm.restype = ctypes.c_int
    L.moe_sym_workspace_size.argtypes = [I64, I64, I64, I64, I64]
    L.moe_sym_workspace_size.restype = SZ
    L.moe_sym_workspace_layout.argtypes = [I64, I64, I64, I64, I64, P]
    L.moe_sym_workspace_layout.restype = ctypes.c_int
    L.moe_sym_forward.argtypes = [P, P, P, P, P, P, P, P, I64, I64, I64, I64, I64, P, SZ, P]
    L.moe_sym_forward.restype = ctypes.c_int
    L.gdn_workspace_size.argtypes = [I64, I64, I64, I64]
    L.gdn_workspace_size.restype = SZ
    L.gdn_chunked_scan.argtypes = [P, P, P, P, P, P, P, P, I64, I64, I64, I64, P, SZ, P]
    L.gdn_chunked_scan.restype = ctypes.c_int
    F64, INT, KV, RO = ctypes.c_double, ctypes.c_int, ctypes.POINTER(_KvArgs), \
        ctypes.POINTER(_RopeArgs)
    L.rope_frequencies.argtypes = [P, I64, F64, INT, F64, F64, F64, F64, P]
    L.rope_rotate.argtypes = [RO, P, I64, P, I64, I64, I64, I64, P]
    L.kv_q4_tile_bytes.argtypes = [I64, ctypes.c_int32]
    L.kv_q4_tile_bytes.restype = SZ
    L.kv_q4_append.argtypes = [KV, RO, P, I64, P, I64, P, I64, P, I64, I64, P]
    L.kv_q4_read.argtypes = [KV, P, P, I64, P]
    L.attn_q4_workspace_size.argtypes = [KV, I64, I64]
    L.attn_q4_workspace_size.restype = SZ
    L.attn_q4_forward.argtypes = [KV, P, I64, P, P, I64, I64, ctypes.c_float, I64, P, SZ, P]
    L.token_logprobs_workspace_size.argtypes = [I64, I64, I64]
    L.token_logprobs_workspace_size.restype = SZ
    L.token_logprobs.argtypes = [P, I64, P, P, P, P, P, I64, I64, I64, P, SZ, P]
    SEQ, SSM = ctypes.POINTER(_SeqArgs), ctypes.POINTER(_SsmArgs)
    L.q8_row_bytes.argtypes = [I64]
    L.q8_row_bytes.restype = SZ
    L.q8_row_quantize.argtypes = [P, I64, P, P, I64, I64, P]
    L.q8q8_gemm.argtypes = [P, P, P, P, P, P, I64, I64, I64, I64, P]
    L.short_conv.argtypes = [SEQ, P, I64, P, P, P, P, I64, I64, I64, I64, ctypes.c_int32, P]
    L.ssm_workspace_size.argtypes = [SEQ, SSM, I64]
    L.ssm_workspace_size.restype = SZ
    L.ssm_scan.argtypes = [SEQ, SSM, P, P, I64, I64, P, SZ, P]
    for name in ("rope_frequencies", "rope_rotate", "kv_q4_append", "kv_q4_read",
                 "attn_q4_forward", "token_logprobs", "q8_row_quantize", "q8q8_gemm", "short_conv",
                 "ssm_scan"):
        getattr(L, name).restype = INT
    _lib = L
    return L


def strerror(code: int) -> str:
    return lib().w4a8_strerror(code).decode()


def _check(rc: int, where: str):
    if rc != OK:
        raise W4A8Error(rc, where)


def _stream(stream):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _empty(shape, dtype, device, stream):
    """A call's own output, of the memory of the stream that writes it: the
    current stream's pending work may still use what it has freed."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(shape, dtype=dtype, device=device)


def _p(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _u8(t):
    import torch
    assert t.dtype == torch.uint8 and t.is_contiguous()
    return t


# ------------------------------------------------------------------ entry points
def q8_0_quantize(x, out=None, stream=None):
    """Q8_0 of fp32 rows x [rows, K] -> uint8 [rows, K/32*34] on x's device."""
    import torch
    assert x.dtype == torch.float32 and x.is_contiguous()
    rows, K = (1, x.numel()) if x.dim() == 1 else (x.numel() // x.shape[-1], x.shape[-1])
    if out is None:
        out = _empty((rows, K // 32 * Q8_0_BLOCK_BYTES), torch.uint8, x.device, stream)
    _check(lib().q8_0_quantize(_p(x), _p(_u8(out)), rows, K, _stream(stream)), "q8_0_quantize")
    return out


def q4_0_quantize(w, out=None, stream=None):
    """Q4_0 of fp32 rows w [rows, K] -> uint8 [rows, K/32*18] on w's device."""
    import torch
    assert w.dtype == torch.float32 and w.is_contiguous()
    rows, K = (1, w.numel()) if w.dim() == 1 else (w.numel() // w.shape[-1], w.shape[-1])
    if out is None:
        out = _empty((rows, K // 32 * Q4_0_BLOCK_BYTES), torch.uint8, w.device, stream)
    _check(lib().q4_0_quantize(_p(w), _p(_u8(out)), rows, K, _stream(stream)), "q4_0_quantize")
    return out


def q4q8_gemv(w, xq, N, K, y=None, stream=None):
    """y[N] = W4A8(w [N, K/32 Q4_0 blocks], xq [K/32 Q8_0 blocks]) in fp32."""
    import torch
    if y is None:
        y = _empty(N, torch.float32, w.device, stream)
    _check(lib().q4q8_gemv(_p(_u8(w)), _p(_u8(xq)), _p(y), N, K, _stream(stream)), "q4q8_gemv")
    return y


def gemm_workspace(M, K, device="cuda", stream=None):
    """A workspace for q4q8_gemm with M activation rows of length K."""
    import torch
    n = int(lib().q4q8_gemm_workspace_size(M, K))
    if n == 0:
        raise W4A8Error(ESHAPE, "q4q8_gemm_workspace_size")
    return _empty(n, torch.uint8, device, stream)


def q4q8_gemm(w, xq, M, N, K, y=None, workspace=None, stream=None):
    """y[M, N] = W4A8(xq [M, K/32 Q8_0 blocks], w [N, K/32 Q4_0 blocks]) in fp32."""
    import torch
    if y is None:
        y = _empty((M, N), torch.float32, w.device, stream)
    if workspace is None and M > 1:
        workspace = gemm_workspace(M, K, w.device, stream)
    nbytes = 0 if workspace is None else workspace.numel()
    _check(lib().q4q8_gemm(_p(_u8(w)), _p(_u8(xq)), _p(y), M, N, K, _p(workspace), nbytes,
                           _stream(stream)), "q4q8_gemm")
    return y


def moe_sym_workspace(T, H, I, E, k, device="cuda"):
    """A workspace for moe_sym_forward."""
    import torch
    n = int(lib().moe_sym_workspace_size(T, H, I, E, k))
    if n == 0:
        raise W4A8Error(ESHAPE, "moe_sym_workspace_size")
    return torch.empty(n, dtype=torch.uint8, device=device)


def moe_sym_workspace_layout(T, H, I, E, k) -> dict:
    offs = (ctypes.c_size_t * 3)()
    _check(lib().moe_sym_workspace_layout(T, H, I, E, k, offs), "moe_sym_workspace_layout")
    return {"xq": offs[0], "h": offs[1], "hq": offs[2]}


def moe_sym_forward(hidden, topk_ids, topk_w, w_gate_up, w_down, ws_gate_up, ws_down,
                    H, I, E, k, workspace, out=None, stream=None):
    """The MoE layer in the paper's own format (Q4_SYM weights, Q8_F32
    activations); returns out [T, H] fp32."""
    import torch
    T = hidden.shape[0]
    assert hidden.dtype == torch.float32 and hidden.is_contiguous()
    assert topk_ids.dtype == torch.int32 and topk_ids.is_contiguous()
    assert topk_w.dtype == torch.float32 and topk_w.is_contiguous()
    if out is None:
        out = _empty((T, H), torch.float32, hidden.device, stream)
    rc = lib().moe_sym_forward(_p(hidden), _p(topk_ids), _p(topk_w), _p(_u8(w_gate_up)),
                               _p(_u8(w_down)), _p(ws_gate_up), _p(ws_down), _p(out),
                               T, H, I, E, k, _p(workspace), workspace.numel(), _stream(stream))
    _check(rc, "moe_sym_forward")
    return out


def gdn_scan(q, k, v, g, beta, s0=None, out=None, s_out=None, workspace=None, stream=None):
    """The gated-delta-net recurrence as a chunked scan (gdn_chunked_scan):
    q, k [T, NH, DK], v [T, NH, DV], g and beta [T, NH], s0 [NH, DK, DV] or
    None; returns (out [T, NH, DV], s_out [NH, DK, DV]), fp32."""
    import torch
    T, NH, DK = k.shape
    DV = v.shape[2]
    for t in (q, k, v, g, beta, s0):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous())
    if out is None:
        out = _empty((T, NH, DV), torch.float32, k.device, stream)
    if s_out is None:
        s_out = _empty((NH, DK, DV), torch.float32, k.device, stream)
    if workspace is None:
        n = int(lib().gdn_workspace_size(T, NH, DK, DV))
        if n == 0:
            raise W4A8Error(ESHAPE, "gdn_workspace_size")
        workspace = _empty(n, torch.uint8, k.device, stream)
    _check(lib().gdn_chunked_scan(_p(q), _p(k), _p(v), _p(g), _p(beta), _p(s0), _p(out),
                                  _p(s_out), T, NH, DK, DV, _p(workspace), workspace.numel(),
                                  _stream(stream)), "gdn_chunked_scan")
    return out, s_out


def q4_sym_quantize(w, out=None, stream=None):
    """The paper's symmetric 4-bit weights ({-7..7}, fp32 scale per 32) of fp32
    rows w [rows, K] -> uint8 [rows, K/32*20] on w's device."""
    import torch
    assert w.dtype == torch.float32 and w.is_contiguous()
    rows, K = (1, w.numel()) if w.dim() == 1 else (w.numel() // w.shape[-1], w.shape[-1])
    if out is None:
        out = _empty((rows, K // 32 * Q4_SYM_BLOCK_BYTES), torch.uint8, w.device, stream)
    _check(lib().q4_sym_quantize(_p(w), _p(_u8(out)), rows, K, _stream(stream)), "q4_sym_quantize")
    return out


def q8_f32_quantize(x, out=None, stream=None):
    """8-bit activations with an fp32 scale per 32 of fp32 rows x [rows, K] ->
    uint8 [rows, K/32*36] on x's device."""
    import torch
    assert x.dtype == torch.float32 and x.is_contiguous()
    rows, K = (1, x.numel()) if x.dim() == 1 else (x.numel() // x.shape[-1], x.shape[-1])
    if out is None:
        out = _empty((rows, K // 32 * Q8_F32_BLOCK_BYTES), torch.uint8, x.device, stream)
    _check(lib().q8_f32_quantize(_p(x), _p(_u8(out)), rows, K, _stream(stream)), "q8_f32_quantize")
    return out


def q4sym_q8f32_gemv(w, xq, N, K, y=None, stream=None):
    """y[N] = product of w [N, K/32 Q4_SYM blocks] and xq [K/32 Q8_F32 blocks]."""
    import torch
    if y is None:
        y = _empty(N, torch.float32, w.device, stream)
    _check(lib().q4sym_q8f32_gemv(_p(_u8(w)), _p(_u8(xq)), _p(y), N, K, _stream(stream)),
           "q4sym_q8f32_gemv")
    return y


def router_topk(logits, k, ids=None, weights=None, stream=None):
    """Top-k of fp32 logits [T, E] (descending, equal logits by increasing
    index) and the softmax weights renormalized over the selection; returns
    (ids int32 [T, k], weights fp32 [T, k])."""
    import torch
    assert logits.dtype == torch.float32 and logits.is_contiguous() and logits.dim() == 2
    T, E = logits.shape
    if ids is None:
        ids = _empty((T, k), torch.int32, logits.device, stream)
    if weights is None:
        weights = _empty((T, k), torch.float32, logits.device, stream)
    _check(lib().moe_router_topk(_p(logits), _p(ids), _p(weights), T, E, k, _stream(stream)),
           "moe_router_topk")
    return ids, weights


def moe_workspace_size(T, H, I, E, k) -> int:
    return int(lib().moe_w4a8_workspace_size(T, H, I, E, k))


def moe_workspace(T, H, I, E, k, device="cuda", stream=None):
    """Allocate and zero-fill a workspace for these sizes."""
    import torch
    n = moe_workspace_size(T, H, I, E, k)
    if n == 0:
        raise W4A8Error(ESHAPE, "moe_workspace_size")
    ws = _empty(n, torch.uint8, device, stream)
    _check(lib().moe_w4a8_workspace_init(_p(ws), n, _stream(stream)), "moe_w4a8_workspace_init")
    return ws


def moe_workspace_layout(T, H, I, E, k) -> dict:
    offs = (ctypes.c_size_t * WS_NFIELDS)()
    _check(lib().moe_w4a8_workspace_layout(T, H, I, E, k, offs), "moe_w4a8_workspace_layout")
    return {"xq": offs[WS_XQ], "h": offs[WS_H], "hq": offs[WS_HQ], "perm": offs[WS_PERM],
            "count": offs[WS_COUNT], "sync": offs[WS_SYNC], "sync_end": offs[WS_SYNC_END],
            "xn": offs[WS_XN]}


def moe_forward(hidden, topk_ids, topk_w, w_gate_up, w_down, ws_gate_up, ws_down,
                H, I, E, k, workspace, out=None, stream=None):
    """One routed + shared W4A8 MoE layer; returns out [T, H] fp32."""
    import torch
    T = hidden.shape[0]
    assert hidden.dtype == torch.float32 and hidden.is_contiguous()
    assert topk_ids.dtype == torch.int32 and topk_ids.is_contiguous()
    assert topk_w.dtype == torch.float32 and topk_w.is_contiguous()
    if out is None:
        out = _empty((T, H), torch.float32, hidden.device, stream)
    rc = lib().moe_w4a8_forward(_p(hidden), _p(topk_ids), _p(topk_w), _p(_u8(w_gate_up)),
                                _p(_u8(w_down)), _p(ws_gate_up), _p(ws_down), _p(out),
                                T, H, I, E, k, _p(workspace), workspace.numel(),
                                _stream(stream))
    _check(rc, "moe_w4a8_forward")
    return out


def rmsnorm_residual(x, y, gamma, eps=1e-6, x_out=None, xn=None, want_norm=True, stream=None):
    """x_out = x + y (y may be None) and xn = RMSNorm(x_out) * gamma per row of
    [T, H] fp32; returns (x_out, xn).  x_out may be x itself (in place)."""
    import torch
    T, H = x.shape
    for t in (x, y, gamma):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous())
    if x_out is None:
        x_out = _empty(x.shape, x.dtype, x.device, stream)
    if want_norm and xn is None:
        xn = _empty(x.shape, x.dtype, x.device, stream)
    rc = lib().rmsnorm_residual(_p(x), _p(y), _p(gamma if want_norm else None), _p(x_out),
                                _p(xn if want_norm else None), T, H, float(eps), _stream(stream))
    _check(rc, "rmsnorm_residual")
    return x_out, (xn if want_norm else None)


def moe_layer(x, y_prev, gamma, topk_ids, topk_w, w_gate_up, w_down, ws_gate_up, ws_down,
              H, I, E, k, workspace, eps=1e-6, x_out=None, out=None, stream=None):
    """One pre-norm residual MoE step: x_out = x + y_prev, out = MoE(RMSNorm(x_out)
    * gamma); returns (x_out, out)."""
    import torch
    T = x.shape[0]
    for t in (x, y_prev, gamma, topk_w):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous())
    assert topk_ids.dtype == torch.int32 and topk_ids.is_contiguous()
    if x_out is None:
        x_out = _empty(x.shape, x.dtype, x.device, stream)
    if out is None:
        out = _empty(x.shape, x.dtype, x.device, stream)
    rc = lib().moe_w4a8_layer(_p(x), _p(y_prev), _p(gamma), float(eps), _p(x_out), _p(topk_ids),
                              _p(topk_w), _p(_u8(w_gate_up)), _p(_u8(w_down)), _p(ws_gate_up),
                              _p(ws_down), _p(out), T, H, I, E, k, _p(workspace),
                              workspace.numel(), _stream(stream))
    _check(rc, "moe_w4a8_layer")
    return x_out, out


def moe_layer_routed(x, y_prev, gamma, router_logits, w_gate_up, w_down, ws_gate_up, ws_down,
                     H, I, E, k, workspace, shared_gate=None, eps=1e-6, x_out=None, out=None,
                     topk_ids=None, topk_w=None, stream=None):
    """moe_layer with the router in front: top-k of router_logits [T, E] and
    the renormalized softmax weights, an optional sigmoid gate [T] on the
    shared expert; returns (x_out, out, topk_ids, topk_w)."""
    import torch
    T = x.shape[0]
    for t in (x, y_prev, gamma, router_logits, shared_gate):
        assert t is None or (t.dtype == torch.float32 and t.is_contiguous())
    if x_out is None:
        x_out = _empty(x.shape, x.dtype, x.device, stream)
    if out is None:
        out = _empty(x.shape, x.dtype, x.device, stream)
    if topk_ids is None:
        topk_ids = _empty((T, k), torch.int32, x.device, stream)
    if topk_w is None:
        topk_w = _empty((T, k), torch.float32, x.device, stream)
    rc = lib().moe_w4a8_layer_routed(_p(x), _p(y_prev), _p(gamma), float(eps), _p(x_out),
                                     _p(router_logits), _p(shared_gate), _p(_u8(w_gate_up)),
                                     _p(_u8(w_down)), _p(ws_gate_up), _p(ws_down), _p(out),
                                     _p(topk_ids), _p(topk_w), T, H, I, E, k, _p(workspace),
                                     workspace.numel(), _stream(stream))
    _check(rc, "moe_w4a8_layer_routed")
    return x_out, out, topk_ids, topk_w


def decode_wait_bound(rounds: int = -1) -> int:
    """Set the single-token kernel's bound on poll rounds (rounds >= 0);
    returns the previous bound."""
    return int(lib().w4a8_decode_wait_bound(int(rounds)))


def moe_forward_noalloc(hidden, topk_ids, topk_w, w_gate_up, w_down, ws_gate_up, ws_down,
                        H, I, E, k, out=None, stream=None):
    """moe_forward without a workspace argument: the library's fixed per-GPU
    scratch array serves as the workspace (moe_w4a8_forward_noalloc).  With
    `out` given, nothing is allocated."""
    import torch
    T = hidden.shape[0]
    assert hidden.dtype == torch.float32 and hidden.is_contiguous()
    assert topk_ids.dtype == torch.int32 and topk_ids.is_contiguous()
    assert topk_w.dtype == torch.float32 and topk_w.is_contiguous()
    if out is None:
        out = _empty((T, H), torch.float32, hidden.device, stream)
    rc = lib().moe_w4a8_forward_noalloc(_p(hidden), _p(topk_ids), _p(topk_w), _p(_u8(w_gate_up)),
                                        _p(_u8(w_down)), _p(ws_gate_up), _p(ws_down), _p(out),
                                        T, H, I, E, k, _stream(stream))
    _check(rc, "moe_w4a8_forward_noalloc")
    return out


# ------------------------------------------------------------------ attention and logits
# These calls are short (a token's rotation takes 3 us on the GPU), so their
# checks are written for few Python operations each.
def _call(what, stream, tensors, *args):
    """Entry point `what` with `args` and a stream (None: the current one) on
    the GPU that all of `tensors` are on, made current for the call."""
    dev = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise ValueError(f"tensors on {tensors[0].device} and {t.device} in one call")
    if dev < 0:
        raise ValueError(f"tensors on {tensors[0].device}: a GPU's are needed")
    C, f = torch._C, getattr(_lib or lib(), what)
    here = C._cuda_getDevice()
    if here == dev:
        rc = f(*args, stream.cuda_stream if stream is not None else C._cuda_getCurrentRawStream(dev))
    else:
        C._cuda_setDevice(dev)
        try:
            rc = f(*args, stream.cuda_stream if stream is not None else C._cuda_getCurrentRawStream(dev))
        finally:
            C._cuda_setDevice(here)
    if rc != OK:
        raise W4A8Error(rc, what)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _zeros(n, device, stream=None):
    """A workspace, zero-filled and held on the stream that uses it."""
    with torch.cuda.stream(stream):
        return torch.zeros(n, dtype=torch.uint8, device=device)


def _is(t, dtype, shape, what):
    """A contiguous tensor of this type and shape (None: any size)."""
    if t.dtype is dtype and t.is_contiguous():
        if t.shape == shape or \
                None in shape and t.dim() == len(shape) and all(n in (None, m) for n, m in zip(shape, t.shape)):
            return
    raise ValueError(f"{what}: a contiguous {dtype} tensor of shape {shape} is needed, "
                     f"got {t.dtype} {tuple(t.shape)} with strides {t.stride()}")


def _heads(x, shape, what):
    """[rows, heads, D] fp32 of this shape with contiguous heads; returns the
    row stride."""
    if x.dtype is torch.float32 and x.shape == shape and len(shape) == 3:
        if x.is_contiguous():
            return shape[1] * shape[2]
        T, NH, D = shape
        s0, s1, s2 = x.stride()
        if s2 == 1 and (NH == 1 or s1 == D):
            return s0 if T > 1 else max(s0, NH * D)
    raise ValueError(f"{what}: fp32 [rows, heads, D] = {tuple(shape)} with contiguous heads is needed, "
                     f"got {x.dtype} {tuple(x.shape)} with strides {x.stride()}")


def _rope(pos, inv_freq, layout, mscale, T):
    _is(pos, torch.int32, (T,), "pos")
    if inv_freq.dtype is not torch.float64 or inv_freq.dim() != 1 or not inv_freq.is_contiguous():
        _is(inv_freq, torch.float64, (None,), "inv_freq")
    if layout not in ROPE_LAYOUTS:
        raise ValueError(f"layout {layout!r}: one of {sorted(ROPE_LAYOUTS)}")
    return _RopeArgs(inv_freq.data_ptr(), pos.data_ptr(), 2 * inv_freq.numel(),
                     ROPE_LAYOUTS[layout], mscale)


def rope_frequencies(n_rot, base=10000.0, kind="none", factor=1.0, orig_len=0, beta_fast=32.0,
                     beta_slow=1.0, device="cuda", out=None, stream=None):
    """Frequencies of the n_rot / 2 rotated pairs, fp64 radians per position:
    base^(-2i / n_rot), as they are ("none"), over factor ("linear"), or mixed
    by how often a pair turns within orig_len positions ("parts")."""
    if kind not in ROPE_KINDS:
        raise ValueError(f"kind {kind!r}: one of {sorted(ROPE_KINDS)}")
    if out is None:
        out = _empty(max(0, n_rot // 2), torch.float64, device, stream)
    _is(out, torch.float64, (n_rot // 2,), "out")
    _call("rope_frequencies", stream, (out,), _ptr(out), n_rot, base, ROPE_KINDS[kind], factor,
          orig_len, beta_fast, beta_slow)
    return out


def rope_rotate(x, pos, inv_freq, layout="half", mscale=1.0, out=None, stream=None):
    """The heads of x [T, NH, D] turned by their rows' positions pos [T] (the
    first 2 * len(inv_freq) elements; out may be x)."""
    shape = x.shape
    xs = _heads(x, shape, "x")
    T, NH, D = shape
    r = _rope(pos, inv_freq, layout, mscale, T)
    if out is None:
        out = _empty(shape, torch.float32, x.device, stream)
    os_ = _heads(out, shape, "out")
    if T:
        _call("rope_rotate", stream, (x, pos, inv_freq, out), ctypes.byref(r), x.data_ptr(), xs,
              out.data_ptr(), os_, T, NH, D)
    return out


def kv_tile_bytes(D, fmt="q4_0") -> int:
    return int(lib().kv_q4_tile_bytes(D, KV_FORMATS[fmt]))


def kv_pools(n_pages, NKV, D, fmt="q4_0", device="cuda"):
    """Key and value pools of n_pages pages (any contents) for NKV heads."""
    n = kv_tile_bytes(D, fmt)
    if n == 0:
        raise W4A8Error(ESHAPE, "kv_q4_tile_bytes")
    new = lambda: torch.empty((n_pages, NKV, n), dtype=torch.uint8, device=device)
    return new(), new()


class KVCache:
    """A plan of the paged 4-bit cache (w4a8_kv): the pools [n_pages, NKV,
    tile bytes] (kv_pools), page_table [B, max_pages], kv_len [B] (this call's
    rows included) and cu_rows [B + 1].  It keeps the tensors, which are read
    on the device at each call: update them in place between steps."""

    def __init__(self, k_pages, v_pages, page_table, kv_len, cu_rows, D, fmt="q4_0"):
        if fmt not in KV_FORMATS:
            raise ValueError(f"format {fmt!r}: one of {sorted(KV_FORMATS)}")
        n = kv_tile_bytes(D, fmt)
        if n == 0:
            raise W4A8Error(ESHAPE, "KVCache")
        _is(k_pages, torch.uint8, (None, None, n), "k_pages")
        _is(v_pages, torch.uint8, tuple(k_pages.shape), "v_pages")
        _is(page_table, torch.int32, (None, None), "page_table")
        B, max_pages = page_table.shape
        _is(kv_len, torch.int32, (B,), "kv_len")
        _is(cu_rows, torch.int32, (B + 1,), "cu_rows")
        self.tensors = (k_pages, v_pages, page_table, kv_len, cu_rows)
        for t in self.tensors:
            if t.device != k_pages.device:
                raise ValueError(f"tensors on {k_pages.device} and {t.device} in one plan")
        self.NKV, self.D, self.device = k_pages.shape[1], D, k_pages.device
        self.args = _KvArgs(*(t.data_ptr() for t in self.tensors), k_pages.shape[0], max_pages, B,
                            self.NKV, D, KV_FORMATS[fmt])
        self.ref = ctypes.byref(self.args)


def kv_append(kv, k, v, pos=None, inv_freq=None, layout="half", mscale=1.0, q=None, q_out=None,
              stream=None):
    """Stores the rows k, v [T, NKV, D] as the last tokens of kv's sequences,
    the keys rotated when pos [T] and inv_freq are given; with q [T, NH, D] the
    same launch rotates the queries, which are returned."""
    T = k.shape[0]
    shape = (T, kv.NKV, kv.D)
    ks, vs = _heads(k, shape, "k"), _heads(v, shape, "v")
    if (pos is None) != (inv_freq is None):
        raise ValueError("pos and inv_freq go together")
    r = None if pos is None else _rope(pos, inv_freq, layout, mscale, T)
    NH = qs = 0
    if q is not None:
        NH = q.shape[1] if q.dim() == 3 else 0
        shape = (T, NH, kv.D)
        qs = _heads(q, shape, "q")
        if q_out is None:
            q_out = _empty(shape, torch.float32, q.device, stream)
        _is(q_out, torch.float32, shape, "q_out")
    else:
        q_out = None
    if T:
        _call("kv_q4_append", stream, (kv.tensors[0], k, v, pos, inv_freq, q, q_out), kv.ref,
              None if r is None else ctypes.byref(r), k.data_ptr(), ks, v.data_ptr(), vs, _ptr(q), qs,
              _ptr(q_out), NH, T)
    return q_out


def kv_read(kv, T, k_out=None, v_out=None, stream=None):
    """The T rows of kv's sequences as fp32 (k, v) [T, NKV, D]."""
    shape = (T, kv.NKV, kv.D)
    if k_out is None:
        k_out = _empty(shape, torch.float32, kv.device, stream)
    if v_out is None:
        v_out = _empty(shape, torch.float32, kv.device, stream)
    _is(k_out, torch.float32, shape, "k_out")
    _is(v_out, torch.float32, shape, "v_out")
    if T:
        _call("kv_q4_read", stream, (kv.tensors[0], k_out, v_out), kv.ref, k_out.data_ptr(),
              v_out.data_ptr(), T)
    return k_out, v_out


def attn_workspace(kv, T, NH, stream=None):
    """A workspace for attn_forward with T rows of NH heads on kv's plan
    (zero-filled on the stream; each call of attn_forward leaves it ready for
    the next)."""
    n = int(lib().attn_q4_workspace_size(kv.ref, T, NH))
    if n == 0:
        raise W4A8Error(ESHAPE, "attn_q4_workspace_size")
    return _zeros(n, kv.device, stream)


def attn_forward(kv, q, scale, window=0, out=None, lse=None, want_lse=True, workspace=None,
                 stream=None):
    """Softmax attention of q [T, NH, D] (kv's rows) over the 4-bit cache;
    returns (out [T, NH, D], lse [T, NH] or None)."""
    T, NH = q.shape[:2] if q.dim() == 3 else (0, 0)
    shape = (T, NH, kv.D)
    qs = _heads(q, shape, "q")
    if out is None:
        out = _empty(shape, torch.float32, q.device, stream)
    _is(out, torch.float32, shape, "out")
    if lse is None and want_lse:
        lse = _empty((T, NH), torch.float32, q.device, stream)
    if lse is not None:
        _is(lse, torch.float32, (T, NH), "lse")
    if T:
        if workspace is None:
            workspace = attn_workspace(kv, T, NH, stream)
        elif not workspace.is_contiguous():
            raise ValueError("workspace: a contiguous tensor is needed")
        _call("attn_q4_forward", stream, (kv.tensors[0], q, out, lse, workspace), kv.ref, q.data_ptr(),
              qs, out.data_ptr(), _ptr(lse), T, NH, scale, window, workspace.data_ptr(),
              workspace.numel() * workspace.element_size())
    return out, lse


def logprobs_workspace(T, V, n_top=0, device="cuda", stream=None):
    """A workspace for token_logprobs (zero-filled on the stream; each call of
    it leaves it ready for the next)."""
    n = int(lib().token_logprobs_workspace_size(T, V, n_top))
    if n == 0:
        raise W4A8Error(ERANGE, "token_logprobs_workspace_size")
    return _zeros(n, device, stream)


def token_logprobs(logits, targets=None, n_top=0, want_entropy=True, logprob=None, entropy=None,
                   top_ids=None, top_logprobs=None, workspace=None, stream=None):
    """From fp32 logits [T, V] (rows may be strided): (log probability of
    targets [T] int32, entropy [T], the n_top largest logits' ids int32 and log
    probabilities [T, n_top]); None where not asked for."""
    if logits.dtype is not torch.float32 or logits.dim() != 2 or \
            (logits.shape[1] != 1 and logits.stride(1) != 1):
        raise ValueError(f"logits: fp32 [T, V] with contiguous rows is needed, got {logits.dtype} "
                         f"{tuple(logits.shape)} with strides {logits.stride()}")
    T, V = logits.shape
    stride = logits.stride(0)
    if T == 1 and stride < V:
        stride = V
    new = logits.new_empty if stream is None else \
        lambda shape, dtype=torch.float32: _empty(shape, dtype, logits.device, stream)
    if targets is not None:
        _is(targets, torch.int32, (T,), "targets")
        if logprob is None:
            logprob = new((T,))
        else:
            _is(logprob, torch.float32, (T,), "logprob")
    else:
        logprob = None
    if entropy is not None:
        _is(entropy, torch.float32, (T,), "entropy")
    elif want_entropy:
        entropy = new((T,))
    if n_top > 0:
        if top_ids is None:
            top_ids = new((T, n_top), dtype=torch.int32)
        else:
            _is(top_ids, torch.int32, (T, n_top), "top_ids")
        if top_logprobs is None:
            top_logprobs = new((T, n_top))
        else:
            _is(top_logprobs, torch.float32, (T, n_top), "top_logprobs")
    else:
        top_ids = top_logprobs = None
    if T:
        if workspace is None:
            workspace = logprobs_workspace(T, V, n_top, logits.device, stream)
        elif not workspace.is_contiguous():
            raise ValueError("workspace: a contiguous tensor is needed")
        _call("token_logprobs", stream,
              (logits, targets, logprob, entropy, top_ids, top_logprobs, workspace), logits.data_ptr(),
              stride, _ptr(targets), _ptr(logprob), _ptr(entropy), _ptr(top_ids), _ptr(top_logprobs),
              T, V, n_top, workspace.data_ptr(), workspace.numel() * workspace.element_size())
    return logprob, entropy, top_ids, top_logprobs


# ------------------------------------------------------------------ around a layer's recurrence
def _rows(x, shape, what):
    """fp32 [rows, n] of this shape with contiguous rows; returns the row
    stride."""
    if x.dtype is torch.float32 and x.shape == shape and len(shape) == 2:
        T, n = shape
        s0, s1 = x.stride()
        if s1 == 1 or n == 1:
            return s0 if T > 1 else max(s0, n)
    raise ValueError(f"{what}: fp32 [rows, n] = {tuple(shape)} with contiguous rows is needed, "
                     f"got {x.dtype} {tuple(x.shape)} with strides {x.stride()}")


def q8_row_bytes(K) -> int:
    return int(lib().q8_row_bytes(K))


def q8_row_quantize(x, q=None, d=None, stream=None):
    """8-bit rows of fp32 x [rows, K] (rows may be strided): codes int8 [rows,
    K rounded up to 128] and scales fp32 [rows], of activations or weights."""
    shape = x.shape
    xs = _rows(x, shape, "x")
    M, K = shape
    KP = (K + Q8_ROW_PAD - 1) // Q8_ROW_PAD * Q8_ROW_PAD
    if q is None:
        q = x.new_empty((M, KP), dtype=torch.int8) if stream is None else \
            _empty((M, KP), torch.int8, x.device, stream)
    else:
        _is(q, torch.int8, (M, KP), "q")
    if d is None:
        d = x.new_empty(M) if stream is None else _empty((M,), torch.float32, x.device, stream)
    else:
        _is(d, torch.float32, (M,), "d")
    if M:
        _call("q8_row_quantize", stream, (x, q, d), x.data_ptr(), xs, q.data_ptr(), d.data_ptr(), M, K)
    return q, d


def _q8_rows(q, d, what):
    """8-bit rows: codes [rows, multiple of 128] and scales [rows]; returns
    that shape."""
    if q.dtype is torch.int8 and q.dim() == 2 and q.is_contiguous() and d.dtype is torch.float32 and \
            d.dim() == 1 and d.is_contiguous():
        rows, KP = q.shape
        if KP % Q8_ROW_PAD == 0 and d.numel() == rows:
            return rows, KP
    raise ValueError(f"{what}: contiguous int8 codes [rows, multiple of {Q8_ROW_PAD}] and fp32 scales [rows] are "
                     f"needed, got {q.dtype} {tuple(q.shape)} and {d.dtype} {tuple(d.shape)} with strides "
                     f"{q.stride()} and {d.stride()}")


def q8q8_gemm(xq, xd, wq, wd, bias=None, out=None, stream=None):
    """out [M, N] fp32 (rows may be strided) = the product of 8-bit rows xq [M,
    KP] with scales xd [M] and weight rows wq [N, KP] with scales wd [N], plus
    bias [N]."""
    M, KP = _q8_rows(xq, xd, "xq, xd")
    N, KW = _q8_rows(wq, wd, "wq, wd")
    if KP != KW:
        raise ValueError(f"xq and wq: rows of {KP} and {KW} codes")
    if bias is not None:
        _is(bias, torch.float32, (N,), "bias")
    if out is None:
        out = _empty((M, N), torch.float32, xq.device, stream)
    ys = _rows(out, (M, N), "out")
    if M:
        # (rows of 2^17 codes end with at least one of the padding: K is below 2^17)
        _call("q8q8_gemm", stream, (xq, xd, wq, wd, bias, out), xq.data_ptr(), xd.data_ptr(),
              wq.data_ptr(), wd.data_ptr(), _ptr(bias), out.data_ptr(), ys, M, N, KP - (KP == 1 << 17))
    return out


class SeqPlan:
    """The sequences of a call of the recurrent operators (w4a8_seqs): cu_rows
    [B + 1], and the slots of a pool of n_slots states that each reads (src
    [B], default its number; outside the pool: none, zeros) and writes (dst
    [B], default the one it reads; outside the pool: not kept).  It keeps the
    tensors, int32, which are read on the device at each call."""

    def __init__(self, cu_rows, n_slots, src=None, dst=None):
        _is(cu_rows, torch.int32, (None,), "cu_rows")
        B = cu_rows.shape[0] - 1
        if B < 0:
            raise ValueError("cu_rows: [B + 1] is needed, got an empty tensor")
        for t, what in ((src, "src"), (dst, "dst")):
            if t is not None:
                _is(t, torch.int32, (B,), what)
                if t.device != cu_rows.device:
                    raise ValueError(f"tensors on {cu_rows.device} and {t.device} in one plan")
        self.tensors = (cu_rows, src, dst)
        self.B, self.n_slots, self.device = B, n_slots, cu_rows.device
        self.args = _SeqArgs(cu_rows.data_ptr(), _ptr(src), _ptr(dst), n_slots, B)
        self.ref = ctypes.byref(self.args)


def short_conv(plan, x, w, state, bias=None, act="silu", out=None, stream=None):
    """The causal convolution of x [T, CH] (rows may be strided) with w [W, CH]
    along plan's sequences, and its activation ("silu" or "none"); state
    [n_slots, W - 1, CH] holds the sequences' last inputs (None without slots).
    Returns out [T, CH]."""
    xs = _rows(x, x.shape, "x")
    T, CH = x.shape
    _is(w, torch.float32, (None, CH), "w")
    W = w.shape[0]
    if state is not None:
        _is(state, torch.float32, (plan.n_slots, W - 1, CH), "state")
    elif plan.n_slots > 0:
        raise ValueError("state: the plan has slots")
    if bias is not None:
        _is(bias, torch.float32, (CH,), "bias")
    if act not in CONV_ACTS:
        raise ValueError(f"act {act!r}: one of {sorted(CONV_ACTS)}")
    if out is None:
        out = _empty((T, CH), torch.float32, x.device, stream)
    os_ = _rows(out, (T, CH), "out")
    if T:
        _call("short_conv", stream, (plan.tensors[0], x, w, state, bias, out), plan.ref, x.data_ptr(), xs,
              w.data_ptr(), _ptr(bias), _ptr(state), out.data_ptr(), os_, T, CH, W, CONV_ACTS[act])
    return out


def _ssm_sizes(plan, T, NH, NG, N, P):
    a = _SsmArgs(NH=NH, NG=NG, N=N, P=P)
    return int(lib().ssm_workspace_size(plan.ref, ctypes.byref(a), T))


def ssm_workspace(plan, T, NH, NG, N, P, stream=None):
    """A workspace for ssm_scan with T rows on plan's sequences."""
    n = _ssm_sizes(plan, T, NH, NG, N, P)
    if n == 0:
        raise W4A8Error(ESHAPE, "ssm_workspace_size")
    return _empty(n, torch.uint8, plan.device, stream)


def ssm_scan(plan, x, dt, A, B, C, state, D=None, z=None, dt_bias=None, softplus=True, out=None,
             workspace=None, stream=None):
    """The selective state space scan of x [T, NH, P] with steps dt [T, NH],
    decays A [NH], B and C [T, NG, N] (rows of all may be strided) along plan's
    sequences; state [n_slots, NH, N, P] (None without slots).  Optional: D and
    dt_bias [NH], the gate z [T, NH, P].  Returns out [T, NH, P]."""
    xs = _heads(x, x.shape, "x")
    T, NH, P = x.shape
    ds = _rows(dt, (T, NH), "dt")
    NG, N = B.shape[1:] if B.dim() == 3 else (0, 0)
    bs, cs = _heads(B, (T, NG, N), "B"), _heads(C, (T, NG, N), "C")
    zs = 0 if z is None else _heads(z, (T, NH, P), "z")
    _is(A, torch.float32, (NH,), "A")
    for t, what in ((D, "D"), (dt_bias, "dt_bias")):
        if t is not None:
            _is(t, torch.float32, (NH,), what)
    if state is not None:
        _is(state, torch.float32, (plan.n_slots, NH, N, P), "state")
    elif plan.n_slots > 0:
        raise ValueError("state: the plan has slots")
    if out is None:
        out = _empty((T, NH, P), torch.float32, x.device, stream)
    os_ = _heads(out, (T, NH, P), "out")
    if T:
        if workspace is None:
            workspace = ssm_workspace(plan, T, NH, NG, N, P, stream)
        elif not workspace.is_contiguous():
            raise ValueError("workspace: a contiguous tensor is needed")
        a = _SsmArgs(x.data_ptr(), dt.data_ptr(), B.data_ptr(), C.data_ptr(), _ptr(z), A.data_ptr(), _ptr(D),
                     _ptr(dt_bias), xs, ds, bs, cs, zs, NH, NG, N, P, 1 if softplus else 0)
        _call("ssm_scan", stream, (plan.tensors[0], x, dt, A, B, C, state, D, z, dt_bias, out, workspace),
              plan.ref, ctypes.byref(a), _ptr(state), out.data_ptr(), os_, T, workspace.data_ptr(),
              workspace.numel() * workspace.element_size())
    return out
