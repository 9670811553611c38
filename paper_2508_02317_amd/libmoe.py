"""ctypes binding of libmoe_gfx950.so: argument marshalling only.

Every function here has the name of the C entry point it calls (include/moe.h) and does
nothing but check tensor dtypes / contiguity, allocate outputs and workspaces with torch
when the caller did not pass them, and hand raw device pointers and the current HIP
stream to the library.  All arithmetic of the MoE layer runs inside the library's
kernels.  There is no fallback: if the shared library has not been built, importing this
module raises.
"""
import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmoe_gfx950.so")

MOE_OK, MOE_ERR_INVALID_ARG, MOE_ERR_UNSUPPORTED, MOE_ERR_WORKSPACE, MOE_ERR_HIP = range(5)
MOE_F32, MOE_BF16, MOE_MX8 = 0, 1, 2

EXPORTS = [
    "moe_version", "moe_last_error",
    "moe_route_topk_workspace_bytes", "moe_route_topk", "moe_route_topk_bwd",
    "moe_route_topk_noalloc_max_bytes", "moe_route_topk_noalloc",
    "moe_expert_offsets_workspace_bytes", "moe_expert_offsets",
    "moe_permute_workspace_bytes", "moe_permute",
    "moe_grouped_gemm_swiglu_fwd_workspace_bytes", "moe_grouped_gemm_swiglu_fwd",
    "moe_grouped_gemm_swiglu_bwd_workspace_bytes", "moe_grouped_gemm_swiglu_bwd",
    "moe_grouped_gemm_swiglu_fwd_gather_workspace_bytes", "moe_grouped_gemm_swiglu_fwd_gather",
    "moe_grouped_gemm_swiglu_bwd_gather_workspace_bytes", "moe_grouped_gemm_swiglu_bwd_gather",
    "moe_unpermute_combine_fwd", "moe_unpermute_combine_bwd",
    "moe_router_logits_workspace_bytes", "moe_router_logits", "moe_router_bwd_workspace_bytes", "moe_router_bwd",
    "moe_mx8_quantise", "moe_grouped_gemm_swiglu_fwd_mx8_workspace_bytes", "moe_grouped_gemm_swiglu_fwd_mx8",
    "moe_grouped_gemm_down_mx8",
    "moe_rope_table", "moe_rope_fwd", "moe_rope_bwd", "moe_kv_cache_write", "moe_kv_cache_read",
    "moe_paged_attn_decode_workspace_bytes", "moe_paged_attn_decode",
    "moe_set_launch_hook",
]


# void hook(const char* kernel_name, int phase, void* stream, void* user)
LAUNCH_HOOK = ctypes.CFUNCTYPE(None, ctypes.c_char_p, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p)


class moe_kv_cache_t(ctypes.Structure):
    """The cache descriptor of include/moe.h."""
    _fields_ = ([(n, ctypes.c_int32) for n in ("dtype", "pages", "heads", "page_size", "dim", "reserved")] +
                [(n, ctypes.c_void_p) for n in ("k", "v", "k_scales", "v_scales")] +
                [(n, ctypes.c_int64) for n in ("page_stride", "scale_page_stride")])


class MoEError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("libmoe status %d: %s" % (code, message))
        self.code = code


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            "libmoe_gfx950.so is not built (%s missing). Build it with "
            "`python -m paper_2508_02317_amd.build`; there is no fallback path." % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
    lib.moe_version.restype = ctypes.c_char_p
    lib.moe_version.argtypes = []
    lib.moe_last_error.restype = ctypes.c_char_p
    lib.moe_last_error.argtypes = []
    lib.moe_route_topk_workspace_bytes.restype = sz
    lib.moe_route_topk_workspace_bytes.argtypes = [i32, i32, i32]
    lib.moe_route_topk.restype = ctypes.c_int32
    lib.moe_route_topk.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_route_topk_noalloc_max_bytes.restype = sz
    lib.moe_route_topk_noalloc_max_bytes.argtypes = []
    lib.moe_route_topk_noalloc.restype = ctypes.c_int32
    lib.moe_route_topk_noalloc.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.moe_route_topk_bwd.restype = ctypes.c_int32
    lib.moe_route_topk_bwd.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp]
    lib.moe_expert_offsets_workspace_bytes.restype = sz
    lib.moe_expert_offsets_workspace_bytes.argtypes = [i32, i32]
    lib.moe_expert_offsets.restype = ctypes.c_int32
    lib.moe_expert_offsets.argtypes = [vp, i32, i32, vp, vp, vp, sz, vp]
    lib.moe_permute_workspace_bytes.restype = sz
    lib.moe_permute_workspace_bytes.argtypes = [i32, i32, i32]
    lib.moe_permute.restype = ctypes.c_int32
    lib.moe_permute.argtypes = [vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_grouped_gemm_swiglu_fwd_workspace_bytes.restype = sz
    lib.moe_grouped_gemm_swiglu_fwd_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.moe_grouped_gemm_swiglu_fwd.restype = ctypes.c_int32
    lib.moe_grouped_gemm_swiglu_fwd.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_grouped_gemm_swiglu_bwd_workspace_bytes.restype = sz
    lib.moe_grouped_gemm_swiglu_bwd_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.moe_grouped_gemm_swiglu_bwd.restype = ctypes.c_int32
    lib.moe_grouped_gemm_swiglu_bwd.argtypes = [vp] * 8 + [i32] * 5 + [vp] * 6 + [sz, vp]
    lib.moe_grouped_gemm_swiglu_fwd_gather_workspace_bytes.restype = sz
    lib.moe_grouped_gemm_swiglu_fwd_gather_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.moe_grouped_gemm_swiglu_fwd_gather.restype = ctypes.c_int32
    lib.moe_grouped_gemm_swiglu_fwd_gather.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_grouped_gemm_swiglu_bwd_gather_workspace_bytes.restype = sz
    lib.moe_grouped_gemm_swiglu_bwd_gather_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
    lib.moe_grouped_gemm_swiglu_bwd_gather.restype = ctypes.c_int32
    lib.moe_grouped_gemm_swiglu_bwd_gather.argtypes = [vp, vp, i32, i32, vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp]
    lib.moe_unpermute_combine_fwd.restype = ctypes.c_int32
    lib.moe_unpermute_combine_fwd.argtypes = [vp, i32, i32, i32, i32, vp, vp, vp, vp]
    lib.moe_unpermute_combine_bwd.restype = ctypes.c_int32
    lib.moe_unpermute_combine_bwd.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, vp, vp, vp]
    lib.moe_router_logits_workspace_bytes.restype = sz
    lib.moe_router_logits_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.moe_router_logits.restype = ctypes.c_int32
    lib.moe_router_logits.argtypes = [vp, vp, i32, i32, i32, i32, vp, vp, sz, vp]
    lib.moe_router_bwd_workspace_bytes.restype = sz
    lib.moe_router_bwd_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.moe_router_bwd.restype = ctypes.c_int32
    lib.moe_router_bwd.argtypes = [vp, vp, vp, i32, i32, i32, i32, i32, vp, vp, vp, sz, vp]
    lib.moe_mx8_quantise.restype = ctypes.c_int32
    lib.moe_mx8_quantise.argtypes = [vp, ctypes.c_int64, i32, vp, vp, vp]
    lib.moe_grouped_gemm_swiglu_fwd_mx8_workspace_bytes.restype = sz
    lib.moe_grouped_gemm_swiglu_fwd_mx8_workspace_bytes.argtypes = [i32, i32, i32, i32]
    lib.moe_grouped_gemm_swiglu_fwd_mx8.restype = ctypes.c_int32
    lib.moe_grouped_gemm_swiglu_fwd_mx8.argtypes = [vp, vp, i32, i32, vp] + [vp] * 6 + [i32] * 4 + [vp] * 5 + [sz, vp]
    lib.moe_grouped_gemm_down_mx8.restype = ctypes.c_int32
    lib.moe_grouped_gemm_down_mx8.argtypes = [vp] * 4 + [i32] * 4 + [vp] * 3 + [sz, vp]
    i64, f32 = ctypes.c_int64, ctypes.c_float
    lib.moe_rope_table.restype = ctypes.c_int32
    lib.moe_rope_table.argtypes = [vp, i32, i32, ctypes.c_double, vp, vp, vp]
    for turn in (lib.moe_rope_fwd, lib.moe_rope_bwd):
        turn.restype = ctypes.c_int32
        turn.argtypes = [vp, i64, i64] * 2 + [i32] * 6 + [vp] * 3 + [i32] * 2 + [vp, i64, i64] * 2 + [vp]
    lib.moe_kv_cache_write.restype = ctypes.c_int32
    lib.moe_kv_cache_write.argtypes = [vp] + [vp, i64, i64] * 2 + [i32, vp] + [vp, i64, i64] + [i32] * 2 + [vp] * 3 + [i32] * 2 + [vp, i64, i64, vp]
    lib.moe_kv_cache_read.restype = ctypes.c_int32
    lib.moe_kv_cache_read.argtypes = [vp, vp, i32, vp, vp, i32, i32, vp, vp, vp]
    lib.moe_paged_attn_decode_workspace_bytes.restype = sz
    lib.moe_paged_attn_decode_workspace_bytes.argtypes = [i32] * 6
    lib.moe_paged_attn_decode.restype = ctypes.c_int32
    lib.moe_paged_attn_decode.argtypes = [vp, i64, i64, vp, vp, i32, vp, i32, i32, f32, i32, vp, vp, vp, sz, vp]
    lib.moe_set_launch_hook.restype = ctypes.c_int32
    lib.moe_set_launch_hook.argtypes = [LAUNCH_HOOK, vp]
    return lib


lib = _load()
try:
    from . import _marshal              # csrc/marshal.cpp: the checks and the call of the functions that a generation step makes most
except ImportError:                     # not built on this host: the same through ctypes
    _marshal = None
_raw_stream, _current_device = getattr(torch._C, "_cuda_getCurrentRawStream", None), torch.cuda.current_device


def moe_version():
    return lib.moe_version().decode()


def moe_last_error():
    return lib.moe_last_error().decode()


def moe_set_launch_hook(hook):
    """hook: a LAUNCH_HOOK instance (kept alive by the caller) or None to remove it."""
    _check(lib.moe_set_launch_hook(hook if hook is not None else LAUNCH_HOOK(), None))


def _check(status):
    if status != MOE_OK:
        raise MoEError(status, moe_last_error())


# The host's share of a call is marshalling, and a small layer's ten calls take longer there than their kernels on the GPU.  So pointers
# go as plain integers, the stream as its raw handle, and the workspace size is asked for only where a workspace has to be made.  fp32
# step of 256 tokens, all in one process: kernels alone (20 steps replayed from a graph) 45 us a step; steps in a row 78 -> 57 us, all of
# it the host's time; one step enqueued on an idle GPU 89 -> 67 us.  A forward of 16 tokens on an idle GPU: 41 -> 29 us to enqueue.

def _ptr(t):
    return None if t is None else t.data_ptr()


def _dtype_code(t):
    if t.dtype == torch.float32:
        return MOE_F32
    if t.dtype == torch.bfloat16:
        return MOE_BF16
    raise TypeError("libmoe supports float32 and bfloat16 tensors, got %s" % t.dtype)


def _need(t, dtype=None, name="tensor"):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError("%s must be a contiguous device tensor" % name)
    if dtype is not None and t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return t


if _raw_stream is not None:
    def _stream():
        """The current stream of the current device (torch.cuda.current_stream() makes an object of it, 1 us)."""
        return _raw_stream(_current_device())
else:                                     # the shortcut is not public, and absent from a torch without devices
    def _stream():
        return torch.cuda.current_stream().cuda_stream


def _ws(query, args, ws, device):
    """ws, or a new workspace of query(*args) bytes, and its size."""
    if ws is None:
        ws = torch.empty(max(int(query(*args)), 256), dtype=torch.uint8, device=device)
    return ws, ws.numel()


# --------------------------------------------------------------------------------------------

def moe_route_topk(logits, k, renorm=1, out=None, ws=None):
    """-> topk_idx [T,k] i32, topk_w [T,k] f32, counts [E] i32, offsets [E+1] i32."""
    _need(logits, torch.float32, "logits")
    T, E = logits.shape
    dev = logits.device
    if out is None:
        out = (torch.empty((T, k), dtype=torch.int32, device=dev), torch.empty((T, k), dtype=torch.float32, device=dev),
               torch.empty(E, dtype=torch.int32, device=dev), torch.empty(E + 1, dtype=torch.int32, device=dev))
    idx, w, counts, offsets = out
    ws, nbytes = _ws(lib.moe_route_topk_workspace_bytes, (T, E, k), ws, dev)
    _check(lib.moe_route_topk(_ptr(logits), T, E, k, int(renorm), _ptr(idx), _ptr(w), _ptr(counts), _ptr(offsets),
                              _ptr(ws), nbytes, _stream()))
    return idx, w, counts, offsets


def moe_route_topk_noalloc(logits, k, renorm, out):
    """moe_route_topk without a workspace (histogram rows in the library's static device array); `out` =
    (topk_idx, topk_w, counts, offsets) must be given: nothing is allocated here either."""
    _need(logits, torch.float32, "logits")
    T, E = logits.shape
    idx, w, counts, offsets = out
    _check(lib.moe_route_topk_noalloc(_ptr(logits), T, E, k, int(renorm), _ptr(idx), _ptr(w), _ptr(counts), _ptr(offsets),
                                      _stream()))
    return idx, w, counts, offsets


def moe_expert_offsets(topk_idx, E, out=None, ws=None):
    """-> counts [E] i32, offsets [E+1] i32 of a known assignment."""
    _need(topk_idx, torch.int32, "topk_idx")
    n = topk_idx.numel()
    dev = topk_idx.device
    if out is None:
        out = (torch.empty(E, dtype=torch.int32, device=dev), torch.empty(E + 1, dtype=torch.int32, device=dev))
    counts, offsets = out
    ws, nbytes = _ws(lib.moe_expert_offsets_workspace_bytes, (n, E), ws, dev)
    _check(lib.moe_expert_offsets(_ptr(topk_idx), n, E, _ptr(counts), _ptr(offsets), _ptr(ws), nbytes, _stream()))
    return counts, offsets


def moe_route_topk_bwd(dw, topk_w, topk_idx, logits, E, renorm=1, out=None):
    """-> dlogits [T,E] f32."""
    _need(dw, torch.float32, "dw"); _need(topk_w, torch.float32, "topk_w"); _need(topk_idx, torch.int32, "topk_idx")
    T, k = topk_idx.shape
    if out is None:
        out = torch.empty((T, E), dtype=torch.float32, device=dw.device)
    _check(lib.moe_route_topk_bwd(_ptr(dw), _ptr(topk_w), _ptr(topk_idx), _ptr(logits), T, E, k, int(renorm),
                                  _ptr(out), _stream()))
    return out


def moe_permute(x, topk_idx, offsets, E, out=None, ws=None):
    """-> xp [P,d], row_of_pair [P] i32, pair_of_row [P] i32.  x None: only the two maps (xp is None)."""
    _need(topk_idx, torch.int32, "topk_idx"); _need(offsets, torch.int32, "offsets")
    T, k = topk_idx.shape
    P = T * k
    dev = topk_idx.device
    if x is not None:
        _need(x, None, "x")
        d = x.shape[1]
    else:
        d = 8
    if out is None:
        out = (torch.empty((P, d), dtype=x.dtype, device=dev) if x is not None else None,
               torch.empty(P, dtype=torch.int32, device=dev), torch.empty(P, dtype=torch.int32, device=dev))
    xp, row_of_pair, pair_of_row = out
    if x is None:
        xp = None
    ws, nbytes = _ws(lib.moe_permute_workspace_bytes, (T, E, k), ws, dev)
    _check(lib.moe_permute(_ptr(x), _dtype_code(x) if x is not None else MOE_BF16, T, d, E, k, _ptr(topk_idx), _ptr(offsets),
                           _ptr(xp), _ptr(row_of_pair), _ptr(pair_of_row), _ptr(ws), nbytes, _stream()))
    return xp, row_of_pair, pair_of_row


def moe_grouped_gemm_swiglu_fwd(xp, w_gate, w_up, w_down, offsets, save_gu=True, out=None, ws=None):
    """-> act [P,f], yp [P,d], g_save, u_save ([P,f] or None)."""
    _need(xp, None, "xp"); _need(offsets, torch.int32, "offsets")
    for name, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(w, xp.dtype, name)
    P, d = xp.shape
    E, f, _ = w_gate.shape
    dev = xp.device
    if out is None:
        mk = lambda *s: torch.empty(s, dtype=xp.dtype, device=dev)
        out = (mk(P, f), mk(P, d), mk(P, f) if save_gu else None, mk(P, f) if save_gu else None)
    act, yp, g, u = out
    code = _dtype_code(xp)
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_fwd_workspace_bytes, (code, P, d, f, E), ws, dev)
    _check(lib.moe_grouped_gemm_swiglu_fwd(_ptr(xp), _ptr(w_gate), _ptr(w_up), _ptr(w_down), code, P, d, f, E,
                                           _ptr(offsets), _ptr(g), _ptr(u), _ptr(act), _ptr(yp), _ptr(ws), nbytes,
                                           _stream()))
    return act, yp, g, u


def moe_grouped_gemm_swiglu_bwd(dyp, xp, g_save, u_save, act, w_gate, w_up, w_down, offsets, out=None, ws=None):
    """-> dxp [P,d], dw_gate [E,f,d], dw_up [E,f,d], dw_down [E,d,f]."""
    _need(dyp, xp.dtype, "dyp"); _need(xp, None, "xp"); _need(act, xp.dtype, "act")
    P, d = xp.shape
    E, f, _ = w_gate.shape
    if out is None:
        out = (torch.empty_like(xp), torch.empty_like(w_gate), torch.empty_like(w_up), torch.empty_like(w_down))
    dxp, dwg, dwu, dwd = out
    code = _dtype_code(xp)
    have_saved = int(g_save is not None)
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_bwd_workspace_bytes, (code, P, d, f, E, have_saved), ws, xp.device)
    _check(lib.moe_grouped_gemm_swiglu_bwd(_ptr(dyp), _ptr(xp), _ptr(g_save), _ptr(u_save), _ptr(act), _ptr(w_gate),
                                           _ptr(w_up), _ptr(w_down), code, P, d, f, E, _ptr(offsets), _ptr(dxp),
                                           _ptr(dwg), _ptr(dwu), _ptr(dwd), _ptr(ws), nbytes, _stream()))
    return dxp, dwg, dwu, dwd


def moe_grouped_gemm_swiglu_fwd_gather(x, k, pair_of_row, w_gate, w_up, w_down, offsets, save_gu=True, out=None, ws=None, topk_w=None):
    """Forward without xp: rows are read as x[pair_of_row[r] // k].  -> act [P,f], yp [P,d], g_save, u_save.
    With topk_w [T,k], act and yp leave scaled by each row's combine weight."""
    if topk_w is not None:
        _need(topk_w, torch.float32, "topk_w")
    _need(x, None, "x"); _need(pair_of_row, torch.int32, "pair_of_row"); _need(offsets, torch.int32, "offsets")
    for name, w in (("w_gate", w_gate), ("w_up", w_up), ("w_down", w_down)):
        _need(w, x.dtype, name)
    T, d = x.shape
    P = T * k
    E, f, _ = w_gate.shape
    dev = x.device
    if out is None:
        mk = lambda *s: torch.empty(s, dtype=x.dtype, device=dev)
        out = (mk(P, f), mk(P, d), mk(P, f) if save_gu else None, mk(P, f) if save_gu else None)
    act, yp, g, u = out
    code = _dtype_code(x)
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_fwd_gather_workspace_bytes, (code, P, d, f, E), ws, dev)
    _check(lib.moe_grouped_gemm_swiglu_fwd_gather(_ptr(x), T, k, _ptr(pair_of_row), _ptr(topk_w), _ptr(w_gate), _ptr(w_up), _ptr(w_down),
                                                  code, P, d, f, E, _ptr(offsets), _ptr(g), _ptr(u), _ptr(act), _ptr(yp),
                                                  _ptr(ws), nbytes, _stream()))
    return act, yp, g, u


def moe_mx8_quantise(src, out=None):
    """bf16 [..., K] -> (E4M3 codes uint8 [..., K], packed scale words int32 [K/128, rows]) with rows = the product of the
    leading dimensions; byte j of word (g, row) is the power-of-two scale code of elements 128 g + 32 j .. + 31 of the row."""
    _need(src, torch.bfloat16, "src")
    K = src.shape[-1]
    rows = src.numel() // K if K else 0
    if out is None:
        out = (torch.empty(src.shape, dtype=torch.uint8, device=src.device),
               torch.empty((max(K // 128, 0), rows), dtype=torch.int32, device=src.device))
    codes, scales = out
    _check(lib.moe_mx8_quantise(_ptr(src), rows, K, _ptr(codes), _ptr(scales), _stream()))
    return codes, scales


def moe_grouped_gemm_swiglu_fwd_mx8(xq, xs, wgq, wgs, wuq, wus, wdq, wds, offsets, pair_of_row=None, k=1, out=None, ws=None):
    """Expert forward with 8-bit block-scaled operands (from moe_mx8_quantise).  xq [T, d] codes read by token through
    pair_of_row [P] (P = T * k), or [P, d] in expert order when pair_of_row is None.
    -> act codes uint8 [P, f], act scale words int32 [f/128, P], yp bf16 [P, d]."""
    _need(xq, torch.uint8, "xq"); _need(xs, torch.int32, "xs"); _need(offsets, torch.int32, "offsets")
    for name, w in (("wgq", wgq), ("wuq", wuq), ("wdq", wdq)):
        _need(w, torch.uint8, name)
    for name, w in (("wgs", wgs), ("wus", wus), ("wds", wds)):
        _need(w, torch.int32, name)
    T, d = xq.shape
    E, f, _ = wgq.shape
    if pair_of_row is not None:
        _need(pair_of_row, torch.int32, "pair_of_row")
        P = T * k
    else:
        P, k = T, 1
    dev = xq.device
    if out is None:
        out = (torch.empty((P, f), dtype=torch.uint8, device=dev), torch.empty((max(f // 128, 0), P), dtype=torch.int32, device=dev),
               torch.empty((P, d), dtype=torch.bfloat16, device=dev))
    actq, acts, yp = out
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_fwd_mx8_workspace_bytes, (P, d, f, E), ws, dev)
    _check(lib.moe_grouped_gemm_swiglu_fwd_mx8(_ptr(xq), _ptr(xs), T, k, _ptr(pair_of_row), _ptr(wgq), _ptr(wgs), _ptr(wuq), _ptr(wus),
                                               _ptr(wdq), _ptr(wds), P, d, f, E, _ptr(offsets), _ptr(actq), _ptr(acts), _ptr(yp),
                                               _ptr(ws), nbytes, _stream()))
    return actq, acts, yp


def moe_grouped_gemm_down_mx8(actq, acts, wdq, wds, offsets, out=None, ws=None):
    """The second product alone on given activation codes [P, f] and scale words [f/128, P].  -> yp bf16 [P, d]."""
    _need(actq, torch.uint8, "actq"); _need(acts, torch.int32, "acts"); _need(wdq, torch.uint8, "wdq"); _need(wds, torch.int32, "wds")
    _need(offsets, torch.int32, "offsets")
    P, f = actq.shape
    E, d, _ = wdq.shape
    yp = out if out is not None else torch.empty((P, d), dtype=torch.bfloat16, device=actq.device)
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_fwd_mx8_workspace_bytes, (P, d, f, E), ws, actq.device)
    _check(lib.moe_grouped_gemm_down_mx8(_ptr(actq), _ptr(acts), _ptr(wdq), _ptr(wds), P, d, f, E, _ptr(offsets), _ptr(yp),
                                         _ptr(ws), nbytes, _stream()))
    return yp


def moe_grouped_gemm_swiglu_bwd_gather(dy, x, topk_w, pair_of_row, g_save, u_save, w_gate, w_up, w_down, offsets,
                                       out=None, ws=None, act_w=None):
    """Combine backward and FFN backward without dyp / xp.
    -> dxp [P,d], dw_gate [E,f,d], dw_up [E,f,d], dw_down [E,d,f], dtopk_w [T,k] f32.
    act_w [P,f]: the weighted activation the forward wrote when it was given topk_w (None: formed here)."""
    if act_w is not None:
        _need(act_w, x.dtype, "act_w")
    _need(dy, x.dtype, "dy"); _need(x, None, "x"); _need(topk_w, torch.float32, "topk_w")
    _need(pair_of_row, torch.int32, "pair_of_row"); _need(offsets, torch.int32, "offsets")
    T, d = x.shape
    k = topk_w.shape[1]
    P = T * k
    E, f, _ = w_gate.shape
    if out is None:
        out = (torch.empty((P, d), dtype=x.dtype, device=x.device), torch.empty_like(w_gate), torch.empty_like(w_up),
               torch.empty_like(w_down), torch.empty((T, k), dtype=torch.float32, device=x.device))
    dxp, dwg, dwu, dwd, dtw = out
    code = _dtype_code(x)
    have_saved = int(g_save is not None)
    ws, nbytes = _ws(lib.moe_grouped_gemm_swiglu_bwd_gather_workspace_bytes, (code, P, d, f, E, have_saved), ws, x.device)
    _check(lib.moe_grouped_gemm_swiglu_bwd_gather(_ptr(dy), _ptr(x), T, k, _ptr(topk_w), _ptr(pair_of_row), _ptr(g_save),
                                                  _ptr(u_save), _ptr(act_w), _ptr(w_gate), _ptr(w_up), _ptr(w_down), code, P, d, f, E,
                                                  _ptr(offsets), _ptr(dxp), _ptr(dwg), _ptr(dwu), _ptr(dwd), _ptr(dtw),
                                                  _ptr(ws), nbytes, _stream()))
    return dxp, dwg, dwu, dwd, dtw


def moe_unpermute_combine_fwd(yp, topk_w, row_of_pair, T, k, out=None):
    """-> y [T,d]; topk_w None = unit weights (backward of moe_permute)."""
    _need(yp, None, "yp"); _need(row_of_pair, torch.int32, "row_of_pair")
    if topk_w is not None:
        _need(topk_w, torch.float32, "topk_w")
    d = yp.shape[1]
    if out is None:
        out = torch.empty((T, d), dtype=yp.dtype, device=yp.device)
    _check(lib.moe_unpermute_combine_fwd(_ptr(yp), _dtype_code(yp), T, d, k, _ptr(topk_w), _ptr(row_of_pair),
                                         _ptr(out), _stream()))
    return out


def moe_unpermute_combine_bwd(dy, yp, topk_w, row_of_pair, out=None):
    """-> dyp [P,d], dw [T,k] f32."""
    _need(dy, yp.dtype, "dy"); _need(yp, None, "yp"); _need(topk_w, torch.float32, "topk_w")
    T, d = dy.shape
    k = topk_w.shape[1]
    if out is None:
        out = (torch.empty_like(yp), torch.empty((T, k), dtype=torch.float32, device=dy.device))
    dyp, dw = out
    _check(lib.moe_unpermute_combine_bwd(_ptr(dy), _ptr(yp), _dtype_code(yp), T, d, k, _ptr(topk_w), _ptr(row_of_pair),
                                         _ptr(dyp), _ptr(dw), _stream()))
    return dyp, dw


def moe_router_logits(x, w_router, out=None, ws=None):
    """-> logits [T,E] f32 = x [T,d] @ w_router [E,d]^T."""
    _need(x, None, "x"); _need(w_router, x.dtype, "w_router")
    T, d = x.shape
    E = w_router.shape[0]
    dt = _dtype_code(x)
    if out is None:
        out = torch.empty((T, E), dtype=torch.float32, device=x.device)
    ws, n = _ws(lib.moe_router_logits_workspace_bytes, (dt, T, d, E), ws, x.device)
    _check(lib.moe_router_logits(_ptr(x), _ptr(w_router), dt, T, d, E, _ptr(out), _ptr(ws), n, _stream()))
    return out


def moe_router_bwd(dlogits, x, w_router, dx=None, out_dw=None, ws=None):
    """-> dx [T,d] (dx given: the router term is added to it in place), dw_router [E,d]."""
    _need(dlogits, torch.float32, "dlogits"); _need(x, None, "x"); _need(w_router, x.dtype, "w_router")
    T, d = x.shape
    E = w_router.shape[0]
    dt = _dtype_code(x)
    accumulate = dx is not None
    if dx is None:
        dx = torch.empty_like(x)
    else:
        _need(dx, x.dtype, "dx")
    if out_dw is None:
        out_dw = torch.empty_like(w_router)
    ws, n = _ws(lib.moe_router_bwd_workspace_bytes, (dt, T, d, E), ws, x.device)
    _check(lib.moe_router_bwd(_ptr(dlogits), _ptr(x), _ptr(w_router), dt, T, d, E, int(accumulate), _ptr(dx), _ptr(out_dw),
                              _ptr(ws), n, _stream()))
    return dx, out_dw


# ---- rotary positions, the paged key/value cache, attention of one token over it -----------------------------------

def _heads(t, dtype, name, shape=None):
    """A [T, heads, dim] device tensor whose heads are contiguous: its pointer and the strides of tokens and heads."""
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    st = t.stride()
    if len(st) != 3 or not t.is_cuda:
        raise ValueError("%s must be a [tokens, heads, dim] device tensor" % name)
    if st[2] != 1 and t.shape[2] != 1:
        raise ValueError("%s: the elements of a head must be contiguous" % name)
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    return t.data_ptr(), st[0] if t.shape[0] > 1 else 0, st[1] if t.shape[1] > 1 else 0   # the stride of one token or one head is never taken


_NO_HEADS = (None, 0, 0)


def _table(cos, sin, positions, T):
    """The pointers of positions and a rotation's table, its n_pos and rot; cos None: no rotation."""
    if cos is None:
        return None, None, None, 0, 0
    n = cos.stride()
    shape = cos.shape
    if not (len(n) == 2 and n[1] == 1 and n[0] == shape[1] and sin.stride() == n and sin.shape == shape and positions.numel() == T):
        raise ValueError("cos and sin must be [n_pos, rot / 2], contiguous, and positions [%d], got %s, %s and %s"
                         % (T, tuple(shape), tuple(sin.shape), tuple(positions.shape)))
    if cos.dtype is not torch.float32 or sin.dtype is not torch.float32 or positions.dtype is not torch.int32:
        raise TypeError("cos and sin must be float32 and positions int32, got %s, %s and %s" % (cos.dtype, sin.dtype, positions.dtype))
    if not (cos.is_cuda and sin.is_cuda and positions.is_cuda and positions.is_contiguous()):
        raise ValueError("cos, sin and positions must be contiguous device tensors")
    return positions.data_ptr(), cos.data_ptr(), sin.data_ptr(), shape[0], 2 * shape[1]


def moe_rope_table(freq, n_pos, amplitude=1.0, out=None):
    """freq [half] f64 -> cos, sin [n_pos, half] f32 of the angles p * freq[i], times amplitude."""
    _need(freq, torch.float64, "freq")
    if out is None:
        out = tuple(torch.empty((n_pos, freq.numel()), dtype=torch.float32, device=freq.device) for _ in range(2))
    cos, sin = out
    _need(cos, torch.float32, "cos"); _need(sin, torch.float32, "sin")
    if cos.shape != (n_pos, freq.numel()) or sin.shape != cos.shape:
        raise ValueError("out must be two tensors [%d, %d]" % (n_pos, freq.numel()))
    _check(lib.moe_rope_table(_ptr(freq), n_pos, freq.numel(), amplitude, _ptr(cos), _ptr(sin), _stream()))
    return cos, sin


def _rope(back, q, k, positions, cos, sin, interleaved, out):
    if out is None:
        out = tuple(None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
    if _marshal is not None:
        _check(_marshal.rope(back, q, k, positions, cos, sin, interleaved, out[0], out[1], _stream()))
        return out
    some = q if q is not None else k
    dtype, (T, _, D) = some.dtype, some.shape
    qi = qo = ki = ko = _NO_HEADS
    Hq = Hk = 0
    if q is not None:
        shape = q.shape
        Hq = shape[1]
        qi, qo = _heads(q, dtype, "q"), _heads(out[0], dtype, "q out", shape)
    if k is not None:
        shape = k.shape
        Hk = shape[1]
        if shape[0] != T or shape[2] != D:
            raise ValueError("q and k must have the same tokens and head size")
        ki, ko = _heads(k, dtype, "k"), _heads(out[1], dtype, "k out", shape)
    p_pos, p_cos, p_sin, n_pos, rot = _table(cos, sin, positions, T)
    call = lib.moe_rope_bwd if back else lib.moe_rope_fwd
    _check(call(*qi, *ki, _dtype_code(some), T, Hq, Hk, D, rot, p_pos, p_cos, p_sin, n_pos, interleaved, *qo, *ko, _stream()))
    return out


def moe_rope_fwd(q, k, positions, cos, sin, interleaved=False, out=None):
    """q [T, Hq, D], k [T, Hk, D] (either may be None) rotated by positions [T] i32 with the table cos, sin [n_pos, rot / 2] f32.
    -> q_out, k_out; out = (q, k) rotates in place."""
    return _rope(False, q, k, positions, cos, sin, interleaved, out)


def moe_rope_bwd(dq, dk, positions, cos, sin, interleaved=False, out=None):
    """Gradients of moe_rope_fwd's inputs from those of its outputs."""
    return _rope(True, dq, dk, positions, cos, sin, interleaved, out)


class KVCacheView:
    """A paged cache as the calls below take it: the tensors it lies in and their descriptor, made once."""

    def __init__(self, k, v, k_scales=None, v_scales=None):
        if k.dtype is torch.uint8:
            code, self.dtype = MOE_MX8, torch.bfloat16
        else:
            code, self.dtype = _dtype_code(k), k.dtype
        pages, heads, page_size, dim = k.shape
        for name, t, row in (("k", k, dim), ("v", v, dim)) + ((("k_scales", k_scales, dim // 32), ("v_scales", v_scales, dim // 32)) if code == MOE_MX8 else ()):
            if t is None or not t.is_cuda or t.dtype is not (torch.uint8 if name.endswith("scales") else k.dtype):
                raise ValueError("%s must be a device tensor, uint8 for scales and the type of k otherwise" % name)
            if t.shape != (pages, heads, page_size, row) or t.stride()[1:] != (page_size * row, row, 1):
                raise ValueError("%s must be [pages, heads, page_size, %d] = %s, dense within a page" % (name, row, (pages, heads, page_size, row)))
        if v.stride(0) != k.stride(0) or (code == MOE_MX8 and v_scales.stride(0) != k_scales.stride(0)):
            raise ValueError("keys and values must have the same stride between pages")
        if code != MOE_MX8 and (k_scales is not None or v_scales is not None):
            raise ValueError("scales belong to a cache of 8-bit codes")
        self.k, self.v, self.k_scales, self.v_scales = k, v, k_scales, v_scales
        self.heads, self.dim, self.page_size, self.scale = heads, dim, page_size, dim ** -0.5
        self.desc = moe_kv_cache_t(code, pages, heads, page_size, dim, 0, _ptr(k), _ptr(v), _ptr(k_scales), _ptr(v_scales), k.stride(0),
                                   k_scales.stride(0) if code == MOE_MX8 else 0)
        self._ref = ctypes.addressof(self.desc)
        self._at = tuple((name, getattr(self, name).data_ptr()) for name in ("k", "v", "k_scales", "v_scales")[:4 if code == MOE_MX8 else 2])

    @property
    def ref(self):
        """The descriptor's address, for a call.  It holds the tensors' addresses: one whose storage has been swapped, resized or freed since may
        not be reached through it any more."""
        for name, at in self._at:
            if getattr(self, name).data_ptr() != at:
                raise ValueError("%s of the cache has moved since its view was made" % name)
        return self._ref


def moe_kv_cache(k, v, k_scales=None, v_scales=None):
    """k, v [pages, heads, page_size, dim] f32, bf16, or uint8 codes with scales uint8 [pages, heads, page_size, dim / 32].
    -> the view of them that moe_kv_cache_write, moe_kv_cache_read and moe_paged_attn_decode take (it keeps the tensors, which stay where they are)."""
    return KVCacheView(k, v, k_scales, v_scales)


def moe_kv_cache_write(cache, k, v, slots, q=None, positions=None, cos=None, sin=None, interleaved=False, q_out=None):
    """k, v [T, heads, dim] into the cache at slots [T] i64, the keys rotated if a table is given; q [T, Hq, dim] rotated into q_out.
    -> q_out (None without q)."""
    ref = cache.ref
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=cache.dtype, device=q.device)
    if _marshal is not None:
        _check(_marshal.kv_cache_write(ref, k, v, slots, q, positions, cos, sin, interleaved, q_out, _stream()))
        return q_out
    T, dt = k.shape[0], cache.dtype
    shape = (T, cache.heads, cache.dim)
    ki, vi = _heads(k, dt, "k", shape), _heads(v, dt, "v", shape)
    _need(slots, torch.int64, "slots")
    if slots.numel() != T:
        raise ValueError("slots must be [%d]" % T)
    qi = qo = _NO_HEADS
    Hq = 0
    if q is not None:
        Hq = q.shape[1]
        qi, qo = _heads(q, dt, "q", (T, Hq, cache.dim)), _heads(q_out, dt, "q_out", q.shape)
    p_pos, p_cos, p_sin, n_pos, rot = _table(cos, sin, positions, T)
    _check(lib.moe_kv_cache_write(ref, *ki, *vi, T, slots.data_ptr(), *qi, Hq, rot, p_pos, p_cos, p_sin, n_pos, interleaved, *qo, _stream()))
    return q_out


def moe_kv_cache_read(cache, pages, row_start, rows=None, first=None, out=None):
    """Tokens first[b] .. of every sequence b (first None: from its first on) into the rows row_start[b] .. row_start[b + 1] - 1.
    pages [B, max_pages] i32, row_start [B + 1] i32, first [B] i32; rows: row_start[B], needed without out.
    -> k, v [rows, heads, dim] in the cache's type (bf16 for 8-bit codes)."""
    ref = cache.ref
    if out is None:
        if rows is None:
            raise ValueError("rows (the last of row_start, on the host) or out must be given")
        out = tuple(torch.empty((rows, cache.heads, cache.dim), dtype=cache.dtype, device=pages.device) for _ in range(2))
    k, v = out
    if _marshal is not None:
        _check(_marshal.kv_cache_read(ref, pages, row_start, first, k, v, _stream()))
        return out
    _need(pages, torch.int32, "pages"); _need(row_start, torch.int32, "row_start")
    if pages.dim() != 2 or row_start.numel() != pages.shape[0] + 1:
        raise ValueError("pages must be [sequences, max_pages] and row_start have one entry more than there are sequences")
    B, max_pages = pages.shape
    if first is not None:
        _need(first, torch.int32, "first")
        if first.numel() != B:
            raise ValueError("first must be [%d]" % B)
    _need(k, cache.dtype, "k out"); _need(v, cache.dtype, "v out")
    if k.dim() != 3 or k.shape[1:] != (cache.heads, cache.dim) or v.shape != k.shape:
        raise ValueError("out must be two tensors [rows, %d, %d]" % (cache.heads, cache.dim))
    _check(lib.moe_kv_cache_read(ref, pages.data_ptr(), max_pages, row_start.data_ptr(), _ptr(first), B, k.shape[0], k.data_ptr(), v.data_ptr(),
                                 _stream()))
    return out


def moe_paged_attn_decode(q, cache, pages, lens, scale=None, window=0, out=None, lse=None, ws=None):
    """Attention of one token per sequence: q [B, Hq, dim] over the first lens[b] tokens of the pages pages[b, :] (the last `window` of them
    where it is not 0).  scale None: dim ** -0.5.  -> out [B, Hq, dim], lse [B, Hq] f32 (None where lse is not given; True makes one)."""
    ref = cache.ref
    if scale is None:
        scale = cache.scale
    if out is None:
        out = torch.empty(q.shape, dtype=cache.dtype, device=q.device)
    if lse is True:
        lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    if ws is None:
        B, Hq, _ = q.shape
        ws, _ = _ws(lib.moe_paged_attn_decode_workspace_bytes, (B, Hq, cache.heads, cache.dim, cache.page_size, pages.shape[1]), None, q.device)
    if _marshal is not None:
        _check(_marshal.paged_attn_decode(ref, q, pages, lens, scale, window, out, lse, ws, _stream()))
        return out, lse
    dt = cache.dtype
    B, Hq, _ = q.shape
    qi = _heads(q, dt, "q", (B, Hq, cache.dim))
    _need(pages, torch.int32, "pages"); _need(lens, torch.int32, "lens")
    if pages.dim() != 2 or pages.shape[0] != B or lens.numel() != B:
        raise ValueError("pages must be [%d, max_pages] and lens [%d]" % (B, B))
    if _need(out, dt, "out").shape != q.shape:
        raise ValueError("out must have the shape of q")
    if lse is not None and _need(lse, torch.float32, "lse").shape != (B, Hq):
        raise ValueError("lse must be [%d, %d]" % (B, Hq))
    if window != ctypes.c_int32(window).value:
        raise OverflowError("window does not fit 32 bits")
    _check(lib.moe_paged_attn_decode(*qi, ref, pages.data_ptr(), pages.shape[1], lens.data_ptr(), B, Hq, scale, window, out.data_ptr(), _ptr(lse),
                                     ws.data_ptr(), ws.numel() * ws.element_size(), _stream()))
    return out, lse
