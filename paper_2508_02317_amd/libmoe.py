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
    "moe_rope_axes_fwd", "moe_rope_axes_bwd", "moe_kv_cache_write_axes",
    "moe_norm_fwd", "moe_norm_bwd_workspace_bytes", "moe_norm_bwd",
    "moe_balance_loss_fwd_workspace_bytes", "moe_balance_loss_fwd", "moe_balance_loss_bwd",
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
    for turn in (lib.moe_rope_axes_fwd, lib.moe_rope_axes_bwd):
        turn.restype = ctypes.c_int32
        turn.argtypes = [vp, i64, i64] * 2 + [i32] * 6 + [vp, i32, vp] + [vp] * 2 + [i32] * 2 + [vp, i64, i64] * 2 + [vp]
    lib.moe_kv_cache_write_axes.restype = ctypes.c_int32
    lib.moe_kv_cache_write_axes.argtypes = ([vp] + [vp, i64, i64] * 2 + [i32, vp] + [vp, i64, i64] + [i32] * 2 + [vp, i32, vp] + [vp] * 2 + [i32] * 2 +
                                            [vp, i64, i64, vp])
    lib.moe_norm_fwd.restype = ctypes.c_int32
    lib.moe_norm_fwd.argtypes = [vp, i64, i64] * 2 + [i32] * 5 + [vp, vp, i32, f32] + [vp, i64, i64] * 2 + [vp] * 3
    lib.moe_norm_bwd_workspace_bytes.restype = sz
    lib.moe_norm_bwd_workspace_bytes.argtypes = [i32] * 3
    lib.moe_norm_bwd.restype = ctypes.c_int32
    lib.moe_norm_bwd.argtypes = [vp, i64, i64] * 2 + [i32] * 4 + [vp] * 3 + [i32] + [vp, i64, i64] * 2 + [vp] * 3 + [sz, vp]
    lib.moe_balance_loss_fwd_workspace_bytes.restype = sz
    lib.moe_balance_loss_fwd_workspace_bytes.argtypes = [i32] * 3
    lib.moe_balance_loss_fwd.restype = ctypes.c_int32
    lib.moe_balance_loss_fwd.argtypes = [vp] * 3 + [i32] * 3 + [vp] * 5 + [sz, vp]
    lib.moe_balance_loss_bwd.restype = ctypes.c_int32
    lib.moe_balance_loss_bwd.argtypes = [vp] * 4 + [i32] * 3 + [f32] * 2 + [vp] * 4
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


# ---- positions with several axes, the norm, the router's losses ------------------------------------------------------
# These refuse tensors that are not on the current device, whose stream the call goes to.

if _raw_stream is not None:
    _device_now = getattr(torch._C, "_cuda_getDevice", _current_device)   # torch.cuda.current_device() looks first whether torch has a device at all, 0.2 us

    def _where():
        """The current stream of the current device, and the device."""
        device = _device_now()
        return _raw_stream(device), device
else:
    def _where():
        return _stream(), _current_device()


def _on(t, name):
    if not t.is_cuda:
        raise ValueError("%s must be a device tensor" % name)
    if t.get_device() != _current_device():
        raise ValueError("%s is not on the current device" % name)
    return t


def _flat(t, dtype, n, name):
    """The pointer of a contiguous tensor of n elements on the current device (None: null)."""
    if t is None:
        return None
    _need(_on(t, name), dtype, name)
    if n is not None and t.numel() != n:
        raise ValueError("%s must have %d elements" % (name, n))
    return t.data_ptr()


def _axes(positions, cos, sin, pair_axis, T):
    if not isinstance(pair_axis, bytes):
        raise TypeError("pair_axis must be bytes, the axis of every pair")
    if positions is None or cos is None or sin is None:
        raise ValueError("positions, cos and sin must be given")
    at = _flat(positions, torch.int32, None, "positions"), _flat(cos, torch.float32, None, "cos"), _flat(sin, torch.float32, None, "sin")
    if cos.dim() != 2 or sin.shape != cos.shape or positions.dim() != 2 or positions.shape[1] != T:
        raise ValueError("cos and sin must be [n_pos, rot / 2] and positions [axes, %d]" % T)
    if len(pair_axis) != cos.shape[1]:
        raise ValueError("pair_axis must have one entry per pair")
    return at[0], positions.shape[0], pair_axis, at[1], at[2], cos.shape[0], 2 * cos.shape[1]


def _rope_axes(back, q, k, positions, cos, sin, pair_axis, interleaved, out):
    if out is None:
        out = tuple(None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k))
    if _marshal is not None:
        _check(_marshal.rope_axes(back, q, k, positions, cos, sin, pair_axis, interleaved, out[0], out[1], *_where()))
        return out
    some = q if q is not None else k
    if some is None:
        raise ValueError("q or k must be given")
    code, (T, _, D) = _dtype_code(some), some.shape
    qi = qo = ki = ko = _NO_HEADS
    Hq = Hk = 0
    if q is not None:
        Hq = q.shape[1]
        qi, qo = _heads(_on(q, "q"), some.dtype, "q"), _heads(_on(out[0], "q out"), some.dtype, "q out", q.shape)
    if k is not None:
        Hk = k.shape[1]
        ki, ko = _heads(_on(k, "k"), some.dtype, "k", (T, Hk, D)), _heads(_on(out[1], "k out"), some.dtype, "k out", k.shape)
    p_pos, n_axes, pairs, p_cos, p_sin, n_pos, rot = _axes(positions, cos, sin, pair_axis, T)
    call = lib.moe_rope_axes_bwd if back else lib.moe_rope_axes_fwd
    _check(call(*qi, *ki, code, T, Hq, Hk, D, rot, p_pos, n_axes, pairs, p_cos, p_sin, n_pos, interleaved, *qo, *ko, _stream()))
    return out


def moe_rope_axes_fwd(q, k, positions, cos, sin, pair_axis, interleaved=False, out=None):
    """moe_rope_fwd with positions [axes, T] i32 of up to four axes; pair_axis: bytes, the axis of each of the rot / 2 pairs (generation.rope_axes).
    -> q_out, k_out; out = (q, k) rotates in place."""
    return _rope_axes(False, q, k, positions, cos, sin, pair_axis, interleaved, out)


def moe_rope_axes_bwd(dq, dk, positions, cos, sin, pair_axis, interleaved=False, out=None):
    """Gradients of moe_rope_axes_fwd's inputs from those of its outputs."""
    return _rope_axes(True, dq, dk, positions, cos, sin, pair_axis, interleaved, out)


def moe_kv_cache_write_axes(cache, k, v, slots, q, positions, cos, sin, pair_axis, interleaved=False, q_out=None):
    """moe_kv_cache_write with positions [axes, T] i32 and pair_axis as in moe_rope_axes_fwd; q may be None.  -> q_out (None without q)."""
    ref = cache.ref
    if q is not None and q_out is None:
        q_out = torch.empty(q.shape, dtype=cache.dtype, device=q.device)
    if _marshal is not None:
        _check(_marshal.kv_cache_write_axes(ref, cache.k.get_device(), k, v, slots, q, positions, cos, sin, pair_axis, interleaved, q_out, *_where()))
        return q_out
    _on(cache.k, "cache")
    T, dt = k.shape[0], cache.dtype
    shape = (T, cache.heads, cache.dim)
    ki, vi = _heads(_on(k, "k"), dt, "k", shape), _heads(_on(v, "v"), dt, "v", shape)
    p_slots = _flat(slots, torch.int64, T, "slots")
    qi = qo = _NO_HEADS
    Hq = 0
    if q is not None:
        Hq = q.shape[1]
        qi, qo = _heads(_on(q, "q"), dt, "q", (T, Hq, cache.dim)), _heads(_on(q_out, "q_out"), dt, "q_out", q.shape)
    p_pos, n_axes, pairs, p_cos, p_sin, n_pos, rot = _axes(positions, cos, sin, pair_axis, T)
    _check(lib.moe_kv_cache_write_axes(ref, *ki, *vi, T, p_slots, *qi, Hq, rot, p_pos, n_axes, pairs, p_cos, p_sin, n_pos, interleaved, *qo, _stream()))
    return q_out


def _rows(t, like, name):
    """[tokens, dim] or [tokens, heads, dim] whose rows are contiguous: pointer, strides of tokens and heads (None: null)."""
    if t is None:
        return _NO_HEADS
    _on(t, name)
    if t.dim() not in (2, 3):
        raise ValueError("%s must be [tokens, dim] or [tokens, heads, dim]" % name)
    st = t.stride()
    if st[-1] != 1 and t.shape[-1] != 1:
        raise ValueError("%s: the elements of a row must be contiguous" % name)
    if t.dtype is not like.dtype:
        raise TypeError("%s has another element type" % name)
    if t.shape != like.shape:
        raise ValueError("%s has another shape" % name)
    return t.data_ptr(), st[0] if t.shape[0] > 1 else 0, st[1] if t.dim() == 3 and t.shape[1] > 1 else 0


def _vectors(D, **named):
    """The pointers of weights [D] of one type, and its code."""
    code, out = None, []
    for name, t in named.items():
        if t is not None:
            _on(t, name)
            c = _dtype_code(t)
            if code is not None and c != code:
                raise TypeError("%s has another type than the other weights" % name)
            if t.shape != (D,) or not t.is_contiguous():
                raise ValueError("%s must be contiguous, one number per column" % name)
            code = c
        out.append(_ptr(t))
    return out, MOE_F32 if code is None else code


def moe_norm_fwd(x, weight=None, bias=None, eps=1e-6, rms=False, residual=None, stats=True, out=None):
    """Layer norm (rms: rms norm) of the rows of x [T, D] or [T, heads, D], or of h = x + residual; weight, bias [D] f32 or bf16 (None: 1 and 0).
    -> y, h (None without residual), mean (None with rms), rstd f32 (both None where stats is false); out: the four of them, each as above or, for mean and
    rstd, None."""
    if out is None:
        mk = lambda: torch.empty(x.shape, dtype=x.dtype, device=x.device)
        stat = lambda wanted: torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if wanted and stats else None
        out = mk(), None if residual is None else mk(), stat(not rms), stat(True)
    y, h, mean, rstd = out
    if _marshal is not None:
        _check(_marshal.norm_fwd(x, weight, bias, eps, rms, residual, y, h, mean, rstd, *_where()))
        return out
    if x is None or y is None:
        raise ValueError("x and y must be given")
    xi, ri, yo, so = _rows(x, x, "x"), _rows(residual, x, "residual"), _rows(y, x, "y"), _rows(h, x, "h")
    T, H, D = x.shape[0], x.shape[1] if x.dim() == 3 else 1, x.shape[-1]
    (p_w, p_b), code = _vectors(D, weight=weight, bias=bias)
    _check(lib.moe_norm_fwd(*xi, *ri, _dtype_code(x), T, H, D, rms, p_w, p_b, code, eps, *so, *yo, _flat(mean, torch.float32, T * H, "mean"),
                            _flat(rstd, torch.float32, T * H, "rstd"), _stream()))
    return out


def moe_norm_bwd(dy, x, rstd, mean=None, weight=None, add=None, with_weight=True, with_bias=False, out=None, ws=None):
    """Gradients of moe_norm_fwd: dy and x (what was normed) like its x, rstd and mean as it gave them (mean None: rms norm), add: a gradient of x from elsewhere.
    -> dx, dweight, dbias [D] in the type of weight (f32 without one; None unless wanted); out: the three of them."""
    if out is None:
        kind = torch.float32 if weight is None else weight.dtype
        vec = lambda wanted: torch.empty(x.shape[-1], dtype=kind, device=x.device) if wanted else None
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device), vec(with_weight), vec(with_bias)
    dx, dweight, dbias = out
    T, H, D = x.shape[0], x.shape[1] if x.dim() == 3 else 1, x.shape[-1]
    if ws is None and (dweight is not None or dbias is not None):
        ws, _ = _ws(lib.moe_norm_bwd_workspace_bytes, (T, H, D), None, x.device)
    if _marshal is not None:
        _check(_marshal.norm_bwd(dy, x, rstd, mean, weight, add, dx, dweight, dbias, ws, *_where()))
        return out
    if dy is None or dx is None or rstd is None:
        raise ValueError("dy, rstd and dx must be given")
    di, xi, ai, do = _rows(dy, x, "dy"), _rows(x, x, "x"), _rows(add, x, "add"), _rows(dx, x, "dx")
    (p_w, p_dw, p_db), code = _vectors(D, weight=weight, dweight=dweight, dbias=dbias)
    _check(lib.moe_norm_bwd(*di, *xi, _dtype_code(x), T, H, D, _flat(mean, torch.float32, T * H, "mean"), _flat(rstd, torch.float32, T * H, "rstd"), p_w, code, *ai, *do,
                            p_dw, p_db, _flat(ws, None, None, "ws"), 0 if ws is None else ws.numel() * ws.element_size(), _stream()))
    return out


def _logits(t):
    if t is None or t.dim() != 2:
        raise ValueError("logits must be [tokens, experts]")
    return _flat(t, torch.float32, None, "logits")


def _mask(t, n):
    if t is None:
        return None
    if t.dtype not in (torch.bool, torch.uint8):
        raise TypeError("valid must be bool or uint8")
    return _flat(t, None, n, "valid")


def moe_balance_loss_fwd(logits, topk_idx, valid=None, out=None, ws=None):
    """Balance loss and z loss of a router: logits [T, E] f32, topk_idx [T, k] i32, valid [T] bool or uint8 (None: all tokens count).
    -> losses [2] f32, counts [E + 1] i32 (the last one the number of valid tokens), importance [E] f32 (mean probabilities), lse [T] f32."""
    T, E = logits.shape
    if out is None:
        mk = lambda n, t: torch.empty(n, dtype=t, device=logits.device)
        out = mk(2, torch.float32), mk(E + 1, torch.int32), mk(E, torch.float32), mk(T, torch.float32)
    losses, counts, importance, lse = out
    k = topk_idx.shape[-1]
    if ws is None:
        ws, _ = _ws(lib.moe_balance_loss_fwd_workspace_bytes, (T, E, k), None, logits.device)
    if _marshal is not None:
        _check(_marshal.balance_loss_fwd(logits, topk_idx, valid, losses, counts, importance, lse, ws, *_where()))
        return out
    p_logits, p_idx = _logits(logits), _flat(topk_idx, torch.int32, None, "topk_idx")
    if topk_idx.dim() != 2 or topk_idx.shape[0] != T:
        raise ValueError("topk_idx must be [tokens, k]")
    if losses is None or counts is None or importance is None or lse is None:
        raise ValueError("losses, counts, importance and lse must be given")
    _check(lib.moe_balance_loss_fwd(p_logits, p_idx, _mask(valid, T), T, E, k, _flat(losses, torch.float32, 2, "losses"), _flat(counts, torch.int32, E + 1, "counts"),
                                    _flat(importance, torch.float32, E, "importance"), _flat(lse, torch.float32, T, "lse"), _flat(ws, None, None, "ws"),
                                    ws.numel() * ws.element_size(), _stream()))
    return out


def moe_balance_loss_bwd(logits, counts, lse, k, balance=1.0, z=0.0, dlosses=None, valid=None, add=None, out=None):
    """Gradient of balance * losses[0] + z * losses[1] (times dlosses [2] f32 on the device, where given) with respect to the logits, counts and lse as
    moe_balance_loss_fwd gave them, plus add [T, E] (which may be out).  -> dlogits [T, E] f32."""
    if out is None:
        out = torch.empty(logits.shape, dtype=torch.float32, device=logits.device)
    if _marshal is not None:
        _check(_marshal.balance_loss_bwd(logits, counts, lse, k, balance, z, dlosses, valid, add, out, *_where()))
        return out
    p_logits = _logits(logits)
    T, E = logits.shape
    if counts is None or lse is None:
        raise ValueError("counts and lse must be given")
    _check(lib.moe_balance_loss_bwd(p_logits, _flat(counts, torch.int32, E + 1, "counts"), _flat(lse, torch.float32, T, "lse"), _mask(valid, T), T, E, k, balance, z,
                                    _flat(dlosses, torch.float32, 2, "dlosses"), _flat(add, torch.float32, T * E, "add"), _flat(out, torch.float32, T * E, "dlogits"),
                                    _stream()))
    return out
