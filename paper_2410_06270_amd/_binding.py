"""ctypes binding of the C-ABI (argument marshalling only).

Functions carry the C names without the ``mc_`` prefix.  Device buffers are
torch tensors on the current CUDA (HIP) device; the library never allocates,
so ``PackedLayer`` and ``Routing`` allocate their buffers with torch and build
the descriptors over them.
"""
from __future__ import annotations

import ctypes
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libmcmoe.so")
_lib = None

MC_OK, MC_EINVAL, MC_ENOSPACE, MC_EHIP, MC_EUNSUPPORTED = range(5)
MAX_EXPERTS = 256
MAX_TOPK = 8


class MCError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("mc status %d: %s" % (status, msg))
        self.status = status


class _Layer(ctypes.Structure):
    _fields_ = [("E", ctypes.c_int), ("d", ctypes.c_int), ("ffn", ctypes.c_int),
                ("group", ctypes.c_int), ("bits_host", ctypes.POINTER(ctypes.c_int)),
                ("words", ctypes.c_void_p), ("sz", ctypes.c_void_p),
                ("words_bytes", ctypes.c_size_t), ("sz_bytes", ctypes.c_size_t)]


class _Routing(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int), ("E", ctypes.c_int), ("k", ctypes.c_int),
                ("topk_idx", ctypes.c_void_p), ("topk_w", ctypes.c_void_p),
                ("kept", ctypes.c_void_p), ("counts", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p), ("pair_token", ctypes.c_void_p),
                ("pair_rank", ctypes.c_void_p), ("pair_w", ctypes.c_void_p),
                ("pair_pos", ctypes.c_void_p), ("n_pruned", ctypes.c_void_p)]


class _KVCache(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int), ("page", ctypes.c_int), ("Hkv", ctypes.c_int), ("D", ctypes.c_int),
                ("dtype", ctypes.c_int), ("k", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("page_stride", ctypes.c_size_t), ("k_bytes", ctypes.c_size_t), ("v_bytes", ctypes.c_size_t),
                ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p)]


class _KVBatch(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int), ("T", ctypes.c_int), ("max_pages", ctypes.c_int), ("max_len", ctypes.c_int),
                ("q_start", ctypes.c_void_p), ("kv_len", ctypes.c_void_p), ("page_table", ctypes.c_void_p)]


class _QKPrep(ctypes.Structure):
    _fields_ = [("q_norm", ctypes.c_void_p), ("k_norm", ctypes.c_void_p), ("norm_row", ctypes.c_int),
                ("eps", ctypes.c_float), ("rot", ctypes.c_int), ("rope_pairs", ctypes.c_int),
                ("rope", ctypes.c_void_p), ("n_pos", ctypes.c_int)]


class _Attention(ctypes.Structure):
    _fields_ = [("Hq", ctypes.c_int), ("scale", ctypes.c_float), ("softcap", ctypes.c_float),
                ("window", ctypes.c_int), ("slopes", ctypes.c_void_p), ("prefix", ctypes.c_void_p)]


class _KVPool(ctypes.Structure):
    _fields_ = [("n_pages", ctypes.c_int), ("page", ctypes.c_int), ("free_list", ctypes.c_void_p),
                ("n_free", ctypes.c_void_p), ("n_free_out", ctypes.c_void_p)]


class _KVTables(ctypes.Structure):
    _fields_ = [("S", ctypes.c_int), ("T", ctypes.c_int), ("max_pages", ctypes.c_int), ("q_start", ctypes.c_void_p),
                ("kv_len", ctypes.c_void_p), ("page_table", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("slots", ctypes.c_void_p)]


class _KVSummary(ctypes.Structure):
    _fields_ = [("bounds", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("bounds_bytes", ctypes.c_size_t),
                ("scale_bytes", ctypes.c_size_t)]


def lib_path() -> str:
    return _LIB_PATH


def load():
    """Load libmcmoe.so; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libmcmoe.so is not built (run __graft_entry__.build())")
        lib = ctypes.CDLL(_LIB_PATH)
        P, I, S = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t
        st = ctypes.c_int
        lib.mc_last_error.restype = ctypes.c_char_p
        lib.mc_last_error.argtypes = []
        lib.mc_pack_sizes.restype = st
        lib.mc_pack_sizes.argtypes = [I, I, I, P, I, ctypes.POINTER(S), ctypes.POINTER(S)]
        lib.mc_pack.restype = st
        lib.mc_pack.argtypes = [P, P, P, ctypes.POINTER(_Layer), P]
        lib.mc_pack_methods.restype = st
        lib.mc_pack_methods.argtypes = [P, P, P, ctypes.POINTER(_Layer), P, P]
        lib.mc_dequant_export.restype = st
        lib.mc_dequant_export.argtypes = [ctypes.POINTER(_Layer), I, I, P, P]
        lib.mc_codes_export.restype = st
        lib.mc_codes_export.argtypes = [ctypes.POINTER(_Layer), I, I, P, P]
        lib.mc_gptq_workspace.restype = st
        lib.mc_gptq_workspace.argtypes = [I, I, ctypes.POINTER(S)]
        lib.mc_gptq_hessian.restype = st
        lib.mc_gptq_hessian.argtypes = [P, I, I, P, I, P]
        lib.mc_gptq_factor.restype = st
        lib.mc_gptq_factor.argtypes = [P, I, ctypes.c_double, P, P, P, S, P]
        lib.mc_gptq_quantize.restype = st
        lib.mc_gptq_quantize.argtypes = [ctypes.POINTER(_Layer), I, I, P, P, P, P, P, S, P]
        lib.mc_router_logits.restype = st
        lib.mc_router_logits.argtypes = [P, P, I, I, I, P, P]
        lib.mc_route_and_prune.restype = st
        lib.mc_route_and_prune.argtypes = [P, P, ctypes.c_float, ctypes.POINTER(_Routing), P]
        lib.mc_forward_workspace.restype = st
        lib.mc_forward_workspace.argtypes = [I, I, I, I, I, ctypes.POINTER(S)]
        lib.mc_moe_forward.restype = st
        lib.mc_moe_forward.argtypes = [P, ctypes.POINTER(_Routing), ctypes.POINTER(_Layer), P, P,
                                       S, P]
        lib.mc_moe_forward_noalloc.restype = st
        lib.mc_moe_forward_noalloc.argtypes = [P, ctypes.POINTER(_Routing), ctypes.POINTER(_Layer), P, P]
        lib.mc_moe_route_forward.restype = st
        lib.mc_moe_route_forward.argtypes = [P, P, P, ctypes.c_float, ctypes.POINTER(_Routing),
                                             ctypes.POINTER(_Layer), P, P, S, P]
        lib.mc_stack_workspace.restype = st
        lib.mc_stack_workspace.argtypes = [I, I, I, I, I, ctypes.POINTER(S)]
        lib.mc_moe_stack_forward.restype = st
        lib.mc_moe_stack_forward.argtypes = [P, I, ctypes.POINTER(_Layer), P, P, ctypes.c_float,
                                             ctypes.POINTER(_Routing), P, P, P, S, P]
        lib.mc_importance_workspace.restype = st
        lib.mc_importance_workspace.argtypes = [I, I, ctypes.POINTER(S)]
        lib.mc_token_importance.restype = st
        lib.mc_token_importance.argtypes = [P, I, I, P, I, ctypes.c_float, P, P, P, S, P]
        lib.mc_odp_threshold.restype = st
        lib.mc_odp_threshold.argtypes = [P, I, I, ctypes.POINTER(ctypes.c_double),
                                         ctypes.POINTER(ctypes.c_double)]
        D = ctypes.c_double
        lib.mc_pmq_significance.restype = st
        lib.mc_pmq_significance.argtypes = [P, I, I, I, P, P]
        lib.mc_pmq_allocate.restype = st
        lib.mc_pmq_allocate.argtypes = [P, P, P, I, D, D, D, I, P, ctypes.POINTER(D)]
        lib.mc_pmq_error_workspace.restype = st
        lib.mc_pmq_error_workspace.argtypes = [I, I, I, I, I, I, ctypes.POINTER(S)]
        lib.mc_pmq_expert_error.restype = st
        lib.mc_pmq_expert_error.argtypes = [P, P, P, I, I, I, I, P, ctypes.POINTER(_Routing), P, P, S, P]
        KC, KB, AT = (ctypes.POINTER(t) for t in (_KVCache, _KVBatch, _Attention))
        lib.mc_kv_page_bytes.restype = st
        lib.mc_kv_page_bytes.argtypes = [I, I, I, I, ctypes.POINTER(S)]
        lib.mc_kv_append.restype = st
        lib.mc_kv_append.argtypes = [P, S, P, S, P, S, I, ctypes.POINTER(_QKPrep), KB, KC, P, S, P]
        lib.mc_attn_workspace.restype = st
        lib.mc_attn_workspace.argtypes = [I, I, I, I, ctypes.POINTER(S)]
        for f in (lib.mc_attn_decode, lib.mc_attn_prefill):
            f.restype = st
            f.argtypes = [P, S, KB, KC, AT, P, S, P, P, S, P]
        lib.mc_attn_importance_workspace.restype = st
        lib.mc_attn_importance_workspace.argtypes = [I, I, ctypes.POINTER(S)]
        lib.mc_attn_importance.restype = st
        lib.mc_attn_importance.argtypes = [P, S, P, KB, KC, AT, P, I, ctypes.c_float, P, P, P, S, P]
        KP, KT, KS = (ctypes.POINTER(t) for t in (_KVPool, _KVTables, _KVSummary))
        lib.mc_kv_read.restype = st
        lib.mc_kv_read.argtypes = [KB, KC, P, S, P, S, P]
        lib.mc_kv_tables_workspace.restype = st
        lib.mc_kv_tables_workspace.argtypes = [I, ctypes.POINTER(S)]
        for f in (lib.mc_kv_reserve, lib.mc_kv_release):
            f.restype = st
            f.argtypes = [P, P, KP, KT, P, S, P]
        lib.mc_kv_summarize.restype = st
        lib.mc_kv_summarize.argtypes = [KB, KC, KS, P]
        lib.mc_attn_select_workspace.restype = st
        lib.mc_attn_select_workspace.argtypes = [I, I, I, ctypes.POINTER(S)]
        lib.mc_attn_select.restype = st
        lib.mc_attn_select.argtypes = [P, S, KB, KC, KS, AT, I, I, I, P, P, P, S, P]
        lib.mc_attn_sparse.restype = st
        lib.mc_attn_sparse.argtypes = [P, S, KB, KC, AT, P, P, I, P, S, P, P, S, P]
        lib.mc_timing_enable.restype = st
        lib.mc_timing_enable.argtypes = [I]
        lib.mc_timing_read.restype = st
        lib.mc_timing_read.argtypes = [ctypes.c_char_p, ctypes.POINTER(ctypes.c_double),
                                       ctypes.POINTER(I)]
        _lib = lib
    return _lib


def _check(status: int):
    if status != MC_OK:
        raise MCError(status, load().mc_last_error().decode())


def _stream(stream=None):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def pack_sizes(E: int, d: int, ffn: int, bits, group: int):
    arr = (ctypes.c_int * len(bits))(*[int(b) for b in bits])
    wb, szb = ctypes.c_size_t(), ctypes.c_size_t()
    _check(load().mc_pack_sizes(E, d, ffn, arr, group, ctypes.byref(wb), ctypes.byref(szb)))
    return wb.value, szb.value


class PackedLayer:
    """Device buffers + descriptor of one packed layer (torch-allocated)."""

    def __init__(self, E: int, d: int, ffn: int, bits, group: int, device=None):
        self.E, self.d, self.ffn, self.group = E, d, ffn, group
        self.bits = [int(b) for b in bits]
        wb, szb = pack_sizes(E, d, ffn, self.bits, group)
        device = device or torch.device("cuda")
        self.words = torch.empty(wb // 4, dtype=torch.int32, device=device)
        self.sz = torch.empty(szb // 4, dtype=torch.int32, device=device)
        self._bits_c = (ctypes.c_int * E)(*self.bits)
        self.desc = _Layer(E, d, ffn, group, self._bits_c, self.words.data_ptr(),
                           self.sz.data_ptr(), wb, szb)

    @property
    def nbytes(self) -> int:
        return self.words.numel() * 4 + self.sz.numel() * 4


class Routing:
    """Device buffers + descriptor of a routing result for T tokens."""

    def __init__(self, T: int, E: int, k: int, device=None):
        device = device or torch.device("cuda")
        self.T, self.E, self.k = T, E, k
        i32 = dict(dtype=torch.int32, device=device)
        self.topk_idx = torch.empty((T, k), **i32)
        self.topk_w = torch.empty((T, k), dtype=torch.float32, device=device)
        self.kept = torch.empty((T, k), dtype=torch.uint8, device=device)
        self.counts = torch.empty(E, **i32)
        self.offsets = torch.empty(E + 1, **i32)
        self.pair_token = torch.full((T * k,), -1, **i32)
        self.pair_rank = torch.full((T * k,), -1, **i32)
        self.pair_w = torch.zeros(T * k, dtype=torch.float32, device=device)
        self.pair_pos = torch.empty((T, k), **i32)
        self.n_pruned = torch.empty(1, **i32)
        self.desc = _Routing(T, E, k, *[t.data_ptr() for t in (
            self.topk_idx, self.topk_w, self.kept, self.counts, self.offsets, self.pair_token,
            self.pair_rank, self.pair_w, self.pair_pos, self.n_pruned)])


QUANT_RTN, QUANT_SIGN = 0, 1


def pack(w_gate, w_up, w_down, layer: PackedLayer, stream=None, methods=None):
    """Quantize and pack; methods (per expert, QUANT_RTN or QUANT_SIGN for
    1-bit sign binarization) defaults to RTN everywhere."""
    for t in (w_gate, w_up, w_down):
        assert t.dtype == torch.float32 and t.is_contiguous() and t.is_cuda
    if methods is None:
        _check(load().mc_pack(_ptr(w_gate), _ptr(w_up), _ptr(w_down), ctypes.byref(layer.desc),
                              _stream(stream)))
    else:
        arr = (ctypes.c_int * layer.E)(*[int(m) for m in methods])
        _check(load().mc_pack_methods(_ptr(w_gate), _ptr(w_up), _ptr(w_down), ctypes.byref(layer.desc),
                                      arr, _stream(stream)))


def dequant_export(layer: PackedLayer, e: int, mat: int, out, stream=None):
    assert out.dtype in (torch.float16, torch.int16) and out.is_contiguous()
    _check(load().mc_dequant_export(ctypes.byref(layer.desc), e, mat, _ptr(out), _stream(stream)))


def codes_export(layer: PackedLayer, e: int, mat: int, out, stream=None):
    assert out.dtype == torch.uint8 and out.is_contiguous()
    _check(load().mc_codes_export(ctypes.byref(layer.desc), e, mat, _ptr(out), _stream(stream)))


def gptq_workspace(R: int, K: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_gptq_workspace(R, K, ctypes.byref(b)))
    return b.value


def gptq_hessian(x, H, accumulate: bool = False, stream=None):
    """x: [N][K] bf16 (or int16 bits); H: [K][K] float64."""
    assert x.is_contiguous() and x.element_size() == 2 and H.is_contiguous() and H.dtype == torch.float64
    N, K = x.shape
    assert tuple(H.shape) == (K, K)
    _check(load().mc_gptq_hessian(_ptr(x), N, K, _ptr(H), int(bool(accumulate)), _stream(stream)))


def gptq_factor(H, U, dead, workspace, damp: float = 0.01, stream=None):
    """H, U: [K][K] float64; dead: [K] uint8."""
    K = H.shape[0]
    assert H.is_contiguous() and U.is_contiguous() and H.dtype == torch.float64 and U.dtype == torch.float64
    assert dead.dtype == torch.uint8 and dead.numel() == K
    _check(load().mc_gptq_factor(_ptr(H), K, float(damp), _ptr(U), _ptr(dead), _ptr(workspace),
                                 workspace.numel() * workspace.element_size(), _stream(stream)))


def gptq_quantize(layer: PackedLayer, e: int, mat: int, W, U, dead, workspace, loss=None, stream=None):
    """W: [R][K] float32 (the fp32 weights of matrix `mat` of expert e)."""
    assert W.is_contiguous() and W.dtype == torch.float32 and U.dtype == torch.float64
    _check(load().mc_gptq_quantize(ctypes.byref(layer.desc), e, mat, _ptr(W), _ptr(U), _ptr(dead), _ptr(loss),
                                   _ptr(workspace), workspace.numel() * workspace.element_size(),
                                   _stream(stream)))


def router_logits(x, w_router, logits, stream=None):
    """x [T][d], w_router [E][d]: bf16 (or int16 bit patterns); logits [T][E] fp32."""
    assert x.is_contiguous() and w_router.is_contiguous() and logits.is_contiguous()
    assert x.element_size() == 2 and w_router.element_size() == 2 and logits.dtype == torch.float32
    T, d = x.shape
    E = w_router.shape[0]
    assert w_router.shape[1] == d and tuple(logits.shape) == (T, E)
    _check(load().mc_router_logits(_ptr(x), _ptr(w_router), T, d, E, _ptr(logits), _stream(stream)))


def route_and_prune(logits, important, threshold: float, routing: Routing, stream=None):
    assert logits.dtype == torch.float32 and logits.is_contiguous()
    if important is not None:
        assert important.dtype == torch.uint8 and important.is_contiguous()
    _check(load().mc_route_and_prune(_ptr(logits), _ptr(important), float(threshold),
                                     ctypes.byref(routing.desc), _stream(stream)))


def forward_workspace(T: int, E: int, k: int, d: int, ffn: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_forward_workspace(T, E, k, d, ffn, ctypes.byref(b)))
    return b.value


def moe_forward(x, routing: Routing, layer: PackedLayer, y, workspace, stream=None):
    """x, y: bf16 (or int16 bit patterns) [T][d] device tensors."""
    assert x.is_contiguous() and y.is_contiguous() and x.element_size() == 2
    _check(load().mc_moe_forward(_ptr(x), ctypes.byref(routing.desc), ctypes.byref(layer.desc),
                                 _ptr(y), _ptr(workspace), workspace.numel() * workspace.element_size(),
                                 _stream(stream)))


def moe_forward_noalloc(x, routing: Routing, layer: PackedLayer, y, stream=None):
    """moe_forward with the library's own device workspace (no allocation)."""
    assert x.is_contiguous() and y.is_contiguous() and x.element_size() == 2
    _check(load().mc_moe_forward_noalloc(_ptr(x), ctypes.byref(routing.desc), ctypes.byref(layer.desc),
                                         _ptr(y), _stream(stream)))


def route_forward(x, logits, important, threshold: float, routing: Routing, layer: PackedLayer, y, workspace,
                  stream=None):
    """route_and_prune + moe_forward in one call (same results)."""
    assert x.is_contiguous() and y.is_contiguous() and x.element_size() == 2
    assert logits.dtype == torch.float32 and logits.is_contiguous()
    if important is not None:
        assert important.dtype == torch.uint8 and important.is_contiguous()
    _check(load().mc_moe_route_forward(_ptr(x), _ptr(logits), _ptr(important), float(threshold),
                                       ctypes.byref(routing.desc), ctypes.byref(layer.desc), _ptr(y),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream)))


def stack_workspace(T: int, E: int, k: int, d: int, ffn: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_stack_workspace(T, E, k, d, ffn, ctypes.byref(b)))
    return b.value


def stack_forward(x, layers, logits, important, threshold: float, routing: Routing, y, tmp,
                  workspace, stream=None):
    """Residual MoE stack: y = h_n with h_{l+1} = bf16(h_l + MoE_l(RMSNorm(h_l))).
    x, y, tmp: bf16 bits [T][d]; logits: float32 [n][T][E]; important: uint8
    [n][T] or None; layers: list of PackedLayer sharing E, d, ffn, group."""
    n = len(layers)
    arr = (_Layer * n)(*[l.desc for l in layers])
    assert logits.dtype == torch.float32 and logits.is_contiguous()
    for t in (x, y) + (() if tmp is None else (tmp,)):
        assert t.is_contiguous() and t.element_size() == 2
    _check(load().mc_moe_stack_forward(_ptr(x), n, arr, _ptr(logits), _ptr(important),
                                       float(threshold), ctypes.byref(routing.desc), _ptr(y), _ptr(tmp),
                                       _ptr(workspace), workspace.numel() * workspace.element_size(),
                                       _stream(stream)))


def importance_workspace(H: int, L: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_importance_workspace(H, L, ctypes.byref(b)))
    return b.value


def token_importance(attn, x, rho: float, important, workspace, importance=None, stream=None):
    """attn: [H][L][L] bf16 bits (int16 tensor), x: [L][d] bf16 bits; writes the
    protected mask (uint8 [L]) and, if given, the importance (float32 [L])."""
    H, L, _ = attn.shape
    d = x.shape[1]
    _check(load().mc_token_importance(_ptr(attn), H, L, _ptr(x), d, ctypes.c_float(rho),
                                      None if importance is None else _ptr(importance), _ptr(important),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream(stream)))


def odp_threshold(logits_host):
    """(mu, tau) from calibration logits (a C-contiguous float32 numpy array [T][E])."""
    import numpy as np
    lg = np.ascontiguousarray(logits_host, dtype=np.float32)
    mu, tau = ctypes.c_double(), ctypes.c_double()
    _check(load().mc_odp_threshold(lg.ctypes.data_as(ctypes.c_void_p), lg.shape[0], lg.shape[1],
                                   ctypes.byref(mu), ctypes.byref(tau)))
    return mu.value, tau.value


def pmq_significance(logits_host, k: int):
    """(phi, w) per expert from calibration logits (float32 numpy [T][E])."""
    import numpy as np
    lg = np.ascontiguousarray(logits_host, dtype=np.float32)
    T, E = lg.shape
    phi, w = np.empty(E, np.float64), np.empty(E, np.float64)
    _check(load().mc_pmq_significance(lg.ctypes.data_as(ctypes.c_void_p), T, E, k,
                                      phi.ctypes.data_as(ctypes.c_void_p), w.ctypes.data_as(ctypes.c_void_p)))
    return phi, w


def pmq_allocate(phi, w, eps, total_bits: int, alpha: float = 1.0, beta: float = 1.0, gamma: float = 2.0):
    """Eq. 4 widths: (bits list, objective).  eps: [E][3] errors at 1, 2, 3 bits."""
    import numpy as np
    phi = np.ascontiguousarray(phi, dtype=np.float64)
    w = np.ascontiguousarray(w, dtype=np.float64)
    eps = np.ascontiguousarray(eps, dtype=np.float64)
    E = phi.shape[0]
    bits = np.empty(E, np.int32)
    obj = ctypes.c_double()
    _check(load().mc_pmq_allocate(phi.ctypes.data_as(ctypes.c_void_p), w.ctypes.data_as(ctypes.c_void_p),
                                  eps.ctypes.data_as(ctypes.c_void_p), E, float(alpha), float(beta),
                                  float(gamma), int(total_bits), bits.ctypes.data_as(ctypes.c_void_p),
                                  ctypes.byref(obj)))
    return [int(b) for b in bits], obj.value


def pmq_error_workspace(T: int, E: int, k: int, d: int, ffn: int, group: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_pmq_error_workspace(T, E, k, d, ffn, group, ctypes.byref(b)))
    return b.value


def pmq_expert_error(w_gate, w_up, w_down, x, routing: Routing, group: int, workspace, stream=None):
    """eps [E][3] (numpy fp64): the reconstruction error of each expert at 1,
    2 and 3 bits on the calibration batch x [T][d] (bf16 or int16 bits) routed
    by ``routing``; fp32 device weights as for pack()."""
    import numpy as np
    for t in (w_gate, w_up, w_down):
        assert t.dtype == torch.float32 and t.is_contiguous() and t.is_cuda
    assert x.is_contiguous() and x.element_size() == 2 and workspace.is_contiguous()
    E, ffn, d = w_gate.shape
    eps = np.empty((E, 3), np.float64)
    _check(load().mc_pmq_expert_error(_ptr(w_gate), _ptr(w_up), _ptr(w_down), E, d, ffn, int(group), _ptr(x),
                                      ctypes.byref(routing.desc), eps.ctypes.data_as(ctypes.c_void_p),
                                      _ptr(workspace), workspace.numel() * workspace.element_size(),
                                      _stream(stream)))
    return eps


def kv_page_bytes(page: int, Hkv: int, D: int, dtype=torch.bfloat16) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_kv_page_bytes(page, Hkv, D, _kv_dtype(dtype), ctypes.byref(b)))
    return b.value


_KV_DTYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1}
if hasattr(torch, "float4_e2m1fn_x2"):           # (all the rest works under a torch without it)
    _KV_DTYPES[torch.float4_e2m1fn_x2] = 4


def _kv_dtype(dtype) -> int:
    assert dtype in _KV_DTYPES, "a cache holds bfloat16, float8_e4m3fn or float4_e2m1fn_x2 (where torch has it)"
    return _KV_DTYPES[dtype]


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_on(dev: int, stream):
    """The given stream, or the current one of device dev, as an address."""
    if stream is not None:
        return stream.cuda_stream
    return _raw_stream(dev) if _raw_stream is not None else torch.cuda.current_stream().cuda_stream


def _here(*tensors) -> int:
    """The current device, on which the kernels run and on which the tensors
    (None aside) have to be."""
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() != dev:
            raise AssertionError("tensors must be on the current device")
    return dev


def _here_too(dev: int, *descriptors):
    """The descriptors' tensors (None and descriptors without any aside) lie on device dev."""
    for d in descriptors:
        if d is not None and d.dev is not None and d.dev != dev:
            raise AssertionError("the descriptors' tensors must be on the current device")


def _device_of(*tensors):
    """The one CUDA device of a descriptor's tensors (None aside; None if there are none)."""
    found = {t.get_device() for t in tensors if t is not None}
    assert len(found) <= 1 and -1 not in found, "a descriptor's tensors lie on one GPU"
    return found.pop() if found else None


def _bounded(n) -> int:
    """A window or length as a C int: any negative number stays one (and is refused), any
    past the largest says as much as that (a ctypes field would take it modulo 2^32)."""
    return max(-1, min(int(n), 2 ** 31 - 1))


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)      # bf16, or its bits


class KVCache:
    """Device buffers + descriptor of a paged cache (torch-allocated, or the
    given k and v: [n_pages][..] with contiguous pages, which may be slices of
    an allocation that layers share).  k_scale, v_scale: float32 [Hkv], for
    float8_e4m3fn caches.  float4_e2m1fn_x2 caches are uint8 arrays (a page holds
    codes and their scales)."""

    def __init__(self, n_pages: int, page: int, Hkv: int, D: int, dtype=torch.bfloat16, k=None, v=None,
                 k_scale=None, v_scale=None, device=None):
        kind = _kv_dtype(dtype)
        per = kv_page_bytes(page, Hkv, D, dtype)
        e = 1 if kind else 2
        device = device or torch.device("cuda")
        held = torch.uint8 if kind == 4 else dtype
        if k is None:
            k = torch.zeros((n_pages, per // e), dtype=held, device=device)
        if v is None:
            v = torch.zeros((n_pages, per // e), dtype=held, device=device)
        for t in (k, v):
            assert t.dtype in ((held, torch.uint8) if kind else _BF16) and t.shape[0] == n_pages
            assert t.numel() * e == n_pages * per and t[0].is_contiguous()
        stride = k.stride(0) * e if n_pages > 1 else per
        assert n_pages == 1 or v.stride(0) * e == stride, "k and v differ in their page stride"
        if kind == 1:
            for t in (k_scale, v_scale):
                assert t is not None and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == Hkv
        self.n_pages, self.page, self.Hkv, self.D, self.dtype = n_pages, page, Hkv, D, dtype
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.dev = _device_of(k, v, k_scale, v_scale)
        nb = (n_pages - 1) * stride + per
        self.desc = _KVCache(n_pages, page, Hkv, D, kind, k.data_ptr(), v.data_ptr(), stride, nb, nb,
                             k_scale.data_ptr() if k_scale is not None else None,
                             v_scale.data_ptr() if v_scale is not None else None)
        self.ref = ctypes.byref(self.desc)


class KVBatch:
    """Descriptor over a batch's device arrays (int32): kv_len [S], page_table
    [S][max_pages] and, for calls on several new tokens a sequence, q_start
    [S + 1] with T rows.  max_len: a length that few sequences exceed.  rows:
    those that attn_select and attn_sparse take, T, or without q_start S."""

    def __init__(self, kv_len, page_table, q_start=None, T=None, max_len: int = 0):
        S, max_pages = page_table.shape
        for t in (kv_len, page_table) + (() if q_start is None else (q_start,)):
            assert t.dtype == torch.int32 and t.is_contiguous()
        assert kv_len.numel() == S and (q_start is None or q_start.numel() == S + 1)
        assert q_start is None or T is not None, "q_start comes with T, the number of rows"
        self.S, self.T, self.max_pages = S, S if T is None else int(T), max_pages
        self.rows = S if q_start is None else self.T
        self.kv_len, self.page_table, self.q_start = kv_len, page_table, q_start
        self.dev = _device_of(kv_len, page_table, q_start)
        self.desc = _KVBatch(S, self.T, max_pages, _bounded(max_len), None if q_start is None else q_start.data_ptr(),
                             kv_len.data_ptr(), page_table.data_ptr())
        self.ref = ctypes.byref(self.desc)


class QKPrep:
    """Norm and rotation of kv_append.  rope: float32 [n_pos][rot/2][2] (cosine,
    sine); q_norm, k_norm: bfloat16 weights of a head, or with norm_row of the
    whole row."""

    def __init__(self, rope=None, rope_pairs: bool = False, q_norm=None, k_norm=None, norm_row: bool = False,
                 eps: float = 1e-5):
        if rope is not None:
            assert rope.dtype == torch.float32 and rope.is_contiguous() and rope.dim() == 3 and rope.shape[2] == 2
        for t in (q_norm, k_norm):
            assert t is None or (t.dtype in _BF16 and t.is_contiguous())
        self.dev = _device_of(rope, q_norm, k_norm)
        self.rope, self.q_norm, self.k_norm, self.norm_row = rope, q_norm, k_norm, bool(norm_row)
        ptr = lambda t: None if t is None else t.data_ptr()  # noqa: E731
        self.desc = _QKPrep(ptr(q_norm), ptr(k_norm), int(norm_row), float(eps),
                            0 if rope is None else 2 * rope.shape[1], int(rope_pairs), ptr(rope),
                            0 if rope is None else rope.shape[0])
        self.ref = ctypes.byref(self.desc)


class Attention:
    """Scores and masks of the attention calls.  slopes: float32 [Hq]; prefix:
    int32 [S]."""

    def __init__(self, Hq: int, scale: float, softcap: float = 0.0, window: int = 0, slopes=None, prefix=None):
        assert slopes is None or (slopes.dtype == torch.float32 and slopes.is_contiguous() and slopes.numel() == Hq)
        assert prefix is None or (prefix.dtype == torch.int32 and prefix.is_contiguous())
        self.dev = _device_of(slopes, prefix)
        self.Hq, self.slopes, self.prefix = Hq, slopes, prefix
        self.desc = _Attention(Hq, float(scale), float(softcap), _bounded(window),
                               None if slopes is None else slopes.data_ptr(),
                               None if prefix is None else prefix.data_ptr())
        self.ref = ctypes.byref(self.desc)


def _row_matrix(t, rows: int, width: int):
    """(address, elements between rows) of a bf16 matrix with contiguous rows."""
    s0, s1 = t.stride()
    assert t.shape == (rows, width) and t.dtype in _BF16 and s1 == 1
    return t.data_ptr(), s0 if rows > 1 else width


def kv_append(q, k, v, prep, batch: KVBatch, cache: KVCache, q_out, stream=None):
    """q [T][Hq*D], k and v [T][Hkv*D], q_out [T][Hq*D]: bf16, rows may be slices
    of wider ones; q and q_out may be None.  prep: QKPrep or None."""
    dev = _here(q, k, v, q_out)
    _here_too(dev, cache, batch, prep)
    assert batch.q_start is not None
    T, D, kw = batch.T, cache.D, cache.Hkv * cache.D
    qp, qs, op, os_, qw = None, 0, None, 0, D
    if q is not None:
        qw = q.shape[1]
        assert qw % D == 0
        qp, qs = _row_matrix(q, T, qw)
    if q_out is not None:
        op, os_ = _row_matrix(q_out, T, qw)
    kp, ks = _row_matrix(k, T, kw)
    vp, vs = _row_matrix(v, T, kw)
    if prep is not None and prep.q_norm is not None:
        assert prep.k_norm is None or prep.k_norm.numel() == (kw if prep.norm_row else D)
        assert q is None or prep.q_norm.numel() == (qw if prep.norm_row else D)
    _check(load().mc_kv_append(qp, qs, kp, ks, vp, vs, qw // D, None if prep is None else prep.ref, batch.ref,
                               cache.ref, op, os_, _stream_on(dev, stream)))


def attn_workspace(T: int, Hq: int, Hkv: int, D: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_attn_workspace(T, Hq, Hkv, D, ctypes.byref(b)))
    return b.value


def _attn(fn, rows, q, batch, cache, attn, o, workspace, lse, stream):
    dev = _here(q, o, lse, workspace)
    _here_too(dev, cache, batch, attn)
    width = attn.Hq * cache.D
    assert lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == rows * attn.Hq)
    assert attn.prefix is None or attn.prefix.numel() == batch.S
    qp, qs = _row_matrix(q, rows, width)
    op, os_ = _row_matrix(o, rows, width)
    _check(fn(qp, qs, batch.ref, cache.ref, attn.ref, op, os_, None if lse is None else lse.data_ptr(),
              workspace.data_ptr(), workspace.nbytes, _stream_on(dev, stream)))


def attn_decode(q, batch: KVBatch, cache: KVCache, attn: Attention, o, workspace, lse=None, stream=None):
    """q, o [S][Hq*D] bf16 (rows may be slices of wider ones); lse [S][Hq] float32."""
    _attn(load().mc_attn_decode, batch.S, q, batch, cache, attn, o, workspace, lse, stream)


def attn_prefill(q, batch: KVBatch, cache: KVCache, attn: Attention, o, workspace, lse=None, stream=None):
    """q, o [T][Hq*D] bf16 (rows may be slices of wider ones); lse [T][Hq] float32."""
    assert batch.q_start is not None
    _attn(load().mc_attn_prefill, batch.T, q, batch, cache, attn, o, workspace, lse, stream)


def kv_read(batch: KVBatch, cache: KVCache, k=None, v=None, stream=None):
    """The batch's new tokens as the cache stands for them: k, v [T][Hkv*D] bf16 (rows may be
    slices of wider ones), either may be None."""
    dev = _here(k, v)
    _here_too(dev, cache, batch)
    assert batch.q_start is not None
    width = cache.Hkv * cache.D
    kp, ks = (None, 0) if k is None else _row_matrix(k, batch.T, width)
    vp, vs = (None, 0) if v is None else _row_matrix(v, batch.T, width)
    _check(load().mc_kv_read(batch.ref, cache.ref, kp, ks, vp, vs, _stream_on(dev, stream)))


class KVPool:
    """Free pages of a cache: free_list int32 [n_pages] of which the first n_free (int32 [1]) are
    free, the top last.  n_free_out: where a call leaves the new height (n_free itself if None)."""

    def __init__(self, page: int, free_list, n_free, n_free_out=None):
        n_free_out = n_free if n_free_out is None else n_free_out
        for t in (free_list, n_free, n_free_out):
            assert t.dtype == torch.int32 and t.is_contiguous()
        assert n_free.numel() == 1 and n_free_out.numel() == 1
        self.page, self.free_list, self.n_free, self.n_free_out = page, free_list, n_free, n_free_out
        self.dev = _device_of(free_list, n_free, n_free_out)
        self.desc = _KVPool(free_list.numel(), page, free_list.data_ptr(), n_free.data_ptr(), n_free_out.data_ptr())
        self.ref = ctypes.byref(self.desc)


def kv_tables_workspace(S: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_kv_tables_workspace(S, ctypes.byref(b)))
    return b.value


def _tables(batch: KVBatch, positions=None, slots=None):
    """The batch's arrays as the tables calls take them."""
    return ctypes.byref(_KVTables(
        batch.S, batch.T, batch.max_pages, None if batch.q_start is None else batch.q_start.data_ptr(),
        batch.kv_len.data_ptr(), batch.page_table.data_ptr(), None if positions is None else positions.data_ptr(),
        None if slots is None else slots.data_ptr()))


def kv_reserve(want, past, pool: KVPool, batch: KVBatch, workspace, positions=None, slots=None, stream=None):
    """want, past: int32 [S] (past may be batch.kv_len).  Writes the batch's q_start, kv_len and new
    page table entries, and, if given, positions (int32 [T]) and slots (int64 [T])."""
    dev = _here(want, past, workspace, positions, slots)
    _here_too(dev, pool, batch)
    assert batch.q_start is not None
    for t in (want, past):
        assert t.dtype == torch.int32 and t.is_contiguous() and t.numel() == batch.S
    assert positions is None or (positions.dtype == torch.int32 and positions.is_contiguous()
                                 and positions.numel() == batch.T)
    assert slots is None or (slots.dtype == torch.int64 and slots.is_contiguous() and slots.numel() == batch.T)
    _check(load().mc_kv_reserve(want.data_ptr(), past.data_ptr(), pool.ref, _tables(batch, positions, slots),
                                workspace.data_ptr(), workspace.nbytes, _stream_on(dev, stream)))


def kv_release(done, past, pool: KVPool, batch: KVBatch, workspace, stream=None):
    """done: uint8 [S], past: int32 [S] (may be batch.kv_len).  Pushes the pages of requests that are
    done, and writes the batch's kv_len."""
    dev = _here(done, past, workspace)
    _here_too(dev, pool, batch)
    assert done.dtype == torch.uint8 and done.is_contiguous() and done.numel() == batch.S
    assert past.dtype == torch.int32 and past.is_contiguous() and past.numel() == batch.S
    _check(load().mc_kv_release(done.data_ptr(), past.data_ptr(), pool.ref, _tables(batch), workspace.data_ptr(),
                                workspace.nbytes, _stream_on(dev, stream)))


class KVSummary:
    """Bounds on the keys of a cache's pages: bounds int8 [n_pages][Hkv][2][D], scale float32
    [n_pages][Hkv] (torch-allocated, or given)."""

    def __init__(self, cache: KVCache, bounds=None, scale=None):
        if bounds is None:
            bounds = torch.zeros((cache.n_pages, cache.Hkv, 2, cache.D), dtype=torch.int8, device=cache.k.device)
        if scale is None:
            scale = torch.zeros((cache.n_pages, cache.Hkv), dtype=torch.float32, device=cache.k.device)
        assert bounds.dtype == torch.int8 and bounds.is_contiguous() and scale.dtype == torch.float32
        assert scale.is_contiguous()
        self.bounds, self.scale = bounds, scale
        self.dev = _device_of(bounds, scale)
        self.desc = _KVSummary(bounds.data_ptr(), scale.data_ptr(), bounds.nbytes, scale.nbytes)
        self.ref = ctypes.byref(self.desc)


def kv_summarize(batch: KVBatch, cache: KVCache, summary: KVSummary, stream=None):
    """Renews the bounds of the pages that the batch's new tokens lie on (without q_start: the last
    token of each sequence)."""
    dev = _here(batch.kv_len)
    _here_too(dev, cache, batch, summary)
    _check(load().mc_kv_summarize(batch.ref, cache.ref, summary.ref, _stream_on(dev, stream)))


def attn_select_workspace(T: int, Hkv: int, max_pages: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_attn_select_workspace(T, Hkv, max_pages, ctypes.byref(b)))
    return b.value


def _selection(sel, count, rows: int, Hkv: int) -> int:
    assert sel.dtype == torch.int32 and sel.is_contiguous() and sel.dim() == 3 and sel.shape[:2] == (rows, Hkv)
    assert count.dtype == torch.int32 and count.is_contiguous() and count.numel() == rows * Hkv
    return sel.shape[2]


def attn_select(q, batch: KVBatch, cache: KVCache, summary: KVSummary, attn: Attention, sel, count, workspace,
                keep_first: int = 1, keep_last: int = 1, stream=None):
    """q [rows][Hq*D] bf16; writes the selected pages sel (int32 [rows][Hkv][n_sel], places in the
    sequence) and their number count (int32 [rows][Hkv]).  rows: batch.rows."""
    dev = _here(q, sel, count, workspace)
    _here_too(dev, cache, batch, summary, attn)
    n_sel = _selection(sel, count, batch.rows, cache.Hkv)
    qp, qs = _row_matrix(q, batch.rows, attn.Hq * cache.D)
    _check(load().mc_attn_select(qp, qs, batch.ref, cache.ref, summary.ref, attn.ref, n_sel, _bounded(keep_first),
                                 _bounded(keep_last), sel.data_ptr(), count.data_ptr(), workspace.data_ptr(),
                                 workspace.nbytes, _stream_on(dev, stream)))


def attn_sparse(q, batch: KVBatch, cache: KVCache, attn: Attention, sel, count, o, workspace, lse=None, stream=None):
    """Attention to the pages sel[row][head][:count]: q, o [rows][Hq*D] bf16 (rows may be slices of
    wider ones), lse [rows][Hq] float32.  Rows as for attn_select."""
    dev = _here(q, sel, count, o, lse, workspace)
    _here_too(dev, cache, batch, attn)
    rows, width = batch.rows, attn.Hq * cache.D
    n_sel = _selection(sel, count, rows, cache.Hkv)
    assert lse is None or (lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == rows * attn.Hq)
    qp, qs = _row_matrix(q, rows, width)
    op, os_ = _row_matrix(o, rows, width)
    _check(load().mc_attn_sparse(qp, qs, batch.ref, cache.ref, attn.ref, sel.data_ptr(), count.data_ptr(), n_sel, op,
                                 os_, None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes,
                                 _stream_on(dev, stream)))


def attn_importance_workspace(Hq: int, L: int) -> int:
    b = ctypes.c_size_t()
    _check(load().mc_attn_importance_workspace(Hq, L, ctypes.byref(b)))
    return b.value


def attn_importance(q, lse, batch: KVBatch, cache: KVCache, attn: Attention, x, rho: float, important, workspace,
                    importance=None, stream=None):
    """q [L][Hq*D] bf16, lse [L][Hq] float32 (as attn_prefill wrote it), x [L][d] bf16;
    writes the protected mask (uint8 [L]) and, if given, the importance (float32 [L])."""
    dev = _here(q, lse, x, important, importance, workspace)
    _here_too(dev, cache, batch, attn)
    L, d = batch.T, x.shape[1]
    assert x.shape[0] == L and x.is_contiguous() and x.dtype in _BF16
    assert lse.dtype == torch.float32 and lse.is_contiguous() and lse.numel() == L * attn.Hq
    assert important.dtype == torch.uint8 and important.is_contiguous() and important.numel() == L
    assert importance is None or (importance.dtype == torch.float32 and importance.is_contiguous()
                                  and importance.numel() == L)
    qp, qs = _row_matrix(q, L, attn.Hq * cache.D)
    _check(load().mc_attn_importance(qp, qs, lse.data_ptr(), batch.ref, cache.ref, attn.ref, x.data_ptr(), d, rho,
                                     None if importance is None else importance.data_ptr(), important.data_ptr(),
                                     workspace.data_ptr(), workspace.nbytes, _stream_on(dev, stream)))


def timing_enable(on: bool = True):
    _check(load().mc_timing_enable(1 if on else 0))


def timing_read(kernel: str):
    """(summed ms, launches) of the events recorded for one kernel."""
    ms, n = ctypes.c_double(), ctypes.c_int()
    _check(load().mc_timing_read(kernel.encode(), ctypes.byref(ms), ctypes.byref(n)))
    return ms.value, n.value
