"""Thin Python binding of libminikv.so: argument marshalling only.

Every function here has the name and the argument order of its C entry point in include/minikv.h and
forwards device pointers of torch tensors (torch is used for device memory and streams, nothing else).  Some go through _bind.so first,
which does the same in compiled code.
There is no CPU fallback: if the HIP library is missing, loading raises.
"""
import ctypes as C
import os
import warnings

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libminikv.so")

BUF_NAMES = ("Kc", "Ks", "Kz", "Vc", "Vs", "Vz", "q_len", "Rk", "Rv", "r_len")
_BUF_DTYPE = dict(Kc=torch.int32, Vc=torch.int32, q_len=torch.int32, r_len=torch.int32,
                  Ks=torch.float16, Kz=torch.float16, Vs=torch.float16, Vz=torch.float16,
                  Rk=torch.float16, Rv=torch.float16)


class MinikvShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "D", "G", "Tcap", "Rcap")]


class MinikvCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in BUF_NAMES]


class MinikvPtShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "D", "G", "bits", "Tcap")]


PT_BUF_NAMES = ("Kc", "Ks", "Kz", "Vc", "Vs", "Vz", "q_len")


class MinikvPtCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in PT_BUF_NAMES]


class MinikvBlkShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("R", "Hq", "Hkv", "D", "block", "n_blocks", "max_blocks", "dtype")]


class MinikvBlkCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("K", "V", "Ks", "Vs")]


DTYPES = {torch.float16: 0, torch.bfloat16: 1}         # minikv_dtype


class MinikvError(RuntimeError):
    def __init__(self, status, where):
        self.status = status
        super().__init__("%s: %s (%d)" % (where, lib().minikv_strerror(status).decode(), status))


_lib = _bind = None


def lib():
    """Load libminikv.so, and _bind.so if it is there (built in-tree by `python -m paper_2411_18077_amd.build`)."""
    global _lib, _bind
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("libminikv.so is not built: run `python -m paper_2411_18077_amd.build` "
                              "(there is no fallback path)")
        l = C.CDLL(LIB_PATH)
        l.minikv_abi_version.restype = C.c_int
        l.minikv_strerror.restype = C.c_char_p
        l.minikv_strerror.argtypes = [C.c_int]
        l.minikv_strvariant.restype = C.c_char_p
        l.minikv_strvariant.argtypes = [C.c_int]
        l.minikv_set_variant.restype = C.c_int
        l.minikv_set_variant.argtypes = [C.c_int]
        l.minikv_diag_decode_weights.restype = C.c_int
        l.minikv_diag_decode_weights.argtypes = [C.c_int]
        l.minikv_diag_select_path.restype = C.c_int
        l.minikv_diag_select_path.argtypes = [C.c_int]
        l.minikv_buffer_bytes.restype = C.c_size_t
        l.minikv_buffer_bytes.argtypes = [C.POINTER(MinikvShape), C.c_int]
        l.minikv_cache_bytes.restype = C.c_size_t
        l.minikv_cache_bytes.argtypes = [C.POINTER(MinikvShape), C.c_int]
        l.minikv_workspace_bytes.restype = C.c_size_t
        l.minikv_workspace_bytes.argtypes = [C.POINTER(MinikvShape)]
        P = C.c_void_p
        l.kv_quantize_pack.restype = C.c_int
        l.kv_quantize_pack.argtypes = [C.POINTER(MinikvShape), P, P, C.c_int64, P, C.c_int64, P, C.c_int32,
                                       C.POINTER(MinikvCache), P]
        l.kv_append_residual.restype = C.c_int
        l.kv_append_residual.argtypes = [C.POINTER(MinikvShape), P, P, C.POINTER(MinikvCache), P]
        l.kv_flush_residual.restype = C.c_int
        l.kv_flush_residual.argtypes = [C.POINTER(MinikvShape), C.POINTER(MinikvCache), P]
        l.minikv_decode_attn.restype = C.c_int
        l.minikv_decode_attn.argtypes = [C.POINTER(MinikvShape), P, C.POINTER(MinikvCache), C.c_float, P, P,
                                         C.c_size_t, P]
        l.minikv_decode_step.restype = C.c_int
        l.minikv_decode_step.argtypes = [C.POINTER(MinikvShape), P, P, P, C.POINTER(MinikvCache), P, C.c_float, P, P,
                                         C.c_size_t, P]
        l.minikv_decode_attn_static.restype = C.c_int
        l.minikv_decode_attn_static.argtypes = [C.POINTER(MinikvShape), P, C.POINTER(MinikvCache), C.c_float, P, P]
        l.minikv_static_workspace_units.restype = C.c_size_t
        l.minikv_static_workspace_units.argtypes = []
        l.minikv_pt_cache_bytes.restype = C.c_size_t
        l.minikv_pt_cache_bytes.argtypes = [C.POINTER(MinikvPtShape), C.c_int]
        l.minikv_pt_workspace_bytes.restype = C.c_size_t
        l.minikv_pt_workspace_bytes.argtypes = [C.POINTER(MinikvPtShape)]
        l.kv_quantize_pack_pt.restype = C.c_int
        l.kv_quantize_pack_pt.argtypes = [C.POINTER(MinikvPtShape), P, P, C.c_int64, P, C.c_int64, P, C.c_int32,
                                          C.POINTER(MinikvPtCache), P]
        l.minikv_decode_attn_pt.restype = C.c_int
        l.minikv_decode_attn_pt.argtypes = [C.POINTER(MinikvPtShape), P, C.POINTER(MinikvPtCache), C.c_float, P, P,
                                            C.c_size_t, P]
        l.selective_flash_attn.restype = C.c_int
        l.selective_flash_attn.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int64, P, P, P, C.c_float, P, P, P, P,
                                           C.c_size_t, P]
        l.selective_flash_attn_workspace_bytes.restype = C.c_size_t
        l.selective_flash_attn_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int64]
        S = C.POINTER(MinikvBlkShape)
        l.minikv_blk_cache_bytes.restype = C.c_size_t
        l.minikv_blk_cache_bytes.argtypes = [S, C.c_int]
        l.minikv_blk_workspace_bytes.restype = C.c_size_t
        l.minikv_blk_workspace_bytes.argtypes = [S]
        l.kv_assign_blk.restype = C.c_int
        l.kv_assign_blk.argtypes = [S, P, P, P, P, P, P, P, P, P, C.c_int32, P]
        l.kv_quantize_blk.restype = C.c_int
        l.kv_quantize_blk.argtypes = [S, C.c_int32, P, C.c_int64, P, C.c_int64, P, C.POINTER(MinikvBlkCache), P]
        l.minikv_decode_attn_blk.restype = C.c_int
        l.minikv_decode_attn_blk.argtypes = [S, P, C.c_int64, C.POINTER(MinikvBlkCache), P, P, C.c_float, P, P, C.c_size_t, P]
        l.selective_flash_attn_packed.restype = C.c_int
        l.selective_flash_attn_packed.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_int32, P, C.c_int64,
                                                  P, C.c_int64, P, C.c_int64, P, C.c_float, P, P, P, P]
        l.minikv_prompt_blk_workspace_bytes.restype = C.c_size_t
        l.minikv_prompt_blk_workspace_bytes.argtypes = [S, C.c_int32]
        l.minikv_prompt_attn_blk.restype = C.c_int
        l.minikv_prompt_attn_blk.argtypes = [S, C.c_int32, P, C.c_int64, C.POINTER(MinikvBlkCache), P, P, P, C.c_float, P, P, P, C.c_size_t, P]
        l.minikv_norm_rope.restype = C.c_int
        l.minikv_norm_rope.argtypes = [C.c_int32, C.c_int32, C.c_int32, C.c_int32, P, C.c_int64, P, C.c_int64, P, P, C.c_float, P, C.c_int32,
                                       C.c_int32, P, P, C.c_int64, P, C.c_int64, P]
        l.kv_fork_blk.restype = C.c_int
        l.kv_fork_blk.argtypes = [S] + [P] * 12
        l.kv_copy_blk.restype = C.c_int
        l.kv_copy_blk.argtypes = [S, C.c_int32, C.POINTER(MinikvBlkCache), C.c_int32, P, P, P]
        l.kv_free_workspace_bytes.restype = C.c_size_t
        l.kv_free_workspace_bytes.argtypes = [S]
        l.kv_free_blk.restype = C.c_int
        l.kv_free_blk.argtypes = [S, P, P, P, P, P, C.c_size_t, P]
        l.kv_compact_blk.restype = C.c_int
        l.kv_compact_blk.argtypes = [S, P, P, P, P, P, C.c_int32, P, P, P, C.c_size_t, P]
        l.minikv_diag_redo_count.restype = C.c_int
        l.minikv_diag_redo_count.argtypes = [C.POINTER(MinikvShape), P, C.POINTER(C.c_int32)]
        l.minikv_stream_read_probe.restype = C.c_int
        l.minikv_stream_read_probe.argtypes = [P, C.c_size_t, P, P]
        l.kv_select_workspace_bytes.restype = C.c_size_t
        l.kv_select_workspace_bytes.argtypes = [C.c_int32, C.c_int32, C.c_int64]
        l.kv_select_hh_rw.restype = C.c_int
        l.kv_select_hh_rw.argtypes = [C.c_int32, C.c_int32, C.c_int64, P, P, P, P, C.c_int64, P, P, C.c_size_t, P]
        l.kv_pyramid_budget.restype = C.c_int
        l.kv_pyramid_budget.argtypes = [C.c_int32, C.c_double, C.c_int32, C.c_int32, C.POINTER(C.c_double)]
        _lib, _bind = l, _compiled()
    return _lib


def _compiled():
    """_bind.so, or None, and a warning, where it cannot be used: its calls are then made from here."""
    from .build import bound_to
    try:
        from . import _bind as bind
        what = getattr(bind, "built_for", "something that it does not name")
        if what == bound_to():
            return bind
        why = "it is built for %s" % what
    except ImportError as e:
        why = str(e)
    warnings.warn("the compiled calls of _bind.so are not in use, some calls take longer (`python -m paper_2411_18077_amd.build` makes it for %s): %s"
                  % (bound_to(), why), RuntimeWarning, stacklevel=3)
    return None


def _ptr(t):
    return None if t is None else t.data_ptr()         # (the argument types make pointers of the integers)


# The current stream's handle without the Python object torch.cuda.current_stream() builds around it: 0.2 instead of 3 of
# the 8.4 microseconds that a call with one launch took the host (5.2 now, 3.5 of them in the library and the runtime).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_device = getattr(torch._C, "_cuda_getDevice", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(_device())
        stream = torch.cuda.current_stream()
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc, where):
    if rc != 0:
        raise MinikvError(rc, where)


def make_shape(B, Hq, Hkv, D, G, Tcap, Rcap):
    return MinikvShape(B, Hq, Hkv, D, G, Tcap, Rcap)


def buffer_bytes(shape, which):
    return int(lib().minikv_buffer_bytes(C.byref(shape), which))


def cache_bytes(shape, which):
    return int(lib().minikv_cache_bytes(C.byref(shape), which))


def workspace_bytes(shape):
    return int(lib().minikv_workspace_bytes(C.byref(shape)))


class Cache:
    """Caller-owned device buffers of one cache (torch tensors), sized by minikv_cache_bytes."""

    def __init__(self, shape, device="cuda", fill=None):
        self.shape = shape
        self.t = {}
        for i, name in enumerate(BUF_NAMES):
            nbytes = cache_bytes(shape, i)
            dt = _BUF_DTYPE[name]
            n = max(nbytes // dt.itemsize, 1)         # Rcap == 0: a 1-element placeholder
            self.t[name] = torch.zeros(n, dtype=dt, device=device)
        self.workspace = torch.zeros(max(workspace_bytes(shape), 16), dtype=torch.uint8, device=device)   # zeroed once

    def __getattr__(self, name):
        t = self.__dict__.get("t", {})
        if name in t:
            return t[name]
        raise AttributeError(name)

    def c(self):
        t = self.t                                     # (written out: half the time of a generator, on every call)
        return MinikvCache(t["Kc"].data_ptr(), t["Ks"].data_ptr(), t["Kz"].data_ptr(), t["Vc"].data_ptr(), t["Vs"].data_ptr(),
                           t["Vz"].data_ptr(), t["q_len"].data_ptr(), t["Rk"].data_ptr(), t["Rv"].data_ptr(), t["r_len"].data_ptr())

    def nbytes(self):
        return sum(v.numel() * v.element_size() for v in self.t.values())

    def swap_r_len(self, other):
        """After minikv_decode_step: `other` (the array it wrote) becomes the cache's r_len; returns the old one."""
        old = self.t["r_len"]
        self.t["r_len"] = other
        return old


def kv_quantize_pack(shape, K, V, L, idx, idx_stride, n_tok, max_tok, cache, stream=None):
    cc = cache.c()
    _check(lib().kv_quantize_pack(C.byref(shape), _ptr(K), _ptr(V), int(L), _ptr(idx), int(idx_stride),
                                  _ptr(n_tok), int(max_tok), C.byref(cc), _stream(stream)), "kv_quantize_pack")


def kv_append_residual(shape, k_new, v_new, cache, stream=None):
    cc = cache.c()
    _check(lib().kv_append_residual(C.byref(shape), _ptr(k_new), _ptr(v_new), C.byref(cc), _stream(stream)),
           "kv_append_residual")


def kv_flush_residual(shape, cache, stream=None):
    cc = cache.c()
    _check(lib().kv_flush_residual(C.byref(shape), C.byref(cc), _stream(stream)), "kv_flush_residual")


def minikv_decode_attn(shape, q, cache, sm_scale, out, workspace=None, stream=None):
    cc = cache.c()
    ws = cache.workspace if workspace is None else workspace
    _check(lib().minikv_decode_attn(C.byref(shape), _ptr(q), C.byref(cc), float(sm_scale), _ptr(out), _ptr(ws),
                                    ws.numel() * ws.element_size(), _stream(stream)), "minikv_decode_attn")


def minikv_decode_attn_static(shape, q, cache, sm_scale, out, stream=None):
    cc = cache.c()
    _check(lib().minikv_decode_attn_static(C.byref(shape), _ptr(q), C.byref(cc), float(sm_scale), _ptr(out),
                                           _stream(stream)), "minikv_decode_attn_static")


def selective_flash_attn_workspace_bytes(B, Hkv, L):
    return int(lib().selective_flash_attn_workspace_bytes(int(B), int(Hkv), int(L)))


def selective_flash_attn(B, Hq, Hkv, L, Q, K, V, sm_scale, X_O, lse, A_cumul, workspace, stream=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().selective_flash_attn(int(B), int(Hq), int(Hkv), int(L), _ptr(Q), _ptr(K), _ptr(V), float(sm_scale),
                                      _ptr(X_O), _ptr(lse), _ptr(A_cumul), _ptr(workspace), nbytes, _stream(stream)),
           "selective_flash_attn")


def kv_select_workspace_bytes(units, rep, L):
    return int(lib().kv_select_workspace_bytes(int(units), int(rep), int(L)))


def kv_select_hh_rw(units, rep, L, A_cumul, n_hh, n_rw, idx, idx_stride, n_tok, workspace=None, stream=None):
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check(lib().kv_select_hh_rw(int(units), int(rep), int(L), _ptr(A_cumul), _ptr(n_hh), _ptr(n_rw), _ptr(idx),
                                 int(idx_stride), _ptr(n_tok), _ptr(workspace), nbytes, _stream(stream)),
           "kv_select_hh_rw")


def kv_pyramid_budget(n_layers, x, d, bottom_heavy):
    out = (C.c_double * max(int(n_layers), 1))()
    _check(lib().kv_pyramid_budget(int(n_layers), float(x), int(d), int(bottom_heavy), out), "kv_pyramid_budget")
    return list(out)[: int(n_layers)]


def minikv_stream_read_probe(src, sums, stream=None):
    _check(lib().minikv_stream_read_probe(_ptr(src), src.numel() * src.element_size(), _ptr(sums), _stream(stream)),
           "minikv_stream_read_probe")


def minikv_diag_redo_count(shape, workspace):
    n = C.c_int32(0)
    _check(lib().minikv_diag_redo_count(C.byref(shape), _ptr(workspace), C.byref(n)), "minikv_diag_redo_count")
    return int(n.value)


def minikv_decode_step(shape, q, k_new, v_new, cache, r_len_next, sm_scale, out, stream=None):
    """Append + attend in one launch; afterwards r_len_next holds the residual lengths (the caller swaps it with
    cache.r_len: see Cache.swap_r_len)."""
    cc = cache.c()
    _check(lib().minikv_decode_step(C.byref(shape), _ptr(q), _ptr(k_new), _ptr(v_new), C.byref(cc), _ptr(r_len_next),
                                    float(sm_scale), _ptr(out), _ptr(cache.workspace),
                                    cache.workspace.numel() * cache.workspace.element_size(), _stream(stream)),
           "minikv_decode_step")


def minikv_diag_decode_weights(mode):
    _check(lib().minikv_diag_decode_weights(int(mode)), "minikv_diag_decode_weights")


def minikv_diag_select_path(path):
    _check(lib().minikv_diag_select_path(int(path)), "minikv_diag_select_path")


def minikv_set_variant(v):
    _check(lib().minikv_set_variant(int(v)), "minikv_set_variant")


# ---------------------------------------------------------------------------------------------------------
# per-token quantized variant

def make_pt_shape(B, Hq, Hkv, D, G, bits, Tcap):
    return MinikvPtShape(B, Hq, Hkv, D, G, bits, Tcap)


class PtCache:
    """Caller-owned device buffers of one per-token quantized cache, sized by minikv_pt_cache_bytes."""

    def __init__(self, shape, device="cuda"):
        self.shape = shape
        self.t = {}
        for name in PT_BUF_NAMES:
            nbytes = int(lib().minikv_pt_cache_bytes(C.byref(shape), BUF_NAMES.index(name)))
            dt = _BUF_DTYPE[name]
            self.t[name] = torch.zeros(max(nbytes // dt.itemsize, 1), dtype=dt, device=device)
        self.workspace = torch.empty(max(int(lib().minikv_pt_workspace_bytes(C.byref(shape))), 16), dtype=torch.uint8,
                                     device=device)

    def __getattr__(self, name):
        t = self.__dict__.get("t", {})
        if name in t:
            return t[name]
        raise AttributeError(name)

    def c(self):
        t = self.t
        return MinikvPtCache(t["Kc"].data_ptr(), t["Ks"].data_ptr(), t["Kz"].data_ptr(), t["Vc"].data_ptr(), t["Vs"].data_ptr(),
                             t["Vz"].data_ptr(), t["q_len"].data_ptr())

    def nbytes(self):
        return sum(v.numel() * v.element_size() for v in self.t.values())


def kv_quantize_pack_pt(shape, K, V, L, idx, idx_stride, n_tok, max_tok, cache, stream=None):
    cc = cache.c()
    _check(lib().kv_quantize_pack_pt(C.byref(shape), _ptr(K), _ptr(V), int(L), _ptr(idx), int(idx_stride),
                                     _ptr(n_tok), int(max_tok), C.byref(cc), _stream(stream)), "kv_quantize_pack_pt")


def minikv_decode_attn_pt(shape, q, cache, sm_scale, out, stream=None):
    cc = cache.c()
    ws = cache.workspace
    _check(lib().minikv_decode_attn_pt(C.byref(shape), _ptr(q), C.byref(cc), float(sm_scale), _ptr(out), _ptr(ws),
                                       ws.numel(), _stream(stream)), "minikv_decode_attn_pt")


# ---------------------------------------------------------------------------------------------------------
# paged 8-bit cache and packed prompts

def _stride(x, heads):
    """Elements between the tokens of x [tokens][heads][128], whose heads lie side by side."""
    n, h, d = x.shape
    t, s, one = x.stride()
    if h != heads or d != 128 or one != 1 or (s != 128 and h > 1):
        raise ValueError("rows are [tokens][%d][128] with the heads of a token side by side: got shape %s, strides %s"
                         % (heads, tuple(x.shape), x.stride()))
    return t if n > 1 else heads * 128                 # (one token: any stride will do)


def _home(stream):
    """The current GPU's index, which is where a call runs (None where no GPU is in use), and the stream's handle."""
    if not torch.cuda.is_initialized():
        return None, 0 if stream is None else _stream(stream)
    home = _device()
    return home, _raw_stream(home) if stream is None else _stream(stream)


def _here(t, home, name):
    if t.get_device() != home:                         # (-1: host memory)
        raise ValueError("%s is on %s, the call runs on %s" % (name, t.device, "no GPU" if home is None else "cuda:%d" % home))
    return t.data_ptr()


def _need(t, dtype, n, name, home):
    """What a raw pointer does not tell the library: the type, that n elements lie one behind the other, and where."""
    if t.dtype is not dtype or t.numel() < n or not t.is_contiguous():
        raise ValueError("%s: a contiguous tensor of at least %d %s is needed, got %s of %s" % (name, n, dtype, t.dtype, tuple(t.shape)))
    return _here(t, home, name)


def make_blk_shape(R, Hq, Hkv, D, block, n_blocks, max_blocks, dtype):
    """dtype: torch.float16 or torch.bfloat16, of queries, keys, values and outputs."""
    if dtype not in DTYPES:
        raise ValueError("rows are torch.float16 or torch.bfloat16: got %s" % dtype)
    return MinikvBlkShape(R, Hq, Hkv, D, block, n_blocks, max_blocks, DTYPES[dtype])


class BlkCache:
    """Caller-owned device buffers of one paged 8-bit cache, sized by minikv_blk_cache_bytes; given ones are taken as they are.
    K, V: float8_e4m3fn [n_blocks][Hkv][block][128]; Ks, Vs: float32 [n_blocks][Hkv]; and a workspace of the attention, for calls on
    one stream at a time."""

    def __init__(self, shape, device="cuda", K=None, V=None, Ks=None, Vs=None):
        self.shape = shape
        codes, scales = int(lib().minikv_blk_cache_bytes(C.byref(shape), 0)), int(lib().minikv_blk_cache_bytes(C.byref(shape), 1))
        if not codes:
            raise ValueError("invalid shape")
        if K is not None:
            device = K.device
        rows = (shape.n_blocks, shape.Hkv)
        e4m3, f32 = torch.float8_e4m3fn, torch.float32

        def made(t, size, dtype, n, name):
            if t is None:
                return torch.zeros(size, dtype=torch.uint8 if dtype is e4m3 else dtype, device=device).view(dtype)
            _need(t, dtype, n, name, torch.empty(0, device=device).get_device())
            return t
        self._t = (made(K, rows + (shape.block, 128), e4m3, codes, "K"), made(V, rows + (shape.block, 128), e4m3, codes, "V"),
                   made(Ks, rows, f32, scales // 4, "Ks"), made(Vs, rows, f32, scales // 4, "Vs"))
        self._c = MinikvBlkCache(*(t.data_ptr() for t in self._t))
        self.workspace = torch.zeros(int(lib().minikv_blk_workspace_bytes(C.byref(shape))), dtype=torch.uint8, device=device)   # zeroed once

    K, V, Ks, Vs = (property(lambda self, i=i: self._t[i]) for i in range(4))          # (not to be replaced: the pointers are kept)

    def c(self):
        return self._c


def _fits(shape, cache, home):
    """The cache's buffers are big enough for the shape, and here."""
    own = cache.shape
    if own is not shape and (own.n_blocks < shape.n_blocks or own.Hkv != shape.Hkv or own.block != shape.block):
        raise ValueError("the cache is one of %d blocks of %d tokens and %d heads" % (own.n_blocks, own.block, own.Hkv))
    _here(cache.K, home, "the cache")
    return C.byref(cache.c())


_ASSIGN = ("q_len", "n_new", "table", "ring", "ring_state", "q_len_next", "ring_state_next", "cu", "slots")


def kv_assign_blk(shape, q_len, n_new, table, ring, ring_state, q_len_next, ring_state_next, cu, slots, stream=None):
    i32, R, (home, st) = torch.int32, shape.R, _home(stream)
    tensors = (q_len, n_new, table, ring, ring_state, q_len_next, ring_state_next, cu, slots)
    sizes = (R, R, R * shape.max_blocks, shape.n_blocks, 2, R, 2, R + 1, 0)
    for t, n in zip(tensors, sizes):                   # (_need written out: nine of them are half the call)
        if t.dtype is not i32 or t.numel() < n or not t.is_contiguous() or t.get_device() != home:
            for t, n, name in zip(tensors, sizes, _ASSIGN):
                _need(t, i32, n, name, home)
    _check(lib().kv_assign_blk(C.byref(shape), *[t.data_ptr() for t in tensors], slots.numel(), st), "kv_assign_blk")


def _rows(x, dtype, heads, name, home):
    if DTYPES.get(x.dtype) != dtype:
        raise ValueError("%s: got %s" % (name, x.dtype))
    return _stride(x, heads), _here(x, home, name)


def kv_quantize_blk(shape, K, V, slots, cache, stream=None):
    """K, V: [tokens][Hkv][128], possibly slices of a fused projection; slots: one per token."""
    n, (home, st) = K.shape[0], _home(stream)
    if V.shape[0] != n:
        raise ValueError("K has %d tokens, V %d" % (n, V.shape[0]))
    (ks, k), (vs, v) = _rows(K, shape.dtype, shape.Hkv, "K", home), _rows(V, shape.dtype, shape.Hkv, "V", home)
    _check(lib().kv_quantize_blk(C.byref(shape), n, k, ks, v, vs, _need(slots, torch.int32, n, "slots", home), _fits(shape, cache, home),
                                 st), "kv_quantize_blk")


def minikv_decode_attn_blk(shape, q, cache, table, q_len, sm_scale, out, workspace=None, stream=None):
    """q: [R][Hq][128], possibly a slice of a fused projection; out: contiguous.  q_len counts filed tokens: in a step of one new
    token each it is kv_assign_blk's q_len_next, behind kv_quantize_blk.  workspace: the cache's own if not given; calls on different
    streams that may overlap need one each (zero-filled once)."""
    home, st = _home(stream)
    (qs, p), ws = _rows(q, shape.dtype, shape.Hq, "q", home), cache.workspace if workspace is None else workspace
    if q.shape[0] < shape.R:
        raise ValueError("q has %d rows, the shape %d requests" % (q.shape[0], shape.R))
    if not ws.is_contiguous():
        raise ValueError("workspace: a contiguous tensor is needed")
    _check(lib().minikv_decode_attn_blk(C.byref(shape), p, qs, _fits(shape, cache, home),
                                        _need(table, torch.int32, shape.R * shape.max_blocks, "table", home),
                                        _need(q_len, torch.int32, shape.R, "q_len", home), float(sm_scale),
                                        _need(out, q.dtype, shape.R * shape.Hq * 128, "out", home), _here(ws, home, "workspace"),
                                        ws.numel() * ws.element_size(), st), "minikv_decode_attn_blk")


def selective_flash_attn_packed(B, Hq, Hkv, T, max_len, Q, K, V, cu, sm_scale, X_O, lse, A_cumul, stream=None):
    """Q: [T][Hq][128], K, V: [T][Hkv][128], possibly slices of a fused projection; X_O: contiguous; A_cumul may be None."""
    dtype, (home, st) = DTYPES.get(Q.dtype, -1), _home(stream)
    (qs, q), (ks, k), (vs, v) = _rows(Q, dtype, Hq, "Q", home), _rows(K, dtype, Hkv, "K", home), _rows(V, dtype, Hkv, "V", home)
    if min(Q.shape[0], K.shape[0], V.shape[0]) < T:
        raise ValueError("fewer than %d rows" % T)
    _check(lib().selective_flash_attn_packed(int(B), int(Hq), int(Hkv), int(T), int(max_len), dtype, q, qs, k, ks, v, vs,
                                             _need(cu, torch.int32, B + 1, "cu", home), float(sm_scale),
                                             _need(X_O, Q.dtype, T * Hq * 128, "X_O", home), _need(lse, torch.float32, T * Hq, "lse", home),
                                             None if A_cumul is None else _need(A_cumul, torch.float32, T * Hq, "A_cumul", home), st),
           "selective_flash_attn_packed")


def _quick(home):
    """The compiled calls: each checks its arguments as the function here that uses it does and makes the call, or returns None
    where one is not plainly right (or no GPU is in use), and has done nothing."""
    if _lib is None:
        lib()
    return _bind if home is not None else None


def _int_ptrs(home, names, tensors, sizes):
    """Pointers of contiguous int32 tensors of at least these sizes (_need written out: one after the other they are half of a call)."""
    i32 = torch.int32
    for t, n in zip(tensors, sizes):
        if t.dtype is not i32 or t.numel() < n or not t.is_contiguous() or t.get_device() != home:
            for t, n, name in zip(tensors, sizes, names):
                _need(t, i32, n, name, home)
    return [t.data_ptr() for t in tensors]


def minikv_prompt_blk_workspace_bytes(shape, T):
    return int(lib().minikv_prompt_blk_workspace_bytes(C.byref(shape), int(T)))


def _space(ws, home):
    if not ws.is_contiguous():
        raise ValueError("workspace: a contiguous tensor is needed")
    return _here(ws, home, "workspace"), ws.numel() * ws.element_size()


_PROMPT = ("table", "q_len", "cu")


def minikv_prompt_attn_blk(shape, T, q, cache, table, q_len, cu, sm_scale, out, lse, workspace, stream=None):
    """q: [T][Hq][128], possibly a slice of a fused projection; out: contiguous; lse: [T][Hq] or None.  cu and q_len are kv_assign_blk's cu
    and q_len_next, behind kv_quantize_blk."""
    home, st = _home(stream)
    quick = _quick(home)
    if quick and cache.shape is shape:
        rc = quick.prompt_attn_blk(home, st, C.addressof(shape), T, q, C.addressof(cache._c), cache._t[0], table, q_len, cu, sm_scale, out, lse, workspace)
        if rc is not None:
            return _check(rc, "minikv_prompt_attn_blk")
    R, Hq = shape.R, shape.Hq
    (qs, p), (ws, n) = _rows(q, shape.dtype, Hq, "q", home), _space(workspace, home)
    if q.shape[0] < T:
        raise ValueError("q has %d rows, fewer than %d" % (q.shape[0], T))
    _check(lib().minikv_prompt_attn_blk(C.byref(shape), T, p, qs, _fits(shape, cache, home),
                                        *_int_ptrs(home, _PROMPT, (table, q_len, cu), (R * shape.max_blocks, R, R + 1)),
                                        sm_scale, _need(out, q.dtype, T * Hq * 128, "out", home),
                                        None if lse is None else _need(lse, torch.float32, T * Hq, "lse", home), ws, n, st),
           "minikv_prompt_attn_blk")


def minikv_norm_rope(Hq, Hkv, T, Q, K, w_q, w_k, eps, inv_freq, rot_dim, adjacent, pos, Q_out, K_out, stream=None):
    """Q, Q_out: [T][Hq][128], K, K_out: [T][Hkv][128], possibly slices of a fused projection; Q_out and K_out may be Q and K.  w_q, w_k:
    [128] of the rows' type, or None; inv_freq: float32 [rot_dim / 2]."""
    home, st = _home(stream)
    quick = _quick(home)
    if quick:
        rc = quick.norm_rope(home, st, Hq, Hkv, T, Q, K, w_q, w_k, eps, inv_freq, rot_dim, adjacent, pos, Q_out, K_out)
        if rc is not None:
            return _check(rc, "minikv_norm_rope")
    dt = Q.dtype
    dtype, rows = DTYPES.get(dt, -1), []
    for x, heads, name in ((Q, Hq, "Q"), (K, Hkv, "K"), (Q_out, Hq, "Q_out"), (K_out, Hkv, "K_out")):
        (n, h, d), (t, side, one) = x.shape, x.stride()                # (_rows written out: four of them are half of the call)
        if x.dtype is not dt or n < T or h != heads or d != 128 or one != 1 or (side != 128 and h > 1) or x.get_device() != home:
            _rows(x, dtype, heads, name, home)
            raise ValueError("%s: fewer than %d rows" % (name, T))
        rows += (x.data_ptr(), t if n > 1 else heads * 128)
    q, qs, k, ks, qo, qos, ko, kos = rows
    if T == 1:                                         # (one row has no stride of its own)
        qos, kos = qs if qo == q else qos, ks if ko == k else kos
    _check(lib().minikv_norm_rope(Hq, Hkv, T, dtype, q, qs, k, ks, None if w_q is None else _need(w_q, dt, 128, "w_q", home),
                                  None if w_k is None else _need(w_k, dt, 128, "w_k", home), eps,
                                  _need(inv_freq, torch.float32, rot_dim // 2, "inv_freq", home) if rot_dim else None, rot_dim,
                                  1 if adjacent else 0, _need(pos, torch.int32, T, "pos", home), qo, qos, ko, kos, st), "minikv_norm_rope")


class BlkCaches:
    """The caches of a program's layers, all of one shape, for kv_copy_blk: BlkCache objects, or dicts of their buffers K, V, Ks, Vs."""

    def __init__(self, shape, layers):
        self.shape = shape
        self._t = []
        for x in layers:
            t = x._t if isinstance(x, BlkCache) else (x["K"], x["V"], x["Ks"], x["Vs"])
            home = t[0].get_device() if not self._t else self._t[0][0].get_device()
            codes, scales = int(lib().minikv_blk_cache_bytes(C.byref(shape), 0)), int(lib().minikv_blk_cache_bytes(C.byref(shape), 1)) // 4
            if not codes:
                raise ValueError("invalid shape")
            for y, dtype, n, name in zip(t, (torch.float8_e4m3fn,) * 2 + (torch.float32,) * 2, (codes, codes, scales, scales), ("K", "V", "Ks", "Vs")):
                _need(y, dtype, n, name, home)
            self._t.append(t)
        self._c = (MinikvBlkCache * max(len(self._t), 1))(*(MinikvBlkCache(*(y.data_ptr() for y in t)) for t in self._t))

    def __len__(self):
        return len(self._t)


_FORK = ("q_len", "parent", "n_keep", "table", "ring", "ring_state", "q_len_next", "table_next", "ring_state_next", "src", "dst")


def kv_fork_blk(shape, q_len, parent, n_keep, table, ring, ring_state, q_len_next, table_next, ring_state_next, src, dst, stream=None):
    home, st = _home(stream)
    quick = _quick(home)
    if quick:
        rc = quick.fork_blk(home, st, C.addressof(shape), q_len, parent, n_keep, table, ring, ring_state, q_len_next, table_next, ring_state_next, src, dst)
        if rc is not None:
            return _check(rc, "kv_fork_blk")
    R = shape.R
    rows = R * shape.max_blocks
    _check(lib().kv_fork_blk(C.byref(shape), *_int_ptrs(
        home, _FORK, (q_len, parent, n_keep, table, ring, ring_state, q_len_next, table_next, ring_state_next, src, dst),
        (R, R, R, rows, shape.n_blocks, 2, R, rows, 2, R, R)), st), "kv_fork_blk")


_PAIRS = ("src", "dst")


def _pairs(src):
    n = src.numel()
    if n > 1 << 30:
        raise ValueError("%d pairs, at most 2^30" % n)
    return n


def kv_copy_blk(shape, caches, src, dst, stream=None):
    """caches: BlkCaches; src, dst: a pair per element."""
    home, st = _home(stream)
    own, layers, quick = caches.shape, caches._t, _quick(home)
    if quick and own is shape and layers:
        rc = quick.copy_blk(home, st, C.addressof(shape), len(layers), C.addressof(caches._c), layers[0][0], src, dst)
        if rc is not None:
            return _check(rc, "kv_copy_blk")
    n = _pairs(src)
    if dst.numel() != n:
        raise ValueError("%d sources, %d destinations" % (n, dst.numel()))
    if own is not shape and (own.n_blocks < shape.n_blocks or own.Hkv != shape.Hkv or own.block != shape.block):
        raise ValueError("the caches are ones of %d blocks of %d tokens and %d heads" % (own.n_blocks, own.block, own.Hkv))
    if layers:
        _here(layers[0][0], home, "the caches")
    _check(lib().kv_copy_blk(C.byref(shape), len(layers), caches._c, n, *_int_ptrs(home, _PAIRS, (src, dst), (n, n)), st), "kv_copy_blk")


def kv_free_workspace_bytes(shape):
    return int(lib().kv_free_workspace_bytes(C.byref(shape)))


_FREE = ("q_len", "table", "ring", "ring_state")


def kv_free_blk(shape, q_len, table, ring, ring_state, workspace, stream=None):
    home, st = _home(stream)
    quick = _quick(home)
    if quick:
        rc = quick.free_blk(home, st, C.addressof(shape), q_len, table, ring, ring_state, workspace)
        if rc is not None:
            return _check(rc, "kv_free_blk")
    R, (ws, n) = shape.R, _space(workspace, home)
    _check(lib().kv_free_blk(C.byref(shape), *_int_ptrs(home, _FREE, (q_len, table, ring, ring_state),
                                                        (R, R * shape.max_blocks, shape.n_blocks, 2)), ws, n, st), "kv_free_blk")


_COMPACT = ("q_len", "table", "table_next", "ring", "ring_state", "src", "dst")


def kv_compact_blk(shape, q_len, table, table_next, ring, ring_state, src, dst, workspace, stream=None):
    """At most src.numel() blocks move."""
    home, st = _home(stream)
    quick = _quick(home)
    if quick:
        rc = quick.compact_blk(home, st, C.addressof(shape), q_len, table, table_next, ring, ring_state, src, dst, workspace)
        if rc is not None:
            return _check(rc, "kv_compact_blk")
    R = shape.R
    (ws, n), pairs, rows = _space(workspace, home), _pairs(src), R * shape.max_blocks
    p = _int_ptrs(home, _COMPACT, (q_len, table, table_next, ring, ring_state, src, dst), (R, rows, rows, shape.n_blocks, 2, pairs, pairs))
    _check(lib().kv_compact_blk(C.byref(shape), *p[:5], pairs, p[5], p[6], ws, n, st), "kv_compact_blk")
