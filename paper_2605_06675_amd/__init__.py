"""Python binding of librq (the RateQuant hot path on MI355X).

Argument marshalling only: every step of the path runs in the HIP library.
Functions carry the C names; they raise RQError on a non-OK status.  Device
arguments are torch tensors on a HIP device (torch provides device memory
and streams), host arrays are numpy arrays.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "librq.so")

RQ_OK, RQ_EINVAL, RQ_EINFEASIBLE, RQ_EUNSUPPORTED, RQ_EDEVICE, RQ_ESMALLWS = (
    0, -1, -2, -3, -4, -5)
RQ_KIVI, RQ_QUAROT, RQ_TURBO, RQ_RTN, RQ_KIVI_RTN = 0, 1, 2, 3, 4
RQ_F16, RQ_BF16, RQ_F32 = 0, 1, 2
RQ_INT8, RQ_E4M3 = 0, 1
RQ_MAX_KV_HEADS = 32
RQ_MAX_NODES = 1024

EXPORTS = ("rq_version", "rq_last_error", "rq_cache_sizes", "rq_region_offset",
           "rq_quantize_kv", "rq_decode_workspace", "rq_decode_attention",
           "rq_calibrate_workspace", "rq_calibrate_distortion",
           "rq_fit_distortion", "rq_allocate_bits", "rq_turbo_codebook",
           "rq_sensitivity_workspace", "rq_sensitivity", "rq_cap_weights",
           "rq_fallback_beta", "rq_decode_static_bytes",
           "rq_decode_attention_static", "rq_read_probe", "rq_decode_step",
           "rq_block_sizes", "rq_block_append", "rq_block_advance",
           "rq_block_attention_workspace", "rq_block_attention",
           "rq_block_evict_workspace", "rq_block_evict", "rq_tree_mask",
           "rq_block_tree_attention_workspace", "rq_block_tree_attention",
           "rq_tree_verify_workspace", "rq_tree_verify", "rq_block_accept")
RQ_TURBO_TABLE_FLOATS = 8 * 2 * 256


class RQError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"status {status}: {msg}")
        self.status = status


class RqCache(C.Structure):
    _fields_ = [("family", C.c_int32), ("dtype", C.c_int32),
                ("n_layers", C.c_int32), ("batch", C.c_int32),
                ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("capacity", C.c_int32),
                ("residual", C.c_int32), ("bits", C.POINTER(C.c_int8)),
                ("codes", C.c_void_p), ("meta", C.c_void_p),
                ("resid", C.c_void_p), ("rotation", C.c_void_p),
                ("codebook", C.c_void_p)]


class RqBlockCache(C.Structure):
    _fields_ = [("format", C.c_int32), ("dtype", C.c_int32),
                ("n_layers", C.c_int32), ("batch", C.c_int32),
                ("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32),
                ("head_dim", C.c_int32), ("capacity", C.c_int32),
                ("codes", C.c_void_p), ("scales", C.c_void_p),
                ("tail", C.c_void_p), ("positions", C.c_void_p),
                ("weights", C.c_void_p), ("counters", C.c_void_p)]


class RqBlockRows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_batch", C.c_int64),
                ("stride_head", C.c_int64), ("stride_token", C.c_int64)]


class RqBlockQuery(C.Structure):
    _fields_ = [("n_new", C.c_int32), ("max_tokens", C.c_int32),
                ("past", C.c_void_p), ("new_len", C.c_void_p),
                ("q", RqBlockRows), ("out", RqBlockRows),
                ("out_dtype", C.c_int32), ("scale", C.c_float),
                ("cap", C.c_float), ("window", C.c_int32),
                ("slopes", C.c_void_p), ("accumulate", C.c_int32)]


class RqBlockTree(C.Structure):
    _fields_ = [("n_nodes", C.c_int32), ("max_tokens", C.c_int32),
                ("past", C.c_void_p), ("new_len", C.c_void_p),
                ("mask", C.c_void_p), ("depth", C.c_void_p),
                ("q", RqBlockRows), ("k", RqBlockRows), ("v", RqBlockRows),
                ("out", RqBlockRows), ("out_dtype", C.c_int32),
                ("scale", C.c_float), ("cap", C.c_float),
                ("window", C.c_int32), ("slopes", C.c_void_p)]


class RqTreeDraft(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_nodes", C.c_int32),
                ("vocab", C.c_int32), ("dtype", C.c_int32),
                ("tokens", C.c_void_p), ("parents", C.c_void_p),
                ("new_len", C.c_void_p), ("target", C.c_void_p),
                ("target_stride_batch", C.c_int64),
                ("target_stride_node", C.c_int64), ("draft", C.c_void_p),
                ("draft_stride_batch", C.c_int64),
                ("draft_stride_node", C.c_int64), ("uniforms", C.c_void_p),
                ("n_path", C.c_int32), ("path", C.c_void_p),
                ("count", C.c_void_p), ("next", C.c_void_p)]


class RqBlockLayers(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride_layer", C.c_int64),
                ("stride_batch", C.c_int64), ("stride_head", C.c_int64),
                ("stride_token", C.c_int64)]


_lib = None


def lib():
    """Load librq.so (built in-tree by build.py).  Raises if it is absent:
    there is no fallback path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with "
                "`python -m paper_2605_06675_amd.build`")
        L = C.CDLL(LIB_PATH)
        i32, u64, vp = C.c_int32, C.c_uint64, C.c_void_p
        pd, pi = C.POINTER(C.c_double), C.POINTER(C.c_int32)
        pu64 = C.POINTER(C.c_uint64)
        pc = C.POINTER(RqCache)
        sig = {
            "rq_version": (i32, []),
            "rq_last_error": (C.c_char_p, []),
            "rq_cache_sizes": (i32, [pc, pu64, pu64, pu64]),
            "rq_region_offset": (i32, [pc, i32, i32, i32, pu64]),
            "rq_quantize_kv": (i32, [pc, i32, i32, vp, vp, i32, vp]),
            "rq_decode_workspace": (i32, [pc, i32, pu64]),
            "rq_decode_attention": (i32, [pc, i32, i32, vp, vp, C.c_float, vp,
                                          u64, vp]),
            "rq_calibrate_workspace": (i32, [i32, i32, i32, pu64]),
            "rq_calibrate_distortion": (i32, [i32, i32, vp, i32, i32, i32, pi,
                                              i32, vp, vp, pd, pd, pd, pd, vp,
                                              u64, vp]),
            "rq_fit_distortion": (i32, [pd, i32, pi, i32, pd, pd, pd]),
            "rq_allocate_bits": (i32, [i32, pd, pd, pd, C.c_double, i32, i32,
                                       pi, pd, pd]),
            "rq_turbo_codebook": (i32, [C.POINTER(C.c_float)]),
            "rq_sensitivity_workspace": (i32, [i32, i32, i32, i32, pu64]),
            "rq_sensitivity": (i32, [i32, vp, i32, i32, i32, pd, vp, u64, vp]),
            "rq_cap_weights": (i32, [i32, pd, C.c_double]),
            "rq_fallback_beta": (i32, [i32, pd, pd, C.c_double]),
            "rq_decode_static_bytes": (u64, []),
            "rq_read_probe": (i32, [vp, u64, vp, i32, vp]),
            "rq_decode_attention_static": (i32, [pc, i32, i32, vp, vp,
                                                 C.c_float, vp]),
            "rq_decode_step": (i32, [pc, i32, i32, vp, vp, vp, vp, C.c_float,
                                     vp, u64, vp]),
        }
        pb, pq = C.POINTER(RqBlockCache), C.POINTER(RqBlockQuery)
        sig.update({
            "rq_block_sizes": (i32, [pb] + [pu64] * 6),
            "rq_block_append": (i32, [pb, i32, vp, i32, vp, vp, vp, vp]),
            "rq_block_advance": (i32, [pb, vp, i32, vp, vp, vp, vp, vp]),
            "rq_block_attention_workspace": (i32, [pb, pq, pu64]),
            "rq_block_attention": (i32, [pb, i32, vp, vp, u64, vp]),
            "rq_block_evict_workspace": (i32, [pb, i32, pu64]),
            "rq_block_evict": (i32, [pb, pb, i32, vp, i32, i32, i32, vp, vp,
                                     u64, vp]),
        })
        pt, pd_ = C.POINTER(RqBlockTree), C.POINTER(RqTreeDraft)
        sig.update({
            "rq_tree_mask": (i32, [i32, i32, vp, vp, vp, vp, vp]),
            "rq_block_tree_attention_workspace": (i32, [pb, pt, pu64]),
            "rq_block_tree_attention": (i32, [pb, i32, vp, vp, u64, vp]),
            "rq_tree_verify_workspace": (i32, [pd_, pu64]),
            "rq_tree_verify": (i32, [vp, vp, u64, vp]),
            "rq_block_accept": (i32, [pb, vp, i32, i32, vp, vp, vp, vp, vp, vp,
                                      vp, vp, vp]),
        })
        for name, (res, args) in sig.items():
            f = getattr(L, name)
            f.restype, f.argtypes = res, args
        _lib = L
    return _lib


def _check(status):
    if status != RQ_OK:
        raise RQError(status, lib().rq_last_error().decode())


def _dptr(a, dtype):
    a = np.ascontiguousarray(a, dtype=dtype)
    return a, a.ctypes.data_as(C.POINTER(np.ctypeslib.as_ctypes_type(dtype)))


def _tptr(t):
    """Device pointer of a contiguous torch tensor (None -> NULL)."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("device tensors must be contiguous")
    return C.c_void_p(t.data_ptr())


def _stream(stream=None):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return C.c_void_p(s.cuda_stream)


# ----------------------------------------------------------------- host calls
def rq_version():
    return lib().rq_version()


def rq_last_error():
    return lib().rq_last_error().decode()


def rq_fit_distortion(mse, bits):
    mse = np.atleast_2d(np.asarray(mse, dtype=np.float64))
    n_comp, n_bits = mse.shape
    m, mp = _dptr(mse, np.float64)
    b, bp = _dptr(bits, np.int32)
    out = [np.empty(n_comp) for _ in range(3)]
    ptrs = [o.ctypes.data_as(C.POINTER(C.c_double)) for o in out]
    _check(lib().rq_fit_distortion(mp, n_comp, bp, n_bits, *ptrs))
    return tuple(out)


def rq_allocate_bits(w, alpha, beta, avg_bits, bmin, bmax, want_cont=True):
    """Returns (bits int32[n], continuous float64[n] or None, J)."""
    w, wp = _dptr(w, np.float64)
    a, ap = _dptr(alpha, np.float64)
    be, bp = _dptr(beta, np.float64)
    n = w.size
    bits = np.empty(n, dtype=np.int32)
    cont = np.empty(n) if want_cont else None
    J = C.c_double()
    _check(lib().rq_allocate_bits(
        n, wp, ap, bp, float(avg_bits), int(bmin), int(bmax),
        bits.ctypes.data_as(C.POINTER(C.c_int32)),
        cont.ctypes.data_as(C.POINTER(C.c_double)) if want_cont else None,
        C.byref(J)))
    return bits, cont, J.value


def rq_turbo_codebook():
    """The TurboQuant codebook table, float32 [8][2][256]: [b-1][0] the
    thresholds, [b-1][1] the centroids of the b-bit Lloyd-Max quantizer."""
    t = np.empty(RQ_TURBO_TABLE_FLOATS, dtype=np.float32)
    _check(lib().rq_turbo_codebook(t.ctypes.data_as(C.POINTER(C.c_float))))
    return t.reshape(8, 2, 256)


def rq_calibrate_workspace(n_comp, n_tokens, n_bits):
    v = C.c_uint64()
    _check(lib().rq_calibrate_workspace(n_comp, n_tokens, n_bits, C.byref(v)))
    return v.value


def make_cache(family, dtype, n_layers, batch, n_kv_heads, n_q_heads,
               capacity, residual, bits, codes=None, meta=None, resid=None,
               rotation=None, codebook=None):
    """Fill an RqCache descriptor.  bits: int8 [n_layers][n_kv_heads][2];
    rotation, codebook: device tensors (TurboQuant only).  The numpy bit
    table is kept alive on the returned object."""
    bt = np.ascontiguousarray(bits, dtype=np.int8).reshape(-1)
    c = RqCache(family, dtype, n_layers, batch, n_kv_heads, n_q_heads, 128,
                capacity, residual, bt.ctypes.data_as(C.POINTER(C.c_int8)),
                _tptr(codes) if codes is not None else None,
                _tptr(meta) if meta is not None else None,
                _tptr(resid) if resid is not None else None,
                _tptr(rotation) if rotation is not None else None,
                _tptr(codebook) if codebook is not None else None)
    c._bits = bt
    return c


def rq_cache_sizes(cache):
    a, b, c = C.c_uint64(), C.c_uint64(), C.c_uint64()
    _check(lib().rq_cache_sizes(C.byref(cache), C.byref(a), C.byref(b),
                                C.byref(c)))
    return a.value, b.value, c.value


def rq_region_offset(cache, layer, head, kind):
    v = C.c_uint64()
    _check(lib().rq_region_offset(C.byref(cache), layer, head, kind,
                                  C.byref(v)))
    return v.value


def rq_decode_workspace(cache, n_tokens):
    v = C.c_uint64()
    _check(lib().rq_decode_workspace(C.byref(cache), n_tokens, C.byref(v)))
    return v.value


# --------------------------------------------------------------- device calls
def _need_device(t, what, shape, elem):
    """The C side sees raw pointers only: check what it cannot (shape,
    element size, device, contiguity) before a kernel reads or writes the
    buffer."""
    if not t.is_cuda:
        raise ValueError(f"{what} must be a device tensor")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.element_size() != elem:
        raise ValueError(f"{what} has {t.element_size()}-byte elements, expected {elem}")
    if not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")


def _check_attention_args(cache, q, out):
    import torch
    shape = (cache.batch, cache.n_q_heads, 128)
    _need_device(q, "q", shape, 2)
    _need_device(out, "out", shape, 4)
    if out.dtype != torch.float32 or q.device != out.device:
        raise ValueError("out must be float32 on q's device")


def rq_quantize_kv(cache, layer, n_past, k, v, stream=None):
    """k, v: torch [batch][n_kv_heads][n_new][128] (fp16/bf16, device)."""
    n_new = k.shape[2] if k.dim() == 4 else -1
    shape = (cache.batch, cache.n_kv_heads, n_new, 128)
    _need_device(k, "k", shape, 2)
    _need_device(v, "v", shape, 2)
    _check(lib().rq_quantize_kv(C.byref(cache), layer, n_past, _tptr(k),
                                _tptr(v), n_new, _stream(stream)))


def rq_decode_attention(cache, layer, n_tokens, q, out, ws, scale=None,
                        stream=None):
    """q: torch [batch][n_q_heads][128]; out: fp32 same shape; ws: device
    byte tensor of at least rq_decode_workspace bytes."""
    if scale is None:
        scale = 1.0 / np.sqrt(128.0)
    _check_attention_args(cache, q, out)
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous device tensor")
    _check(lib().rq_decode_attention(
        C.byref(cache), layer, n_tokens, _tptr(q), _tptr(out), float(scale),
        _tptr(ws), ws.numel() * ws.element_size(), _stream(stream)))


def rq_decode_step(cache, layer, n_past, k, v, q, out, ws, scale=None,
                   stream=None):
    """Append one token (k, v: [batch][n_kv_heads][1][128]) after n_past and
    attend over n_past + 1 tokens with q in one fused call; out, ws as for
    rq_decode_attention (ws sized for n_past + 1 tokens)."""
    if scale is None:
        scale = 1.0 / np.sqrt(128.0)
    shape = (cache.batch, cache.n_kv_heads, 1, 128)
    _need_device(k, "k", shape, 2)
    _need_device(v, "v", shape, 2)
    _check_attention_args(cache, q, out)
    if not ws.is_cuda or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous device tensor")
    _check(lib().rq_decode_step(
        C.byref(cache), layer, n_past, _tptr(k), _tptr(v), _tptr(q), _tptr(out),
        float(scale), _tptr(ws), ws.numel() * ws.element_size(),
        _stream(stream)))


def rq_decode_attention_static(cache, layer, n_tokens, q, out, scale=None,
                               stream=None):
    """rq_decode_attention with the library's own scratch: allocates
    nothing (for callers that cannot allocate)."""
    if scale is None:
        scale = 1.0 / np.sqrt(128.0)
    _check_attention_args(cache, q, out)
    _check(lib().rq_decode_attention_static(
        C.byref(cache), layer, n_tokens, _tptr(q), _tptr(out), float(scale),
        _stream(stream)))


def rq_read_probe(buf, sink, n_blocks, stream=None):
    """Read the whole device tensor buf once (measurement utility); sink:
    device int32/uint32 tensor of n_blocks elements."""
    _check(lib().rq_read_probe(_tptr(buf), buf.numel() * buf.element_size(),
                               _tptr(sink), int(n_blocks), _stream(stream)))


def rq_calibrate_distortion(family, dtype, x, is_value, bits, ws=None,
                            fit=True, rotation=None, codebook=None,
                            stream=None):
    """x: torch [n_comp][n_tokens][128] (device); rotation (bf16
    [n_comp][128][128]) and codebook (float32 table) on the device for
    TurboQuant.  Returns (mse[n_comp][n_bits], alpha, beta, r2) as numpy
    arrays (None when fit is False)."""
    import torch
    n_comp, T = x.shape[0], x.shape[1]
    b, bp = _dptr(bits, np.int32)
    need = rq_calibrate_workspace(n_comp, T, b.size)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=x.device)
    mse = np.empty((n_comp, b.size))
    outs = [np.empty(n_comp) for _ in range(3)] if fit else [None] * 3
    dp = C.POINTER(C.c_double)
    ptrs = [o.ctypes.data_as(dp) if o is not None else None for o in outs]
    _check(lib().rq_calibrate_distortion(
        family, dtype, _tptr(x), n_comp, T, int(bool(is_value)), bp, b.size,
        _tptr(rotation), _tptr(codebook), mse.ctypes.data_as(dp), *ptrs,
        _tptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))
    return (mse, *outs)


def rq_sensitivity_workspace(gdtype, n_seq, n_comp, n_tokens):
    v = C.c_uint64()
    _check(lib().rq_sensitivity_workspace(gdtype, n_seq, n_comp, n_tokens,
                                          C.byref(v)))
    return v.value


def rq_sensitivity(gdtype, grad, ws=None, stream=None):
    """grad: torch [n_seq][n_comp][n_tokens][128] on the device (float32,
    float16 or bfloat16 as gdtype says).  Returns w float64[n_comp]."""
    import torch
    n_seq, n_comp, T = grad.shape[0], grad.shape[1], grad.shape[2]
    need = rq_sensitivity_workspace(gdtype, n_seq, n_comp, T)
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=grad.device)
    w = np.empty(n_comp)
    _check(lib().rq_sensitivity(
        gdtype, _tptr(grad), n_seq, n_comp, T,
        w.ctypes.data_as(C.POINTER(C.c_double)), _tptr(ws),
        ws.numel() * ws.element_size(), _stream(stream)))
    return w


def rq_cap_weights(w, factor=5.0):
    """Returns a capped copy of w."""
    w = np.array(w, dtype=np.float64)
    _check(lib().rq_cap_weights(w.size, w.ctypes.data_as(C.POINTER(C.c_double)),
                                float(factor)))
    return w


def rq_fallback_beta(beta, r2, r2_min=0.96):
    """Returns a copy of beta with the fallback applied."""
    beta = np.array(beta, dtype=np.float64)
    r, rp = _dptr(r2, np.float64)
    if r.size != beta.size:
        raise ValueError("beta and r2 differ in length")
    _check(lib().rq_fallback_beta(beta.size,
                                  beta.ctypes.data_as(C.POINTER(C.c_double)),
                                  rp, float(r2_min)))
    return beta


class KVCache:
    """Device buffers (torch) plus the descriptor of one quantized cache."""

    def __init__(self, family, dtype, n_layers, batch, n_kv_heads, n_q_heads,
                 capacity, residual, bits, device="cuda", rotation=None):
        """rotation (TurboQuant only): device tensor of the bf16 rotations
        [n_layers][n_kv_heads][128][128] (y = R x); the codebook table is
        computed by the library and copied to the device here."""
        import torch
        self.desc = make_cache(family, dtype, n_layers, batch, n_kv_heads,
                               n_q_heads, capacity, residual, bits)
        self.rotation = self.codebook = None
        if family == RQ_TURBO:
            if rotation is None:
                raise ValueError("TurboQuant needs the rotations")
            if tuple(rotation.shape) != (n_layers, n_kv_heads, 128, 128) \
                    or rotation.element_size() != 2:
                raise ValueError("rotation must be 16-bit [L][H][128][128]")
            self.rotation = rotation.contiguous()
            self.codebook = torch.from_numpy(
                rq_turbo_codebook().reshape(-1)).to(device)
            self.desc.rotation = self.rotation.data_ptr()
            self.desc.codebook = self.codebook.data_ptr()
        cb, mb, rb = rq_cache_sizes(self.desc)
        self.codes = torch.zeros(max(cb, 1), dtype=torch.uint8, device=device)
        self.meta = torch.zeros(max(mb, 1), dtype=torch.uint8, device=device)
        self.resid = torch.zeros(max(rb, 2) // 2, dtype=torch.int16,
                                 device=device)
        self.desc.codes = self.codes.data_ptr()
        self.desc.meta = self.meta.data_ptr()
        self.desc.resid = self.resid.data_ptr()
        self.n_tokens = [0] * n_layers
        self._ws = None

    def append(self, layer, k, v, stream=None):
        rq_quantize_kv(self.desc, layer, self.n_tokens[layer], k, v, stream)
        self.n_tokens[layer] += k.shape[2]

    def workspace(self, n_tokens, stream=None):
        import torch
        need = rq_decode_workspace(self.desc, n_tokens)
        if self._ws is None or self._ws.numel() < need:
            # zeroed once, on the stream of the call that first uses it (a
            # zeroed counter is always read as stale, whatever the call's
            # number on this workspace)
            s = torch.cuda.current_stream() if stream is None else stream
            with torch.cuda.stream(s):
                self._ws = torch.zeros(need, dtype=torch.uint8,
                                       device=self.codes.device)
        return self._ws

    def attention(self, layer, q, out=None, scale=None, stream=None):
        import torch
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        n = self.n_tokens[layer]
        rq_decode_attention(self.desc, layer, n, q, out,
                            self.workspace(n, stream), scale, stream)
        return out

    def decode_step(self, layer, k, v, q, out=None, scale=None, stream=None):
        """Append one token to `layer` and attend over the cache with q
        (rq_decode_step)."""
        import torch
        if out is None:
            out = torch.empty(q.shape, dtype=torch.float32, device=q.device)
        n = self.n_tokens[layer]
        rq_decode_step(self.desc, layer, n, k, v, q, out,
                       self.workspace(n + 1, stream), scale, stream)
        self.n_tokens[layer] = n + 1
        return out

    def attention_static(self, layer, q, out, scale=None, stream=None):
        """Decode attention through rq_decode_attention_static (the
        library's own scratch; no allocation: out is the caller's)."""
        rq_decode_attention_static(self.desc, layer, self.n_tokens[layer], q,
                                   out, scale, stream)
        return out


# ------------------------------------------------- block-scaled 8-bit cache
def make_block_cache(format, dtype, n_layers, batch, n_kv_heads, n_q_heads,
                     head_dim, capacity, codes=None, scales=None, tail=None,
                     positions=None, weights=None):
    """Fill an RqBlockCache descriptor.  The device tensors must have the
    sizes rq_block_sizes reports; they are kept alive on the returned object,
    as are its counters, which are made here."""
    c = RqBlockCache(format, dtype, n_layers, batch, n_kv_heads, n_q_heads,
                     head_dim, capacity)
    buffers = (codes, scales, tail, positions, weights)
    given = [t for t in buffers if t is not None]
    if given:
        sizes = rq_block_sizes(c)
        for name, t, size in zip(("codes", "scales", "tail", "positions",
                                  "weights"), buffers, sizes):
            if t is None:
                continue
            if not t.is_cuda or t.device != given[0].device:
                raise ValueError(f"{name} must be on the cache's device")
            if t.numel() * t.element_size() < size:
                raise ValueError(f"{name} has {t.numel() * t.element_size()} "
                                 f"bytes, needs {size}")
            setattr(c, name, _tptr(t))
        import torch
        c._device = given[0].device
        c._calls = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        c._lengths = torch.int32
        # (the inputs' type, and the outputs')
        c._type = torch.bfloat16 if dtype == RQ_BF16 else torch.float16,
        c._out_types = {torch.float32: RQ_F32, torch.float16: RQ_F16,
                        torch.bfloat16: RQ_BF16}
        counters = torch.zeros(sizes[5] // 4, dtype=torch.int32, device=c._device)
        # calls may come on any stream
        torch.cuda.current_stream(c._device).synchronize()
        c.counters = counters.data_ptr()
        buffers += (counters,)
    c._buffers = buffers
    return c


def rq_block_sizes(cache):
    """Bytes of (codes, scales, tail, positions, weights, counters)."""
    v = [C.c_uint64() for _ in range(6)]
    _check(lib().rq_block_sizes(C.byref(cache), *(C.byref(x) for x in v)))
    return tuple(x.value for x in v)


# rq_block_rows and rq_block_query as packed bytes (a tenth of the time that
# filling ctypes structures takes, where a call takes ten microseconds)
_ROWS = struct.Struct("@Pqqq")
_QUERY = struct.Struct("@iiPPPqqqPqqqiffiPi4x")
_TREE = struct.Struct("@iiPPPPPqqqPqqqPqqqPqqqiffiP")
_DRAFT = struct.Struct("@iiiiPPPPqqPqqPiPPP")
_LAYERS = struct.Struct("@Pqqqq")
assert _ROWS.size == C.sizeof(RqBlockRows)
assert _QUERY.size == C.sizeof(RqBlockQuery)
assert _TREE.size == C.sizeof(RqBlockTree)
assert _DRAFT.size == C.sizeof(RqTreeDraft)
assert _LAYERS.size == C.sizeof(RqBlockLayers)


def _block_call(cache, stream, f, *args):
    """Launch on the given stream, or the current one of the cache's device,
    with that device current."""
    _device_call(cache._device, cache._calls, stream, f, *args)


def _device_call(device, calls, stream, f, *args):
    current, raw_stream = calls
    if stream is None:
        s = raw_stream(device.index)
    elif stream.device != device:
        raise ValueError(f"the stream is on {stream.device}, the cache on {device}")
    else:
        s = stream.cuda_stream
    if current() == device.index:
        status = f(*args, s)
    else:
        import torch
        with torch.cuda.device(device):
            status = f(*args, s)
    if status != RQ_OK:
        _check(status)


def _block_rows(cache, t, what, heads, n, dtypes):
    """Pointer and strides of t [batch][heads][n][head_dim] (any strides,
    contiguous rows)."""
    shape = (cache.batch, heads, n, cache.head_dim)
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {shape}")
    if t.device != cache._device:
        raise ValueError(f"{what} is on {t.device}, the cache on {cache._device}")
    if t.dtype not in dtypes:
        raise ValueError(f"{what} has dtype {t.dtype}, expected {next(iter(dtypes))}")
    sb, sh, st, sd = t.stride()
    if sd != 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    if what == "out" and (not sb and shape[0] > 1 or not sh and heads > 1
                          or not st and n > 1):
        raise ValueError("rows of out share memory")
    return t.data_ptr(), sb, sh, st


def _block_lengths(cache, t, what):
    """Pointer of an int32 [batch] tensor (0 for None)."""
    if t is None:
        return 0
    if t.dtype is not cache._lengths or t.device != cache._device \
            or t.shape != (cache.batch,) or not t.is_contiguous():
        raise ValueError(f"{what} must be int32 [{cache.batch}] on the cache's device")
    return t.data_ptr()


def _block_slopes(cache, slopes):
    if slopes is not None and (slopes.device != cache._device
                               or cache._out_types.get(slopes.dtype) != RQ_F32
                               or slopes.shape != (cache.n_q_heads,)
                               or not slopes.is_contiguous()):
        raise ValueError(f"slopes must be float32 [{cache.n_q_heads}] on the cache's device")


def _block_ws(cache, ws):
    if ws.device != cache._device or not ws.is_contiguous():
        raise ValueError("ws must be a contiguous tensor on the cache's device")
    return ws.data_ptr(), ws.numel() * ws.element_size()


def rq_block_append(cache, layer, past, k, v, new_len=None, stream=None):
    """k, v: torch [batch][n_kv_heads][n_new][head_dim] in the cache's dtype
    (any strides, contiguous rows); past, new_len: device int32 [batch]."""
    n = k.shape[2] if k.dim() == 4 else -1
    rk = _block_rows(cache, k, "k", cache.n_kv_heads, n, cache._type)
    rv = _block_rows(cache, v, "v", cache.n_kv_heads, n, cache._type)
    if past is None:
        raise ValueError("past is missing")
    _block_call(cache, stream, lib().rq_block_append, C.byref(cache), layer,
                _block_lengths(cache, past, "past"), n,
                _block_lengths(cache, new_len, "new_len"), _ROWS.pack(*rk),
                _ROWS.pack(*rv))


def rq_block_advance(cache, lengths, n_new, new_len=None, past=None,
                     fitting=None, dropped=None, stream=None):
    """lengths grow by the tokens of an append that fit; all device int32
    [batch]."""
    if lengths is None:
        raise ValueError("lengths is missing")
    _block_call(cache, stream, lib().rq_block_advance, C.byref(cache),
                _block_lengths(cache, lengths, "lengths"), n_new,
                _block_lengths(cache, new_len, "new_len"),
                _block_lengths(cache, past, "past"),
                _block_lengths(cache, fitting, "fitting"),
                _block_lengths(cache, dropped, "dropped"))


def rq_block_attention_workspace(cache, n_new, max_tokens=None,
                                 accumulate=False, window=0):
    """Workspace bytes of an attention call (a call with a window needs no
    more than one without)."""
    a = RqBlockQuery(n_new, cache.capacity if max_tokens is None else max_tokens)
    a.window, a.accumulate = int(window), int(bool(accumulate))
    v = C.c_uint64()
    _check(lib().rq_block_attention_workspace(C.byref(cache), C.byref(a),
                                              C.byref(v)))
    return v.value


def rq_block_attention(cache, layer, past, q, out, ws, new_len=None,
                       max_tokens=None, scale=None, cap=0.0, window=0,
                       slopes=None, accumulate=False, stream=None):
    """q: torch [batch][n_q_heads][n_new][head_dim] in the cache's dtype; out:
    the same shape in float32, float16 or bfloat16 (both any strides,
    contiguous rows); past, new_len: device int32 [batch]; slopes: device
    float32 [n_q_heads]; ws: device byte tensor of at least
    rq_block_attention_workspace bytes; max_tokens: bound on the sequences'
    lengths (the capacity by default)."""
    n = q.shape[2] if q.dim() == 4 else -1
    if past is None:
        raise ValueError("past is missing")
    _block_slopes(cache, slopes)
    rq_ = _block_rows(cache, q, "q", cache.n_q_heads, n, cache._type)
    ro = _block_rows(cache, out, "out", cache.n_q_heads, n, cache._out_types)
    a = _QUERY.pack(
        n, cache.capacity if max_tokens is None else max_tokens,
        _block_lengths(cache, past, "past"),
        _block_lengths(cache, new_len, "new_len"), *rq_, *ro,
        cache._out_types[out.dtype],
        cache.head_dim ** -0.5 if scale is None else scale, cap, window,
        0 if slopes is None else slopes.data_ptr(), 1 if accumulate else 0)
    _block_call(cache, stream, lib().rq_block_attention, C.byref(cache), layer,
                a, *_block_ws(cache, ws))


# ------------------------------------------------------ trees of drafted tokens
class _Torch:
    """What the calls below need of torch, looked up once (an import statement in
    each call takes as long as three of its checks)."""

    def __init__(self):
        import torch
        self.calls = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        self.int32, self.float32 = torch.int32, torch.float32
        self.types = {torch.float32: RQ_F32, torch.float16: RQ_F16,
                      torch.bfloat16: RQ_BF16}


_torch = None


def _the_torch():
    global _torch
    if _torch is None:
        _torch = _Torch()
    return _torch


def _tree_array(t, what, device, shape, dtype):
    """Pointer of a contiguous tensor."""
    if t.dtype is not dtype or t.shape != shape or t.device != device \
            or not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous {dtype} {list(shape)} on {device}")
    return t.data_ptr()


def _tree_call(device, stream, f, *args):
    if device.type != "cuda":
        raise ValueError(f"the tensors are on {device}, not on a GPU")
    _device_call(device, _the_torch().calls, stream, f, *args)


def rq_tree_mask(parents, mask, depth=None, new_len=None, stream=None):
    """Which nodes each drafted token sees.  parents: device int32
    [batch][n_nodes]; mask: int32 [batch][n_nodes][ceil(n_nodes / 32)], 32 nodes a
    word; depth: int32 [batch][n_nodes] (both are written); new_len: int32
    [batch]."""
    if parents.dim() != 2:
        raise ValueError(f"parents has shape {tuple(parents.shape)}, expected two axes")
    shape = B, n = parents.shape
    at, i32 = parents.device, _the_torch().int32
    _tree_call(at, stream, lib().rq_tree_mask, B, n,
               _tree_array(parents, "parents", at, shape, i32),
               0 if new_len is None else _tree_array(new_len, "new_len", at, (B,), i32),
               _tree_array(mask, "mask", at, (B, n, (n + 31) // 32), i32),
               0 if depth is None else _tree_array(depth, "depth", at, shape, i32))


def rq_block_tree_attention_workspace(cache, n_nodes, max_tokens=None, window=0):
    """Workspace bytes of a tree's attention call."""
    a = RqBlockTree(n_nodes, cache.capacity if max_tokens is None else max_tokens)
    a.window = int(window)
    v = C.c_uint64()
    _check(lib().rq_block_tree_attention_workspace(C.byref(cache), C.byref(a),
                                                   C.byref(v)))
    return v.value


def rq_block_tree_attention(cache, layer, past, q, k, v, mask, out, ws,
                            depth=None, new_len=None, max_tokens=None,
                            scale=None, cap=0.0, window=0, slopes=None,
                            stream=None):
    """Attention of drafted tokens over the cached ones and each other: q: torch
    [batch][n_q_heads][n_nodes][head_dim], k, v: [batch][n_kv_heads][n_nodes]
    [head_dim] in the cache's dtype; out: q's shape in float32, float16 or
    bfloat16 (all any strides, contiguous rows; a sequence's are finite, also where
    the mask hides a node); mask, depth: rq_tree_mask's (depth where there is a window
    or slopes); past: device int32 [batch], cached tokens; max_tokens: bound on them
    (the capacity by default); the rest as rq_block_attention."""
    n = q.shape[2] if q.dim() == 4 else -1
    if past is None:
        raise ValueError("past is missing")
    _block_slopes(cache, slopes)
    B, at, i32 = cache.batch, cache._device, cache._lengths
    rq_ = _block_rows(cache, q, "q", cache.n_q_heads, n, cache._type)
    rk = _block_rows(cache, k, "k", cache.n_kv_heads, n, cache._type)
    rv = _block_rows(cache, v, "v", cache.n_kv_heads, n, cache._type)
    ro = _block_rows(cache, out, "out", cache.n_q_heads, n, cache._out_types)
    a = _TREE.pack(
        n, cache.capacity if max_tokens is None else max_tokens,
        _block_lengths(cache, past, "past"),
        _block_lengths(cache, new_len, "new_len"),
        _tree_array(mask, "mask", at, (B, n, (n + 31) // 32), i32),
        0 if depth is None else _tree_array(depth, "depth", at, (B, n), i32),
        *rq_, *rk, *rv, *ro, cache._out_types[out.dtype],
        cache.head_dim ** -0.5 if scale is None else scale, cap, window,
        0 if slopes is None else slopes.data_ptr())
    _block_call(cache, stream, lib().rq_block_tree_attention, C.byref(cache),
                layer, a, *_block_ws(cache, ws))


def rq_tree_verify_workspace(batch, n_nodes, vocab):
    """Workspace bytes of rq_tree_verify."""
    d = RqTreeDraft(batch, n_nodes, vocab)
    v = C.c_uint64()
    _check(lib().rq_tree_verify_workspace(C.byref(d), C.byref(v)))
    return v.value


def _tree_rows(t, what, shape, dtype, device):
    """Pointer and strides of probabilities [batch][n_nodes][vocab]."""
    if t.shape != shape or t.dtype is not dtype or t.device != device:
        raise ValueError(f"{what} must be {dtype} {list(shape)} on {device}")
    sb, sn, sv = t.stride()
    if sv != 1 and shape[2] > 1:
        raise ValueError(f"the rows of {what} must be contiguous")
    return t.data_ptr(), sb, sn


def rq_tree_verify(tokens, parents, target, draft, uniforms, path, count, next,
                   ws, new_len=None, stream=None):
    """Verify drafted trees.  tokens, parents: device int32 [batch][n_nodes];
    target: float32, float16 or bfloat16 [batch][n_nodes][vocab], the target's
    probabilities behind each node; draft: the draft's, of its type and shape (both
    any strides, contiguous rows), or None: the drafted tokens were not drawn;
    uniforms: float32 [batch][n_nodes], 0..1; new_len: int32 [batch].
    Receives path: int32 [batch][room], the accepted nodes; count: int32 [batch];
    next: int32 [batch], the token drawn behind them.  ws: device byte tensor of at
    least rq_tree_verify_workspace bytes, zeroed before its first call (every call
    leaves it zero)."""
    if target.dim() != 3 or path.dim() != 2:
        raise ValueError("target must have three axes and path two")
    t, dtype = _the_torch(), target.dtype
    if dtype not in t.types:
        raise ValueError(f"target has dtype {dtype}")
    shape, at, i32 = target.shape, target.device, t.int32
    B, n, V = shape
    nodes = B, n
    if ws.device != at or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous tensor on {at}")
    d = _DRAFT.pack(
        B, n, V, t.types[dtype], _tree_array(tokens, "tokens", at, nodes, i32),
        _tree_array(parents, "parents", at, nodes, i32),
        0 if new_len is None else _tree_array(new_len, "new_len", at, (B,), i32),
        *_tree_rows(target, "target", shape, dtype, at),
        *((0, 0, 0) if draft is None
          else _tree_rows(draft, "draft", shape, dtype, at)),
        _tree_array(uniforms, "uniforms", at, nodes, t.float32),
        path.shape[1], _tree_array(path, "path", at, (B, path.shape[1]), i32),
        _tree_array(count, "count", at, (B,), i32),
        _tree_array(next, "next", at, (B,), i32))
    _tree_call(at, stream, lib().rq_tree_verify, d, ws.data_ptr(),
               ws.numel() * ws.element_size())


def rq_block_accept(cache, lengths, path, count, k, v, new_lengths, past=None,
                    fitting=None, dropped=None, stream=None):
    """Append a path of drafted tokens to every layer.  lengths: device int32
    [n_layers][batch], tokens held; path: int32 [batch][room] and count: int32
    [batch], as rq_tree_verify leaves them; k, v: torch [n_layers][batch]
    [n_kv_heads][n_nodes][head_dim] in the cache's dtype (any strides, contiguous
    rows).  new_lengths (lengths itself, or another tensor), past, fitting and
    dropped are written, as by rq_block_advance, each int32 [n_layers][batch]."""
    L, B, at = cache.n_layers, cache.batch, cache._device
    if path.dim() != 2:
        raise ValueError("path must have two axes")
    n = k.shape[3] if k.dim() == 5 else -1
    shape = (L, B, cache.n_kv_heads, n, cache.head_dim)
    packed = []
    for t, what in ((k, "k"), (v, "v")):
        if t.shape != shape or t.device != at or t.dtype not in cache._type:
            raise ValueError(f"{what} must be {cache._type[0]} {list(shape)} on {at}")
        if t.stride(4) != 1:
            raise ValueError(f"the rows of {what} must be contiguous")
        packed.append(_LAYERS.pack(t.data_ptr(), *t.stride()[:4]))

    i32, layers = cache._lengths, (L, B)

    def each(t, what):
        return 0 if t is None else _tree_array(t, what, at, layers, i32)
    if lengths is None or new_lengths is None:
        raise ValueError("lengths and new_lengths are needed")
    _block_call(cache, stream, lib().rq_block_accept, C.byref(cache),
                each(lengths, "lengths"), n, path.shape[1],
                _tree_array(path, "path", at, (B, path.shape[1]), i32),
                _tree_array(count, "count", at, (B,), i32), *packed,
                each(new_lengths, "new_lengths"), each(past, "past"),
                each(fitting, "fitting"), each(dropped, "dropped"))


def rq_block_evict_workspace(cache, keep):
    v = C.c_uint64()
    _check(lib().rq_block_evict_workspace(C.byref(cache), keep, C.byref(v)))
    return v.value


def rq_block_evict(src, dst, layer, lengths, keep, new_lengths, ws, n_sink=4,
                   n_recent=32, stream=None):
    """Shrink one layer of src into dst; lengths, new_lengths: device int32
    [batch], not the same memory; ws: device byte tensor of at least
    rq_block_evict_workspace bytes."""
    if lengths is None or new_lengths is None:
        raise ValueError("lengths and new_lengths are needed")
    if dst._device != src._device:
        raise ValueError("the caches are on different devices")
    _block_call(src, stream, lib().rq_block_evict, C.byref(src), C.byref(dst),
                layer, _block_lengths(src, lengths, "lengths"), keep, n_sink,
                n_recent, _block_lengths(src, new_lengths, "new_lengths"),
                *_block_ws(src, ws))


class DraftTree:
    """Drafted tokens of one step: which of them each one sees, and, verified,
    which are accepted.  parents: device int32 [batch][n_nodes] (a node's parent
    comes before it; node 0 is the root); new_len: device int32 [batch], how many
    of the nodes each sequence uses.

    The calls of one tree share its tensors: they go to one stream, or follow each
    other by the caller's events.  All can be captured into a graph."""

    def __init__(self, parents, new_len=None, stream=None):
        import torch
        B, n = parents.shape
        self.parents, self.new_len = parents, new_len
        s = torch.cuda.current_stream(parents.device) if stream is None else stream
        with torch.cuda.stream(s):
            # (rows that no sequence uses hold zeros)
            self.mask = torch.zeros(B, n, (n + 31) // 32, dtype=torch.int32,
                                    device=parents.device)
            self.depth = torch.zeros_like(parents)
        self._results = self._ws = None
        self._held = []             # tensors that a graph writes to
        self.layout(stream)

    def layout(self, stream=None):
        """Lay out again what parents and new_len hold now."""
        rq_tree_mask(self.parents, self.mask, self.depth, self.new_len, stream)

    def verify(self, tokens, target, uniforms, draft=None, room=None, stream=None):
        """(path, count, next) of rq_tree_verify: the accepted nodes ([batch]
        [room]), how many, and the token drawn behind them.  The tensors are this
        tree's own: a later call writes them again.  room: n_nodes by default; no
        path is longer than the tree's depth + 1, and BlockCache.accept plans for
        the whole room."""
        import torch
        B, n = self.parents.shape
        room = n if room is None else room
        s = torch.cuda.current_stream(target.device) if stream is None else stream
        need = rq_tree_verify_workspace(B, n, target.shape[-1])
        with torch.cuda.stream(s):
            capturing = torch.cuda.is_current_stream_capturing()
            ws = self._ws
            if ws is None or ws.numel() < need:
                if ws is not None:
                    ws.record_stream(s)
                ws = torch.zeros(need, dtype=torch.uint8, device=target.device)
                if not capturing:       # (else its zeros are the graph's work)
                    self._ws = ws
            if self._results is None or self._results[0].shape[1] != room:
                for t in self._results or ():
                    t.record_stream(s)
                self._results = tuple(
                    torch.empty(shape, dtype=torch.int32, device=target.device)
                    for shape in ((B, room), (B,), (B,)))
            if capturing:
                self._held.append((ws, self._results))
        rq_tree_verify(tokens, self.parents, target, draft, uniforms,
                       *self._results, ws, self.new_len, stream)
        return self._results


class BlockCache:
    """Device buffers (torch), lengths and the descriptor of one block-scaled
    8-bit cache.  `lengths` (device int32 [n_layers][batch]) says what each
    sequence holds, `bound` (host) at most how much any does.

    The calls of one cache share a workspace: they go to one stream, or follow
    each other by the caller's events.  All can be captured into a graph
    (evict with a given `into`).  A captured call is planned for the whole
    capacity; its replays move the lengths on, and drop tokens that do not
    fit: these are not attended and do not attend (their rows of `out` are left
    as they were, or 0 where the call made it).  From then on the layer's
    `bound` is the capacity, and a call that appends to it outside a graph may
    wait to read the lengths."""

    def __init__(self, format, dtype, n_layers, batch, n_kv_heads, n_q_heads,
                 head_dim, capacity, device="cuda", weights=False):
        import torch
        self.shape = (format, dtype, n_layers, batch, n_kv_heads, n_q_heads,
                      head_dim)
        sizes = rq_block_sizes(make_block_cache(*self.shape, capacity))
        types = (torch.uint8, torch.float32,
                 torch.bfloat16 if dtype == RQ_BF16 else torch.float16,
                 torch.int32, torch.float32)
        names = ("codes", "scales", "tail", "positions", "weights")
        for name, size, t in zip(names, sizes, types):
            new = torch.zeros(size // t.itemsize, dtype=t, device=device)
            setattr(self, name, new if name != "weights" or weights else None)
        self.lengths = torch.zeros(n_layers, batch, dtype=torch.int32,
                                   device=device)
        # of the tokens appended last: those before, those that fitted and those
        # that did not; layers where it may be any
        self._last = torch.zeros(3, n_layers, batch, dtype=torch.int32,
                                 device=device)
        self._drops = set()
        # (which waits for the buffers' zeros, these included)
        self.desc = make_block_cache(*self.shape, capacity,
                                     **{n: getattr(self, n) for n in names})
        self.bound = [0] * n_layers
        self._replayed = set()      # layers that a graph appends to
        self._ws = None
        self._held = []             # workspaces that a graph writes to

    def _on(self, stream):
        """The call's stream, and whether it is being captured."""
        import torch
        if stream is None:
            stream = torch.cuda.current_stream(self.codes.device)
        with torch.cuda.stream(stream):
            return stream, torch.cuda.is_current_stream_capturing()

    def _workspace(self, need, stream):
        import torch
        s, capturing = self._on(stream)
        if self._ws is None or self._ws.numel() < need:
            if self._ws is not None:
                self._ws.record_stream(s)
            with torch.cuda.stream(s):
                self._ws = torch.empty(max(need, 16), dtype=torch.uint8,
                                       device=self.codes.device)
        if capturing and not any(w is self._ws for w in self._held):
            self._held.append(self._ws)
        return self._ws

    def _grow(self, layer, n, new_len, stream):
        import torch
        row = self.lengths[layer]
        if layer in self._drops:
            rq_block_advance(self.desc, row, n, new_len,
                             *self._last[:, layer].unbind(), stream=stream)
        else:
            with torch.cuda.stream(self._on(stream)[0]):
                row += n if new_len is None else new_len.clamp(0, n)
        if layer not in self._replayed:
            self.bound[layer] += n

    def _room(self, layer, n, stream):
        """Bound on the tokens after n more."""
        import torch
        capacity = self.desc.capacity
        s, capturing = self._on(stream)
        if capturing:
            self._replayed.add(layer)
            self._drops.add(layer)
            self.bound[layer] = capacity
            return capacity
        held = self.bound[layer]
        if held + n > capacity:          # (an upper bound: padding counts)
            with torch.cuda.stream(s):
                held = int(self.lengths[layer].max())
            if held + n > capacity:
                raise ValueError(f"tokens {held} + {n} exceed the capacity "
                                 f"{capacity}")
            if layer not in self._replayed:
                self.bound[layer] = held
        return min(self.bound[layer] + n, capacity)

    def append(self, layer, k, v, new_len=None, stream=None):
        """Append k, v ([batch][n_kv_heads][n][head_dim]); new_len: how many
        of the n rows each sequence takes.  Where `bound` would pass the
        capacity, the lengths are read (a wait) before it is refused."""
        self._room(layer, k.shape[2], stream)
        rq_block_append(self.desc, layer, self.lengths[layer], k, v, new_len,
                        stream)
        self._grow(layer, k.shape[2], new_len, stream)

    def _attend(self, layer, past, bound, q, out, new_len, stream, kw):
        import torch
        need = rq_block_attention_workspace(self.desc, q.shape[2], bound,
                                            kw.get("accumulate", False),
                                            kw.get("window", 0))
        ws = self._workspace(need, stream)
        s = self._on(stream)[0]
        if out is None:
            with torch.cuda.stream(s):
                out = torch.zeros_like(q) if new_len is not None else torch.empty_like(q)
        rq_block_attention(self.desc, layer, past, q, out, ws, new_len, bound,
                           stream=stream, **kw)
        return out

    def attention(self, layer, q, out=None, new_len=None, stream=None, **kw):
        """Attention of the tokens appended last (q: [batch][n_q_heads][n]
        [head_dim]; scale, cap, window, slopes, accumulate as
        rq_block_attention)."""
        import torch
        s, capturing = self._on(stream)
        bound = self.desc.capacity if capturing else self.bound[layer]
        if new_len is not None:         # (padding may be more rows than tokens)
            bound = max(bound, q.shape[2])
        with torch.cuda.stream(s):
            new = q.shape[2] if new_len is None else new_len.clamp(0, q.shape[2])
            if capturing or layer in self._drops:
                new = new_len = (new - self._last[2, layer]).clamp_(min=0)
            past = self.lengths[layer] - new
        return self._attend(layer, past, bound, q, out, new_len, stream, kw)

    def step(self, layer, k, v, q, out=None, new_len=None, stream=None, **kw):
        """Append k, v and attend with the same tokens' q.  Where the
        attention is refused, the tokens are appended all the same."""
        bound = self._room(layer, k.shape[2], stream)
        past = self.lengths[layer]
        rq_block_append(self.desc, layer, past, k, v, new_len, stream)
        if layer in self._drops:
            self._grow(layer, k.shape[2], new_len, stream)
            past, fitting, _ = self._last[:, layer].unbind()
            return self._attend(layer, past, bound, q, out, fitting, stream, kw)
        try:
            return self._attend(layer, past, bound, q, out, new_len, stream, kw)
        finally:
            self._grow(layer, k.shape[2], new_len, stream)

    def tree_attention(self, layer, q, k, v, tree, out=None, stream=None, **kw):
        """Attention of drafted tokens (tree: a DraftTree; q: [batch][n_q_heads]
        [n_nodes][head_dim], k, v: [batch][n_kv_heads][n_nodes][head_dim]; scale,
        cap, window, slopes as rq_block_attention) over the layer's tokens and each
        other.  A sequence's nodes are finite, also those that no other sees.  The
        cache is left as it was: accept appends what is verified."""
        import torch
        s, capturing = self._on(stream)
        bound = self.desc.capacity if capturing else self.bound[layer]
        ws = self._workspace(rq_block_tree_attention_workspace(
            self.desc, q.shape[2], bound, kw.get("window", 0)), stream)
        if out is None:
            with torch.cuda.stream(s):
                out = torch.zeros_like(q) if tree.new_len is not None else torch.empty_like(q)
        rq_block_tree_attention(self.desc, layer, self.lengths[layer], q, k, v,
                                tree.mask, out, ws, tree.depth, tree.new_len,
                                bound, stream=stream, **kw)
        return out

    def accept(self, k, v, path, count, stream=None):
        """Append verified drafted tokens to every layer: the rows of k, v
        ([n_layers][batch][n_kv_heads][n_nodes][head_dim]) that path ([batch][room])
        names, count ([batch]) of each sequence (DraftTree.verify's).  `bound` grows
        by path's room; where it would pass the capacity, lengths and counts are
        read (a wait): a call is refused where its counts do not fit, else what the
        sequences then hold is the bound."""
        import torch
        room, layers, capacity = path.shape[1], self.desc.n_layers, self.desc.capacity
        s, capturing = self._on(stream)
        if capturing:
            bounds = [self._room(layer, room, stream) for layer in range(layers)]
        else:
            bounds = [held + room for held in self.bound]
        if max(bounds) > capacity:
            _tree_array(count, "count", self.desc._device, (self.desc.batch,), torch.int32)
            with torch.cuda.stream(s):
                held = (self.lengths + count.clamp(0, room)).amax(1).tolist()
            if max(held) > capacity:
                raise ValueError(f"tokens {max(held)} exceed the capacity {capacity}")
            bounds = [capacity if layer in self._replayed else n
                      for layer, n in enumerate(held)]
        past, fitting, dropped = self._last.unbind()
        rq_block_accept(self.desc, self.lengths, path, count, k, v, self.lengths,
                        past, fitting, dropped, stream)
        self.bound = bounds

    def evict(self, keep, n_sink=4, n_recent=32, into=None, stream=None):
        """Shrink every layer to at most `keep` tokens a sequence: into
        another BlockCache of this shape, or a new one of the least
        capacity."""
        import torch
        s, capturing = self._on(stream)
        if into is None:
            with torch.cuda.stream(s):
                into = BlockCache(*self.shape, (keep + 31) // 32 * 32,
                                  device=self.codes.device, weights=True)
        ws = self._workspace(rq_block_evict_workspace(self.desc, keep), stream)
        for layer in range(self.desc.n_layers):
            rq_block_evict(self.desc, into.desc, layer, self.lengths[layer],
                           keep, into.lengths[layer], ws, n_sink, n_recent,
                           stream)
            if capturing:
                into._replayed.add(layer)
            into.bound[layer] = (into.desc.capacity if layer in into._replayed
                                 else min(self.bound[layer], keep))
        if capturing:
            into._drops.update(range(self.desc.n_layers))
        if self._drops or into._drops:      # (the last tokens stay the last)
            with torch.cuda.stream(s):
                into._last.copy_(self._last)
            into._drops |= self._drops
        return into
