"""ctypes binding of libfreqattn.so: the same entry points as include/freqattn.h, argument marshalling only.

Device tensors are torch tensors (torch is used for device memory and streams, nothing else); every computation
happens inside the library.  Loading fails loudly when the library has not been built.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libfreqattn.so")

OK, EINVAL, ENOMEM, EHIP, EUNSUPPORTED, ERANGE = 0, 1, 2, 3, 4, 5
F32, BF16 = 0, 1
LAUNCH_FUSED, LAUNCH_SEPARATE = 0, 1
PATH_AUTO, PATH_GENERIC, PATH_MFMA, PATH_TABLES_ONLY = 0, 1, 2, 3
TRANSFORM_DCT, TRANSFORM_HAAR = 0, 1
ROTARY_HALF, ROTARY_INTERLEAVED = 0, 1
ROTARY_PLAIN, ROTARY_LINEAR, ROTARY_NTK, ROTARY_BY_PARTS = 0, 1, 2, 3


class Shape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "heads", "head_dim", "T", "H", "W", "dtype")]


class BandCfg(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("low_num", "low_den", "mid_num", "mid_den", "low_compress", "mid_block",
                                         "mid_diag", "mid_stride", "mid_block0", "high_window", "n_summary")] + \
               [("softmax_scale", C.c_float), ("transform", C.c_int32), ("mid2_num", C.c_int32), ("mid2_den", C.c_int32)]


class Heads(C.Structure):
    """freqattn_heads: a device tensor [batch][rows][heads][channels] by its address and strides (elements)."""
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]


class RotaryCfg(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("axes", C.c_int32), ("axis_dim", C.c_int32 * 4), ("layout", C.c_int32), ("scaling", C.c_int32),
                ("context", C.c_int32), ("grid", C.c_int32 * 4), ("base", C.c_double), ("factor", C.c_double), ("beta_fast", C.c_double),
                ("beta_slow", C.c_double), ("amplitude", C.c_double)]


class QkShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "tokens", "q_heads", "k_heads", "head_dim", "dtype")] + [("eps", C.c_float)]


class SequenceShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("sequences", "q_heads", "kv_heads", "head_dim", "q_rows", "k_rows", "dtype", "causal")] + \
               [("softmax_scale", C.c_float)]


class SequenceRows(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q_offsets", "k_offsets", "q_lengths", "k_lengths")]


class Rows(C.Structure):
    """freqattn_rows: a device tensor [batch][rows][channels] by its address and strides (elements)."""
    _fields_ = [("data", C.c_void_p), ("batch_stride", C.c_int64), ("row_stride", C.c_int64)]


class NormShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("batch", "rows", "channels", "dtype", "weights_per_batch")] + [("eps", C.c_float)]


class ProductShape(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rows", "channels", "outputs", "dtype")]


class Cache8(C.Structure):
    """freqattn_cache8: codes of keys and values (freqattn_heads, field by field), their scales, rows of a block."""
    _fields_ = [f for x in "kv" for f in ((x + "_data", C.c_void_p), (x + "_batch_stride", C.c_int64), (x + "_row_stride", C.c_int64), (x + "_head_stride", C.c_int64))] + \
               [("k_scales", C.c_void_p), ("v_scales", C.c_void_p), ("block_rows", C.c_int32)]


_H, _P = C.POINTER(Heads), C.c_void_p
_R, _N, _C8 = C.POINTER(Rows), C.POINTER(NormShape), C.POINTER(Cache8)
_SEQ = [C.POINTER(SequenceShape), C.POINTER(SequenceRows)]
_ROT = [_P, _P, C.c_int64]     # rotary, positions, positions_stride

EXPORTS = {
    "freqattn_create": (C.c_int, [C.POINTER(Shape), C.POINTER(BandCfg), C.c_int32, C.POINTER(C.c_void_p)]),
    "freqattn_forward": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(BandCfg),
                                   C.POINTER(C.c_int32), C.c_void_p, C.c_void_p]),
    "freqattn_forward_static": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(BandCfg),
                                          C.POINTER(C.c_int32), C.c_void_p, C.c_void_p]),
    "freqattn_forward_projected": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p,
                                             C.c_void_p, C.POINTER(BandCfg), C.POINTER(C.c_int32), C.c_void_p, C.c_void_p]),
    "freqattn_destroy": (None, [C.c_void_p]),
    "freqattn_last_error": (C.c_char_p, [C.c_void_p]),
    "freqattn_set_launch_mode": (C.c_int, [C.c_void_p, C.c_int32]),
    "freqattn_get_path": (C.c_int32, [C.c_void_p]),
    "freqattn_set_exchange_fusion": (C.c_int, [C.c_void_p, C.c_int32]),
    "freqattn_set_alloc_prediction": (C.c_int, [C.c_void_p, C.c_int32]),
    "freqattn_band_sizes": (C.c_int, [C.c_void_p, C.POINTER(C.c_int64)]),
    "freqattn_band_index": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]),
    "freqattn_mid_blocks": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int64)]),
    "freqattn_mid2_blocks": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_int32), C.POINTER(C.c_int64)]),
    "freqattn_dct_matrix": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_double)]),
    "freqattn_get_v_box": (C.c_int32, [C.c_void_p]),
    "freqattn_summary_weights": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_float)]),
    "freqattn_read_spectral": (C.c_int, [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_float), C.c_void_p]),
    "freqattn_route_fixed": (C.c_int, [C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_int32)]),
    "freqattn_load_balance": (C.c_int, [C.POINTER(C.c_float), C.c_int32, C.c_float, C.POINTER(C.c_float)]),
    "freqattn_route_mlp": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_int32,
                                     C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_float),
                                     C.POINTER(C.c_float), C.POINTER(C.c_int32), C.POINTER(C.c_float),
                                     C.POINTER(C.c_float), C.c_void_p]),
    "freqattn_forward_routed": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.POINTER(BandCfg), C.c_float,
                                          C.c_int32, C.POINTER(C.c_float), C.POINTER(C.c_float), C.POINTER(C.c_float),
                                          C.POINTER(C.c_float), C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_float),
                                          C.c_void_p]),
    "freqattn_dense_forward": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "freqattn_set_stage_timing": (C.c_int, [C.c_void_p, C.c_int32]),
    "freqattn_stage_times": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(C.c_char_p), C.POINTER(C.c_float),
                                       C.POINTER(C.c_int32)]),
    "freqattn_workspace_bytes": (C.c_int64, [C.c_void_p]),
    "freqattn_check_range": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.c_void_p]),
    "freqattn_measure_peaks": (C.c_int, [C.c_void_p, C.POINTER(C.c_double), C.POINTER(C.c_double), C.c_void_p]),
    "freqattn_forward_tokens": (C.c_int, [_P, _H, _H, _H, _P, _P, C.c_float] + _ROT + [C.POINTER(BandCfg), C.POINTER(C.c_int32), _P, _P]),
    "freqattn_rotary_create": (C.c_int, [C.POINTER(RotaryCfg), C.POINTER(_P)]),
    "freqattn_rotary_destroy": (None, [_P]),
    "freqattn_rotary_frequencies": (C.c_int, [_P, C.POINTER(C.c_double), C.POINTER(C.c_double)]),
    "freqattn_rotary_apply": (C.c_int, [_P, C.c_int32, C.c_int32, C.c_int32, C.c_int32, _H, _P, C.c_int64, C.c_int32, _H, _P]),
    "freqattn_qk_norm": (C.c_int, [C.POINTER(QkShape)] + _ROT + [_H, _H, _P, _P, _H, _H, _P]),
    "freqattn_qk_norm_workspace": (C.c_int64, [C.c_int32]),
    "freqattn_qk_norm_backward": (C.c_int, [C.POINTER(QkShape)] + _ROT + [_H, _H, _P, _P, _H, _H, _H, _H, _P, _P, _P, C.c_int64, _P]),
    "freqattn_sequence_attention_workspace": (C.c_int64, _SEQ),
    "freqattn_sequence_attention": (C.c_int, _SEQ + [_H, _H, _H, _H, _P, _P, C.c_int64, _P]),
    "freqattn_sequence_attention_backward_workspace": (C.c_int64, _SEQ),
    "freqattn_sequence_attention_backward": (C.c_int, _SEQ + [_H] * 5 + [_P] + [_H] * 3 + [_P, C.c_int64, _P]),
    "freqattn_layer_norm": (C.c_int, [_N, _R, _P, _P, _R, _P]),
    "freqattn_layer_norm_workspace": (C.c_int64, [_N]),
    "freqattn_layer_norm_backward": (C.c_int, [_N, _R, _P, _R, _R, _P, _P, _P, C.c_int64, _P]),
    "freqattn_quantize_rows": (C.c_int, [C.c_int32] * 4 + [_R, _R, _P, _P]),
    "freqattn_product_i8": (C.c_int, [C.POINTER(ProductShape), _P, C.c_int64, _P, _P, C.c_int64, _P, _P, _P, C.c_int64, _P]),
    "freqattn_cache8_append": (C.c_int, _SEQ + [_H, _H, _C8, _P]),
    "freqattn_cache8_read": (C.c_int, _SEQ + [_C8, _H, _H, _P]),
    "freqattn_cache8_attention_workspace": (C.c_int64, _SEQ),
    "freqattn_cache8_attention": (C.c_int, _SEQ + [_H, _C8, _H, _P, _P, C.c_int64, _P]),
}

_lib = None


def lib():
    """The loaded library; raises if it has not been built (there is no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -c 'import __graft_entry__ as g; g.build()'` "
                               "(or python paper_2604_22808_amd/build.py) first")
        # torch ships its own HIP runtime (same soname): load it first so that the library binds to the runtime
        # that owns torch's device memory and streams instead of bringing a second one into the process.
        import torch  # noqa: F401
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in EXPORTS.items():
            fn = getattr(l, name)
            fn.restype = res
            fn.argtypes = args
        _lib = l
    return _lib


class FreqAttnError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__(f"freqattn status {status}: {msg}")
        self.status = status


def _ptr(t):
    return C.c_void_p(t.data_ptr())


def _stream():
    import torch
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def make_cfg(**kw) -> BandCfg:
    base = dict(low_num=1, low_den=4, mid_num=1, mid_den=2, low_compress=4, mid_block=64, mid_diag=1, mid_stride=8,
                mid_block0=1, high_window=256, n_summary=16, softmax_scale=0.0, transform=0, mid2_num=0, mid2_den=1)
    base.update(kw)
    return BandCfg(**base)


class Context:
    """Owns one freqattn_ctx.  Methods carry the names of the C entry points without the prefix."""

    def __init__(self, batch, heads, head_dim, grid, dtype, cfg: BandCfg, path=PATH_AUTO):
        self.shape = Shape(batch, heads, head_dim, grid[0], grid[1], grid[2], dtype)
        self.cfg = cfg
        self._h = C.c_void_p()
        st = lib().freqattn_create(C.byref(self.shape), C.byref(cfg), path, C.byref(self._h))
        if st != OK:
            raise FreqAttnError(st, lib().freqattn_last_error(None).decode())

    def _check(self, st):
        if st != OK:
            raise FreqAttnError(st, lib().freqattn_last_error(self._h).decode())

    def destroy(self):
        if self._h:
            lib().freqattn_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.destroy()
        except Exception:
            pass

    def _check_tensors(self, who, **tensors):
        """The library sees raw addresses only: a tensor on the host, of another type, shape or layout would make its
        kernels read or write out of bounds, so every device tensor is checked here before its pointer is taken."""
        import torch
        s = self.shape
        want_shape = (s.batch, s.heads, s.T * s.H * s.W, s.head_dim)
        want_dtype = torch.bfloat16 if s.dtype == BF16 else torch.float32
        for name, t in tensors.items():
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{who}: {name} must be a torch tensor")
            if not t.is_cuda:
                raise ValueError(f"{who}: {name} must be a device tensor")
            if t.dtype != want_dtype:
                raise ValueError(f"{who}: {name} has dtype {t.dtype}, the context was created for {want_dtype}")
            if tuple(t.shape) != want_shape:
                raise ValueError(f"{who}: {name} has shape {tuple(t.shape)}, expected {want_shape}")
            if not t.is_contiguous():
                raise ValueError(f"{who}: {name} must be contiguous")

    # ---- hot path
    def forward(self, q, k, v, head_alloc, out, cfg=None):
        self._check_tensors("forward", q=q, k=k, v=v, out=out)
        ha = np.ascontiguousarray(head_alloc, dtype=np.int32)
        if ha.shape != (self.shape.heads,):
            raise ValueError(f"forward: head_alloc must hold {self.shape.heads} entries, got shape {ha.shape}")
        cfg = cfg or self.cfg
        self._check(lib().freqattn_forward(self._h, _ptr(q), _ptr(k), _ptr(v), C.byref(cfg),
                                           ha.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(out), _stream()))
        return out

    def forward_tokens(self, q, k, v, head_alloc, out, wq=None, wk=None, eps=1e-6, rotary=None, positions=None, cfg=None):
        """freqattn_forward_tokens: q, k, v [batch, N, heads, head_dim] with adjacent channels (views of a fused projection, say), out as in
        forward; eps None: no norms."""
        who = "forward_tokens"
        self._check_tensors(who, out=out)
        s = self.shape
        want = (s.batch, s.T * s.H * s.W, s.heads, s.head_dim)
        hq, hk, hv = (_heads(who, name, x, out, want) for name, x in (("q", q), ("k", k), ("v", v)))
        wq, wk = (_vector(who, name, x, out, s.head_dim, out.dtype) for name, x in (("wq", wq), ("wk", wk)))
        ha = np.ascontiguousarray(head_alloc, dtype=np.int32)
        if ha.shape != (s.heads,):
            raise ValueError(f"{who}: head_alloc must hold {s.heads} entries, got shape {ha.shape}")
        if rotary is not None and isinstance(rotary, Rotary) and rotary.head_dim != s.head_dim:
            raise ValueError(f"{who}: head_dim {s.head_dim}, the rotary was made for {rotary.head_dim}")
        rot, at, stride = _positions(who, rotary, positions, want[0], want[1], out)
        self._check(lib().freqattn_forward_tokens(self._h, hq, hk, hv, wq, wk, -1.0 if eps is None else float(eps), rot, at, stride,
                                                  C.byref(cfg or self.cfg), ha.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(out), _stream()))
        return out

    def forward_projected(self, x, wq, wk, wv, wo, head_alloc, out, cfg=None):
        import torch
        s = self.shape
        hd = s.heads * s.head_dim
        if not isinstance(x, torch.Tensor) or x.dim() != 3:
            raise ValueError("forward_projected: x must be a [batch, N, d_model] tensor")
        d_model = int(x.shape[2])
        want = {"x": (s.batch, s.T * s.H * s.W, d_model), "out": (s.batch, s.T * s.H * s.W, d_model),
                "wq": (d_model, hd), "wk": (d_model, hd), "wv": (d_model, hd), "wo": (hd, d_model)}
        for name, t in (("x", x), ("out", out), ("wq", wq), ("wk", wk), ("wv", wv), ("wo", wo)):
            if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.bfloat16 or not t.is_contiguous() \
                    or tuple(t.shape) != want[name]:
                raise ValueError(f"forward_projected: {name} must be a contiguous bf16 device tensor of shape {want[name]}")
        ha = np.ascontiguousarray(head_alloc, dtype=np.int32)
        if ha.shape != (s.heads,):
            raise ValueError(f"forward_projected: head_alloc must hold {s.heads} entries")
        cfg = cfg or self.cfg
        self._check(lib().freqattn_forward_projected(self._h, _ptr(x), d_model, _ptr(wq), _ptr(wk), _ptr(wv), _ptr(wo),
                                                     C.byref(cfg), ha.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(out),
                                                     _stream()))
        return out

    def forward_static(self, q, k, v, head_alloc, out, cfg=None):
        self._check_tensors("forward_static", q=q, k=k, v=v, out=out)
        ha = np.ascontiguousarray(head_alloc, dtype=np.int32)
        if ha.shape != (self.shape.heads,):
            raise ValueError(f"forward_static: head_alloc must hold {self.shape.heads} entries, got shape {ha.shape}")
        cfg = cfg or self.cfg
        self._check(lib().freqattn_forward_static(self._h, _ptr(q), _ptr(k), _ptr(v), C.byref(cfg),
                                                  ha.ctypes.data_as(C.POINTER(C.c_int32)), _ptr(out), _stream()))
        return out

    @staticmethod
    def _router_weights(who, w1, b1, w2, b2):
        f = lambda a: np.ascontiguousarray(a, dtype=np.float32)
        w1, b1, w2, b2 = f(w1), f(b1), f(w2), f(b2)
        hidden = int(w1.shape[1]) if w1.ndim == 2 else -1
        if w1.shape != (256, hidden) or b1.shape != (hidden,) or w2.shape != (hidden, 3) or b2.shape != (3,) or hidden < 1:
            raise ValueError(f"{who}: router weights must be w1 [256, hidden], b1 [hidden], w2 [hidden, 3], b2 [3]")
        return hidden, w1, b1, w2, b2

    def forward_routed(self, q, k, v, t, w1, b1, w2, b2, out, cfg=None):
        self._check_tensors("forward_routed", q=q, k=k, v=v, out=out)
        hidden, w1, b1, w2, b2 = self._router_weights("forward_routed", w1, b1, w2, b2)
        alloc = np.zeros(self.shape.heads, np.int32)
        pi = np.zeros(3, np.float32)
        P = lambda a: a.ctypes.data_as(C.POINTER(C.c_float))
        cfg = cfg or self.cfg
        self._check(lib().freqattn_forward_routed(self._h, _ptr(q), _ptr(k), _ptr(v), C.byref(cfg), float(t), hidden,
                                                  P(w1), P(b1), P(w2), P(b2), _ptr(out),
                                                  alloc.ctypes.data_as(C.POINTER(C.c_int32)), P(pi), _stream()))
        return alloc, pi

    def dense_forward(self, q, k, v, out):
        self._check_tensors("dense_forward", q=q, k=k, v=v, out=out)
        self._check(lib().freqattn_dense_forward(self._h, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _stream()))
        return out

    def route_mlp(self, q, k, v, t, w1, b1, w2, b2):
        self._check_tensors("route_mlp", q=q, k=k, v=v)
        hidden, w1, b1, w2, b2 = self._router_weights("route_mlp", w1, b1, w2, b2)
        alloc = np.zeros(self.shape.heads, np.int32)
        pi = np.zeros(3, np.float32)
        stats = np.zeros(192, np.float32)
        P = lambda a: a.ctypes.data_as(C.POINTER(C.c_float))
        self._check(lib().freqattn_route_mlp(self._h, _ptr(q), _ptr(k), _ptr(v), float(t), hidden, P(w1), P(b1), P(w2),
                                             P(b2), alloc.ctypes.data_as(C.POINTER(C.c_int32)), P(pi), P(stats),
                                             _stream()))
        return alloc, pi, stats

    # ---- options and introspection
    def set_launch_mode(self, mode):
        self._check(lib().freqattn_set_launch_mode(self._h, mode))

    def set_exchange_fusion(self, enabled):
        self._check(lib().freqattn_set_exchange_fusion(self._h, 1 if enabled else 0))

    def set_alloc_prediction(self, enabled):
        self._check(lib().freqattn_set_alloc_prediction(self._h, 1 if enabled else 0))

    def get_path(self):
        return lib().freqattn_get_path(self._h)

    def check_range(self):
        """Synchronises; raises FreqAttnError (ERANGE) if a forward since the last check left the fp16 range."""
        flag = C.c_int32(0)
        self._check(lib().freqattn_check_range(self._h, C.byref(flag), _stream()))
        return int(flag.value)

    def workspace_bytes(self):
        return lib().freqattn_workspace_bytes(self._h)

    def measure_peaks(self):
        """(bytes/s of a plain streaming copy, flop/s of an MFMA loop) on this machine; synchronises."""
        cp, mf = C.c_double(0.0), C.c_double(0.0)
        self._check(lib().freqattn_measure_peaks(self._h, C.byref(cp), C.byref(mf), _stream()))
        return cp.value, mf.value

    @property
    def n_bands(self):
        return 4 if self.cfg.mid2_num > 0 else 3

    def band_sizes(self):
        n = (C.c_int64 * 4)()
        self._check(lib().freqattn_band_sizes(self._h, n))
        return [int(x) for x in n][:self.n_bands]

    def band_index(self, band):
        out = np.zeros(self.band_sizes()[band], np.int32)
        self._check(lib().freqattn_band_index(self._h, band, out.ctypes.data_as(C.POINTER(C.c_int32))))
        return out

    def _blocks(self, fn, band):
        nnz = C.c_int64()
        self._check(fn(self._h, None, None, C.byref(nnz)))
        nb = -(-self.band_sizes()[band] // self.cfg.mid_block)
        rp = np.zeros(nb + 1, np.int32)
        ci = np.zeros(nnz.value, np.int32)
        self._check(fn(self._h, rp.ctypes.data_as(C.POINTER(C.c_int32)), ci.ctypes.data_as(C.POINTER(C.c_int32)),
                       C.byref(nnz)))
        return rp, ci

    def mid_blocks(self):
        return self._blocks(lib().freqattn_mid_blocks, 1)

    def mid2_blocks(self):
        if self.n_bands < 4:
            return np.zeros(1, np.int32), np.zeros(0, np.int32)
        return self._blocks(lib().freqattn_mid2_blocks, 3)

    def get_v_box(self):
        return int(lib().freqattn_get_v_box(self._h))

    def summary_weights(self, band):
        m = min(self.cfg.n_summary, int(self.band_sizes()[band]))
        n = self.shape.T * self.shape.H * self.shape.W
        out = np.zeros((m, n), np.float32)
        self._check(lib().freqattn_summary_weights(self._h, band, out.ctypes.data_as(C.POINTER(C.c_float))))
        return out

    def dct_matrix(self, axis):
        n = (self.shape.T, self.shape.H, self.shape.W)[axis]
        out = np.zeros((n, n), np.float64)
        self._check(lib().freqattn_dct_matrix(self._h, axis, out.ctypes.data_as(C.POINTER(C.c_double))))
        return out

    def read_spectral(self, which, slice_, band):
        out = np.zeros((self.band_sizes()[band], self.shape.head_dim), np.float32)
        self._check(lib().freqattn_read_spectral(self._h, which, slice_, band, out.ctypes.data_as(C.POINTER(C.c_float)),
                                                 _stream()))
        return out

    def set_stage_timing(self, enabled):
        self._check(lib().freqattn_set_stage_timing(self._h, int(enabled)))

    def stage_times(self):
        names = (C.c_char_p * 16)()
        ms = (C.c_float * 16)()
        n = C.c_int32()
        self._check(lib().freqattn_stage_times(self._h, 16, names, ms, C.byref(n)))
        return [(names[i].decode(), float(ms[i])) for i in range(n.value)]


def load_balance(pi_heads, lam):
    p = np.ascontiguousarray(pi_heads, dtype=np.float32)
    if p.ndim != 2 or p.shape[1] != 3:
        raise ValueError("load_balance: pi_heads must be [heads, 3]")
    out = C.c_float(0.0)
    st = lib().freqattn_load_balance(p.ctypes.data_as(C.POINTER(C.c_float)), p.shape[0], float(lam), C.byref(out))
    if st != OK:
        raise FreqAttnError(st, "freqattn_load_balance: bad arguments")
    return float(out.value)


def route_fixed(heads, n_low, n_mid, n_high):
    out = np.zeros(heads, np.int32)
    st = lib().freqattn_route_fixed(heads, n_low, n_mid, n_high, out.ctypes.data_as(C.POINTER(C.c_int32)))
    if st != OK:
        raise FreqAttnError(st, "freqattn_route_fixed: bad arguments")
    return out


# ---- operators next to the layer: rotary positions, norms of Q and K, attention over sequences ---------------------------
# They need no context.  A tensor of heads is [batch, rows, heads, head_dim] (packed sequences: [rows, heads, head_dim]) with adjacent
# channels and any other strides: a head-major tensor is passed as x.transpose(1, 2), a part of a fused projection as the slice that it is.

_Tensor = None     # torch.Tensor and the two I/O types, once torch is there (these calls are short: what they look up counts)


def _torch_names():
    global _Tensor, _BF16, _F32, _INT32, _INT8, _CODES, _BYTE, _device, _raw_stream
    import torch
    _BF16, _F32, _INT32, _INT8, _BYTE = torch.bfloat16, torch.float32, torch.int32, torch.int8, torch.uint8
    _CODES = (torch.float8_e4m3fn, torch.uint8)
    _device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
    _Tensor = torch.Tensor


def _count(who, name, n):
    """The library counts in int32."""
    if n > 0x7fffffff:
        raise ValueError(f"{who}: {name} has an axis of 2^31 entries or more")


def _heads(who, name, t, like=None, shape=None, written=False):
    """The freqattn_heads of a tensor, after the checks that the library cannot make on an address."""
    if _Tensor is None:
        _torch_names()
    if not isinstance(t, _Tensor):
        raise TypeError(f"{who}: {name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{who}: {name} must be a device tensor")
    sh, st, dtype = t.shape, t.stride(), t.dtype
    dim = len(st)
    if dim != 3 and dim != 4:
        raise ValueError(f"{who}: {name} must be [batch, rows, heads, head_dim] or [rows, heads, head_dim], got {tuple(sh)}")
    if like is None:
        if dtype is not _BF16 and dtype is not _F32:
            raise ValueError(f"{who}: {name} has dtype {dtype}, expected bfloat16 or float32")
    elif dtype is not like.dtype:
        raise ValueError(f"{who}: {name} has dtype {dtype}, expected {like.dtype}")
    elif t.device != like.device:
        raise ValueError(f"{who}: {name} is on {t.device}, expected {like.device}")
    if shape is None:
        _count(who, name, max(sh))
    elif sh != shape:
        raise ValueError(f"{who}: {name} has shape {tuple(sh)}, expected {tuple(shape)}")
    if st[-1] != 1 and sh[-1] > 1:
        raise ValueError(f"{who}: the channels of {name} must be adjacent")
    if written and 0 in st and any(s == 0 and n > 1 for s, n in zip(st, sh)):
        raise ValueError(f"{who}: {name} is written and must not be expanded")
    return Heads(t.data_ptr(), st[0] if dim == 4 else 0, st[-3], st[-2])


def _int32(who, name, t, like, *shapes):
    """Address of a contiguous int32 device tensor of one of the shapes; None passes."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or t.dtype is not _INT32 or t.device != like.device or not t.is_contiguous() or t.shape not in shapes:
        raise ValueError(f"{who}: {name} must be a contiguous int32 tensor on {like.device} of shape {' or '.join(map(str, shapes))}")
    return t.data_ptr()


def _vector(who, name, t, like, n, dtype):
    if t is None:
        return None
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.device != like.device or not t.is_contiguous() or t.shape != (n,):
        raise ValueError(f"{who}: {name} must be a contiguous {dtype} tensor of shape {(n,)} on {like.device}")
    return t.data_ptr()


def _call(fn, t, *args):
    """fn(*args, stream) on the device of t, with its current stream; raises on failure."""
    index = t.get_device()
    if index == _device():
        st = fn(*args, _raw_stream(index))
    else:
        import torch
        with torch.cuda.device(index):
            st = fn(*args, _raw_stream(index))
    if st != OK:
        raise FreqAttnError(st, lib().freqattn_last_error(None).decode())


def _workspace(who, t, need, like):
    """Address and size of the caller's workspace, or of one from torch's allocator (on the stream that the call uses)."""
    if need == 0:
        return None, 0, None
    if t is None:
        import torch
        t = torch.empty(need, dtype=torch.uint8, device=like.device)
    elif not isinstance(t, _Tensor) or t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{who}: workspace must be a contiguous tensor on {like.device}")
    return t.data_ptr(), t.numel() * t.element_size(), t


def _io(t):
    return BF16 if t.dtype is _BF16 else F32


class Rotary:
    """Rotary positions (freqattn_rotary): `axis_dims` channels rotate per position axis, the rest of head_dim stays."""

    def __init__(self, head_dim, axis_dims, layout=ROTARY_HALF, base=10000.0, scaling=ROTARY_PLAIN, factor=1.0, context=0, grid=None,
                 beta_fast=32.0, beta_slow=1.0, amplitude=0.0):
        axis_dims = [int(x) for x in (axis_dims if hasattr(axis_dims, "__len__") else [axis_dims])]
        self._h = C.c_void_p()
        if not 1 <= len(axis_dims) <= 4 or (grid is not None and len(grid) != len(axis_dims)):
            raise ValueError("Rotary: 1 to 4 axes, and one grid extent for each")
        self.head_dim, self.axes, self.pairs = int(head_dim), len(axis_dims), sum(axis_dims) // 2
        cfg = RotaryCfg(head_dim, self.axes, (C.c_int32 * 4)(*axis_dims), layout, scaling, context, (C.c_int32 * 4)(*(grid or ())), base, factor,
                        beta_fast, beta_slow, amplitude)
        st = lib().freqattn_rotary_create(C.byref(cfg), C.byref(self._h))
        if st != OK:
            raise FreqAttnError(st, lib().freqattn_last_error(None).decode())

    def frequencies(self):
        """(radians per position of every pair, amplitude)."""
        out, amp = np.zeros(self.pairs, np.float64), C.c_double(0.0)
        st = lib().freqattn_rotary_frequencies(self._h, out.ctypes.data_as(C.POINTER(C.c_double)), C.byref(amp))
        if st != OK:
            raise FreqAttnError(st, lib().freqattn_last_error(None).decode())
        return out, amp.value

    def __del__(self):
        try:
            if self._h:
                lib().freqattn_rotary_destroy(self._h)
                self._h = C.c_void_p()
        except Exception:
            pass


def _positions(who, rotary, positions, batch, tokens, like):
    """(rotary handle, positions address, batch stride): positions int32 [batch, tokens, axes] or, one list for all, [tokens, axes]; the last axis may
    be left out where there is one."""
    if rotary is None:
        if positions is not None:
            raise ValueError(f"{who}: positions without a rotary")
        return None, None, 0
    if not isinstance(rotary, Rotary):
        raise TypeError(f"{who}: rotary must be a Rotary")
    n = rotary.axes
    each, one = [(batch, tokens, n)], [(tokens, n)]
    if n == 1:
        each.append((batch, tokens))
        one.append((tokens,))
    at = _int32(who, "positions", positions, like, *each, *one)
    return rotary._h, at, tokens * n if at is not None and positions.shape in each else 0


def rotary_apply(rotary, x, out, positions=None, inverse=False):
    """freqattn_rotary_apply: x, out [batch, tokens, heads, head_dim]; out may be x."""
    who = "rotary_apply"
    if not isinstance(rotary, Rotary):
        raise TypeError(f"{who}: rotary must be a Rotary")
    hx = _heads(who, "x", x)
    if x.dim() != 4:
        raise ValueError(f"{who}: x must be [batch, tokens, heads, head_dim]")
    ho = _heads(who, "out", out, x, x.shape, True)
    b, n, h, d = x.shape
    if d != rotary.head_dim:
        raise ValueError(f"{who}: head_dim {d}, the rotary was made for {rotary.head_dim}")
    hr, at, stride = _positions(who, rotary, positions, b, n, x)
    _call(lib().freqattn_rotary_apply, x, hr, _io(x), b, n, h, hx, at, stride, 1 if inverse else 0, ho)
    return out


def _qk_args(who, q, k, wq, wk, eps, rotary, positions):
    hq = _heads(who, "q", q)
    if q.dim() != 4:
        raise ValueError(f"{who}: q must be [batch, tokens, heads, head_dim]")
    b, n, h, d = q.shape
    hk, kh = None, 0
    if k is not None:
        if getattr(k, "dim", lambda: 0)() != 4:
            raise ValueError(f"{who}: k must be [batch, tokens, heads, head_dim]")
        kh = k.shape[2]
        _count(who, "k", kh)
        hk = _heads(who, "k", k, q, q.shape[:2] + (kh, d))
    w = [_vector(who, name, x, q, d, q.dtype) for name, x in (("wq", wq), ("wk", wk))]
    rot = _positions(who, rotary, positions, b, n, q)
    if rotary is not None and d != rotary.head_dim:
        raise ValueError(f"{who}: head_dim {d}, the rotary was made for {rotary.head_dim}")
    return QkShape(b, n, h, kh, d, _io(q), eps), rot, hq, hk, w


def qk_norm(q, k, wq, wk, q_out, k_out, eps=1e-6, rotary=None, positions=None):
    """freqattn_qk_norm: q [batch, tokens, heads, head_dim], k likewise with its own number of heads (or None); weights [head_dim] or None."""
    who = "qk_norm"
    shape, rot, hq, hk, w = _qk_args(who, q, k, wq, wk, eps, rotary, positions)
    oq = _heads(who, "q_out", q_out, q, q.shape, True)
    ok = None if k is None else _heads(who, "k_out", k_out, q, k.shape, True)
    _call(lib().freqattn_qk_norm, q, shape, *rot, hq, hk, *w, oq, ok)
    return q_out, k_out


def qk_norm_backward(q, k, wq, wk, dq_out, dk_out, dq, dk, dwq=None, dwk=None, eps=1e-6, rotary=None, positions=None, workspace=None):
    """freqattn_qk_norm_backward: q, k, wq, wk, rotary, positions as in qk_norm; dwq, dwk fp32 [head_dim] or None."""
    who = "qk_norm_backward"
    shape, rot, hq, hk, w = _qk_args(who, q, k, wq, wk, eps, rotary, positions)
    yq, xq = _heads(who, "dq_out", dq_out, q, q.shape), _heads(who, "dq", dq, q, q.shape, True)
    yk = xk = None
    if k is not None:
        yk, xk = _heads(who, "dk_out", dk_out, q, k.shape), _heads(who, "dk", dk, q, k.shape, True)
    dw = [_vector(who, name, x, q, q.shape[3], _F32) for name, x in (("dwq", dwq), ("dwk", dwk))]
    need = 0 if dwq is None and dwk is None else lib().freqattn_qk_norm_workspace(q.shape[3])
    ws, size, keep = _workspace(who, workspace, need, q)
    _call(lib().freqattn_qk_norm_backward, q, shape, *rot, hq, hk, *w, yq, yk, xq, xk, *dw, ws, size)
    return dq, dk, dwq, dwk


def _sequence_args(who, q, k, v, causal, scale, q_offsets, k_offsets, q_lengths, k_lengths):
    hq, hk = _heads(who, "q", q), _heads(who, "k", k, q)
    hv = _heads(who, "v", v, k, k.shape)
    for name, t, off in (("q", q, q_offsets), ("k", k, k_offsets)):
        if off is not None and not hasattr(off, "numel"):
            raise ValueError(f"{who}: {name}_offsets must be a tensor")
        if t.dim() != (4 if off is None else 3):
            raise ValueError(f"{who}: {name} must be [rows, heads, head_dim] with {name}_offsets, [sequences, rows, heads, head_dim] without")
    n = q.shape[0] if q_offsets is None else q_offsets.numel() - 1
    if (k.shape[0] if k_offsets is None else k_offsets.numel() - 1) != n or n < 0:
        raise ValueError(f"{who}: q and k must have the same number of sequences")
    _count(who, "q_offsets", n)
    if q.shape[-1] != k.shape[-1]:
        raise ValueError(f"{who}: q and k must have the same head_dim")
    rows = SequenceRows(_int32(who, "q_offsets", q_offsets, q, (n + 1,)), _int32(who, "k_offsets", k_offsets, q, (n + 1,)),
                        _int32(who, "q_lengths", q_lengths, q, (n,)), _int32(who, "k_lengths", k_lengths, q, (n,)))
    shape = SequenceShape(n, q.shape[-2], k.shape[-2], q.shape[-1], q.shape[-3], k.shape[-3], _io(q), 1 if causal else 0, scale)
    return shape, rows, hq, hk, hv


def _lse(who, lse, q, q_offsets, heads):
    shape = (heads, q.shape[0] if q_offsets is not None else q.shape[0] * q.shape[1])
    if not isinstance(lse, _Tensor) or lse.dtype is not _F32 or lse.device != q.device or not lse.is_contiguous() or lse.shape != shape:
        raise ValueError(f"{who}: lse must be a contiguous float32 tensor of shape {shape} on {q.device}")
    return lse.data_ptr()


def sequence_attention(q, k, v, out, lse=None, causal=False, scale=0.0, q_offsets=None, k_offsets=None, q_lengths=None, k_lengths=None,
                       workspace=None):
    """freqattn_sequence_attention: q, out [rows, heads, head_dim] with q_offsets (packed sequences) or [sequences, rows, heads, head_dim]; k, v
    likewise with k_offsets and their own number of heads; lse [heads, rows] or [heads, sequences * rows] fp32."""
    who = "sequence_attention"
    shape, rows, hq, hk, hv = _sequence_args(who, q, k, v, causal, scale, q_offsets, k_offsets, q_lengths, k_lengths)
    ho = _heads(who, "out", out, q, q.shape, True)
    at = None if lse is None else _lse(who, lse, q, q_offsets, shape.q_heads)
    ws, size, keep = _workspace(who, workspace, lib().freqattn_sequence_attention_workspace(shape, rows), q)
    _call(lib().freqattn_sequence_attention, q, shape, rows, hq, hk, hv, ho, at, ws, size)
    return out


def sequence_attention_backward(dout, q, k, v, out, lse, dq, dk, dv, causal=False, scale=0.0, q_offsets=None, k_offsets=None, q_lengths=None,
                                k_lengths=None, workspace=None):
    """freqattn_sequence_attention_backward: arguments as in sequence_attention, out and lse as that call left them."""
    who = "sequence_attention_backward"
    shape, rows, hq, hk, hv = _sequence_args(who, q, k, v, causal, scale, q_offsets, k_offsets, q_lengths, k_lengths)
    hg, ho, xq = _heads(who, "dout", dout, q, q.shape), _heads(who, "out", out, q, q.shape), _heads(who, "dq", dq, q, q.shape, True)
    xk, xv = _heads(who, "dk", dk, q, k.shape, True), _heads(who, "dv", dv, q, k.shape, True)
    at = _lse(who, lse, q, q_offsets, shape.q_heads)
    ws, size, keep = _workspace(who, workspace, lib().freqattn_sequence_attention_backward_workspace(shape, rows), q)
    _call(lib().freqattn_sequence_attention_backward, q, shape, rows, hg, hq, hk, hv, ho, at, xq, xk, xv, ws, size)
    return dq, dk, dv


# ---- on token rows: layer norm, products in 8-bit integers, caches held in 8 bits ---------------------------------------
# A tensor of rows is [batch, rows, channels] or [rows, channels] with adjacent channels and any other strides.

def _rows(who, name, t, like=None, shape=None, dtype=None, written=False):
    """The freqattn_rows of a tensor and its sizes as three axes, after the checks that the library cannot make on an address."""
    if _Tensor is None:
        _torch_names()
    if not isinstance(t, _Tensor):
        raise TypeError(f"{who}: {name} must be a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{who}: {name} must be a device tensor")
    sh, st = t.shape, t.stride()
    dim = len(st)
    if dim != 2 and dim != 3:
        raise ValueError(f"{who}: {name} must be [batch, rows, channels] or [rows, channels], got {tuple(sh)}")
    if dtype is not None:
        if t.dtype is not dtype:
            raise ValueError(f"{who}: {name} has dtype {t.dtype}, expected {dtype}")
    elif t.dtype is not _BF16 and t.dtype is not _F32:
        raise ValueError(f"{who}: {name} has dtype {t.dtype}, expected bfloat16 or float32")
    if like is not None and t.device != like.device:
        raise ValueError(f"{who}: {name} is on {t.device}, expected {like.device}")
    if shape is None:
        _count(who, name, max(sh))
    elif sh != shape:
        raise ValueError(f"{who}: {name} has shape {tuple(sh)}, expected {tuple(shape)}")
    if st[-1] != 1 and sh[-1] > 1:
        raise ValueError(f"{who}: the channels of {name} must be adjacent")
    if written and 0 in st and any(s == 0 and n > 1 for s, n in zip(st, sh)):
        raise ValueError(f"{who}: {name} is written and must not be expanded")
    return Rows(t.data_ptr(), st[0] if dim == 3 else 0, st[-2])


def _filled(who, name, t, like, dtype, shape):
    """Address of a contiguous device tensor of the type and shape; None passes."""
    if t is None:
        return None
    if not isinstance(t, _Tensor) or t.dtype is not dtype or t.device != like.device or not t.is_contiguous() or t.shape != shape:
        raise ValueError(f"{who}: {name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {like.device}")
    return t.data_ptr()


def _weights(who, name, t, x, dtype, b, c):
    """Address of weights or their gradients, and whether they are [batch, channels] instead of [channels]; None passes as (None, None)."""
    if t is None:
        return None, None
    each = isinstance(t, _Tensor) and t.dim() == 2 and x.dim() == 3
    return _filled(who, name, t, x, dtype, (b, c) if each else (c,)), each


def _one_form(who, *each):
    """Whether weights are given for every batch entry; they all have to be, or none."""
    e = [x for x in each if x is not None]
    if e and any(x != e[0] for x in e):
        raise ValueError(f"{who}: weights must be all [channels] or all [batch, channels]")
    return 1 if e and e[0] else 0


def _sizes(x):
    sh = x.shape
    return sh if len(sh) == 3 else (1, sh[0], sh[1])


def layer_norm(x, w, b, out, eps=1e-6):
    """freqattn_layer_norm: x, out [batch, rows, channels] or [rows, channels]; w, b [channels] or [batch, channels], or None; out may be x."""
    who = "layer_norm"
    hx = _rows(who, "x", x)
    n, r, c = _sizes(x)
    dtype = x.dtype
    (aw, ew), (ab, eb) = _weights(who, "w", w, x, dtype, n, c), _weights(who, "b", b, x, dtype, n, c)
    each = _one_form(who, ew, eb)
    ho = _rows(who, "out", out, x, x.shape, dtype, True)
    _call(lib().freqattn_layer_norm, x, NormShape(n, r, c, _io(x), each, eps), hx, aw, ab, ho)
    return out


def layer_norm_backward(x, w, dout, dx, dw=None, db=None, eps=1e-6, workspace=None):
    """freqattn_layer_norm_backward: x, w as in layer_norm; dw, db fp32 [channels] or [batch, channels] (as w, where there is one), or None."""
    who = "layer_norm_backward"
    hx = _rows(who, "x", x)
    n, r, c = _sizes(x)
    dtype = x.dtype
    (aw, ew), (adw, edw), (adb, edb) = _weights(who, "w", w, x, dtype, n, c), _weights(who, "dw", dw, x, _F32, n, c), _weights(who, "db", db, x, _F32, n, c)
    shape = NormShape(n, r, c, _io(x), _one_form(who, ew, edw, edb), eps)
    hy, ho = _rows(who, "dout", dout, x, x.shape, dtype), _rows(who, "dx", dx, x, x.shape, dtype, True)
    need = 0 if dw is None and db is None else lib().freqattn_layer_norm_workspace(shape)
    ws, size, keep = _workspace(who, workspace, need, x)
    _call(lib().freqattn_layer_norm_backward, x, shape, hx, aw, hy, ho, adw, adb, ws, size)
    return dx, dw, db


def quantize_rows(x, codes, scales):
    """freqattn_quantize_rows: x [batch, rows, channels] or [rows, channels], codes int8 of its shape, scales fp32 of its shape without the channels."""
    who = "quantize_rows"
    hx = _rows(who, "x", x)
    sh = x.shape
    hc = _rows(who, "codes", codes, x, sh, _INT8, True)
    at = _filled(who, "scales", scales, x, _F32, sh[:-1])
    if at is None:
        raise ValueError(f"{who}: scales must be a tensor")
    _call(lib().freqattn_quantize_rows, x, _io(x), *_sizes(x), hx, hc, at)
    return codes, scales


def _flat(who, name, t):
    """Rows and row stride of a tensor whose leading axes are one axis of rows in memory."""
    sh, st = t.shape, t.stride()
    if len(sh) == 2:
        return sh[0], st[0]
    if sh[0] > 1 and sh[1] > 1 and st[0] != sh[1] * st[1]:
        raise ValueError(f"{who}: the rows of {name} must lie at one stride")
    return sh[0] * sh[1], st[1] if sh[1] > 1 else st[0]


def product_i8(a, a_scales, w, w_scales, out, bias=None):
    """freqattn_product_i8: a int8 [batch, rows, channels] or [rows, channels], w int8 [outputs, channels], a_scales and w_scales fp32 without the channels, out
    bfloat16 or float32 of a's shape with the outputs in place of the channels, bias [outputs] of out's type or None."""
    who = "product_i8"
    if _Tensor is None:
        _torch_names()
    ha, hw = _rows(who, "a", a, None, None, _INT8), _rows(who, "w", w, a, None, _INT8)
    ash, wsh = a.shape, w.shape
    if len(wsh) != 2 or wsh[1] != ash[-1]:
        raise ValueError(f"{who}: w must be [outputs, {ash[-1]}], got {tuple(wsh)}")
    n, lead = wsh[0], ash[:-1]
    ho = _rows(who, "out", out, a, lead + (n,), None, True)
    sa, sw = _filled(who, "a_scales", a_scales, a, _F32, lead), _filled(who, "w_scales", w_scales, a, _F32, (n,))
    if sa is None or sw is None:
        raise ValueError(f"{who}: a_scales and w_scales must be tensors")
    if len(ash) == 2:
        rows, a_stride, out_stride = ash[0], ha.row_stride, ho.row_stride
    else:
        (rows, a_stride), (_, out_stride) = _flat(who, "a", a), _flat(who, "out", out)
        _count(who, "a", rows)
    _call(lib().freqattn_product_i8, a, ProductShape(rows, ash[-1], n, _io(out)), ha.data, a_stride, sa, hw.data, hw.row_stride, sw,
          _filled(who, "bias", bias, a, out.dtype, (n,)), ho.data, out_stride)
    return out


_BLOCKS = (16, 32, 64, 128, 256)


def _cache8(who, cache_k, cache_v, k_scales, v_scales, block):
    """The freqattn_cache8 of a cache's tensors."""
    if _Tensor is None:
        _torch_names()
    at = []
    for name, t in (("cache_k", cache_k), ("cache_v", cache_v)):
        if not isinstance(t, _Tensor):
            raise TypeError(f"{who}: {name} must be a torch tensor")
        if not t.is_cuda:
            raise ValueError(f"{who}: {name} must be a device tensor")
        st = t.stride()
        if t.dtype not in _CODES or len(st) != 4:
            raise ValueError(f"{who}: {name} must be a float8_e4m3fn or uint8 tensor [sequences, rows, heads, head_dim], got {t.dtype} {tuple(t.shape)}")
        if st[3] != 1 and t.shape[3] > 1:
            raise ValueError(f"{who}: the channels of {name} must be adjacent")
        at += (t.data_ptr(), st[0], st[1], st[2])
    sh = cache_k.shape
    if cache_v.shape != sh or cache_v.device != cache_k.device:
        raise ValueError(f"{who}: cache_k and cache_v must have one shape and device")
    _count(who, "cache_k", max(sh))
    if block not in _BLOCKS:
        raise ValueError(f"{who}: block must be 16, 32, 64, 128 or 256")
    scales = (sh[0], -(-sh[1] // block), sh[2])
    at += (_filled(who, "k_scales", k_scales, cache_k, _BYTE, scales), _filled(who, "v_scales", v_scales, cache_k, _BYTE, scales))
    if None in at[8:]:
        raise ValueError(f"{who}: k_scales and v_scales must be tensors")
    return Cache8(*at, block)


def _apart(who, name, t):
    if 0 in t.stride() and any(s == 0 and n > 1 for s, n in zip(t.stride(), t.shape)):
        raise ValueError(f"{who}: {name} is written and must not be expanded")


def cache8_append(k, v, cache_k, cache_v, k_scales, v_scales, block, q_offsets=None, q_lengths=None, k_lengths=None):
    """freqattn_cache8_append: new rows k, v [rows, heads, head_dim] with q_offsets (packed sequences) or [sequences, rows, heads, head_dim] become the last of the
    k_lengths filled rows of cache_k, cache_v [sequences, capacity, heads, head_dim]; k_scales, v_scales uint8 [sequences, blocks of `block` rows, heads]."""
    who = "cache8_append"
    cache = _cache8(who, cache_k, cache_v, k_scales, v_scales, block)
    _apart(who, "cache_k", cache_k)
    _apart(who, "cache_v", cache_v)
    hk = _heads(who, "k", k)
    hv = _heads(who, "v", v, k, k.shape)
    n, rows, heads, d = cache_k.shape
    if k.dim() != (4 if q_offsets is None else 3):
        raise ValueError(f"{who}: k must be [rows, heads, head_dim] with q_offsets, [sequences, rows, heads, head_dim] without")
    if k.device != cache_k.device or k.shape[-2:] != (heads, d) or (q_offsets is None and k.shape[0] != n):
        raise ValueError(f"{who}: k has shape {tuple(k.shape)} on {k.device}, the cache {tuple(cache_k.shape)} on {cache_k.device}")
    at = SequenceRows(_int32(who, "q_offsets", q_offsets, k, (n + 1,)), None, _int32(who, "q_lengths", q_lengths, k, (n,)),
                      _int32(who, "k_lengths", k_lengths, k, (n,)))
    shape = SequenceShape(n, heads, heads, d, k.shape[-3], rows, _io(k), 0, 0.0)
    _call(lib().freqattn_cache8_append, k, shape, at, hk, hv, cache)


def cache8_read(cache_k, cache_v, k_scales, v_scales, block, k, v, k_lengths=None):
    """freqattn_cache8_read: the values of the filled rows into k, v of the cache's shape, bfloat16 or float32."""
    who = "cache8_read"
    cache = _cache8(who, cache_k, cache_v, k_scales, v_scales, block)
    hk = _heads(who, "k", k, None, cache_k.shape, True)
    hv = _heads(who, "v", v, k, cache_k.shape, True)
    if k.device != cache_k.device:
        raise ValueError(f"{who}: k is on {k.device}, expected {cache_k.device}")
    n, rows, heads, d = cache_k.shape
    at = SequenceRows(None, None, None, _int32(who, "k_lengths", k_lengths, k, (n,)))
    _call(lib().freqattn_cache8_read, k, SequenceShape(n, heads, heads, d, 0, rows, _io(k), 0, 0.0), at, cache, hk, hv)
    return k, v


def cache8_attention(q, cache_k, cache_v, k_scales, v_scales, block, out, lse=None, causal=False, scale=0.0, q_offsets=None, q_lengths=None, k_lengths=None,
                     workspace=None):
    """freqattn_cache8_attention: q, out, lse, causal, scale as in sequence_attention, the cache as in cache8_append."""
    who = "cache8_attention"
    cache = _cache8(who, cache_k, cache_v, k_scales, v_scales, block)
    hq = _heads(who, "q", q)
    ho = _heads(who, "out", out, q, q.shape, True)
    n, rows, heads, d = cache_k.shape
    if q.dim() != (4 if q_offsets is None else 3):
        raise ValueError(f"{who}: q must be [rows, heads, head_dim] with q_offsets, [sequences, rows, heads, head_dim] without")
    if q.device != cache_k.device or q.shape[-1] != d or (q_offsets is None and q.shape[0] != n):
        raise ValueError(f"{who}: q has shape {tuple(q.shape)} on {q.device}, the cache {tuple(cache_k.shape)} on {cache_k.device}")
    at = SequenceRows(_int32(who, "q_offsets", q_offsets, q, (n + 1,)), None, _int32(who, "q_lengths", q_lengths, q, (n,)),
                      _int32(who, "k_lengths", k_lengths, q, (n,)))
    shape = SequenceShape(n, q.shape[-2], heads, d, q.shape[-3], rows, _io(q), 1 if causal else 0, scale)
    where = None if lse is None else _lse(who, lse, q, q_offsets, shape.q_heads)
    ws, size, keep = _workspace(who, workspace, lib().freqattn_cache8_attention_workspace(shape, at), q)
    _call(lib().freqattn_cache8_attention, q, shape, at, hq, cache, ho, where, ws, size)
    return out
