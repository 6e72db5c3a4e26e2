"""ctypes binding of libdyllm.so: argument marshalling only.

Every function mirrors one entry point of include/dyllm.h and passes raw
device pointers of torch tensors (torch is used for device memory and streams
only).  There is no fallback: if the HIP library is missing or fails, calls
raise.
"""
from __future__ import annotations

import ctypes as C
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdyllm.so")

F32, BF16 = 0, 1
OK, ERR_INVALID_ARG, ERR_BAD_SHAPE, ERR_UNSUPPORTED, ERR_NO_MEM, ERR_HIP, ERR_CAPACITY = 0, -1, -2, -3, -4, -5, -6

SYMBOLS = [
    "dyllm_workspace_bytes", "dyllm_create", "dyllm_destroy", "dyllm_strerror", "dyllm_last_error",
    "dyllm_poll_status", "dyllm_saliency", "dyllm_compact", "dyllm_compact_static", "dyllm_qkv_refresh",
    "dyllm_partial_attention", "dyllm_salient_ffn", "dyllm_layer_step", "dyllm_layer_step_approx",
    "dyllm_stack_step_approx", "dyllm_merge_lists", "dyllm_step_kind", "dyllm_denoise_step", "dyllm_full_step",
    "dyllm_stack_step", "dyllm_stack_full_step", "dyllm_pack_weight",
    "dyllm_head_norm_rope", "dyllm_head_norm_rope_quant", "dyllm_quant_write", "dyllm_quant_read",
    "dyllm_partial_attention_quant", "dyllm_qkv_refresh_normed", "dyllm_layer_step_quant",
    "dyllm_profile_begin", "dyllm_profile_end", "dyllm_stage_count", "dyllm_stage_name",
]


class DyllmError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("dyllm error %d: %s" % (code, msg))
        self.code = code


class LayerCfg(C.Structure):
    _fields_ = [
        ("hidden", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
        ("head_dim", C.c_int32), ("ffn_dim", C.c_int32), ("max_batch", C.c_int32),
        ("max_seq", C.c_int32), ("max_rows", C.c_int32), ("dtype", C.c_int32),
        ("rms_eps", C.c_float), ("rope_theta", C.c_float),
    ]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in (
        "wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down", "bq", "bk", "bv", "g_attn", "g_ffn")]


class LayerCache(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v", "c", "out", "lse")]


class IndexListC(C.Structure):
    _fields_ = [("idx", C.c_void_p), ("offsets", C.c_void_p), ("cap", C.c_int32)]


class QuantCacheC(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("format", C.c_int32)]


class Schedule(C.Structure):
    _fields_ = [("t_full", C.c_int32), ("full_period", C.c_int32), ("prompt_len", C.c_int32),
                ("approx", C.c_int32), ("tau", C.c_float)]


STEP_DENSE, STEP_FULL, STEP_RESPONSE = 0, 1, 2


_lib = None


def load_library() -> C.CDLL:
    """Loads the built library; raises if it is not there (build it with build.py)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            "%s not found: build it first (python -m paper_2603_08026_amd.build)" % LIB_PATH)
    lib = C.CDLL(LIB_PATH)
    vp, i32, f32 = C.c_void_p, C.c_int32, C.c_float
    P = C.POINTER
    lib.dyllm_workspace_bytes.argtypes = [P(LayerCfg), P(C.c_size_t)]
    lib.dyllm_create.argtypes = [P(LayerCfg), P(vp)]
    lib.dyllm_destroy.argtypes = [vp]
    lib.dyllm_strerror.argtypes = [C.c_int]
    lib.dyllm_strerror.restype = C.c_char_p
    lib.dyllm_last_error.argtypes = [vp]
    lib.dyllm_last_error.restype = C.c_char_p
    lib.dyllm_poll_status.argtypes = [vp, P(i32), vp]
    lib.dyllm_saliency.argtypes = [vp, vp, vp, P(IndexListC), i32, i32, f32, vp, vp, C.c_int, vp]
    lib.dyllm_compact.argtypes = [vp, vp, P(IndexListC), i32, i32, P(IndexListC), vp]
    lib.dyllm_compact_static.argtypes = [vp, P(IndexListC), i32, i32, P(IndexListC), vp, vp]
    lib.dyllm_qkv_refresh.argtypes = [vp, P(LayerWeights), vp, P(IndexListC), i32, i32, P(LayerCache), vp, vp]
    lib.dyllm_partial_attention.argtypes = [vp, vp, vp, vp, P(IndexListC), i32, i32, vp, vp]
    lib.dyllm_salient_ffn.argtypes = [vp, P(LayerWeights), vp, vp, P(IndexListC), i32, i32, vp, vp]
    lib.dyllm_layer_step.argtypes = [vp, P(LayerWeights), P(LayerCache), vp, P(IndexListC), i32, i32, f32,
                                     P(IndexListC), vp, vp]
    lib.dyllm_layer_step_approx.argtypes = [vp, P(LayerWeights), P(LayerCache), vp, P(IndexListC), i32, i32, i32,
                                            f32, i32, P(IndexListC), vp, vp]
    lib.dyllm_stack_step_approx.argtypes = [vp, i32, P(LayerWeights), P(LayerCache), vp, P(IndexListC), i32, i32,
                                            i32, f32, i32, P(IndexListC), vp, vp]
    lib.dyllm_merge_lists.argtypes = [vp, P(IndexListC), P(IndexListC), i32, i32, i32, P(IndexListC), vp]
    lib.dyllm_step_kind.argtypes = [P(Schedule), i32]
    lib.dyllm_denoise_step.argtypes = [vp, P(Schedule), i32, i32, P(LayerWeights), P(LayerCache), vp,
                                       P(IndexListC), P(IndexListC), i32, i32, P(IndexListC), P(IndexListC), vp]
    lib.dyllm_full_step.argtypes = [vp, P(LayerWeights), P(LayerCache), vp, i32, i32, vp]
    lib.dyllm_stack_step.argtypes = [vp, i32, P(LayerWeights), P(LayerCache), vp, P(IndexListC), i32, i32, f32,
                                     P(IndexListC), vp, vp]
    lib.dyllm_stack_full_step.argtypes = [vp, i32, P(LayerWeights), P(LayerCache), vp, i32, i32, vp]
    P_idx, P_q, i64 = P(IndexListC), P(QuantCacheC), C.c_int64
    lib.dyllm_head_norm_rope.argtypes = [vp, vp, i64, vp, vp, P_idx, i32, i32, P(LayerCache), vp, vp]
    lib.dyllm_head_norm_rope_quant.argtypes = [vp, vp, i64, vp, vp, P_idx, i32, i32, P_q, vp, vp]
    lib.dyllm_quant_write.argtypes = [vp, vp, vp, P_idx, i32, i32, P_q, vp]
    lib.dyllm_quant_read.argtypes = [vp, P_q, P_idx, i32, i32, vp, vp, vp]
    lib.dyllm_partial_attention_quant.argtypes = [vp, vp, P_q, vp, P_idx, i32, i32, vp, vp]
    lib.dyllm_qkv_refresh_normed.argtypes = [vp, P(LayerWeights), vp, vp, vp, P_idx, i32, i32, P(LayerCache), P_q, vp, vp]
    lib.dyllm_layer_step_quant.argtypes = [vp, P(LayerWeights), vp, vp, P(LayerCache), P_q, vp, vp, P_idx, i32, i32, f32,
                                           P_idx, vp, vp]
    lib.dyllm_profile_begin.argtypes = [vp, i32]
    lib.dyllm_profile_end.argtypes = [vp, P(f32), P(i32)]
    lib.dyllm_stage_count.argtypes = []
    lib.dyllm_stage_name.argtypes = [C.c_int]
    lib.dyllm_stage_name.restype = C.c_char_p
    for name in SYMBOLS:
        fn = getattr(lib, name)
        if name not in ("dyllm_strerror", "dyllm_last_error", "dyllm_stage_name"):
            fn.restype = C.c_int
    _lib = lib
    return lib


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return C.c_void_p(t.data_ptr())


def _device() -> int:
    return torch.cuda.current_device()


try:  # the handle without a Stream object around it: 0.1 us of a call's 7, the public way 1.1
    from torch._C import _cuda_getCurrentRawStream as _raw_stream
except ImportError:
    def _raw_stream(device: int) -> int:
        """The current stream of a device."""
        return torch.cuda.current_stream(device).cuda_stream


def _stream() -> C.c_void_p:
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


@dataclass
class IndexList:
    """Device-resident token list: idx int32 [cap], offsets int32 [B+1]."""
    idx: torch.Tensor
    offsets: torch.Tensor

    @property
    def cap(self) -> int:
        return int(self.idx.numel())

    def c(self) -> IndexListC:
        assert self.idx.dtype == torch.int32 and self.offsets.dtype == torch.int32
        return IndexListC(self.idx.data_ptr(), self.offsets.data_ptr(), self.cap)

    @staticmethod
    def empty(cap: int, B: int, device="cuda") -> "IndexList":
        return IndexList(torch.zeros(max(cap, 1), dtype=torch.int32, device=device)[:cap],
                         torch.zeros(B + 1, dtype=torch.int32, device=device))


E4M3, INT8 = 0, 1
CODES = {torch.float8_e4m3fn: E4M3, torch.int8: INT8}


def _powers_of_two(s: torch.Tensor) -> bool:
    """Whether an fp32 tensor holds normal powers of two, +0 and NaN alone."""
    bits = s.view(torch.int32)
    whole = ((bits & ~0x7f800000) == 0) & (bits != 0x7f800000)  # neither sign nor fraction, no infinity
    return bool((whole | torch.isnan(s)).all())


class QuantCache:
    """Key/value cache in 8 bits: codes k, v [B, L, Hkv, dh] (torch.float8_e4m3fn or torch.int8), scales [B, Hkv, L] fp32.
    The scales of e4m3 codes have to be powers of two (or 0, or NaN for vectors that hold no number): attention reads the exponent alone of some.
    Those of another kind are refused here, fresh memory that nobody has cleared among them (`empty` makes a cache of zeros).  Looking waits for the
    GPU; it is left out under stream capture, and what is written into the scales later is not looked at."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dtype not in CODES or v.dtype != k.dtype or k.dim() != 4 or v.shape != k.shape:
            raise ValueError("codes are two [B, L, Hkv, dh] tensors of float8_e4m3fn or int8")
        B, L, Hkv, _ = k.shape
        for s in (k_scale, v_scale):
            if s.dtype != torch.float32 or tuple(s.shape) != (B, Hkv, L):
                raise ValueError("scales are fp32 [B, Hkv, L] tensors")
        for t in (v, k_scale, v_scale):
            if t.device != k.device:
                raise ValueError("the cache's tensors are on different devices")
        if CODES[k.dtype] == E4M3 and not (k.is_cuda and torch.cuda.is_current_stream_capturing()):
            if not (_powers_of_two(k_scale) and _powers_of_two(v_scale)):
                raise ValueError("the scales of e4m3 codes have to be powers of two (fresh memory: zeros)")
        self.k, self.v, self.k_scale, self.v_scale, self.format = k, v, k_scale, v_scale, CODES[k.dtype]
        self.shape, self.device = tuple(k.shape), k.get_device()
        self.c = QuantCacheC(_ptr(k), _ptr(v), _ptr(k_scale), _ptr(v_scale), self.format)

    @staticmethod
    def empty(B: int, L: int, Hkv: int, dh: int, codes=torch.float8_e4m3fn, device="cuda") -> "QuantCache":
        """A cache of zeros."""
        c = [torch.zeros(B, L, Hkv, dh, dtype=torch.int8, device=device).view(codes) for _ in range(2)]
        return QuantCache(*c, *(torch.zeros(B, Hkv, L, dtype=torch.float32, device=device) for _ in range(2)))


def make_weights(tensors: dict) -> LayerWeights:
    w = LayerWeights()
    for name, _ in LayerWeights._fields_:
        t = tensors.get(name)
        setattr(w, name, None if t is None else t.data_ptr())
    return w


def make_cache(k, v, c, out, lse=None) -> LayerCache:
    """lse: fp32 [B, L, H] tensor for the log-normaliser cache, or None.  k, v: None where they are held in 8 bits."""
    return LayerCache(*(None if t is None else t.data_ptr() for t in (k, v, c, out, lse)))


def pack_weight(src: torch.Tensor, dst: torch.Tensor) -> None:
    """Row-major bf16 [n_out, n_in] device matrix -> the panel layout bf16 contexts read (dst: same size)."""
    if src.dim() != 2 or src.dtype != torch.bfloat16 or dst.dtype != torch.bfloat16 or dst.numel() != src.numel():
        raise ValueError("pack_weight takes a 2-D bf16 matrix and a bf16 destination of the same size")
    lib = load_library()
    rc = lib.dyllm_pack_weight(_ptr(src), C.c_int32(src.shape[0]), C.c_int32(src.shape[1]), _ptr(dst), _stream())
    if rc:
        raise DyllmError(rc, lib.dyllm_strerror(rc).decode())


COMPACT_STATIC_MAX_ROWS = 1 << 20


def compact_static(flag: torch.Tensor, rows: Optional["IndexList"], B: int, L: int, out: "IndexList",
                   status: Optional[torch.Tensor] = None) -> None:
    """dyllm_compact without a context: no device memory is allocated by the call."""
    lib = load_library()
    r = rows.c() if rows is not None else None
    o = out.c()
    rc = lib.dyllm_compact_static(_ptr(flag), C.byref(r) if r is not None else None, C.c_int32(B), C.c_int32(L),
                                  C.byref(o), _ptr(status), _stream())
    if rc:
        raise DyllmError(rc, lib.dyllm_strerror(rc).decode())


def workspace_bytes(cfg: LayerCfg) -> int:
    n = C.c_size_t(0)
    rc = load_library().dyllm_workspace_bytes(C.byref(cfg), C.byref(n))
    if rc:
        raise DyllmError(rc, load_library().dyllm_strerror(rc).decode())
    return int(n.value)


class Context:
    """Owns a dyllm_ctx (device scratch only)."""

    def __init__(self, cfg: LayerCfg):
        self.lib = load_library()
        self.cfg = cfg
        h = C.c_void_p()
        rc = self.lib.dyllm_create(C.byref(cfg), C.byref(h))
        if rc:
            raise DyllmError(rc, self.lib.dyllm_strerror(rc).decode())
        self.h = h
        self._dtype = torch.float32 if cfg.dtype == F32 else torch.bfloat16
        self._dh, self._dq, self._dkv = cfg.head_dim, cfg.n_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim
        self._width, self._kv_shape = self._dq + 2 * self._dkv, (cfg.n_kv_heads, cfg.head_dim)
        self._dev = torch.cuda.current_device()  # where the scratch memory is

    def close(self):
        if getattr(self, "h", None):
            torch.cuda.synchronize()
            self.lib.dyllm_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int):
        if rc:
            raise DyllmError(rc, self.lib.dyllm_last_error(self.h).decode())

    def poll_status(self) -> int:
        st = C.c_int32(0)
        self._check(self.lib.dyllm_poll_status(self.h, C.byref(st), _stream()))
        return int(st.value)

    def profile_begin(self, max_calls: int):
        self._check(self.lib.dyllm_profile_begin(self.h, max_calls))

    def profile_end(self):
        """Returns ({stage name: mean ms}, calls)."""
        n = self.lib.dyllm_stage_count()
        ms = (C.c_float * n)()
        calls = C.c_int32(0)
        self._check(self.lib.dyllm_profile_end(self.h, ms, C.byref(calls)))
        return {self.lib.dyllm_stage_name(i).decode(): float(ms[i]) for i in range(n)}, int(calls.value)

    def saliency(self, c_new, c_cache, rows: Optional[IndexList], B, L, tau, cos_out, flag_out, commit=False):
        r = rows.c() if rows is not None else None
        self._check(self.lib.dyllm_saliency(self.h, _ptr(c_new), _ptr(c_cache),
                                            C.byref(r) if r is not None else None, B, L, tau,
                                            _ptr(cos_out), _ptr(flag_out), int(commit), _stream()))

    def compact(self, flag, rows: Optional[IndexList], B, L, out: IndexList):
        r = rows.c() if rows is not None else None
        o = out.c()
        self._check(self.lib.dyllm_compact(self.h, _ptr(flag), C.byref(r) if r is not None else None,
                                           B, L, C.byref(o), _stream()))

    def qkv_refresh(self, w: LayerWeights, x, rows: IndexList, B, L, cache: LayerCache, q_sal_out):
        r = rows.c()
        self._check(self.lib.dyllm_qkv_refresh(self.h, C.byref(w), _ptr(x), C.byref(r), B, L,
                                               C.byref(cache), _ptr(q_sal_out), _stream()))

    def partial_attention(self, q_sal, k_cache, v_cache, rows: IndexList, B, L, c_sal_out):
        r = rows.c()
        self._check(self.lib.dyllm_partial_attention(self.h, _ptr(q_sal), _ptr(k_cache), _ptr(v_cache),
                                                     C.byref(r), B, L, _ptr(c_sal_out), _stream()))

    def salient_ffn(self, w: LayerWeights, x, c, rows_out: IndexList, B, L, out_cache):
        r = rows_out.c()
        self._check(self.lib.dyllm_salient_ffn(self.h, C.byref(w), _ptr(x), _ptr(c), C.byref(r), B, L,
                                               _ptr(out_cache), _stream()))

    def layer_step(self, w: LayerWeights, cache: LayerCache, x, idx_in: IndexList, B, L, tau,
                   idx_out: IndexList, cos_out=None):
        i, o = idx_in.c(), idx_out.c()
        self._check(self.lib.dyllm_layer_step(self.h, C.byref(w), C.byref(cache), _ptr(x), C.byref(i),
                                              B, L, tau, C.byref(o), _ptr(cos_out), _stream()))

    def layer_step_approx(self, w: LayerWeights, cache: LayerCache, x, idx_in: IndexList, B, L, tau,
                          idx_out: IndexList, cos_out=None, row_lo=0, cached_norm=False):
        i, o = idx_in.c(), idx_out.c()
        self._check(self.lib.dyllm_layer_step_approx(self.h, C.byref(w), C.byref(cache), _ptr(x), C.byref(i),
                                                     B, L, row_lo, tau, int(cached_norm), C.byref(o),
                                                     _ptr(cos_out), _stream()))

    def stack_step_approx(self, ws, caches, x, idx_in: IndexList, B, L, tau, idx_outs, cos_out=None, row_lo=0,
                          cached_norm=False):
        n = len(ws)
        wa = (LayerWeights * n)(*ws)
        ca = (LayerCache * n)(*caches)
        oa = (IndexListC * n)(*[o.c() for o in idx_outs])
        i = idx_in.c()
        self._check(self.lib.dyllm_stack_step_approx(self.h, n, wa, ca, _ptr(x), C.byref(i), B, L, row_lo, tau,
                                                     int(cached_norm), oa, _ptr(cos_out), _stream()))

    def merge_lists(self, a, b, B, L, pos_lo, out: IndexList):
        """a, b: IndexList or None."""
        ac, bc, oc = (a.c() if a is not None else None), (b.c() if b is not None else None), out.c()
        self._check(self.lib.dyllm_merge_lists(self.h, C.byref(ac) if ac is not None else None,
                                               C.byref(bc) if bc is not None else None, B, L, pos_lo,
                                               C.byref(oc), _stream()))

    def denoise_step(self, sched: Schedule, t, ws, caches, x, decoded, carry, B, L, cand: IndexList, idx_outs):
        """decoded, carry: IndexList or None.  Returns the step kind (STEP_*)."""
        n = len(ws)
        wa = (LayerWeights * n)(*ws)
        ca = (LayerCache * n)(*caches)
        oa = (IndexListC * n)(*[o.c() for o in idx_outs])
        dc, cc, kc = (decoded.c() if decoded is not None else None), (carry.c() if carry is not None else None), cand.c()
        self._check(self.lib.dyllm_denoise_step(self.h, C.byref(sched), t, n, wa, ca, _ptr(x),
                                                C.byref(dc) if dc is not None else None,
                                                C.byref(cc) if cc is not None else None, B, L, C.byref(kc), oa,
                                                _stream()))
        return int(self.lib.dyllm_step_kind(C.byref(sched), t))

    # ---- normalised query and key heads; the cache in 8 bits.  Tensors are checked against the context: type, number of elements, device, no
    # strides (rows of qkv excepted).  LayerWeights and LayerCache are addresses, which the caller answers for.
    # (A call takes the host about as long as a short kernel the GPU, so what it asks of torch is asked once.)

    def _here(self) -> int:
        dev = _device()
        if dev != self._dev:
            raise ValueError("the context is on device %d, the current one is %d" % (self._dev, dev))
        return dev

    def _arg(self, t, numel, what, dev, dtype=None):
        if t.dtype is not (dtype or self._dtype) or t.numel() < numel or not t.is_contiguous():
            raise ValueError("%s: a contiguous %s tensor of at least %d elements is wanted" % (what, dtype or self._dtype, numel))
        if t.get_device() != dev:
            raise ValueError("%s: not on the current device" % what)
        return t.data_ptr()

    def _gain(self, g, what, dev):
        return None if g is None else self._arg(g, self._dh, what, dev)

    def _lens(self, kv_len, B, dev):
        return None if kv_len is None else self._arg(kv_len, B, "kv_len", dev, torch.int32)

    def _rows(self, rows, B, L, dev):
        """(the list's structure or None, rows at most)"""
        if rows is None:
            return None, B * L
        idx, offsets = rows.idx, rows.offsets
        if offsets.numel() < B + 1:
            raise ValueError("rows: %d offsets are wanted" % (B + 1))
        if idx.dtype is not torch.int32 or offsets.dtype is not torch.int32:
            raise ValueError("rows: int32 tensors are wanted")
        if not (idx.is_contiguous() and offsets.is_contiguous()):
            raise ValueError("rows: contiguous tensors are wanted")
        if idx.get_device() != dev or offsets.get_device() != dev:
            raise ValueError("rows: not on the current device")
        n = idx.numel()
        return C.byref(IndexListC(idx.data_ptr(), offsets.data_ptr(), n)), n

    def _quant(self, cache: QuantCache, B, L, dev):
        if cache.shape != (B, L, *self._kv_shape):
            raise ValueError("the 8-bit cache is %s, the call's %s" % (cache.shape, (B, L, *self._kv_shape)))
        if cache.device != dev:
            raise ValueError("the 8-bit cache is not on the current device")
        return C.byref(cache.c)

    def _qkv(self, qkv, n, dev):
        """(pointer, row stride) of raw projections [n, (H + 2 Hkv) dh], whose rows may lie further apart than they are long"""
        shape, width = qkv.shape, self._width
        if len(shape) != 2 or shape[1] != width or shape[0] < n:
            raise ValueError("qkv: [%d, %d] is wanted" % (n, width))
        ld = width
        if not qkv.is_contiguous():
            ld = qkv.stride(0) if shape[0] > 1 else width
            if qkv.stride(1) != 1 or (n > 1 and ld < width):
                raise ValueError("qkv: neighbouring columns and rows that do not overlap are wanted")
        if qkv.dtype is not self._dtype or qkv.get_device() != dev:
            raise ValueError("qkv: of another type or device than the context's")
        return qkv.data_ptr(), ld

    def head_norm_rope(self, qkv, g_q, g_k, rows: Optional[IndexList], B, L, cache: LayerCache, q_out):
        """qkv: [n, (H + 2 Hkv) dh], rows may be strided; g_q, g_k: [dh] or None; rows None: all B*L tokens."""
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        p, ld = self._qkv(qkv, n, dev)
        q = self._arg(q_out, n * self._dq, "q_out", dev)
        self._check(self.lib.dyllm_head_norm_rope(self.h, p, ld, self._gain(g_q, "g_q", dev), self._gain(g_k, "g_k", dev), r, B,
                                                  L, C.byref(cache), q, _raw_stream(dev)))

    def head_norm_rope_quant(self, qkv, g_q, g_k, rows: Optional[IndexList], B, L, cache: QuantCache, q_out):
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        p, ld = self._qkv(qkv, n, dev)
        q = self._arg(q_out, n * self._dq, "q_out", dev)
        self._check(self.lib.dyllm_head_norm_rope_quant(self.h, p, ld, self._gain(g_q, "g_q", dev), self._gain(g_k, "g_k", dev), r,
                                                        B, L, self._quant(cache, B, L, dev), q, _raw_stream(dev)))

    def quant_write(self, k, v, rows: Optional[IndexList], B, L, cache: QuantCache):
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        n *= self._dkv
        self._check(self.lib.dyllm_quant_write(self.h, self._arg(k, n, "k", dev), self._arg(v, n, "v", dev), r, B, L,
                                               self._quant(cache, B, L, dev), _raw_stream(dev)))

    def quant_read(self, cache: QuantCache, rows: Optional[IndexList], B, L, k_out, v_out):
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        n *= self._dkv
        self._check(self.lib.dyllm_quant_read(self.h, self._quant(cache, B, L, dev), r, B, L, self._arg(k_out, n, "k_out", dev),
                                              self._arg(v_out, n, "v_out", dev), _raw_stream(dev)))

    def partial_attention_quant(self, q_sal, cache: QuantCache, rows: Optional[IndexList], B, L, c_sal_out, kv_len=None):
        """kv_len: int32 [B] device tensor (keys of each sequence) or None."""
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        n *= self._dq
        self._check(self.lib.dyllm_partial_attention_quant(
            self.h, self._arg(q_sal, n, "q_sal", dev), self._quant(cache, B, L, dev), self._lens(kv_len, B, dev), r, B, L,
            self._arg(c_sal_out, n, "c_sal_out", dev), _raw_stream(dev)))

    def qkv_refresh_normed(self, w: LayerWeights, g_q, g_k, x, rows: Optional[IndexList], B, L, cache, q_sal_out):
        """cache: LayerCache (storage type) or QuantCache."""
        dev = self._here()
        r, n = self._rows(rows, B, L, dev)
        quant = isinstance(cache, QuantCache)
        self._check(self.lib.dyllm_qkv_refresh_normed(
            self.h, C.byref(w), self._gain(g_q, "g_q", dev), self._gain(g_k, "g_k", dev),
            self._arg(x, B * L * self.cfg.hidden, "x", dev), r, B, L, None if quant else C.byref(cache),
            self._quant(cache, B, L, dev) if quant else None, self._arg(q_sal_out, n * self._dq, "q_sal_out", dev),
            _raw_stream(dev)))

    def layer_step_quant(self, w: LayerWeights, g_q, g_k, cache: LayerCache, quant: QuantCache, x, idx_in: IndexList, B, L,
                         tau, idx_out: IndexList, cos_out=None, kv_len=None):
        """Of cache only c and out are used."""
        dev = self._here()
        i, n = self._rows(idx_in, B, L, dev)
        o, _ = self._rows(idx_out, B, L, dev)
        self._check(self.lib.dyllm_layer_step_quant(
            self.h, C.byref(w), self._gain(g_q, "g_q", dev), self._gain(g_k, "g_k", dev), C.byref(cache),
            self._quant(quant, B, L, dev), self._lens(kv_len, B, dev), self._arg(x, B * L * self.cfg.hidden, "x", dev), i, B, L,
            tau, o, None if cos_out is None else self._arg(cos_out, n, "cos_out", dev, torch.float32), _raw_stream(dev)))

    def full_step(self, w: LayerWeights, cache: LayerCache, x, B, L):
        self._check(self.lib.dyllm_full_step(self.h, C.byref(w), C.byref(cache), _ptr(x), B, L, _stream()))

    def stack_step(self, ws, caches, x, idx_in: IndexList, B, L, tau, idx_outs, cos_out=None):
        """ws / caches / idx_outs: one LayerWeights / LayerCache / IndexList per layer."""
        n = len(ws)
        wa = (LayerWeights * n)(*ws)
        ca = (LayerCache * n)(*caches)
        oa = (IndexListC * n)(*[o.c() for o in idx_outs])
        i = idx_in.c()
        self._check(self.lib.dyllm_stack_step(self.h, n, wa, ca, _ptr(x), C.byref(i), B, L, tau, oa,
                                              _ptr(cos_out), _stream()))

    def stack_full_step(self, ws, caches, x, B, L):
        n = len(ws)
        wa = (LayerWeights * n)(*ws)
        ca = (LayerCache * n)(*caches)
        self._check(self.lib.dyllm_stack_full_step(self.h, n, wa, ca, _ptr(x), B, L, _stream()))
