"""Python binding of libqstate (the C ABI in include/qstate.h).

Argument marshalling only: every step of the hot path runs in the CUDA library.  Tensors are
torch tensors on a CUDA device (torch supplies device memory and streams); the library is
loaded from this package's in-tree build and there is no fallback -- without the compiled
library every call raises.
"""
from __future__ import annotations

import ctypes as ct
import os
from dataclasses import dataclass, field, fields

from . import build as _build

QSTATE_OK, QSTATE_EINVAL, QSTATE_EBUDGET, QSTATE_ECUDA, QSTATE_EDEVICE, QSTATE_ETIMEOUT = range(6)
DECAY_ROW, DECAY_HEAD = 0, 1
ERASE_DELTA, ERASE_NONE, ERASE_GENERAL = 0, 1, 2
ALLOC_LAGGED, ALLOC_CURRENT = 0, 1
FORM_TOKEN, FORM_CHUNK = 0, 1
UNIT_ROW, UNIT_HEAD = 0, 1
# allocation weights (Eq. 3 and the alternatives of Table 1; see include/qstate.h)
(WEIGHT_OURS, WEIGHT_RANGE, WEIGHT_GAMMA_RAW, WEIGHT_NRANGE, WEIGHT_PERSIST, WEIGHT_WBFACTOR,
 WEIGHT_NOERASE, WEIGHT_SHUFFLE, WEIGHT_UNIFORM) = range(9)

# paged cache of attention layers (see include/qstate.h)
KV_HEADS, KV_LATENT = 0, 1
KV_BF16, KV_F16 = 0, 1
KV_16, KV_E4M3 = 0, 1


class QstateError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"qstate error {code}: {msg}")
        self.code = code


class _Cfg(ct.Structure):
    _fields_ = [("B", ct.c_int32), ("H", ct.c_int32), ("dk", ct.c_int32), ("dv", ct.c_int32),
                ("decay_kind", ct.c_int32), ("erase_kind", ct.c_int32),
                ("unit_kind", ct.c_int32), ("group_heads", ct.c_int32),
                ("bbar_num", ct.c_int32), ("bbar_den", ct.c_int32), ("bmin", ct.c_int32),
                ("bmax", ct.c_int32), ("C", ct.c_int32), ("fit_every", ct.c_int32),
                ("ema_span", ct.c_float), ("gate_bits", ct.c_int32),
                ("weight_kind", ct.c_int32), ("alloc_mode", ct.c_int32),
                ("interval_form", ct.c_int32)]


class _Buf(ct.Structure):
    _fields_ = [("payload", ct.c_void_p), ("scales", ct.c_void_p), ("widths", ct.c_void_p),
                ("head_off", ct.c_void_p), ("fidx", ct.c_void_p)]


class _Stats(ct.Structure):
    _fields_ = [("ema_s", ct.c_void_p), ("ema_r", ct.c_void_p), ("range", ct.c_void_p)]


class _Inputs(ct.Structure):
    _fields_ = [("q", ct.c_void_p), ("k", ct.c_void_p), ("v", ct.c_void_p), ("s", ct.c_void_p),
                ("s_code", ct.c_void_p), ("s_lut", ct.c_void_p), ("beta", ct.c_void_p),
                ("T", ct.c_int32), ("a", ct.c_void_p), ("w", ct.c_void_p)]


class _KvCfg(ct.Structure):
    _fields_ = [("kind", ct.c_int32), ("Hq", ct.c_int32), ("Hkv", ct.c_int32), ("dk", ct.c_int32), ("dv", ct.c_int32),
                ("page", ct.c_int32), ("n_pages", ct.c_int32), ("max_pages", ct.c_int32), ("dtype", ct.c_int32),
                ("store", ct.c_int32), ("window", ct.c_int32), ("scale", ct.c_float)]


class _KvCache(ct.Structure):
    _fields_ = [("k", ct.c_void_p), ("v", ct.c_void_p), ("k_exp", ct.c_void_p), ("v_exp", ct.c_void_p)]


class _KvPages(ct.Structure):
    _fields_ = [("table", ct.c_void_p), ("lens", ct.c_void_p), ("lens_out", ct.c_void_p), ("free_list", ct.c_void_p),
                ("free_count", ct.c_void_p), ("free_out", ct.c_void_p)]


class _KvSlots(ct.Structure):
    _fields_ = [("cu", ct.c_void_p), ("slot", ct.c_void_p), ("pos", ct.c_void_p), ("req", ct.c_void_p),
                ("ok", ct.c_void_p), ("T", ct.c_int32)]


class _KvMoves(ct.Structure):
    _fields_ = [("src", ct.c_void_p), ("dst", ct.c_void_p), ("n", ct.c_int32)]


EXPORTS = ["qstate_validate", "qstate_region_bytes", "qstate_units", "qstate_scale_groups",
           "qstate_bits_per_element", "qstate_init", "qstate_alloc_bits", "qstate_pack",
           "qstate_unpack", "qstate_quant_decay", "qstate_quant_decay_noalloc", "qstate_step",
           "qstate_scan", "qstate_scan_host",
           "qstate_scan_fp32", "qstate_check", "qstate_set_wait_limit", "qstate_set_scan_partitions",
           "qstate_scan_partition_count", "qstate_last_error", "qstate_kv_validate", "qstate_kv_cache_bytes",
           "qstate_kv_work_bytes", "qstate_kv_plan", "qstate_kv_append", "qstate_kv_attend",
           "qstate_kv_pages_work_bytes", "qstate_kv_fork", "qstate_kv_compact", "qstate_kv_copy",
           "qstate_kv_group_bytes", "qstate_kv_shared_work_bytes", "qstate_kv_group", "qstate_kv_attend_shared",
           "qstate_set_shared_gain"]

_lib = None


def library_path() -> str:
    return _build.LIB


def load(path: str | None = None, build_if_missing: bool = False):
    """Load libqstate.so (build it first if asked).  Raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    path = path or _build.LIB
    if not os.path.exists(path):
        if not build_if_missing:
            raise QstateError(QSTATE_ECUDA, f"CUDA library not built: {path} (run build())")
        _build.build()
    L = ct.CDLL(path)
    P, PC = ct.c_void_p, ct.POINTER(_Cfg)
    L.qstate_validate.argtypes = [PC]
    L.qstate_region_bytes.argtypes = [PC]
    L.qstate_region_bytes.restype = ct.c_size_t
    L.qstate_units.argtypes = [PC]
    L.qstate_units.restype = ct.c_size_t
    L.qstate_scale_groups.argtypes = [PC]
    L.qstate_scale_groups.restype = ct.c_size_t
    L.qstate_bits_per_element.argtypes = [PC]
    L.qstate_bits_per_element.restype = ct.c_double
    L.qstate_init.argtypes = [PC, ct.POINTER(_Buf), ct.POINTER(_Buf), P]
    L.qstate_alloc_bits.argtypes = [PC, ct.POINTER(_Stats), P, P, P]
    L.qstate_pack.argtypes = [PC, P, ct.POINTER(_Buf), P, P]
    L.qstate_unpack.argtypes = [PC, ct.POINTER(_Buf), P, P]
    L.qstate_quant_decay.argtypes = [PC, P, ct.c_int32, P, P, P, P]
    L.qstate_quant_decay_noalloc.argtypes = [PC, P, ct.c_int32, P, P, P]
    L.qstate_step.argtypes = [PC, ct.POINTER(_Buf), ct.POINTER(_Buf), ct.POINTER(_Inputs),
                              ct.c_int32, ct.c_int32, ct.c_int32, P, ct.POINTER(_Stats), P]
    L.qstate_scan.argtypes = [PC, ct.POINTER(_Buf), ct.POINTER(_Buf), ct.POINTER(_Inputs),
                              ct.c_int32, ct.c_int32, ct.c_int32, P, ct.POINTER(_Stats),
                              ct.POINTER(ct.c_int32), P]
    L.qstate_scan_host.argtypes = [PC, ct.POINTER(_Buf), ct.POINTER(_Buf), ct.POINTER(_Inputs),
                                   ct.POINTER(_Inputs), ct.c_int32, ct.c_int32, ct.c_int32, P, P,
                                   ct.POINTER(_Stats), ct.c_int32, ct.POINTER(ct.c_int32), P, P]
    L.qstate_scan_fp32.argtypes = [PC, P, ct.POINTER(_Inputs), ct.c_int32, ct.c_int32, P, P]
    L.qstate_check.argtypes = [P]
    L.qstate_set_wait_limit.argtypes = [ct.c_int32]
    L.qstate_set_scan_partitions.argtypes = [ct.c_int32]
    L.qstate_scan_partition_count.argtypes = [ct.c_void_p, ct.c_void_p, ct.c_void_p]
    L.qstate_last_error.restype = ct.c_char_p
    KC, I32, I64 = ct.POINTER(_KvCfg), ct.c_int32, ct.c_int64
    L.qstate_kv_validate.argtypes = [KC]
    L.qstate_kv_cache_bytes.argtypes = [KC, I32]
    L.qstate_kv_cache_bytes.restype = ct.c_size_t
    L.qstate_kv_work_bytes.argtypes = [KC]
    L.qstate_kv_work_bytes.restype = ct.c_size_t
    L.qstate_kv_plan.argtypes = [P, P, P, I32, P, P, P]
    L.qstate_kv_append.argtypes = [P, P, P, I64, I64, P, I64, I64, P, I32, P]
    L.qstate_kv_attend.argtypes = [P, P, P, I64, I64, P, P, I32, P, P, P, P]
    for name in ("qstate_kv_pages_work_bytes", "qstate_kv_group_bytes", "qstate_kv_shared_work_bytes"):
        getattr(L, name).argtypes = [KC, I32]
        getattr(L, name).restype = ct.c_size_t
    L.qstate_kv_fork.argtypes = [P, P, P, P, P, I32, P, P, P, P]
    L.qstate_kv_compact.argtypes = [P, P, P, I32, I32, P, P, P, P, P]
    L.qstate_kv_copy.argtypes = [P, P, P, P]
    L.qstate_set_shared_gain.argtypes = [I32]
    L.qstate_kv_group.argtypes = [P, P, I32, P, P, I32, P, P]
    L.qstate_kv_attend_shared.argtypes = [P, P, P, I64, I64, P, P, I32, P, P, P, P, P]
    for name in EXPORTS:
        if name not in ("qstate_region_bytes", "qstate_units", "qstate_scale_groups",
                        "qstate_bits_per_element", "qstate_last_error", "qstate_kv_cache_bytes",
                        "qstate_kv_work_bytes", "qstate_kv_pages_work_bytes", "qstate_kv_group_bytes",
                        "qstate_kv_shared_work_bytes"):
            getattr(L, name).restype = ct.c_int
    _lib = L
    return L


def _lib_or_raise():
    return _lib if _lib is not None else load()


def _check(rc: int):
    if rc != QSTATE_OK:
        raise QstateError(rc, _lib_or_raise().qstate_last_error().decode())


# A decode loop calls once per token and layer with some twenty tensors, so marshalling is kept
# short: pointers and streams are plain integers (ctypes takes them for void pointers), structures
# are filled field by field, and the current stream comes as a handle without a Stream object
# (one step of 32 heads: 24 us of host time, 34 us without).
def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("tensor must live on a CUDA device")
    if not t.is_contiguous():
        raise ValueError("tensor must be contiguous")
    return t.data_ptr()


_raw_stream = None


def _current_stream():
    """Handle of torch's current stream on the current device."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        torch.cuda.init()
        get, dev = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
        _raw_stream = ((lambda: get(dev())) if get and dev else
                       (lambda: torch.cuda.current_stream().cuda_stream))
    return _raw_stream()


def _stream(stream):
    return stream.cuda_stream if stream is not None else _current_stream()


@dataclass
class Config:
    """Method configuration (mirrors ``qstate_cfg``)."""
    B: int
    H: int
    dk: int
    dv: int
    decay_kind: int = DECAY_ROW
    erase_kind: int = ERASE_DELTA
    unit_kind: int = UNIT_ROW
    group_heads: int = 1
    bbar_num: int = 4
    bbar_den: int = 1
    bmin: int = 1
    bmax: int = 8
    C: int = 1
    fit_every: int = 1
    ema_span: float = 64.0
    gate_bits: int = 0
    weight_kind: int = 0
    alloc_mode: int = 0
    interval_form: int = 0

    def c(self) -> _Cfg:
        return _Cfg(self.B, self.H, self.dk, self.dv, self.decay_kind, self.erase_kind, self.unit_kind,
                    self.group_heads, self.bbar_num, self.bbar_den, self.bmin, self.bmax, self.C,
                    self.fit_every, self.ema_span, self.gate_bits, self.weight_kind, self.alloc_mode,
                    self.interval_form)

    @classmethod
    def from_workload(cls, w, **over) -> "Config":
        kw = dict(B=w.B, H=w.H, dk=w.dk, dv=w.dv,
                  decay_kind=DECAY_ROW if w.per_row_decay else DECAY_HEAD,
                  erase_kind=(ERASE_GENERAL if getattr(w, "general", False)
                            else ERASE_DELTA if w.erase else ERASE_NONE),
                  unit_kind=UNIT_ROW if w.unit == "row" else UNIT_HEAD,
                  group_heads=w.group_heads, bbar_num=w.bbar, bbar_den=1, bmin=w.bmin,
                  bmax=w.bmax, C=w.C, gate_bits=w.gate_bits)
        kw.update(over)
        return cls(**kw)

    @property
    def units(self) -> int:
        return self.H * self.dk if self.unit_kind == UNIT_ROW else self.H

    @property
    def scale_groups(self) -> int:
        return self.H * self.dk if self.unit_kind == UNIT_ROW else self.H * (self.dk // 32) * self.dv


def validate(cfg: Config) -> None:
    c = cfg.c()
    _check(_lib_or_raise().qstate_validate(ct.byref(c)))


def region_bytes(cfg: Config) -> int:
    validate(cfg)
    c = cfg.c()
    return int(_lib_or_raise().qstate_region_bytes(ct.byref(c)))


def bits_per_element(cfg: Config) -> float:
    validate(cfg)
    c = cfg.c()
    return float(_lib_or_raise().qstate_bits_per_element(ct.byref(c)))


@dataclass
class State:
    """One packed state (device tensors, caller-owned)."""
    payload: object
    scales: object
    widths: object
    head_off: object
    fidx: object

    def c(self) -> _Buf:
        return _Buf(_ptr(self.payload), _ptr(self.scales), _ptr(self.widths), _ptr(self.head_off), _ptr(self.fidx))


def new_state(cfg: Config, device="cuda") -> State:
    import torch
    rb = region_bytes(cfg)
    return State(torch.zeros(cfg.B * rb, dtype=torch.uint8, device=device),
                 torch.zeros(cfg.B * cfg.scale_groups, dtype=torch.int16, device=device),
                 torch.zeros(cfg.B * cfg.units, dtype=torch.uint8, device=device),
                 torch.zeros(cfg.B * cfg.H, dtype=torch.int32, device=device),
                 torch.full((cfg.B * cfg.scale_groups,), 15, dtype=torch.uint8, device=device))


@dataclass
class Stats:
    ema_s: object
    ema_r: object
    range: object

    def c(self) -> _Stats:
        return _Stats(_ptr(self.ema_s), _ptr(self.ema_r), _ptr(self.range))


def new_stats(cfg: Config, device="cuda") -> Stats:
    import torch
    n = cfg.B * cfg.units
    return Stats(*(torch.zeros(n, dtype=torch.float32, device=device) for _ in range(3)))


@dataclass
class Inputs:
    q: object
    k: object
    v: object
    s: object = None
    s_code: object = None
    s_lut: object = None
    beta: object = None
    T: int = field(default=0)
    a: object = None
    w: object = None

    def c(self) -> _Inputs:
        T = self.T or int(self.q.shape[1])
        return _Inputs(_ptr(self.q), _ptr(self.k), _ptr(self.v), _ptr(self.s), _ptr(self.s_code),
                       _ptr(self.s_lut), _ptr(self.beta), T, _ptr(self.a), _ptr(self.w))


def qstate_init(cfg: Config, a: State, b: State, stream=None) -> None:
    c, ba, bb = cfg.c(), a.c(), b.c()
    _check(_lib_or_raise().qstate_init(ct.byref(c), ct.byref(ba), ct.byref(bb), _stream(stream)))


def qstate_alloc_bits(cfg: Config, stats: Stats, widths_out, head_off_out, stream=None) -> None:
    c, st = cfg.c(), stats.c()
    _check(_lib_or_raise().qstate_alloc_bits(ct.byref(c), ct.byref(st), _ptr(widths_out),
                                             _ptr(head_off_out), _stream(stream)))


def qstate_pack(cfg: Config, S, out: State, range_out=None, stream=None) -> None:
    c, bo = cfg.c(), out.c()
    _check(_lib_or_raise().qstate_pack(ct.byref(c), _ptr(S), ct.byref(bo), _ptr(range_out),
                                       _stream(stream)))


def qstate_unpack(cfg: Config, src: State, S_out, stream=None) -> None:
    c, bi = cfg.c(), src.c()
    _check(_lib_or_raise().qstate_unpack(ct.byref(c), ct.byref(bi), _ptr(S_out), _stream(stream)))


def qstate_quant_decay(cfg: Config, s, code_out, lut_out, thr_out, stream=None) -> None:
    c = cfg.c()
    _check(_lib_or_raise().qstate_quant_decay(ct.byref(c), _ptr(s), int(s.shape[1]), _ptr(code_out),
                                              _ptr(lut_out), _ptr(thr_out), _stream(stream)))


def qstate_quant_decay_noalloc(cfg: Config, s, code_out, lut_out, stream=None) -> None:
    """qstate_quant_decay without a threshold buffer (see include/qstate.h)."""
    c = cfg.c()
    _check(_lib_or_raise().qstate_quant_decay_noalloc(ct.byref(c), _ptr(s), int(s.shape[1]),
                                                      _ptr(code_out), _ptr(lut_out),
                                                      _stream(stream)))


def qstate_step(cfg: Config, src: State, dst: State, x: Inputs, t_begin: int, t_end: int,
                w_index: int, o, stats: Stats, stream=None) -> None:
    c, bi, bo, xi, st = cfg.c(), src.c(), dst.c(), x.c(), stats.c()
    _check(_lib_or_raise().qstate_step(ct.byref(c), ct.byref(bi), ct.byref(bo), ct.byref(xi),
                                       t_begin, t_end, w_index, _ptr(o), ct.byref(st),
                                       _stream(stream)))


def qstate_scan(cfg: Config, ping: State, pong: State, x: Inputs, t_begin: int, t_end: int,
                w_index0: int, o, stats: Stats, stream=None) -> bool:
    """Returns True if the final state is in ``pong``."""
    c, bi, bo, xi, st = cfg.c(), ping.c(), pong.c(), x.c(), stats.c()
    flag = ct.c_int32(0)
    _check(_lib_or_raise().qstate_scan(ct.byref(c), ct.byref(bi), ct.byref(bo), ct.byref(xi),
                                       t_begin, t_end, w_index0, _ptr(o), ct.byref(st),
                                       ct.byref(flag), _stream(stream)))
    return bool(flag.value)


def _hptr(t):
    """Pointer of a host (CPU) tensor; pinned memory keeps the copies asynchronous."""
    if t is None:
        return None
    if t.is_cuda or not t.is_contiguous():
        raise ValueError("host tensor must be a contiguous CPU tensor")
    return t.data_ptr()


def qstate_scan_host(cfg: Config, ping: State, pong: State, x_host: Inputs, x_dev: Inputs,
                     t_begin: int, t_end: int, w_index0: int, o_host, o_dev, stats: Stats,
                     chunk: int, stream, copy_stream) -> bool:
    """qstate_scan with inputs staged from host tensors chunk by chunk (see include/qstate.h).
    Returns True if the final state is in ``pong``."""
    c, bi, bo, st = cfg.c(), ping.c(), pong.c(), stats.c()
    xh = _Inputs(*(_hptr(getattr(x_host, n)) for n in ("q", "k", "v", "s", "s_code", "s_lut", "beta")),
                 x_host.T or int(x_host.q.shape[1]), _hptr(x_host.a), _hptr(x_host.w))
    xd = x_dev.c()
    flag = ct.c_int32(0)
    _check(_lib_or_raise().qstate_scan_host(ct.byref(c), ct.byref(bi), ct.byref(bo), ct.byref(xh),
                                            ct.byref(xd), t_begin, t_end, w_index0, _hptr(o_host),
                                            _ptr(o_dev), ct.byref(st), chunk, ct.byref(flag),
                                            stream.cuda_stream, copy_stream.cuda_stream))
    return bool(flag.value)


def qstate_scan_fp32(cfg: Config, S, x: Inputs, t_begin: int, t_end: int, o, stream=None) -> None:
    c, xi = cfg.c(), x.c()
    _check(_lib_or_raise().qstate_scan_fp32(ct.byref(c), _ptr(S), ct.byref(xi), t_begin, t_end,
                                            _ptr(o), _stream(stream)))


def qstate_check(stream=None) -> None:
    _check(_lib_or_raise().qstate_check(_stream(stream)))


def qstate_set_wait_limit(polls: int) -> None:
    """Limit of the chunked form's waits for its tensor-core products in later calls (polls;
    0 gives up at once, negative restores the default)."""
    _check(_lib_or_raise().qstate_set_wait_limit(int(polls)))


def qstate_set_scan_partitions(n: int) -> None:
    """Batch partitions of later scans, each on its own stream (1..8; 0 chooses per
    configuration).  Results are identical for every choice."""
    _check(_lib_or_raise().qstate_set_scan_partitions(int(n)))


def qstate_scan_partition_count(cfg: Config, x: Inputs, stats: Stats) -> int:
    """Batch partitions a scan with these arguments would use now (0 if they are invalid)."""
    c, xi, st = cfg.c(), x.c(), stats.c()
    return int(_lib_or_raise().qstate_scan_partition_count(ct.byref(c), ct.byref(xi), ct.byref(st)))


# ---- paged cache of attention layers -------------------------------------------------------------
# Descriptions and tensors of these calls stay the same from step to step, so their structures are made
# once, with the frozen object that holds them.
class _Kept:
    """Copies (copy, deepcopy, pickle) are made again from the fields, so that their addresses are their own."""

    def __reduce__(self):
        return type(self), tuple(getattr(self, f.name) for f in fields(self))


def _keep(obj, struct=None, **more):
    """Keeps a structure, its address and whatever else belongs to a frozen object."""
    if struct is not None:
        more.update(_c=struct, _at=ct.addressof(struct))
    for name, value in more.items():
        object.__setattr__(obj, name, value)


@dataclass(frozen=True)
class KvConfig(_Kept):
    """One attention layer's paged cache (mirrors ``qstate_kv_cfg``).  A description for
    qstate_kv_plan alone needs page, n_pages and max_pages only."""
    page: int
    n_pages: int
    max_pages: int
    kind: int = KV_HEADS
    Hq: int = 1
    Hkv: int = 1
    dk: int = 64
    dv: int = 64
    dtype: int = KV_BF16
    store: int = KV_16
    window: int = 0
    scale: float = 1.0

    def __post_init__(self):
        import torch
        _keep(self, _KvCfg(self.kind, self.Hq, self.Hkv, self.dk, self.dv, self.page, self.n_pages, self.max_pages,
                           self.dtype, self.store, self.window, self.scale),
              torch_dtype=torch.float16 if self.dtype == KV_F16 else torch.bfloat16, _i32=torch.int32, _f32=torch.float32)


def kv_validate(cfg: KvConfig) -> None:
    _check(_lib_or_raise().qstate_kv_validate(ct.byref(cfg._c)))


def _typed(t, name, *dtypes):
    """Address of a contiguous CUDA tensor of one of the types (None stays None)."""
    if t is None:
        return None
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    return _ptr(t)


def _sized(t, name, n):
    if t is not None and t.numel() != n:
        raise ValueError(f"{name} must have {n} entries, got {t.numel()}")


@dataclass(frozen=True)
class KvCache(_Kept):
    """One layer's cache (device tensors, caller-owned): k (n_pages, Hkv, page, dk), v (n_pages, Hkv, page, dv)
    or None for latents, and for e4m3 the exponent bytes (n_pages, Hkv, page).  The tensors keep their storage
    for as long as the object is in use; so do those of KvPages and KvSlots."""
    k: object
    v: object = None
    k_exp: object = None
    v_exp: object = None

    def __post_init__(self):
        import torch
        types = (torch.bfloat16, torch.float16, torch.float8_e4m3fn)
        _keep(self, _KvCache(_typed(self.k, "k", *types), _typed(self.v, "v", *types),
                             _typed(self.k_exp, "k_exp", torch.uint8), _typed(self.v_exp, "v_exp", torch.uint8)), _fits=None)

    def _check(self, cfg):
        """The cache belongs to the description; looked at once for each description."""
        if self._fits is cfg:
            return
        import torch
        kv_validate(cfg)
        rows = cfg.n_pages * cfg.Hkv * cfg.page
        dtype = torch.float8_e4m3fn if cfg.store == KV_E4M3 else cfg.torch_dtype
        for t, name, d in ((self.k, "k", cfg.dk), (self.v, "v", cfg.dv)):
            _sized(t, name, rows * d)
            if t is not None and t.dtype != dtype:
                raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
        _sized(self.k_exp, "k_exp", rows)
        _sized(self.v_exp, "v_exp", rows)
        _keep(self, _fits=cfg)


def new_kv_cache(cfg: KvConfig, device="cuda") -> KvCache:
    import torch
    kv_validate(cfg)
    e4m3 = cfg.store == KV_E4M3
    shape = (cfg.n_pages, cfg.Hkv, cfg.page)
    arr = lambda d: torch.zeros(shape + (d,), dtype=torch.float8_e4m3fn if e4m3 else cfg.torch_dtype, device=device)  # noqa: E731
    exp = lambda: torch.full(shape, 127, dtype=torch.uint8, device=device) if e4m3 else None  # noqa: E731
    return KvCache(arr(cfg.dk), None if cfg.kind == KV_LATENT else arr(cfg.dv), exp(), exp())


@dataclass(frozen=True)
class KvPages(_Kept):
    """Who holds which page: table (R, max_pages), lens (R), free_list (n_pages), free_count (1), int32."""
    table: object
    lens: object
    free_list: object
    free_count: object

    def __post_init__(self):
        import torch
        names = ("table", "lens", "free_list", "free_count")
        _keep(self, _args=[_typed(getattr(self, n), n, torch.int32) for n in names], R=self.lens.numel(),
              _sizes=(self.table.numel(), self.free_list.numel()))


def new_kv_pages(cfg: KvConfig, R: int, device="cuda") -> KvPages:
    """Tables of R requests without tokens; every page is free, the lowest on top."""
    import torch
    return KvPages(torch.full((R, cfg.max_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(R, dtype=torch.int32, device=device),
                   torch.arange(cfg.n_pages - 1, -1, -1, dtype=torch.int32, device=device),
                   torch.full((1,), cfg.n_pages, dtype=torch.int32, device=device))


@dataclass(frozen=True)
class KvSlots(_Kept):
    """A step's tokens, as qstate_kv_plan lays them out: cu (R + 1), slot, pos, req (T; pos and req may
    be None), int32, and ok (R), uint8."""
    cu: object
    slot: object
    pos: object
    req: object
    ok: object

    def __post_init__(self):
        import torch
        ptrs = [_typed(getattr(self, n), n, torch.int32) for n in ("cu", "slot", "pos", "req")]
        T = self.slot.numel()
        _sized(self.pos, "pos", T)
        _sized(self.req, "req", T)
        _keep(self, _KvSlots(*ptrs, _typed(self.ok, "ok", torch.uint8), T), T=T, _sizes=(self.cu.numel(), self.ok.numel()))


def new_kv_slots(R: int, T: int, device="cuda") -> KvSlots:
    import torch
    i32 = lambda n: torch.empty(n, dtype=torch.int32, device=device)  # noqa: E731
    return KvSlots(i32(R + 1), i32(T), i32(T), i32(T), torch.empty(R, dtype=torch.uint8, device=device))


def new_kv_work(cfg: KvConfig, device="cuda"):
    """Work space of a layer's calls (zeroed); serves any number of calls in stream order."""
    import torch
    n = int(_lib_or_raise().qstate_kv_work_bytes(ct.byref(cfg._c)))
    if n == 0:
        kv_validate(cfg)
    return torch.zeros(n, dtype=torch.uint8, device=device)


def _work(cfg, work):
    """The work space's address; its size is looked at once for each description."""
    if getattr(work, "_kv_fits", None) is not cfg:
        need = int(_lib_or_raise().qstate_kv_work_bytes(ct.byref(cfg._c)))
        if work.numel() * work.element_size() < need:
            raise ValueError(f"the work space needs {need} bytes")
        _ptr(work)
        work._kv_fits = cfg
    return work.data_ptr()


# The three calls of a serving step are short (a launch or two of a few microseconds each), so what they look
# at is written out here instead of going through a function for each tensor: 5.7 us of host time a call
# against 7.0.
def _refuse(name, what):
    raise ValueError(f"{name} must be a contiguous CUDA tensor of {what}")


def qstate_kv_plan(cfg: KvConfig, pages: KvPages, n_new, slots: KvSlots, work, lens_out=None, free_out=None,
                   stream=None) -> None:
    """Pages and slots of a step (see include/qstate.h).  The new lengths and free count go to lens_out and
    free_out, in place without them."""
    R, i32 = pages.R, cfg._i32
    if n_new.dtype is not i32 or n_new.numel() != R or not n_new.is_cuda or not n_new.is_contiguous():
        _refuse("n_new", f"{R} int32")
    if pages._sizes != (R * cfg.max_pages, cfg.n_pages) or slots._sizes != (R + 1, R):
        raise ValueError(f"table must have {R} x {cfg.max_pages} entries, free_list {cfg.n_pages}, cu {R + 1} and ok {R}")
    table, lens, free_list, free = pages._args
    to, free_to = lens, free
    if lens_out is not None:
        if lens_out.dtype is not i32 or lens_out.numel() != R or not lens_out.is_cuda or not lens_out.is_contiguous():
            _refuse("lens_out", f"{R} int32")
        to = lens_out.data_ptr()
    if free_out is not None:
        if free_out.dtype is not i32 or free_out.numel() != 1 or not free_out.is_cuda:
            _refuse("free_out", "one int32")
        free_to = free_out.data_ptr()
    c = _KvPages(table, lens, to, free_list, free, free_to)
    rc = (_lib or load()).qstate_kv_plan(cfg._at, ct.addressof(c), n_new.data_ptr(), R, slots._at, _work(cfg, work),
                                         _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


def _refuse_rows(name, cfg, rows, heads, d):
    raise ValueError(f"{name} must be a CUDA tensor of {rows} x {heads} x {d} {cfg.torch_dtype} with entries side by side")


def qstate_kv_append(cfg: KvConfig, cache: KvCache, k, v, slot, stream=None) -> None:
    """Rows k, v (T, Hkv, d), any strides but the last, into slots slot[0..T); v is None for latents."""
    if cache._fits is not cfg:
        cache._check(cfg)
    T, H, dtype = slot.numel(), cfg.Hkv, cfg.torch_dtype
    if slot.dtype is not cfg._i32 or not slot.is_cuda or not slot.is_contiguous():
        _refuse("slot", "int32")
    if k.dtype is not dtype or k.shape != (T, H, cfg.dk) or k.stride(2) != 1 or not k.is_cuda:
        _refuse_rows("k", cfg, T, H, cfg.dk)
    kr, kh, _ = k.stride()
    vp, vr, vh = None, 0, 0
    if v is not None:
        if v.dtype is not dtype or v.shape != (T, H, cfg.dv) or v.stride(2) != 1 or not v.is_cuda:
            _refuse_rows("v", cfg, T, H, cfg.dv)
        vp = v.data_ptr()
        vr, vh, _ = v.stride()
    rc = (_lib or load()).qstate_kv_append(cfg._at, cache._at, k.data_ptr(), kr, kh, vp, vr, vh, slot.data_ptr(), T,
                                           _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


def qstate_kv_attend(cfg: KvConfig, cache: KvCache, q, table, lens, o, lse, work, stream=None) -> None:
    """One token of each request: q (R, Hq, dk), any strides but the last, against its pages; o (R, Hq, dv),
    lse (R, Hq) float32 or None."""
    if cache._fits is not cfg:
        cache._check(cfg)
    R, H, dtype, i32 = lens.numel(), cfg.Hq, cfg.torch_dtype, cfg._i32
    if q.dtype is not dtype or q.shape != (R, H, cfg.dk) or q.stride(2) != 1 or not q.is_cuda:
        _refuse_rows("q", cfg, R, H, cfg.dk)
    qr, qh, _ = q.stride()
    if lens.dtype is not i32 or not lens.is_cuda or not lens.is_contiguous():
        _refuse("lens", "int32")
    if table.dtype is not i32 or table.numel() != R * cfg.max_pages or not table.is_cuda or not table.is_contiguous():
        _refuse("table", f"{R} x {cfg.max_pages} int32")
    if o.dtype is not dtype or o.numel() != R * H * cfg.dv or not o.is_cuda or not o.is_contiguous():
        _refuse("o", f"{R} x {H} x {cfg.dv} {dtype}")
    sums = None
    if lse is not None:
        if lse.dtype is not cfg._f32 or lse.numel() != R * H or not lse.is_cuda or not lse.is_contiguous():
            _refuse("lse", f"{R} x {H} float32")
        sums = lse.data_ptr()
    rc = (_lib or load()).qstate_kv_attend(cfg._at, cache._at, q.data_ptr(), qr, qh, table.data_ptr(), lens.data_ptr(), R,
                                           o.data_ptr(), sums, _work(cfg, work),
                                           _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


# ---- requests that hold pages together ---------------------------------------------------------------
@dataclass(frozen=True)
class KvMoves(_Kept):
    """Pages to copy, src[i] to dst[i] (int32, one length; -1 in both where there is nothing to copy)."""
    src: object
    dst: object

    def __post_init__(self):
        import torch
        at = [_typed(getattr(self, n), n, torch.int32) for n in ("src", "dst")]
        _sized(self.dst, "dst", self.src.numel())
        _keep(self, _KvMoves(*at, self.src.numel()), n=self.src.numel())


def new_kv_moves(n: int, device="cuda") -> KvMoves:
    import torch
    return KvMoves(*(torch.full((n,), -1, dtype=torch.int32, device=device) for _ in range(2)))


@dataclass(frozen=True)
class KvGroups(_Kept):
    """What qstate_kv_group leaves for qstate_kv_attend_shared, for R requests."""
    data: object
    R: int

    def __post_init__(self):
        import torch
        _keep(self, _at=_typed(self.data, "data", torch.uint8), _fits=None, _made=None)

    def _check(self, cfg):
        """The memory is enough for the description; looked at once for each description."""
        need = _bytes("qstate_kv_group_bytes", cfg, self.R)
        if self.data.numel() < need:
            raise ValueError(f"groups of {self.R} requests need {need} bytes")
        _keep(self, _fits=cfg)


def _bytes(name, cfg, R):
    lib = _lib_or_raise()
    n = int(getattr(lib, name)(ct.byref(cfg._c), R))
    if n == 0:
        raise QstateError(QSTATE_EINVAL, lib.qstate_last_error().decode())
    return n


def new_kv_groups(cfg: KvConfig, R: int, device="cuda") -> KvGroups:
    import torch
    return KvGroups(torch.zeros(_bytes("qstate_kv_group_bytes", cfg, R), dtype=torch.uint8, device=device), R)


def new_kv_pages_work(cfg: KvConfig, R: int, device="cuda"):
    """Work space of qstate_kv_fork and qstate_kv_compact for up to R requests (zeroed)."""
    import torch
    return torch.zeros(_bytes("qstate_kv_pages_work_bytes", cfg, R), dtype=torch.uint8, device=device)


def new_kv_shared_work(cfg: KvConfig, R: int, device="cuda"):
    """Work space of qstate_kv_attend_shared for up to R requests (zeroed); serves qstate_kv_attend too."""
    import torch
    return torch.zeros(_bytes("qstate_kv_shared_work_bytes", cfg, R), dtype=torch.uint8, device=device)


def _work_of(name, cfg, work, R):
    """The address of a work space for R requests; its size is looked at once for each description and R."""
    if getattr(work, "_kv_fits_R", None) != (name, R) or getattr(work, "_kv_fits_cfg", None) is not cfg:
        need = _bytes(name, cfg, R)
        if work.numel() * work.element_size() < need:
            raise ValueError(f"the work space needs {need} bytes")
        _ptr(work)
        work._kv_fits_R, work._kv_fits_cfg = (name, R), cfg
    return work.data_ptr()


def _ints(t, name, n, none=False):
    """Address of n int32 (None stays None where it may be)."""
    import torch
    if t is None and none:
        return None
    if t is None or t.dtype is not torch.int32 or t.numel() != n or not t.is_cuda or not t.is_contiguous():
        _refuse(name, f"{n} int32")
    return t.data_ptr()


def _pages_struct(cfg, pages, lens_out, free_out):
    R = pages.R
    if pages._sizes != (R * cfg.max_pages, cfg.n_pages):
        raise ValueError(f"table must have {R} x {cfg.max_pages} entries and free_list {cfg.n_pages}")
    table, lens, free_list, free = pages._args
    return _KvPages(table, lens, lens if lens_out is None else _ints(lens_out, "lens_out", R), free_list, free,
                    free if free_out is None else _ints(free_out, "free_out", 1))


def qstate_kv_fork(cfg: KvConfig, pages: KvPages, others, parent, keep, moves: KvMoves, ok, work, lens_out=None, free_out=None,
                   stream=None) -> None:
    """Requests take over the first keep[r] tokens of request parent[r] (see include/qstate.h): others (n_pages), parent
    (R), keep (R, or None for all tokens), int32, ok (R), uint8, moves of R entries or more.  The new lengths and free
    count go to lens_out and free_out, in place without them."""
    import torch
    R = pages.R
    c = _pages_struct(cfg, pages, lens_out, free_out)
    if ok.dtype is not torch.uint8 or ok.numel() != R or not ok.is_cuda or not ok.is_contiguous():
        _refuse("ok", f"{R} uint8")
    if moves.n < R:
        raise ValueError(f"moves must have {R} entries or more, got {moves.n}")
    rc = (_lib or load()).qstate_kv_fork(cfg._at, ct.addressof(c), _ints(others, "others", cfg.n_pages), _ints(parent, "parent", R),
                                         _ints(keep, "keep", R, none=True), R, moves._at, ok.data_ptr(),
                                         _work_of("qstate_kv_pages_work_bytes", cfg, work, R),
                                         _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


def qstate_kv_compact(cfg: KvConfig, pages: KvPages, others, limit: int, moves: KvMoves, left, work, table_out=None,
                      free_out=None, stream=None) -> None:
    """Held pages from `limit` on move in front of it (see include/qstate.h): others (n_pages) and left (1), int32,
    may be None.  The new table and free count go to table_out and free_out, in place without them."""
    R = pages.R
    c = _pages_struct(cfg, pages, None, free_out)
    to = c.table if table_out is None else _ints(table_out, "table_out", R * cfg.max_pages)
    rc = (_lib or load()).qstate_kv_compact(cfg._at, ct.addressof(c), _ints(others, "others", cfg.n_pages, none=True), R, limit,
                                            moves._at, _ints(left, "left", 1, none=True), to,
                                            _work_of("qstate_kv_pages_work_bytes", cfg, work, R),
                                            _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


def qstate_kv_copy(cfg: KvConfig, cache: KvCache, moves: KvMoves, stream=None) -> None:
    """Copies the pages of `moves` in one layer's cache."""
    if cache._fits is not cfg:
        cache._check(cfg)
    rc = (_lib or load()).qstate_kv_copy(cfg._at, cache._at, moves._at, _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)


def qstate_set_shared_gain(ns: int) -> None:
    """What sharing has to gain for later calls of qstate_kv_group (ns; 0: share wherever two can, negative: the default)."""
    _check(_lib_or_raise().qstate_set_shared_gain(int(ns)))


def qstate_kv_group(cfg: KvConfig, lens, start, common, groups: KvGroups, stream=None) -> None:
    """Which requests share their first tokens (see include/qstate.h): lens (R), start (N + 1), common (N), int32."""
    if groups._fits is not cfg:
        groups._check(cfg)
    N = common.numel()
    rc = (_lib or load()).qstate_kv_group(cfg._at, _ints(lens, "lens", groups.R), groups.R, _ints(start, "start", N + 1),
                                          _ints(common, "common", N), N, groups._at,
                                          _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)
    if groups._made is not cfg:
        _keep(groups, _made=cfg)


def _attend_args(cfg, cache, q, table, lens, o, lse):
    """What an attention takes, looked at: q's strides, requests, lse's address."""
    if cache._fits is not cfg:
        cache._check(cfg)
    R, H, dtype, i32 = lens.numel(), cfg.Hq, cfg.torch_dtype, cfg._i32
    if q.dtype is not dtype or q.shape != (R, H, cfg.dk) or q.stride(2) != 1 or not q.is_cuda:
        _refuse_rows("q", cfg, R, H, cfg.dk)
    qr, qh, _ = q.stride()
    if lens.dtype is not i32 or not lens.is_cuda or not lens.is_contiguous():
        _refuse("lens", "int32")
    if table.dtype is not i32 or table.numel() != R * cfg.max_pages or not table.is_cuda or not table.is_contiguous():
        _refuse("table", f"{R} x {cfg.max_pages} int32")
    if o.dtype is not dtype or o.numel() != R * H * cfg.dv or not o.is_cuda or not o.is_contiguous():
        _refuse("o", f"{R} x {H} x {cfg.dv} {dtype}")
    sums = None
    if lse is not None:
        if lse.dtype is not cfg._f32 or lse.numel() != R * H or not lse.is_cuda or not lse.is_contiguous():
            _refuse("lse", f"{R} x {H} float32")
        sums = lse.data_ptr()
    return qr, qh, R, sums


def qstate_kv_attend_shared(cfg: KvConfig, cache: KvCache, q, table, lens, groups: KvGroups, o, lse, work, stream=None) -> None:
    """qstate_kv_attend with the groups' common tokens read once for all of their requests; `groups` as qstate_kv_group
    left them for these lengths."""
    qr, qh, R, sums = _attend_args(cfg, cache, q, table, lens, o, lse)
    if groups._fits is not cfg:
        groups._check(cfg)
    if groups.R != R:
        raise ValueError(f"groups were made for {groups.R} requests, got {R}")
    made = groups._made
    if made is not None and made is not cfg and (made.Hq, made.Hkv, made.dk, made.window, made.store) != (
            cfg.Hq, cfg.Hkv, cfg.dk, cfg.window, cfg.store):
        raise ValueError("groups were made for a layer of other heads, another window or another store")
    rc = (_lib or load()).qstate_kv_attend_shared(cfg._at, cache._at, q.data_ptr(), qr, qh, table.data_ptr(), lens.data_ptr(), R,
                                                  groups._at, o.data_ptr(), sums,
                                                  _work_of("qstate_kv_shared_work_bytes", cfg, work, R),
                                                  _current_stream() if stream is None else stream.cuda_stream)
    if rc:
        _check(rc)
