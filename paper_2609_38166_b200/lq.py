"""Thin Python binding of the C-ABI library (``include/lq.h``): argument marshalling only.

Every entry point has the name of its C symbol without the ``lq_`` prefix and takes torch tensors
(device memory and streams are PyTorch's; every step of the computation runs in the library's kernels).
There is no fallback of any kind: if ``liblq.so`` is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from dataclasses import dataclass
from typing import Optional

import torch

GATE_SCALAR = 0
GATE_DIAG = 1

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "liblq.so")
_lib = None

EXPORTS = ["lq_decode_step", "lq_decode_step_profiled", "lq_decode_step_host", "lq_decode_step_host_pipelined", "lq_decode_step_host_static", "lq_decode_stage_bytes", "lq_head_bytes", "lq_record_floats",
           "lq_window_flush",
           "lq_quantize_state", "lq_dequantize_state", "lq_ref_decode_step_f32", "lq_ref_decode_step_bf16",
           "lq_decode_launches", "lq_step_launches", "lq_check_device", "lq_clear_device_flags", "lq_selftest_bounded_wait",
           "lq_conv_prompt", "lq_conv_step", "lq_norm_rotate", "lq_scan_prompt", "lq_scan_prompt_bytes", "lq_scan_step",
           "lq_norm_add", "lq_norm_gate", "lq_product", "lq_product_groups",
           "lq_static_stage_bytes", "lq_import_state", "lq_export_state", "lq_status_string", "lq_version"]


class LqError(RuntimeError):
    pass


class _Shape(C.Structure):
    _fields_ = [(n, C.c_int) for n in
                ("batch", "heads_v", "heads_qk", "d_k", "d_v", "W", "r", "n_iter", "gate", "smooth", "delta", "rec16", "state_bf16")]


class _State(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("heads", "records", "decays", "win_pos", "work")]


def lib() -> C.CDLL:
    """The loaded shared library; raises if it has not been built (``python -m paper_2609_38166_b200.build``)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise LqError(f"{_LIB_PATH} is missing: build it with `python -m paper_2609_38166_b200.build`")
        L = C.CDLL(_LIB_PATH)
        L.lq_status_string.restype = C.c_char_p
        L.lq_status_string.argtypes = [C.c_int]
        L.lq_version.restype = C.c_int
        L.lq_decode_stage_bytes.restype = C.c_uint64
        L.lq_decode_stage_bytes.argtypes = [C.c_void_p]
        for name in ("lq_head_bytes", "lq_record_floats"):
            getattr(L, name).restype = C.c_uint64
            getattr(L, name).argtypes = [C.c_void_p]
        L.lq_decode_launches.restype = C.c_int
        L.lq_decode_launches.argtypes = [C.c_void_p]
        L.lq_step_launches.restype = C.c_int
        L.lq_step_launches.argtypes = [C.c_void_p, C.c_void_p]
        L.lq_static_stage_bytes.restype = C.c_uint64
        L.lq_static_stage_bytes.argtypes = []
        L.lq_clear_device_flags.restype = C.c_int
        L.lq_clear_device_flags.argtypes = []
        L.lq_selftest_bounded_wait.restype = C.c_int
        L.lq_selftest_bounded_wait.argtypes = [C.c_void_p]
        for name in ("lq_import_state", "lq_export_state"):
            getattr(L, name).restype = C.c_int
        for name in ("lq_decode_step", "lq_decode_step_profiled", "lq_decode_step_host", "lq_decode_step_host_pipelined",
                     "lq_decode_step_host_static", "lq_check_device", "lq_window_flush", "lq_quantize_state",
                     "lq_dequantize_state", "lq_ref_decode_step_f32", "lq_ref_decode_step_bf16"):
            getattr(L, name).restype = C.c_int
        vp = C.c_void_p                      # (declared, so that plain integers can be handed over as addresses)
        L.lq_decode_step.argtypes = [vp] * 9
        L.lq_decode_step_profiled.argtypes = [vp] * 10
        for name in ("lq_decode_step_host", "lq_decode_step_host_pipelined"):
            getattr(L, name).argtypes = [vp] * 10
        L.lq_decode_step_host_static.argtypes = [vp] * 9
        L.lq_window_flush.argtypes = [vp, vp, C.c_int, vp]
        L.lq_quantize_state.argtypes = L.lq_dequantize_state.argtypes = [vp] * 4
        L.lq_ref_decode_step_f32.argtypes = L.lq_ref_decode_step_bf16.argtypes = [vp] * 9
        L.lq_import_state.argtypes = L.lq_export_state.argtypes = [vp] * 4
        i64 = C.c_int64
        L.lq_conv_prompt.argtypes = [vp, vp, i64, vp, vp, vp, vp, i64, vp, vp, vp, vp]
        L.lq_conv_step.argtypes = [vp, vp, i64, vp, vp, vp, vp, i64, vp, vp]
        L.lq_norm_rotate.argtypes = [vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp]
        L.lq_scan_prompt.argtypes = [vp, vp, vp, i64, vp, vp]
        L.lq_scan_step.argtypes = [vp, vp, vp, i64, vp]
        L.lq_norm_add.argtypes = L.lq_norm_gate.argtypes = L.lq_product.argtypes = L.lq_product_groups.argtypes = [vp] * 3
        for name in ("lq_conv_prompt", "lq_conv_step", "lq_norm_rotate", "lq_scan_prompt", "lq_scan_step", "lq_norm_add", "lq_norm_gate", "lq_product",
                     "lq_product_groups"):
            getattr(L, name).restype = C.c_int
        L.lq_scan_prompt_bytes.restype = C.c_uint64
        L.lq_scan_prompt_bytes.argtypes = [vp]
        _lib = L
    return _lib


class _Kept:
    """A place for the C struct of a shape outside of the instance's dict, which holds the fields and nothing else."""
    __slots__ = ("_kept",)

    def ref(self):
        """A reference to the shape as the C struct, for a call of the library.  The struct is built once and kept until a
        field changes, however it is changed: a decode step is one call per token and layer, and at small batches its
        marshalling took longer than its kernels (10.1 us of host time a call, 2.7 us with the struct kept; comparing the
        fields is 0.2 us of it)."""
        try:
            of, kept = self._kept
            if of == self.__dict__:
                return kept[0]
        except AttributeError:
            pass
        return self._keep()[0]

    def kept(self):
        """The same with what the binding wants of the tensors (``wants``)."""
        try:
            of, kept = self._kept
            if of == self.__dict__:
                return kept
        except AttributeError:
            pass
        return self._keep()

    def _keep(self):
        of, kept = dict(self.__dict__), (C.byref(self.c()), self.wants())
        if of == self.__dict__:              # (another thread may be changing a field)
            self._kept = (of, kept)
        return kept

    def wants(self):
        return None

    def __getstate__(self):                  # (copies and pickles carry the fields only)
        return self.__dict__


@dataclass
class Shape(_Kept):
    batch: int
    heads_v: int
    heads_qk: int
    d_k: int = 128
    d_v: int = 128
    W: int = 16
    r: int = 4
    n_iter: int = 1
    gate: int = GATE_SCALAR
    smooth: int = 1
    delta: int = 1
    rec16: int = 0
    state_bf16: int = 0

    def c(self, batch: Optional[int] = None) -> _Shape:
        return _Shape(self.batch if batch is None else batch, self.heads_v, self.heads_qk, self.d_k, self.d_v, self.W, self.r,
                      self.n_iter, self.gate, self.smooth, self.delta, self.rec16, self.state_bf16)


def head_bytes(sh: Shape) -> int:
    return int(lib().lq_head_bytes(sh.ref()))


def record_floats(sh: Shape) -> int:
    return int(lib().lq_record_floats(sh.ref()))


class State:
    """Device tensors of the window representation of B x Hv heads, in the layout of ``lq_state``:
    ``heads`` (one contiguous byte block per head), ``records`` (one fp32 row per buffered record),
    ``decays`` (scalar gate) and ``win_pos``.  The named pieces (codes, col_scale, row_smooth, comp_k,
    comp_u, buf_k, buf_u, buf_a) are strided views into those tensors."""

    def __init__(self, sh: Shape, device="cuda", storage=None, work=True):
        """``storage``: optionally the four tensors (heads, records, decays, win_pos) to use instead of fresh
        ones - contiguous, of the shapes and dtypes below (callers that place the state in memory of their own).
        ``work``: give the state the ``work`` words (LQ_WORK_WORDS).  With them a step of many shapes is one launch instead
        of two (``step_launches``), and the decode kernel of the others hands out the heads of its last rounds to the CTAs that
        get there first; without them every CTA takes the same number."""
        B, H, K, V, W, r = sh.batch, sh.heads_v, sh.d_k, sh.d_v, sh.W, sh.r
        self.shape = sh
        self.work = torch.zeros((8,), dtype=torch.int32, device=device) if work else None
        hb, rf = head_bytes(sh), record_floats(sh)
        assert hb > 0 and rf > 0, "shape not supported by the library"
        rec_dtype = torch.float16 if sh.rec16 else torch.float32
        if storage is None:
            self.heads = torch.zeros((B, H, hb), dtype=torch.uint8, device=device)
            self.records = torch.zeros((B, H, W, rf), dtype=rec_dtype, device=device)
            self.decays = torch.zeros((B, H, W), dtype=torch.float32, device=device)
            self.win_pos = torch.zeros((B,), dtype=torch.int32, device=device)
        else:
            self.heads, self.records, self.decays, self.win_pos = storage
            for t, shape, dt in ((self.heads, (B, H, hb), torch.uint8), (self.records, (B, H, W, rf), rec_dtype),
                                 (self.decays, (B, H, W), torch.float32), (self.win_pos, (B,), torch.int32)):
                assert tuple(t.shape) == shape and t.dtype == dt and t.is_contiguous(), (tuple(t.shape), shape, t.dtype, dt)
        if sh.state_bf16:                    # per-window BF16: the head block is S^T in bfloat16, nothing else
            assert hb == 2 * K * V
            self.state16 = self.heads.view(torch.bfloat16).unflatten(-1, (V, K))
            self.codes = self.col_scale = self.row_smooth = self.comp_k = self.comp_u = None
            self._record_views(sh)
            return
        o = 0
        self.codes = self.heads[..., o:o + K * V].view(torch.int8).unflatten(-1, (V, K)); o += K * V   # Z^T
        self.col_scale = self.heads[..., o:o + 4 * V].view(torch.float32); o += 4 * V
        self.row_smooth = self.heads[..., o:o + 4 * K].view(torch.float32); o += 4 * K
        self.comp_k = self.heads[..., o:o + 2 * r * K].view(torch.float16).unflatten(-1, (r, K)); o += 2 * r * K
        self.comp_u = self.heads[..., o:o + 2 * r * V].view(torch.float16).unflatten(-1, (r, V)); o += 2 * r * V
        assert o == hb
        if storage is None:
            self.row_smooth.fill_(1.0)
        self._record_views(sh)

    def _record_views(self, sh: Shape) -> None:
        K, V = sh.d_k, sh.d_v
        self.buf_k = self.records[..., 0:K]
        self.buf_u = self.records[..., K:K + V]
        self.buf_a = self.records[..., K + V:K + V + K] if sh.gate == GATE_DIAG else self.decays

    def tensors(self):
        return (self.heads, self.records, self.decays, self.win_pos)

    def c(self, b0: int = 0) -> _State:
        """ctypes view; ``b0`` offsets every array to sequence b0 (sub-batches are addressed by pointer)."""
        work = self.work.data_ptr() if self.work is not None else None
        if b0:
            return _State(*[t.data_ptr() + b0 * t.stride(0) * t.element_size() for t in self.tensors()], work)
        return _State(self.heads.data_ptr(), self.records.data_ptr(), self.decays.data_ptr(), self.win_pos.data_ptr(), work)

    def nbytes_quantized(self) -> int:
        return self.heads.numel()


def _stream(stream) -> int:
    if stream is None:                       # (building torch's Stream object for this takes 3.4 us)
        return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _check(rc: int, what: str) -> None:
    if rc != 0:
        raise LqError(f"{what}: {lib().lq_status_string(rc).decode()} (status {rc})")


def _ptr(t: Optional[torch.Tensor], b0: int = 0) -> Optional[int]:
    if t is None:
        return None
    assert t.is_contiguous()
    return t.data_ptr() + b0 * t.stride(0) * t.element_size() if b0 else t.data_ptr()


def _sub(sh: Shape, b0: int, nb: Optional[int]):
    """Sequences [b0, b0+nb) of a shape, as a reference to the C struct."""
    if nb is None and not b0:
        return sh.ref()
    nb = sh.batch - b0 if nb is None else nb
    return C.byref(sh.c(nb))


def decode_step(sh: Shape, st: State, q, k, v, beta, alpha, o, stream=None, b0: int = 0, nb: Optional[int] = None):
    """lq_decode_step on sequences [b0, b0+nb) of the tensors (all of them by default)."""
    s = sh.ref() if nb is None and not b0 else _sub(sh, b0, nb)
    cs = C.byref(st.c(b0))
    rc = (_lib or lib()).lq_decode_step(s, cs, _ptr(q, b0), _ptr(k, b0), _ptr(v, b0), _ptr(beta, b0), _ptr(alpha, b0), _ptr(o, b0),
                                        _stream(stream))
    if rc:
        _check(rc, "lq_decode_step")


def decode_step_profiled(sh: Shape, st: State, q, k, v, beta, alpha, o, event_between, stream=None):
    """lq_decode_step_profiled: ``event_between`` is a torch.cuda.Event that has been recorded once before
    (so that its CUDA handle exists); it is re-recorded between the two kernels of the step."""
    s = sh.ref()
    cs = C.byref(st.c())
    _check(lib().lq_decode_step_profiled(s, cs, _ptr(q), _ptr(k), _ptr(v), _ptr(beta),
                                         _ptr(alpha), _ptr(o), _stream(stream), event_between.cuda_event),
           "lq_decode_step_profiled")


def decode_stage_bytes(sh: Shape) -> int:
    return int(lib().lq_decode_stage_bytes(sh.ref()))


def decode_launches(sh: Shape) -> int:
    return int(lib().lq_decode_launches(sh.ref()))


def step_launches(sh: Shape, st: State) -> int:
    return int(lib().lq_step_launches(sh.ref(), C.byref(st.c())))


def decode_step_host(sh: Shape, st: State, q_h, k_h, v_h, beta_h, alpha_h, o_h, stage, stream=None):
    """lq_decode_step_host: the token's tensors are (pinned) CPU tensors, ``stage`` a device byte buffer."""
    for t in (q_h, k_h, v_h, beta_h, alpha_h, o_h):
        assert t.device.type == "cpu" and t.is_contiguous()
    s = sh.ref()
    cs = C.byref(st.c())
    _check(lib().lq_decode_step_host(s, cs, _ptr(q_h), _ptr(k_h), _ptr(v_h), _ptr(beta_h),
                                     _ptr(alpha_h), _ptr(o_h), _ptr(stage), _stream(stream)), "lq_decode_step_host")


def decode_step_host_pipelined(sh: Shape, st: State, q_h, k_h, v_h, beta_h, alpha_h, o_h, stage, stream=None):
    """lq_decode_step_host_pipelined: same arguments as decode_step_host; copies and kernels overlap."""
    for t in (q_h, k_h, v_h, beta_h, alpha_h, o_h):
        assert t.device.type == "cpu" and t.is_contiguous()
    s = sh.ref()
    cs = C.byref(st.c())
    _check(lib().lq_decode_step_host_pipelined(s, cs, _ptr(q_h), _ptr(k_h), _ptr(v_h), _ptr(beta_h),
                                               _ptr(alpha_h), _ptr(o_h), _ptr(stage), _stream(stream)),
           "lq_decode_step_host_pipelined")


STATIC_STAGE_BYTES = 16 << 20


def decode_step_host_static(sh: Shape, st: State, q_h, k_h, v_h, beta_h, alpha_h, o_h, stream=None):
    """lq_decode_step_host_static: like decode_step_host, for callers that cannot allocate the staging
    buffer; the staging is a fixed array inside the library (requests above STATIC_STAGE_BYTES are refused)."""
    for t in (q_h, k_h, v_h, beta_h, alpha_h, o_h):
        assert t.device.type == "cpu" and t.is_contiguous()
    s = sh.ref()
    cs = C.byref(st.c())
    _check(lib().lq_decode_step_host_static(s, cs, _ptr(q_h), _ptr(k_h), _ptr(v_h), _ptr(beta_h),
                                            _ptr(alpha_h), _ptr(o_h), _stream(stream)), "lq_decode_step_host_static")


def window_flush(sh: Shape, st: State, force: bool = False, stream=None):
    s = sh.ref()
    cs = C.byref(st.c())
    _check(lib().lq_window_flush(s, cs, 1 if force else 0, _stream(stream)),
           "lq_window_flush")


def quantize_state(sh: Shape, S, st: State, stream=None, b0: int = 0, nb: Optional[int] = None):
    s = _sub(sh, b0, nb)
    cs = C.byref(st.c(b0))
    _check(lib().lq_quantize_state(s, _ptr(S, b0), cs, _stream(stream)), "lq_quantize_state")


def dequantize_state(sh: Shape, st: State, S, stream=None, b0: int = 0, nb: Optional[int] = None):
    """lq_dequantize_state on sequences [b0, b0+nb) of the state; ``S`` receives exactly those sequences."""
    s = _sub(sh, b0, nb)
    cs = C.byref(st.c(b0))
    _check(lib().lq_dequantize_state(s, cs, _ptr(S), _stream(stream)), "lq_dequantize_state")


def ref_decode_step_f32(sh: Shape, S, q, k, v, beta, alpha, o, stream=None, b0: int = 0, nb: Optional[int] = None):
    s = _sub(sh, b0, nb)
    _check(lib().lq_ref_decode_step_f32(s, _ptr(S, b0), _ptr(q, b0), _ptr(k, b0), _ptr(v, b0),
                                        _ptr(beta, b0), _ptr(alpha, b0), _ptr(o, b0), _stream(stream)),
           "lq_ref_decode_step_f32")


def ref_decode_step_bf16(sh: Shape, S16, q, k, v, beta, alpha, o, stream=None):
    s = sh.ref()
    _check(lib().lq_ref_decode_step_bf16(s, _ptr(S16), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(alpha),
                                         _ptr(o), _stream(stream)), "lq_ref_decode_step_bf16")


def check_device() -> int:
    """lq_check_device: synchronises the device and returns the kernels' error flags (0 = none)."""
    flags = C.c_int(0)
    _check(lib().lq_check_device(C.byref(flags)), "lq_check_device")
    return int(flags.value)


class _StateArrays(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("codes", "col_scale", "row_smooth", "comp_k", "comp_u", "buf_k", "buf_u", "buf_a", "win_pos")]


class StateArrays:
    """The window representation as separate device tensors in the paper's orientation (``lq_state_arrays``):
    codes int8 [B,Hv,d_k,d_v], col_scale / row_smooth fp32, comp_k / comp_u fp16, buf_k / buf_u / buf_a fp32,
    win_pos int32 [B]."""

    def __init__(self, sh: Shape, device="cuda"):
        B, H, K, V, W, r = sh.batch, sh.heads_v, sh.d_k, sh.d_v, sh.W, sh.r
        z = lambda shape, dt: torch.zeros(shape, dtype=dt, device=device)
        self.codes = z((B, H, K, V), torch.int8)
        self.col_scale = z((B, H, V), torch.float32)
        self.row_smooth = z((B, H, K), torch.float32)
        self.comp_k = z((B, H, r, K), torch.float16)
        self.comp_u = z((B, H, r, V), torch.float16)
        self.buf_k = z((B, H, W, K), torch.float32)
        self.buf_u = z((B, H, W, V), torch.float32)
        self.buf_a = z((B, H, W, K) if sh.gate == GATE_DIAG else (B, H, W), torch.float32)
        self.win_pos = z((B,), torch.int32)

    def c(self) -> _StateArrays:
        ptr = lambda t: t.data_ptr() if t.numel() else None
        return _StateArrays(ptr(self.codes), ptr(self.col_scale), ptr(self.row_smooth), ptr(self.comp_k), ptr(self.comp_u),
                            ptr(self.buf_k), ptr(self.buf_u), ptr(self.buf_a), ptr(self.win_pos))


def import_state(sh: Shape, arrays: StateArrays, st: State, stream=None) -> None:
    """lq_import_state: fill the packed state from the separate arrays."""
    s, a, cs = sh.ref(), C.byref(arrays.c()), C.byref(st.c())
    _check(lib().lq_import_state(s, a, cs, _stream(stream)), "lq_import_state")


def export_state(sh: Shape, st: State, arrays: StateArrays, stream=None) -> None:
    """lq_export_state: write the packed state out as separate arrays."""
    s, a, cs = sh.ref(), C.byref(arrays.c()), C.byref(st.c())
    _check(lib().lq_export_state(s, cs, a, _stream(stream)), "lq_export_state")


# ---- what surrounds the decode step in a layer: the operators on packed rows ----

BF16, F16, F32 = 0, 1, 2                     # lq_type
TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}
_DTYPES = {v: k for k, v in TYPES.items()}
NORM_NONE, NORM_L2, NORM_RMS = 0, 1, 2


class _Conv(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "seqs", "channels", "width", "n_slots", "silu", "type")]


class _Norm(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "heads_q", "heads_k", "dim", "rot", "pairs", "norm", "type")] + \
               [(n, C.c_float) for n in ("eps", "scale_q", "scale_k")]


class _Scan(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "seqs", "max_len", "heads_v", "heads_qk", "d_k", "d_v", "n_slots", "select", "gate_type")]


class _ScanIo(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q", "k", "v")] + [(n, C.c_int64) for n in ("q_stride", "k_stride", "v_stride")] + \
               [(n, C.c_void_p) for n in ("beta", "alpha")] + [(n, C.c_int64) for n in ("beta_stride", "alpha_stride")] + \
               [(n, C.c_void_p) for n in ("A", "dt_bias", "skip", "S0", "S", "seq_start", "slots", "resume")]


@dataclass
class ConvShape(_Kept):
    """``lq_conv``: ``tokens`` packed rows of ``seqs`` sequences (``conv_step``: one row each), states in ``n_slots`` slots."""
    tokens: int
    seqs: int
    channels: int
    width: int = 4
    n_slots: int = 0
    silu: int = 1
    type: int = BF16

    def c(self) -> _Conv:
        return _Conv(self.tokens, self.seqs, self.channels, self.width, self.n_slots, self.silu, self.type)

    def wants(self):
        return (_DTYPES.get(self.type), (self.tokens, self.channels), (self.channels, self.width), (self.channels,),
                (self.n_slots, self.width - 1, self.channels), (self.seqs + 1,), (self.seqs,))


@dataclass
class NormShape(_Kept):
    """``lq_norm``: heads of ``dim`` channels, of which the first ``rot`` are rotated."""
    tokens: int
    heads_q: int
    heads_k: int
    dim: int = 128
    rot: int = 0
    pairs: int = 0
    norm: int = NORM_L2
    type: int = BF16
    eps: float = 1e-6
    scale_q: float = 1.0
    scale_k: float = 1.0

    def c(self) -> _Norm:
        return _Norm(self.tokens, self.heads_q, self.heads_k, self.dim, self.rot, self.pairs, self.norm, self.type, self.eps, self.scale_q,
                     self.scale_k)

    def wants(self):
        return (_DTYPES.get(self.type), (self.tokens, self.heads_q, self.dim), (self.tokens, self.heads_k, self.dim), (self.dim,), (self.tokens,),
                (self.rot // 2,))


@dataclass
class ScanShape(_Kept):
    """``lq_scan``: ``max_len`` is at least the length of the longest sequence (``scan_step`` does not look at it)."""
    tokens: int
    seqs: int
    heads_v: int
    heads_qk: int
    max_len: int = 1
    d_k: int = 128
    d_v: int = 128
    n_slots: int = 0
    select: int = 0
    gate_type: int = BF16

    def c(self) -> _Scan:
        return _Scan(self.tokens, self.seqs, self.max_len, self.heads_v, self.heads_qk, self.d_k, self.d_v, self.n_slots, self.select, self.gate_type)

    def wants(self):
        T, H = self.tokens, self.heads_v
        return (_DTYPES.get(self.gate_type), (T, self.heads_qk, self.d_k), (T, H, self.d_v), (T, H), (H,), (self.n_slots, H, self.d_k, self.d_v),
                (self.seqs + 1,), (self.seqs,))


class _Add(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "dim", "norm", "type")] + [("eps", C.c_float)]


class _Gated(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("tokens", "heads", "dim", "norm", "silu", "o_type", "type")] + [("eps", C.c_float)]


class _NormIo(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_stride", C.c_int64), ("residual", C.c_void_p), ("residual_stride", C.c_int64), ("z", C.c_void_p), ("z_stride", C.c_int64),
                ("w", C.c_void_p), ("out", C.c_void_p), ("out_stride", C.c_int64), ("out8", C.c_void_p), ("out8_stride", C.c_int64), ("scale", C.c_void_p),
                ("scale_stride", C.c_int64)]


class _ProductIo(C.Structure):
    _fields_ = [("x", C.c_void_p), ("x_stride", C.c_int64), ("x_scale", C.c_void_p), ("x_scale_stride", C.c_int64), ("w", C.c_void_p), ("w_scale", C.c_void_p),
                ("out", C.c_void_p), ("out_stride", C.c_int64), ("group_start", C.c_void_p)]


class _Linear(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("rows", "in_", "out", "groups", "type")]


E4M3 = torch.float8_e4m3fn
BLOCK = 128                                  # channels of a row to a scale, and output channels of weights


@dataclass
class AddShape(_Kept):
    """``lq_add``: rows of ``dim`` channels, normalised as a whole."""
    tokens: int
    dim: int
    norm: int = NORM_RMS
    type: int = BF16
    eps: float = 1e-6

    def c(self) -> _Add:
        return _Add(self.tokens, self.dim, self.norm, self.type, self.eps)

    def wants(self):
        return _DTYPES.get(self.type), (self.tokens, self.dim), (self.dim,), (-(-self.dim // BLOCK), self.tokens)


@dataclass
class GatedShape(_Kept):
    """``lq_gated``: ``heads`` heads of ``dim`` channels, outputs of a recurrence of ``o_type``."""
    tokens: int
    heads: int
    dim: int = 128
    norm: int = NORM_RMS
    silu: int = 1
    o_type: int = F32
    type: int = BF16
    eps: float = 1e-6

    def c(self) -> _Gated:
        return _Gated(self.tokens, self.heads, self.dim, self.norm, self.silu, self.o_type, self.type, self.eps)

    def wants(self):
        width = self.heads * self.dim
        return (_DTYPES.get(self.o_type), _DTYPES.get(self.type), (self.tokens, self.heads, self.dim), (self.tokens, width), (self.dim,),
                (-(-width // BLOCK), self.tokens))


@dataclass
class ProductShape(_Kept):
    """``lq_linear``: ``rows`` rows of ``channels_in`` channels, weights of ``channels_out`` (of every group)."""
    rows: int
    channels_in: int
    channels_out: int
    groups: int = 1
    type: int = BF16

    def c(self) -> _Linear:
        return _Linear(self.rows, self.channels_in, self.channels_out, self.groups, self.type)

    def wants(self):
        n, k = self.channels_out, self.channels_in
        scales = (-(-n // BLOCK), -(-k // BLOCK))
        return (_DTYPES.get(self.type), (self.rows, k), (scales[1], self.rows), (n, k), scales, (self.rows, n), (self.groups, n, k), (self.groups, *scales),
                (self.groups + 1,))


_SCAN_IO = struct.Struct("=3Q3q2Q2q8Q")        # lq_scan_io, as _ScanIo
_NORM_IO = struct.Struct("=QqQqQqQQqQqQq")     # lq_norm_io, as _NormIo
_PRODUCT_IO = struct.Struct("=QqQqQQQqQ")      # lq_product_io, as _ProductIo
_device = torch._C._cuda_getDevice


def _refuse(t, what: str, want) -> None:
    raise LqError(f"{what}: " + ("missing" if t is None else f"{t.dtype} {tuple(t.shape)} with strides {t.stride()} on {t.device}") +
                  f", wanted {want} on cuda:{torch.cuda.current_device()}")


def _rows(t, what: str, dtype, shape, device: int):
    """(address, row stride) of a tensor of ``shape``, [rows, ...], and ``dtype`` whose rows are contiguous, on the current device."""
    if t is None or t.dtype is not dtype or t.shape != shape or t.get_device() != device:
        _refuse(t, what, (dtype, shape))
    if len(shape) == 2:                      # (most of them: a call is marshalled in half the time)
        stride, one = t.stride()
        if one != 1 and shape[1] != 1 and shape[0] > 0:
            _refuse(t, what, (dtype, shape, "contiguous rows"))
        return t.data_ptr(), stride if shape[0] > 1 else shape[1]
    if t.is_contiguous():
        return t.data_ptr(), t.stride(0) if shape[0] > 1 else math.prod(shape[1:])
    stride, run = t.stride(), 1
    for n, s in zip(shape[:0:-1], stride[:0:-1]):
        if n != 1 and s != run:
            _refuse(t, what, (dtype, shape, "contiguous rows"))
        run *= n
    return t.data_ptr(), stride[0] if shape[0] > 1 else max(stride[0], run)


def _dense(t, what: str, dtype, shape, device: int):
    """Address of a contiguous tensor of that shape on the current device; None stays None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != device or not t.is_contiguous():
        _refuse(t, what, (dtype, shape, "contiguous"))
    return t.data_ptr()


def conv_prompt(sh: ConvShape, x, w, bias, state, out, seq_start, slots=None, resume=None, stream=None) -> None:
    """lq_conv_prompt: ``x``, ``out`` [tokens, channels] (rows may be strided), ``w`` [channels, width], ``bias`` [channels] or None,
    ``state`` [n_slots, width-1, channels] or None, ``seq_start`` int32 [seqs+1], ``slots``, ``resume`` int32 [seqs] or None."""
    ref, (dt, rows, taps, chan, states, starts, seqs) = sh.kept()
    d, i32 = _device(), torch.int32
    px, sx = _rows(x, "x", dt, rows, d)
    po, so = _rows(out, "out", dt, rows, d)
    rc = (_lib or lib()).lq_conv_prompt(ref, px, sx, _dense(w, "w", dt, taps, d), _dense(bias, "bias", dt, chan, d), _dense(state, "state", dt, states, d), po, so,
                                        _dense(seq_start, "seq_start", i32, starts, d), _dense(slots, "slots", i32, seqs, d),
                                        _dense(resume, "resume", i32, seqs, d), _stream(stream))
    if rc:
        _check(rc, "lq_conv_prompt")


def conv_step(sh: ConvShape, x, w, bias, state, out, slots=None, stream=None) -> None:
    """lq_conv_step: one row per sequence; ``out`` may be ``x``."""
    ref, (dt, rows, taps, chan, states, _, seqs) = sh.kept()
    d = _device()
    px, sx = _rows(x, "x", dt, rows, d)
    po, so = (px, sx) if out is x else _rows(out, "out", dt, rows, d)
    rc = (_lib or lib()).lq_conv_step(ref, px, sx, _dense(w, "w", dt, taps, d), _dense(bias, "bias", dt, chan, d), _dense(state, "state", dt, states, d), po, so,
                                      _dense(slots, "slots", torch.int32, seqs, d), _stream(stream))
    if rc:
        _check(rc, "lq_conv_step")


def norm_rotate(sh: NormShape, q, k, out_q, out_k, w_q=None, w_k=None, positions=None, inv_freq=None, stream=None) -> None:
    """lq_norm_rotate: ``q``, ``out_q`` [tokens, heads_q, dim], ``k``, ``out_k`` [tokens, heads_k, dim] (rows may be strided; an output
    may be its input), ``w_q``, ``w_k`` fp32 [dim] or None, ``positions`` int32 [tokens], ``inv_freq`` fp32 [rot/2]."""
    ref, (dt, rows_q, rows_k, dim, toks, freqs) = sh.kept()
    d, f32 = _device(), torch.float32
    none = (None, 0)
    pq, sq = _rows(q, "q", dt, rows_q, d) if rows_q[1] else none
    pk, sk = _rows(k, "k", dt, rows_k, d) if rows_k[1] else none
    poq, soq = _rows(out_q, "out_q", dt, rows_q, d) if rows_q[1] else none
    pok, sok = _rows(out_k, "out_k", dt, rows_k, d) if rows_k[1] else none
    rc = (_lib or lib()).lq_norm_rotate(ref, pq, sq, pk, sk, poq, soq, pok, sok, _dense(w_q, "w_q", f32, dim, d), _dense(w_k, "w_k", f32, dim, d),
                                        _dense(positions, "positions", torch.int32, toks, d), _dense(inv_freq, "inv_freq", f32, freqs, d), _stream(stream))
    if rc:
        _check(rc, "lq_norm_rotate")


def _scan_io(want, d: int, q, k, v, beta, alpha, S0, S, seq_start, slots, resume, A, dt_bias, skip) -> bytes:
    gate, qk, vo, gates, heads, states, starts, seqs = want
    bf, f32, i32 = torch.bfloat16, torch.float32, torch.int32
    pq, sq = _rows(q, "q", bf, qk, d)
    pk, sk = _rows(k, "k", bf, qk, d)
    pv, sv = _rows(v, "v", bf, vo, d)
    pb, sb = _rows(beta, "beta", gate, gates, d)
    pa, sa = (0, 0) if alpha is None else _rows(alpha, "alpha", gate, gates, d)
    return _SCAN_IO.pack(pq, pk, pv, sq, sk, sv, pb, pa, sb, sa, _dense(A, "A", f32, heads, d) or 0, _dense(dt_bias, "dt_bias", f32, heads, d) or 0,
                         _dense(skip, "skip", f32, heads, d) or 0, _dense(S0, "S0", f32, states, d) or 0, _dense(S, "S", f32, states, d) or 0,
                         _dense(seq_start, "seq_start", i32, starts, d) or 0, _dense(slots, "slots", i32, seqs, d) or 0,
                         _dense(resume, "resume", i32, seqs, d) or 0)


def scan_prompt_bytes(sh: ScanShape) -> int:
    """lq_scan_prompt_bytes: the size of the workspace of ``scan_prompt``."""
    return int(lib().lq_scan_prompt_bytes(sh.ref()))


def scan_prompt(sh: ScanShape, q, k, v, beta, alpha, o, S, seq_start, slots=None, resume=None, A=None, dt_bias=None, skip=None, S0=None,
                work=None, stream=None) -> None:
    """lq_scan_prompt: ``q``, ``k`` bf16 [tokens, heads_qk, d_k], ``v``, ``o`` bf16 [tokens, heads_v, d_v], ``beta``, ``alpha``
    [tokens, heads_v] (rows of all of them may be strided; with ``sh.select`` beta is dt and alpha None), ``S`` fp32 [n_slots, heads_v,
    d_k, d_v], ``S0`` the same or None (resumed from S), ``A``, ``dt_bias``, ``skip`` fp32 [heads_v], ``work`` uint8 [scan_prompt_bytes]
    (None where that is 0)."""
    ref, want = sh.kept()
    d = _device()
    io = _scan_io(want, d, q, k, v, beta, alpha, S0, S, seq_start, slots, resume, A, dt_bias, skip)
    po, so = _rows(o, "o", torch.bfloat16, want[2], d)
    pw = None
    if work is not None and work.numel():
        need = scan_prompt_bytes(sh)
        if work.dtype is not torch.uint8 or not work.is_contiguous() or work.numel() < need or work.get_device() != d:
            _refuse(work, "work", f"{need} bytes of torch.uint8")
        pw = work.data_ptr()
    rc = (_lib or lib()).lq_scan_prompt(ref, io, po, so, pw, _stream(stream))
    if rc:
        _check(rc, "lq_scan_prompt")


def scan_step(sh: ScanShape, q, k, v, beta, alpha, o, S, slots=None, A=None, dt_bias=None, skip=None, S0=None, stream=None) -> None:
    """lq_scan_step: one row per sequence, as in ``scan_prompt``; ``o`` is fp32 [seqs, heads_v, d_v]."""
    ref, want = sh.kept()
    d = _device()
    io = _scan_io(want, d, q, k, v, beta, alpha, S0, S, None, slots, None, A, dt_bias, skip)
    po, so = _rows(o, "o", torch.float32, want[2], d)
    rc = (_lib or lib()).lq_scan_step(ref, io, po, so, _stream(stream))
    if rc:
        _check(rc, "lq_scan_step")


def _norm_io(d: int, x, residual, z, w, dim, out, out8, scale, dt, rows, scales) -> bytes:
    """lq_norm_io; x, residual and z as (address, stride)."""
    po, so = (0, 0) if out is None else _rows(out, "out", dt, rows, d)
    p8, s8 = (0, 0) if out8 is None else _rows(out8, "out8", E4M3, rows, d)
    ps, ss = (0, 0) if scale is None else _rows(scale, "scale", torch.float32, scales, d)
    return _NORM_IO.pack(*x, *residual, *z, _dense(w, "w", torch.float32, dim, d) or 0, po, so, p8, s8, ps, ss)


def norm_add(sh: AddShape, x, residual=None, w=None, out=None, out8=None, scale=None, stream=None) -> None:
    """lq_norm_add: ``x``, ``out``, ``residual`` [tokens, dim] (``residual`` in and out, or None; ``out`` may be ``x``), ``w`` fp32 [dim] or None,
    ``out8`` float8_e4m3fn [tokens, dim] with ``scale`` fp32 [ceil(dim/128), tokens]; ``out`` or ``out8`` may be None.  Rows of all may be strided."""
    ref, (dt, rows, dim, scales) = sh.kept()
    d = _device()
    px = _rows(x, "x", dt, rows, d)
    pr = (0, 0) if residual is None else _rows(residual, "residual", dt, rows, d)
    rc = (_lib or lib()).lq_norm_add(ref, _norm_io(d, px, pr, (0, 0), w, dim, out, out8, scale, dt, rows, scales), _stream(stream))
    if rc:
        _check(rc, "lq_norm_add")


def norm_gate(sh: GatedShape, o, z, w=None, out=None, out8=None, scale=None, stream=None) -> None:
    """lq_norm_gate: ``o``, ``z`` [tokens, heads, dim], ``w`` fp32 [dim] or None, ``out`` [tokens, heads * dim], ``out8`` float8_e4m3fn
    [tokens, heads * dim] with ``scale`` fp32 [ceil(heads * dim / 128), tokens]; ``out`` or ``out8`` may be None.  Rows of all may be strided."""
    ref, (odt, dt, heads, rows, dim, scales) = sh.kept()
    d = _device()
    po = _rows(o, "o", odt, heads, d)
    pz = _rows(z, "z", dt, heads, d)
    rc = (_lib or lib()).lq_norm_gate(ref, _norm_io(d, po, (0, 0), pz, w, dim, out, out8, scale, dt, rows, scales), _stream(stream))
    if rc:
        _check(rc, "lq_norm_gate")


def product(sh: ProductShape, x, x_scale, w, w_scale, out, stream=None) -> None:
    """lq_product: ``x`` float8_e4m3fn [rows, channels_in], ``x_scale`` fp32 [ceil(channels_in/128), rows], ``out`` [rows, channels_out] (rows of all
    three may be strided), ``w`` float8_e4m3fn [channels_out, channels_in], ``w_scale`` fp32 [ceil(channels_out/128), ceil(channels_in/128)]."""
    ref, (dt, rows, scales, weights, w_scales, outs, _, _, _) = sh.kept()
    d, f32 = _device(), torch.float32
    io = _PRODUCT_IO.pack(*_rows(x, "x", E4M3, rows, d), *_rows(x_scale, "x_scale", f32, scales, d), _dense(w, "w", E4M3, weights, d) or 0,
                          _dense(w_scale, "w_scale", f32, w_scales, d) or 0, *_rows(out, "out", dt, outs, d), 0)
    rc = (_lib or lib()).lq_product(ref, io, _stream(stream))
    if rc:
        _check(rc, "lq_product")


def product_groups(sh: ProductShape, x, x_scale, w, w_scale, out, group_start, stream=None) -> None:
    """lq_product_groups: as ``product`` with ``w`` [groups, channels_out, channels_in], ``w_scale`` [groups, ceil(channels_out/128),
    ceil(channels_in/128)]; ``group_start`` int32 [groups + 1]."""
    ref, (dt, rows, scales, _, _, outs, weights, w_scales, starts) = sh.kept()
    d, f32 = _device(), torch.float32
    io = _PRODUCT_IO.pack(*_rows(x, "x", E4M3, rows, d), *_rows(x_scale, "x_scale", f32, scales, d), _dense(w, "w", E4M3, weights, d) or 0,
                          _dense(w_scale, "w_scale", f32, w_scales, d) or 0, *_rows(out, "out", dt, outs, d),
                          _dense(group_start, "group_start", torch.int32, starts, d) or 0)
    rc = (_lib or lib()).lq_product_groups(ref, io, _stream(stream))
    if rc:
        _check(rc, "lq_product_groups")


def clear_device_flags() -> None:
    """lq_clear_device_flags: the error flags stay set until this is called."""
    _check(lib().lq_clear_device_flags(), "lq_clear_device_flags")


def selftest_bounded_wait(stream=None) -> None:
    """lq_selftest_bounded_wait: one warp lets a bounded wait run out; sets bit 3 of the error flags."""
    _check(lib().lq_selftest_bounded_wait(_stream(stream)), "lq_selftest_bounded_wait")


def static_stage_bytes() -> int:
    """LQ_STATIC_STAGE_BYTES as the loaded library was built with."""
    return int(lib().lq_static_stage_bytes())


def version() -> int:
    return int(lib().lq_version())
