"""Python binding of the AdamW step (edit_adamw_* of include/edit_outer.h).

As in `outer`, this module checks tensors and passes pointers and streams; the
arithmetic runs in the library's kernels and there is no fallback.
"""
from __future__ import annotations

import ctypes
import math
from array import array
from dataclasses import dataclass
from typing import List, Optional, Sequence, Union

import torch

from .outer import (
    ADAMW_BLOCK, ADAMW_E4M3, ADAMW_F32, ADAMW_STOCHASTIC, BF16, F32, _AdamWCall, _AdamWConfig, _AdamWState, _AdamWTensors,
    _check, _stream_handle, load_library,
)

_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@dataclass
class AdamWConfig:
    """The tensors of one optimizer and its hyper-parameters."""
    numel: Sequence[int]                        # elements of each tensor
    dtype: str = "bf16"                         # of the parameters: "bf16" or "f32"
    grad_dtype: Optional[str] = None            # of the gradients; None: as the parameters
    state: str = "f32"                          # how m and v are held: "f32" or "e4m3" (8 bits)
    betas: Sequence[float] = (0.9, 0.999)
    eps: float = 1e-8
    weight_decay: float = 0.01
    decay: Optional[Sequence[float]] = None     # each tensor's factor of weight_decay; None: 1
    stochastic: bool = False                    # round bf16 parameters stochastically


@dataclass
class AdamWState:
    """m and v of every tensor: fp32, or torch.float8_e4m3fn with an fp32 scale
    for every 256 elements.  The values they stand for: code * scale."""
    exp_avg: List[torch.Tensor]
    exp_avg_sq: List[torch.Tensor]
    exp_avg_scale: Optional[List[torch.Tensor]] = None
    exp_avg_sq_scale: Optional[List[torch.Tensor]] = None


@dataclass
class AdamWRecord:
    step: int         # t
    skipped: int      # calls left out: their gradients were not finite, or their rate no rate
    norm: float       # of the last call that took one
    clip_coef: float  # c of the last call; 0 if it was left out


def _whole(value, bits: int, name: str) -> int:
    if int(value) != value or abs(int(value)) >= 2 ** bits:
        raise ValueError(f"{name} must be a whole number below 2^{bits}")
    return int(value)


class AdamW:
    """AdamW over a list of tensors, e.g. a replica's sync units, or the gains
    beside Orthogonalizer.local_step.  The handle holds t; states are the
    caller's (new_state()).  Calls on one handle, replays of graphs that hold
    them included, must not overlap: order them on one stream or with events."""

    def __init__(self, cfg: AdamWConfig, device: Optional[torch.device] = None):
        self._h = None
        self.cfg = cfg
        device = torch.device("cuda") if device is None else torch.device(device)
        if device.type != "cuda":
            raise ValueError("the handle needs a GPU device")
        c, keep = self._c_config(cfg)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self.device = device
        self._numel = [int(n) for n in cfg.numel]
        self._held = cfg.state == "e4m3"
        self._dtype, self._grad_dtype = _TYPES[cfg.dtype], _TYPES[cfg.grad_dtype or cfg.dtype]
        self._lib = load_library()
        h = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            _check(self._lib.edit_adamw_init(ctypes.byref(c), ctypes.byref(h)), "edit_adamw_init")
        self._h = h
        del keep  # the arrays that the configuration points to

    @staticmethod
    def _c_config(cfg: AdamWConfig):
        """The C configuration, and the arrays it points to."""
        grad = cfg.grad_dtype or cfg.dtype
        for name, value in (("dtype", cfg.dtype), ("grad_dtype", grad)):
            if value not in _TYPES:
                raise ValueError(f"{name} must be 'bf16' or 'f32'")
        if cfg.state not in ("f32", "e4m3"):
            raise ValueError("state must be 'f32' or 'e4m3'")
        if len(cfg.betas) != 2:
            raise ValueError("betas must be two numbers")
        count = len(cfg.numel)
        numel = (ctypes.c_int64 * max(1, count))(*[_whole(n, 63, "numel") for n in cfg.numel])
        decay = None
        if cfg.decay is not None:
            if len(cfg.decay) != count:
                raise ValueError(f"expected {count} decay factors, got {len(cfg.decay)}")
            decay = (ctypes.c_double * max(1, count))(*[float(x) for x in cfg.decay])
        c = _AdamWConfig(count, numel, decay, BF16 if cfg.dtype == "bf16" else F32, BF16 if grad == "bf16" else F32,
                         ADAMW_E4M3 if cfg.state == "e4m3" else ADAMW_F32, ADAMW_STOCHASTIC if cfg.stochastic else 0,
                         float(cfg.betas[0]), float(cfg.betas[1]), float(cfg.eps), float(cfg.weight_decay))
        return c, (numel, decay)

    # -- lifetime ------------------------------------------------------------
    def close(self) -> None:
        if getattr(self, "_h", None) is not None and self._h.value:
            with torch.cuda.device(self.device):
                self._lib.edit_adamw_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # -- tensors -------------------------------------------------------------
    def _call(self, fn, what: str, *args) -> None:
        if torch.cuda.current_device() != self.device.index:
            with torch.cuda.device(self.device):
                status = fn(self._h, *args)
        else:
            status = fn(self._h, *args)
        _check(status, what)

    def _pointers(self, tensors: Sequence, dtype: torch.dtype, what: str, per: int = 1, optional: bool = False):
        """Host array of the tensors' pointers; `per`: elements for each of theirs."""
        if len(tensors) != len(self._numel):
            raise ValueError(f"expected {len(self._numel)} tensors in {what}, got {len(tensors)}")
        place = self.device.index if self.device.type == "cuda" else -1
        out = array("Q")
        for t, n in zip(tensors, self._numel):
            if t is None and optional:
                out.append(0)
                continue
            if per != 1:
                n = -(-n // per)
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{what}[{len(out)}] must be a torch.Tensor")
            if t.dtype is not dtype or t.get_device() != place or t.numel() != n or not t.is_contiguous():
                raise ValueError(f"{what}[{len(out)}] must be a contiguous {dtype} tensor of {n} elements on {self.device}")
            out.append(t.data_ptr())
        return (ctypes.c_void_p * max(1, len(out))).from_buffer(out if out else array("Q", [0]))

    def _state_pointers(self, state: AdamWState) -> list:
        if not isinstance(state, AdamWState):
            raise TypeError("state must be an AdamWState")
        dtype = torch.float8_e4m3fn if self._held else torch.float32
        out = [self._pointers(state.exp_avg, dtype, "exp_avg"), self._pointers(state.exp_avg_sq, dtype, "exp_avg_sq")]
        scales = (state.exp_avg_scale, state.exp_avg_sq_scale)
        if not self._held:
            if any(s is not None for s in scales):
                raise ValueError("states in fp32 have no scales")
            return out + [None, None]
        for s, what in zip(scales, ("exp_avg_scale", "exp_avg_sq_scale")):
            if s is None:
                raise ValueError(f"{what} is missing")
            out.append(self._pointers(s, torch.float32, what, per=ADAMW_BLOCK))
        return out

    def _flat_views(self, dtype: torch.dtype, per: int = 1) -> List[torch.Tensor]:
        """Zeros for every tensor, in one buffer; each begins at a multiple of 256 elements."""
        sizes = [-(-n // per) for n in self._numel]
        step = ADAMW_BLOCK if per == 1 else 1
        room = [-(-n // step) * step for n in sizes]
        total = sum(room)
        if dtype == torch.float8_e4m3fn:
            flat = torch.zeros(total, dtype=torch.uint8, device=self.device).view(dtype)
        else:
            flat = torch.zeros(total, dtype=dtype, device=self.device)
        out, at = [], 0
        for n, r in zip(sizes, room):
            out.append(flat[at:at + n])
            at += r
        return out

    def new_state(self) -> AdamWState:
        """States of zeros, made on the current stream."""
        if not self._held:
            return AdamWState(self._flat_views(torch.float32), self._flat_views(torch.float32))
        codes, scale = torch.float8_e4m3fn, torch.float32
        return AdamWState(self._flat_views(codes), self._flat_views(codes), self._flat_views(scale, ADAMW_BLOCK),
                          self._flat_views(scale, ADAMW_BLOCK))

    # -- the step --------------------------------------------------------------
    def prepare_grads(self, grads: Sequence[Optional[torch.Tensor]]) -> "GradPlan":
        """Check the gradients once, for calls that take only them."""
        return GradPlan(self, grads)

    def prepare(self, params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]],
                state: AdamWState) -> "AdamWPlan":
        """Check a step's tensors once; AdamWPlan.run() is then one
        edit_adamw_step call with no per-tensor Python work."""
        return AdamWPlan(self, params, grads, state)

    def step(self, params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]], state: AdamWState,
             lr: Union[float, torch.Tensor], max_norm: Optional[float] = None, sumsq: Optional[torch.Tensor] = None,
             seed: int = 0, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Enqueue one step of all tensors, in place on `params` and `state`; see AdamWPlan.run."""
        AdamWPlan(self, params, grads, state).run(lr, max_norm, sumsq, seed, stream)

    def sum_squares(self, grads: Sequence[Optional[torch.Tensor]], out: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Enqueue S = sum of g^2 over all gradients; see GradPlan.sum_squares."""
        return GradPlan(self, grads).sum_squares(out, stream)

    # -- states ----------------------------------------------------------------
    def pack(self, exp_avg: Sequence[torch.Tensor], exp_avg_sq: Sequence[torch.Tensor], state: Optional[AdamWState] = None,
             seed: int = 0, stream: Optional[torch.cuda.Stream] = None) -> AdamWState:
        """Enqueue the change of fp32 states to 8-bit ones (edit_adamw_pack) and return those."""
        m = self._pointers(exp_avg, torch.float32, "exp_avg")
        v = self._pointers(exp_avg_sq, torch.float32, "exp_avg_sq")
        if state is None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
                state = self.new_state()
        tensors = _AdamWTensors(None, None, *self._state_pointers(state))
        self._call(self._lib.edit_adamw_pack, "edit_adamw_pack", m, v, ctypes.byref(tensors), _seed(seed),
                   _stream_handle(stream, self.device))
        return state

    def unpack(self, state: AdamWState, exp_avg: Optional[Sequence[torch.Tensor]] = None,
               exp_avg_sq: Optional[Sequence[torch.Tensor]] = None, stream: Optional[torch.cuda.Stream] = None) -> tuple:
        """Enqueue the values of 8-bit states in fp32 (edit_adamw_unpack) and return (exp_avg, exp_avg_sq)."""
        tensors = _AdamWTensors(None, None, *self._state_pointers(state))
        if exp_avg is None or exp_avg_sq is None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(self.device)):
                exp_avg = self._flat_views(torch.float32) if exp_avg is None else exp_avg
                exp_avg_sq = self._flat_views(torch.float32) if exp_avg_sq is None else exp_avg_sq
        self._call(self._lib.edit_adamw_unpack, "edit_adamw_unpack", ctypes.byref(tensors),
                   self._pointers(exp_avg, torch.float32, "exp_avg"),
                   self._pointers(exp_avg_sq, torch.float32, "exp_avg_sq"), _stream_handle(stream, self.device))
        return exp_avg, exp_avg_sq

    def state_get(self) -> AdamWRecord:
        """The record of the last call, after waiting for the device."""
        st = _AdamWState()
        self._call(self._lib.edit_adamw_state_get, "edit_adamw_state_get", ctypes.byref(st))
        return AdamWRecord(int(st.step), int(st.skipped), float(st.norm), float(st.clip_coef))

    def state_set(self, step: int) -> None:
        """t of a run that is resumed; waits for the device."""
        self._call(self._lib.edit_adamw_state_set, "edit_adamw_state_set", _whole(step, 63, "step"))


def _seed(seed: int) -> int:
    if int(seed) != seed or not 0 <= int(seed) < 2 ** 64:
        raise ValueError("seed must be a whole number from 0 to 2^64 - 1")
    return int(seed)


class GradPlan:
    """Checked gradients.  The plan keeps the tensors alive; their storage must
    not be reallocated while it is used."""

    def __init__(self, handle: AdamW, grads: Sequence[Optional[torch.Tensor]]):
        self._handle = handle
        self._grads = list(grads)
        self._grad = handle._pointers(self._grads, handle._grad_dtype, "grads", optional=True)

    def sum_squares(self, out: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
        """Enqueue S = sum of g^2 (edit_adamw_sumsq) and return `out`, one fp64
        element.  The shards of a module add theirs up for AdamWPlan.run's `sumsq`."""
        h = self._handle
        if out is None:
            with torch.cuda.stream(stream if stream is not None else torch.cuda.current_stream(h.device)):
                out = torch.empty(1, dtype=torch.float64, device=h.device)
        h._call(h._lib.edit_adamw_sumsq, "edit_adamw_sumsq", self._grad, _scalar(h, out, "out"),
                _stream_handle(stream, h.device))
        return out


class AdamWPlan(GradPlan):
    """A step's checked tensors.  The plan keeps them alive; their storage must
    not be reallocated while it is used."""

    def __init__(self, handle: AdamW, params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]],
                 state: AdamWState):
        super().__init__(handle, grads)
        self._params = list(params)
        self._tensors = _AdamWTensors(handle._pointers(self._params, handle._dtype, "params"), self._grad,
                                      *handle._state_pointers(state))
        self._call_args = _AdamWCall()
        # the tensors, whatever becomes of the caller's lists
        self._state = [list(x or []) for x in (state.exp_avg, state.exp_avg_sq, state.exp_avg_scale, state.exp_avg_sq_scale)]

    def run(self, lr: Union[float, torch.Tensor], max_norm: Optional[float] = None, sumsq: Optional[torch.Tensor] = None,
            seed: int = 0, stream: Optional[torch.cuda.Stream] = None) -> None:
        """Enqueue one step (edit_adamw_step).  `lr`: a number, or one fp64
        element on the device, read when the step runs; one that is negative or not
        finite leaves the whole call out.  `max_norm` clips the gradients' norm;
        `sumsq` is its square where it covers more than these gradients.  With
        either, gradients that are not finite leave the call out too.  `seed`: of
        the random numbers, which differ from step to step."""
        h = self._handle
        if max_norm is not None and not (max_norm > 0.0 and math.isfinite(max_norm)):
            raise ValueError("max_norm must be finite and > 0, or None")
        call = self._call_args
        device_lr = isinstance(lr, torch.Tensor)
        call.lr, call.lr_device = (0.0, _scalar(h, lr, "lr")) if device_lr else (float(lr), None)
        call.max_norm = 0.0 if max_norm is None else float(max_norm)
        call.sumsq = None if sumsq is None else _scalar(h, sumsq, "sumsq")
        call.seed = _seed(seed)
        h._call(h._lib.edit_adamw_step, "edit_adamw_step", ctypes.byref(self._tensors), ctypes.byref(call),
                _stream_handle(stream, h.device))


def _scalar(h: AdamW, t: torch.Tensor, what: str) -> int:
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch.Tensor")
    if t.device != h.device or t.dtype != torch.float64 or t.numel() != 1:
        raise ValueError(f"{what} must be one float64 element on {h.device}")
    return t.data_ptr()
