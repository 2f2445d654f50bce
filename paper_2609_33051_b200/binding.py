"""ctypes binding of libsketchssm.so: argument marshalling only.

Every step of the decode path runs in the CUDA library; this module converts
torch tensors to raw device pointers, forwards the calls with the same names as
the C ABI and raises on a non-zero status.  There is no fallback: if the shared
library is missing or CUDA is unavailable the calls fail.
"""
from __future__ import annotations

import contextlib
import ctypes
import importlib.util
import os
from typing import Optional

import torch

from . import build as _build

KIND = {"mamba2": 0, "gdn": 1, "kda": 2}
DTYPE = {"f32": 0, "bf16": 1}
TORCH_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
NO_SKETCH = 0x1
NO_APPEND = 0x1
SILU = 0x1
SIGMOID = 0x1

EXPORTED = (
    "sketchssm_create", "sketchssm_destroy", "sketchssm_query_sizes", "sketchssm_bind",
    "sketchssm_state_update", "sketchssm_decode_step", "sketchssm_full_read_decode",
    "sketchssm_read_status", "sketchssm_last_launch_count", "sketchssm_tune",
    "sketchssm_status_string", "sketchssm_version", "sketchssm_last_cuda_error", "sketchssm_step_host",
    "sketchssm_decode_step_static", "sketchssm_selftest_wait_timeout", "sketchssm_step_mixed",
    "sketchssm_causal_conv", "sketchssm_conv_step", "sketchssm_prompt_work_bytes", "sketchssm_prompt_scan",
    "sketchssm_rms_norm", "sketchssm_scaled_matmul",
    "sketchssm_delta_step", "sketchssm_delta_work_bytes", "sketchssm_delta_scan", "sketchssm_integer_norm", "sketchssm_integer_matmul",
)
OP_DECODE, OP_FULL_READ, OP_UPDATE = 0, 1, 2


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in
                ("kind", "batch", "heads", "dk", "dv", "rank", "buf_len", "io_dtype", "out_dtype", "device",
                 "coef_per_seq", "coef_pivots")] + [("ridge_lambda", ctypes.c_float), ("sketch_dtype", ctypes.c_int32),
                                                            ("erase_factors", ctypes.c_int32)]


class Sizes(ctypes.Structure):
    _fields_ = [(n, ctypes.c_size_t) for n in
                ("state_bytes", "sketch_bytes", "ring_bytes", "omega_bytes", "coef_bytes", "status_bytes",
                 "work_bytes", "ring_head_bytes", "ring_v_offset", "ring_beta_offset", "ring_decay_offset", "alignment",
                 "erase_bytes")]


class Buffers(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("state", "sketch", "ring", "omega", "coef", "status", "work", "head_rank",
                                                "erase")]


class Staging(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("q", "k", "v", "beta", "decay", "out")]


class PromptBatch(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int32), ("tokens", ctypes.c_int32)] + [(n, ctypes.c_void_p) for n in
                                                                             ("starts", "slots", "resume")]


class Prompts:
    """Prompts packed one behind another along the token axis: sequence i is the rows starts[i] .. starts[i + 1] - 1 of `tokens`.

    starts [N + 1], slots [N] (the batch entry that keeps a sequence's state; None: i) and resume [N] (the batch entry whose
    state it goes on from, -1: none; None: no sequence does) are int32 tensors on the device, read when the kernels run."""

    def __init__(self, starts: torch.Tensor, tokens: int, slots: Optional[torch.Tensor] = None,
                 resume: Optional[torch.Tensor] = None):
        self.sequences, self.tokens = starts.numel() - 1, int(tokens)
        if self.sequences < 0 or not 0 <= self.tokens < 2 ** 31:
            raise ValueError("starts holds one row number more than there are sequences, and tokens is not negative (and an int32)")
        for name, t, n in (("starts", starts, self.sequences + 1), ("slots", slots, self.sequences), ("resume", resume, self.sequences)):
            if t is not None and (t.dtype != torch.int32 or t.dim() != 1 or t.numel() != n or not t.is_contiguous()):
                raise ValueError(f"{name} is a dense int32 tensor of {n} entries")
        self.starts, self.slots, self.resume = starts, slots, resume
        self.c = PromptBatch(self.sequences, self.tokens, _ptr(starts), _ptr(slots), _ptr(resume))
        self.address, self.device = ctypes.addressof(self.c), starts.device
        if any(t is not None and t.device != starts.device for t in (slots, resume)):
            raise ValueError("starts, slots and resume lie on one device")

    def on(self, device: torch.device) -> bool:
        return self.device == device


def on_stream(stream):
    """Tensors made under it may be dropped as soon as what uses them is in `stream`'s queue (None: the current stream, as always):
    their memory is then given only to later work of that stream."""
    return contextlib.nullcontext() if stream is None else torch.cuda.stream(stream)


class SketchSSMError(RuntimeError):
    def __init__(self, fn: str, status: int, text: str):
        super().__init__(f"{fn} failed: {text} ({status})")
        self.status = status


_LIB = None
_CALLS = None       # the extension module that checks tensors and calls the library for the operators around the recurrence


def load_library(path: Optional[str] = None) -> ctypes.CDLL:
    """Load libsketchssm.so (built in-tree by build.py) and declare the prototypes."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    path = path or _build.LIB_PATH
    if not os.path.exists(path):
        raise FileNotFoundError(
            f"{path} not found: build it with `python -m paper_2609_33051_b200.build` (needs nvcc)")
    lib = ctypes.CDLL(path)
    vp, i32, u32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint32
    lib.sketchssm_create.argtypes = [ctypes.POINTER(Config), ctypes.POINTER(vp)]
    lib.sketchssm_destroy.argtypes = [vp]
    lib.sketchssm_query_sizes.argtypes = [vp, ctypes.POINTER(Sizes)]
    lib.sketchssm_bind.argtypes = [vp, ctypes.POINTER(Buffers)]
    for name in ("sketchssm_state_update", "sketchssm_decode_step", "sketchssm_full_read_decode",
                 "sketchssm_decode_step_static"):
        getattr(lib, name).argtypes = [vp, i32, vp, vp, vp, vp, vp, vp, u32, vp]
    lib.sketchssm_step_mixed.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, u32, vp]
    lib.sketchssm_step_host.argtypes = [vp, i32, i32, vp, vp, vp, vp, vp, vp, ctypes.POINTER(Staging), u32, vp]
    lib.sketchssm_selftest_wait_timeout.argtypes = [vp, i32, i32, vp]
    i64 = ctypes.c_int64
    pb = ctypes.POINTER(PromptBatch)
    lib.sketchssm_causal_conv.argtypes = [vp, pb, i32, i32, vp, vp, vp, vp, i64, vp, i64, u32, vp]
    lib.sketchssm_conv_step.argtypes = [vp, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sketchssm_prompt_work_bytes.argtypes = [vp, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.sketchssm_prompt_scan.argtypes = [vp, pb, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, i64, i32, vp,
                                          ctypes.c_size_t, vp]
    lib.sketchssm_rms_norm.argtypes = [vp, i32, i32, i32, ctypes.c_float, vp, i64, i32, vp, vp, vp, vp, i64, vp, i64, vp, i32,
                                       vp, vp, vp, vp]
    lib.sketchssm_scaled_matmul.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, i64, i32, vp]
    f32 = ctypes.c_float
    lib.sketchssm_delta_step.argtypes = [vp, i32, i32, f32, f32, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, vp, vp, vp, vp, vp, vp, vp]
    lib.sketchssm_delta_work_bytes.argtypes = [vp, i32, i32, ctypes.POINTER(ctypes.c_size_t)]
    lib.sketchssm_delta_scan.argtypes = [vp, pb, i32, f32, f32, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp, vp, vp, i64, i32, vp,
                                         ctypes.c_size_t, vp]
    lib.sketchssm_integer_norm.argtypes = [vp, i32, i32, i32, f32, vp, i64, i32, vp, vp, vp, vp, i64, u32, vp, vp, vp, vp]
    lib.sketchssm_integer_matmul.argtypes = [vp, i32, i32, i32, vp, vp, vp, vp, vp, i64, i32, vp]
    lib.sketchssm_read_status.argtypes = [vp, ctypes.POINTER(ctypes.c_int32 * 4), vp]
    lib.sketchssm_last_launch_count.argtypes = [vp]
    lib.sketchssm_tune.argtypes = [vp, ctypes.c_char_p, i32]
    lib.sketchssm_status_string.argtypes = [i32]
    lib.sketchssm_status_string.restype = ctypes.c_char_p
    lib.sketchssm_version.restype = ctypes.c_char_p
    lib.sketchssm_last_cuda_error.argtypes = [vp]
    lib.sketchssm_last_cuda_error.restype = ctypes.c_char_p
    for name in EXPORTED:
        if name not in ("sketchssm_status_string", "sketchssm_version", "sketchssm_last_cuda_error"):
            getattr(lib, name).restype = ctypes.c_int
    if path == _build.LIB_PATH:
        _LIB = lib
    return lib


def _calls():
    """The extension module, loaded with the first call that needs it: the decode calls do without."""
    global _CALLS
    if _CALLS is None:
        path = _build.calls_path()
        if not os.path.exists(path):
            raise FileNotFoundError(
                f"{path} not found: build it with `python -m paper_2609_33051_b200.build` (needs a C++ compiler and torch's headers)")
        spec = importlib.util.spec_from_file_location(__package__ + "._layer_calls", path)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _CALLS = module
    return _CALLS


_RAW_STREAM, _DEVICE = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()       # (the declared argument types make the C pointer of it)


class SketchSSM:
    """One layer's decode state on one GPU: owns the torch buffers, forwards to the C ABI.

    Tensors (all on `device`): state [B,H,K,V] f32, sketch [B,H,r,V] f32, ring (bytes),
    omega [H,K,r] f32, coef [H,r,K] f32 (or [B,H,r,K] with coef_per_seq: the state-dependent map that every
    state update rebuilds).  Token arguments follow the C header:
    q,k [B,H,K] io; v [B,H,V] io; beta [B,H] f32; decay [B,H] f32 or [B,H,K] io (KDA).
    With erase_factors (GDN / KDA) the decode step forms c_t from projected erase vectors kept in `erase` [B,H,L,r] f32.
    """

    def __init__(self, kind: str, batch: int, heads: int, dk: int, dv: int, rank: int, buf_len: int,
                 io: str = "bf16", out: str = "f32", device: int = 0, allocate: bool = True,
                 coef_per_seq: bool = False, coef_pivots: int = 4, ridge_lambda: float = 0.1, sketch: str = "f32",
                 erase_factors: bool = False):
        self.lib = load_library()
        self.kind, self.io, self.out = kind, io, out
        self.B, self.H, self.K, self.V, self.R, self.L = batch, heads, dk, dv, rank, buf_len
        self.device = torch.device("cuda", device)
        self.coef_per_seq = bool(coef_per_seq)
        self.cfg = Config(KIND[kind], batch, heads, dk, dv, rank, buf_len, DTYPE[io], DTYPE[out], device,
                          int(self.coef_per_seq), coef_pivots, ridge_lambda, DTYPE[sketch], int(bool(erase_factors)))
        self.erase_factors = bool(erase_factors)
        self.sketch_dtype = sketch
        self._ctx = ctypes.c_void_p()
        self._check("sketchssm_create", self.lib.sketchssm_create(ctypes.byref(self.cfg), ctypes.byref(self._ctx)))
        self.sizes = Sizes()
        self._check("sketchssm_query_sizes", self.lib.sketchssm_query_sizes(self._ctx, ctypes.byref(self.sizes)))
        self.state = self.sketch = self.ring = self.omega = self.coef = self.status = self.work = self.erase = None
        self._heads()
        self.head_rank = None        # optional int32 [H] device tensor: per-head sketch rank (0 = full-state read); set, then bind()
        if allocate:
            self.allocate()

    # -- memory -----------------------------------------------------------------------------
    def allocate(self):
        d = self.device
        self.state = torch.zeros(self.B, self.H, self.K, self.V, dtype=torch.float32, device=d)
        self.sketch = torch.zeros(self.B, self.H, self.R, self.V, dtype=TORCH_DTYPE[self.sketch_dtype], device=d)
        self.ring = torch.zeros(self.sizes.ring_bytes, dtype=torch.uint8, device=d)
        self.omega = torch.zeros(self.H, self.K, self.R, dtype=torch.float32, device=d)
        self.coef = torch.zeros(*((self.B,) if self.coef_per_seq else ()), self.H, self.R, self.K,
                                dtype=TORCH_DTYPE[self.sketch_dtype], device=d)
        self.status = torch.zeros(self.sizes.status_bytes // 4, dtype=torch.int32, device=d)
        self.work = torch.zeros(self.sizes.work_bytes // 4, dtype=torch.float32, device=d)
        if self.erase_factors:
            self.erase = torch.zeros(self.B, self.H, self.L, self.R, dtype=TORCH_DTYPE[self.sketch_dtype], device=d)
        self.bind()

    def bind(self):
        assert self.state.numel() * 4 == self.sizes.state_bytes
        assert self.sketch.numel() * self.sketch.element_size() == self.sizes.sketch_bytes
        assert self.ring.numel() == self.sizes.ring_bytes
        b = Buffers(self.state.data_ptr(), self.sketch.data_ptr(), self.ring.data_ptr(),
                    self.omega.data_ptr(), self.coef.data_ptr(), self.status.data_ptr(), self.work.data_ptr(),
                    self.head_rank.data_ptr() if self.head_rank is not None else None,
                    self.erase.data_ptr() if self.erase is not None else None)
        self._check("sketchssm_bind", self.lib.sketchssm_bind(self._ctx, ctypes.byref(b)))

    def _heads(self):
        """What the calls of _layer_calls begin with: the C function, the context, the device and the layer's sizes."""
        def head(fn):
            return (ctypes.cast(fn, ctypes.c_void_p).value, self._ctx.value or 0, self.device.index or 0, self.B, self.H, self.K,
                    self.V, DTYPE[self.io])
        lib = self.lib
        self._conv, self._step, self._scan = (head(f) for f in (lib.sketchssm_causal_conv, lib.sketchssm_conv_step, lib.sketchssm_prompt_scan))
        self._norm, self._matmul = head(lib.sketchssm_rms_norm), head(lib.sketchssm_scaled_matmul)
        self._delta_step, self._delta_scan = (head(f) + (KIND[self.kind],) for f in (lib.sketchssm_delta_step, lib.sketchssm_delta_scan))
        self._norm8, self._matmul8 = head(lib.sketchssm_integer_norm), head(lib.sketchssm_integer_matmul)

    def close(self):
        if self._ctx:
            self.lib.sketchssm_destroy(self._ctx)
            self._ctx = ctypes.c_void_p()
            self._heads()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- helpers ------------------------------------------------------------------------------
    def _check(self, fn: str, rc: int):
        if rc != 0:
            text = self.lib.sketchssm_status_string(rc).decode()
            if rc == -4 and self._ctx:
                text += ": " + self.lib.sketchssm_last_cuda_error(self._ctx).decode()
            raise SketchSSMError(fn, rc, text)

    @staticmethod
    def _stream(stream) -> int:
        """The stream's handle; None: the current stream of the current device (where torch offers it, read without
        building a Stream object, which costs as much as the rest of a call's marshalling)."""
        if stream is not None:
            return stream.cuda_stream
        if _RAW_STREAM is None or _DEVICE is None:
            return torch.cuda.current_stream().cuda_stream
        return _RAW_STREAM(_DEVICE())

    def new_output(self) -> torch.Tensor:
        return torch.empty(self.B, self.H, self.V, dtype=TORCH_DTYPE[self.out], device=self.device)

    def ring_views(self):
        """Typed views of the ring: k [B,H,L,K], v [B,H,L,V], beta [B,H,L], decay [B,H,L] or [B,H,L,K]."""
        hb = self.sizes.ring_head_bytes
        raw = self.ring.view(self.B, self.H, hb)
        iod = TORCH_DTYPE[self.io]
        k = raw[..., : self.sizes.ring_v_offset].view(iod).view(self.B, self.H, self.L, self.K)
        v = raw[..., self.sizes.ring_v_offset: self.sizes.ring_beta_offset].view(iod).view(self.B, self.H, self.L, self.V)
        beta = raw[..., self.sizes.ring_beta_offset: self.sizes.ring_decay_offset].view(torch.float32)
        dec = raw[..., self.sizes.ring_decay_offset:]
        dec = dec.view(iod).view(self.B, self.H, self.L, self.K) if self.kind == "kda" else dec.view(torch.float32)
        return k, v, beta, dec

    # -- the C ABI calls --------------------------------------------------------------------
    def state_update(self, n_before: int, q=None, k=None, v=None, beta=None, decay=None, out=None,
                     flags: int = 0, stream=None):
        rc = self.lib.sketchssm_state_update(self._ctx, n_before, _ptr(q), _ptr(k), _ptr(v), _ptr(beta),
                                             _ptr(decay), _ptr(out), flags, self._stream(stream))
        if rc:
            self._check("sketchssm_state_update", rc)
        return out

    def decode_step(self, n_before: int, q, k, v, beta, decay, out, flags: int = 0, stream=None):
        rc = self.lib.sketchssm_decode_step(self._ctx, n_before, _ptr(q), _ptr(k), _ptr(v), _ptr(beta),
                                            _ptr(decay), _ptr(out), flags, self._stream(stream))
        if rc:
            self._check("sketchssm_decode_step", rc)
        return out

    def decode_step_static(self, n_before: int, q, k, v, beta, decay, out, flags: int = 0, stream=None):
        """sketchssm_decode_step_static: the decode step for callers that can neither allocate nor supply
        scratch; its kernel-to-kernel hand-off uses the library's fixed 4 MiB device array."""
        rc = self.lib.sketchssm_decode_step_static(self._ctx, n_before, _ptr(q), _ptr(k), _ptr(v), _ptr(beta),
                                                   _ptr(decay), _ptr(out), flags, self._stream(stream))
        if rc:
            self._check("sketchssm_decode_step_static", rc)
        return out

    def step_mixed(self, phase: torch.Tensor, q, k, v, beta, decay, out, stream=None):
        """sketchssm_step_mixed: one step for sequences at different window phases; phase is an int32 [B] device tensor
        (n >= 0: decode step at ring fill n; -(n + 1): flush with n buffered tokens plus the current one)."""
        assert phase.dtype == torch.int32 and phase.is_cuda and phase.numel() == self.B
        rc = self.lib.sketchssm_step_mixed(self._ctx, _ptr(phase), _ptr(q), _ptr(k), _ptr(v), _ptr(beta), _ptr(decay),
                                           _ptr(out), 0, self._stream(stream))
        if rc:
            self._check("sketchssm_step_mixed", rc)
        return out

    def full_read_decode(self, n_before: int, q, k, v, beta, decay, out, flags: int = 0, stream=None):
        rc = self.lib.sketchssm_full_read_decode(self._ctx, n_before, _ptr(q), _ptr(k), _ptr(v), _ptr(beta),
                                                 _ptr(decay), _ptr(out), flags, self._stream(stream))
        if rc:
            self._check("sketchssm_full_read_decode", rc)
        return out

    def new_token_buffers(self, pinned_host: bool = False):
        """Empty q, k, v, beta, decay, out tensors of the C ABI's shapes: on the device, or page-locked host."""
        iod = TORCH_DTYPE[self.io]
        kw = dict(device="cpu", pin_memory=True) if pinned_host else dict(device=self.device)
        dec = (torch.empty(self.B, self.H, self.K, dtype=iod, **kw) if self.kind == "kda"
               else torch.empty(self.B, self.H, dtype=torch.float32, **kw))
        return dict(q=torch.empty(self.B, self.H, self.K, dtype=iod, **kw),
                    k=torch.empty(self.B, self.H, self.K, dtype=iod, **kw),
                    v=torch.empty(self.B, self.H, self.V, dtype=iod, **kw),
                    beta=torch.empty(self.B, self.H, dtype=torch.float32, **kw), decay=dec,
                    out=torch.empty(self.B, self.H, self.V, dtype=TORCH_DTYPE[self.out], **kw))

    def step_host(self, op: int, n_before: int, host: dict, staging: dict, flags: int = 0, stream=None):
        """sketchssm_step_host: host token tensors in, host output out, copies and kernel on one stream."""
        st = Staging(*[staging[n].data_ptr() for n in ("q", "k", "v", "beta", "decay", "out")])
        rc = self.lib.sketchssm_step_host(self._ctx, op, n_before, _ptr(host["q"]), _ptr(host["k"]), _ptr(host["v"]),
                                          _ptr(host["beta"]), _ptr(host["decay"]), _ptr(host["out"]),
                                          ctypes.byref(st), flags, self._stream(stream))
        if rc:
            self._check("sketchssm_step_host", rc)
        return host["out"]

    # -- the operators around the recurrence ---------------------------------------------------
    def new_conv_state(self, channels: int, width: int) -> torch.Tensor:
        """Zeroed stored rows [B, width - 1, channels] of the short convolution."""
        return torch.zeros(self.B, width - 1, channels, dtype=TORCH_DTYPE[self.io], device=self.device)

    def causal_conv(self, prompts: Prompts, x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor],
                    state: torch.Tensor, out: torch.Tensor, silu: bool = True, stream=None) -> torch.Tensor:
        """sketchssm_causal_conv: the short causal convolution of packed prompts x [T, C] into out; weight [C, W] f32, bias [C]
        f32 or None, state [B, W - 1, C] holds the stored rows and is moved on."""
        if not prompts.on(self.device):
            raise ValueError("prompts lie on the layer's device")
        rc = (_CALLS or _calls()).causal_conv(*self._conv, prompts.address, prompts.tokens, x, weight, bias, state, out, SILU if silu else 0,
                                self._stream(stream))
        if rc:
            self._check("sketchssm_causal_conv", rc)
        return out

    def conv_step(self, x: torch.Tensor, dt: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor],
                  state: torch.Tensor, a: torch.Tensor, dt_bias: Optional[torch.Tensor], token: dict, groups: int = 1,
                  stream=None) -> dict:
        """sketchssm_conv_step: one token of every batch entry, x [B, H V + 2 G K] and dt [B, H], into the q, k, v, beta, decay of
        `token` (new_token_buffers), which the decode calls take."""
        rc = (_CALLS or _calls()).conv_step(*self._step, x, dt, weight, bias, state, a, dt_bias, token["q"], token["k"], token["v"], token["beta"],
                              token["decay"], groups, self._stream(stream))
        if rc:
            self._check("sketchssm_conv_step", rc)
        return token

    def new_prompt_work(self, sequences: int, tokens: int) -> Optional[torch.Tensor]:
        """Scratch of prompt_scan for batches of at most this many sequences and tokens (None: none is needed)."""
        n = ctypes.c_size_t()
        self._check("sketchssm_prompt_work_bytes", self.lib.sketchssm_prompt_work_bytes(self._ctx, sequences, tokens, ctypes.byref(n)))
        return torch.empty(n.value, dtype=torch.uint8, device=self.device) if n.value else None

    def prompt_scan(self, prompts: Prompts, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, dt: torch.Tensor, a: torch.Tensor,
                    out: torch.Tensor, dt_bias: Optional[torch.Tensor] = None, skip: Optional[torch.Tensor] = None,
                    work: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """sketchssm_prompt_scan: the selective scan of packed prompts, q, k [T, G, K], v [T, H, V], dt [T, H] in io, a [H] f32, into
        out [T, H, V] (f32 or bf16) and the bound state.  work: new_prompt_work (allocated here if None)."""
        if not prompts.on(self.device):
            raise ValueError("prompts lie on the layer's device")
        if work is None:
            with on_stream(stream):
                work = self.new_prompt_work(prompts.sequences, prompts.tokens)
        rc = (_CALLS or _calls()).prompt_scan(*self._scan, prompts.address, prompts.tokens, q, k, v, dt, a, out, dt_bias, skip, work, self._stream(stream))
        if rc:
            self._check("sketchssm_prompt_scan", rc)
        return out

    def rms_norm(self, x: torch.Tensor, weight: torch.Tensor, out: Optional[torch.Tensor] = None,
                 out8: Optional[torch.Tensor] = None, scale: Optional[torch.Tensor] = None,
                 residual: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None,
                 gate: Optional[torch.Tensor] = None, skip: Optional[torch.Tensor] = None,
                 skip_weight: Optional[torch.Tensor] = None, eps: float = 1e-5, group: int = 0, stream=None):
        """sketchssm_rms_norm: the norm of x [T, D] (f32 or bf16) with the residual's addition, or the skip and the gate, before it;
        into out (io) and/or out8 [T, D] e4m3 with scale [T, ceil(D / 128)]."""
        rc = (_CALLS or _calls()).rms_norm(*self._norm, x, weight, out, out8, scale, residual, residual_out, gate, skip, skip_weight, eps, group,
                             self._stream(stream))
        if rc:
            self._check("sketchssm_rms_norm", rc)
        return out if out is not None else out8

    def scaled_matmul(self, a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, out: torch.Tensor,
                      stream=None) -> torch.Tensor:
        """sketchssm_scaled_matmul: out [M, N] (f32 or bf16) = a [M, K] w [N, K]^T in e4m3, with a_scale [M, ceil(K / 128)] and
        w_scale [ceil(N / 128), ceil(K / 128)]."""
        rc = (_CALLS or _calls()).scaled_matmul(*self._matmul, a, a_scale, w, w_scale, out, self._stream(stream))
        if rc:
            self._check("sketchssm_scaled_matmul", rc)
        return out

    # -- the delta rule's layer, and 8-bit integers ---------------------------------------------
    def delta_step(self, x: torch.Tensor, b: torch.Tensor, dt: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor],
                   state: torch.Tensor, a: torch.Tensor, dt_bias: Optional[torch.Tensor], token: dict, groups: int = 1, eps: float = 1e-6,
                   q_scale: Optional[float] = None, stream=None) -> dict:
        """sketchssm_delta_step (GDN, KDA): one token of every batch entry, x [B, H V + 2 G K], b [B, H] and dt [B, H] (GDN) or [B, H K] (KDA),
        into the q, k, v, beta, decay of `token` (new_token_buffers), which the decode calls take.  dt_bias [H] or [H, K].
        q_scale: None for 1 / sqrt(K)."""
        rc = (_CALLS or _calls()).delta_step(*self._delta_step, x, b, dt, weight, bias, state, a, dt_bias, token["q"], token["k"], token["v"],
                               token["beta"], token["decay"], groups, eps, self.K ** -0.5 if q_scale is None else q_scale, self._stream(stream))
        if rc:
            self._check("sketchssm_delta_step", rc)
        return token

    def new_delta_work(self, sequences: int, tokens: int) -> Optional[torch.Tensor]:
        """Scratch of delta_scan for batches of at most this many sequences and tokens (None: none is needed)."""
        n = ctypes.c_size_t()
        self._check("sketchssm_delta_work_bytes", self.lib.sketchssm_delta_work_bytes(self._ctx, sequences, tokens, ctypes.byref(n)))
        return torch.empty(n.value, dtype=torch.uint8, device=self.device) if n.value else None

    def delta_scan(self, prompts: Prompts, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, b: torch.Tensor, dt: torch.Tensor,
                   a: torch.Tensor, out: torch.Tensor, dt_bias: Optional[torch.Tensor] = None, eps: float = 1e-6,
                   q_scale: Optional[float] = None, work: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """sketchssm_delta_scan (GDN, KDA): the gated delta rule over packed prompts, q, k [T, G, K] (not normalised), v [T, H, V], b [T, H],
        dt [T, H] (GDN) or [T, H K] (KDA) in io, a [H] f32, dt_bias [H] or [H, K] f32, into out [T, H, V] (f32 or bf16) and the
        bound state.  q_scale: None for 1 / sqrt(K).  work: new_delta_work (allocated here if None and needed)."""
        if not prompts.on(self.device):
            raise ValueError("prompts lie on the layer's device")
        if work is None and not (self.kind == "gdn" and out.dtype == torch.float32):      # (needs none)
            with on_stream(stream):
                work = self.new_delta_work(prompts.sequences, prompts.tokens)
        rc = (_CALLS or _calls()).delta_scan(*self._delta_scan, prompts.address, prompts.tokens, q, k, v, b, dt, a, out, dt_bias, work, eps,
                               self.K ** -0.5 if q_scale is None else q_scale, self._stream(stream))
        if rc:
            self._check("sketchssm_delta_scan", rc)
        return out

    def integer_norm(self, x: torch.Tensor, weight: torch.Tensor, out8: torch.Tensor, scale: torch.Tensor, out: Optional[torch.Tensor] = None,
                  residual: Optional[torch.Tensor] = None, residual_out: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                  act: str = "silu", eps: float = 1e-5, stream=None) -> torch.Tensor:
        """sketchssm_integer_norm: the norm of x [T, D] (f32 or bf16) in groups of len(weight), after the residual's addition, or with the gate
        (through `act`, "silu" or "sigmoid") behind it; into out8 [T, D] int8 with scale [T], and out (io) if wanted."""
        if act not in ("silu", "sigmoid"):
            raise ValueError("act is silu or sigmoid")
        rc = (_CALLS or _calls()).integer_norm(*self._norm8, x, weight, out8, scale, out, residual, residual_out, gate, SIGMOID if act == "sigmoid" else 0,
                              eps, self._stream(stream))
        if rc:
            self._check("sketchssm_integer_norm", rc)
        return out8

    def integer_matmul(self, a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor, out: torch.Tensor,
                    stream=None) -> torch.Tensor:
        """sketchssm_integer_matmul: out [M, N] (f32 or bf16) = a [M, K] w [N, K]^T of 8-bit integers, with a_scale [M] and w_scale [N]."""
        rc = (_CALLS or _calls()).integer_matmul(*self._matmul8, a, a_scale, w, w_scale, out, self._stream(stream))
        if rc:
            self._check("sketchssm_integer_matmul", rc)
        return out

    def selftest_wait_timeout(self, poll_limit: int = 2048, where: int = 99, stream=None):
        """sketchssm_selftest_wait_timeout: one warp whose bounded wait runs out and reports through the status block."""
        self._check("sketchssm_selftest_wait_timeout",
                    self.lib.sketchssm_selftest_wait_timeout(self._ctx, poll_limit, where, self._stream(stream)))

    def read_status(self, stream=None):
        detail = (ctypes.c_int32 * 4)()
        rc = self.lib.sketchssm_read_status(self._ctx, ctypes.byref(detail), self._stream(stream))
        return rc, list(detail)

    def check_status(self, stream=None):
        rc, detail = self.read_status(stream)
        if rc != 0:
            raise SketchSSMError("sketchssm_read_status", rc,
                                 self.lib.sketchssm_status_string(rc).decode() + f" detail={detail}")

    def last_launch_count(self) -> int:
        return self.lib.sketchssm_last_launch_count(self._ctx)

    def tune(self, key: str, value: int):
        self._check("sketchssm_tune", self.lib.sketchssm_tune(self._ctx, key.encode(), value))
