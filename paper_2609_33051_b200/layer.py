"""Layers served with the library: prompts first, then one token after another through the sketched decode.

Mamba2Layer:

    x -> norm (with the residual's addition, 8 bits) -> first projection -> [gate | values, keys, queries | step sizes]
      -> short convolution -> recurrence (scan of a prompt, or a step of the windowed decode) + skip
      -> gate and norm (8 bits) -> second projection

DeltaLayer (GDN, KDA):

    x -> norm (with the residual's addition, 8-bit integers) -> first projection -> [gate | values, keys, queries | step sizes | decays]
      -> short convolution -> recurrence with unit keys and queries (scan of a prompt, or a step of the windowed decode)
      -> every head's norm and gate (8-bit integers) -> second projection

Every step runs in the CUDA library (binding.SketchSSM); this module holds the weights and the order of the calls.  The
projections' weights are kept in e4m3 with a scale for each block of 128 x 128 (Mamba-2), or in 8-bit integers with a scale for each
channel.
"""
from __future__ import annotations

from typing import Optional

import torch

from . import binding

_E4M3 = torch.float8_e4m3fn


def quantise_weight(w: torch.Tensor):
    """(e4m3 values [N, K], scales [ceil(N / 128), ceil(K / 128)]) of a weight matrix; done once, when a layer is loaded."""
    n, k = w.shape
    nb, kb = -(-n // 128), -(-k // 128)
    p = torch.nn.functional.pad(w.float(), (0, kb * 128 - k, 0, nb * 128 - n)).view(nb, 128, kb, 128)
    scale = (p.abs().amax(dim=(1, 3)) / 448.0).clamp(min=1e-30)
    q = (p / scale[:, None, :, None]).view(nb * 128, kb * 128)[:n, :k].to(_E4M3)
    return q.contiguous(), scale.contiguous()


def quantise_integer(w: torch.Tensor):
    """(8-bit integers [N, K], scales [N]) of a weight matrix, a scale for each of its rows; done once, when a layer is loaded."""
    w = w.float()
    scale = (w.abs().amax(dim=1) / 127.0).clamp(min=1e-30)
    return torch.round(w / scale[:, None]).to(torch.int8).contiguous(), scale.contiguous()


class Mamba2Layer:
    """One layer of `width` channels for `batch` sequences.  Tensors between layers are bf16; weights come in as floats:
    norm [width], w_in [2 H V + 2 G K + H, width] (rows: gate, values, keys, queries, step sizes), conv_weight [C, W] and conv_bias [C]
    with C = H V + 2 G K, a [H] (negative), dt_bias and skip [H], gate_norm [H V], w_out [width, H V].
    norm_group: how many of the H V inner elements the gated norm takes together, a multiple of 128 (0: all of them; models with several groups
    of heads mostly norm each group's H V / G by itself).
    The whole batch is at one phase of the decode window: a step takes a token of every sequence, and prompts are taken in while the ring is
    empty (end_window).
    stream (None: the current one): what runs, and what it allocates, the results among it, belongs to that stream."""

    def __init__(self, batch: int, heads: int, dk: int, dv: int, groups: int, rank: int, buf_len: int, norm, w_in, conv_weight,
                 conv_bias, a, dt_bias, skip, gate_norm, w_out, eps: float = 1e-5, device: int = 0,
                 norm_group: int = 0, **kw):
        self.m = binding.SketchSSM("mamba2", batch, heads, dk, dv, rank, buf_len, io="bf16", out="f32", device=device, **kw)
        dev = self.m.device
        f32 = lambda t: t.to(device=dev, dtype=torch.float32).contiguous()  # noqa: E731
        self.groups, self.eps, self.inner, self.norm_group = groups, eps, heads * dv, norm_group
        self.channels = self.inner + 2 * groups * dk
        self.norm, self.conv_weight, self.conv_bias = f32(norm), f32(conv_weight), f32(conv_bias)
        self.a, self.dt_bias, self.skip, self.gate_norm = f32(a), f32(dt_bias), f32(skip), f32(gate_norm)
        # (rows of zeros up to a multiple of eight: the projection's rows, and the column ranges of them, are then 16-byte aligned)
        self.w_in, self.w_in_scale = quantise_weight(torch.nn.functional.pad(f32(w_in), (0, 0, 0, -w_in.shape[0] % 8)))
        self.w_out, self.w_out_scale = quantise_weight(f32(w_out))
        self.conv_state = self.m.new_conv_state(self.channels, self.conv_weight.shape[1])
        self.token = self.m.new_token_buffers()

    def _new(self, rows: int, cols: int, dtype=torch.bfloat16) -> torch.Tensor:
        return torch.empty(rows, cols, dtype=dtype, device=self.m.device)

    def _project_in(self, x: torch.Tensor, residual: Optional[torch.Tensor], stream):
        """Norm and first projection: (gate, convolved channels, step sizes) as column ranges of one matrix.  `residual` is moved on
        in place: afterwards it holds residual + x."""
        t, d = x.shape
        x8, scale = self._new(t, d, _E4M3), self._new(t, -(-d // 128), torch.float32)
        self.m.rms_norm(x, self.norm, out8=x8, scale=scale, residual=residual, residual_out=residual, eps=self.eps, stream=stream)
        p = self.m.scaled_matmul(x8, scale, self.w_in, self.w_in_scale, self._new(t, self.w_in.shape[0]), stream=stream)
        return p[:, :self.inner], p[:, self.inner:self.inner + self.channels], p[:, self.inner + self.channels:self.inner + self.channels + self.m.H]

    def _project_out(self, y: torch.Tensor, gate: torch.Tensor, stream, **kw) -> torch.Tensor:
        t = y.shape[0]
        y8, scale = self._new(t, self.inner, _E4M3), self._new(t, -(-self.inner // 128), torch.float32)
        self.m.rms_norm(y, self.gate_norm, out8=y8, scale=scale, gate=gate, eps=self.eps, group=self.norm_group, stream=stream,
                        **kw)
        return self.m.scaled_matmul(y8, scale, self.w_out, self.w_out_scale, self._new(t, self.w_out.shape[0]), stream=stream)

    def prompt(self, prompts: binding.Prompts, x: torch.Tensor, residual: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The layer over packed prompts x [T, width]; leaves the states and the convolution's rows of the prompts' slots.  Before the
        first decode step of a window begin_window builds the sketch.  After decode steps end_window comes first: tokens that are still in
        the ring are no part of the states that prompts go on from, and begin_window forgets them."""
        with binding.on_stream(stream):
            return self._prompt(prompts, x, residual, stream)

    def _prompt(self, prompts, x, residual, stream):
        m, h, k = self.m, self.m.H, self.m.K
        gate, xbc, dt = self._project_in(x, residual, stream)
        t = x.shape[0]
        c = m.causal_conv(prompts, xbc, self.conv_weight, self.conv_bias, self.conv_state, self._new(t, self.channels), stream=stream)
        v = c[:, :self.inner].unflatten(1, (h, m.V))
        key = c[:, self.inner:self.inner + self.groups * k].unflatten(1, (self.groups, k))
        q = c[:, self.inner + self.groups * k:].unflatten(1, (self.groups, k))
        y = self._new(t, self.inner)
        m.prompt_scan(prompts, q, key, v, dt, self.a, y.unflatten(1, (h, m.V)), dt_bias=self.dt_bias, skip=self.skip, stream=stream)
        return self._project_out(y, gate, stream)

    def begin_window(self, stream=None):
        """The sketch (and the maps) of the states as they are: after prompts, before decode steps.  The ring is empty afterwards."""
        self.m.state_update(0, stream=stream)

    def end_window(self, n_before: int, stream=None):
        """The n_before tokens in the ring go into the states, and the ring is empty: before prompts that come between the steps of a window
        (begin_window follows them, for the next step)."""
        self.m.state_update(n_before, flags=binding.NO_SKETCH, stream=stream)

    def step(self, n_before: int, x: torch.Tensor, residual: Optional[torch.Tensor] = None, exact: bool = False, stream=None) -> torch.Tensor:
        """One token of every sequence, x [B, width], with n_before tokens in the ring: a decode step, and at the end of the window the
        state update, after which the ring is empty.  exact: the full state is read instead of the sketch."""
        with binding.on_stream(stream):
            return self._step(n_before, x, residual, exact, stream)

    def _step(self, n_before, x, residual, exact, stream):
        m = self.m
        gate, xbc, dt = self._project_in(x, residual, stream)
        t = m.conv_step(xbc, dt, self.conv_weight, self.conv_bias, self.conv_state, self.a, self.dt_bias, self.token, groups=self.groups,
                        stream=stream)
        args = [t[n] for n in ("q", "k", "v", "beta", "decay", "out")]
        if n_before == m.L - 1:
            m.state_update(n_before, *args, stream=stream)
        elif exact:
            m.full_read_decode(n_before, *args, stream=stream)
        else:
            m.decode_step(n_before, *args, stream=stream)
        return self._project_out(t["out"].view(m.B, self.inner), gate, stream, skip=t["v"].view(m.B, self.inner), skip_weight=self.skip)


class DeltaLayer:
    """One layer of `width` channels for `batch` sequences, with the recurrence of kind "gdn" (a decay for each head) or "kda" (one for each channel of
    a key).  Tensors between layers are bf16; weights come in as floats: norm [width], w_in [2 H V + 2 G K + H + D, width] (rows: gate,
    values, keys, queries, step sizes, arguments of the decays: D = H, or H K), conv_weight [C, W] and conv_bias [C] (or None) with
    C = H V + 2 G K, a [H] (negative), dt_bias [H] or [H, K], head_norm [V] (the same for every head), w_out [width, H V].  inner and width
    are multiples of 16.
    act: what the gate goes through, "silu" or "sigmoid".  The whole batch is at one phase of the decode window, as in Mamba2Layer.
    stream (None: the current one): what runs, and what it allocates, the results among it, belongs to that stream."""

    def __init__(self, kind: str, batch: int, heads: int, dk: int, dv: int, groups: int, rank: int, buf_len: int, norm, w_in, conv_weight,
                 conv_bias, a, dt_bias, head_norm, w_out, eps: float = 1e-5, qk_eps: float = 1e-6, act: str = "silu", device: int = 0, **kw):
        if kind not in ("gdn", "kda"):
            raise ValueError("kind is gdn or kda")
        if act not in ("silu", "sigmoid"):
            raise ValueError("act is silu or sigmoid")
        self.m = binding.SketchSSM(kind, batch, heads, dk, dv, rank, buf_len, io="bf16", out="f32", device=device, **kw)
        dev = self.m.device
        f32 = lambda t: t.to(device=dev, dtype=torch.float32).contiguous()  # noqa: E731
        self.groups, self.eps, self.qk_eps, self.act, self.inner = groups, eps, qk_eps, act, heads * dv
        self.channels, self.decays = self.inner + 2 * groups * dk, heads * dk if kind == "kda" else heads
        self.norm, self.conv_weight, self.a, self.dt_bias, self.head_norm = f32(norm), f32(conv_weight), f32(a), f32(dt_bias), f32(head_norm)
        self.conv_bias = None if conv_bias is None else f32(conv_bias)
        # Rows of zeros behind the step sizes and at the end, up to multiples of eight: the projection's rows, and the column ranges of them, are
        # then 16-byte aligned.
        w, cut, pad = f32(w_in), self.inner + self.channels + heads, torch.nn.functional.pad
        if w.shape[0] != cut + self.decays:
            raise ValueError(f"w_in has {cut + self.decays} rows")
        self.dt_at = cut + -cut % 8
        w = torch.cat([pad(w[:cut], (0, 0, 0, self.dt_at - cut)), pad(w[cut:], (0, 0, 0, -self.decays % 8))])
        self.w_in, self.w_in_scale = quantise_integer(w)
        self.w_out, self.w_out_scale = quantise_integer(f32(w_out))
        self.conv_state = self.m.new_conv_state(self.channels, self.conv_weight.shape[1])
        self.token = self.m.new_token_buffers()

    def _new(self, *size: int, dtype=torch.bfloat16) -> torch.Tensor:
        return torch.empty(*size, dtype=dtype, device=self.m.device)

    def _project_in(self, x: torch.Tensor, residual: Optional[torch.Tensor], stream):
        """Norm and first projection: (gate, channels to convolve, step sizes, arguments of the decays) as column ranges of one matrix.
        `residual` is moved on in place: afterwards it holds residual + x."""
        t, d = x.shape
        x8, scale = self._new(t, d, dtype=torch.int8), self._new(t, dtype=torch.float32)
        self.m.integer_norm(x, self.norm, x8, scale, residual=residual, residual_out=residual, eps=self.eps, stream=stream)
        p = self.m.integer_matmul(x8, scale, self.w_in, self.w_in_scale, self._new(t, self.w_in.shape[0]), stream=stream)
        at = self.inner + self.channels
        return p[:, :self.inner], p[:, self.inner:at], p[:, at:at + self.m.H], p[:, self.dt_at:self.dt_at + self.decays]

    def _project_out(self, y: torch.Tensor, gate: torch.Tensor, stream) -> torch.Tensor:
        t = y.shape[0]
        y8, scale = self._new(t, self.inner, dtype=torch.int8), self._new(t, dtype=torch.float32)
        self.m.integer_norm(y, self.head_norm, y8, scale, gate=gate, act=self.act, eps=self.eps, stream=stream)
        return self.m.integer_matmul(y8, scale, self.w_out, self.w_out_scale, self._new(t, self.w_out.shape[0]), stream=stream)

    def prompt(self, prompts: binding.Prompts, x: torch.Tensor, residual: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
        """The layer over packed prompts x [T, width]; leaves the states and the convolution's rows of the prompts' slots.  begin_window and
        end_window stand between prompts and decode steps as in Mamba2Layer."""
        with binding.on_stream(stream):
            m, h, k = self.m, self.m.H, self.m.K
            gate, xbc, b, dt = self._project_in(x, residual, stream)
            t = x.shape[0]
            c = m.causal_conv(prompts, xbc, self.conv_weight, self.conv_bias, self.conv_state, self._new(t, self.channels), stream=stream)
            v = c[:, :self.inner].unflatten(1, (h, m.V))
            key = c[:, self.inner:self.inner + self.groups * k].unflatten(1, (self.groups, k))
            q = c[:, self.inner + self.groups * k:].unflatten(1, (self.groups, k))
            y = self._new(t, self.inner)
            m.delta_scan(prompts, q, key, v, b, dt, self.a, y.unflatten(1, (h, m.V)), dt_bias=self.dt_bias, eps=self.qk_eps, stream=stream)
            return self._project_out(y, gate, stream)

    def begin_window(self, stream=None):
        """The sketch (and the maps) of the states as they are: after prompts, before decode steps.  The ring is empty afterwards."""
        self.m.state_update(0, stream=stream)

    def end_window(self, n_before: int, stream=None):
        """The n_before tokens in the ring go into the states, and the ring is empty: before prompts that come between the steps of a window
        (begin_window follows them, for the next step)."""
        self.m.state_update(n_before, flags=binding.NO_SKETCH, stream=stream)

    def step(self, n_before: int, x: torch.Tensor, residual: Optional[torch.Tensor] = None, exact: bool = False, stream=None) -> torch.Tensor:
        """One token of every sequence, x [B, width], with n_before tokens in the ring: a decode step, and at the end of the window the
        state update, after which the ring is empty.  exact: the full state is read instead of the sketch."""
        with binding.on_stream(stream):
            m = self.m
            gate, xbc, b, dt = self._project_in(x, residual, stream)
            t = m.delta_step(xbc, b, dt, self.conv_weight, self.conv_bias, self.conv_state, self.a, self.dt_bias, self.token, groups=self.groups,
                             eps=self.qk_eps, stream=stream)
            args = [t[n] for n in ("q", "k", "v", "beta", "decay", "out")]
            if n_before == m.L - 1:
                m.state_update(n_before, *args, stream=stream)
            elif exact:
                m.full_read_decode(n_before, *args, stream=stream)
            else:
                m.decode_step(n_before, *args, stream=stream)
            return self._project_out(t["out"].view(m.B, self.inner), gate, stream)
