"""Plain 64-bit forms of the operators around the recurrence, one sequence, row and head after the other, on the CPU.

Beside each result stands the same sum over absolute values: what rounding errors of its terms are measured by."""
import numpy as np
import torch


def f64(t):
    return t.detach().cpu().double()


def silu(x):
    return x / (1 + torch.exp(-x))


def softplus(x):
    return torch.logaddexp(x, torch.zeros_like(x))


def conv(starts, slots, resume, x, weight, bias, state, act, batch):
    """(out, sum of absolute terms, state afterwards); rows outside the sequences are NaN."""
    x, w, new = f64(x), f64(weight), f64(state).clone()
    old, W = f64(state), weight.shape[1]
    b = f64(bias) if bias is not None else torch.zeros(w.shape[0], dtype=torch.float64)
    out, mag = torch.full_like(x, float("nan")), torch.full_like(x, float("nan"))
    for i in range(len(starts) - 1):
        lo, hi = starts[i], starts[i + 1]
        src = resume[i] if resume is not None else -1
        hist = old[src] if 0 <= src < batch else torch.zeros(W - 1, x.shape[1], dtype=torch.float64)
        full = torch.cat([hist, x[lo:hi]])
        for t in range(lo, hi):
            rows = full[t - lo:t - lo + W]
            y = b + (rows * w.T).sum(0)
            out[t] = silu(y) if act else y
            mag[t] = b.abs() + (rows * w.T).abs().sum(0)
        dst = slots[i] if slots is not None else i
        if 0 <= dst < batch:
            new[dst] = full[hi - lo:]
    return out, mag, new


def scan(starts, slots, resume, q, k, v, dt, a, dt_bias, skip, state, batch):
    """(out, its absolute sum, state afterwards, its absolute sum)."""
    q, k, v, dt, a, old = (f64(t) for t in (q, k, v, dt, a, state))
    T, H, V = v.shape
    per = H // q.shape[1]
    q, k = q.repeat_interleave(per, 1), k.repeat_interleave(per, 1)
    beta = softplus(dt + (f64(dt_bias) if dt_bias is not None else 0.0))
    d = f64(skip) if skip is not None else torch.zeros(H, dtype=torch.float64)
    out, mag = torch.full_like(v, float("nan")), torch.full_like(v, float("nan"))
    new, new_mag = old.clone(), old.abs()
    for i in range(len(starts) - 1):
        src = resume[i] if resume is not None else -1
        S = old[src].clone() if 0 <= src < batch else torch.zeros_like(old[0])
        A = S.abs()
        for t in range(starts[i], starts[i + 1]):
            dec = torch.exp(a * beta[t])[:, None, None]
            kv = beta[t][:, None, None] * k[t][:, :, None] * v[t][:, None, :]
            S, A = dec * S + kv, dec * A + kv.abs()
            out[t] = torch.einsum("hkv,hk->hv", S, q[t]) + d[:, None] * v[t]
            mag[t] = torch.einsum("hkv,hk->hv", A, q[t].abs()) + (d[:, None] * v[t]).abs()
        dst = slots[i] if slots is not None else i
        if 0 <= dst < batch:
            new[dst], new_mag[dst] = S, A
    return out, mag, new, new_mag


def norm(x, weight, eps, group, residual=None, gate=None, skip=None, skip_weight=None):
    """(h, y)."""
    h = f64(x)
    D = h.shape[1]
    if residual is not None:
        h = h + f64(residual)
    if gate is not None:
        if skip is not None:
            h = h + f64(skip) * f64(skip_weight).repeat_interleave(D // skip_weight.numel())
        h = h * silu(f64(gate))
    y = torch.empty_like(h)
    for g in range(0, D, group or D):
        p = h[:, g:g + (group or D)]
        y[:, g:g + (group or D)] = p / torch.sqrt((p * p).mean(1, keepdim=True) + eps)
    return h, y * f64(weight)


def matmul(a, a_scale, w, w_scale):
    """(out, sum of absolute terms)."""
    K, N = a.shape[1], w.shape[0]
    A = f64(a.float()) * f64(a_scale).repeat_interleave(128, 1)[:, :K]
    W = f64(w.float()) * f64(w_scale).repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
    return A @ W.T, A.abs() @ W.abs().T


def half_step(dtype):
    """The largest relative error of one rounding to the type."""
    return torch.finfo(dtype).eps / 2


def close(got, ref, bound, what=""):
    """Every element of `got` is within `bound` (a tensor) of `ref`; NaN in ref has to be NaN in got."""
    got = f64(got)
    nan = torch.isnan(ref)
    assert torch.equal(torch.isnan(got), nan), what + ": NaN where there is none, or none where there is one"
    over = ((got - ref).abs() - bound)[~nan]
    assert over.numel() == 0 or over.max() <= 0, f"{what}: worst {((got - ref).abs() / bound)[~nan].max():.3g} of the bound"


def starts_of(lengths, first=0):
    return [int(s) for s in np.cumsum([first] + list(lengths))]
