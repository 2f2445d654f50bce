"""Plain 64-bit forms of a delta-rule layer's operators, token by token, on the CPU, and bounds of what fp32 arithmetic may be off by."""
import torch

from tests.layer_ref import f64, silu, softplus

U = 2.0 ** -24


def unit(x, eps):
    return x / torch.sqrt((x * x).sum(-1, keepdim=True) + eps)


def decays(dt, a, dt_bias):
    """[T, H, 1 or K] of dt [T, H] or [T, H, K]."""
    x = f64(dt)
    if x.dim() == 2:
        x = x[..., None]
    if dt_bias is not None:
        x = x + f64(dt_bias).reshape(x.shape[1:])
    return torch.exp(softplus(x) * f64(a)[:, None])


def scan(starts, slots, resume, q, k, v, b, dt, a, dt_bias, state, batch, eps=1e-6, q_scale=None, rel=40 * U):
    """(out, its bound, state afterwards, its bound).

    The bound.  S <- (I - beta k k^T) D S + beta k v^T is a contraction of every column of S (|k| <= 1, beta and D in 0..1), so an error of
    a column, as a length, grows by what a token adds and shrinks by its largest decay.  A token adds at most `rel` times (the column's
    length + |v|): sums of K products in at most sixteen partial sums and five joins, norms, gates (expf, log1pf, divisions of a few ulp;
    the error of a decay's exponent x is a few u x, and x exp(-x) < 0.37) and the update: below 40 u where all of it is fp32.  An
    output is |q| <= q_scale times the column's error off, and by `rel` times (the column's length) itself."""
    q, k, v, old = f64(q), f64(k), f64(v), f64(state)
    T, H, V = v.shape
    K, per = q.shape[2], H // q.shape[1]
    q_scale = K ** -0.5 if q_scale is None else q_scale
    q, k = (unit(z, eps).repeat_interleave(per, 1) for z in (q, k))
    q = q * q_scale
    beta = 1 / (1 + torch.exp(-f64(b)))
    D = decays(dt, a, dt_bias)
    out, tol = torch.full_like(v, float("nan")), torch.full_like(v, float("nan"))
    new, new_tol = old.clone(), torch.zeros_like(old)
    for i in range(len(starts) - 1):
        src = resume[i] if resume is not None else -1
        S = old[src].clone() if 0 <= src < batch else torch.zeros_like(old[0])
        err = torch.zeros(H, V, dtype=torch.float64)
        for t in range(starts[i], starts[i + 1]):
            size = S.norm(dim=1)
            S = D[t][:, :, None] * S
            x = beta[t][:, None] * (v[t] - torch.einsum("hkv,hk->hv", S, k[t]))
            S = S + k[t][:, :, None] * x[:, None, :]
            err = D[t].amax(1)[:, None] * err + rel * (size + v[t].abs())
            out[t] = torch.einsum("hkv,hk->hv", S, q[t])
            tol[t] = abs(q_scale) * (err + rel * S.norm(dim=1))
        dst = slots[i] if slots is not None else i
        if 0 <= dst < batch:
            new[dst], new_tol[dst] = S, err[:, None, :].expand_as(S)
    return out, tol, new, new_tol


def norm8(x, weight, eps, residual=None, gate=None, act="silu"):
    """(h, y): weight of one group."""
    h = f64(x)
    if residual is not None:
        h = h + f64(residual)
    g = weight.numel()
    y = torch.cat([p / torch.sqrt((p * p).mean(1, keepdim=True) + eps) * f64(weight) for p in h.split(g, 1)], 1)
    if gate is not None:
        z = f64(gate)
        y = y * (silu(z) if act == "silu" else 1 / (1 + torch.exp(-z)))
    return h, y
