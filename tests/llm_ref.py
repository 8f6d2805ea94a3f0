"""The operators of include/attnfuse_llm.h in 64 bits, from their definitions (CPU tensors)."""
import math

import torch

U32 = 2.0 ** -24   # half a step of fp32, relative


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().cpu().double()


def rotate(x, pos, rope, theta, sign=1.0):
    """Rows of x [..., D] (fp64) turned by sign * the angles of their positions (pos broadcasts against the rows)."""
    if rope == "none":
        return x
    D = x.shape[-1]
    w = float(theta) ** (-2.0 * torch.arange(D // 2, dtype=torch.float64) / D)
    a = pos.double()[..., None] * w
    c, s = torch.cos(a), sign * torch.sin(a)
    if rope == "neox":
        x0, x1 = x[..., : D // 2], x[..., D // 2:]
        return torch.cat((x0 * c - x1 * s, x0 * s + x1 * c), -1)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * c - x1 * s, x0 * s + x1 * c), -1).flatten(-2)


def qknorm(x, w, pos, rope, theta, eps):
    """Output rows, and the largest |w x r| of each row (what the roundings of a row are relative to)."""
    x = f64(x)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    y = x * r * (1.0 if w is None else f64(w))
    return rotate(y, pos, rope, theta), y.abs().amax(-1, keepdim=True)


def qknorm_bwd(x, w, dout, pos, rope, theta, eps):
    """dx, dw, and what their roundings are relative to: a row's r (max|g| + max|xh| mean|g xh|), and sum |dy xh|."""
    x = f64(x)
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else f64(w)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    xh, dy = x * r, rotate(f64(dout), pos, rope, theta, -1.0)
    g = dy * w
    dx = r * (g - xh * (g * xh).mean(-1, keepdim=True))
    size = r * (g.abs().amax(-1, keepdim=True) + xh.abs().amax(-1, keepdim=True) * (g * xh).abs().mean(-1, keepdim=True))
    dims = tuple(range(x.dim() - 1))
    return dx, (dy * xh).sum(dims), size, (dy.abs() * xh.abs()).sum(dims)


def assert_within(got, want, tol, what):
    got = f64(got)
    assert got.shape == want.shape, f"{what}: shape {tuple(got.shape)}, {tuple(want.shape)} expected"
    err = (got - want).abs()
    over = ~(err <= tol)   # NaN is over
    assert not over.any(), f"{what}: off by {err[over].max().item():.3e} where {(tol + 0 * err)[over].min().item():.3e} is allowed"


def visible(S, window, sinks):
    i, j = torch.arange(S)[:, None], torch.arange(S)[None, :]
    return (j <= i) & ((j > i - window) | (j < sinks))


def scale_of(D, scale):
    return 1.0 / math.sqrt(D) if scale is None else scale


def decode(q, keys, values, seen, pos, *, rope="none", theta=10000.0, slopes=None, scale=None):
    """One query of each head, q [H, D] at position pos, against the visible keys ``seen`` (their positions) of keys and
    values [H_kv, n, D]: O [H, D], LSE [H], the sum of p |v|, and the largest scale sum |q' k| of a head (what the scores'
    roundings are relative to)."""
    H, D = q.shape
    G = H // keys.shape[0]
    o, lse, pv, mag = torch.zeros(H, D, dtype=torch.float64), torch.full((H,), -math.inf, dtype=torch.float64), None, None
    pv, mag = torch.zeros_like(o), torch.zeros(H, dtype=torch.float64)
    if len(seen) == 0:
        return o, lse, pv, mag
    qr = rotate(f64(q), torch.full((H,), pos), rope, theta)
    for h in range(H):
        k, v = f64(keys[h // G])[seen], f64(values[h // G])[seen]
        s = scale_of(D, scale) * (k @ qr[h])
        if slopes is not None:
            s = s - float(slopes[h]) * (pos - seen.double())
        lse[h] = torch.logsumexp(s, 0)
        p = torch.softmax(s, 0)
        o[h], pv[h] = p @ v, p @ v.abs()
        mag[h] = scale_of(D, scale) * (k.abs() @ qr[h].abs()).max() + (0 if slopes is None else abs(float(slopes[h])) * pos)
    return o, lse, pv, mag
