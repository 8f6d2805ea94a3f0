"""Rotation at positions of several axes in 64 bits, from its definition (CPU tensors)."""
import torch

from llm_ref import f64


def pairs(D, sections, order, ladder, theta):
    """The axis and the frequency of every pair."""
    half, left, axis, rung = D // 2, list(sections), [], []
    a = 0
    for i in range(half):
        if order == "turns" and i:
            a = (a + 1) % len(left)
        while left[a] == 0:
            a = (a + 1) % len(left)
        axis.append(a)
        rung.append(i / half if ladder == "shared" else (sections[a] - left[a]) / sections[a])
        left[a] -= 1
    return axis, float(theta) ** -torch.tensor(rung, dtype=torch.float64)


def turn(x, pos, rope, theta, sections, order, ladder, sign=1.0):
    """Rows of x [..., D] (fp64), row r turned by the positions pos[:, r] (pos [axes, ...] broadcasts against the rows)."""
    D = x.shape[-1]
    axis, w = pairs(D, sections, order, ladder, theta)
    a = pos.double()[axis].movedim(0, -1) * w
    c, s = torch.cos(a), sign * torch.sin(a)
    if rope == "neox":
        x0, x1 = x[..., : D // 2], x[..., D // 2:]
        return torch.cat((x0 * c - x1 * s, x0 * s + x1 * c), -1)
    x0, x1 = x[..., 0::2], x[..., 1::2]
    return torch.stack((x0 * c - x1 * s, x0 * s + x1 * c), -1).flatten(-2)


def axes_fwd(x, w, pos, variant, norm, eps):
    """Output rows, and the largest magnitude of each row before its rotation."""
    x = f64(x)
    y = x * (x.square().mean(-1, keepdim=True) + eps).rsqrt() * (1.0 if w is None else f64(w)) if norm else x
    return turn(y, pos, *variant), y.abs().amax(-1, keepdim=True)


def axes_bwd(x, w, dout, pos, variant, norm, eps):
    """dx, dw, and what their roundings are relative to (as llm_ref.qknorm_bwd)."""
    dy = turn(f64(dout), pos, *variant, sign=-1.0)
    if not norm:
        return dy, None, f64(dout).abs().amax(-1, keepdim=True), None
    x = f64(x)
    w = torch.ones(x.shape[-1], dtype=torch.float64) if w is None else f64(w)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    xh, g = x * r, dy * w
    dx = r * (g - xh * (g * xh).mean(-1, keepdim=True))
    size = r * (g.abs().amax(-1, keepdim=True) + xh.abs().amax(-1, keepdim=True) * (g * xh).abs().mean(-1, keepdim=True))
    dims = tuple(range(x.dim() - 1))
    return dx, (dy * xh).sum(dims), size, (dy.abs() * xh.abs()).sum(dims)
