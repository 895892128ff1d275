"""Plain 64-bit forms of the operators of a transformer layer, and bounds for what the kernels may differ by."""
import torch

from paper_2607_10071_b200 import binding as fb

#: Half a step of a result's type, relative to the value.
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def activation(z, act):
    if act == fb.ACT_RELU:
        return z.clamp_min(0)
    if act == fb.ACT_GELU:
        return z * torch.special.ndtr(z)
    if act == fb.ACT_SILU:
        return z * torch.sigmoid(z)
    return z


def activation_slope(z, act):
    z = z.detach().clone().requires_grad_(True)
    if act == fb.ACT_NONE:
        return torch.ones_like(z)
    if act == fb.ACT_RELU:
        return (z > 0).to(z.dtype)
    return torch.autograd.grad(activation(z, act).sum(), z)[0]


def sum_bound(a, b, long):
    """What a sum of products a b^T over `long` terms may be off by: the tensor cores take 16 terms at a time and cut the sum off each
    time, by at most a step of the partial sum, 2^-23 of the terms' absolute sum; shares and running sums add a few roundings.  (float32
    operands: the three products left out are 3 x 2^-25 of it.)"""
    return (a.abs() @ b.abs().transpose(-1, -2)) * ((long / 16 + 16) * 2.0 ** -23)


def linear(x, w, b=None, act=0, residual=None):
    """(result, z, bound of the result without its rounding, bound of z without its rounding)"""
    x, w = x.double(), w.double()
    z = x @ w.T + (0 if b is None else b.double())
    off_z = sum_bound(x, w, x.shape[-1]) + 2.0 ** -23 * z.abs()
    out = activation(z, act) + (0 if residual is None else residual.double())
    # slopes of the activations are at most 1.13; their formulas: 3e-5 of |z| Phi(-|z|), at most 0.17, where the result is bf16, a few steps of
    # float32 otherwise; one more sum for the residual
    off = 1.13 * off_z + 2.0 ** -21 * (z.abs() + out.abs())
    return out, z, off, off_z


def linear_backward(g, x, w, act=0, z=None):
    """Three gradients and their bounds without their own rounding.  bf16: the gradient before the activation is rounded as well."""
    low = x.dtype == torch.bfloat16
    g, x, w = g.double(), x.double(), w.double()
    dz = g * activation_slope(z.double(), act) if act else g
    # The slope's formula.  It is a sum of two terms, s + z s (1 - s) or Phi + z phi, that have opposite signs for z < 0 and cancel at the function's
    # minimum: their roundings, about eight of 2^-24 of terms up to 1.3, stay when the sum does not.
    off = dz.abs() * 2.0 ** -20 + (g.abs() * (3.1e-5 if low else 1.3 * 8 * 2.0 ** -24) if act in (fb.ACT_GELU, fb.ACT_SILU) else 0)
    rough = off + (HALF_STEP[torch.bfloat16] * dz.abs() if low else 0)
    grads = (dz @ w, dz.T @ x, dz.sum(0))
    n, rows = w.shape[0], x.shape[0]
    bounds = (rough @ w.abs() + sum_bound(dz, w.T, n), rough.T @ x.abs() + sum_bound(dz.T, x.T, rows),
              off.sum(0) + dz.abs().sum(0) * (rows ** 0.5 + 40) * 2.0 ** -24)
    return grads, bounds


def check(got, want, off, what=""):
    """Every element within its bound plus the rounding of the result's type."""
    assert got.shape == want.shape, (what, got.shape, want.shape)
    diff = (got.double() - want).abs()
    tol = HALF_STEP[got.dtype] * want.abs() * 1.001 + off * 1.001 + 1e-37
    worst = (diff / tol).max().item() if diff.numel() else 0.0
    assert not diff.numel() or worst <= 1.0, f"{what}: {worst:.3g} times the bound, {diff.max().item():.3g} off"


def whiten(v, kind, eps):
    if kind == fb.NORM_NONE:
        return v
    if kind == fb.NORM_LAYER:
        v = v - v.mean(-1, keepdim=True)
    return v / (v.pow(2).mean(-1, keepdim=True) + eps).sqrt()


def block_norm(x, y, gate, scale, after, aw, ab, before, bw, bb, eps):
    """(h, n) in 64 bits; differentiable."""
    def affine(v, kind, w, b):
        if kind == fb.NORM_NONE:
            return v
        v = whiten(v, kind, eps)
        v = v if w is None else v * w
        return v if b is None else v + b
    h = x
    if y is not None:
        m = affine(y, after, aw, ab)
        if gate is not None:
            g = gate.reshape(-1, x.shape[-1])
            m = m * g.repeat_interleave(x.shape[0] // g.shape[0], 0)
        h = x + scale * m
    return h, (None if before == fb.NORM_NONE else affine(h, before, bw, bb))
