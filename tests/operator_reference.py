"""The transformer operators in 64 bits, straight from their definitions, and how far a result may be from them.

A bound counts roundings: storing costs half a step of the result's type (HALF[dtype] relative), a sum of n terms in binary32
at most n roundings of 2^-24 relative to the sum of magnitudes, a library function a few more.
"""
import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
ULP = 2.0 ** -24
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def close(got, want, bound, what=""):
    got, want, bound = got.double().cpu(), want.double().cpu(), bound.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    off = (got - want).abs()
    bad = (off > bound) & ~torch.isnan(want)
    if bad.any():
        worst = int(torch.argmax(torch.where(bad, off - bound, torch.zeros_like(off))))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} too far; at {worst}: {got.flatten()[worst]} for {want.flatten()[worst]}, "
                             f"bound {bound.flatten()[worst]}")


def frequencies(rotated, base=10000.0, factor=1.0):
    return torch.tensor([base ** (-2.0 * i / rotated) / factor for i in range(rotated // 2)], dtype=torch.float64)


def rotary(x, positions, freq, interleaved=False, inverse=False, scale=1.0):
    """(result, bound) for x [tokens, .., dim]."""
    x64 = x.double().cpu()
    shape = x64.shape
    x64 = x64.reshape(shape[0], -1, shape[-1])
    p = freq.numel()
    angle = positions.double().cpu()[:, None, None] * freq[None, None, :] * (-1.0 if inverse else 1.0)
    c, s = scale * torch.cos(angle), scale * torch.sin(angle)
    i0 = torch.arange(p) * 2 if interleaved else torch.arange(p)
    i1 = i0 + 1 if interleaved else i0 + p
    a, b = x64[..., i0], x64[..., i1]
    out, slack = x64.clone(), torch.zeros_like(x64)
    out[..., i0], out[..., i1] = a * c - b * s, a * s + b * c
    # cos and sin to 2 units in the last place, the angle to 2^-24 of itself (under half a turn), two products and a sum
    slack[..., i0] = slack[..., i1] = (a.abs() + b.abs()) * abs(scale) * 16 * ULP
    touched = torch.zeros_like(x64)
    touched[..., i0] = touched[..., i1] = 1.0
    return out.reshape(shape), (slack + out.abs() * HALF[x.dtype] * touched).reshape(shape)


def attention(q, cache, table, lengths, scale, head_major):
    """(result, bound), one sequence and head at a time."""
    if head_major:
        cache = cache.transpose(2, 3)
    pages, _, page, kv_heads, dim = cache.shape
    batch, heads, _ = q.shape
    group = heads // kv_heads
    out, bound = torch.zeros(batch, heads, dim, dtype=torch.float64), torch.zeros(batch, heads, dim, dtype=torch.float64)
    for b in range(batch):
        n = max(0, min(int(lengths[b]), table.shape[1] * page))
        if n == 0:
            continue
        ids = [int(t) for t in table[b, : -(-n // page)]]
        keep = torch.tensor([0 <= ids[i // page] < pages for i in range(n)])
        held = cache[[t if 0 <= t < pages else 0 for t in ids]].double().cpu().transpose(0, 1).reshape(2, -1, kv_heads, dim)[:, :n][:, keep]
        if held.shape[1] == 0:
            continue
        for h in range(heads):
            k, v, qq = held[0, :, h // group], held[1, :, h // group], q[b, h].double().cpu()
            s = scale * (k @ qq)
            w = torch.softmax(s, 0)
            out[b, h] = w @ v
            # a score: dim products and sums; its exponential: the argument's rounding, and 2 units of exp2
            ds = (abs(scale) * (dim + 8) * ULP * (k.abs() @ qq.abs()) + s.abs() * 4 * ULP).max() + 4 * ULP
            spread = w @ v.abs()
            bound[b, h] = spread * (2 * ds + 2 * (n + 64) * ULP) + out[b, h].abs() * HALF[q.dtype]
            if q.dtype == torch.bfloat16:  # the weights go into the product as two bf16 parts
                bound[b, h] += spread * 2.0 ** -15
    return out, bound


def rms_norm(x, gamma, residual, eps):
    """(y, bound of its 32-bit value, h, bound of it) without the roundings of storing."""
    h = x.double().cpu() + (0.0 if residual is None else residual.double().cpu())
    cols = h.shape[-1]
    y = gamma.double().cpu() * h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    return y, y.abs() * (cols / 2 + 16) * ULP, h, h.abs() * ULP


def rms_norm_grad(dy, h, gamma, dh, eps):
    """(dx, bound, dgamma, bound)."""
    dtype = h.dtype
    dy, h, gamma = dy.double().cpu(), h.double().cpu(), gamma.double().cpu()
    cols = h.shape[-1]
    inv = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + eps)
    u, d = h * inv, dy * gamma
    direct = 0.0 if dh is None else dh.double().cpu()
    dx = direct + inv * (d - u * (d * u).mean(-1, keepdim=True))
    size = inv * (d.abs() + u.abs() * (d * u).abs().mean(-1, keepdim=True)) + (0.0 if dh is None else direct.abs())
    dims = tuple(range(h.dim() - 1))
    dgamma, total = (dy * u).sum(dims), (dy * u).abs().sum(dims)
    rows = h.numel() // cols
    return dx, dx.abs() * HALF[dtype] + size * (2 * cols + 64) * ULP, dgamma, total * (rows + cols + 64) * ULP
