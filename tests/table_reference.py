"""Lookup in a table, cross entropy against it, and their gradients in 64 bits, straight from their definitions, and how far a
result may be from them (see operator_reference: bounds count roundings)."""
import torch

from operator_reference import HALF, ULP

TINY = 2.0 ** -126
WHERE = ["cpu"]  # (where the references are made: "cuda" for sizes that take too long otherwise)


def _64(x):
    return x.to(WHERE[0]).double()


def embedding(table, ids, scale=1.0):
    """(result, bound): a product in binary32, and what storing costs."""
    t, i = _64(table), ids.to(WHERE[0]).long()
    there = (i >= 0) & (i < t.shape[0])
    out = torch.where(there[..., None], t[torch.where(there, i, 0)] * scale, 0.0)
    return out, out.abs() * (HALF[table.dtype] + 2 * ULP)


def embedding_grad(dy, ids, rows, base=None, scale=1.0):
    """(result, bound): a row is a sum of as many terms as tokens name it."""
    dtype = dy.dtype if base is None else base.dtype
    d, i = _64(dy).reshape(-1, dy.shape[-1]), ids.to(WHERE[0]).long().flatten()
    there = (i >= 0) & (i < rows)
    d, i = d[there], i[there]
    total = torch.zeros(rows, d.shape[-1], dtype=torch.float64, device=d.device).index_add_(0, i, d)
    size = torch.zeros(rows, d.shape[-1], dtype=torch.float64, device=d.device).index_add_(0, i, d.abs())
    count = torch.bincount(i, minlength=rows)[:, None].double()
    out = scale * total + (0.0 if base is None else _64(base))
    return out, abs(scale) * size * (count + 2) * ULP + out.abs() * (HALF[dtype] + 2 * ULP)


def _scores(x, table, scale):
    """Scores and how far they may be: products of bf16 are exact in binary32 and those of f32, taken as three bf16 parts each, leave
    out less than 4 units; a matrix unit's sum may cut a whole unit off each time, and there are at most as many sums as columns (six
    products of 16 columns each at a time)."""
    x, w = _64(x).reshape(-1, x.shape[-1]), _64(table)
    return scale * x @ w.T, abs(scale) * (2 * (x.shape[-1] + 16) * ULP * (x.abs() @ w.abs().T))


def loss(x, table, targets, scale=1.0):
    """(loss, bound, lse, bound), flat."""
    z, dz = _scores(x, table, scale)
    t = targets.to(WHERE[0]).long().flatten()
    there = (t >= 0) & (t < table.shape[0])
    lse = torch.logsumexp(z, -1)
    # the exponent: a few roundings of the score; sums of up to 256 scores, then one for each 256; logarithm
    far = (z.abs() * 8 * ULP + dz).amax(-1) + (table.shape[0] / 256 + 320) * ULP + lse.abs() * 4 * ULP
    at = torch.where(there, t, 0)[:, None]
    out = torch.where(there, lse - z.gather(1, at)[:, 0], 0.0)
    return out, torch.where(there, far + dz.gather(1, at)[:, 0] + (out.abs() + z.gather(1, at)[:, 0].abs()) * 4 * ULP, 0.0), lse, far


def loss_grad(x, table, targets, lse, dloss, scale=1.0):
    """(dx, bound, dtable, bound): for bf16, P and x dloss go into the products rounded to bf16; for f32 as three parts."""
    z, dz = _scores(x, table, scale)
    t = targets.to(WHERE[0]).long().flatten()
    there = (t >= 0) & (t < table.shape[0])
    lse, dloss = torch.where(there, _64(lse).flatten(), 0.0)[:, None], torch.where(there, _64(dloss).flatten(), 0.0)[:, None]
    hot = torch.zeros_like(z).scatter_(1, torch.where(there, t, 0)[:, None], 1.0)
    e = torch.where(there[:, None], torch.exp(z - lse), 0.0)
    p = torch.where(there[:, None], scale * dloss * (e - hot), 0.0)
    dp = abs(scale) * dloss.abs() * (e * (dz + 8 * ULP * (z.abs() + lse.abs() + 1)) + 4 * ULP * (e + hot)) * there[:, None]
    # binary32 has no full precision below its smallest normal number, 2^-126, to which an exponential, P and a result may be off at
    # any size: exp(z - lse) for scores 88 below the largest is there
    dp = dp + abs(scale) * dloss.abs() * TINY + TINY
    dp = dp + p.abs() * (HALF[torch.bfloat16] if x.dtype == torch.bfloat16 else 4 * ULP)
    x64, w = torch.where(there[:, None], _64(x).reshape(-1, x.shape[-1]), 0.0), _64(table)
    n, v = p.shape
    dx, dtable = p @ w, p.T @ x64
    more = p.abs().T @ x64.abs() * (HALF[torch.bfloat16] if x.dtype == torch.bfloat16 else 4 * ULP)
    return (dx, dp @ w.abs() + 2 * (v + 64) * ULP * (p.abs() @ w.abs()) + dx.abs() * HALF[x.dtype] + TINY,
            dtable, dp.T @ x64.abs() + more + 2 * (n + 64) * ULP * (p.abs().T @ x64.abs()) + dtable.abs() * HALF[x.dtype] + TINY)
