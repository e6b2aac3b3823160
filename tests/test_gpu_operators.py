"""The transformer operators on the GPU against their definitions in 64 bits (operator_reference), through the public
entry points: types, head layouts, lengths from none to long, odd sizes, slices read in place, unaligned memory, results in
place, padded batches, other streams, captured flushes, and a run of them together."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import operator_reference as ref
from operator_reference import HALF, TYPES, ULP, close

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def lt():
    import paper_2102_13267_b200 as lt
    return lt


@pytest.fixture()
def ctx(lt):
    c = lt.LazyContext(device=0)
    yield c
    c.close()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def fetch(ctx, t):
    a = ctx.fetch(t)
    if t.dtype == "bf16":
        return torch.from_numpy(a.view(np.int16)).view(torch.bfloat16)
    return torch.from_numpy(a)


def unaligned(ctx, x, name, by=1):
    """A copy of x that starts `by` elements behind a 16-byte boundary."""
    room = torch.empty(x.numel() + 64, device="cuda", dtype=x.dtype)
    room[by: by + x.numel()] = x.flatten()
    return ctx.from_device_ptr(room.data_ptr() + by * x.element_size(), name, tuple(x.shape), keep=room)


# ------------------------------------------------------------------------------------------------ rotary
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,heads,dim,rotated,interleaved,inverse", [
    (1, 1, 2, 2, False, False), (1, 32, 128, 128, False, False), (3, 5, 128, 128, True, False), (7, 4, 80, 40, True, True),
    (33, 3, 96, 32, False, True), (64, 8, 64, 64, False, False), (5, 2, 33, 6, True, False), (129, 1, 256, 256, False, True),
    (2, 7, 20, 20, False, False), (257, 40, 64, 32, True, False), (300, 2, 12, 4, False, False), (2, 1, 4096, 4096, False, False)])
def test_rotary(ctx, lt, dtype, tokens, heads, dim, rotated, interleaved, inverse):
    t, g = TYPES[dtype], gen(tokens * 31 + dim)
    x = normal(g, tokens, heads, dim, dtype=t)
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    pos[0] = 0 if tokens > 1 else 131071
    pos[-1] = (1 << 31) - 1 if tokens > 2 else pos[-1]
    want, bound = ref.rotary(x, pos, ref.frequencies(rotated), interleaved, inverse, 1.25)
    y = ctx.rotary(ctx.from_torch(x), ctx.from_torch(pos), ctx.leaf(lt.rotary_table(rotated), "u32"), interleaved=interleaved, inverse=inverse, scale=1.25)
    close(fetch(ctx, y), want, bound)


@pytest.mark.parametrize("tokens,heads,dim,rotated,interleaved", [
    (1, 3, 80, 40, False), (40, 6, 80, 40, False), (9000, 3, 100, 24, False), (70, 5, 20, 16, True), (33, 2, 12, 8, False), (300, 40, 36, 36, True), (5000, 33, 68, 56, False)])
def test_rotary_and_append_in_pieces_of_eight_bytes(ctx, lt, tokens, heads, dim, rotated, interleaved):
    """bf16 heads whose pairs do not come in eights."""
    g, t = gen(tokens + dim), torch.bfloat16
    k, v = normal(g, tokens, heads, dim, dtype=t), normal(g, tokens, heads, dim, dtype=t)
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    want, bound = ref.rotary(k, pos, ref.frequencies(rotated), interleaved)
    turned = (ctx.from_torch(pos), ctx.leaf(lt.rotary_table(rotated), "u32"))
    close(fetch(ctx, ctx.rotary(ctx.from_torch(k), *turned, interleaved=interleaved)), want, bound)
    pages = (tokens + 15) // 16
    cache = empty_cache(g, pages, 16, heads, dim, True, t)
    slots = torch.randperm(pages * 16, generator=g, device="cuda")[:tokens].to(torch.int32)
    lc = ctx.from_torch(cache)
    ctx.cache_append(lc, ctx.from_torch(k), ctx.from_torch(v), ctx.from_torch(slots), *turned, head_major=True, interleaved=interleaved)
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lc) == cache.data_ptr()
    after, at = token_view(cache, True).cpu(), slots.cpu().long()
    close(after[0][at], want, bound, "keys")
    assert torch.equal(after[1][at], v.cpu())


def test_rotary_gradient_is_the_transposed_rotation(ctx, lt):
    """<dy, rotary(x)> differentiated: the inverse applied to dy is the gradient, checked against differences in 64 bits."""
    g = gen(5)
    x, dy = normal(g, 4, 3, 16), normal(g, 4, 3, 16)
    pos = torch.tensor([0, 1, 77, 100000], dtype=torch.int32, device="cuda")
    f = ref.frequencies(16)
    dx = fetch(ctx, ctx.rotary(ctx.from_torch(dy), ctx.from_torch(pos), ctx.leaf(lt.rotary_table(16), "u32"), inverse=True, scale=0.5))
    for at in [(0, 0, 0), (1, 2, 7), (2, 1, 15), (3, 0, 8)]:
        up, down = x.double().cpu().clone(), x.double().cpu().clone()
        up[at] += 0.5
        down[at] -= 0.5
        d = (dy.double().cpu() * (_rot64(up, pos, f, 0.5) - _rot64(down, pos, f, 0.5))).sum()
        assert abs(float(d) - float(dx[at])) < 64 * ULP * float(dy.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,rotated", [(50001, 1, 64, 64), (60000, 1, 16, 8), (20000, 1, 256, 256), (3001, 1, 1024, 1024), (700, 1, 2048, 2048), (9000, 3, 128, 128)])
def test_rotary_more_tokens_than_the_blocks_have_at_once(ctx, lt, dtype, interleaved, tokens, heads, dim, rotated):
    t, g = TYPES[dtype], gen(tokens)
    x = normal(g, tokens, heads, dim, dtype=t)
    pos = torch.randint(0, 1 << 20, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    y = ctx.rotary(ctx.from_torch(x), ctx.from_torch(pos), ctx.leaf(lt.rotary_table(rotated), "u32"), interleaved=interleaved)
    close(fetch(ctx, y), *ref.rotary(x, pos, ref.frequencies(rotated), interleaved))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotated", [128, 6])
def test_rotary_angles(ctx, lt, interleaved, rotated):
    """Pairs (1, 0) turn into the cosine and the sine themselves.  The angle is taken to 2^-28 of a turn, which moves neither by
    more than 2 pi 2^-28 sqrt(1/2); the functions themselves are good to one unit in the last place, 2^-24 at most."""
    tokens, p = 40000, rotated // 2
    table = lt.rotary_table(rotated)
    pos = torch.randint(-(1 << 31), 1 << 31, (tokens,), generator=gen(rotated), device="cuda").to(torch.int32)
    x = torch.zeros(tokens, 1, rotated, device="cuda")
    (x[..., ::2] if interleaved else x[..., :p]).fill_(1.0)
    y = fetch(ctx, ctx.rotary(ctx.from_torch(x), ctx.from_torch(pos), ctx.leaf(table, "u32"), interleaved=interleaved))[:, 0].double().numpy()
    c, s = (y[:, ::2], y[:, 1::2]) if interleaved else (y[:, :p], y[:, p:])
    f = table[:, 0].astype(np.uint64) | (table[:, 1].astype(np.uint64) << np.uint64(32))
    turns = (pos.cpu().numpy().astype(np.int64).view(np.uint64)[:, None] * f[None, :]).view(np.int64) / 2.0 ** 64
    most = 2.0 ** -24 + 2 * math.pi * 2.0 ** -28 * math.sqrt(0.5)
    for got, want in ((c, np.cos(2 * math.pi * turns)), (s, np.sin(2 * math.pi * turns))):
        assert np.abs(got - want).max() <= most


def _rot64(x, pos, f, scale):
    z = torch.polar(torch.full((), scale, dtype=torch.float64), pos.double().cpu()[:, None, None] * f)
    p = f.numel()
    w = torch.complex(x[..., :p], x[..., p: 2 * p]) * z
    return torch.cat((w.real, w.imag), -1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotary_slices_unaligned_and_in_place(ctx, lt, dtype, interleaved):
    t, g = TYPES[dtype], gen(9)
    packed = normal(g, 19, 12, 64, dtype=t)
    pos = torch.arange(1000, 1019, device="cuda", dtype=torch.int32)
    table = ctx.leaf(lt.rotary_table(64), "u32")
    f = ref.frequencies(64)
    lp, lpos = ctx.from_torch(packed), ctx.from_torch(pos)
    for start, count in ((0, 8), (8, 2), (3, 5)):
        y = ctx.rotary(ctx.op("narrow", lp, dim=1, start=start, length=count), lpos, table, interleaved=interleaved)
        ctx.barrier()
        assert "copy kernel" not in ctx.dump_plan()
        close(fetch(ctx, y), *ref.rotary(packed[:, start: start + count], pos, f, interleaved))
    # a slice of the tokens, and one of a computed value (copied first)
    y = ctx.rotary(ctx.op("narrow", lp, dim=0, start=4, length=9), ctx.op("narrow", lpos, dim=0, start=4, length=9), table, interleaved=interleaved)
    close(fetch(ctx, y), *ref.rotary(packed[4:13], pos[4:13], f, interleaved))
    y = ctx.rotary(ctx.op("narrow", ctx.op("neg", lp), dim=1, start=1, length=3), lpos, table, interleaved=interleaved)
    close(fetch(ctx, y), *ref.rotary(-packed[:, 1:4], pos, f, interleaved))
    for by in (1, 2, 4):
        y = ctx.rotary(unaligned(ctx, packed, dtype, by), lpos, table, interleaved=interleaved)
        close(fetch(ctx, y), *ref.rotary(packed, pos, f, interleaved))
    # over its own input
    want, bound = ref.rotary(packed, pos, f, interleaved)
    own = packed.clone()
    lo = ctx.from_torch(own)
    ctx.assign(lo, ctx.rotary(lo, lpos, table, interleaved=interleaved))
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lo) == own.data_ptr()
    close(own, want, bound)


# ------------------------------------------------------------------------------------------------ cache_append
def empty_cache(g, pages, page, heads, dim, head_major, dtype):
    return normal(g, *((pages, 2, heads, page, dim) if head_major else (pages, 2, page, heads, dim)), dtype=dtype)


def token_view(cache, head_major):
    """[2, slots, heads, dim]"""
    c = cache.transpose(2, 3) if head_major else cache
    return c.movedim(1, 0).reshape(2, -1, c.shape[3], c.shape[4])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,rotated,interleaved,page,pages", [
    (30001, 1, 64, 64, False, 32, 960), (20001, 1, 128, 128, True, 16, 1300),
    (1, 1, 8, 8, False, 1, 3), (1, 8, 128, 128, False, 16, 4), (33, 2, 80, 40, True, 7, 9), (64, 8, 64, 0, False, 16, 40), (300, 4, 256, 256, False, 48, 8),
    (5, 3, 33, 16, True, 5, 5), (90, 1, 96, 32, False, 64, 2)])
def test_cache_append(ctx, lt, dtype, head_major, tokens, heads, dim, rotated, interleaved, page, pages):
    t, g = TYPES[dtype], gen(tokens + 7 * dim)
    cache = empty_cache(g, pages, page, heads, dim, head_major, t)
    k, v = normal(g, tokens, heads, dim, dtype=t), normal(g, tokens, heads, dim, dtype=t)
    slots = torch.randperm(pages * page, generator=g, device="cuda")[:tokens].to(torch.int32)
    if tokens > 4:
        slots[tokens // 2] = -1
        slots[-2:] = -7  # rows behind the last sequence
    pos = torch.randint(0, 100000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    before = token_view(cache, head_major).cpu()
    lc = ctx.from_torch(cache)
    turned = (ctx.from_torch(pos), ctx.leaf(lt.rotary_table(rotated), "u32")) if rotated else ()
    ctx.cache_append(lc, ctx.from_torch(k), ctx.from_torch(v), ctx.from_torch(slots), *turned, head_major=head_major, interleaved=interleaved)
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lc) == cache.data_ptr()  # only the slots were written
    want, bound = ref.rotary(k, pos, ref.frequencies(rotated), interleaved) if rotated else (k.double().cpu(), torch.zeros(k.shape))
    after = token_view(cache, head_major).cpu()
    at = slots.cpu().long()
    kept = at >= 0
    close(after[0][at[kept]], want[kept], bound[kept], "keys")
    assert torch.equal(after[1][at[kept]], v.cpu()[kept])
    rest = torch.ones(pages * page, dtype=torch.bool)
    rest[at[kept]] = False
    assert torch.equal(after[:, rest], before[:, rest])


def test_cache_append_packed_slices_and_unaligned(ctx, lt):
    g = gen(3)
    qkv = normal(g, 21, 12, 64, dtype=torch.bfloat16)
    pos = torch.arange(21, device="cuda", dtype=torch.int32) * 11
    slots = torch.randperm(64, generator=g, device="cuda")[:21].to(torch.int32)
    want, bound = ref.rotary(qkv[:, 8:10], pos, ref.frequencies(64))
    lq, table = ctx.from_torch(qkv), ctx.leaf(lt.rotary_table(64), "u32")
    for by in (0, 1):
        cache = empty_cache(g, 8, 8, 2, 64, True, torch.bfloat16)
        lc = unaligned(ctx, cache, "bf16", by)
        ctx.cache_append(lc, ctx.op("narrow", lq, dim=1, start=8, length=2), ctx.op("narrow", lq, dim=1, start=10, length=2), ctx.from_torch(slots),
                         ctx.from_torch(pos), table, head_major=True)
        ctx.barrier()
        assert "copy kernel" not in ctx.dump_plan()
        after = token_view(fetch(ctx, lc), True)
        close(after[0][slots.cpu().long()], want, bound)
        assert torch.equal(after[1][slots.cpu().long()], qkv[:, 10:].cpu())


def test_cache_append_as_a_value_leaves_the_old_cache(ctx, lt):
    """Not assigned, the result is a new cache; two appends to one cache in one flush keep their order."""
    g = gen(4)
    cache = empty_cache(g, 4, 8, 2, 16, False, torch.float32)
    k1, v1, k2, v2 = (normal(g, 2, 2, 16) for _ in range(4))
    s1, s2 = torch.tensor([3, 9], dtype=torch.int32, device="cuda"), torch.tensor([9, 20], dtype=torch.int32, device="cuda")
    lc = ctx.from_torch(cache)
    old = cache.clone()
    new = ctx.op("cache_append", lc, *(ctx.from_torch(a) for a in (k1, v1, s1)), head_major=False, interleaved=False, scale=1.0)
    got = token_view(fetch(ctx, new), False)
    assert torch.equal(cache, old)
    want = token_view(old, False).clone().cpu()
    want[0, [3, 9]], want[1, [3, 9]] = k1.cpu(), v1.cpu()
    assert torch.equal(got, want)
    ctx.cache_append(lc, *(ctx.from_torch(a) for a in (k1, v1, s1)))
    ctx.cache_append(lc, *(ctx.from_torch(a) for a in (k2, v2, s2)))
    ctx.barrier(blocking=True)
    want[0, [9, 20]], want[1, [9, 20]] = k2.cpu(), v2.cpu()
    assert torch.equal(token_view(fetch(ctx, lc), False), want)


def test_slots_beyond_the_cache_are_left_out_and_reported(ctx, lt):
    g = gen(6)
    cache = empty_cache(g, 2, 4, 1, 8, False, torch.float32)
    k, v = normal(g, 3, 1, 8), normal(g, 3, 1, 8)
    before = token_view(cache, False).clone().cpu()
    slots = torch.tensor([8, 5, 2147483647], dtype=torch.int32, device="cuda")
    lc = ctx.from_torch(cache)
    ctx.cache_append(lc, ctx.from_torch(k), ctx.from_torch(v), ctx.from_torch(slots))
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*slot"):
        ctx.barrier(blocking=True)
    before[0, 5], before[1, 5] = k[1].cpu(), v[1].cpu()
    assert torch.equal(token_view(cache, False).cpu(), before)
    ctx.cache_append(lc, ctx.from_torch(k), ctx.from_torch(v), ctx.from_torch(slots.clamp(max=6)[1:2].expand(3).contiguous() - torch.arange(3, device="cuda", dtype=torch.int32)))
    ctx.barrier(blocking=True)  # reported once


def test_a_bad_slot_is_reported_to_the_context_that_met_it(lt):
    g = gen(7)
    a, b = lt.LazyContext(device=0), lt.LazyContext(device=0)
    k = normal(g, 2, 1, 8)
    kept = []

    def append(c, slots):
        cache = torch.zeros(2, 2, 4, 1, 8, device="cuda")
        hs = [c.from_torch(t) for t in (cache, k, k, torch.tensor(slots, dtype=torch.int32, device="cuda"))]
        kept.append(hs)
        c.cache_append(*hs)

    append(a, [8, 1]), append(b, [0, 1])
    a.barrier()
    torch.cuda.synchronize()
    b.barrier(blocking=True)
    append(b, [2, 3])
    b.barrier(blocking=True)
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*slot"):
        a.barrier(blocking=True)
    a.barrier(blocking=True)  # reported once
    kept.clear()
    a.close(), b.close()


# ------------------------------------------------------------------------------------------------ paged_attention
def paged(g, lengths, page, kv_heads, dim, head_major, dtype, spare=2, width=None):
    """(cache, page table): pages in random order, everything that no token lies in being NaN, entries behind the last page invalid."""
    per = [-(-n // page) for n in lengths]
    pages = sum(per) + spare
    cache = empty_cache(g, pages, page, kv_heads, dim, head_major, dtype)
    order = torch.randperm(pages, generator=g, device="cuda").tolist()
    width = width or max(1, max(per))
    table = torch.full((len(lengths), width), -5, dtype=torch.int32)
    held = torch.zeros(pages, page, dtype=torch.bool)
    for b, n in enumerate(lengths):
        for i in range(per[b]):
            p = order.pop()
            table[b, i] = p
            held[p, : min(page, n - i * page)] = True
    lost = ~held.cuda()
    if head_major:
        cache.masked_fill_(lost[:, None, None, :, None], math.nan)
    else:
        cache.masked_fill_(lost[:, None, :, None, None], math.nan)
    return cache, table.cuda()


LENGTHS = {"edges": [0, 1, 15, 16, 17, 63, 64, 65, 0], "one": [1], "long": [1000], "ragged": [3, 500, 129, 1, 257, 2], "two_tiles": [128, 5, 127], "none": [0, 0], "longer": [2500, 40]}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("head_major", [False, True])
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths", [
    (8, 2, 128, 16, "edges"), (32, 8, 128, 16, "long"), (1, 1, 64, 16, "one"), (16, 16, 64, 32, "ragged"), (5, 1, 128, 48, "ragged"), (16, 1, 128, 64, "long"),
    (12, 1, 64, 7, "edges"), (8, 4, 80, 16, "ragged"), (4, 2, 96, 8, "two_tiles"), (8, 1, 256, 16, "ragged"), (24, 1, 256, 16, "long"), (3, 3, 33, 5, "ragged"), (2, 2, 8, 1, "edges"),
    (4, 2, 128, 16, "none"), (40, 1, 64, 16, "long"), (8, 8, 72, 16, "longer"), (64, 2, 128, 32, "two_tiles"), (7, 7, 1, 3, "edges"), (16, 2, 192, 16, "ragged"), (17, 1, 136, 16, "edges")])
def test_paged_attention(ctx, dtype, head_major, heads, kv_heads, dim, page, lengths):
    t, g, n = TYPES[dtype], gen(heads * 100 + dim + page), LENGTHS[lengths]
    cache, table = paged(g, n, page, kv_heads, dim, head_major, t)
    q = normal(g, len(n), heads, dim, dtype=t, std=2.0)
    out = torch.full_like(q, 7.0)
    scale = dim ** -0.5
    want, bound = ref.attention(q, cache, table, n, scale, head_major)
    ln = torch.tensor(n, dtype=torch.int32, device="cuda")
    args = [ctx.from_torch(a) for a in (q, cache, table, ln)]
    lo = ctx.from_torch(out)
    ctx.paged_attention(*args, scale=scale, head_major=head_major, out=lo)
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lo) == out.data_ptr()
    close(out, want, bound)
    again = fetch(ctx, ctx.paged_attention(*args, scale=scale, head_major=head_major))
    assert torch.equal(again, out.cpu())  # the same bits every time


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("batch", [33, 300, 1025, 2100])
def test_paged_attention_many_sequences(ctx, dtype, batch):
    """More sequences than a block has threads, most of them empty, and a table far wider than any sequence."""
    t, g = TYPES[dtype], gen(12)
    n = [0] * batch
    for b, x in ((0, 3), (31, 130), (32, 5), (127, 200), (128, 1), (129, 65), (250, 0), (1023, 64), (1024, 66), (2047, 9), (batch - 1, 331)):
        if b < batch:
            n[b] = x
    cache, table = paged(g, n, 16, 2, 64, True, t, width=500)
    q = normal(g, batch, 8, 64, dtype=t)
    want, bound = ref.attention(q, cache, table, n, 0.2, True)
    y = ctx.paged_attention(*(ctx.from_torch(a) for a in (q, cache, table, torch.tensor(n, dtype=torch.int32, device="cuda"))), scale=0.2, head_major=True)
    close(fetch(ctx, y), want, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths", [
    (8, 1, 128, 64, [20000]), (4, 1, 256, 16, [9001, 0, 12]), (16, 2, 64, 48, [300, 7000, 64, 1]), (3, 3, 72, 16, [4097, 129]), (32, 1, 128, 16, [5000, 3000]),
    (8, 2, 128, 16, [1500, 17, 900, 2100, 64, 65, 0, 1300, 800, 1999, 33, 1024])])
def test_paged_attention_spread_over_blocks(ctx, dtype, heads, kv_heads, dim, page, lengths):
    """Sequences that many blocks share (up to as many as one may be spread over), beside short ones; unaligned as well,
    where the kernel for any shape shares them out."""
    t, g = TYPES[dtype], gen(heads + dim + page)
    cache, table = paged(g, lengths, page, kv_heads, dim, True, t)
    q = normal(g, len(lengths), heads, dim, dtype=t, std=1.5)
    want, bound = ref.attention(q, cache, table, lengths, dim ** -0.5, True)
    rest = [ctx.from_torch(table), ctx.from_torch(torch.tensor(lengths, dtype=torch.int32, device="cuda"))]
    lq, first = ctx.from_torch(q), None
    for lc in (ctx.from_torch(cache), unaligned(ctx, cache, dtype)):
        for again in range(3):
            y = fetch(ctx, ctx.paged_attention(lq, lc, *rest, scale=dim ** -0.5, head_major=True))
            if again == 0:
                close(y, want, bound)
                first = y
            assert torch.equal(y, first)  # whichever block comes last


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,dim,page,lengths", [(8, 1, 128, 16, [100000]), (5, 1, 64, 24, [31000, 70000, 40]), (40, 1, 64, 64, [40000]), (2, 1, 36, 16, [50000]), (6, 2, 256, 32, [33, 30000])])
def test_paged_attention_joined_in_two_steps(ctx, dtype, heads, kv_heads, dim, page, lengths):
    """So few and so long sequences that hundreds of blocks share each."""
    test_paged_attention_spread_over_blocks(ctx, dtype, heads, kv_heads, dim, page, lengths)


@pytest.mark.parametrize("by", [1, 2, 4])
def test_paged_attention_unaligned_and_sliced(ctx, by):
    g, n = gen(13), [70, 1, 200]
    cache, table = paged(g, n, 16, 2, 64, False, torch.bfloat16)
    qkv = normal(g, 3, 12, 64, dtype=torch.bfloat16)
    ln = torch.tensor(n, dtype=torch.int32, device="cuda")
    want, bound = ref.attention(qkv[:, 2:10], cache, table, n, 0.125, False)
    rest = [ctx.from_torch(table), ctx.from_torch(ln)]
    sliced = ctx.op("narrow", ctx.from_torch(qkv), dim=1, start=2, length=8)
    close(fetch(ctx, ctx.paged_attention(sliced, ctx.from_torch(cache), *rest, scale=0.125)), want, bound)
    close(fetch(ctx, ctx.paged_attention(sliced, unaligned(ctx, cache, "bf16", by), *rest, scale=0.125)), want, bound)
    lq = unaligned(ctx, qkv[:, 2:10].contiguous(), "bf16", by)
    close(fetch(ctx, ctx.paged_attention(lq, ctx.from_torch(cache), *rest, scale=0.125)), want, bound)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_paged_attention_extreme_scores(ctx, dtype):
    """Scores of hundreds, one token that takes all, infinities in the keys (weight nothing), a NaN that has to show."""
    t, g, n = TYPES[dtype], gen(14), [100, 100, 100, 100]
    cache, table = paged(g, n, 16, 1, 64, True, t)
    q = normal(g, 4, 4, 64, dtype=t)
    q[0] *= 300
    q[1] = q[1].abs()
    view = lambda b, i: (int(table[b, i // 16]), i % 16)  # noqa: E731
    p, o = view(1, 33)
    cache[p, 0, 0, o] = -math.inf  # score -inf for positive queries
    p, o = view(2, 99)
    cache[p, 1, 0, o, 5] = math.nan
    want, bound = ref.attention(q, cache, table, n, 0.125, True)
    assert torch.isnan(want[2, :, 5]).all() and not torch.isnan(want[[0, 3]]).any()
    bound = torch.nan_to_num(bound)
    y = fetch(ctx, ctx.paged_attention(*(ctx.from_torch(a) for a in (q, cache, table, torch.tensor(n, dtype=torch.int32, device="cuda"))), scale=0.125, head_major=True))
    close(y[[0, 2, 3]], want[[0, 2, 3]], bound[[0, 2, 3]])
    # without the token of weight nothing
    keep = [i for i in range(100) if i != 33]
    flat = token_view(cache, True).double().cpu()
    ids = [int(table[1, i // 16]) * 16 + i % 16 for i in keep]
    w = torch.softmax(0.125 * q[1].double().cpu() @ flat[0, ids, 0].T, -1)
    close(y[1], w @ flat[1, ids, 0], (w @ flat[1, ids, 0].abs()) * 2.0 ** -7)


def test_pages_and_lengths_outside_are_left_out_and_reported(ctx, lt):
    g, n = gen(15), [40, 40, 20]
    for t in (torch.bfloat16, torch.float32):
        cache, table = paged(g, n, 16, 2, 64, False, t)
        q = normal(g, 3, 4, 64, dtype=t)
        lq, lc = ctx.from_torch(q), ctx.from_torch(cache)
        bad = table.clone()
        bad[0, 1], bad[1, 0], bad[1, 1], bad[1, 2] = cache.shape[0], -1, 2147483647, -2147483648
        ln = torch.tensor(n, dtype=torch.int32, device="cuda")
        want, bound = ref.attention(q, cache, bad, n, 0.125, False)
        assert (want[1] == 0).all()
        out = torch.empty_like(q)
        lo = ctx.from_torch(out)
        ctx.paged_attention(lq, lc, ctx.from_torch(bad), ctx.from_torch(ln), scale=0.125, out=lo)
        with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*page"):
            ctx.barrier(blocking=True)
        close(out, want, bound)
        far = torch.tensor([40, -3, 2147483647], dtype=torch.int32, device="cuda")
        cut = table.clone()
        cut[2] = table[0]
        full = cut[:, :2].contiguous()  # two pages: 32 tokens
        want, bound = ref.attention(q, cache, full, [32, 0, 32], 0.125, False)
        ctx.paged_attention(lq, lc, ctx.from_torch(full), ctx.from_torch(far), scale=0.125, out=lo)
        with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX"):
            ctx.barrier(blocking=True)
        close(out, want, bound)
        ctx.barrier(blocking=True)


@pytest.mark.parametrize("head_major", [False, True])
def test_cache_of_more_than_2_to_the_32_values(ctx, lt, head_major):
    """Append to, and attend over, pages whose offsets do not fit 32 bits."""
    heads, dim, page = 8, 128, 64
    pages = (1 << 32) // (2 * page * heads * dim) + 40
    shape = (pages, 2, heads, page, dim) if head_major else (pages, 2, page, heads, dim)
    cache = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    assert cache.numel() > (1 << 32)
    g = gen(16)
    n = 300
    table = torch.arange(pages - 5, pages, dtype=torch.int32, device="cuda")[None].flip(1).contiguous()
    k, v = normal(g, n, heads, dim, dtype=torch.bfloat16), normal(g, n, heads, dim, dtype=torch.bfloat16)
    slots = (table[0, torch.arange(n, device="cuda") // page] * page + torch.arange(n, device="cuda") % page).to(torch.int32)
    q = normal(g, 1, 16, dim, dtype=torch.bfloat16)
    lc, out = ctx.from_torch(cache), torch.empty_like(q)
    lo = ctx.from_torch(out)
    ctx.cache_append(lc, ctx.from_torch(k), ctx.from_torch(v), ctx.from_torch(slots), head_major=head_major)
    ctx.paged_attention(ctx.from_torch(q), lc, ctx.from_torch(table), ctx.from_torch(torch.tensor([n], dtype=torch.int32, device="cuda")), scale=0.1,
                        head_major=head_major, out=lo)
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lc) == cache.data_ptr()
    small = torch.zeros((5, *shape[1:]), dtype=torch.bfloat16, device="cuda")
    small[:] = cache[pages - 5:]
    at = (slots - (pages - 5) * page).cpu().long()
    assert torch.equal(token_view(small, head_major)[0].cpu()[at], k.cpu())
    want, bound = ref.attention(q, small, table - (pages - 5), [n], 0.1, head_major)
    close(out, want, bound)


# ------------------------------------------------------------------------------------------------ norms
def decoded(codes):
    return codes.view(torch.float8_e4m3fn).float().double()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gamma_type", ["f32", "same"])
@pytest.mark.parametrize("rows,cols,residual", [(1, 1, False), (1, 4096, True), (5, 7, True), (3, 1000, False), (33, 1024, True), (2, 4095, True), (300, 136, True),
                                                (2, 16384, True), (2, 40000, False), (1, 65544, True), (700, 64, False)])
def test_rms_norm(ctx, dtype, gamma_type, rows, cols, residual):
    t, g = TYPES[dtype], gen(rows * 7 + cols)
    x = normal(g, rows, cols, dtype=t)
    r = normal(g, rows, cols, dtype=t, std=2.0) if residual else None
    gamma = (1 + normal(g, cols, std=0.2)).to(torch.float32 if gamma_type == "f32" else t)
    y, slack, h, hs = ref.rms_norm(x, gamma, r, 1e-5)
    got = ctx.rms_norm(ctx.from_torch(x), ctx.from_torch(gamma), residual=None if r is None else ctx.from_torch(r), eps=1e-5)
    ctx.barrier()
    assert ctx.dump_plan().count("launch ") == 1
    close(fetch(ctx, got[0]), y, slack + y.abs() * HALF[t])
    if residual:
        close(fetch(ctx, got[1]), h, hs + h.abs() * HALF[t])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
@pytest.mark.parametrize("rows,cols,residual", [(1, 1, False), (4, 4096, True), (3, 1000, True), (5, 100, False), (2, 8200, True), (1, 40000, False), (600, 256, True)])
def test_rms_norm_in_8_bits(ctx, dtype, group, rows, cols, residual):
    t, g = TYPES[dtype], gen(rows * 5 + cols + group)
    x = normal(g, rows, cols, dtype=t)
    r = normal(g, rows, cols, dtype=t) if residual else None
    if rows > 2:
        x[1] = 0  # a row of zeros
        if residual:
            r[1] = 0
    gamma = 1 + normal(g, cols, std=0.2)
    y, slack, h, hs = ref.rms_norm(x, gamma, r, 1e-6)
    got = ctx.rms_norm(ctx.from_torch(x), ctx.from_torch(gamma), residual=None if r is None else ctx.from_torch(r), eps=1e-6, eight_bit=True, group=group)
    ctx.barrier()
    assert ctx.dump_plan().count("launch ") == 1
    codes, scales = decoded(fetch(ctx, got[0])), fetch(ctx, got[1]).double()
    width = group or cols
    parts = y.split(width, -1)
    top = torch.stack([p.abs().amax(-1) for p in parts], -1)
    assert scales.shape == top.shape
    rel = (cols / 2 + 32) * ULP
    close(scales, top / 448, top / 448 * rel)
    value = torch.cat([p * torch.where(top[:, i: i + 1] > 0, 448 / top[:, i: i + 1], 0.0) for i, p in enumerate(parts)], -1)
    # half a step of e4m3: 2^-4 of the value, 2^-10 among the subnormal ones
    close(codes, value, torch.maximum(value.abs() * 2.0 ** -4, torch.tensor(2.0 ** -10, dtype=torch.float64)) + value.abs() * 2 * rel)
    if rows > 2:
        assert (codes[1] == 0).all() and (scales[1] == 0).all()
    if residual:
        close(fetch(ctx, got[2]), h, hs + h.abs() * HALF[t])


def test_rms_norm_with_nan_infinity_and_tiny_values(ctx):
    x = torch.ones(5, 512, device="cuda")
    x[0, 3], x[1, 200], x[2] = math.nan, math.inf, 1e-30
    x[4] = 3e18  # (a square fits, the sum of the squares does not)
    gamma = torch.ones(512, device="cuda")
    y, codes, scales = ctx.rms_norm(ctx.from_torch(x), ctx.from_torch(gamma))[0], *ctx.rms_norm(ctx.from_torch(x), ctx.from_torch(gamma), eight_bit=True, group=128)
    y, codes, scales = fetch(ctx, y), decoded(fetch(ctx, codes)), fetch(ctx, scales)
    assert torch.isnan(y[0]).all() and torch.isnan(codes[0]).all() and torch.isnan(scales[0]).all()
    assert torch.isnan(y[1, 200]) and (y[1, :200] == 0).all()  # infinity over infinity; the rest over infinity
    assert torch.isnan(scales[1, 1]) and (scales[1, [0, 2, 3]] == 0).all() and (codes[1, :128] == 0).all()
    close(y[2:], torch.tensor([1e-30 / 1e-3, 1.0, 1.0])[:, None].expand(3, 512), torch.tensor([1e-27, 1e-6, 1e-6])[:, None].expand(3, 512) * 300 * ULP + 1e-6 * torch.tensor([0.0, 1, 1])[:, None])
    assert (codes[3:] == 448).all()


@pytest.mark.parametrize("top", [1e-35, 1e-36, 1e-37, 1e-38, 1e-40])
@pytest.mark.parametrize("cols", [512, 500, 499, 8195])
def test_rms_norm_in_8_bits_of_groups_next_to_nothing(ctx, cols, top):
    """y / scale, however small the largest y of a group is: 448, 224 and 112 for it, its half and its quarter."""
    x = torch.ones(3, cols, device="cuda")
    x[:, 1::3] *= 0.5
    x[:, 2::3] *= -0.25
    gamma = torch.full((cols,), top * math.sqrt(0.4375), device="cuda")  # (the mean of the squares is about 0.4375)
    for group in (0, 128):
        codes, scales = ctx.rms_norm(ctx.from_torch(x), ctx.from_torch(gamma), eight_bit=True, group=group)
        assert torch.equal(decoded(fetch(ctx, codes)), (448 * x).cpu().double())
        y = ref.rms_norm(x, gamma, None, 1e-6)[0].abs().amax()
        # what y loses where its last bit is worth 2^-149, and the scale
        assert float((fetch(ctx, scales).double() - y / 448).abs().max()) <= float(y / 448) * 600 * ULP + 2 * 2.0 ** -149


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rms_norm_slices_unaligned_and_in_place(ctx, dtype):
    t, g = TYPES[dtype], gen(21)
    wide = normal(g, 9, 3, 512, dtype=t)
    r = normal(g, 9, 512, dtype=t)
    gamma = 1 + normal(g, 512, std=0.1)
    lw, lr, lg = ctx.from_torch(wide.view(9, 1536)), ctx.from_torch(r), ctx.from_torch(gamma)
    for i, cols in ((0, 512), (2, 512)):
        y, slack, h, hs = ref.rms_norm(wide[:, i], gamma, r, 1e-6)
        got = ctx.rms_norm(ctx.op("narrow", lw, dim=1, start=512 * i, length=512), lg, residual=lr)
        ctx.barrier()
        assert "copy kernel" not in ctx.dump_plan()
        close(fetch(ctx, got[0]), y, slack + y.abs() * HALF[t])
        close(fetch(ctx, got[1]), h, hs + h.abs() * HALF[t])
    odd = ctx.op("narrow", lw, dim=1, start=3, length=512)  # rows that start off the 16-byte grid
    y, slack, h, hs = ref.rms_norm(wide.view(9, 1536)[:, 3:515], gamma, None, 1e-6)
    close(fetch(ctx, ctx.rms_norm(odd, lg)[0]), y, slack + y.abs() * HALF[t])
    x = wide[:, 1].contiguous()
    y, slack, h, hs = ref.rms_norm(x, gamma, r, 1e-6)
    got = ctx.rms_norm(unaligned(ctx, x, dtype), unaligned(ctx, gamma, "f32"), residual=unaligned(ctx, r, dtype, 3))
    close(fetch(ctx, got[0]), y, slack + y.abs() * HALF[t])
    # the residual stream updated in place, the normalised values over x
    lx, own, res = ctx.from_torch(x), x, r.clone()
    lres = ctx.from_torch(res)
    ctx.rms_norm(lx, lg, residual=lres, out=(lx, lres))
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lx) == own.data_ptr() and ctx.device_ptr(lres) == res.data_ptr()
    close(own, y, slack + y.abs() * HALF[t])
    close(res, h, hs + h.abs() * HALF[t])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gamma_type", ["f32", "same"])
@pytest.mark.parametrize("rows,cols,direct", [(1, 1, False), (1, 1000, True), (7, 33, True), (64, 1024, False), (1500, 64, True), (3, 8192, True), (2, 40000, False), (1300, 520, False)])
def test_rms_norm_grad(ctx, dtype, gamma_type, rows, cols, direct):
    t, g = TYPES[dtype], gen(rows + cols)
    dy, h = normal(g, rows, cols, dtype=t), normal(g, rows, cols, dtype=t, std=2.0)
    dh = normal(g, rows, cols, dtype=t) if direct else None
    gt = torch.float32 if gamma_type == "f32" else t
    gamma = (1 + normal(g, cols, std=0.2)).to(gt)
    dx, bx, dg, bg = ref.rms_norm_grad(dy, h, gamma, dh, 1e-6)
    got = ctx.rms_norm_grad(*(ctx.from_torch(a) for a in (dy, h, gamma)), residual_grad=None if dh is None else ctx.from_torch(dh))
    a, b = fetch(ctx, got[0]), fetch(ctx, got[1])
    close(a, dx, bx, "dx")
    close(b, dg, bg + dg.abs() * HALF[gt], "dgamma")
    alone = ctx.op("rms_norm_grad", *(ctx.from_torch(x) for x in (dy, h, gamma)), *(() if dh is None else (ctx.from_torch(dh),)), result=1, residual=direct, eps=1e-6)
    assert torch.equal(fetch(ctx, alone), b)  # alone or together, the same bits


def test_rms_norm_grad_against_differences(ctx):
    g = gen(31)
    h, dy, gamma = normal(g, 3, 24), normal(g, 3, 24), 1 + normal(g, 24, std=0.3)
    dx, dg = (fetch(ctx, t).double() for t in ctx.rms_norm_grad(*(ctx.from_torch(a) for a in (dy, h, gamma)), eps=1e-3))

    def loss(h, gamma):
        return float((dy.double().cpu() * gamma * h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-3)).sum())

    h64, g64, step = h.double().cpu(), gamma.double().cpu(), 1e-5
    for r, c in ((0, 0), (1, 7), (2, 23)):
        e = torch.zeros_like(h64)
        e[r, c] = step
        assert abs((loss(h64 + e, g64) - loss(h64 - e, g64)) / (2 * step) - float(dx[r, c])) < 1e-5
        e = torch.zeros_like(g64)
        e[c] = step
        assert abs((loss(h64, g64 + e) - loss(h64, g64 - e)) / (2 * step) - float(dg[c])) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", [(3, 64), (400, 1024), (2, 16384), (5, 33), (40, 999), (3, 2001), (2, 40000)])
def test_rms_norm_grad_of_large_values(ctx, dtype, rows, cols):
    """The sum of dy gamma h does not fit into binary32; the mean of dy gamma h / rms does, and so do the gradients."""
    t, g = TYPES[dtype], gen(rows + cols)
    dy, h = normal(g, rows, cols, dtype=t, std=1e24), normal(g, rows, cols, dtype=t, std=1e18)
    gamma = 1 + normal(g, cols, std=0.2)
    dx, bx, dg, bg = ref.rms_norm_grad(dy, h, gamma, None, 1e-6)
    got = ctx.rms_norm_grad(*(ctx.from_torch(a) for a in (dy, h, gamma)))
    close(fetch(ctx, got[0]), dx, bx, "dx")
    close(fetch(ctx, got[1]), dg, bg + dg.abs() * ULP, "dgamma")


def test_rms_norm_grad_slices_and_in_place(ctx):
    g = gen(33)
    for dtype, t in TYPES.items():
        wide = normal(g, 40, 3 * 256, dtype=t)
        gamma = 1 + normal(g, 256, std=0.1)
        lw, lg = ctx.from_torch(wide), ctx.from_torch(gamma)
        a, b, c = (wide[:, 256 * i: 256 * i + 256] for i in range(3))
        dx, bx, dg, bg = ref.rms_norm_grad(a, b, gamma, c, 1e-6)
        la, lb, lc = (ctx.op("narrow", lw, dim=1, start=256 * i, length=256) for i in range(3))
        got = ctx.rms_norm_grad(la, lb, lg, residual_grad=lc)
        del la, lb, lc  # (slices that are still named are results of their own)
        ctx.barrier()
        assert "copy kernel" not in ctx.dump_plan()
        close(fetch(ctx, got[0]), dx, bx)
        close(fetch(ctx, got[1]), dg, bg + dg.abs() * ULP)
        la, lb = (ctx.op("narrow", lw, dim=1, start=256 * i, length=256) for i in range(2))
        own = c.contiguous()
        lo, into = ctx.from_torch(own), torch.empty(256, device="cuda")
        li = ctx.from_torch(into)
        ctx.rms_norm_grad(la, lb, lg, residual_grad=lo, out=(lo, li))
        ctx.barrier(blocking=True)
        assert ctx.device_ptr(lo) == own.data_ptr()
        close(own, dx, bx)
        close(into, dg, bg + dg.abs() * ULP)


# ------------------------------------------------------------------------------------------------ many rows
# More rows than the blocks have at once, several times over: rows to come, their rings and what blocks keep from row to row.
MANY = [(40000, 64), (8192, 4096), (3000, 8192), (1500, 16384), (8000, 999), (12000, 333), (30000, 131), (3000, 4095), (2500, 1400)]


def near(got, want, bound, what):
    """As close(), on the GPU."""
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    if bool(bad.any()):
        at = int(torch.argmax(torch.where(bad, off - bound, torch.zeros_like(off))))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} too far; at {at}: {got.flatten()[at]} for {want.flatten()[at]}, bound {bound.flatten()[at]}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", MANY)
def test_rms_norm_many_rows(ctx, dtype, rows, cols):
    t, g = TYPES[dtype], gen(rows + cols)
    gamma = 1 + normal(g, cols, std=0.2)
    for residual, group in ((True, None), (False, None), (True, 0), (True, 128), (False, 64)):
        x = normal(g, rows, cols, dtype=t)
        r = normal(g, rows, cols, dtype=t, std=2.0) if residual else None
        h = x.double() + (r.double() if residual else 0.0)
        y = gamma.double() * h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6)
        rel = (cols / 2 + 32) * ULP
        lx, lg, lr = ctx.from_torch(x), ctx.from_torch(gamma), ctx.from_torch(r) if residual else None
        if group is None:  # in place: y over x, the sum over the residual
            ctx.rms_norm(lx, lg, residual=lr, out=(lx, lr) if residual else (lx,))
        else:
            width = group or cols
            parts = y.split(width, -1)
            top = torch.stack([p.abs().amax(-1) for p in parts], -1)
            codes = torch.empty(rows, cols, dtype=torch.uint8, device="cuda")
            scales = torch.empty(rows, len(parts), device="cuda")
            kept = [ctx.from_torch(codes), ctx.from_torch(scales)] + ([lr] if residual else [])  # (named until the barrier)
            ctx.rms_norm(lx, lg, residual=lr, eight_bit=True, group=group, out=kept)
        ctx.barrier(blocking=True)
        what = (residual, group)
        if group is None:
            assert ctx.device_ptr(lx) == x.data_ptr()
            near(x, y, y.abs() * (rel + HALF[t]), what)
        else:
            near(scales, top / 448, top / 448 * rel, what)
            value = torch.cat([p * (448 / top[:, i: i + 1]) for i, p in enumerate(parts)], -1)
            near(codes.view(torch.float8_e4m3fn), value, (value.abs() * 2.0 ** -4).clamp(min=2.0 ** -10) + value.abs() * 2 * rel, what)
        if residual:
            assert ctx.device_ptr(lr) == r.data_ptr()
            near(r, h, h.abs() * (ULP + HALF[t]), what)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,cols", MANY + [(16384, 1024)])
def test_rms_norm_grad_many_rows(ctx, dtype, rows, cols):
    t, g = TYPES[dtype], gen(rows + cols + 1)
    gamma = 1 + normal(g, cols, std=0.2)
    for direct in (True, False):
        dy, h = normal(g, rows, cols, dtype=t), normal(g, rows, cols, dtype=t, std=2.0)
        dh = normal(g, rows, cols, dtype=t) if direct else None
        h64, d = h.double(), dy.double() * gamma.double()
        inv = 1 / torch.sqrt((h64 * h64).mean(-1, keepdim=True) + 1e-6)
        u = h64 * inv
        e = dh.double() if direct else torch.zeros((), device="cuda", dtype=torch.float64)
        dx = e + inv * (d - u * (d * u).mean(-1, keepdim=True))
        size = inv * (d.abs() + u.abs() * (d * u).abs().mean(-1, keepdim=True)) + e.abs()
        dgamma, total = (dy.double() * u).sum(0), (dy.double() * u).abs().sum(0)
        into = torch.empty(cols, device="cuda")
        lh, li = ctx.from_torch(h), ctx.from_torch(into)
        ctx.rms_norm_grad(ctx.from_torch(dy), lh, ctx.from_torch(gamma), residual_grad=ctx.from_torch(dh) if direct else None, out=(lh, li))
        ctx.barrier(blocking=True)
        assert ctx.device_ptr(lh) == h.data_ptr()
        near(h, dx, dx.abs() * HALF[t] + size * (2 * cols + 64) * ULP, ("dx", direct))
        # u: a sum over the row; then the rows of a block one after the other (there are as many blocks as SMs at least), blocks in 64 bits
        near(into, dgamma, total * (cols / 2 + 32 + rows / 148 + 16) * ULP, ("dgamma", direct))


# ------------------------------------------------------------------------------------------------ together
class Decoder:
    """One layer's operators of a decode step, as a program records them: norm in, rotation, append, attention, norm out."""

    def __init__(self, lt, ctx, g, batch=5, heads=8, kv_heads=2, dim=64, page=16, most=8, dtype=torch.bfloat16):
        self.lt, self.ctx, self.heads, self.kv, self.dim, self.page, self.t = lt, ctx, heads, kv_heads, dim, page, dtype
        self.cols = heads * dim
        self.table = torch.randperm(batch * most, generator=g, device="cuda").to(torch.int32).view(batch, most)
        self.cache = torch.full((batch * most, 2, kv_heads, page, dim), math.nan, device="cuda", dtype=dtype)
        self.gamma = 1 + normal(g, self.cols, std=0.1)
        self.x, self.res = normal(g, batch, self.cols, dtype=dtype), normal(g, batch, self.cols, dtype=dtype)
        self.qkv = torch.zeros(batch, heads + 2 * kv_heads, dim, device="cuda", dtype=dtype)
        self.pos, self.slots, self.len = (torch.zeros(batch, dtype=torch.int32, device="cuda") for _ in range(3))
        self.att, self.y = torch.empty(batch, heads, dim, device="cuda", dtype=dtype), torch.empty(batch, self.cols, device="cuda", dtype=dtype)
        b = lt.Batch()
        hs = []

        def use(t):
            hs.append(ctx.from_torch(t))
            return b.input()

        cache, qkv, pos, slots, ln, table, att = (use(t) for t in (self.cache, self.qkv, self.pos, self.slots, self.len, self.table, self.att))
        f = use(torch.from_numpy(lt.rotary_table(dim).view(np.int32)).cuda().view(torch.uint32))
        q = b.rotary(b.op("narrow", qkv, dim=1, start=0, length=heads), pos, f)
        b.cache_append(cache, b.op("narrow", qkv, dim=1, start=heads, length=kv_heads), b.op("narrow", qkv, dim=1, start=heads + kv_heads, length=kv_heads), slots, pos, f,
                       head_major=True)
        b.paged_attention(q, cache, table, ln, scale=dim ** -0.5, head_major=True, out=att)
        x, res, gamma, y = (use(t) for t in (self.x, self.res, self.gamma, self.y))
        b.rms_norm(x, gamma, residual=res, out=(y, res))
        self.batch, self.handles = b, hs

    def step(self, g, n, flush=None):
        """One token for every sequence with n[b] >= 0 tokens before it (n[b] < 0: padding); returns what it has to give."""
        alive = torch.tensor([x >= 0 for x in n])
        at = torch.tensor([max(x, 0) for x in n], device="cuda")
        self.qkv.copy_(normal(g, *self.qkv.shape, dtype=self.t))
        self.x.copy_(normal(g, *self.x.shape, dtype=self.t))
        self.pos.copy_(at)
        self.len.copy_(torch.where(alive.cuda(), at + 1, 0))
        slot = torch.gather(self.table, 1, (at // self.page)[:, None].long())[:, 0] * self.page + at % self.page
        self.slots.copy_(torch.where(alive.cuda(), slot, -1))
        res = self.res.clone()
        self.ctx.record(self.batch, self.handles)
        (flush or self.ctx.barrier)()
        torch.cuda.synchronize()
        f = ref.frequencies(self.dim)
        q, _ = ref.rotary(self.qkv[:, : self.heads], self.pos, f)
        k, kb = ref.rotary(self.qkv[:, self.heads: self.heads + self.kv], self.pos, f)
        flat = token_view(self.cache, True).cpu()
        s = self.slots.cpu().long()
        close(flat[0][s[alive]], k[alive], kb[alive], "cache")
        assert torch.equal(flat[1][s[alive]], self.qkv[:, self.heads + self.kv:].cpu()[alive])
        want, bound = ref.attention(q.to(self.t), self.cache, self.table, self.len.tolist(), self.dim ** -0.5, True)
        # the rotated query is rounded to bf16: half a step of it, or the whole one where 32 bits put it on the other side of a border;
        # a score moves by at most 2^-8 of |q| |k| scale, about 16 / 8, and the weights with it
        close(self.att, want, bound + want.abs() * 2 ** -5 + 0.05, "attention")
        y, slack, h, hs = ref.rms_norm(self.x, self.gamma, res, 1e-6)
        close(self.y, y, slack + y.abs() * HALF[self.t], "norm")
        close(self.res, h, hs + h.abs() * HALF[self.t], "residual")


def test_decode_steps(ctx, lt):
    """Steps of a batch whose sequences grow past page borders and whose rows come and go, recorded the same way every time."""
    g = gen(41)
    d = Decoder(lt, ctx, g)
    n = [0, 0, -1, 0, 0]
    for i in range(20):
        d.step(g, n)
        n = [x + 1 if x >= 0 else x for x in n]
    st = ctx.stats()
    assert st["compiles"] == 1 and st["cache_hits"] == 19
    plan = ctx.dump_plan()
    assert plan.count("launch ") == 4 and "copy kernel" not in plan


def test_on_another_stream_and_device_current(ctx, lt):
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = lt.LazyContext(device=0, stream=s.cuda_stream)
        g = gen(42)
        d = Decoder(lt, c, g)
        s.synchronize()
        for i in range(3):
            d.step(g, [i, i, i, -1, i])
        c.close()


def test_captured_flushes(lt):
    """Steps captured into graphs and replayed on new values: results go to the caller's buffers, temporaries to the
    static scratch.  Two graphs of one context replay one after the other."""
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c = lt.LazyContext(device=0, stream=s.cuda_stream)
        g = gen(43)
        a, b = Decoder(lt, c, g, batch=3), Decoder(lt, c, g, batch=4, heads=16, kv_heads=2)
        att_a, att_b = a.att, b.att
        table = c.leaf(lt.rotary_table(64), "u32")
        x = normal(g, 6, 8, 64)
        pos = torch.arange(6, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(x)
        lx, lp, lo = c.from_torch(x), c.from_torch(pos), c.from_torch(out)
        cache, tb = paged(g, [200, 90], 16, 2, 64, True, torch.bfloat16)
        q, q2 = normal(g, 2, 8, 64, dtype=torch.bfloat16), normal(g, 2, 8, 64, dtype=torch.bfloat16)
        ln = torch.tensor([200, 90], dtype=torch.int32, device="cuda")
        o1, o2 = torch.zeros_like(q), torch.zeros_like(q)
        args = [c.from_torch(t) for t in (cache, tb, ln)]
        lq, lq2, lo1, lo2 = (c.from_torch(t) for t in (q, q2, o1, o2))

        def one():
            c.rotary(lx, lp, table, out=lo)
            c.paged_attention(lq, *args, scale=0.125, head_major=True, out=lo1)
            c.barrier_static_scratch()

        def two():
            c.paged_attention(lq2, *args, scale=0.25, head_major=True, out=lo2)
            c.barrier_static_scratch()

        one(), two()
        s.synchronize()
        graphs = []
        for f in (one, two):
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=s):
                f()
            graphs.append(gr)
        q.copy_(normal(g, 2, 8, 64, dtype=torch.bfloat16)), q2.copy_(normal(g, 2, 8, 64, dtype=torch.bfloat16))
        x.copy_(normal(g, 6, 8, 64))
        o1.zero_(), o2.zero_(), out.zero_()
        for gr in graphs * 2:
            gr.replay()
        s.synchronize()
        close(out, *ref.rotary(x, pos, ref.frequencies(64)))
        close(o1, *ref.attention(q, cache, tb, [200, 90], 0.125, True))
        close(o2, *ref.attention(q2, cache, tb, [200, 90], 0.25, True))
        del graphs, gr, att_a, att_b
        c.close()


def test_first_attention_of_a_context_is_captured(lt):
    """An ordinary barrier under capture, in a context that has flushed no attention yet: the graph and the flushes after
    it do not depend on counters that only the graph sets."""
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        warm, c = lt.LazyContext(device=0, stream=s.cuda_stream), lt.LazyContext(device=0, stream=s.cuda_stream)
        g = gen(47)
        n = [5000, 300]
        cache, table = paged(g, n, 16, 2, 64, False, torch.bfloat16)
        q, out, ln = normal(g, 2, 8, 64, dtype=torch.bfloat16), torch.zeros(2, 8, 64, device="cuda", dtype=torch.bfloat16), torch.tensor(n, dtype=torch.int32, device="cuda")

        def step(ctx):
            handles = [ctx.from_torch(t) for t in (q, cache, table, ln, out)]
            ctx.paged_attention(*handles[:4], scale=0.125, out=handles[4])
            ctx.barrier()
            return handles

        kept = [step(warm)]
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            kept.append(step(c))
        kept.append(step(c))
        s.synchronize()
        want = ref.attention(q, cache, table, n, 0.125, False)
        close(out, *want)
        for _ in range(2):
            out.zero_()
            graph.replay()
            s.synchronize()
            close(out, *want)
        del graph, kept
        warm.close(), c.close()


def captured_attention(lt, seed, stream, n, warm, allocator="torch"):
    """(graph of one ordinary barrier with an attention, context, tensors, what it has to give) on `stream`."""
    with torch.cuda.stream(stream):
        c, g = lt.LazyContext(device=0, stream=stream.cuda_stream, allocator=allocator), gen(seed)
        cache, table = paged(g, n, 16, 2, 64, False, torch.bfloat16)
        q, ln = normal(g, len(n), 8, 64, dtype=torch.bfloat16), torch.tensor(n, dtype=torch.int32, device="cuda")
        out = torch.zeros_like(q)
        handles = [c.from_torch(t) for t in (q, cache, table, ln, out)]

        def step():
            c.paged_attention(*handles[:4], scale=0.125, out=handles[4])
            c.barrier()

        if warm:
            step()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        stream.synchronize()
    return graph, c, (q, cache, table, ln, out, handles), ref.attention(q, cache, table, n, 0.125, False)


def test_captured_barriers_share_nothing_and_outlive_their_contexts(lt):
    """Graphs of ordinary barriers, of contexts that have flushed an attention before and of new ones, replayed side by side on
    their streams; then once more when the contexts are closed and what they gave back is somebody else's."""
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    lengths = ([5000, 300], [9000], [40, 3000, 2000])
    made = [captured_attention(lt, 60 + i, s, n, warm) for i, (s, n, warm) in enumerate(zip(streams, lengths, (False, False, True)))]

    def replay():
        for _, _, t, _ in made:
            t[4].zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for (graph, *_), s in zip(made, streams):
                with torch.cuda.stream(s):
                    graph.replay()
        torch.cuda.synchronize()
        for _, _, t, want in made:
            close(t[4], *want)

    replay()
    for _, c, t, _ in made:
        t[5].clear()
        c.close()
    torch.cuda.synchronize()
    taken = []
    for s in streams:  # what the contexts held goes to whoever asks on their streams
        with torch.cuda.stream(s):
            taken += [torch.full((size,), 0x7fc07fc0, dtype=torch.int32, device="cuda") for size in [2048] * 64 + [1 << 17] * 16 + [1 << 20] * 8]
    torch.cuda.synchronize()
    replay()
    for t in taken:
        assert bool((t == 0x7fc07fc0).all())


@pytest.mark.parametrize("allocator", ["torch", "none"])
def test_two_graphs_of_one_context_replay_side_by_side(lt, allocator):
    """Attention and the norm's gradient, whose blocks leave parts in temporaries; the context flushes between the replays."""
    s, others = torch.cuda.Stream(), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c, g = lt.LazyContext(device=0, stream=s.cuda_stream, allocator=allocator), gen(82)
        n = [7000, 900]
        cache, table = paged(g, n, 16, 2, 64, False, torch.bfloat16)
        ln, gamma = torch.tensor(n, dtype=torch.int32, device="cuda"), 1 + normal(g, 640, std=0.2)
        dy = normal(g, 3000, 640)
        data, graphs = [], []
        for i in range(3):
            q, h = normal(g, 2, 8, 64, dtype=torch.bfloat16), normal(g, 3000, 640)
            outs = torch.zeros_like(q), torch.zeros_like(h), torch.zeros(640, device="cuda")
            data.append((q, h, *outs, [c.from_torch(t) for t in (q, cache, table, ln, dy, h, gamma, *outs)]))

        def step(i):
            q, ca, tb, l, d, h, ga, att, dx, dg = data[i][5]
            c.paged_attention(q, ca, tb, l, scale=0.125, out=att)
            c.rms_norm_grad(d, h, ga, out=(dx, dg))
            c.barrier()

        step(2)
        s.synchronize()
        for i in range(2):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                step(i)
            graphs.append(graph)
        s.synchronize()
    for _ in range(20):
        for graph, o in zip(graphs, others):
            with torch.cuda.stream(o):
                graph.replay()
        step(2)
    torch.cuda.synchronize()
    for q, h, att, dx, dg, _ in data:
        close(att, *ref.attention(q, cache, table, n, 0.125, False))
        a, b, e, f = ref.rms_norm_grad(dy, h, gamma, None, 1e-6)
        close(dx, a, b)
        close(dg, e, f + e.abs() * ULP)
    for d in data:
        d[5].clear()
    c.close()


def test_captured_barrier_without_allocator_callbacks(lt):
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for warm in (False, True):
        graph, c, t, want = captured_attention(lt, 70, s, [5000, 300], warm, allocator="none")
        for _ in range(3):
            with torch.cuda.stream(s):
                t[4].zero_()
                graph.replay()
            s.synchronize()
            close(t[4], *want)
        with torch.cuda.stream(s):
            t[4].zero_()
            c.paged_attention(*t[5][:4], scale=0.125, out=t[5][4])
            c.barrier(blocking=True)
        close(t[4], *want)
        t[5].clear()
        c.close()


@pytest.mark.parametrize("warm", [False, True])
def test_results_of_a_captured_barrier_are_not_handed_out_again(lt, warm):
    """Results without a buffer of the caller's, and what passes between a graph's kernels: neither is what a later flush gets."""
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        c, g = lt.LazyContext(device=0, stream=s.cuda_stream), gen(81)
        x, gamma = normal(g, 64, 512), 1 + normal(g, 512, std=0.2)
        lx, lg = c.from_torch(x), c.from_torch(gamma)

        def step():
            y, = c.rms_norm(lx, lg)
            z, = c.rms_norm(y, lg)
            del y
            c.barrier()
            return z

        if warm:
            z = step()
            del z
            c.barrier(blocking=True)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            z = step()

        def want():
            return ref.rms_norm(ref.rms_norm(x, gamma, None, 1e-6)[0], gamma, None, 1e-6)[0]

        for _ in range(2):
            x.copy_(normal(g, 64, 512))
            graph.replay()
            close(fetch(c, z), want(), want().abs() * 2000 * ULP)
        taken = c.device_ptr(z)
        del z
        c.barrier(blocking=True)
        later = [step() for _ in range(3)]
        kept = [fetch(c, z) for z in later]
        assert all(c.device_ptr(z) != taken for z in later)
        x.copy_(normal(g, 64, 512))
        graph.replay()
        s.synchronize()
        for z, k in zip(later, kept):
            assert torch.equal(fetch(c, z), k)
        del later, z
        c.close()


def test_bad_pages_in_a_replayed_graph_are_reported(lt):
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph, c, (q, cache, table, ln, out, handles), want = captured_attention(lt, 75, s, [300, 500], True)
    with torch.cuda.stream(s):
        c.barrier(blocking=True)
        for i in range(3):
            good = table.clone()
            graph.replay()
            c.barrier(blocking=True)
            close(out, *want)
            table[1, i] = cache.shape[0] + i
            graph.replay()
            with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*page"):
                c.barrier(blocking=True)
            close(out, *ref.attention(q, cache, table, [300, 500], 0.125, False))
            table.copy_(good)
    handles.clear()
    c.close()


FIRST_CONTEXT_UNDER_CAPTURE = """
import torch
import paper_2102_13267_b200 as lt

s = torch.cuda.Stream()
with torch.cuda.stream(s):
    x = torch.ones(4, 2, 8, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    table = torch.from_numpy(lt.rotary_table(8).view("int32")).cuda()
    out = torch.zeros_like(x)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        c = lt.LazyContext(device=0, stream=s.cuda_stream)
        handles = [c.from_torch(x), c.from_torch(pos), c.from_torch(table, "u32"), c.from_torch(out)]
        c.rotary(*handles[:3], out=handles[3])
        c.barrier()
    graph.replay()
    s.synchronize()
    assert torch.equal(out, x), out
    handles.clear()
    c.close()
print("replayed")
"""


def test_first_context_of_a_process_is_made_under_capture():
    done = subprocess.run([sys.executable, "-c", FIRST_CONTEXT_UNDER_CAPTURE], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), capture_output=True, text=True, timeout=300)
    assert done.returncode == 0 and "replayed" in done.stdout, done.stderr[-2000:]


def test_replay(ctx, lt):
    """lt_replay runs the step again on the tensors' current values."""
    g = gen(44)
    d = Decoder(lt, ctx, g)
    d.step(g, [0, 0, 0, 0, 0])
    d.step(g, [1, 1, 1, 1, 1])

    class Again:
        def record(self, *a):
            pass
    real, d.ctx = d.ctx, Again()
    for i in range(2, 5):
        d.step(g, [i] * 5, flush=real.replay)


def test_unfused_and_static_scratch_give_the_same(lt):
    g = gen(45)
    x, r, gamma = normal(g, 20, 512, dtype=torch.bfloat16), normal(g, 20, 512, dtype=torch.bfloat16), 1 + normal(g, 512, std=0.1)
    got = []
    for fusion in (1, 0):
        c = lt.LazyContext(device=0)
        c.set_option("fusion", fusion)
        t = c.rms_norm(c.from_torch(x), c.from_torch(gamma), residual=c.from_torch(r), eight_bit=True, group=64)
        c.barrier()
        assert c.dump_plan().count("launch ") == (1 if fusion else 3)
        got.append([c.fetch(v) for v in t])
        del t
        c.close()
    for a, b in zip(*got):
        np.testing.assert_array_equal(a, b)


def test_operators_among_traced_operations(ctx, lt):
    """Operators read what fused groups compute and are read by them."""
    g = gen(46)
    x, gamma = normal(g, 12, 256, dtype=torch.bfloat16), 1 + normal(g, 256, std=0.1)
    lx = ctx.from_torch(x)
    twice = lx + lx
    y = ctx.rms_norm(twice, ctx.from_torch(gamma), residual=lx)
    z = ctx.op("relu", y[0]) + y[1]
    want, slack, h, hs = ref.rms_norm((2 * x.float()).to(torch.bfloat16), gamma, x, 1e-6)
    yy, hh = fetch(ctx, y[0]), fetch(ctx, y[1])
    close(yy, want, slack + want.abs() * HALF[torch.bfloat16])
    close(hh, h, hs + h.abs() * HALF[torch.bfloat16])
    zz = fetch(ctx, z)
    close(zz, (yy.float().clamp(min=0) + hh.float()).to(torch.bfloat16), zz.double().abs() * 0)
