"""Lookup in a table, cross entropy against it, and their gradients on the GPU against their definitions in 64 bits
(table_reference), through the public entry points."""
import math

import numpy as np
import pytest
import torch

import table_reference as ref
from operator_reference import HALF, TYPES, ULP, close
from test_gpu_operators import ctx, fetch, gen, lt, normal, unaligned  # noqa: F401

pytestmark = pytest.mark.gpu


def tokens_of(g, n, vocab, skew=True):
    u = torch.rand(n, device="cuda", dtype=torch.float64, generator=g)
    return ((torch.exp(u * math.log(vocab + 1)).long() - 1 if skew else (u * vocab).long()).clamp(0, vocab - 1)).to(torch.int32)


# ------------------------------------------------------------------------------------------------ lookup
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (1, 32000, 4096), (3, 7, 8), (37, 100, 33), (5000, 300, 64), (129, 1000, 2056), (70, 50, 12), (4097, 65, 1000), (9, 3, 16384)])
def test_embedding(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    g, t = gen(tokens + cols), TYPES[dtype]
    table, ids = normal(g, vocab, cols, dtype=t), tokens_of(g, tokens, vocab, False)
    if tokens > 2:
        ids[1], ids[-1] = -1, -(1 << 31)
    close(fetch(ctx, ctx.embedding(ctx.from_torch(table), ctx.from_torch(ids), scale=1.75)), *ref.embedding(table, ids, 1.75))
    got = fetch(ctx, ctx.embedding(ctx.from_torch(table), ctx.from_torch(ids)))
    assert torch.equal(got.double(), ref.embedding(table, ids)[0])  # without a scale nothing is rounded


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embedding_of_a_slice_and_unaligned(ctx, dtype):  # noqa: F811
    g, t = gen(3), TYPES[dtype]
    wide, ids = normal(g, 40, 96, dtype=t), tokens_of(g, 6 * 9, 40).reshape(6, 9)
    for start, length in ((32, 32), (5, 31), (8, 40)):
        part = ctx.op("narrow", ctx.from_torch(wide), dim=1, start=start, length=length)
        y = ctx.embedding(part, ctx.from_torch(ids))
        del part
        assert torch.equal(fetch(ctx, y).double(), ref.embedding(wide[:, start: start + length], ids)[0])
    assert torch.equal(fetch(ctx, ctx.embedding(unaligned(ctx, wide, dtype), unaligned(ctx, ids, "i32"))).double(), ref.embedding(wide, ids)[0])


def test_embedding_far_into_a_large_table(ctx):  # noqa: F811
    """Rows behind 2^31 elements, and results behind 2^31 bytes."""
    table = torch.zeros((1 << 20) + 3, 2056, device="cuda", dtype=torch.bfloat16)
    ids = torch.tensor([(1 << 20) + 2, 0, (1 << 20) + 1], dtype=torch.int32, device="cuda").repeat(180000)
    table[(1 << 20) + 2], table[(1 << 20) + 1], table[0] = 3.0, 5.0, 7.0
    out = torch.empty(540000, 2056, device="cuda", dtype=torch.bfloat16)
    lo = ctx.from_torch(out)
    ctx.embedding(ctx.from_torch(table), ctx.from_torch(ids), out=lo)
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lo) == out.data_ptr()
    want = torch.tensor([3.0, 7.0, 5.0], device="cuda", dtype=torch.bfloat16).repeat(180000)
    assert bool((out == want[:, None]).all())


# ------------------------------------------------------------------------------------------------ its gradient
def check_grad(ctx, dy, ids, rows, base=None, scale=1.0):  # noqa: F811
    got = ctx.embedding_grad(ctx.from_torch(dy), ctx.from_torch(ids), rows, base=None if base is None else ctx.from_torch(base), scale=scale)
    close(fetch(ctx, got), *ref.embedding_grad(dy, ids, rows, base, scale))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (1, 32000, 512), (64, 1, 8), (65, 1, 33), (300, 5003, 200), (4096, 128, 40), (4097, 129, 17), (20000, 3, 24),
                                               (10000, 40000, 64), (999, 300, 2056), (130, 2, 9000)])
def test_embedding_grad(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    g, t = gen(tokens + cols), TYPES[dtype]
    dy, ids = normal(g, tokens, cols, dtype=t), tokens_of(g, tokens, vocab)
    check_grad(ctx, dy, ids, vocab, scale=-0.5)
    if tokens > 2:  # rows of tokens that are padding do not count, whatever they hold
        ids[0] = ids[-1] = -1
        dy[0], dy[-1] = math.nan, math.inf
        check_grad(ctx, dy, ids, vocab)
    check_grad(ctx, dy, ids, vocab, normal(g, vocab, cols, dtype=t), 2.0)
    check_grad(ctx, dy, ids, vocab, normal(g, vocab, cols))


@pytest.mark.parametrize("lengths", [[64, 65, 63], [128, 1, 64, 64, 200], [63, 66, 1, 130], [1000, 1000], [3, 64, 61, 64, 65, 64 * 40 + 7, 5]])
def test_embedding_grad_rows_end_anywhere_in_a_window(ctx, lengths):  # noqa: F811
    """Rows of as many tokens as given; with 128 classes and rows 128 apart they follow one another in the sorted order."""
    g = gen(sum(lengths))
    ids = torch.cat([torch.full((n,), 128 * i, dtype=torch.int32) for i, n in enumerate(lengths)]).cuda()
    ids = ids[torch.randperm(ids.numel(), generator=g, device="cuda")]
    check_grad(ctx, normal(g, ids.numel(), 72), ids, 128 * len(lengths))


def test_embedding_grad_of_one_token_everywhere_and_of_none(ctx):  # noqa: F811
    g = gen(1)
    dy = normal(g, 30000, 40)
    check_grad(ctx, dy, torch.full((30000,), 77, dtype=torch.int32, device="cuda"), 100)
    check_grad(ctx, dy, torch.full((30000,), -1, dtype=torch.int32, device="cuda"), 100)
    check_grad(ctx, dy, torch.full((30000,), -1, dtype=torch.int32, device="cuda"), 100, normal(g, 100, 40))


def test_embedding_grad_of_a_table_of_millions_of_rows(ctx):  # noqa: F811
    g = gen(2)
    rows = 128 * 16384 + 5  # more classes of rows than the fewest
    ids = torch.randint(0, rows, (3000,), generator=g, device="cuda", dtype=torch.int32)
    ids[:100] = rows - 1
    check_grad(ctx, normal(g, 3000, 4), ids, rows)


def test_embedding_grad_is_the_same_every_time(ctx):  # noqa: F811
    g = gen(4)
    dy, ids = normal(g, 20000, 64), tokens_of(g, 20000, 500)
    a, b = (fetch(ctx, ctx.embedding_grad(ctx.from_torch(dy), ctx.from_torch(ids), 500)) for _ in range(2))
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_embedding_grad_added_in_place(ctx, dtype):  # noqa: F811
    g, t = gen(6), TYPES[dtype]
    dy, ids, base = normal(g, 500, 48, dtype=t), tokens_of(g, 500, 1000), normal(g, 1000, 48, dtype=t)
    named = torch.zeros(1000, dtype=torch.bool, device="cuda")
    named[ids.long()] = True
    base[~named] = math.nan  # (rows that no token names are left as they are)
    base.view(torch.int16 if dtype == "bf16" else torch.int32)[~named] += 1
    before = base.clone()
    want, bound = ref.embedding_grad(dy, ids, 1000, base)
    lb = ctx.from_torch(base)
    ctx.assign(lb, ctx.embedding_grad(ctx.from_torch(dy), ctx.from_torch(ids), 1000, base=lb))
    ctx.barrier(blocking=True)
    assert ctx.device_ptr(lb) == base.data_ptr()
    n = named.cpu()
    close(base.cpu()[n], want[n], bound[n])
    i = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(base.view(i)[~named], before.view(i)[~named])


def test_embedding_grad_of_a_slice_and_unaligned(ctx):  # noqa: F811
    g = gen(8)
    wide, ids = normal(g, 400, 96, dtype=torch.bfloat16), tokens_of(g, 400, 30)
    for start, length in ((32, 32), (5, 31)):
        y = ctx.embedding_grad(ctx.op("narrow", ctx.from_torch(wide), dim=1, start=start, length=length), ctx.from_torch(ids), 30)
        close(fetch(ctx, y), *ref.embedding_grad(wide[:, start: start + length], ids, 30))
    base = normal(g, 30, 96, dtype=torch.bfloat16)
    y = ctx.embedding_grad(unaligned(ctx, wide, "bf16"), unaligned(ctx, ids, "i32"), 30, base=unaligned(ctx, base, "bf16"))
    close(fetch(ctx, y), *ref.embedding_grad(wide, ids, 30, base))


def test_embedding_gradient_against_differences(ctx):  # noqa: F811
    """<dy, embedding(table)> is linear in the table: its difference along a direction is the gradient's product with it."""
    g = gen(9)
    table, along, dy, ids = normal(g, 20, 24), normal(g, 20, 24), normal(g, 200, 24), tokens_of(g, 200, 20)
    grad = fetch(ctx, ctx.embedding_grad(ctx.from_torch(dy), ctx.from_torch(ids), 20, scale=0.5)).double()
    up, down = (fetch(ctx, ctx.embedding(ctx.from_torch(table + s * along), ctx.from_torch(ids), scale=0.5)).double() for s in (1.0, -1.0))
    diff = float((dy.double().cpu() * (up - down)).sum()) / 2
    size = float((dy.double().cpu().abs() * (up.abs() + down.abs())).sum())
    assert abs(diff - float((grad * along.double().cpu()).sum())) < 300 * ULP * size


@pytest.mark.parametrize("op", ["embedding", "embedding_grad", "loss", "loss_grad"])
def test_tokens_outside_the_table_are_left_out_and_reported(ctx, lt, op):  # noqa: F811
    g = gen(10)
    table, x = normal(g, 30, 16), normal(g, 40, 16)
    ids = tokens_of(g, 40, 30)
    ids[3], ids[7], ids[9] = 30, (1 << 31) - 1, -5
    lt_ids = ctx.from_torch(ids)
    lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
    if op == "embedding":
        got, want = [ctx.embedding(ctx.from_torch(table), lt_ids)], [ref.embedding(table, ids)]
    elif op == "embedding_grad":
        got, want = [ctx.embedding_grad(ctx.from_torch(x), lt_ids, 30)], [ref.embedding_grad(x, ids, 30)]
    elif op == "loss":
        got, r = ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), lt_ids), ref.loss(x, table, ids)
        want = [r[:2], r[2:]]
    else:
        d = normal(g, 40)
        got, r = ctx.vocabulary_loss_grad(ctx.from_torch(x), ctx.from_torch(table), lt_ids, ctx.from_torch(lse), ctx.from_torch(d)), ref.loss_grad(x, table, ids, lse, d)
        want = [r[:2], r[2:]]
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*" + {"loss": "vocabulary_loss", "loss_grad": "vocabulary_loss"}.get(op, op)):
        ctx.barrier(blocking=True)
    ctx.barrier(blocking=True)  # (said once)
    for a, b in zip(got, want):
        close(fetch(ctx, a), *b)


# ------------------------------------------------------------------------------------------------ cross entropy
def check_loss(ctx, x, table, ids, scale=1.0, dloss=None):  # noqa: F811
    lx, lw, li = ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)
    loss, lse = ctx.vocabulary_loss(lx, lw, li, scale=scale)
    a, b, c, d = ref.loss(x, table, ids, scale)
    dloss = torch.ones(ids.shape, device="cuda") if dloss is None else dloss
    dx, dw = ctx.vocabulary_loss_grad(lx, lw, li, lse, ctx.from_torch(dloss), scale=scale)
    got = [fetch(ctx, t).flatten() for t in (loss, lse)]
    close(got[0], a, b, "loss")
    close(got[1], c, d, "lse")
    da, db, dc, dd = ref.loss_grad(x, table, ids, got[1], dloss, scale)
    close(fetch(ctx, dx).reshape(da.shape), da, db, "dx")
    close(fetch(ctx, dw), dc, dd, "dtable")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,cols", [(1, 1, 1), (1, 2, 8), (1, 5003, 64), (3, 257, 72), (64, 256, 64), (127, 255, 128), (129, 513, 192), (256, 1000, 33), (257, 300, 100),
                                               (300, 1024, 520), (513, 257, 256), (40, 20011, 24), (1000, 40, 1024), (2, 130, 4100), (700, 700, 700)])
def test_vocabulary_loss(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    g, t = gen(tokens + vocab + cols), TYPES[dtype]
    x, table, ids = normal(g, tokens, cols, dtype=t, std=2.0), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab)
    ids[-1] = vocab - 1
    check_loss(ctx, x, table, ids, dloss=normal(g, tokens))
    if tokens > 3:
        ids[0], ids[tokens // 2], ids[-2] = -1, -7, -(1 << 31)
        check_loss(ctx, x, table, ids, scale=-1.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocabulary_loss_of_more_tokens_and_rows_than_the_blocks_have_at_once(ctx, dtype):  # noqa: F811
    g, t = gen(12), TYPES[dtype]
    x, table, ids = normal(g, 3001, 136, dtype=t), normal(g, 9001, 136, dtype=t, std=0.1), tokens_of(g, 3001, 9001)
    ids[::7] = -1
    check_loss(ctx, x, table, ids, dloss=normal(g, 3001))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_vocabulary_loss_far_scores(ctx, dtype):  # noqa: F811
    """Scores of hundreds, of one sign, and rows whose target has all or none of the weight."""
    g, t = gen(13), TYPES[dtype]
    x, table = normal(g, 50, 64, dtype=t, std=20.0), normal(g, 700, 64, dtype=t)
    x[3] = 0.0
    ids = tokens_of(g, 50, 700)
    z = x.double() @ table.double().T
    ids[:20] = z[:20].argmax(-1).int()
    ids[20:30] = z[20:30].argmin(-1).int()
    check_loss(ctx, x, table, ids)
    table[:, 0] = 8.0
    x[:, 0] = -40.0
    check_loss(ctx, x, table, ids)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_without_a_target_do_not_count_whatever_they_hold(ctx, dtype):  # noqa: F811
    g, t = gen(14), TYPES[dtype]
    x, table, ids, d = normal(g, 300, 64, dtype=t), normal(g, 400, 64, dtype=t), tokens_of(g, 300, 400), normal(g, 300)
    ids[5], ids[200] = -1, -100
    lw, li, ld = ctx.from_torch(table), ctx.from_torch(ids), ctx.from_torch(d)
    lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
    clean = [fetch(ctx, r) for r in ctx.vocabulary_loss_grad(ctx.from_torch(x), lw, li, ctx.from_torch(lse), ld)]
    x2, lse2 = x.clone(), lse.clone()
    x2[5], x2[200] = math.nan, math.inf
    lse2[5], lse2[200], d[5], d[200] = math.nan, -math.inf, math.inf, math.nan
    dirty = [fetch(ctx, r) for r in ctx.vocabulary_loss_grad(ctx.from_torch(x2), lw, li, ctx.from_torch(lse2), ld)]
    assert all(torch.equal(a, b) for a, b in zip(clean, dirty))
    assert not bool(clean[0][5].any()) and not bool(clean[0][200].any())
    loss, lse3 = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x2), lw, li))
    assert float(loss[5]) == 0.0 and float(loss[200]) == 0.0 and bool(torch.isnan(lse3[5]))
    others = torch.ones(300, dtype=torch.bool)
    others[5] = others[200] = False
    a, b, c, e = ref.loss(torch.where(others.cuda()[:, None], x, 0.0), table, ids)
    close(loss, a, b)
    close(lse3[others], c[others], e[others])


def test_no_target_at_all(ctx):  # noqa: F811
    g = gen(15)
    x, table = normal(g, 70, 40), normal(g, 300, 40)
    check_loss(ctx, x, table, torch.full((70,), -1, dtype=torch.int32, device="cuda"))


def test_infinite_scores(ctx):  # noqa: F811
    """Rows of the table that rule a word out, and hidden states that are not finite, stay in their own rows."""
    g = gen(16)
    x, table = normal(g, 20, 8).abs() + 0.5, normal(g, 300, 8)
    table[7] = -math.inf
    table[299] = -math.inf
    ids = torch.arange(20, device="cuda", dtype=torch.int32) + 10
    loss, lse = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)))
    keep = torch.ones(300, dtype=torch.bool)
    keep[7] = keep[299] = False
    a, b, c, d = ref.loss(x, table[keep.cuda()], torch.where(ids > 7, ids - 1, ids))
    close(loss, a, b)
    close(lse, c, d)
    table[7], x[4], x[5, 0] = 0.0, math.nan, math.inf
    table[:, 0] = table[:, 0].abs() + 0.5
    loss, lse = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)))
    assert bool(torch.isnan(lse).all())  # (the last row of the table now has infinities of both signs)
    table[299] = 0.0
    loss, lse = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)))
    assert bool(torch.isnan(lse[4])) and bool(torch.isnan(lse[5]))  # (infinity times the zero there is no number)
    others = torch.ones(20, dtype=torch.bool, device="cuda")
    others[4] = others[5] = False
    a, b, c, d = ref.loss(x[others], table, ids[others])
    close(loss[others.cpu()], a, b)
    close(lse[others.cpu()], c, d)


def test_vocabulary_loss_of_slices_and_unaligned(ctx):  # noqa: F811
    g = gen(17)
    for dtype in ("bf16", "f32"):
        t = TYPES[dtype]
        wx, wt, ids, d = normal(g, 90, 200, dtype=t), normal(g, 333, 200, dtype=t, std=0.2), tokens_of(g, 90, 333), torch.ones(90, device="cuda")
        for start, length in ((64, 64), (8, 72), (3, 61)):
            lx = ctx.op("narrow", ctx.from_torch(wx), dim=1, start=start, length=length)
            lw = ctx.op("narrow", ctx.from_torch(wt), dim=1, start=start, length=length)
            x, w = wx[:, start: start + length], wt[:, start: start + length]
            loss, lse = ctx.vocabulary_loss(lx, lw, ctx.from_torch(ids))
            dx, dw = ctx.vocabulary_loss_grad(lx, lw, ctx.from_torch(ids), lse, ctx.from_torch(d))
            del lx, lw
            a, b, c, e = ref.loss(x, w, ids)
            got = fetch(ctx, lse)
            close(got, c, e)
            close(fetch(ctx, loss), a, b)
            a, b, c, e = ref.loss_grad(x, w, ids, got, d)
            close(fetch(ctx, dx), a, b)
            close(fetch(ctx, dw), c, e)
        loss, lse = ctx.vocabulary_loss(unaligned(ctx, wx, dtype), unaligned(ctx, wt, dtype), unaligned(ctx, ids, "i32"))
        a, b, c, e = ref.loss(wx, wt, ids)
        close(fetch(ctx, loss), a, b)
        out = [unaligned(ctx, wx, dtype), unaligned(ctx, wt, dtype, 3)]
        lse2 = torch.logsumexp(wx.double() @ wt.double().T, -1).float()
        ctx.vocabulary_loss_grad(unaligned(ctx, wx, dtype), unaligned(ctx, wt, dtype), ctx.from_torch(ids), ctx.from_torch(lse2), ctx.from_torch(d), out=out)
        a, b, c, e = ref.loss_grad(wx, wt, ids, lse2, d)
        close(fetch(ctx, out[0]), a, b)
        close(fetch(ctx, out[1]), c, e)


@pytest.mark.parametrize("which", [0, 1])
def test_one_gradient_alone(ctx, which):  # noqa: F811
    g = gen(18)
    x, table, ids, d = normal(g, 300, 96, dtype=torch.bfloat16), normal(g, 2000, 96, dtype=torch.bfloat16, std=0.1), tokens_of(g, 300, 2000), normal(g, 300)
    lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
    args = [ctx.from_torch(t) for t in (x, table, ids, lse, d)]
    got = fetch(ctx, ctx.op("vocabulary_loss_grad", *args, result=which, scale=1.0))
    r = ref.loss_grad(x, table, ids, lse, d)
    close(got, *r[2 * which: 2 * which + 2])
    loss = fetch(ctx, ctx.op("vocabulary_loss", *args[:3], result=which, scale=1.0))
    r = ref.loss(x, table, ids)
    close(loss, *r[2 * which: 2 * which + 2])


def test_vocabulary_loss_is_the_same_every_time(ctx):  # noqa: F811
    g = gen(19)
    x, table, ids = normal(g, 5, 4096, dtype=torch.bfloat16), normal(g, 3001, 4096, dtype=torch.bfloat16, std=0.02), tokens_of(g, 5, 3001)
    lx, lw, li, one = ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids), ctx.from_torch(torch.ones(5, device="cuda"))
    runs = []
    for _ in range(2):
        loss, lse = ctx.vocabulary_loss(lx, lw, li)
        runs.append([fetch(ctx, r) for r in (loss, lse, *ctx.vocabulary_loss_grad(lx, lw, li, lse, one))])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_vocabulary_loss_gradient_against_differences(ctx):  # noqa: F811
    """The loss in 64 bits, a small step up and down along a direction, against the gradients' products with it."""
    g = gen(20)
    x, table, ids, d = normal(g, 60, 32), normal(g, 90, 32), tokens_of(g, 60, 90), normal(g, 60)
    ids[11] = -1
    lx, lw, li = ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)
    loss, lse = ctx.vocabulary_loss(lx, lw, li, scale=0.5)
    dx, dw = (fetch(ctx, r).double() for r in ctx.vocabulary_loss_grad(lx, lw, li, lse, ctx.from_torch(d), scale=0.5))
    ax, aw, h = normal(g, 60, 32).double().cpu(), normal(g, 90, 32).double().cpu(), 1e-5
    up, down = (float((d.double().cpu() * ref.loss(x.double().cpu() + s * h * ax, table.double().cpu() + s * h * aw, ids, 0.5)[0]).sum()) for s in (1, -1))
    want = float((dx * ax).sum() + (dw * aw).sum())
    # third derivatives of a loss are at most a score's to the third: h^2 (12)^3 per token; the products: about 1e3 ULP each
    size = float((dx.abs() * ax.abs()).sum() + (dw.abs() * aw.abs()).sum())
    assert abs((up - down) / (2 * h) - want) < 60 * h * h * 40 ** 3 + 1000 * ULP * size


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 8, 9, 15, 16, 17, 33, 64, 65, 128])
@pytest.mark.parametrize("vocab,cols", [(3, 64), (1003, 264), (5003, 72), (777, 33)])
def test_vocabulary_loss_of_few_tokens(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    g, t = gen(tokens + vocab), TYPES[dtype]
    x, table, ids = normal(g, tokens, cols, dtype=t, std=2.0), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab)
    ids[-1] = vocab - 1
    if tokens > 2:
        ids[1] = -3
    check_loss(ctx, x, table, ids, scale=1.5, dloss=normal(g, tokens))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens,vocab,cols", [(5, 3, 2504), (129, 90, 2504), (200, 300, 6200), (260, 255, 6145), (17, 1500, 2100), (1000, 600, 2051)])
def test_vocabulary_loss_of_few_scores(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    """Long rows and few tiles: several workers have one, for a part of the columns each."""
    g, t = gen(tokens + vocab), TYPES[dtype]
    x, table, ids = normal(g, tokens, cols, dtype=t, std=2.0), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab)
    ids[1::3] = -1
    check_loss(ctx, x, table, ids, scale=0.75, dloss=normal(g, tokens))
    check_loss(ctx, x, table, ids)


def test_few_infinite_scores(ctx):  # noqa: F811
    """As in test_infinite_scores, for each way in which few and many tokens are scored."""
    g = gen(24)
    for tokens, cols in ((1, 24), (4, 24), (7, 24), (16, 24), (70, 24), (200, 24), (200, 500), (200, 1030)):
        x, table = normal(g, tokens, cols).abs() + 0.5, normal(g, 900, cols) * cols ** -0.5
        table[[0, 255, 256, 700, 899]] = -math.inf
        ids = torch.full((tokens,), 300, dtype=torch.int32, device="cuda")
        keep = torch.isfinite(table[:, 0])
        loss, lse = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)))
        a, b, c, d = ref.loss(x, table[keep], ids - 3)
        close(loss, a, b)
        close(lse, c, d)
        table[300] = math.inf  # the target itself: everything else vanishes beside it
        loss, lse = (fetch(ctx, r) for r in ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids)))
        assert bool((lse == math.inf).all()) and bool(torch.isnan(loss).all())
        x[-1, 3] = math.nan
        lse = fetch(ctx, ctx.vocabulary_loss(ctx.from_torch(x), ctx.from_torch(table), ctx.from_torch(ids))[1])
        assert bool(torch.isnan(lse[-1])) and bool((lse[:-1] == math.inf).all())


@pytest.mark.parametrize("dtype,tokens,vocab,cols,where", [("f32", 70, 3, 8210, None), ("f32", 300, 20011, 1000, None), ("bf16", 300, 5001, 1000, "table"), ("bf16", 4500, 300, 1000, "x"),
                                                           ("bf16", 5, 40, 8210, "table")])
def test_vocabulary_loss_in_pieces(ctx, dtype, tokens, vocab, cols, where):  # noqa: F811
    """More than one piece of a packed table, of packed tokens, and long rows; bf16 rows are packed where they begin at odd places."""
    g, t = gen(tokens), TYPES[dtype]
    x, table, ids, d = normal(g, tokens, cols, dtype=t), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab), normal(g, tokens)
    ids[::5] = -1
    lx, lw = (unaligned(ctx, v, dtype) if where == n else ctx.from_torch(v) for n, v in (("x", x), ("table", table)))
    loss, lse = ctx.vocabulary_loss(lx, lw, ctx.from_torch(ids))
    dx, dw = ctx.vocabulary_loss_grad(lx, lw, ctx.from_torch(ids), lse, ctx.from_torch(d))
    a, b, c, e = ref.loss(x, table, ids)
    got = fetch(ctx, lse)
    close(got, c, e)
    close(fetch(ctx, loss), a, b)
    a, b, c, e = ref.loss_grad(x, table, ids, got, d)
    close(fetch(ctx, dx), a, b)
    close(fetch(ctx, dw), c, e)


@pytest.fixture()
def on_the_gpu(monkeypatch):
    monkeypatch.setattr(ref, "WHERE", ["cuda"])


def test_vocabulary_loss_of_so_many_scores_that_p_is_made_in_pieces(ctx, on_the_gpu):  # noqa: F811
    g, t = gen(25), torch.bfloat16
    x, table, ids, d = normal(g, 9001, 72, dtype=t), normal(g, 20001, 72, dtype=t, std=0.1), tokens_of(g, 9001, 20001), normal(g, 9001)
    ids[::5] = -1
    check_loss(ctx, x, table, ids, dloss=d)


@pytest.mark.parametrize("tokens,vocab,cols,tied", [(20000, 3000, 1032, True), (20000, 300, 2056, False), (40001, 5000, 2048, True), (70001, 40, 1024, False)])
def test_embedding_grad_of_large_windows(ctx, on_the_gpu, tokens, vocab, cols, tied):  # noqa: F811
    """So many tokens that windows of 16, 32 and 64 of them are summed, and that they are sorted in several steps."""
    g, t = gen(tokens), torch.bfloat16
    dy, ids = normal(g, tokens, cols, dtype=t), tokens_of(g, tokens, vocab)
    ids[:: 7] = -1
    check_grad(ctx, dy, ids, vocab, normal(g, vocab, cols, dtype=t) if tied else None)


@pytest.mark.parametrize("tokens", [33000, 100000])
def test_embedding_grad_where_one_token_is_most_of_them(ctx, on_the_gpu, tokens):  # noqa: F811
    g = gen(tokens)
    dy, ids = normal(g, tokens, 40), tokens_of(g, tokens, 1000)
    ids[torch.rand(tokens, generator=g, device="cuda") < 0.6] = 128 * 3 + 5
    ids[torch.rand(tokens, generator=g, device="cuda") < 0.1] = 128 * 4 + 5  # (of the same class)
    check_grad(ctx, dy, ids, 1000)


# ------------------------------------------------------------------------------------------------ together, on streams, captured
def step(c, t, out):
    """Both ends of a model on one table: lookup, (a norm stands for the model), loss, gradients, all into the table's."""
    e = c.embedding(t["table"], t["ids"], scale=t["scale"])
    (x,) = c.rms_norm(e, t["gamma"])
    _, lse = c.vocabulary_loss(x, t["table"], t["targets"], out=[out[0], None])
    dx, dw = c.vocabulary_loss_grad(x, t["table"], t["targets"], lse, t["dloss"])
    de, _ = c.rms_norm_grad(dx, e, t["gamma"], out=[None, out[2]])
    c.embedding_grad(de, t["ids"], t["rows"], base=dw, scale=t["scale"], out=out[1])


def make_step(seed, tokens=200, vocab=700, cols=64):
    g = gen(seed)
    s = dict(table=normal(g, vocab, cols, std=0.2), ids=tokens_of(g, tokens, vocab), targets=tokens_of(g, tokens, vocab), dloss=torch.full((tokens,), 1.0 / tokens, device="cuda"),
             gamma=1 + normal(g, cols, std=0.1))
    s["targets"][::9] = -1
    return s, [torch.zeros(tokens, device="cuda"), torch.zeros(vocab, cols, device="cuda"), torch.zeros(cols, device="cuda")]


def step64(s):
    table, gamma = s["table"].double().cpu().requires_grad_(), s["gamma"].double().cpu().requires_grad_()
    e = 2.0 * torch.nn.functional.embedding(s["ids"].long().cpu(), table)
    x = gamma * e / torch.sqrt((e * e).mean(-1, keepdim=True) + 1e-6)
    loss = torch.nn.functional.cross_entropy(x @ table.T, torch.where(s["targets"] < 0, -100, s["targets"]).long().cpu(), reduction="none")
    return [loss.detach(), *torch.autograd.grad(loss, (table, gamma), s["dloss"].double().cpu())]


def check_step(s, out):
    for got, want in zip(out, step64(s)):
        # (hundreds of roundings of 2^-24 of sums whose terms are some tens of the result's root mean square)
        assert float((got.double().cpu() - want).abs().max()) < 4000 * ULP * max(1.0, float(want.abs().max()) * 20)


def handles(c, s, out):
    t = {k: c.from_torch(v) for k, v in s.items()}
    t["rows"], t["scale"] = s["table"].shape[0], 2.0
    return t, [c.from_torch(o) for o in out]


def test_a_training_step_on_one_table(ctx):  # noqa: F811
    s, out = make_step(21)
    t, lo = handles(ctx, s, out)
    for _ in range(3):  # (planned, then matched)
        for o in out:
            o.zero_()
        step(ctx, t, lo)
        ctx.barrier(blocking=True)
        check_step(s, out)
        assert [ctx.device_ptr(o) for o in lo] == [o.data_ptr() for o in out]
    out[1].fill_(math.nan)
    ctx.replay(blocking=True)
    check_step(s, out)


@pytest.mark.parametrize("static", [False, True])
def test_captured_on_a_stream_and_replayed_on_new_values(lt, static):  # noqa: F811
    stream = torch.cuda.Stream()
    s, out = make_step(22)
    other, _ = make_step(23)
    with torch.cuda.stream(stream):
        c = lt.LazyContext(device=0, stream=stream.cuda_stream)
        x, lse = normal(gen(1), 200, 64), torch.zeros(200, device="cuda")
        dx, dw = torch.zeros_like(x), torch.zeros_like(s["table"])
        lx, lw, li, ld, lo, ll = (c.from_torch(v) for v in (x, s["table"], s["targets"], s["dloss"], out[0], lse))
        ldx, ldw, lg = c.from_torch(dx), c.from_torch(dw), c.from_torch(out[1])

        def record():
            _, e = c.vocabulary_loss(lx, lw, li, out=[lo, ll])
            c.vocabulary_loss_grad(lx, lw, li, e, ld, out=[ldx, ldw])
            c.embedding_grad(lx, li, 700, out=lg)

        flush = c.barrier_static_scratch if static else c.barrier
        record()
        flush(blocking=True)
        graph = torch.cuda.CUDAGraph()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            record()
            flush()
        for k in range(2):
            s["table"].copy_(other["table"])
            s["targets"].copy_(other["targets"])
            s["dloss"].copy_(other["dloss"] * (k + 1))
            for o in (out[0], lse, dx, dw, out[1]):
                o.fill_(math.nan)
            graph.replay()
            stream.synchronize()
            r = ref.loss(x, s["table"], s["targets"])
            close(out[0], *r[:2])
            close(lse, *r[2:])
            r = ref.loss_grad(x, s["table"], s["targets"], lse, s["dloss"])
            close(dx, *r[:2])
            close(dw, *r[2:])
            close(out[1], *ref.embedding_grad(x, s["targets"], 700))
        c.barrier(blocking=True)
        del graph
        c.close()


def test_two_contexts_on_two_streams_at_once(lt):  # noqa: F811
    made = []
    for k in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            s, out = make_step(30 + k, tokens=500, vocab=3000, cols=128)
            c = lt.LazyContext(device=0, stream=stream.cuda_stream)
            made.append((stream, s, out, c, handles(c, s, out)))
    torch.cuda.synchronize()
    for _ in range(4):
        for stream, s, out, c, (t, lo) in made:
            step(c, t, lo)
            c.barrier()
    for stream, s, out, c, (t, lo) in made:
        c.barrier(blocking=True)
        check_step(s, out)
        c.close()


@pytest.mark.parametrize("dtype,tokens,vocab,cols", [("bf16", 1, 700, 4096), ("bf16", 2, 3, 8), ("bf16", 2, 1201, 333), ("bf16", 1, 2000, 4104), ("f32", 1, 1, 1), ("f32", 2, 901, 2048), ("f32", 3, 1500, 4096),
                                                     ("f32", 4, 5, 36), ("f32", 7, 2001, 260), ("f32", 9, 800, 516), ("f32", 13, 1003, 77), ("f32", 16, 3001, 1024), ("f32", 16, 300, 4100), ("f32", 17, 900, 512)])
def test_gradients_of_few_tokens(ctx, dtype, tokens, vocab, cols):  # noqa: F811
    g, t = gen(tokens + vocab + cols), TYPES[dtype]
    x, table, ids = normal(g, tokens, cols, dtype=t, std=2.0), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab)
    ids[-1] = vocab - 1
    check_loss(ctx, x, table, ids, dloss=normal(g, tokens))
    odd = torch.empty(table.numel() + 1, device="cuda", dtype=t)[1:].view(vocab, cols)  # (begins behind a 16-byte boundary)
    odd.copy_(table)
    check_loss(ctx, x, odd, ids, scale=-0.75)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients_of_few_tokens_report_a_target_outside_the_table(ctx, lt, dtype):  # noqa: F811
    g, t = gen(3), TYPES[dtype]
    x, table, ids = normal(g, 2, 64, dtype=t), normal(g, 30, 64, dtype=t), torch.tensor([30, 29], dtype=torch.int32, device="cuda")
    lse, d = torch.logsumexp(x.double() @ table.double().T, -1).float(), normal(g, 2)
    got, r = ctx.vocabulary_loss_grad(*(ctx.from_torch(v) for v in (x, table, ids, lse, d))), ref.loss_grad(x, table, ids, lse, d)
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*vocabulary_loss"):
        ctx.barrier(blocking=True)
    for a, b in zip(got, (r[:2], r[2:])):
        close(fetch(ctx, a), *b)


@pytest.mark.parametrize("dtype,tokens", [("bf16", 2), ("f32", 2), ("f32", 16)])
def test_gradients_of_few_tokens_that_do_not_count_and_one_alone(ctx, dtype, tokens):  # noqa: F811
    """Rows without a target hold NaN; each gradient is the same when it is asked for alone."""
    g, t = gen(tokens), TYPES[dtype]
    x, table, targets, dloss = normal(g, tokens, 260, dtype=t), normal(g, 501, 260, dtype=t), tokens_of(g, tokens, 501), normal(g, tokens)
    targets[0] = -1
    tt = [ctx.from_torch(v) for v in (x, table, targets, dloss)]
    lse = ctx.vocabulary_loss(*tt[:3])[1]
    ctx.barrier()
    out = [torch.full_like(x, 7.0), torch.full_like(table, 7.0)]
    buffers = [ctx.from_torch(o) for o in out]
    ctx.vocabulary_loss_grad(*tt[:3], lse, tt[3], out=buffers)
    ctx.barrier()
    torch.cuda.synchronize()
    x2, dloss2 = x.clone(), dloss.clone()
    x2[0], dloss2[0] = math.nan, math.nan
    hurt = ctx.from_torch(x2), ctx.from_torch(dloss2)
    for which in (0, 1):
        alone = torch.full_like(out[which], 7.0)
        buffers = [None, None]
        buffers[which] = ctx.from_torch(alone)
        results = ctx.vocabulary_loss_grad(hurt[0], *tt[1:3], lse, hurt[1], out=buffers)
        ctx.release(results[1 - which])
        ctx.barrier()
        torch.cuda.synchronize()
        assert torch.equal(alone, out[which])
    assert bool((out[0][0] == 0).all()) and bool(torch.isfinite(out[1].float()).all())
