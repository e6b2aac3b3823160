"""Lookup in a table, cross entropy against it, and their gradients on a record-and-plan-only context: shapes, refusals, which
launches a graph becomes and what is written in place.  No GPU."""
import math

import pytest

import paper_2102_13267_b200 as lt
from test_operators_host import ctx, fake, plan, refused  # noqa: F401

LOOK = dict(scale=1.0)
GRAD = dict(rows=50, base=False, scale=1.0)
LOSS = dict(result=0, scale=1.0)


def test_result_shapes(ctx):  # noqa: F811
    f = lambda *a: fake(ctx, *a)  # noqa: E731
    table = f((50, 16), "bf16")
    y = ctx.embedding(table, f((3, 7), "i32"))
    assert (y.shape, y.dtype) == ((3, 7, 16), "bf16")
    g = ctx.embedding_grad(f((3, 7, 16), "bf16"), f((3, 7), "i32"), 50)
    assert (g.shape, g.dtype) == ((50, 16), "bf16")
    assert ctx.embedding_grad(f((3, 7, 16), "bf16"), f((3, 7), "i32"), 50, base=f((50, 16))).dtype == "f32"
    loss, lse = ctx.vocabulary_loss(f((3, 7, 16), "bf16"), table, f((3, 7), "i32"))
    assert (loss.shape, loss.dtype, lse.shape, lse.dtype) == ((3, 7), "f32", (3, 7), "f32")
    dx, dw = ctx.vocabulary_loss_grad(f((3, 7, 16), "bf16"), table, f((3, 7), "i32"), lse, f((3, 7)))
    assert (dx.shape, dx.dtype, dw.shape, dw.dtype) == ((3, 7, 16), "bf16", (50, 16), "bf16")
    text = ctx.dump_ir()
    for name in ("embedding", "embedding_grad", "vocabulary_loss", "vocabulary_loss_grad"):
        assert f"lt::{name}(" in text


TAB, IDS, DY = ((50, 16), "bf16"), ((5,), "i32"), ((5, 16), "bf16")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [TAB], LOOK), ("INVALID_ARG", [TAB, IDS, DY, DY], LOOK), ("DTYPE", [((50, 16), "i32"), IDS], LOOK), ("SHAPE", [((50,), "f32"), IDS], LOOK),
    ("DTYPE", [TAB, ((5,), "f32")], LOOK), ("DTYPE", [TAB, ((5,), "u32")], LOOK), ("SHAPE", [TAB, IDS, ((5, 15), "bf16")], LOOK), ("SHAPE", [TAB, IDS, ((5, 16), "f32")], LOOK),
    ("SHAPE", [TAB, ((1, 1, 1, 1, 1, 5), "i32")], LOOK), ("INVALID_ARG", [TAB, IDS], dict(scale=math.inf)), ("INVALID_ARG", [TAB, IDS], dict(scale=1e39)),
    ("UNSUPPORTED", [((1 << 31, 16), "bf16"), IDS], LOOK)])
def test_embedding_refusals(ctx, status, shapes, attrs):  # noqa: F811
    refused(ctx, status, "embedding", shapes, **attrs)


BASE = dict(GRAD, base=True)


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [DY], GRAD), ("INVALID_ARG", [DY, IDS], BASE), ("INVALID_ARG", [DY, IDS, TAB, TAB], GRAD), ("DTYPE", [((5, 16), "i32"), IDS], GRAD),
    ("DTYPE", [DY, ((5,), "u32")], GRAD), ("SHAPE", [DY, ((4,), "i32")], GRAD), ("SHAPE", [((5,), "bf16"), IDS], GRAD), ("SHAPE", [DY, ((5, 1), "i32")], GRAD),
    ("INVALID_ARG", [DY, IDS], dict(GRAD, rows=0)), ("INVALID_ARG", [DY, IDS], dict(GRAD, rows=-1)), ("UNSUPPORTED", [DY, IDS], dict(GRAD, rows=1 << 31)),
    ("SHAPE", [DY, IDS, ((49, 16), "bf16")], BASE), ("SHAPE", [DY, IDS, ((50, 15), "bf16")], BASE), ("DTYPE", [DY, IDS, ((50, 16), "i32")], BASE),
    ("DTYPE", [((5, 16), "f32"), IDS, TAB], BASE), ("SHAPE", [DY, IDS, ((50, 16), "f32")], GRAD), ("INVALID_ARG", [DY, IDS], dict(GRAD, scale=math.nan))])
def test_embedding_grad_refusals(ctx, status, shapes, attrs):  # noqa: F811
    refused(ctx, status, "embedding_grad", shapes, **attrs)


VEC = ((5,), "f32")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [DY, TAB], LOSS), ("INVALID_ARG", [DY, TAB, IDS, VEC, VEC], LOSS), ("DTYPE", [((5, 16), "f32"), TAB, IDS], LOSS), ("DTYPE", [DY, ((50, 16), "i32"), IDS], LOSS),
    ("SHAPE", [((5, 15), "bf16"), TAB, IDS], LOSS), ("SHAPE", [DY, TAB, ((4,), "i32")], LOSS), ("DTYPE", [DY, TAB, VEC], LOSS), ("SHAPE", [((16,), "bf16"), TAB, IDS], LOSS),
    ("SHAPE", [DY, ((2, 25, 16), "bf16"), IDS], LOSS), ("SHAPE", [DY, TAB, IDS, ((6,), "f32")], LOSS), ("INVALID_ARG", [DY, TAB, IDS], dict(LOSS, result=2)),
    ("INVALID_ARG", [DY, TAB, IDS], dict(LOSS, scale=math.nan)), ("UNSUPPORTED", [((5, 1 << 20), "bf16"), ((50, 1 << 20), "bf16"), IDS], LOSS),
    ("UNSUPPORTED", [((1 << 24, 16), "bf16"), TAB, ((1 << 24,), "i32")], LOSS)])
def test_vocabulary_loss_refusals(ctx, status, shapes, attrs):  # noqa: F811
    refused(ctx, status, "vocabulary_loss", shapes, **attrs)


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [DY, TAB, IDS, VEC], LOSS), ("DTYPE", [DY, TAB, IDS, ((5,), "bf16"), VEC], LOSS), ("DTYPE", [DY, TAB, IDS, VEC, ((5,), "i32")], LOSS),
    ("SHAPE", [DY, TAB, IDS, ((4,), "f32"), VEC], LOSS), ("SHAPE", [DY, TAB, IDS, VEC, ((5, 1), "f32")], LOSS), ("SHAPE", [DY, TAB, IDS, VEC, VEC, TAB], LOSS),
    ("SHAPE", [DY, TAB, IDS, VEC, VEC, DY], dict(LOSS, result=1)), ("INVALID_ARG", [DY, TAB, IDS, VEC, VEC], dict(LOSS, result=-1))])
def test_vocabulary_loss_grad_refusals(ctx, status, shapes, attrs):  # noqa: F811
    refused(ctx, status, "vocabulary_loss_grad", shapes, **attrs)


def test_both_results_are_one_launch(ctx):  # noqa: F811
    x, table, ids = fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16"), fake(ctx, (5,), "i32")
    loss, lse = ctx.vocabulary_loss(x, table, ids)
    dx, dw = ctx.vocabulary_loss_grad(x, table, ids, lse, fake(ctx, (5,)))
    text = plan(ctx)
    assert text.count("operator: vocabulary_loss, results=2") == 1 and text.count("operator: vocabulary_loss_grad, results=2") == 1
    other, _ = ctx.vocabulary_loss(x, table, ids, scale=0.5)
    first, _ = ctx.vocabulary_loss(x, table, ids)
    text = plan(ctx)
    assert text.count("operator: vocabulary_loss") == 2
    del loss, dx, dw, other, first


def test_in_place_on_the_base_only(ctx):  # noqa: F811
    dy, ids, base, shape = fake(ctx, (5, 16), "bf16"), fake(ctx, (5,), "i32"), fake(ctx, (50, 16), "bf16"), (50, 16)
    ctx.assign(base, ctx.embedding_grad(dy, ids, 50, base=base))
    ctx.barrier()
    assert ctx.stats()["outputs_donated"] == 1 and base.shape == shape
    # over the table that is looked up: never
    table, every = fake(ctx, (50, 16), "bf16"), fake(ctx, (50,), "i32")
    before = ctx.stats()["outputs_donated"]
    ctx.assign(table, ctx.embedding(table, every))
    ctx.barrier()
    assert ctx.stats()["outputs_donated"] == before
    # nor the gradient over x
    x, t2, lse = fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16"), fake(ctx, (5,))
    dx, _ = ctx.vocabulary_loss_grad(x, t2, ids, lse, lse)
    ctx.assign(x, dx)
    ctx.barrier()
    assert ctx.stats()["outputs_donated"] == before


def test_buffers_meant_for_results(ctx):  # noqa: F811
    x, table, ids, lse = fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16"), fake(ctx, (5,), "i32"), fake(ctx, (5,))
    out = [fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16")]
    ctx.vocabulary_loss_grad(x, table, ids, lse, lse, out=out)
    ctx.vocabulary_loss(x, table, ids, out=[fake(ctx, (5,)), None])
    y = fake(ctx, (5, 16), "bf16")
    ctx.embedding(table, ids, out=y)
    ctx.barrier()
    assert ctx.stats()["outputs_donated"] >= 3
    with pytest.raises(ValueError):
        ctx.vocabulary_loss(x, table, ids, out=[y])


def test_slices_are_read_in_place(ctx):  # noqa: F811
    wide, ids = fake(ctx, (5, 48), "bf16"), fake(ctx, (5,), "i32")
    table = ctx.op("narrow", fake(ctx, (50, 48), "bf16"), dim=1, start=16, length=16)
    x = ctx.op("narrow", wide, dim=1, start=0, length=16)
    loss, lse = ctx.vocabulary_loss(x, table, ids)
    y = ctx.embedding(table, ids)
    g = ctx.embedding_grad(x, ids, 50)
    ctx.release(x)
    ctx.release(table)
    assert "view" not in plan(ctx) and ctx.stats()["launches_view"] == 0
    del loss, lse, y, g


def test_a_batch_records_the_same(ctx):  # noqa: F811
    x, table, ids, d = fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16"), fake(ctx, (5,), "i32"), fake(ctx, (5,))
    out = [fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16")]
    loss, lse = ctx.vocabulary_loss(x, table, ids)
    ctx.vocabulary_loss_grad(x, table, ids, lse, d, out=out)
    ctx.release(lse)
    ctx.barrier()
    compiles = ctx.stats()["compiles"]
    b = lt.Batch()
    bx, bt, bi, bd, b0, b1 = (b.input() for _ in range(6))
    bl, be = b.vocabulary_loss(bx, bt, bi)
    b.keep(bl)
    b.vocabulary_loss_grad(bx, bt, bi, be, bd, out=[b0, b1])
    kept = ctx.record(b, [x, table, ids, d, *out])
    ctx.barrier()
    assert len(kept) == 1 and kept[0].shape == (5,) and ctx.stats()["compiles"] == compiles
    del loss


@pytest.mark.parametrize("scale", [2.4e38, -3e38, 1e39])
def test_a_scale_that_is_infinite_base_two_is_refused(ctx, scale):  # noqa: F811
    refused(ctx, "INVALID_ARG", "vocabulary_loss", [DY, TAB, IDS], result=0, scale=scale)
    refused(ctx, "INVALID_ARG", "vocabulary_loss_grad", [DY, TAB, IDS, VEC, VEC], result=0, scale=scale)
    x, table, ids = fake(ctx, (5, 16), "bf16"), fake(ctx, (50, 16), "bf16"), fake(ctx, (5,), "i32")
    ctx.vocabulary_loss(x, table, ids, scale=2.3e38)


def test_the_products_wait_probe_needs_a_device(ctx):  # noqa: F811
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE"):
        ctx.debug_product_wait_probe(1000)
