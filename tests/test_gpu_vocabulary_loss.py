"""The vocabulary loss and its gradients where sums are long, weights differ widely, rows are wide or a wait gives up."""
import math
import time

import pytest
import torch

import table_reference as ref
from operator_reference import HALF, TYPES, ULP, close
from test_gpu_operators import ctx, fetch, gen, lt, normal, unaligned  # noqa: F401
from test_gpu_table_operators import handles, make_step, step, step64, tokens_of

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------------ waits
def test_the_products_bounded_wait_gives_up_and_is_reported(ctx, lt):  # noqa: F811
    """The wait runs out on a barrier that nobody arrives at, with no copy or product on its way: one warp of the block gives up,
    the other follows, the next blocking call reports it, once, and the context stays usable."""
    x = ctx.from_torch(torch.arange(64, device="cuda", dtype=torch.float32))
    ctx.debug_product_wait_probe(1000)  # (loaded before it is timed)
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_TIMEOUT"):
        ctx.barrier(blocking=True)
    t0 = time.monotonic()
    ctx.debug_product_wait_probe(20_000_000)  # 20 ms; the second warp's limit is a second
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_TIMEOUT"):
        ctx.barrier(blocking=True)
    assert 0.02 <= time.monotonic() - t0 < 0.6
    ctx.barrier(blocking=True)  # said once
    assert torch.equal(fetch(ctx, x + 1.0).cpu(), torch.arange(64) + 1.0)


def test_the_probe_refuses_more_than_a_second(ctx, lt):  # noqa: F811
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_INVALID_ARG"):
        ctx.debug_product_wait_probe(1_000_000_001)


@pytest.mark.parametrize("op", ["embedding", "loss", "append"])
def test_a_wait_that_gives_up_does_not_hide_an_index_outside(ctx, lt, op):  # noqa: F811
    """Both in one flush: the first blocking call says the one, the next the other."""
    g = gen(1)
    table, ids = normal(g, 30, 16), torch.tensor([3, 30, 5], dtype=torch.int32, device="cuda")
    if op == "embedding":
        kept = ctx.embedding(ctx.from_torch(table), ctx.from_torch(ids))
    elif op == "loss":
        kept = ctx.vocabulary_loss(ctx.from_torch(normal(g, 3, 16)), ctx.from_torch(table), ctx.from_torch(ids))
    else:
        kept = ctx.from_torch(torch.zeros(2, 2, 4, 1, 16, device="cuda"))
        k = ctx.from_torch(normal(g, 3, 1, 16))
        ctx.cache_append(kept, k, k, ctx.from_torch(torch.tensor([1, 8, 2], dtype=torch.int32, device="cuda")))
    ctx.barrier()
    ctx.debug_product_wait_probe(1000)
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_TIMEOUT"):
        ctx.barrier(blocking=True)
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_DEVICE_INDEX.*" + dict(embedding="embedding", loss="vocabulary_loss", append="cache_append")[op]):
        ctx.barrier(blocking=True)
    ctx.barrier(blocking=True)
    del kept


# ------------------------------------------------------------------------------------------------ long sums
# A tensor core's sum cuts each product that it adds off at a unit of 2^-23 of the sum; 64 steps of 64 are 4096 products, and sums
# of so many are added up in binary32.
CUT = 4096 * 2.0 ** -23


@pytest.fixture()
def on_the_gpu(monkeypatch):
    monkeypatch.setattr(ref, "WHERE", ["cuda"])


def test_the_tables_gradient_of_many_tokens_rounds_to_the_right_side(ctx):  # noqa: F811
    """262144 tokens with one and the same P and row of x: a sum of equal terms, whose exact value is just above the middle
    between two bf16 numbers in some columns.  In one sum, all of whose 262144 products are cut off, it would end below."""
    tokens, vocab, cols = 1 << 18, 512, 4864
    p, q = (128 + 69) / 1024, 1 + (torch.arange(cols, device="cuda") % 128).double() / 128
    x = q.to(torch.bfloat16).expand(tokens, cols).contiguous()
    table, ids = torch.zeros(vocab, cols, device="cuda", dtype=torch.bfloat16), torch.zeros(tokens, device="cuda", dtype=torch.int32)
    lse, d, dtable = torch.full((tokens,), -math.log(p), device="cuda"), torch.ones(tokens, device="cuda"), torch.empty_like(table)
    ctx.assign(lo := ctx.from_torch(dtable), ctx.op("vocabulary_loss_grad", *(ctx.from_torch(t) for t in (x, table, ids, lse, d)), lo, result=1, scale=1.0))
    ctx.barrier(blocking=True)
    want = tokens * p * q
    bound = (CUT + (tokens / 4096 + 2) * ULP) * want
    ulp = torch.exp2(torch.frexp(want)[1].double() - 8)
    above = want - (torch.floor(want / ulp) + 0.5) * ulp  # of the middle
    sure = above.abs() > bound
    assert int((sure & (above > 0) & (above < 2e-3 * want)).sum()) >= 38  # (columns that the one sum, 5e-3 or more too small, would get wrong)
    want = want.to(torch.bfloat16)
    assert torch.equal(dtable[1:, sure], want[sure].expand(vocab - 1, -1))


def test_gradients_of_rows_of_262144_columns(ctx, on_the_gpu, monkeypatch):  # noqa: F811
    """Scores of tens, sums of terms of one sign: P is their exponential, so that what is cut off them counts tens of times."""
    tokens, vocab, cols = 130, 300, 1 << 18
    g = gen(40)
    x, table = normal(g, tokens, cols).abs() + 0.5, normal(g, vocab, cols).abs() + 0.5
    table *= (torch.linspace(30.0, 60.0, vocab, device="cuda") / (cols * 1.68))[:, None]
    x, table, ids, d = x.to(torch.bfloat16), table.to(torch.bfloat16), tokens_of(g, tokens, vocab, False), normal(g, tokens)
    monkeypatch.setattr(ref, "_scores", lambda x, w, scale: (lambda a, b: (scale * a @ b.T, abs(scale) * (CUT + (cols / 4096 + 2) * ULP) * (a.abs() @ b.abs().T)))(x.double(), w.double()))
    lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
    # (a table that begins behind a 16-byte boundary is taken in pieces, so that no tile's columns are shared out)
    got = ctx.vocabulary_loss_grad(ctx.from_torch(x), unaligned(ctx, table, "bf16"), *(ctx.from_torch(t) for t in (ids, lse, d)))
    r = ref.loss_grad(x, table, ids, lse, d)
    close(fetch(ctx, got[0]), *r[:2], "dx")
    close(fetch(ctx, got[1]), *r[2:], "dtable")


def test_f32_scores_of_524288_columns(ctx):  # noqa: F811
    """x is 1 and a second bf16 part of one sign, the table powers of two times small numbers: the largest of the six products of parts is exact,
    and what is seen is how the sums of the small ones, 2^-8 of it, are made: 128 steps at a time, 8192 products."""
    tokens, vocab, cols = 70, 300, 1 << 19
    g = gen(41)
    x = 1 + 2.0 ** -8 * (0.9 + 0.09 * torch.rand(tokens, cols, device="cuda", generator=g))
    table = (torch.arange(vocab, device="cuda") % 61 / cols).float()[:, None].expand(vocab, cols).contiguous()
    ids = torch.zeros(tokens, device="cuda", dtype=torch.int32)
    loss, lse = (fetch(ctx, t) for t in ctx.vocabulary_loss(*(ctx.from_torch(t) for t in (x, table, ids))))
    z = (x.double().sum(-1)[:, None] * table[:, 0].double()[None]).cpu()
    want = torch.logsumexp(z, -1)
    far = (z * (8 * ULP + 2.0 ** -8 * (8192 * 2.0 ** -23 + cols / 8192 * ULP) + 4 * 2.0 ** -23)).amax(-1) + (vocab / 256 + 320) * ULP + want * 4 * ULP
    close(lse, want, far)
    close(loss, want, far + want * 4 * ULP)


# ------------------------------------------------------------------------------------------------ weights of very different size
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tokens", [2, 40, 300, 4096, 4097, 9000])
def test_losses_weighted_from_2_to_the_minus_60_to_2_to_the_60(ctx, on_the_gpu, dtype, tokens):  # noqa: F811
    """No product of a gradient, which is 2^70 at most, leaves binary32 on the way, whichever token comes first."""
    g, t = gen(tokens), TYPES[dtype]
    x, table, ids = normal(g, tokens, 72, dtype=t, std=2.0 ** 10), normal(g, 200, 72, dtype=t, std=2.0 ** -13), tokens_of(g, tokens, 200)
    for first, others in ((2.0 ** -60, 2.0 ** 60), (2.0 ** 60, 2.0 ** -60), (0.0, -2.0 ** 100), (math.inf, 3.0), (math.nan, 2.0 ** 90)):
        d = torch.where(torch.rand(tokens, device="cuda", generator=g) < 0.5, others, 1.0)
        d[0], d[-1] = first, others
        ids[0] = 3 if math.isfinite(first) else -1  # (of a token without a target it does not count)
        lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
        got = ctx.vocabulary_loss_grad(*(ctx.from_torch(v) for v in (x, table, ids, lse, d)))
        r = ref.loss_grad(x, table, ids, lse, d)
        close(fetch(ctx, got[0]), *r[:2], "dx")
        close(fetch(ctx, got[1]), *r[2:], "dtable")


@pytest.mark.parametrize("tokens", [300, 5000])
def test_a_weight_that_all_tokens_share_leaves_x_as_it_is(ctx, tokens):  # noqa: F811
    """Gradients of 0 and w for weights are w times those of 0 and 1, to the last bit where w is a power of two."""
    g = gen(tokens)
    x, table, ids = normal(g, tokens, 64, dtype=torch.bfloat16), normal(g, 700, 64, dtype=torch.bfloat16, std=0.2), tokens_of(g, tokens, 700)
    mask = (torch.rand(tokens, device="cuda", generator=g) < 0.7).float()
    mask[0] = 0.0
    lse = torch.logsumexp(x.double() @ table.double().T, -1).float()
    one, other = ([fetch(ctx, r).float() for r in ctx.vocabulary_loss_grad(*(ctx.from_torch(v) for v in (x, table, ids, lse, w * mask)))] for w in (1.0, -2.0 ** -13))
    assert all(torch.equal(b, a * -2.0 ** -13) for a, b in zip(one, other))


# ------------------------------------------------------------------------------------------------ few tokens of long rows
@pytest.mark.parametrize("tokens,cols,launches", [(16, 3328, 2), (9, 3329, 2), (16, 4100, 2), (64, 4096, 2), (33, 6656, 2), (8, 6657, 2), (5, 8200, 2), (64, 8193, 2), (3, 13312, 2), (17, 13312, 2),
                                                  (4, 13313, None), (16, 13400, None)])
def test_few_f32_tokens_are_scored_by_plain_loads_however_long_their_rows(ctx, tokens, cols, launches):  # noqa: F811
    """Fewer of them at a time where not all fit in shared memory: two launches, none of which packs the table."""
    g = gen(tokens + cols)
    x, table, ids = normal(g, tokens, cols, std=2.0), normal(g, 300, cols, std=cols ** -0.5), tokens_of(g, tokens, 300)
    ids[0], ids[-1] = -1, 299
    before = ctx.stats()["kernels_launched"]
    loss, lse = ctx.vocabulary_loss(*(ctx.from_torch(t) for t in (x, table, ids)))
    ctx.barrier(blocking=True)
    if launches:
        assert ctx.stats()["kernels_launched"] - before == launches
    a, b, c, d = ref.loss(x, table, ids)
    close(fetch(ctx, loss), a, b, "loss")
    close(fetch(ctx, lse), c, d, "lse")


# ------------------------------------------------------------------------------------------------ memory
def planned(c, lt, record):  # noqa: F811
    """Bytes of temporaries that what `record` records takes, as a flush that may not allocate says when it refuses it."""
    kept = record()
    with pytest.raises(lt.LazyTensorError, match="LT_ERR_UNSUPPORTED.*bytes of temporaries") as err:
        c.barrier_static_scratch()
    c.barrier(blocking=True)
    del kept
    return int(str(err.value).split("the graph needs ")[1].split()[0])


@pytest.mark.parametrize("tokens,vocab,cols", [(65536, 1000, 512), (16384, 3000, 1024)])
def test_the_gradients_of_bf16_copy_x_once(ctx, lt, tokens, vocab, cols):  # noqa: F811
    """P, x scaled, room for pieces of x and the table (8 MB each), and sums of dx and dtable in binary32."""
    g, t = gen(1), torch.bfloat16
    v = [normal(g, tokens, cols, dtype=t), normal(g, vocab, cols, dtype=t), tokens_of(g, tokens, vocab), torch.zeros(tokens, device="cuda"), torch.ones(tokens, device="cuda")]
    h = [ctx.from_torch(x) for x in v]
    out = [ctx.from_torch(torch.empty_like(x)) for x in v[:2]]
    need = planned(ctx, lt, lambda: ctx.vocabulary_loss_grad(*h, out=out))
    p = min(256 << 20, 2 * tokens * (vocab + 255))
    splits = 4 * (148 // 2) * 256 * 256  # (of products with few tiles: at most a tile's sums for each pair of blocks)
    assert need <= p + 2 * tokens * cols + (16 << 20) + 4 * tokens * cols * (2 * tokens * vocab > p) + 2 * splits + 16 * tokens


@pytest.mark.parametrize("tokens,vocab,cols,where", [(773, 300, 16392, "begins"), (773, 300, 16392, "both"), (60000, 300, 1001, "lies"), (2100, 70000, 4096, "begins")])
def test_gradients_where_x_is_packed_in_pieces(ctx, on_the_gpu, tokens, vocab, cols, where):  # noqa: F811
    """bf16 rows that begin behind a 16-byte boundary (the last piece of few of them), and rows of odd length; pieces of P, too."""
    g, t = gen(tokens), torch.bfloat16
    x, table, ids, d = normal(g, tokens, cols, dtype=t), normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab), normal(g, tokens)
    ids[::5] = -1
    x[0], x[tokens - 1], ids[tokens - 1] = math.nan, math.inf, -1
    lse = torch.where(ids >= 0, torch.logsumexp(x.double() @ table.double().T, -1), 0.0).float()
    lx = ctx.from_torch(x) if where == "lies" else unaligned(ctx, x, "bf16")
    lw = unaligned(ctx, table, "bf16") if where == "both" else ctx.from_torch(table)
    got = ctx.vocabulary_loss_grad(lx, lw, *(ctx.from_torch(v) for v in (ids, lse, d)))
    r = ref.loss_grad(x, table, ids, lse, d)
    close(fetch(ctx, got[0]), *r[:2], "dx")
    close(fetch(ctx, got[1]), *r[2:], "dtable")


# ------------------------------------------------------------------------------------------------ a training step
def step64_bounds(s):
    """The step of test_gpu_table_operators in 64 bits and, for every value, how far binary32 may be from it: the roundings of each
    operator, and what those of the ones before it become in it."""
    table, gamma, ids = s["table"].double().cpu(), s["gamma"].double().cpu(), s["ids"].long().cpu()
    t, d = s["targets"].long().cpu(), s["dloss"].double().cpu()
    n, (v, c) = ids.numel(), table.shape
    e = 2.0 * table[ids]
    r = torch.rsqrt((e * e).mean(-1, keepdim=True) + 1e-6)
    x, dx_ = gamma * e * r, (gamma * e * r).abs() * (c + 8) * ULP
    z = x @ table.T
    dz = dx_ @ table.T.abs() + 2 * (c + 16) * ULP * (x.abs() @ table.T.abs())
    lse = torch.logsumexp(z, -1)
    far = (z.abs() * 8 * ULP + dz).amax(-1) + (v / 256 + 320) * ULP + lse.abs() * 4 * ULP
    there, at = t >= 0, t.clamp(min=0)[:, None]
    loss = torch.where(there, lse - z.gather(1, at)[:, 0], 0.0)
    loss_off = torch.where(there, far + dz.gather(1, at)[:, 0] + (loss.abs() + z.gather(1, at)[:, 0].abs()) * 4 * ULP, 0.0)
    hot = torch.zeros_like(z).scatter_(1, at, 1.0)
    k = torch.where(there, d, 0.0)[:, None]
    ez = torch.exp(z - lse[:, None])
    p, dp = k * (ez - hot), k.abs() * (ez * (dz + far[:, None] + 8 * ULP * (z.abs() + lse.abs()[:, None] + 1)) + 8 * ULP * (ez + hot))
    gx, gx_off = p @ table, dp @ table.abs() + 2 * (v + 64) * ULP * (p.abs() @ table.abs())
    dw, dw_off = p.T @ x, dp.T @ x.abs() + p.abs().T @ dx_ + 2 * (n + 64) * ULP * (p.abs().T @ x.abs())
    # the norm's gradient: r (gamma gx - e r^2 mean(gamma gx e)), and of gamma the sum of gx e r
    q = (gamma * gx * e).mean(-1, keepdim=True)
    q_off = ((gamma.abs() * gx_off * e.abs()).mean(-1, keepdim=True) + (c + 8) * ULP * (gamma * gx * e).abs().mean(-1, keepdim=True))
    ge = r * (gamma * gx - e * r * r * q)
    ge_off = r * (gamma.abs() * gx_off + (c + 16) * ULP * (gamma * gx).abs() + e.abs() * r * r * (q_off + (2 * c + 16) * ULP * q.abs()))
    gg, gg_off = (gx * e * r).sum(0), ((gx_off + (c + n + 16) * ULP * gx.abs()) * (e * r).abs()).sum(0)
    out = dw + 2.0 * torch.zeros_like(table).index_add_(0, ids, ge)
    size = torch.zeros_like(table).index_add_(0, ids, 2 * ge.abs())
    off = dw_off + torch.zeros_like(table).index_add_(0, ids, 2 * ge_off) + (n + 4) * ULP * size + 2 * ULP * out.abs()
    return [(loss, loss_off), (out, off), (gg, gg_off)]


def test_every_value_of_a_training_step(ctx):  # noqa: F811
    """Rows of the table's gradient that few tokens touch are as near as their own terms are, and none is left out."""
    s, out = make_step(21)
    want = step64_bounds(s)
    assert all(torch.allclose(a, b[0], rtol=1e-9, atol=1e-12) for a, b in zip(step64(s), want))
    # (a bound that tells rows from nothing: nine in ten values of the table's gradient are more than ten bounds away from zero)
    assert float((want[1][0].abs() > 10 * want[1][1]).double().mean()) > 0.9
    t, lo = handles(ctx, s, out)
    for _ in range(3):  # (planned, then matched)
        for o in out:
            o.fill_(math.nan)
        step(ctx, t, lo)
        ctx.barrier(blocking=True)
        for got, w, name in zip(out, want, ("loss", "table", "gamma")):
            close(got, *w, name)
    for o in out:
        o.fill_(math.nan)
    ctx.replay(blocking=True)
    for got, w, name in zip(out, want, ("loss", "table", "gamma")):
        close(got, *w, name)


def test_two_streams_at_once_give_the_bits_that_each_gives_alone(lt):  # noqa: F811
    made = []
    for k in range(2):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            s, out = make_step(50 + k, tokens=500 + 131 * k, vocab=3000 - 700 * k, cols=128)
            c = lt.LazyContext(device=0, stream=stream.cuda_stream)
            made.append([stream, out, c, handles(c, s, out), []])
    torch.cuda.synchronize()
    for stream, out, c, (t, lo), alone in made:
        step(c, t, lo)
        c.barrier(blocking=True)
        alone += [o.clone() for o in out]
        torch.cuda.synchronize()
    for _ in range(5):
        for stream, out, c, (t, lo), alone in made:
            with torch.cuda.stream(stream):
                for o in out:
                    o.fill_(math.nan)
            step(c, t, lo)
            c.barrier()
        for stream, out, c, (t, lo), alone in made:
            c.barrier(blocking=True)
        for stream, out, c, (t, lo), alone in made:
            assert all(torch.equal(a, b) for a, b in zip(alone, out))
    for entry in made:
        entry[2].close()


def test_many_tokens_with_weights_of_their_own_captured_and_replayed(lt, on_the_gpu):  # noqa: F811
    """More tokens than a block looks through for the largest weight, x in pieces; the graph is replayed on new weights, targets and rows of x."""
    stream = torch.cuda.Stream()
    g, t = gen(60), torch.bfloat16
    tokens, vocab, cols = 5003, 300, 1024
    room = torch.empty(tokens * cols + 64, device="cuda", dtype=t)
    x = room[1: 1 + tokens * cols].view(tokens, cols)  # (begins behind a 16-byte boundary)
    table, ids, lse, d = normal(g, vocab, cols, dtype=t, std=cols ** -0.5), tokens_of(g, tokens, vocab), torch.zeros(tokens, device="cuda"), normal(g, tokens)
    x.copy_(normal(g, tokens, cols, dtype=t))
    dx, dw = torch.empty(tokens, cols, device="cuda", dtype=t), torch.empty_like(table)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        c = lt.LazyContext(device=0, stream=stream.cuda_stream)
        lx = c.from_device_ptr(x.data_ptr(), "bf16", tuple(x.shape), keep=room)
        h = [lx, *(c.from_torch(v) for v in (table, ids, lse, d))]
        out = [c.from_torch(v) for v in (dx, dw)]
        c.vocabulary_loss_grad(*h, out=out)
        c.barrier(blocking=True)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            c.vocabulary_loss_grad(*h, out=out)
            c.barrier()
        for size in (2.0 ** -40, 2.0 ** 40):
            x.copy_(normal(g, tokens, cols, dtype=t))
            ids.copy_(tokens_of(g, tokens, vocab))
            ids[::11] = -1
            d.copy_(normal(g, tokens) * size)
            lse.copy_(torch.logsumexp(x.double() @ table.double().T, -1))
            dx.fill_(math.nan), dw.fill_(math.nan)
            graph.replay()
            stream.synchronize()
            r = ref.loss_grad(x, table, ids, lse, d)
            close(dx, *r[:2], "dx")
            close(dw, *r[2:], "dtable")
        c.barrier(blocking=True)
        del graph
        c.close()
