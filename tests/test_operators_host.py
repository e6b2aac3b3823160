"""The transformer operators on a record-and-plan-only context: shapes, refusals, which launches a graph becomes, what is
written in place, and the frequencies of rotary positions.  No GPU."""
import math
import threading
import time

import numpy as np
import pytest

import paper_2102_13267_b200 as lt


@pytest.fixture()
def ctx():
    c = lt.LazyContext(device=None)
    yield c
    c.close()


def fake(ctx, shape, dtype="f32", base=[1 << 30]):
    """Device data at an address that is never looked at (nothing is launched)."""
    base[0] += 1 << 28
    return ctx.from_device_ptr(base[0], dtype, shape)


def plan(ctx):
    ctx.barrier()
    return ctx.dump_plan()


ROT = dict(interleaved=False, inverse=False, scale=1.0)
APP = dict(head_major=False, interleaved=False, scale=1.0)
ATT = dict(head_major=False, scale=0.1)
NRM = dict(result=0, residual=False, group=0, eps=1e-6)
GRD = dict(result=0, residual=False, eps=1e-6)


# ------------------------------------------------------------------------------------------------ shapes
def test_result_shapes(ctx):
    f = lambda *a: fake(ctx, *a)  # noqa: E731
    turned = ctx.rotary(f((5, 3, 16), "bf16"), f((5,), "i32"), f((8, 2), "u32"))
    assert (turned.shape, turned.dtype) == ((5, 3, 16), "bf16")
    assert ctx.rotary(f((5, 16)), f((5,), "i32"), f((3, 2), "u32")).shape == (5, 16)
    cache = f((4, 2, 16, 2, 32), "bf16")
    ctx.cache_append(cache, f((3, 2, 32), "bf16"), f((3, 2, 32), "bf16"), f((3,), "i32"))
    assert cache.shape == (4, 2, 16, 2, 32)
    t = ctx.paged_attention(f((7, 6, 32), "bf16"), cache, f((7, 3), "i32"), f((7,), "i32"), scale=1.0)
    assert (t.shape, t.dtype) == ((7, 6, 32), "bf16")
    c, s, h = ctx.rms_norm(f((2, 3, 100), "bf16"), f((100,)), residual=f((2, 3, 100), "bf16"), eight_bit=True, group=32)
    assert [(x.shape, x.dtype) for x in (c, s, h)] == [((2, 3, 100), "u8"), ((2, 3, 4), "f32"), ((2, 3, 100), "bf16")]
    dx, dg = ctx.rms_norm_grad(f((2, 3, 100), "bf16"), f((2, 3, 100), "bf16"), f((100,), "bf16"))
    assert (dx.shape, dx.dtype, dg.shape, dg.dtype) == ((2, 3, 100), "bf16", (100,), "bf16")
    text = ctx.dump_ir()
    for name in ("rotary", "cache_append", "paged_attention", "rms_norm", "rms_norm_grad"):
        assert f"lt::{name}(" in text


# ------------------------------------------------------------------------------------------------ refusals
def refused(ctx, status, name, shapes, **attrs):
    nodes = ctx.stats()["nodes_recorded"]
    ins = [fake(ctx, *s) if isinstance(s, tuple) else s for s in shapes]
    with pytest.raises(lt.LazyTensorError, match=status + ".*" + name):
        ctx.op(name, *ins, **attrs)
    assert ctx.stats()["nodes_recorded"] == nodes + sum(isinstance(s, tuple) for s in shapes)


X, POS, FRQ = ((5, 3, 16), "f32"), ((5,), "i32"), ((8, 2), "u32")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [X, POS], ROT), ("INVALID_ARG", [X, POS, FRQ, X, X], ROT), ("DTYPE", [((5, 3, 16), "i32"), POS, FRQ], ROT), ("SHAPE", [((5,), "f32"), POS, FRQ], ROT),
    ("DTYPE", [X, ((5,), "f32"), FRQ], ROT), ("SHAPE", [X, ((4,), "i32"), FRQ], ROT), ("DTYPE", [X, POS, ((8,), "u32")], ROT), ("DTYPE", [X, POS, ((8, 2), "f32")], ROT),
    ("SHAPE", [X, POS, ((9, 2), "u32")], ROT), ("SHAPE", [X, POS, FRQ, ((5, 3, 15), "f32")], ROT), ("SHAPE", [X, POS, FRQ, ((5, 3, 16), "bf16")], ROT),
    ("INVALID_ARG", [X, POS, FRQ], dict(ROT, scale=math.inf)), ("INVALID_ARG", [X, POS, FRQ], dict(ROT, scale=math.nan))])
def test_rotary_refusals(ctx, status, shapes, attrs):
    refused(ctx, status, "rotary", shapes, **attrs)


CA, K, SL = ((4, 2, 16, 2, 32), "bf16"), ((3, 2, 32), "bf16"), ((3,), "i32")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [CA, K, K], APP), ("INVALID_ARG", [CA, K, K, SL, SL], APP), ("DTYPE", [CA, ((3, 2, 32), "f32"), K, SL], APP), ("SHAPE", [((4, 16, 2, 32), "bf16"), K, K, SL], APP),
    ("SHAPE", [((4, 3, 16, 2, 32), "bf16"), K, K, SL], APP), ("SHAPE", [CA, K, K, SL], dict(APP, head_major=True)), ("SHAPE", [CA, K, ((4, 2, 32), "bf16"), SL], APP),
    ("DTYPE", [CA, K, K, ((3,), "u32")], APP), ("SHAPE", [CA, K, K, ((4,), "i32")], APP), ("SHAPE", [CA, K, K, SL, SL, ((17, 2), "u32")], APP),
    ("DTYPE", [CA, K, K, SL, SL, ((16, 2), "i32")], APP), ("SHAPE", [CA, K, K, SL, ((2,), "i32"), ((16, 2), "u32")], APP),
    ("UNSUPPORTED", [((1 << 28, 2, 16, 2, 32), "bf16"), K, K, SL], APP), ("INVALID_ARG", [CA, K, K, SL], dict(APP, scale=math.nan))])
def test_cache_append_refusals(ctx, status, shapes, attrs):
    refused(ctx, status, "cache_append", shapes, **attrs)


Q, TB, LN = ((7, 6, 32), "bf16"), ((7, 3), "i32"), ((7,), "i32")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [Q, CA, TB], ATT), ("DTYPE", [((7, 6, 32), "f32"), CA, TB, LN], ATT), ("DTYPE", [((7, 6, 32), "u8"), ((4, 2, 16, 2, 32), "u8"), TB, LN], ATT),
    ("SHAPE", [((7, 5, 32), "bf16"), CA, TB, LN], ATT), ("SHAPE", [((7, 6, 16), "bf16"), CA, TB, LN], ATT), ("SHAPE", [((7, 192), "bf16"), CA, TB, LN], ATT),
    ("SHAPE", [Q, CA, ((6, 3), "i32"), LN], ATT), ("SHAPE", [Q, CA, TB, ((6,), "i32")], ATT), ("DTYPE", [Q, CA, ((7, 3), "u32"), LN], ATT), ("DTYPE", [Q, CA, TB, ((7,), "f32")], ATT),
    ("SHAPE", [Q, ((4, 2, 16, 2, 32, 1), "bf16"), TB, LN], ATT), ("SHAPE", [Q, CA, TB, LN, ((7, 6, 31), "bf16")], ATT), ("UNSUPPORTED", [((7, 6, 264), "bf16"), ((4, 2, 16, 2, 264), "bf16"), TB, LN], ATT),
    ("UNSUPPORTED", [((70000, 6, 32), "bf16"), CA, ((70000, 3), "i32"), ((70000,), "i32")], ATT), ("UNSUPPORTED", [Q, CA, ((7, 1 << 28), "i32"), LN], ATT),
    ("UNSUPPORTED", [((1, 2, 32), "bf16"), CA, ((1, (1 << 26) + 1), "i32"), ((1,), "i32")], ATT), ("INVALID_ARG", [Q, CA, TB, LN], dict(ATT, scale=math.inf))])
def test_paged_attention_refusals(ctx, status, shapes, attrs):
    refused(ctx, status, "paged_attention", shapes, **attrs)


R, G = ((4, 64), "bf16"), ((64,), "f32")


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [R], NRM), ("INVALID_ARG", [R, R, G, R], NRM), ("DTYPE", [((4, 64), "i32"), G], NRM), ("SHAPE", [R, ((63,), "f32")], NRM), ("SHAPE", [R, ((1, 64), "f32")], NRM),
    ("DTYPE", [((4, 64), "f32"), ((64,), "bf16")], NRM), ("SHAPE", [R, ((4, 63), "bf16"), G], dict(NRM, residual=True)), ("SHAPE", [R, ((4, 64), "f32"), G], dict(NRM, residual=True)),
    ("INVALID_ARG", [R, G], dict(NRM, result=1)), ("INVALID_ARG", [R, G], dict(NRM, result=4)), ("INVALID_ARG", [R, G], dict(NRM, group=16)), ("INVALID_ARG", [R, G], dict(NRM, group=100)),
    ("INVALID_ARG", [R, G], dict(NRM, eps=-1.0)), ("INVALID_ARG", [R, G], dict(NRM, eps=math.nan)), ("SHAPE", [R, G, R], dict(NRM, result=2)), ("SHAPE", [R, G, ((4, 64), "f32")], dict(NRM, result=3))])
def test_rms_norm_refusals(ctx, status, shapes, attrs):
    refused(ctx, status, "rms_norm", shapes, **attrs)


@pytest.mark.parametrize("status,shapes,attrs", [
    ("INVALID_ARG", [R, R], GRD), ("DTYPE", [R, ((4, 64), "f32"), G], GRD), ("SHAPE", [R, ((5, 64), "bf16"), G], GRD), ("SHAPE", [R, R, G, ((4, 65), "bf16")], dict(GRD, residual=True)),
    ("SHAPE", [R, R, ((65,), "f32")], GRD), ("INVALID_ARG", [R, R, G], dict(GRD, result=2)), ("SHAPE", [R, R, G, R], dict(GRD, result=1)), ("INVALID_ARG", [R, R, G], dict(GRD, eps=math.inf))])
def test_rms_norm_grad_refusals(ctx, status, shapes, attrs):
    refused(ctx, status, "rms_norm_grad", shapes, **attrs)


def test_constants_and_raw_attributes_are_refused(ctx):
    with pytest.raises(lt.LazyTensorError, match="constants"):
        ctx.op("rms_norm", ctx.scalar(2.0), fake(ctx, (1,)), **NRM)
    import ctypes

    h = (ctypes.c_uint64 * 7)(*[fake(ctx, (4, 4)).handle] * 7)
    out, attrs = ctypes.c_uint64(), (ctypes.c_int64 * 4)(0, 0, 0, 0)
    for op in (70, 71, 72, 73, 74):
        for n_in, n_attrs in ((7, 4), (0, 0), (2, 1), (3, 0)):
            assert lt._lib.lt_op(ctx._ctx, op, h, n_in, attrs, n_attrs, ctypes.byref(out)) != 0
    assert lt._lib.lt_op(ctx._ctx, 75, h, 2, attrs, 0, ctypes.byref(out)) == lt.STATUS_NAMES.index("LT_ERR_UNSUPPORTED")
    assert lt._lib.lt_op(ctx._ctx, 1, h, 4, attrs, 0, ctypes.byref(out)) == lt.STATUS_NAMES.index("LT_ERR_INVALID_ARG")


def test_python_argument_checks(ctx):
    c = fake(ctx, *CA)
    with pytest.raises(ValueError):
        ctx.cache_append(c, fake(ctx, *K), fake(ctx, *K), fake(ctx, *SL), fake(ctx, *SL))
    with pytest.raises(ValueError):
        ctx.rms_norm(fake(ctx, *R), fake(ctx, *G), out=(fake(ctx, *R), None))
    with pytest.raises(ValueError):
        ctx.rms_norm_grad(fake(ctx, *R), fake(ctx, *R), fake(ctx, *G), out=(None,))


# ------------------------------------------------------------------------------------------------ plans
def test_results_of_one_operator_are_one_launch(ctx):
    x, r, g = fake(ctx, *R), fake(ctx, *R), fake(ctx, *G)
    a = ctx.rms_norm(x, g, residual=r, eight_bit=True, group=32)
    p = plan(ctx)
    assert p.count("launch ") == 1 and "operator: rms_norm, results=3" in p
    b = ctx.rms_norm(x, g, residual=r, eight_bit=True, group=64) + ctx.rms_norm(x, g, residual=r, eight_bit=True, group=32)
    assert plan(ctx).count("operator: rms_norm, results=3") == 2  # another group is another launch
    two = [ctx.rms_norm(x, g, residual=r), ctx.rms_norm(x, g, residual=r, eps=1e-5), ctx.rms_norm(x, g)]
    assert plan(ctx).count("operator: rms_norm") == 3
    d = ctx.rms_norm_grad(x, r, g)
    assert "operator: rms_norm_grad, results=2" in plan(ctx)
    same = [ctx.op("rms_norm", x, g, **NRM) for _ in range(2)]  # the same result twice: each its own
    assert plan(ctx).count("operator: rms_norm, results=1") == 2
    ctx.set_option("fusion", 0)
    e = ctx.rms_norm_grad(x, r, g)
    assert plan(ctx).count("operator: rms_norm_grad, results=1") == 2
    del a, b, two, d, same, e


def decode(ctx, b, n=1):
    """The operators of a decode step on fake buffers; returns the handles and outputs."""
    t = dict(qkv=fake(ctx, (4, 12, 64), "bf16"), cache=fake(ctx, (9, 2, 2, 16, 64), "bf16"), pos=fake(ctx, (4,), "i32"), slots=fake(ctx, (4,), "i32"), len=fake(ctx, (4,), "i32"),
             table=fake(ctx, (4, 3), "i32"), f=fake(ctx, (32, 2), "u32"), att=fake(ctx, (4, 8, 64), "bf16"), x=fake(ctx, (4, 512), "bf16"), res=fake(ctx, (4, 512), "bf16"),
             g=fake(ctx, (512,)), y=fake(ctx, (4, 512), "bf16"))
    return t


def record(b, t):
    q = b.rotary(b.op("narrow", t["qkv"], dim=1, start=0, length=8), t["pos"], t["f"])
    k, v = (b.op("narrow", t["qkv"], dim=1, start=s, length=2) for s in (8, 10))
    b.cache_append(t["cache"], k, v, t["slots"], t["pos"], t["f"], head_major=True)
    b.paged_attention(q, t["cache"], t["table"], t["len"], scale=0.125, head_major=True, out=t["att"])
    b.rms_norm(t["x"], t["g"], residual=t["res"], out=(t["y"], t["res"]))


def test_a_decode_step_runs_in_place_on_four_launches(ctx):
    t = decode(ctx, ctx)
    where = {k: ctx.device_ptr(v) for k, v in t.items()}
    record(ctx, t)
    p = plan(ctx)
    assert p.count("launch ") == 4 and "copy kernel" not in p
    for k in ("cache", "att", "res", "y"):
        assert ctx.device_ptr(t[k]) == where[k], k
    s = ctx.stats()
    assert s["outputs_donated"] == 4 and s["outputs_allocated"] == 0


def test_recorded_call_by_call_or_in_a_batch_it_is_the_same_plan(ctx):
    t = decode(ctx, ctx)
    record(ctx, t)
    ctx.barrier()
    b = lt.Batch()
    refs = {k: b.input() for k in t}
    record(b, refs)
    for i in range(3):
        ctx.record(b, list(t.values()))
        ctx.barrier()
    s = ctx.stats()
    assert s["compiles"] == 1 and s["cache_hits"] == 3


def test_batch_of_operators_without_shape_operations_is_matched(ctx):
    """The steady state of a loop: the trace repeats and is bound to its plan without being built."""
    x, r, g, y = fake(ctx, *R), fake(ctx, *R), fake(ctx, *G), fake(ctx, *R)
    q, c, tb, ln, o = (fake(ctx, *s) for s in (Q, CA, TB, LN, Q))
    b = lt.Batch()
    i = [b.input() for _ in range(9)]
    b.rms_norm(i[0], i[2], residual=i[1], out=(i[3], i[1]))
    b.paged_attention(i[4], i[5], i[6], i[7], scale=0.3, out=i[8])
    for k in range(5):
        ctx.record(b, [x, r, g, y, q, c, tb, ln, o])
        ctx.barrier()
    s = ctx.stats()
    assert s["compiles"] == 1 and s["traces_matched"] >= 3 and s["outputs_allocated"] == 0
    # one that differs in an attribute only is another graph
    b2 = lt.Batch()
    i = [b2.input() for _ in range(5)]
    b2.paged_attention(*i[:4], scale=0.4, out=i[4])
    ctx.record(b2, [q, c, tb, ln, o])
    ctx.barrier()
    assert ctx.stats()["compiles"] == 2


def test_results_that_may_not_go_in_place(ctx):
    q, c, tb, ln = (fake(ctx, *s) for s in (Q, CA, TB, LN))
    where = ctx.device_ptr(q)
    ctx.assign(q, ctx.op("paged_attention", q, c, tb, ln, **ATT))  # other blocks still read q
    ctx.barrier()
    assert ctx.device_ptr(q) != where
    # a cache that is read after the append, by something that wants the old one
    old = ctx.paged_attention(fake(ctx, *Q), c, tb, ln, scale=1.0)
    where = ctx.device_ptr(c)
    ctx.cache_append(c, fake(ctx, *K), fake(ctx, *K), fake(ctx, *SL))
    new = ctx.paged_attention(fake(ctx, *Q), c, tb, ln, scale=1.0)
    p = plan(ctx)
    before = p.index("operator: paged_attention") < p.index("operator: cache_append")
    assert (ctx.device_ptr(c) == where) == before
    # a buffer somebody else names
    x, g, y = fake(ctx, *R), fake(ctx, *G), fake(ctx, *R)
    other = ctx.op("reshape", y, shape=(64, 4))  # (a value of its own over the same memory, not a view)
    where = ctx.device_ptr(y)
    ctx.rms_norm(x, g, out=(y,))
    ctx.barrier()
    assert ctx.device_ptr(y) != where
    del old, new, other


def test_slices_are_read_in_place_only_where_rows_are_runs(ctx):
    f, pos = fake(ctx, (4, 2), "u32"), fake(ctx, (6,), "i32")
    big = fake(ctx, (6, 10, 16))
    a = ctx.rotary(ctx.op("narrow", big, dim=1, start=2, length=4), pos, f)
    assert "copy kernel" not in plan(ctx)
    b = ctx.rotary(ctx.op("narrow", big, dim=2, start=2, length=8), pos, f)  # a part of every head
    assert "copy kernel" in plan(ctx)
    c = ctx.rotary(ctx.op("narrow", fake(ctx, (9, 4, 16)), dim=0, start=3, length=6), pos, f)
    assert "copy kernel" not in plan(ctx)
    d = ctx.rotary(ctx.op("narrow", fake(ctx, (6, 1, 32)), dim=2, start=3, length=16), pos, f)  # one head: still a run
    assert "copy kernel" not in plan(ctx)
    e = ctx.rms_norm(ctx.op("narrow", fake(ctx, (2, 3, 32)), dim=2, start=3, length=16), fake(ctx, (16,)))
    assert "copy kernel" not in plan(ctx)
    n = ctx.op("narrow", fake(ctx, (6, 10, 16)), dim=1, start=0, length=4)
    h = ctx.rotary(n, pos, f)  # the slice is a result as well
    assert "copy kernel" in plan(ctx)
    i = ctx.rms_norm(fake(ctx, (4, 16)), ctx.op("narrow", fake(ctx, (32,)), dim=0, start=3, length=16))  # not a row operand
    assert "copy kernel" in plan(ctx)
    del a, b, c, d, e, h, i


def test_an_operation_that_a_batch_refuses_leaves_nothing_behind(ctx):
    t = [fake(ctx, *s) for s in (CA, K, K, SL)]
    b = lt.Batch()
    i = [b.input() for _ in t]
    for bad in (lambda: b.op("none such", *i), lambda: b.op("cache_append", i[0], None, i[2], i[3], **APP), lambda: b.op("cache_append", *i[:3], None, **APP)):
        with pytest.raises((KeyError, AttributeError)):
            bad()
    b.cache_append(*i)
    ctx.record(b, t)
    assert "operator: cache_append" in plan(ctx)


def test_more_than_three_operands_in_a_batch(ctx):
    import ctypes

    t = [fake(ctx, *s) for s in (CA, K, K, SL)]
    hs = (ctypes.c_uint64 * 4)(*[x.handle for x in t])
    attrs = (ctypes.c_int64 * 3)(0, 0, lt._double_bits(1.0))

    def run(entries):
        ops, res = (lt.lt_batch_op * len(entries))(), (ctypes.c_uint64 * len(entries))()
        for o, (code, ins, na) in zip(ops, entries):
            o.opcode, o.n_in, o.n_attrs, o.attr_offset, o.keep = code, abs(ins[0]) if isinstance(ins, tuple) else len(ins), na, 0, 0
            for k, v in enumerate((ins[1] if isinstance(ins, tuple) else ins)[:3]):
                o.in_[k] = v
        return lt._lib.lt_op_many(ctx._ctx, ops, len(entries), hs, 4, attrs, res)

    more, app = lt.LT_BATCH_MORE, 71
    assert run([(more, [3], 0), (app, (4, [0, 1, 2]), 3)]) == 0
    for bad in ([(app, (4, [0, 1, 2]), 3)], [(more, [3], 0)], [(more, [3], 0), (more, [3], 0), (app, (4, [0, 1, 2]), 3)], [(more, [3, 3], 0), (app, (4, [0, 1, 2]), 3)],
                [(more, [9], 0), (app, (4, [0, 1, 2]), 3)], [(more, (4, [0, 1, 2]), 0), (app, (7, [0, 1, 2]), 3)], [(more, [3], 0), (lt.LT_BATCH_ASSIGN, [0, 0], 0)], [(more, [], 0), (app, [0, 1, 2], 3)]):
        assert run(bad) == lt.STATUS_NAMES.index("LT_ERR_INVALID_ARG"), bad


def test_other_threads_run_while_a_batch_is_recorded(ctx):
    """The recording call does not hold the interpreter lock: the clock is read on another thread in the middle of it."""
    x = fake(ctx, (4, 4))
    b = lt.Batch()
    r = b.input()
    for _ in range(300000):
        r = b.op("neg", r)
    ctx.record(b, [x])  # (compiles the batch)
    reads, stop = [], threading.Event()

    def watch():
        while not stop.is_set():
            reads.append(time.perf_counter())
            time.sleep(0)

    t = threading.Thread(target=watch)
    t.start()
    try:
        while not reads:
            time.sleep(0.001)
        begin = time.perf_counter()
        ctx.record(b, [x])
        end = time.perf_counter()
    finally:
        stop.set()
        t.join()
    quarter = (end - begin) / 4
    assert any(begin + quarter < at < end - quarter for at in reads), (begin, end, len(reads))


def test_one_batch_on_several_threads(ctx):
    """A batch may be recorded on several threads at once, each on a context of its own."""
    b = lt.Batch()
    i = b.input()
    for _ in range(2000):
        i = b.op("neg", i)
    b.keep(i)
    failed = []

    def work(k):
        c = lt.LazyContext(device=None)
        try:
            for j in range(20):
                r, = c.record(b, [fake(c, (k + 1, j + 1))])
                if r.shape != (k + 1, j + 1):
                    failed.append((k, j, r.shape))
                del r
        except Exception as e:  # noqa: BLE001
            failed.append((k, e))
        finally:
            c.close()

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed, failed[:3]


# ------------------------------------------------------------------------------------------------ frequencies
def radians(table):
    return [((int(hi) << 32 | int(lo)) / 2.0 ** 64) * 2 * math.pi for lo, hi in table]


def test_rotary_table():
    t = lt.rotary_table(128)
    assert t.shape == (64, 2) and t.dtype == np.uint32
    np.testing.assert_allclose(radians(t), [10000.0 ** (-2 * i / 128) for i in range(64)], rtol=1e-14)
    np.testing.assert_allclose(radians(lt.rotary_table(64, kind="linear", factor=4.0)), [10000.0 ** (-2 * i / 64) / 4 for i in range(32)], rtol=1e-14)
    stretched = radians(lt.rotary_table(64, kind="base", factor=8.0))
    np.testing.assert_allclose(stretched, [(10000.0 * 8 ** (64 / 62)) ** (-2 * i / 64) for i in range(32)], rtol=1e-13)
    np.testing.assert_allclose(stretched[-1], 10000.0 ** (-62 / 64) / 8, rtol=1e-12)  # the slowest pair is stretched by the factor
    parts = radians(lt.rotary_table(128, base=500000.0, kind="parts", factor=8.0, original_length=8192, low=1.0, high=4.0))
    plain = [500000.0 ** (-2 * i / 128) for i in range(64)]
    for got, f in zip(parts, plain):
        turns = 8192 * f / (2 * math.pi)
        keep = min(1, max(0, (turns - 1) / 3))
        assert got == pytest.approx(f * (keep + (1 - keep) / 8), rel=1e-13)
    # an angle far out: position x frequency modulo 2^64 is the exact fraction of a turn
    p = 123456789
    f = int(t[1, 1]) << 32 | int(t[1, 0])
    assert ((p * f) % (1 << 64)) / 2.0 ** 64 == pytest.approx((p * 10000.0 ** (-2 / 128) / (2 * math.pi)) % 1.0, abs=1e-7)
    for bad in (dict(rotated=3), dict(rotated=0), dict(rotated=4, kind="none such"), dict(rotated=4, base=-1.0), dict(rotated=4, kind="linear", factor=0.0), dict(rotated=4, kind="parts"),
                dict(rotated=2, kind="base", factor=2.0)):
        with pytest.raises(ValueError):
            lt.rotary_table(**bad)
