"""The vocabulary loss and its gradients where sums are long, weights differ widely, rows are wide or a wait gives up."""
import math
import time

import pytest
import torch

import table_reference as ref
from operator_reference import HALF, TYPES, ULP, close
from test_gpu_operators import ctx, fetch, gen, lt, normal, unaligned  # noqa: F401
from test_gpu_table_operators import tokens_of

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
