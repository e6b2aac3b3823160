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
