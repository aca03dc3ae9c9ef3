"""Calls whose rows or (sequence, head) pairs would take 2^32 threads or more in one launch.  Such a launch runs only
what is left of its threads modulo 2^32 and reports nothing, so these calls have to go out in parts, or be refused."""
import pytest
import torch

import test_gpu_operators as ops
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import harness, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mx", [False, True])
def test_block_of_more_rows_than_a_launch_counts(mx):
    """2^26 rows and some, one head: a norm that gave every row a wavefront in one launch would have 2^32 threads.
    Frames repeat every 15, which the parts of a launch do not: results have to repeat with them, to the bit."""
    ops.say("block of many rows", mx)
    period, N, L = 15, (1 << 16) + 1, 1024
    shape = agg.make_shape(1, N, 32, 32, 0, 1, 64, 1, 1)
    wts = inputs.block_weights(64, seed=49, device="cuda")
    some = inputs.block_input(1, period * L, 64, seed=49, device="cuda").view(period, L * 64)
    x = some.repeat(-(-N // period), 1)[:N].contiguous().view(1, N * L, 64)
    ms = [harness.mx4_quantize(wts["w_" + n]) for n in "qkvo"] if mx else None
    y, _ = harness.block_ex_forward(shape, agg.AGG_BLOCK_FRAME, wts, agg.make_block_options(mx=ms), x)
    y = y.view(N, L * 64)
    first = y[:period].clone()
    assert torch.isfinite(first).all() and not ops.same_bits(first, some)
    for i in range(0, N, 300 * period):
        part = y[i:i + 300 * period]
        want = first.repeat(300, 1)[:len(part)]
        assert ops.same_bits(part, want), i
