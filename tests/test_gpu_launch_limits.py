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


def test_frames_of_one_token_beyond_a_launch():
    """2^24 frames and some, of one token, one head: a key's only query returns its value, and its logit.
    lse: the kernel multiplies q * scale * log2(e) rounded to bf16, which moves each of the 64 products by up to 2^-8 of
    its magnitude; their float32 sum and the way to and from base 2 are under 2^-16 of the magnitudes and 1; the weight,
    rounded to bf16, is off by 2^-8 of itself at most, which is as much in its logarithm."""
    ops.say("frames of one token")
    N = (1 << 24) + 9
    shape = agg.make_shape(1, N, 1, 1, 0, 1, 64, 1, 1)
    g = ops.gen(50)
    q, k, v = (torch.randn((1, N, 1, 64), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "qkv")
    out = harness._buf((1, N, 1, 64), torch.bfloat16, q.device, "O")
    lse = harness._buf((1, N), torch.float32, q.device, "lse")
    out.view(torch.int16).fill_(0x7FC1)
    lse.fill_(float("nan"))
    agg.agg_frame_attn_fwd(shape, q, k, v, out, lse)
    assert ops.same_bits(out, v)
    for at in range(0, N, 1 << 22):
        part = slice(at, min(N, at + (1 << 22)))
        both = q[0, part, 0].double() * k[0, part, 0].double() / 8
        want, size = both.sum(-1), both.abs().sum(-1)
        assert ((lse[0, part].double() - want).abs() <= 1.01 * 2.0 ** -8 + 2.0 ** -8 * size + 2.0 ** -16 * (size + 1)).all(), at


def test_frames_of_some_heads_beyond_a_launch():
    """The same number of pairs as frames of two tokens and several heads of two sequences: what the parts return."""
    ops.say("frames of two tokens")
    B, N, H = 2, 1 << 20, 9
    shape = agg.make_shape(B, N, 1, 2, 0, H, 64, 1, 1)
    g = ops.gen(51)
    q, k, v = (torch.randn((B, 2 * N, H, 64), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "qkv")
    assert B * N * H > 1 << 24
    out, _ = harness.frame_forward(shape, q, k, v)
    part = agg.make_shape(1, 1 << 18, 1, 2, 0, H, 64, 1, 1)
    for b in range(B):
        for at in range(0, 2 * N, 1 << 19):
            rows = slice(at, at + (1 << 19))
            want, _ = harness.frame_forward(part, q[b:b + 1, rows], k[b:b + 1, rows], v[b:b + 1, rows])
            assert ops.same_bits(out[b:b + 1, rows], want), (b, at)


def test_selection_beyond_a_launch():
    """2^26 kept tokens and some, by the grid rule: the host's own list."""
    ops.say("selection of many")
    shape = agg.make_shape(1, (1 << 22) + 1, 8, 8, 0, 1, 64, 2, 2, 0)
    M, _ = agg.agg_kv_count(shape)
    assert M > 1 << 26
    got = harness._buf((M,), torch.int32, torch.device("cuda"), "list")
    got.fill_(-1)
    agg.agg_select_kv_indices(shape, agg.AGG_SELECT_FIRST, 0, None, got)
    assert torch.equal(got.cpu(), torch.from_numpy(agg.agg_kv_indices_host(shape)))


def test_means_beyond_a_launch_are_refused():
    """A workgroup for each of 2^24 sequences and one: an error, and nothing is launched."""
    ops.say("means of many sequences")
    B = (1 << 24) + 1
    shape = agg.make_shape(B, 2, 1, 2, 0, 1, 64, 1, 2, 1)
    k = torch.empty((B, 4, 1, 64), dtype=torch.bfloat16, device="cuda")
    means = torch.empty((2, B, 64), dtype=torch.float32, device="cuda")
    size = agg.agg_workspace_bytes(shape)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    with pytest.raises(agg.AggError) as e:
        agg.agg_kv_subsample(shape, k, k, None, None, None, means[0], means[1], ws, size)
    assert e.value.status == agg.AGG_ERR_LAUNCH
