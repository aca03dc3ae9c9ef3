"""The operators around a block's attention at the ends of their ranges: rotary calls whose wavefronts take several
turns, and every scale of a 4-bit float in values and products.  Tolerances of rotations and norms are those of
test_gpu_operators.py; the others count roundings where they stand."""
import numpy as np
import pytest
import torch

import test_gpu_operators as ops
from oracle import operators_oracle as orc
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import harness

pytestmark = pytest.mark.gpu

# A launch of agg_rope_fwd has at most 4096 workgroups of four wavefronts, and a wavefront's turn is this many tokens
# (two from four heads on, except in calls of up to 4096 tokens).
ROPE_WAVES = 4096 * 4


def turn_tokens(H):
    return 8 // H if H < 4 else 2


# (heads, norm, pairing, channels of the axes, frames or tokens, grid of a frame; no grid: given positions)
TURNS = [(1, "layer", agg.AGG_ROPE_SECTIONS, (0, 32, 32), 2801, (13, 11, 5)),
         (1, "rms", agg.AGG_ROPE_HEAD, (16, 24, 20), 400_003, None),
         (3, "rms", agg.AGG_ROPE_NEIGHBOURS, (16, 24, 20), 99_001, None),
         (3, "none", agg.AGG_ROPE_SECTIONS, (0, 20, 32), 701, (13, 11, 4)),
         (5, "layer", agg.AGG_ROPE_HEAD, (16, 24, 20), 701, (13, 11, 4)),
         (7, "layer", agg.AGG_ROPE_SECTIONS, (16, 24, 24), 98_401, None),
         (8, "none", agg.AGG_ROPE_NEIGHBOURS, (0, 30, 20), 701, (13, 11, 4)),
         (16, "rms", agg.AGG_ROPE_HEAD, (16, 24, 24), 98_403, None)]


@pytest.mark.parametrize("H, kind, pairing, axes, N, grid", TURNS)
def test_rope_several_turns_of_a_wavefront(H, kind, pairing, axes, N, grid):
    """Three turns and more for every wavefront, the last one partial: the bits of calls on parts, in place too, and
    the oracle's values at tokens from all over."""
    ops.say("rope turns", H, kind, pairing, axes, N, grid)
    L = 1 if grid is None else grid[0] * grid[1] + grid[2]
    total = N * L
    assert total > 3 * ROPE_WAVES * turn_tokens(H) and total % turn_tokens(H) != 0
    g = ops.gen(H + N)
    q, k = (ops.normal(g, total, H, 64).mul_(s).to(torch.bfloat16) for s in (1.5, 3.0))
    (qn, qs), (kn, ks) = (ops.make_norm(g, kind, 64) for _ in "qk")
    pos = None
    if grid is None:
        pos = torch.randint(-5000, 5000, (total, 3), generator=g, device="cuda", dtype=torch.int32)

    def run(first, count, in_place=False):  # of frames, or of tokens where there is no grid
        part = slice(first * L, (first + count) * L)
        a, b = (t[part].clone() for t in (q, k))
        rope = agg.make_rope(pairing, *axes, t0=0 if pos is not None else first, patch0=1)
        n_h, n_w, P = grid or (1, 1, 0)
        shape = agg.make_shape(1, count, n_h, n_w, P, H, 64, 1, 1)
        p = None if pos is None else pos[part].contiguous()
        if in_place:
            agg.agg_rope_fwd(shape, rope, qn, kn, p, a, 0, b, 0, a, b)
            return a, b
        return [t.view(-1, H, 64) for t in harness.rope_forward(shape, rope, a, b, qn, kn, p)]

    whole = run(0, N)
    for t, v in zip(run(0, N, True), whole):
        assert ops.same_bits(t, v)
    step = -(-N // 5)  # parts of at most a turn for every wavefront
    assert step * L <= ROPE_WAVES * turn_tokens(H)
    for first in range(0, N, step):
        count = min(step, N - first)
        for t, v in zip(run(first, count), whole):
            assert ops.same_bits(t, v[first * L:(first + count) * L]), first
    some = np.unique(np.concatenate([np.arange(40), total - 1 - np.arange(40),
                                     np.random.default_rng(H).integers(0, total, 400)]))
    if pos is not None:
        at = pos.cpu().numpy()[some].astype(np.int64)
    else:
        at = orc.grid_positions(N, *grid, 0, 1)[some]
    for t, r, spec, name in zip((q, k), whole, (qs, ks), "qk"):
        raw = ops.f64(t[torch.tensor(some, device="cuda")])
        x = orc.norm(raw, *spec)
        want = orc.rope(x, at, pairing, axes, 100.0)
        size, err = np.abs(x), np.broadcast_to(ops.norm_error(raw, spec), x.shape).copy()
        for a, b, _, _ in orc.rope_pairs(pairing, axes, 100.0):
            size[..., a] = size[..., b] = size[..., a] + size[..., b]
            err[..., a] = err[..., b] = err[..., a] + err[..., b]
        ops.within(r[torch.tensor(some, device="cuda")], want, ops.HALF * np.abs(want) + 1e-6 * size + err, name)


# ---- 4-bit floats --------------------------------------------------------------------------------
def matrix(codes, scales, K):
    """codes [rows, K], scales [rows, blocks] as they are held."""
    rows, blocks = len(codes), -(-K // 32)
    full = np.zeros((rows, blocks * 32), dtype=np.int64)
    full[:, :K] = codes
    held = orc.pack(full.reshape(rows, blocks, 32), scales, -(-K // 256) * 128, -(-K // 512) * 16)
    return [torch.tensor(t, device="cuda") for t in held]


def test_every_code_of_every_scale_reads_back():
    """Bytes that no quantisation leaves among them: the smallest values are bf16 subnormals, the largest infinite."""
    ops.say("mx4 every scale")
    codes = np.tile(np.concatenate([np.arange(16), np.arange(15, -1, -1)]), (256, 2))
    scales = np.stack([np.arange(256), np.arange(255, -1, -1)], 1)
    held = matrix(codes, scales, 64)
    got = harness.mx4_dequantize(held, 64).cpu()
    want = torch.tensor(orc.values(*(t.cpu().numpy() for t in held), 64)).float().to(torch.bfloat16)
    nan = torch.isnan(want)
    assert torch.isinf(want).any() and nan.sum() == 64 and (want[0, 1] != 0)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])


# rows that lead to each kernel for 256 channels (test_operator_plan.py: the rule; here by its figures)
SCALE_ROWS = [("few", 256, 32), ("tiles of 64", 1024, 32), ("tiles of 128", 256 * 70, 32), ("tiles of 128, many", 256 * 260, 32),
              ("tiles of 256", 256 * 256, 1056), ("panel", 256 * 1024, 32), ("panel of long rows", 256 * 1024, 520)]


@pytest.mark.parametrize("kernel, rows, K", SCALE_ROWS)
def test_products_of_every_pair_of_scales(kernel, rows, K):
    """Every scale against every other in one block of 32 channels, all others zero.  Of codes without signs a block's
    sum is a multiple of 1/4 below 2^11, so a result is exact in float32 and rounded once, down to where float32 has
    no normal numbers: there it may be off by their smallest, 2^-126."""
    ops.say("product of scales", kernel, rows, K)
    rng = np.random.default_rng(rows + K)
    block = (K - 1) // 32  # the last one, of 32 or of 8 channels
    here = K - 32 * block

    def operand(seed):
        codes = np.zeros((256, K), dtype=np.int64)
        codes[:, 32 * block:] = rng.integers(0, 8, (256, here))
        scales = np.full((256, block + 1), 127)
        scales[:, block] = np.arange(256)
        return matrix(codes, scales, K)

    a, w = operand(0), operand(1)
    av, wv = (orc.values(*(t.cpu().numpy() for t in m), K)[:, 32 * block:] for m in (a, w))
    want = torch.tensor(av @ wv.T).cuda()
    many = [t.repeat(rows // 256, 1) for t in a]
    out, = harness.mx4_linear(many, [w], K)
    out = out.view(-1, 256, 256)
    assert all(ops.same_bits(out[i], out[0]) for i in (0, len(out) // 2, len(out) - 1))
    assert bool((out.view(torch.int16) == out[0].view(torch.int16)).all())
    got, exact = out[0], want.float().to(torch.bfloat16)
    nan = torch.isnan(want)
    assert nan[255].all() and nan[:, 255].all() and nan.sum() == 511 and torch.equal(torch.isnan(got), nan)
    normal = ~nan & (want >= 2.0 ** -126)
    assert torch.equal(got[normal], exact[normal])
    small = ~nan & ~normal
    assert ((got.double() - want).abs() <= 2.0 ** -126)[small].all()
