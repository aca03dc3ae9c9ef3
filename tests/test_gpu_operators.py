"""The operators around a block's attention on the GPU, through the C ABI, against the float64 oracle.

Tolerances count roundings.  A bf16 result is off by at most half a step, 2^-8 of its value, plus the
float32 error in front of that rounding:
  rotation   an angle is good to 2^-25 turns (the float of its reduced turns) + 2 ulp of the sine: under
             6e-7; with three roundings of 2^-24 each, 1e-6 of |x| + |y| of the pair
  norms      sums of up to 8192 values in a tree of lanes: at most 7 + 128 roundings of 2^-24 each one
             after another in a lane, under 2^-16 of the sum of magnitudes; the mean's error counts
             against the largest |x|, the scale's against the value.  2^-15 (max|x - mean| / sigma |gamma| + |beta|) covers both
             where |mean| <= 8 sigma, which the inputs keep
  products   4-bit products and their scales are exact; one rounding of 2^-24 of the magnitudes per 128
             channels, counted twice for the adder's own width, and three for bias, scale, residual
"""
import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import harness, inputs

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
NORMS = {"none": agg.AGG_NORM_NONE, "layer": agg.AGG_NORM_LAYER, "rms": agg.AGG_NORM_RMS}


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def same_bits(a, b):
    return torch.equal(a.view(torch.int16), b.view(torch.int16))


def within(got, want, tol, what):
    got = f64(got)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%s: %d off, worst %.3g of the tolerance" % (
        what, bad.sum(), np.nanmax(np.abs(got - want) / np.maximum(tol, 1e-300)))


def make_norm(g, kind, C, affine=True):
    gamma = 1 + 0.3 * normal(g, C) if affine else None
    beta = 0.3 * normal(g, C) if affine else None
    return agg.make_norm(NORMS[kind], 1e-5, gamma, beta), (NORMS[kind], float(np.float32(1e-5)), f64(gamma), f64(beta))


def norm_error(x, spec):
    """What float32 may lose of a norm, by value (see above)."""
    kind, eps, gamma, beta = spec
    if kind == agg.AGG_NORM_NONE:
        return np.zeros_like(x)
    d = x - x.mean(-1, keepdims=True) if kind == agg.AGG_NORM_LAYER else x
    top = np.abs(d).max(-1, keepdims=True) / np.sqrt((d * d).mean(-1, keepdims=True) + eps)
    return 2.0 ** -15 * (top * (1 if gamma is None else np.abs(gamma)) + (0 if beta is None else np.abs(beta)))


# ---- rotary positions ----------------------------------------------------------------------------
def rope_case(shape, pairing, axes, kind="none", base=100.0, t0=0, patch0=0, pos=None, seed=1, affine=True):
    B, NQ, H = shape.B, shape.NQ, shape.H
    g = gen(seed)
    q, k = (normal(g, B, NQ, H, 64).mul_(s).to(torch.bfloat16) for s in (1.5, 3.0))
    rope = agg.make_rope(pairing, *axes, base=base, t0=t0, patch0=patch0)
    norms = [make_norm(g, kind, 64, affine) for _ in "qk"]
    dev_pos = None if pos is None else torch.tensor(pos, dtype=torch.int32, device="cuda")
    out = harness.rope_forward(shape, rope, q, k, norms[0][0], norms[1][0], dev_pos)
    torch.cuda.synchronize()
    if pos is None:
        at = np.tile(orc.grid_positions(shape.N, shape.n_h, shape.n_w, shape.n_special, t0, patch0), (B, 1))
    else:
        at = np.asarray(pos).reshape(-1, 3)
    # far positions: a float64 angle would lose 2^-53 of itself, up to 2^31 of them: 2.4e-7
    for t, r, (_, spec), name in zip((q, k), out, norms, "qk"):
        x = orc.norm(f64(t).reshape(B * NQ, H, 64), *spec)
        want = orc.rope(x, at, pairing, axes, float(np.float32(base)))
        err = norm_error(f64(t).reshape(B * NQ, H, 64), spec)
        size, err = np.abs(x), np.broadcast_to(err, x.shape).copy()
        for a, b, _, _ in orc.rope_pairs(pairing, axes, base):
            size[..., a] = size[..., b] = size[..., a] + size[..., b]
            err[..., a] = err[..., b] = err[..., a] + err[..., b]
        within(r.view(B * NQ, H, 64), want, HALF * np.abs(want) + 1e-6 * size + err, name)
    return q, k, out, rope, norms, dev_pos


PAIRINGS = [agg.AGG_ROPE_SECTIONS, agg.AGG_ROPE_NEIGHBOURS, agg.AGG_ROPE_HEAD]


@pytest.mark.parametrize("pairing", PAIRINGS)
@pytest.mark.parametrize("axes", [(0, 32, 32), (16, 24, 24), (64, 0, 0), (0, 0, 2), (20, 22, 14), (0, 0, 0)])
def test_rope_pairings_and_axes(pairing, axes):
    say("rope", pairing, axes)
    shape = agg.make_shape(2, 3, 5, 7, 3, 4, 64, 1, 1)
    rope_case(shape, pairing, axes, "layer", t0=-5, patch0=1)


@pytest.mark.parametrize("kind", ["none", "layer", "rms"])
@pytest.mark.parametrize("H", [1, 2, 3, 4, 5, 7, 8, 12, 16, 33])
def test_rope_heads_and_norms(H, kind):
    say("rope heads", H, kind)
    shape = agg.make_shape(1, 2, 3, 3, 2, H, 64, 1, 1)
    rope_case(shape, agg.AGG_ROPE_SECTIONS, (16, 24, 24), kind, patch0=1, affine=H != 5)


@pytest.mark.parametrize("N, n_h, n_w, P", [(1, 1, 1, 0), (1, 1, 1, 1), (1, 1, 1, 5), (2, 1, 9, 0), (17, 2, 1, 4),
                                            (1, 37, 37, 5)])
def test_rope_lengths(N, n_h, n_w, P):
    say("rope lengths", N, n_h, n_w, P)
    rope_case(agg.make_shape(3, N, n_h, n_w, P, 2, 64, 1, 1), agg.AGG_ROPE_HEAD, (16, 24, 24), "rms", 10000.0, 7)


def test_rope_many_tokens():
    """More turns than wavefronts: every wavefront takes several."""
    say("rope many")
    rope_case(agg.make_shape(1, 40, 37, 37, 5, 1, 64, 1, 1), agg.AGG_ROPE_SECTIONS, (0, 32, 32), "layer")
    rope_case(agg.make_shape(1, 40, 37, 37, 5, 4, 64, 1, 1), agg.AGG_ROPE_SECTIONS, (0, 32, 32))


@pytest.mark.parametrize("base", [1.0, 100.0, 10000.0, 3.0e38])
def test_rope_far_positions(base):
    say("rope far", base)
    shape = agg.make_shape(1, 2, 2, 2, 1, 2, 64, 1, 1)
    pos = [[2 ** 31 - 1, 0, 1], [-2 ** 31, 5, -1], [10 ** 9, -10 ** 9, 0], [123456789, 987654321, 1], [0, 0, 0],
           [1 << 20, 1 << 24, 1 << 30], [-1, -2, -3], [3, 2, 1], [65535, 65536, 65537], [5, 5, 5]]
    rope_case(shape, agg.AGG_ROPE_HEAD, (32, 16, 16), pos=[pos], base=base)
    rope_case(shape, agg.AGG_ROPE_NEIGHBOURS, (32, 16, 16), "rms", base=base, t0=2 ** 31 - 3, patch0=-2 ** 31)


def test_rope_given_positions_are_the_grid():
    say("rope given")
    shape = agg.make_shape(2, 3, 4, 5, 2, 8, 64, 1, 1)
    at = np.tile(orc.grid_positions(3, 4, 5, 2, 9, 1), (2, 1, 1)).reshape(2, -1, 3)
    a = rope_case(shape, agg.AGG_ROPE_SECTIONS, (0, 32, 32), "layer", t0=9, patch0=1)
    b = rope_case(shape, agg.AGG_ROPE_SECTIONS, (0, 32, 32), "layer", pos=at)
    assert all(same_bits(x, y) for x, y in zip(a[2], b[2]))


def test_rope_in_place_strided_and_alone():
    say("rope in place, strided, alone")
    shape = agg.make_shape(2, 3, 5, 7, 3, 6, 64, 1, 1)
    C = 6 * 64
    q, k, (rq, rk), rope, ((qn, _), (kn, _)), _ = rope_case(shape, agg.AGG_ROPE_SECTIONS, (16, 24, 24), "layer")
    # one tensor at a time
    only, none = harness.rope_forward(shape, rope, q, None, qn, None)
    assert none is None and same_bits(only, rq)
    none, only = harness.rope_forward(shape, rope, None, k, None, kn)
    assert none is None and same_bits(only, rk)
    # out of the rows of a fused projection, with a ragged end
    fused = torch.full((2 * shape.NQ, 3 * C + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
    fused[:, :C], fused[:, C:2 * C] = q.view(-1, C), k.view(-1, C)
    out = harness.rope_forward(shape, rope, fused, fused[:, C:], qn, kn, None, 3 * C + 8, 3 * C + 8)
    assert same_bits(out[0], rq) and same_bits(out[1], rk)
    # in place
    a, b = q.clone(), k.clone()
    agg.agg_rope_fwd(shape, rope, qn, kn, None, a, 0, b, 0, a, b)
    assert same_bits(a, rq) and same_bits(b, rk)
    # neither a rotation nor a norm: a copy, whatever the bits
    odd = torch.arange(-32768, 32767, 1, dtype=torch.int32, device="cuda").to(torch.int16)[:2 * shape.NQ * C]
    odd = odd.repeat(-(-2 * shape.NQ * C // odd.numel()))[:2 * shape.NQ * C].view(torch.bfloat16).view(q.shape)
    finite = torch.where(torch.isnan(odd), torch.zeros_like(odd), odd).contiguous()
    out = harness.rope_forward(shape, None, finite, finite)
    assert same_bits(out[0], finite) and same_bits(out[1], finite)


def test_rope_leaves_the_other_channels():
    """Infinities and NaN stay where they are: behind the axes' channels and in their own pair."""
    say("rope other channels")
    shape = agg.make_shape(1, 1, 3, 3, 0, 2, 64, 1, 1)
    q = normal(gen(5), 1, 9, 2, 64).to(torch.bfloat16)
    q[0, :, 0, 40], q[0, :, 1, 63], q[0, :, 0, 5] = float("inf"), float("-inf"), float("nan")
    out, _ = harness.rope_forward(shape, agg.make_rope(agg.AGG_ROPE_SECTIONS, 0, 16, 16), q, None)
    assert same_bits(out[..., 32:].contiguous(), q[..., 32:].contiguous())
    nan = torch.isnan(out)
    assert nan[0, :, 0, [5, 13]].all() and nan.sum() == 18


# ---- the seam between branches -------------------------------------------------------------------
@pytest.mark.parametrize("H", [1, 3, 8, 12, 16, 33, 64])
@pytest.mark.parametrize("both", [True, False])
def test_rope_shared_out_heads(H, both):
    """However many wavefronts share a token's heads: the same bits, for few tokens as for many, in place too."""
    say("rope shared heads", H, both)
    g = gen(47)
    total = 5003
    q, k = (normal(g, 1, total, H, 64).to(torch.bfloat16) for _ in "qk")
    pos = torch.randint(-1000, 1000, (1, total, 3), generator=g, device="cuda", dtype=torch.int32)
    n = make_norm(g, "layer", 64)[0]
    rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 16, 24, 20)

    def run(part):
        a, b = (t[:, part].contiguous() for t in (q, k))
        shape = agg.make_shape(1, a.shape[1], 1, 1, 0, H, 64, 1, 1)
        agg.agg_rope_fwd(shape, rope, n, n, pos[:, part].contiguous(), a, 0, b if both else None, 0, a,
                         b if both else None)
        return (a, b) if both else (a,)

    whole = run(slice(0, total))
    for first, size in ((0, 1), (7, 2), (1, 61), (100, 128), (90, 129), (0, 512), (3, 513), (5, 1024), (4, 1025), (0, 2048),
                        (1, 2049), (907, 4096)):
        part = slice(first, first + size)
        for t, v in zip(run(part), whole):
            assert same_bits(t, v[:, part]), (first, size)


def seam_case(rows, C, post="none", pre="layer", scale=True, gate_rows=0, branch=True, want_h=True, seed=3,
              affine=True):
    g = gen(seed)
    x = (normal(g, rows, C) * torch.exp(0.5 * normal(g, C))).to(torch.bfloat16)
    b = (2 * normal(g, rows, C) + 0.5).to(torch.bfloat16) if branch else None
    post_n, post_s = make_norm(g, post, C, affine)
    pre_n, pre_s = make_norm(g, pre, C, affine)
    s = 0.5 * normal(g, C) if scale else None
    gate = normal(g, -(-rows // gate_rows), C).to(torch.bfloat16) if gate_rows else None
    r = agg.make_residual(post_n, pre_n, s, gate, gate_rows)
    h, n = harness.residual_forward(r, x, b, want_h)
    torch.cuda.synchronize()
    want_hh, want_n = orc.seam(f64(x), f64(b), post_s, pre_s, f64(s), f64(gate), gate_rows)
    size, err = np.abs(f64(x)), 0.0
    if branch:
        factor = np.ones((rows, C)) if s is None else np.abs(f64(s)) * np.ones((rows, C))
        if gate is not None:
            factor = factor * np.abs(f64(gate))[np.arange(rows) // gate_rows]
        y = orc.norm(f64(b), *post_s)
        size = size + factor * np.abs(y)
        err = factor * norm_error(f64(b), post_s)
    err = err + 2.0 ** -22 * size  # two products and a sum
    if want_h:
        within(h, want_hh, HALF * np.abs(want_hh) + err, "h")
    if n is not None:
        # an error of h reaches n divided by the deviation, through the value, the mean and the deviation itself
        d = want_hh - want_hh.mean(-1, keepdims=True) if pre == "layer" else want_hh
        sigma = np.sqrt((d * d).mean(-1, keepdims=True) + 1e-5)
        worst = np.broadcast_to(err, want_hh.shape).max(-1, keepdims=True) / sigma
        through = (np.broadcast_to(err, want_hh.shape) / sigma + worst * (1 + np.abs(d) / sigma))
        gamma = 1 if pre_s[2] is None else np.abs(pre_s[2])
        within(n, want_n, HALF * np.abs(want_n) + norm_error(want_hh, pre_s) + through * gamma, "n")
    return r, x, b, h, n


@pytest.mark.parametrize("pre", ["none", "layer", "rms"])
@pytest.mark.parametrize("post", ["none", "layer", "rms"])
@pytest.mark.parametrize("scale, gate_rows", [(False, 0), (True, 0), (False, 1), (True, 5)])
def test_residual_parts(post, pre, scale, gate_rows):
    say("residual", post, pre, scale, gate_rows)
    seam_case(23, 1024, post, pre, scale, gate_rows)


@pytest.mark.parametrize("C", [8, 16, 64, 504, 512, 520, 1024, 1032, 2048, 2056, 2112, 4096, 4104, 8192])
def test_residual_widths(C):
    say("residual width", C)
    seam_case(9, C, "rms", "layer", True, 4)
    seam_case(3, C, "none", "rms", False, 0, affine=False)


@pytest.mark.parametrize("C", [1032, 1536, 1544, 2048, 2056, 2112, 2560, 2568, 3064, 3584, 3592, 4088, 4096, 4104])
def test_residual_long_rows(C):
    """More rows than few, a wavefront each with the parameters in LDS: every width of 512 channels, its ends,
    and the most parameters that there can be."""
    say("residual long rows", C)
    seam_case(1003, C, "layer", "layer", True, 261)
    seam_case(897, C, "none", "rms", False, 0, affine=False)
    seam_case(2501, C, "rms", "none", True)


@pytest.mark.parametrize("rows", [896, 897])
def test_residual_parts_of_long_rows(rows):
    say("residual parts of long rows", rows)
    for post, pre, branch, want_h in (("none", "layer", False, True), ("none", "rms", False, False),
                                      ("layer", "none", True, True), ("none", "none", True, True)):
        seam_case(rows, 1032, post, pre, branch, 5 if branch else 0, branch, want_h)


@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 261, 4099, 20011])
def test_residual_rows(rows):
    say("residual rows", rows)
    seam_case(rows, 192, "layer", "rms", True, 261)
    seam_case(rows, 1024, "none", "layer")


def test_residual_without_branch_or_sum():
    say("residual without branch, without h")
    seam_case(37, 1024, scale=False, branch=False)
    seam_case(37, 1024, scale=False, branch=False, want_h=False)
    seam_case(37, 1024, "rms", "layer", want_h=False)


def test_residual_gate_longer_than_the_rows():
    say("residual one gate for all rows")
    seam_case(11, 256, gate_rows=10 ** 15)


def test_residual_in_place():
    say("residual in place")
    r, x, b, h, n = seam_case(531, 1024, "rms", "layer", True, 100)
    for hh, nn in (("x", "b"), ("b", "x"), ("x", None), (None, "x"), (None, "b")):
        a, c = x.clone(), b.clone()
        ho = {"x": a, "b": c, None: torch.empty_like(x)}[hh]
        no = {"x": a, "b": c, None: torch.empty_like(x)}[nn]
        agg.agg_residual_norm_fwd(531, 1024, r, a, c, ho, no)
        assert same_bits(ho, h) and same_bits(no, n), (hh, nn)


def test_residual_rows_that_are_not_finite():
    """A row with an infinity, a row of one value, a row of zeros: their own results, nobody else's."""
    say("residual special rows")
    g = gen(8)
    x, b = (normal(g, 6, 512).to(torch.bfloat16) for _ in "xb")
    r = agg.make_residual(pre=agg.make_norm(agg.AGG_NORM_LAYER, 1e-5))
    _, clean = harness.residual_forward(r, x, b)
    x[1, 7] = float("inf")
    x[2], b[2] = 3.0, 1.0
    x[3], b[3] = 0.0, 0.0
    x[4, 0] = float("nan")
    h, n = harness.residual_forward(r, x, b)
    assert torch.isnan(n[1]).any() and torch.isnan(n[4]).all() and torch.isinf(h[1, 7])
    assert (h[2] == 4).all() and (n[2] == 0).all() and (h[3] == 0).all() and (n[3] == 0).all()
    assert same_bits(n[[0, 5]], clean[[0, 5]])


# ---- 4-bit floats --------------------------------------------------------------------------------
def held(x, K=None):
    """The oracle's packed bytes of a bf16 matrix on the host."""
    v = f64(x)[:, :K]
    K = v.shape[1]
    return orc.pack(*orc.quantize(v), -(-K // 256) * 128, -(-K // 512) * 16)


def quantize_case(x, K=None):
    K = K or x.shape[1]
    codes, scales = harness.mx4_quantize(x, K)
    back = harness.mx4_dequantize((codes, scales), K)
    c, s = held(x, K)
    assert (codes.cpu().numpy() == c).all() and (scales.cpu().numpy() == s).all()
    want = torch.tensor(orc.values(c, s, K)).to(torch.bfloat16)  # exact
    got = back.cpu()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    return codes, scales


@pytest.mark.parametrize("K", [8, 16, 24, 32, 40, 64, 96, 248, 256, 264, 512, 520, 1024, 1032, 2112, 4096, 8256])
@pytest.mark.parametrize("rows", [1, 5, 67])
def test_mx4_quantize(rows, K):
    say("mx4", rows, K)
    g = gen(K + rows)
    x = (normal(g, rows, K) * torch.exp(3 * normal(g, rows, 1))).to(torch.bfloat16)
    quantize_case(x)


def test_mx4_every_value_against_every_scale():
    """Blocks that hold one large value, which sets the scale, and every smaller bf16 beside it."""
    say("mx4 all values")
    bits = torch.arange(0, 0x7F80, dtype=torch.int32)  # every finite magnitude
    signed = torch.cat((bits, bits | 0x8000))
    for top in (0x0000, 0x0001, 0x0080, 0x00FF, 0x0100, 0x017F, 0x0180, 0x01C0, 0x3F80, 0x3FC0, 0x3FFF, 0x7F00, 0x7F7F):
        ok = signed[(signed & 0x7FFF) <= top]
        if ok.numel() > 12000:  # those near the largest in full, a sample of the far smaller ones
            near = ok[(ok & 0x7FFF) > top - 0x300]
            ok = torch.cat((near, ok[::max(1, ok.numel() // 8000)]))
        rest = torch.zeros(-(-ok.numel() // 31) * 31, dtype=torch.int32)
        rest[:ok.numel()] = ok
        block = torch.cat((torch.full((rest.numel() // 31, 1), top, dtype=torch.int32), rest.view(-1, 31)), 1)
        x = torch.where(block > 32767, block - 65536, block).to(torch.int16).view(torch.bfloat16).cuda()
        quantize_case(x)


def test_mx4_broken_and_empty_blocks():
    say("mx4 broken blocks")
    x = normal(gen(9), 8, 104).to(torch.bfloat16)
    x[0, 3], x[1, 40], x[2, 99] = float("inf"), float("nan"), float("-inf")
    x[3] = 0.0
    x[4, :32] = -0.0
    x[5] = 2.0 ** -133
    x[6] = 3.3e38
    codes, scales = quantize_case(x)
    assert scales[0, 0] == scales[1, 1] == scales[2, 3] == 255 and scales[3, :4].sum() == 0


def test_mx4_long_rows_and_strides():
    say("mx4 strides")
    x = normal(gen(10), 301, 1536).to(torch.bfloat16)
    a = quantize_case(x, 1000)
    b = harness.mx4_quantize(x[:, :1000].contiguous())
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    quantize_case(normal(gen(11), 20011, 64).to(torch.bfloat16))


# ---- products ------------------------------------------------------------------------------------
def product_case(rows, N, K, count=1, bias=True, residual=False, res_scale=True, seed=5, spread=1.0):
    g = gen(seed)
    x = (normal(g, rows, K) * torch.exp(spread * normal(g, rows, 1))).to(torch.bfloat16)
    a = harness.mx4_quantize(x)
    ws = [harness.mx4_quantize((normal(g, N, K) * K ** -0.5).to(torch.bfloat16)) for _ in range(count)]
    bs = [normal(g, N) if bias else None for _ in range(count)]
    res = normal(g, rows, N).to(torch.bfloat16) if residual else None
    rs = normal(g, N) if residual and res_scale else None
    out = harness.mx4_linear(a, ws, K, bs, res, rs)
    torch.cuda.synchronize()
    av = orc.values(*(t.cpu().numpy() for t in a), K)
    for i in range(count):
        wv = orc.values(*(t.cpu().numpy() for t in ws[i]), K)
        want, size = orc.linear(av, wv, f64(bs[i]), f64(res), f64(rs))
        tol = HALF * np.abs(want) + (2 * -(-K // 128) + 4) * 2.0 ** -24 * size
        within(out[i], want, tol, "product %d" % i)
    return a, ws, bs, res, rs, out


@pytest.mark.parametrize("rows", [1, 2, 7, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300])
def test_product_rows(rows):
    say("product rows", rows)
    product_case(rows, 192, 320, 1, True, rows % 2 == 0)


@pytest.mark.parametrize("N", [8, 16, 40, 64, 72, 120, 128, 136, 256, 264, 320, 1000])
@pytest.mark.parametrize("rows", [3, 150])
def test_product_channels(rows, N):
    say("product channels", rows, N)
    product_case(rows, N, 256, 3 if N % 16 else 2)
    product_case(rows, N, 256, 1, False, True)


@pytest.mark.parametrize("K", [8, 24, 32, 64, 120, 128, 136, 192, 256, 264, 384, 512, 520, 768, 1024, 1032, 1536, 2112, 4096, 8200])
@pytest.mark.parametrize("rows", [1, 20, 140])
def test_product_depths(rows, K):
    say("product depth", rows, K)
    product_case(rows, 136, K, 1, True, rows == 20, rows == 20)


@pytest.mark.parametrize("rows, N, K, count", [(522, 1024, 1024, 3), (2048, 1024, 1024, 1), (5496, 512, 512, 2),
                                               (1374, 1024, 4096, 1), (3001, 264, 2112, 3)])
def test_product_sizes(rows, N, K, count):
    say("product size", rows, N, K, count)
    product_case(rows, N, K, count, True, count == 1)


# (rows, N, K, matrices, residual): odd sizes that reach every kernel, and the sizes at which one hands over to the
# next (test_operator_plan.py checks where they lead)
FEW = [(1, 1024, 1024, 3, False), (32, 1024, 1024, 3, False), (63, 1000, 4096, 1, True), (127, 1024, 520, 1, True)]
TILE64 = [(129, 1024, 1024, 1, True), (65, 1000, 4096, 1, False), (1023, 1032, 264, 3, False)]
TILE128 = [(1374, 1024, 1024, 3, False), (5001, 1032, 264, 1, True), (4097, 1032, 1032, 1, False)]
MANY = [(9001, 1032, 264, 1, True), (7601, 1032, 1040, 1, False), (10992, 520, 64, 3, False)]
TILE256 = [(12001, 1032, 2056, 1, True), (12001, 1032, 1288, 2, False)]
SPLIT = [(17001, 1032, 1040, 1, True), (16001, 1032, 1304, 2, False), (16700, 1024, 1288, 1, True)]
PANEL = [(22001, 1000, 1000, 3, False), (22001, 1000, 696, 3, False), (22001, 1000, 264, 3, False),
         (22001, 1000, 200, 3, False), (44000, 1032, 1024, 2, False), (2048 * 512 + 5, 64, 64, 1, False)]


@pytest.mark.parametrize("rows, N, K, count, residual", FEW + TILE64 + TILE128 + MANY + TILE256 + SPLIT + PANEL)
def test_product_kernels(rows, N, K, count, residual):
    """Against float64 products on the GPU, the values themselves being exact."""
    say("product kernel", rows, N, K, count, residual)
    g = gen(rows + N + K)
    x = (normal(g, rows, K) * torch.exp(normal(g, rows, 1))).to(torch.bfloat16)
    a = harness.mx4_quantize(x)
    av = harness.mx4_dequantize(a, K).double()
    ws = [harness.mx4_quantize((normal(g, N, K) * K ** -0.5).to(torch.bfloat16)) for _ in range(count)]
    bs = [normal(g, N) if i != 1 else None for i in range(count)]
    res, rs = (normal(g, rows, N).to(torch.bfloat16), normal(g, N)) if residual else (None, None)
    out = harness.mx4_linear(a, ws, K, bs, res, rs)
    for i in range(count):
        wv = harness.mx4_dequantize(ws[i], K).double().t().contiguous()
        for at in range(0, rows, 1 << 15):
            part = slice(at, min(rows, at + (1 << 15)))
            want, size = av[part] @ wv, av[part].abs() @ wv.abs()
            if bs[i] is not None:
                want, size = want + bs[i].double(), size + bs[i].double().abs()
            if residual:
                want, size = want * rs.double() + res[part].double(), size * rs.double().abs() + res[part].double().abs()
            tol = HALF * want.abs() + (2 * -(-K // 128) + 4) * 2.0 ** -24 * size
            bad = ~((out[i][part].double() - want).abs() <= tol)
            assert not bad.any(), (i, at, bad.nonzero()[:4].tolist())


def test_product_in_place_on_the_residual():
    say("product in place")
    for rows in (5, 700):
        a, ws, bs, res, rs, out = product_case(rows, 512, 512, 1, True, True)
        y = res.clone()
        agg.agg_mx4_linear_fwd(rows, 512, 512, agg.make_mx4_linear(ws, [y], bs, y, rs), *a)
        assert same_bits(y, out[0])


def test_product_of_broken_rows_and_columns():
    """A block that is no number makes its row's, or its channel's, results NaN and no other."""
    say("product with NaN")
    for rows in (5, 300):
        a, ws, bs, _, _, out = product_case(rows, 256, 512, 1)
        a[1][2, 3], ws[0][1][7, 15] = 255, 255
        got = harness.mx4_linear(a, ws, 512, bs)[0]
        nan = torch.isnan(got)
        assert nan[2].all() and nan[:, 7].all() and nan.sum() == rows + 256 - 1
        assert same_bits(got[~nan], out[0][~nan])


def test_product_of_far_scales():
    """Scales at both ends: sums that are tiny, huge, and beyond the range."""
    say("product far scales")
    for rows in (4, 200):
        g = gen(12)
        for ex, ew in ((-60, -60), (60, 60), (-100, 100), (120, -120)):
            x = (normal(g, rows, 256) * 2.0 ** ex).to(torch.bfloat16)
            w = (normal(g, 64, 256) * 2.0 ** ew).to(torch.bfloat16)
            a, b = harness.mx4_quantize(x), harness.mx4_quantize(w)
            out = harness.mx4_linear(a, [b], 256)[0]
            want, size = orc.linear(orc.values(*(t.cpu().numpy() for t in a), 256),
                                    orc.values(*(t.cpu().numpy() for t in b), 256))
            ok = np.abs(want) < 3e38
            assert ok.mean() > 0.4
            tol = HALF * np.abs(want) + 8 * 2.0 ** -24 * size + 2.0 ** -126
            assert (np.abs(f64(out) - want) <= tol)[ok].all()


# ---- as they are used together -------------------------------------------------------------------
def block_parts(shape, seed, gate=True, post="rms", pre="layer", mx=True):
    C = shape.H * 64
    g = gen(seed)
    wts = inputs.block_weights(C, seed=seed, device="cuda")
    x = inputs.block_input(shape.B, shape.NQ, C, seed=seed, device="cuda")
    qn, kn = make_norm(g, "layer", 64)[0], make_norm(g, "rms", 64)[0]
    rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 0, 32, 32, patch0=1)
    gates = normal(g, shape.B * shape.N, C).to(torch.bfloat16) if gate else None
    res = agg.make_residual(make_norm(g, post, C)[0], make_norm(g, pre, C)[0], 0.5 * normal(g, C), gates, shape.L)
    ms = [harness.mx4_quantize(wts["w_" + n]) for n in "qkvo"] if mx else None
    return wts, x, dict(rope=rope, q_norm=qn, k_norm=kn, residual=res, mx=ms)


@pytest.mark.parametrize("mode", [agg.AGG_BLOCK_SGA, agg.AGG_BLOCK_FRAME, agg.AGG_BLOCK_DENSE])
def test_block_is_its_calls_one_after_another(mode):
    say("block of calls", mode)
    shape = agg.make_shape(2, 3, 9, 7, 5, 8, 64, 2, 2, 1)
    rows, C = 2 * shape.NQ, 512
    wts, x, parts = block_parts(shape, 31)
    first = agg.make_residual(pre=agg.make_norm(agg.AGG_NORM_LAYER, wts["ln_eps"], wts["ln_gamma"], wts["ln_beta"]))
    _, xn = harness.residual_forward(first, x.view(rows, C), None, False)
    y, n = harness.block_ex_forward(shape, mode, wts, agg.make_block_options(x_norm=xn, **parts), x)
    # the same, call by call
    bias = [wts["b_" + i] for i in "qkv"]
    q, k, v = harness.mx4_linear(harness.mx4_quantize(xn), parts["mx"][:3], C, bias)
    q, k, v = (t.view(2, shape.NQ, 8, 64) for t in (q, k, v))
    q, k = harness.rope_forward(shape, parts["rope"], q, k, parts["q_norm"], parts["k_norm"])
    if mode == agg.AGG_BLOCK_SGA:
        o = harness.sga_forward(shape, q, k, v).O
    else:
        o = (harness.frame_forward if mode == agg.AGG_BLOCK_FRAME else harness.dense_forward)(shape, q, k, v)[0]
    out = harness.mx4_linear(harness.mx4_quantize(o.view(rows, C)), parts["mx"][3:], C, [wts["b_o"]])[0]
    h, nn = harness.residual_forward(parts["residual"], x.view(rows, C), out)
    assert torch.isfinite(y).all() and same_bits(y.view(rows, C), h) and same_bits(n.view(rows, C), nn)


def test_block_chain_hands_its_norm_on():
    """Two blocks, the second beginning with the norm that the first one wrote; n over x_norm in place."""
    say("block chain")
    shape = agg.make_shape(1, 2, 6, 6, 1, 4, 64, 2, 2, 1)
    wts, x, parts = block_parts(shape, 33)
    wts2, _, parts2 = block_parts(shape, 34)
    pre = agg.make_norm(agg.AGG_NORM_LAYER, wts2["ln_eps"], wts2["ln_gamma"], wts2["ln_beta"])
    r = parts["residual"]
    parts["residual"] = agg.make_residual(r.keep[0], pre, r.keep[2], r.keep[3], r.gate_rows)
    y1, n1 = harness.block_ex_forward(shape, agg.AGG_BLOCK_FRAME, wts, agg.make_block_options(**parts), x)
    y2, n2 = harness.block_ex_forward(shape, agg.AGG_BLOCK_SGA, wts2, agg.make_block_options(x_norm=n1, **parts2), y1)
    held = n1.clone()
    opts = agg.make_block_options(x_norm=held, **parts2)
    cw = agg.make_block_weights(None, None, 0.0, None, None, None, None, wts2["b_q"], wts2["b_k"], wts2["b_v"], wts2["b_o"])
    size = agg.agg_block_ex_workspace_bytes(shape, agg.AGG_BLOCK_SGA, opts)
    ws, y3 = torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty_like(y1)
    agg.agg_global_block_ex_fwd(shape, agg.AGG_BLOCK_SGA, cw, opts, y1, y3, held, ws, size)
    assert same_bits(y3, y2) and same_bits(held, n2)


@pytest.mark.parametrize("H", [1, 5, 8, 16, 33, 64])
def test_block_norm_in_four_bits_is_norm_then_four_bits(H):
    """The block's own norm goes to 4 bits in one pass: the same result as for the norm handed in as a tensor."""
    say("block norm in four bits", H)
    shape = agg.make_shape(1, 2, 3, 5, 1, H, 64, 1, 1)
    C = H * 64
    wts, x, parts = block_parts(shape, 48)
    x[0, 3] = 0.0
    x[0, 4, 7] = float("inf")
    cw = agg.make_block_weights(*(wts[m] for m in ("ln_gamma", "ln_beta", "ln_eps", "w_q", "w_k", "w_v", "w_o",
                                                   "b_q", "b_k", "b_v", "b_o")))
    size = agg.agg_block_workspace_bytes(shape, agg.AGG_BLOCK_FRAME)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    agg.agg_global_block_fwd(shape, agg.AGG_BLOCK_FRAME, cw, x, torch.empty_like(x), ws, size)
    xn = ws[:x.numel() * 2].view(torch.bfloat16).view(x.shape).clone()  # a block's workspace begins with its norm
    want = harness.block_ex_forward(shape, agg.AGG_BLOCK_FRAME, wts, agg.make_block_options(x_norm=xn, **parts), x)
    got = harness.block_ex_forward(shape, agg.AGG_BLOCK_FRAME, wts, agg.make_block_options(**parts), x)
    assert torch.isfinite(want[0][0, shape.L:]).all() and torch.isnan(want[0][0, 4]).any()
    assert same_bits(got[0], want[0]) and same_bits(got[1], want[1])


def test_block_without_options_is_the_plain_block():
    say("block plain")
    shape = agg.make_shape(1, 3, 9, 7, 5, 16, 64, 2, 2, 1)
    wts, x, _ = block_parts(shape, 35, mx=False)
    for mode in (agg.AGG_BLOCK_SGA, agg.AGG_BLOCK_FRAME, agg.AGG_BLOCK_DENSE):
        y, _ = harness.block_forward(shape, mode, wts, x)
        z, n = harness.block_ex_forward(shape, mode, wts, agg.make_block_options(), x)
        assert n is None and same_bits(y, z)


@pytest.mark.parametrize("mx", [False, True])
def test_block_with_a_residual_scale_alone(mx):
    """Layer scale: in 4 bits the projection's epilogue adds it, in bf16 a pass behind it."""
    say("block layer scale", mx)
    shape = agg.make_shape(1, 2, 5, 5, 1, 4, 64, 2, 2, 1)
    wts, x, parts = block_parts(shape, 36, mx=mx)
    rows, C = shape.NQ, 256
    scale = parts["residual"].keep[2]
    parts["residual"] = agg.make_residual(scale=scale)
    y, _ = harness.block_ex_forward(shape, agg.AGG_BLOCK_DENSE, wts, agg.make_block_options(**parts), x)
    # without a scale the branch is y - x
    parts["residual"] = agg.make_residual()
    z, _ = harness.block_ex_forward(shape, agg.AGG_BLOCK_DENSE, wts, agg.make_block_options(**parts), x)
    want = f64(x) + (f64(z) - f64(x)) * f64(scale)
    # y and z rounded once, the branch once more in bf16
    tol = HALF * (np.abs(want) + np.abs(f64(z)) * np.abs(f64(scale)) + np.abs(f64(z) - f64(x)) * np.abs(f64(scale)))
    within(y, want, tol + 1e-5, "layer scale")


@pytest.mark.parametrize("mode", [agg.AGG_BLOCK_SGA, agg.AGG_BLOCK_FRAME, agg.AGG_BLOCK_DENSE])
def test_block_against_the_oracle(mode):
    """The bf16 block with query/key norms, rotary positions and layer scale, in float64 from x to y."""
    from oracle import block_oracle as blk
    from oracle import sga_oracle

    say("block oracle", mode)
    shape = agg.make_shape(1, 3, 9, 7, 5, 8, 64, 2, 2, 1)
    wts, x, parts = block_parts(shape, 37, gate=False, post="none", pre="none", mx=False)
    g = gen(38)
    (qn, qs), (kn, ks) = make_norm(g, "layer", 64), make_norm(g, "rms", 64)
    scale = parts["residual"].keep[2]
    opts = agg.make_block_options(rope=parts["rope"], q_norm=qn, k_norm=kn, residual=agg.make_residual(scale=scale))
    y, _ = harness.block_ex_forward(shape, mode, wts, opts, x)
    w = {k: f64(v) if torch.is_tensor(v) else v for k, v in wts.items()}
    rnd = lambda a: blk.from_bf16_bits(blk.to_bf16_bits(a))
    x64 = f64(x)[0]
    xn = rnd(blk.layernorm(x64, w["ln_gamma"], w["ln_beta"], w["ln_eps"]))
    q, k, v = (rnd(blk.linear(xn, w["w_" + n], w["b_" + n])).reshape(shape.NQ, 8, 64) for n in "qkv")
    pos = orc.grid_positions(3, 9, 7, 5, 0, 1)
    q = orc.rope(orc.norm(q, *qs), pos, orc.SECTIONS, (0, 32, 32), 100.0)
    k = orc.rope(orc.norm(k, *ks), pos, orc.SECTIONS, (0, 32, 32), 100.0)
    o = sga_oracle.Shape(1, 3, 9, 7, 5, 8, 64, 2, 2, 1, 3, 0.125, 0.0)
    qb, kb, vb = (blk.to_bf16_bits(t[None]) for t in (q, k, v))
    at = np.arange(shape.NQ, dtype=np.int64)
    if mode == agg.AGG_BLOCK_SGA:
        attn = sga_oracle.sga(o, qb, kb, vb, rows=at)["O"]
    else:
        attn = (sga_oracle.frame_rows if mode == agg.AGG_BLOCK_FRAME else sga_oracle.dense_rows)(o, qb, kb, vb, at)[0]
    branch = rnd(blk.linear(rnd(attn).reshape(shape.NQ, 512), w["w_o"], w["b_o"]))
    want = x64 + branch * f64(scale)
    err = np.abs(f64(y)[0] - want)
    # the bounds of the plain block, whose attention this is, hold for values up to 4 and a scale up to 1
    assert np.isfinite(f64(y)).all() and err.max() <= 6e-2 and err.mean() <= 4e-3, (err.max(), err.mean())


def test_operators_on_other_streams_and_in_graphs():
    """A captured run of all of them, replayed on new inputs with eager work between the replays; and
    two streams at once on buffers of their own."""
    say("operators in a graph")
    shape = agg.make_shape(1, 2, 9, 7, 5, 8, 64, 2, 2, 1)
    wts, x, parts = block_parts(shape, 41)
    mode = agg.AGG_BLOCK_SGA
    opts = agg.make_block_options(**parts)
    cw = agg.make_block_weights(*(wts[n] for n in ("ln_gamma", "ln_beta", "ln_eps", "w_q", "w_k", "w_v", "w_o",
                                                   "b_q", "b_k", "b_v", "b_o")))
    size = agg.agg_block_ex_workspace_bytes(shape, mode, opts)

    def buffers():
        return torch.empty(size, dtype=torch.uint8, device="cuda"), torch.empty_like(x), torch.empty_like(x)

    ws, y, n = buffers()
    static = x.clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        agg.agg_global_block_ex_fwd(shape, mode, cw, opts, static, y, n, ws, size)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        agg.agg_global_block_ex_fwd(shape, mode, cw, opts, static, y, n, ws, size)
    for i in range(4):
        new = inputs.block_input(1, shape.NQ, 512, seed=50 + i, device="cuda")
        want = harness.block_ex_forward(shape, mode, wts, opts, new)
        static.copy_(new)
        y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert same_bits(y, want[0]) and same_bits(n, want[1]), i
    # two streams
    xs = [inputs.block_input(1, shape.NQ, 512, seed=60 + i, device="cuda") for i in range(2)]
    want = [harness.block_ex_forward(shape, mode, wts, opts, t) for t in xs]
    bufs, streams = [buffers() for _ in xs], [torch.cuda.Stream() for _ in xs]
    torch.cuda.synchronize()
    for _ in range(3):
        for t, (w_, y_, n_), s in zip(xs, bufs, streams):
            with torch.cuda.stream(s):
                agg.agg_global_block_ex_fwd(shape, mode, cw, opts, t, y_, n_, w_, size)
    torch.cuda.synchronize()
    for (_, y_, n_), (a, b) in zip(bufs, want):
        assert same_bits(y_, a) and same_bits(n_, b)


def test_single_operators_in_graphs():
    """Each by itself, the kernels for many rows among them, replayed on inputs that change in between."""
    say("single operators in graphs")
    g = gen(71)
    shape = agg.make_shape(1, 4, 9, 7, 5, 3, 64, 1, 1)
    rope = agg.make_rope(agg.AGG_ROPE_HEAD, 16, 24, 24, t0=3)
    q = normal(g, 1, shape.NQ, 3, 64).to(torch.bfloat16)
    qr, kr = torch.empty_like(q), torch.empty_like(q)
    rows, C = 1003, 4096
    x, b = (normal(g, rows, C).to(torch.bfloat16) for _ in "xb")
    r = agg.make_residual(make_norm(g, "layer", C)[0], make_norm(g, "layer", C)[0], normal(g, C))
    h, n = torch.empty_like(x), torch.empty_like(x)
    a = [harness.mx4_quantize(t) for t in (x, b)]
    w = harness.mx4_quantize((normal(g, 264, C) / 64).to(torch.bfloat16))
    y = [torch.empty((rows, 264), dtype=torch.bfloat16, device="cuda") for _ in "ab"]
    plans = [agg.make_mx4_linear([w], [t]) for t in y]
    many = normal(g, 22000, 512).to(torch.bfloat16)
    held_many = harness.mx4_quantize(many)
    wide = harness.mx4_quantize((normal(g, 3080, 512) / 22).to(torch.bfloat16))
    out = torch.empty((22000, 3080), dtype=torch.bfloat16, device="cuda")
    panel = agg.make_mx4_linear([wide], [out])

    def run():
        agg.agg_rope_fwd(shape, rope, None, None, None, q, 0, q, 0, qr, kr)
        agg.agg_residual_norm_fwd(rows, C, r, x, b, h, n)
        agg.agg_mx4_quantize(rows, C, n, 0, *a[0])
        for plan in plans:
            agg.agg_mx4_linear_fwd(rows, 264, C, plan, *a[0])
        agg.agg_mx4_quantize(22000, 512, many, 0, *held_many)
        agg.agg_mx4_linear_fwd(22000, 3080, 512, panel, *held_many)
        return [t.clone() for t in (qr, kr, h, n, y[0], y[1], out)]

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(3):
        for t in (q, x, b, many):
            t.copy_(normal(g, *t.shape).to(torch.bfloat16))
        want = run()
        for t in (qr, kr, h, n, *y, out):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for t, v in zip((qr, kr, h, n, *y, out), want):
            assert same_bits(t, v), i


@pytest.mark.parametrize("rows, C", [(70003, 488), (35001, 1000), (23003, 1536), (8201, 4104)])
def test_large_tensors_equal_their_parts(rows, C):
    """Tensors of more than 64 MiB are read and written past the caches: the same bits as in parts below that."""
    say("large tensors", rows, C)
    g = gen(44)
    x, b = (normal(g, rows, C).to(torch.bfloat16) for _ in "xb")
    gate = normal(g, (rows + 999) // 1000, C).to(torch.bfloat16)
    post, pre = make_norm(g, "rms", C)[0], make_norm(g, "layer", C)[0]
    scale = normal(g, C)
    r = agg.make_residual(post=post, pre=pre, scale=scale, gate=gate, gate_rows=1000)
    assert rows * C * 2 > 64 << 20 and rows % 1000
    h, n = harness.residual_forward(r, x, b)
    codes, scales = harness.mx4_quantize(n)
    back = harness.mx4_dequantize((codes, scales), C)
    for i in range(0, rows, 20000 if C < 512 else 5000):
        part = slice(i, min(i + (20000 if C < 512 else 5000), rows))
        own = agg.make_residual(post=post, pre=pre, scale=scale, gate=gate[i // 1000:].contiguous(), gate_rows=1000)
        hp, np_ = harness.residual_forward(own, x[part].contiguous(), b[part].contiguous())
        assert same_bits(hp, h[part]) and same_bits(np_, n[part]), i
        cp, sp = harness.mx4_quantize(np_)
        assert torch.equal(cp, codes[part]) and torch.equal(sp, scales[part]), i
        assert same_bits(harness.mx4_dequantize((cp, sp), C), back[part]), i
    # and in place
    a, c = x.clone(), b.clone()
    agg.agg_residual_norm_fwd(rows, C, r, a, c, a, c)
    assert same_bits(a, h) and same_bits(c, n)


def test_more_rows_than_a_launch_counts():
    """2^26 rows and some: more threads than a launch may have, offsets past 32 bits."""
    say("many rows")
    rows, K = (1 << 26) + 5, 8
    x = torch.zeros(rows, K, device="cuda", dtype=torch.bfloat16)
    edges = [0, (1 << 25) - 1, 1 << 25, (1 << 25) + 1, (1 << 26) - 1, 1 << 26, rows - 1]
    x[edges] = normal(gen(45), len(edges), K).to(torch.bfloat16)
    codes, scales = harness.mx4_quantize(x)
    want = harness.mx4_quantize(x[edges].contiguous())
    assert torch.equal(codes[edges], want[0]) and torch.equal(scales[edges], want[1])
    assert int((scales[:, 0] != 0).sum()) == len(edges) and not bool(scales[:, 1:].any())
    back = harness.mx4_dequantize((codes, scales), K)
    assert same_bits(back[edges], harness.mx4_dequantize(want, K))
    assert int((back != 0).any(1).sum()) == len(edges)
    w = harness.mx4_quantize(normal(gen(46), 8, K).to(torch.bfloat16))
    y, = harness.mx4_linear((codes, scales), [w], K)
    few, = harness.mx4_linear(want, [w], K)
    assert same_bits(y[edges], few)  # one step of k: the same sums in every kernel


def test_operators_repeat_to_the_bit():
    say("operators repeat")
    shape = agg.make_shape(1, 3, 13, 11, 5, 16, 64, 2, 2, 1)
    wts, x, parts = block_parts(shape, 43)
    opts = agg.make_block_options(**parts)
    a = harness.block_ex_forward(shape, agg.AGG_BLOCK_SGA, wts, opts, x)
    for _ in range(3):
        b = harness.block_ex_forward(shape, agg.AGG_BLOCK_SGA, wts, opts, x)
        assert same_bits(a[0], b[0]) and same_bits(a[1], b[1])
