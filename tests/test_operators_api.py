"""The operators around a block's attention without a GPU: the oracle's pins, the sizes the host
reports, and every refusal, all of which come before a launch."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import operators_oracle as orc
from paper_2512_02541_amd import binding as agg

FAKE = 0x10000000  # aligned, never dereferenced: validation fails first
FAR = 1 << 40      # distance between fake buffers


def _at(i):
    return FAKE + i * FAR


# ---- the oracle's pins ---------------------------------------------------------------------------
def test_oracle_norms_match_torch():
    gen = torch.Generator().manual_seed(1)
    x = torch.randn((7, 64), generator=gen, dtype=torch.float64)
    g, b = (torch.randn((64,), generator=gen, dtype=torch.float64) for _ in "gb")
    want = torch.nn.functional.layer_norm(x, (64,), g, b, 1e-3)
    assert np.abs(orc.norm(x.numpy(), orc.LAYER, 1e-3, g.numpy(), b.numpy()) - want.numpy()).max() < 1e-12
    want = torch.nn.functional.rms_norm(x, (64,), g, 1e-3)
    assert np.abs(orc.norm(x.numpy(), orc.RMS, 1e-3, g.numpy()) - want.numpy()).max() < 1e-12


@pytest.mark.parametrize("pairing", [orc.SECTIONS, orc.NEIGHBOURS, orc.HEAD])
def test_oracle_rotation(pairing):
    rng = np.random.default_rng(2)
    axes, base = (16, 20, 24), 100.0
    q, k = rng.standard_normal((2, 5, 2, 64))
    pos = rng.integers(-50, 50, (5, 3))
    rq = orc.rope(q, pos, pairing, axes, base)
    assert np.abs(orc.rope(rq, -pos, pairing, axes, base) - q).max() < 1e-12
    assert np.abs((rq ** 2).sum(-1) - (q ** 2).sum(-1)).max() < 1e-10
    # scores depend on the difference of positions alone
    off = rng.integers(-50, 50, (5, 3))
    a = (rq * orc.rope(k, pos + off, pairing, axes, base)).sum(-1)
    b = (q * orc.rope(k, off, pairing, axes, base)).sum(-1)
    assert np.abs(a - b).max() < 1e-10
    # every channel of the axes is in one pair, and each axis has its share
    pairs = orc.rope_pairs(pairing, axes, base)
    assert sorted(c for p in pairs for c in p[:2]) == list(range(60))
    assert [sum(p[2] == a for p in pairs) for a in range(3)] == [8, 10, 12]


def test_oracle_rotation_is_a_complex_product():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 1, 64))
    pos = np.array([[0, 3, 5], [1, 0, 7], [2, 9, 0], [100000, 1, 1]])
    y = orc.rope(x, pos, orc.NEIGHBOURS, (0, 32, 32), 100.0)
    z = (x[..., 0::2] + 1j * x[..., 1::2])[:, 0]
    angle = np.concatenate([pos[:, 1:2] * 100.0 ** (-np.arange(16) / 16), pos[:, 2:3] * 100.0 ** (-np.arange(16) / 16)], 1)
    z = z * np.exp(1j * angle)
    assert np.abs(y[:, 0, 0::2] - z.real).max() < 1e-12 and np.abs(y[:, 0, 1::2] - z.imag).max() < 1e-12


def test_oracle_four_bit_rounding():
    # one block whose scale is 1: its largest magnitude is 4 <= m < 8
    x = np.concatenate([[6.0], np.linspace(-7.9, 7.9, 62)]).reshape(1, -1)
    x = np.pad(x, ((0, 0), (0, 1)))
    codes, scales = orc.quantize(x)
    assert (scales == 127).all()
    got = orc.values(*orc.pack(codes, scales, 128, 16), 64)
    allv = np.concatenate([orc.GRID, -orc.GRID])
    for v, r in zip(x[0], got[0]):
        assert abs(r - v) <= np.abs(allv - v).min() + 1e-15
    ties = np.array([[4.0, .25, .75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 7.5, 0.0]])
    codes, scales = orc.quantize(ties)
    got = orc.values(*orc.pack(codes, scales, 128, 16), 12)
    assert got[0].tolist() == [4, 0, 1, 1, 2, 2, 4, 4, 0, -4, 6, 0]
    # scales: zeros, the smallest, the largest exponents, broken blocks
    tiny, huge = 2.0 ** -133, 1.5 * 2.0 ** 127
    codes, scales = orc.quantize(np.array([[0.0], [tiny], [huge], [np.inf], [np.nan], [1.0]]))
    assert scales[:, 0].tolist() == [0, 0, 252, 255, 255, 125]
    assert codes[:, 0, 0].tolist() == [0, 0, 7 - 0, 0, 0, 6]
    # a quantised matrix is its own quantisation wherever its block's largest is 4 or 6 scales
    rng = np.random.default_rng(4)
    once = orc.values(*orc.pack(*orc.quantize(rng.standard_normal((20, 96))), 128, 16), 96)
    twice = orc.values(*orc.pack(*orc.quantize(once), 128, 16), 96)
    assert (once == twice).all()


def test_oracle_layout():
    codes = np.zeros((1, 2, 32), dtype=np.int64)
    codes[0, 0, 0], codes[0, 0, 1], codes[0, 1, 31] = 3, 12, 9
    c, s = orc.pack(codes, np.array([[130, 7]]), 128, 16)
    assert c[0, 0] == 3 | 12 << 4 and c[0, 31] == 9 << 4 and c[0, 32:].sum() == 0
    assert s[0, :2].tolist() == [130, 7] and s[0, 2:].sum() == 0
    v = orc.values(c, s, 64)
    assert v[0, 0] == 1.5 * 8 and v[0, 1] == -2.0 * 8 and v[0, 63] == -0.5 * 2.0 ** -120


# ---- the host side -------------------------------------------------------------------------------
def test_strides():
    for K in (8, 32, 64, 256, 264, 512, 520, 1024, 2112, 4096):
        assert agg.agg_mx4_code_stride(K) == -(-K // 256) * 128
        assert agg.agg_mx4_scale_stride(K) == -(-K // 512) * 16
    assert agg.agg_mx4_code_stride(0) == agg.agg_mx4_scale_stride(-1) == 0


def _status(call, *args):
    try:
        call(*args, stream=0)
    except agg.AggError as e:
        return e.status
    return 0


def _rope(shape=None, rope="plain", q_norm=None, k_norm=None, pos=None, q=_at(0), qs=0, k=_at(1), ks=0,
          qr=_at(2), kr=_at(3), **fields):
    s = shape or agg.make_shape(1, 2, 16, 16, 5, 16, 64, 1, 1)
    if rope == "plain":
        rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 0, 32, 32)
        for name, value in fields.items():
            setattr(rope, name, value)
    return _status(agg.agg_rope_fwd, s, rope, q_norm, k_norm, pos, q, qs, k, ks, qr, kr)


def test_rope_refusals():
    N, S, U, A, O = (agg.AGG_ERR_NULL, agg.AGG_ERR_SHAPE, agg.AGG_ERR_UNSUPPORTED, agg.AGG_ERR_ALIGN,
                     agg.AGG_ERR_OVERFLOW)
    assert _rope(q=None) == N and _rope(kr=None) == N
    assert _rope(q=None, qr=None, k=None, kr=None) == N
    assert _rope(pairing=3) == S and _rope(pairing=-1) == S
    assert _rope(d_h=31) == S and _rope(d_t=2) == S and _rope(d_w=-2) == S
    assert _rope(d_t=0x7FFFFFFE, d_h=2, d_w=0) == S
    for base in (0.0, 0.5, -3.0, float("inf"), float("nan")):
        assert _rope(base=base) == S
    assert _rope(q=_at(0) + 8) == A and _rope(kr=_at(3) + 2) == A and _rope(pos=_at(4) + 2) == A
    assert _rope(t0=2 ** 31 - 2) == O and _rope(patch0=2 ** 31 - 16) == O
    assert _rope(qs=1016) == S and _rope(qs=1028) == S and _rope(ks=-1024) == S
    assert _rope(qs=1 << 58) == O
    row = 522 * 2048
    # overlaps: shifted in place, the other's input, both outputs, positions, a strided input in place
    assert _rope(qr=_at(0) + 16) == S and _rope(qr=_at(0) - row + 16) == S
    assert _rope(qr=_at(1)) == S and _rope(kr=_at(2) + row - 16) == S
    assert _rope(pos=_at(2)) == S and _rope(qr=_at(0), qs=2048) == S
    assert _rope(shape=agg.make_shape(1, 2, 16, 16, 5, 16, 32, 1, 1)) == U
    assert _rope(shape=agg.make_shape(1, 0, 16, 16, 5, 16, 64, 1, 1)) == S
    for n, want in ((agg.make_norm(3), S), (agg.make_norm(agg.AGG_NORM_RMS, 0.0), S),
                    (agg.make_norm(agg.AGG_NORM_RMS, float("nan")), S),
                    (agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, FAKE + 4), A),
                    (agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, FAKE, FAKE + 8), A)):
        assert _rope(q_norm=n) == want and _rope(k_norm=n) == want


def _seam(rows=10, C=1024, x=_at(0), branch=_at(1), h=_at(2), n=_at(3), pre=agg.AGG_NORM_LAYER, **kw):
    r = agg.make_residual(pre=agg.make_norm(pre), **kw)
    return _status(agg.agg_residual_norm_fwd, rows, C, r, x, branch, h, n)


def test_residual_refusals():
    N, S, U, A, O = (agg.AGG_ERR_NULL, agg.AGG_ERR_SHAPE, agg.AGG_ERR_UNSUPPORTED, agg.AGG_ERR_ALIGN,
                     agg.AGG_ERR_OVERFLOW)
    assert _seam(rows=0) == 0 and _seam(rows=0, x=None, branch=None, h=None) == 0
    assert _seam(rows=-1) == S and _seam(C=0) == S and _seam(C=1020) == S and _seam(C=8200) == U
    assert _seam(rows=1 << 32) == O
    assert _seam(x=None) == N and _seam(n=None) == N and _seam(pre=0) == N
    assert _seam(pre=0, n=None, h=None) == N
    assert _seam(pre=5) == S
    # without a branch there is nothing to scale, gate or normalise
    assert _seam(branch=None, scale=_at(5)) == N and _seam(branch=None, gate=_at(5), gate_rows=1) == N
    assert _seam(branch=None, post=agg.make_norm(agg.AGG_NORM_RMS)) == N
    assert _seam(gate=_at(5), gate_rows=0) == S and _seam(gate=_at(5), gate_rows=-4) == S
    for name, at in (("x", 0), ("branch", 1), ("h", 2), ("n", 3)):
        assert _seam(**{name: _at(at) + 8}) == A
    assert _seam(scale=_at(5) + 4) == A and _seam(gate=_at(5) + 2, gate_rows=1) == A
    for out in ("h", "n"):
        assert _seam(**{out: _at(0) + 16}) == S and _seam(**{out: _at(1) - 16}) == S
        assert _seam(gate=_at(5), gate_rows=3, **{out: _at(5) + 3 * 2048}) == S
    assert _seam(h=_at(3) + 2048) == S
    lib = agg.lib()
    assert lib.agg_residual_norm_fwd(1, 64, None, _at(0), _at(1), _at(2), None, None) == N


def _linear(rows=10, N=1024, K=1024, count=1, a=_at(0), s=_at(1), y=None, **kw):
    y = y or [_at(10 + i) for i in range(count)]
    m = agg.make_mx4_linear([(_at(2), _at(3))] * count, y, **kw)
    return _status(agg.agg_mx4_linear_fwd, rows, N, K, m, a, s)


def test_mx4_refusals():
    N, S, A, O = agg.AGG_ERR_NULL, agg.AGG_ERR_SHAPE, agg.AGG_ERR_ALIGN, agg.AGG_ERR_OVERFLOW

    def quant(rows=10, K=1024, x=_at(0), stride=0, c=_at(1), s=_at(2)):
        return _status(agg.agg_mx4_quantize, rows, K, x, stride, c, s)

    def back(rows=10, K=1024, c=_at(1), s=_at(2), x=_at(0)):
        return _status(agg.agg_mx4_dequantize, rows, K, c, s, x)

    for call in (quant, back):
        assert call(rows=0) == 0 and call(rows=0, x=None) == 0
        assert call(rows=-1) == S and call(K=0) == S and call(K=1020) == S
        assert call(rows=1 << 32) == O and call(K=2 ** 31 - 8) == O
        assert call(x=None) == N and call(c=None) == N and call(s=None) == N
        assert call(x=_at(0) + 8) == A and call(c=_at(1) + 4) == A and call(s=_at(2) + 8) == A
        assert call(c=_at(0) + 16) == S and call(s=_at(0) + 10 * 2048 - 16) == S
    assert quant(stride=1016) == S and quant(stride=1028) == S and quant(stride=-1024) == S
    assert quant(stride=1 << 58) == O and quant(s=_at(1) + 512) == S

    assert _linear(rows=0) == 0 and _linear(rows=0, a=None) == 0
    assert _linear(rows=-1) == S and _linear(N=0) == S and _linear(N=1020) == S and _linear(K=1020) == S
    assert _linear(rows=1 << 32) == O and _linear(N=1 << 22) == O
    assert _linear(a=None) == N and _linear(s=None) == N and _linear(y=[None]) == N
    assert _linear(a=_at(0) + 8) == A and _linear(s=_at(1) + 8) == A and _linear(y=[_at(9) + 2]) == A
    assert _linear(biases=[_at(5) + 4]) == A and _linear(residual=_at(5) + 4) == A
    assert _linear(residual=_at(5), res_scale=_at(6) + 4) == A
    assert _linear(count=2, residual=_at(5)) == S and _linear(res_scale=_at(5)) == S
    assert _linear(count=2, y=[_at(9), _at(9) + 16]) == S and _linear(residual=_at(10) + 2048) == S
    assert _linear(y=[_at(0) + 512]) == S and _linear(y=[_at(1) + 16]) == S
    assert _linear(y=[_at(2) + 512]) == S and _linear(y=[_at(3) - 16]) == S
    assert _linear(K=1 << 23) == O and _linear(rows=1 << 31, N=1 << 21) == O
    m = agg.make_mx4_linear([(_at(2), _at(3))], [_at(9)])
    m.count = 4
    assert _status(agg.agg_mx4_linear_fwd, 1, 64, 64, m, _at(0), _at(1)) == S
    m.count = 0
    assert _status(agg.agg_mx4_linear_fwd, 1, 64, 64, m, _at(0), _at(1)) == S
    m = agg.make_mx4_linear([(None, _at(3))], [_at(9)])
    assert _status(agg.agg_mx4_linear_fwd, 1, 64, 64, m, _at(0), _at(1)) == N
    assert agg.lib().agg_mx4_linear_fwd(1, 64, 64, None, _at(0), _at(1), None) == N
    with pytest.raises(ValueError):
        agg.make_mx4_linear([], [])
    with pytest.raises(ValueError):
        agg.make_mx4_linear([(1, 2)] * 2, [1])


def test_block_refusals():
    N, S, U, A, W = (agg.AGG_ERR_NULL, agg.AGG_ERR_SHAPE, agg.AGG_ERR_UNSUPPORTED, agg.AGG_ERR_ALIGN,
                     agg.AGG_ERR_WORKSPACE)
    shape = agg.make_shape(1, 2, 16, 16, 5, 16, 64, 2, 2)
    weights = agg.agg_block_weights(_at(20), _at(21), 1e-6, _at(22), _at(23), _at(24), _at(25), None, None, None, None)
    mx = [(_at(30 + 2 * i), _at(31 + 2 * i)) for i in range(4)]
    pre = agg.make_residual(pre=agg.make_norm(agg.AGG_NORM_RMS))
    for mode in (agg.AGG_BLOCK_SGA, agg.AGG_BLOCK_FRAME, agg.AGG_BLOCK_DENSE):
        plain, four = agg.make_block_options(), agg.make_block_options(mx=mx)
        nb = agg.agg_block_workspace_bytes(shape, mode)
        assert agg.agg_block_ex_workspace_bytes(shape, mode, plain) == nb
        ns = agg.agg_block_ex_workspace_bytes(shape, mode, four)
        assert ns >= nb + 522 * (512 + 32)

        def call(o, w=weights, x=_at(0), y=_at(1), n=None, ws=_at(2), size=1 << 40, sh=shape):
            return _status(agg.agg_global_block_ex_fwd, sh, mode, w, o, x, y, n, ws, size)

        assert call(plain, size=nb - 1) == W and call(four, size=ns - 1) == W
        assert call(plain, x=None) == N and call(plain, y=None) == N and call(plain, ws=None) == N
        assert call(plain, x=_at(0) + 8) == A and call(plain, ws=_at(2) + 8) == A
        assert call(plain, y=_at(0)) == S and call(plain, y=_at(0) + 2048) == S and call(plain, y=_at(2) + 4096) == S
        assert call(plain, n=_at(3)) == N and call(agg.make_block_options(residual=pre)) == N
        assert call(agg.make_block_options(residual=pre), n=_at(1) + 2048) == S
        assert call(agg.make_block_options(residual=pre, x_norm=_at(4)), y=_at(4), n=_at(5)) == S
        bad = agg.agg_block_weights(_at(20), None, 1e-6, _at(22), _at(23), _at(24), _at(25), None, None, None, None)
        assert call(plain, w=bad) == N
        bare = agg.agg_block_weights(None, None, 0.0, None, None, None, None, None, None, None, None)
        assert call(plain, w=bare) == N
        assert call(agg.make_block_options(x_norm=_at(4)), w=bare) == N     # the matrices are missing
        assert call(agg.make_block_options(mx=mx), w=bare) == N             # the first norm is missing
        o = agg.make_block_options(mx=mx)
        o.first_done = 1
        assert call(o) == N
        o.first_done = 2
        assert call(o) == S
        assert call(agg.make_block_options(mx=mx[:3] + [(None, _at(3))])) == N
        assert call(agg.make_block_options(mx=mx[:3] + [(_at(8) + 8, _at(3))])) == A
        assert call(agg.make_block_options(rope=agg.make_rope(7, 0, 32, 32))) == S
        assert call(agg.make_block_options(q_norm=agg.make_norm(9))) == S
        assert call(agg.make_block_options(residual=agg.make_residual(gate=_at(5)))) == S
        wide = agg.make_shape(1, 2, 16, 16, 5, 65, 64, 2, 2)
        assert call(plain, sh=wide) == U
    assert agg.agg_block_ex_workspace_bytes(shape, 7, agg.make_block_options()) == 0
    with pytest.raises(ValueError):
        agg.make_block_options(mx=mx[:3])
    lib = agg.lib()
    assert lib.agg_global_block_ex_fwd(ctypes.byref(shape), 0, ctypes.byref(weights), None, _at(0), _at(1), None,
                                       _at(2), 1 << 40, None) == N


def test_errors_say_what_the_operators_refuse():
    """A status that several calls share names the reasons of all of them."""
    def message(call):
        with pytest.raises(agg.AggError) as e:
            call()
        return str(e.value)

    r, m = agg.make_residual(), agg.make_mx4_linear([(_at(2), _at(3))], [_at(9)])
    wide = message(lambda: agg.agg_residual_norm_fwd(1, 8200, r, _at(0), _at(1), _at(2), None, stream=0))
    assert "wider" in wide and "head dimension" in wide
    over = message(lambda: agg.agg_residual_norm_fwd(4, 64, r, _at(0), _at(1), _at(0) + 64, None, stream=0))
    assert "overlap" in over and "shape" in over
    deep = message(lambda: agg.agg_mx4_linear_fwd(1, 64, 1 << 23, m, _at(0), _at(1), stream=0))
    far = message(lambda: agg.agg_rope_fwd(agg.make_shape(1, 2, 16, 16, 5, 16, 64, 1, 1),
                                           agg.make_rope(agg.AGG_ROPE_HEAD, 16, 24, 24, t0=2 ** 31 - 2), None, None, None,
                                           _at(0), 0, None, 0, _at(2), None, stream=0))
    assert deep.split(": ")[1] == far.split(": ")[1] and "size" in deep and "position" in far and "token" not in deep


def test_outputs_over_parameters_are_refused():
    """Parameters are read while outputs are written: an overlap would let rows already written change the others."""
    S = agg.AGG_ERR_SHAPE
    rows = 522 * 2048
    for at, out in ((2, "qr"), (3, "kr")):
        for near in (_at(at), _at(at) + rows - 16, _at(at) - 240):
            for n in (agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, near), agg.make_norm(agg.AGG_NORM_RMS, 1e-5, None, near)):
                assert _rope(q_norm=n) == S and _rope(k_norm=n) == S, out
    for at in (2, 3):  # h, n
        for near in (_at(at), _at(at) + 10 * 2048 - 16, _at(at) - 4080):
            assert _seam(scale=near) == S
            for n in (agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, near), agg.make_norm(agg.AGG_NORM_RMS, 1e-5, None, near)):
                assert _seam(post=n) == S
                r = agg.make_residual(pre=n)
                assert _status(agg.agg_residual_norm_fwd, 10, 1024, r, _at(0), _at(1), _at(2), _at(3)) == S
    for near in (_at(10), _at(10) + 10 * 2048 - 16, _at(10) - 4080):
        assert _linear(biases=[near]) == S and _linear(count=2, biases=[None, near]) == S
        assert _linear(residual=_at(5), res_scale=near) == S
    # the y of a block is its residual norm's, or its output projection's
    shape = agg.make_shape(1, 2, 16, 16, 5, 16, 64, 2, 2)
    w = agg.agg_block_weights(_at(20), _at(21), 1e-6, _at(22), _at(23), _at(24), _at(25), None, None, None, _at(1) + 64)
    mx = [(_at(30 + 2 * i), _at(31 + 2 * i)) for i in range(4)]
    scaled = agg.make_residual(scale=_at(1) + 1024)
    for o, weights in ((agg.make_block_options(mx=mx), w), (agg.make_block_options(residual=scaled), w)):
        assert _status(agg.agg_global_block_ex_fwd, shape, agg.AGG_BLOCK_FRAME, weights, o, _at(0), _at(1), None, _at(2),
                       1 << 40) == S


def test_more_pairs_than_a_launch_plan_counts_are_refused():
    """2^34 and 2^33 + 2^5 (frame, head) pairs: numbers whose last 32 bits are 0 and 32."""
    for N in (1 << 30, (1 << 29) + 2):
        shape = agg.make_shape(1, N, 1, 1, 0, 16, 64, 1, 1)
        assert _status(agg.agg_frame_attn_fwd, shape, _at(0), _at(1), _at(2), _at(3), None) == agg.AGG_ERR_LAUNCH
