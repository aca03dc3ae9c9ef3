"""Attention to keys of another length and the paged cache on the GPU, through the C ABI, against the float64 oracle.

Tolerances count roundings.  With A the sum of probability times |v| of a row's channel and S the largest sum of
|scale q k| of its keys:
  O    A probability is rounded to bf16 on its way into the second product, 2^-8 of itself, and the sum may hold the
       rounded or the unrounded ones: 2 * 2^-8 A.  The result is rounded to bf16: 2^-8 |O|.  Logits are sums of 64 exact
       products in float32, 2^-24 of S each, and every other float32 step (exponential, scale, sums of up to
       2^18 keys in lanes and blocks) is under 2^-14 together: 2^-12 (A + S A).
  lse  2^-18 S + 2^-16 (1 + |lse|); where the sum is that of rounded probabilities (more than 32 rows a key head: queries by heads
       that share it) ln(1 + 2^-8) < 2^-8 more.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from oracle import operators_oracle as ops
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import harness

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
FEW = 32


def say(*a):
    print(*a, flush=True)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def bf16(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float32) * scale).to(torch.bfloat16)


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def same_bits(a, b):
    kind = torch.int16 if a.dtype == torch.bfloat16 else torch.int32
    return torch.equal(a.view(kind), b.view(kind))


def check(cross, got, q, k, v, q_lens=None, k_lens=None, what=""):
    """O and lse against the oracle; rows that do not exist have to hold the NaN they held."""
    torch.cuda.synchronize()
    (o, lse), (wo, wl, size, dots) = got, orc.attention(q, k, v, float(np.float32(cross.scale)), q_lens, k_lens)
    absent = torch.isnan(dots).expand_as(wo)
    assert bool((o.view(torch.int16)[absent] == 0x7FC1).all()), what + ": rows behind the last query changed"
    assert bool(torch.isnan(lse[torch.isnan(dots[..., 0]).transpose(1, 2)]).all()), what
    many = cross.NQ * (cross.H // cross.H_kv) > FEW
    tol = (2 * HALF + 2.0 ** -12 * (1 + dots)) * size + HALF * wo.abs()
    off = (o.double() - wo).abs()
    bad = ~(off <= tol) & ~absent
    assert not bool(bad.any()), "%s: %d of O off, worst %.3g of the tolerance" % (
        what, int(bad.sum()), float((off / tol.clamp(min=1e-300))[~absent].nan_to_num(1e9).max()))
    S = dots[..., 0].transpose(1, 2)
    ltol = 2.0 ** -18 * S + 2.0 ** -16 * (1 + wl.abs()) + (HALF if many else 0.0)
    there = ~torch.isnan(S)
    empty = there & torch.isinf(wl)
    assert bool((lse[empty] == -math.inf).all()), what
    loff = (lse.double() - wl).abs()
    lbad = there & ~empty & ~(loff <= ltol)
    assert not bool(lbad.any()), "%s: %d of lse off, worst %.3g of the tolerance" % (
        what, int(lbad.sum()), float((loff / ltol)[there & ~empty].nan_to_num(1e9).max()))


def pages_of(g, B, entries, spare=3):
    """A page table in no order over a pool with pages to spare."""
    n = B * entries + spare
    return torch.randperm(n, generator=g, device="cuda")[:B * entries].to(torch.int32).view(B, entries).contiguous(), n


def put(pools, pages, k, v, lens=None):
    """Writes k and v [B, n, H, 64] into the pools by the oracle's places; rows behind lens stay as they are."""
    B, n, H, _ = k.shape
    for pool, t, place in zip(pools, (k, v), (orc.k_place, orc.v_place)):
        at = orc._places(place, pool.device)
        for b in range(B):
            rows = torch.arange(n if lens is None else min(int(lens[b]), n), device=pool.device)
            for h in range(H):
                pool[pages[b, rows // 64].long()[:, None], h, at[rows % 64]] = t[b, :len(rows), h]


def both(B, NQ, NK, H, H_kv=None, seed=1, q_lens=None, k_lens=None, scale=None, qs=1.3, what=None):
    """The same attention with keys where they are and out of a cache, each against the oracle."""
    H_kv = H_kv or H
    what = what or "B %d NQ %d NK %d H %d/%d" % (B, NQ, NK, H, H_kv)
    say("attention", what)
    g = gen(seed)
    q, k, v = bf16(g, B, NQ, H, 64, scale=qs), bf16(g, B, NK, H_kv, 64), bf16(g, B, NK, H_kv, 64)
    ql, kl = (None if x is None else ints(x) for x in (q_lens, k_lens))
    cross = agg.make_cross(B, NQ, NK, H, H_kv, scale=scale, q_lens=ql, k_lens=kl)
    check(cross, harness.cross_forward(cross, q, k, v), q, k, v, q_lens, k_lens, what)
    pages, n = pages_of(g, B, -(-NK // 64))
    pools = harness.make_pools(n, H_kv, "cuda")
    put(pools, pages, k, v)
    cache = agg.make_cache(*pools, pages, H_kv)
    check(cross, harness.cache_forward(cache, cross, q), q, k, v, q_lens, k_lens, what + " cached")


LENGTHS = [(1, 1, 1), (2, 1, 31), (1, 3, 32), (1, 16, 33), (3, 17, 63), (1, 32, 64), (1, 33, 65), (2, 64, 127),
           (2, 65, 129), (1, 64, 1000), (1, 127, 257), (1, 128, 500), (1, 129, 191), (1, 192, 640), (1, 193, 100),
           (1, 256, 96), (1, 257, 1300), (2, 513, 70), (1, 777, 1029), (2, 300, 1), (1, 40, 2), (1, 1, 4096), (1, 1, 20001),
           (1, 5, 9000), (1, 30, 7001), (1, 61, 5003), (1, 100, 12000), (1, 261, 16384), (1, 1374, 6000)]


@pytest.mark.parametrize("B, NQ, NK", LENGTHS)
def test_lengths(B, NQ, NK):
    both(B, NQ, NK, 2)


# sizes that fill the card with workgroups of every width: B, NQ, NK, H, H_kv
WIDE = [(20, 512, 90, 16, 16), (24, 512, 400, 16, 16), (20, 520, 130, 16, 16), (20, 440, 100, 16, 16), (16, 190, 65, 32, 16), (1, 1374, 9000, 16, 16),
        (2, 700, 6000, 16, 8), (1, 2816, 8000, 16, 16), (6, 128, 700, 4, 4), (3, 500, 1500, 16, 4), (2, 1024, 12000, 16, 16),
        (1, 600, 20000, 2, 2), (3, 380, 9000, 1, 1), (20, 100, 100, 4, 4), (20, 100, 2000, 4, 4), (2, 440, 5000, 12, 12),
        (24, 65, 1029, 4, 4), (6, 65, 2000, 16, 16)]


@pytest.mark.parametrize("B, NQ, NK, H, H_kv", WIDE)
def test_many_rows(B, NQ, NK, H, H_kv):
    both(B, NQ, NK, H, H_kv, seed=12)


@pytest.mark.parametrize("B, NQ, NK, H, H_kv", [(64, 3, 70, 12, 12), (61, 20, 40, 13, 13), (257, 1, 33, 3, 3), (100, 33, 65, 4, 4)])
def test_many_pairs(B, NQ, NK, H, H_kv):
    """Workgroups of few rows dealt out to the XCDs in runs, as many as eight of them hold and some more or fewer."""
    both(B, NQ, NK, H, H_kv, seed=14)


@pytest.mark.parametrize("NQ", [1, 7, 30, 200])
@pytest.mark.parametrize("H, H_kv", [(1, 1), (4, 4), (12, 4), (16, 1), (33, 33), (20, 5), (6, 2)])
def test_heads(H, H_kv, NQ):
    both(2, NQ, 197, H, H_kv, seed=2)


@pytest.mark.parametrize("NQ, NK, H", [(1, 700, 3), (9, 5000, 3), (40, 300, 3), (100, 640, 3), (300, 1400, 3), (520, 9000, 3),
                                       (100, 640, 24), (300, 1400, 16), (700, 500, 16),
                                       (700, 65, 32), (512, 700, 2), (70, 3000, 8), (70, 3000, 2)])
def test_ragged(NQ, NK, H):
    """Lengths of every kind: none, one, inside a tile, on its border, all, and values outside the range."""
    k_lens = [NK, 0, 1, NK // 2, 64, min(65, NK), NK - 1, -3, NK + 100]
    q_lens = [NQ, NQ, 1, NQ // 2, 0, NQ - 1, NQ, NQ, NQ + 7]
    both(9, NQ, NK, H, seed=3, k_lens=k_lens)
    both(9, NQ, NK, H - H % 2, H // 2, seed=4, q_lens=q_lens, k_lens=k_lens)
    both(3, NQ, NK, 2, seed=5, q_lens=[0, 0, 0], k_lens=[0, 5, NK])


def test_no_queries_and_no_keys():
    say("empty calls")
    g = gen(6)
    q, k = bf16(g, 2, 5, 4, 64), bf16(g, 2, 9, 4, 64)
    o, lse = harness.cross_forward(agg.make_cross(2, 5, 0, 4), q, None, None)
    torch.cuda.synchronize()
    assert not bool(o.any()) and bool((lse == -math.inf).all())
    assert agg.agg_cross_workspace_bytes(agg.make_cross(2, 0, 9, 4)) == 0
    agg.agg_cross_attn_fwd(agg.make_cross(2, 0, 9, 4), None, 0, k, 0, k, 0, None)
    many = bf16(g, 1, 400, 2, 64)
    o, lse = harness.cross_forward(agg.make_cross(1, 400, 0, 2), many, None, None)
    torch.cuda.synchronize()
    assert not bool(o.any()) and bool((lse == -math.inf).all())


BEHIND = [(NQ, H, 1000, (1000, 1, 95, 640)) for NQ, H in [(1, 2), (20, 2), (60, 2), (250, 32), (500, 32), (1000, 16)]] + \
         [(1374, 16, 9000, (8963,)), (2816, 16, 8000, (7990,)), (100, 80, 100, (70,)), (512, 350, 400, (391,)), (65, 96, 1029, (1001,))]


@pytest.mark.parametrize("NQ, H, NK, lens", BEHIND)
def test_what_lies_behind_the_keys_does_not_matter(NQ, H, NK, lens):
    """NaN and infinities in rows, and in pages, behind the last key."""
    g = gen(7)
    B, lens = len(lens), list(lens)
    q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H, 64), bf16(g, B, NK, H, 64)
    kl = ints(lens)
    cross = agg.make_cross(B, NQ, NK, H, k_lens=kl)
    want = harness.cross_forward(cross, q, k, v)
    pages, n = pages_of(g, B, -(-NK // 64))
    pools = harness.make_pools(n, H, "cuda", fill=0)
    put(pools, pages, k, v, lens)
    clean = harness.cache_forward(agg.make_cache(*pools, pages, H), cross, q)
    check(cross, want, q, k, v, None, lens, "clean")
    for bad in (math.nan, math.inf, -math.inf):
        say("behind the keys", NQ, bad)
        k2, v2 = k.clone(), v.clone()
        for b, m in enumerate(lens):
            k2[b, m:] = bad
            v2[b, m:] = bad
        got = harness.cross_forward(cross, q, k2, v2)
        pools = harness.make_pools(n, H, "cuda")
        for p in pools:
            p.fill_(bad)
        put(pools, pages, k, v, lens)
        cached = harness.cache_forward(agg.make_cache(*pools, pages, H), cross, q)
        torch.cuda.synchronize()
        for x, y in zip(want + clean, got + cached):
            assert same_bits(x, y), bad


@pytest.mark.parametrize("NQ", [1, 50, 90, 300])
@pytest.mark.parametrize("NK", [130, 5000])
def test_large_logits(NQ, NK):
    """Logits of hundreds, one key that outweighs all others wherever it lies, and rows without one."""
    say("large logits", NQ, NK)
    g = gen(8)
    H = 2
    q, k, v = bf16(g, 1, NQ, H, 64), bf16(g, 1, NK, H, 64, scale=0.3), bf16(g, 1, NK, H, 64)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    cross = agg.make_cross(1, NQ, NK, H)
    for at in (0, 40, NK // 2, NK - 1):
        q2, k2 = q.clone(), k.clone()
        q2[:, ::2] = (8 * u).to(torch.bfloat16)        # logit 64 * 64 / 8 = 512 with that key, at every other query
        k2[:, at] = (8 * u).to(torch.bfloat16)
        k2[:, (at + 7) % NK] = (-8 * u).to(torch.bfloat16)
        check(cross, harness.cross_forward(cross, q2, k2, v), q2, k2, v, what="spike at %d" % at)
        pages, n = pages_of(g, 1, -(-NK // 64))
        pools = harness.make_pools(n, H, "cuda")
        put(pools, pages, k2, v)
        check(cross, harness.cache_forward(agg.make_cache(*pools, pages, H), cross, q2), q2, k2, v, what="cached spike at %d" % at)
    # all logits far below zero, and far above
    for sign in (-1, 1):
        q2, k2 = (8 * u).to(torch.bfloat16).expand_as(q).contiguous(), k.clone()
        k2 += (sign * 6 * u).to(torch.bfloat16)
        check(cross, harness.cross_forward(cross, q2, k2, v), q2, k2, v, what="shifted %d" % sign)


# a size for each wide kernel, with and without shared out keys: B, NQ, NK, H
REDO = [(20, 440, 100, 16), (24, 512, 400, 16), (20, 520, 130, 16), (1, 1374, 9000, 16), (1, 2816, 8000, 16), (2, 440, 5000, 12),
        (20, 100, 100, 4), (20, 100, 2000, 4), (24, 65, 1029, 4), (6, 65, 2000, 16)]


@pytest.mark.parametrize("B, NQ, NK, H", REDO)
def test_rows_redone_on_every_route(B, NQ, NK, H):
    """Logits that leave the fast path's range in one workgroup, and in all, early and late among the keys."""
    say("redone", B, NQ, NK, H)
    g = gen(13)
    q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H, 64, scale=0.5), bf16(g, B, NK, H, 64)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    cross = agg.make_cross(B, NQ, NK, H)
    for rows, at in ((slice(NQ - 1, NQ), 3), (slice(0, NQ, 50), NK - 2)):
        q2, k2 = q.clone(), k.clone()
        q2[:, rows] = (6 * u).to(torch.bfloat16)  # logit 6 * 6 * 64 / 8 = 288 with that key, -288 with its neighbour
        k2[:, at] = (6 * u).to(torch.bfloat16)
        k2[:, at + 1] = (-6 * u).to(torch.bfloat16)
        check(cross, harness.cross_forward(cross, q2, k2, v), q2, k2, v, what="rows %s key %d" % (rows, at))
        pages, n = pages_of(g, B, -(-NK // 64))
        pools = harness.make_pools(n, H, "cuda")
        put(pools, pages, k2, v)
        check(cross, harness.cache_forward(agg.make_cache(*pools, pages, H), cross, q2), q2, k2, v, what="cached, key %d" % at)


@pytest.mark.parametrize("NQ, H", [(3, 2), (50, 2), (300, 2), (300, 16), (600, 32)])
def test_rows_that_are_no_numbers(NQ, H):
    """A query that is NaN spoils its own row, a key that is NaN its sequence, a value that is NaN its channel."""
    say("not numbers", NQ, H)
    g = gen(9)
    q, k, v = bf16(g, 2, NQ, H, 64), bf16(g, 2, 200, H, 64), bf16(g, 2, 200, H, 64)
    cross = agg.make_cross(2, NQ, 200, H)
    want, _ = harness.cross_forward(cross, q, k, v)
    _, _, size, dots = orc.attention(q, k, v, 0.125)
    q2 = q.clone()
    q2[0, 1, 1, 5] = math.nan
    o, lse = harness.cross_forward(cross, q2, k, v)
    torch.cuda.synchronize()
    assert bool(torch.isnan(o[0, 1, 1]).all()) and bool(torch.isnan(lse[0, 1, 1]))
    # (rows that share a workgroup with it may have taken the other path: not the same bits)
    off = (o.double() - want.double()).abs() > (4 * HALF + 2.0 ** -11 * (1 + dots)) * size + 2 * HALF * want.double().abs()
    off[0, 1, 1] = False
    keep = torch.ones_like(off)
    keep[0, 1, 1] = False
    assert not bool((off & keep).any()) and bool(torch.isfinite(o[keep]).all())
    k2, v2 = k.clone(), v.clone()
    k2[1, 70, 0, 3] = math.nan
    v2[0, 199, 1, 9] = math.nan
    o, _ = harness.cross_forward(cross, q, k2, v2)
    torch.cuda.synchronize()
    bad = torch.isnan(o)
    assert bool(bad[1, :, 0].all()) and bool(bad[0, :, 1, 9].all()) and int(bad.sum()) == NQ * 64 + NQ
    k2, v2 = k.clone(), v.clone()
    v2[0, 199, 1, 9] = math.inf  # ... an infinite one its channel, which is infinite
    o, _ = harness.cross_forward(cross, q, k2, v2)
    torch.cuda.synchronize()
    assert bool((o[0, :, 1, 9] == math.inf).all()) and int(torch.isfinite(o).logical_not().sum()) == NQ


@pytest.mark.parametrize("NQ, NK, H_kv", [(1, 3000, 3), (40, 301, 3), (300, 777, 3), (300, 777, 24), (600, 777, 24)])
def test_strides(NQ, NK, H_kv):
    """Keys and values side by side, queries among other channels: the results of contiguous ones, to the bit."""
    say("strides", NQ, NK, H_kv)
    g = gen(10)
    B, H = 2, 2 * H_kv
    q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H_kv, 64), bf16(g, B, NK, H_kv, 64)
    lens = ints([NK - 5, NK])
    cross = agg.make_cross(B, NQ, NK, H, H_kv, k_lens=lens)
    want = harness.cross_forward(cross, q, k, v)
    check(cross, want, q, k, v, None, lens.tolist(), "contiguous")
    wide_q = torch.full((B, NQ, H + 1, 64), math.nan, dtype=torch.bfloat16, device="cuda")
    wide_q[:, :, 1:] = q
    wide = torch.full((B, NK, 2 * H_kv * 64 + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :, :H_kv * 64] = k.reshape(B, NK, -1)
    wide[:, :, H_kv * 64:2 * H_kv * 64] = v.reshape(B, NK, -1)
    s = wide.shape[2]
    got = harness.cross_forward(cross, wide_q[:, :, 1:], wide, wide[:, :, H_kv * 64:], (H + 1) * 64, s, s)
    pages, n = pages_of(g, B, -(-NK // 64))
    pools = harness.make_pools(n, H_kv, "cuda")
    put(pools, pages, k, v)
    cache = agg.make_cache(*pools, pages, H_kv)
    a, b = harness.cache_forward(cache, cross, q), harness.cache_forward(cache, cross, wide_q[:, :, 1:], (H + 1) * 64)
    torch.cuda.synchronize()
    for x, y in zip(want + a, got + b):
        assert same_bits(x, y)


@pytest.mark.parametrize("H", [2, 32])
def test_shared_and_foreign_pages(H):
    """Sequences over one row of the table with lengths of their own, and page numbers outside the pool, which are read as
    the first or the last page."""
    say("pages", H)
    g = gen(11)
    NK = 500
    k, v = bf16(g, 1, NK, H, 64), bf16(g, 1, NK, H, 64)
    pages, n = pages_of(g, 1, 8)
    pools = harness.make_pools(n, H, "cuda", fill=0)
    put(pools, pages, k, v)
    lens = [100, 250, 500, 0, 33]
    for NQ in (2, 150, 600):
        q = bf16(g, 5, NQ, H, 64)
        shared = pages.expand(5, 8).contiguous()
        kl = ints(lens)
        cross = agg.make_cross(5, NQ, NK, H, k_lens=kl)
        got = harness.cache_forward(agg.make_cache(*pools, shared, H), cross, q)
        check(cross, got, q, k.expand(5, -1, -1, -1), v.expand(5, -1, -1, -1), None, lens, "shared pages")
        wild = shared.clone()
        wild[0, 1], wild[1, 3], wild[2, 0] = -5, n + 9, 2 ** 31 - 1
        tame = wild.clamp(0, n - 1)
        a = harness.cache_forward(agg.make_cache(*pools, wild, H), cross, q)
        b = harness.cache_forward(agg.make_cache(*pools, tame, H), cross, q)
        torch.cuda.synchronize()
        assert same_bits(a[0], b[0]) and same_bits(a[1], b[1])


# ---- appending -----------------------------------------------------------------------------------
PAIRINGS = [agg.AGG_ROPE_SECTIONS, agg.AGG_ROPE_NEIGHBOURS, agg.AGG_ROPE_HEAD]
KINDS = {"none": agg.AGG_NORM_NONE, "layer": agg.AGG_NORM_LAYER, "rms": agg.AGG_NORM_RMS}


def f64(t):
    return None if t is None else t.detach().double().cpu().numpy()


def norm_of(g, kind, affine=True):
    gamma = 1 + 0.3 * torch.randn(64, generator=g, device="cuda") if affine else None
    beta = 0.3 * torch.randn(64, generator=g, device="cuda") if affine else None
    return agg.make_norm(KINDS[kind], 1e-5, gamma, beta), (KINDS[kind], float(np.float32(1e-5)), f64(gamma), f64(beta))


def turned(x, spec, at, pairing, axes, base):
    """What norm and rotation have to give of x [tokens, H, 64], and the tolerance: half a step of bf16; 2^-15 of the largest value
    in units of the deviation for the norm's float32 sums of 64; 1e-6 of a pair's magnitudes for angle, sine and sums."""
    n = ops.norm(x, *spec)
    err = np.zeros_like(n)
    if spec[0] != agg.AGG_NORM_NONE:
        d = x - x.mean(-1, keepdims=True) if spec[0] == agg.AGG_NORM_LAYER else x
        top = np.abs(d).max(-1, keepdims=True) / np.sqrt((d * d).mean(-1, keepdims=True) + spec[1])
        err = 2.0 ** -15 * (top * (1 if spec[2] is None else np.abs(spec[2])) + (0 if spec[3] is None else np.abs(spec[3])))
        err = np.broadcast_to(err, n.shape).copy()
    want = ops.rope(n, at, pairing, axes, base)
    size = np.abs(n)
    for a, b, _, _ in ops.rope_pairs(pairing, axes, base):
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
        err[..., a] = err[..., b] = err[..., a] + err[..., b]
    return want, HALF * np.abs(want) + 1e-6 * size + err


def append_case(shape, H_kv, start=None, counts=None, pairing=agg.AGG_ROPE_SECTIONS, axes=(0, 32, 32), kind="layer", base=100.0,
                t0=3, patch0=1, given=False, queries=True, strided=False, max_pages=None, wild=False, seed=21, rope=True):
    B, T, H = shape.B, shape.NQ, shape.H
    say("append B %d T %d H %d/%d start %s counts %s" % (B, T, H, H_kv, start, counts))
    g = gen(seed)
    s0 = [0] * B if start is None else start
    cap = max_pages or max(1, -(-(max(s0) + T) // 64))
    pages, n = pages_of(g, B, cap)
    if wild:
        pages[0, 0], pages[-1, -1] = -7, n + 5
    # the new rows among others, which have to stay
    q, k, v = bf16(g, B, T, H, 64, scale=1.5), bf16(g, B, T, H_kv, 64, scale=3.0), bf16(g, B, T, H_kv, 64)
    stride = 0
    if strided:
        wide = torch.full((B, T, H + 2 * H_kv, 64), math.nan, dtype=torch.bfloat16, device="cuda")
        for t, lo in ((q, 0), (k, H), (v, H + H_kv)):
            wide[:, :, lo:lo + t.shape[2]] = t
        q, k, v = wide[:, :, :H], wide[:, :, H:H + H_kv], wide[:, :, H + H_kv:]
        stride = (H + 2 * H_kv) * 64
    pools = harness.make_pools(n, H_kv, "cuda")
    for p in pools:
        p.copy_(bf16(g, *p.shape))
    before = [p.clone() for p in pools]
    qr = harness._buf((B, T, H, 64), torch.bfloat16, "cuda", "Qr")
    qr.view(torch.int16).fill_(0x7FC1)
    lens = harness._buf((B,), torch.int32, "cuda", "lens")
    lens.fill_(-1)
    r = agg.make_rope(pairing, *axes, base=base, t0=t0, patch0=patch0) if rope else None
    (qn, q_spec), (kn, k_spec) = norm_of(g, kind), norm_of(g, kind, affine=H_kv != 5)
    at = np.tile(ops.grid_positions(shape.N, shape.n_h, shape.n_w, shape.n_special, t0, patch0), (B, 1)).reshape(B, T, 3)
    pos = None
    if given:
        at = np.random.RandomState(seed).randint(-2 ** 31, 2 ** 31, (B, T, 3))
        pos = ints(at)
    cache = agg.make_cache(*pools, pages, H_kv)
    agg.agg_cache_append(cache, shape, r, qn, kn, pos, q if queries else None, stride, k, stride, v, stride,
                         None if start is None else ints(start), None if counts is None else ints(counts), lens,
                         qr if queries else None)
    torch.cuda.synchronize()
    number = [T if counts is None else min(max(c, 0), T) for c in (counts or [T] * B)]
    assert lens.tolist() == [min(max(s + c, 0), 64 * cap) for s, c in zip(s0, number)]
    ax = axes if rope else (0, 0, 0)
    exp_v, exp_k = before[1].clone(), before[0].double()
    tol_k = torch.zeros_like(exp_k)
    for b in range(B):
        want, tol = turned(f64(k[b]), k_spec, at[b], pairing, ax, float(np.float32(base)))
        want, tol = (torch.tensor(x, device="cuda") for x in (want, tol))
        tokens = torch.arange(number[b], device="cuda")
        rows = s0[b] + tokens
        inside = (rows >= 0) & (rows < 64 * cap)
        rows, tokens = rows[inside], tokens[inside]
        page = pages[b, rows // 64].long()
        inside = (page >= 0) & (page < n)
        rows, tokens, page = rows[inside], tokens[inside], page[inside][:, None]
        for h in range(H_kv):
            exp_v[page, h, orc._places(orc.v_place, "cuda")[rows % 64]] = v[b, tokens, h]
            exp_k[page, h, orc._places(orc.k_place, "cuda")[rows % 64]] = want[tokens, h]
            tol_k[page, h, orc._places(orc.k_place, "cuda")[rows % 64]] = tol[tokens, h]
        if queries:
            want, tol = turned(f64(q[b]), q_spec, at[b], pairing, ax, float(np.float32(base)))
            c = number[b]
            assert (np.abs(f64(qr[b, :c]) - want[:c]) <= tol[:c]).all(), "queries"
            assert bool((qr[b, c:].contiguous().view(torch.int16) == 0x7FC1).all()), "queries that do not exist"
    assert same_bits(pools[1], exp_v), "values"
    off = (pools[0].double() - exp_k).abs()
    assert bool((off <= tol_k).all()), "keys: %d off" % int((off > tol_k).sum())


def frames(B, N, n_h, n_w, P, H):
    return agg.make_shape(B, N, n_h, n_w, P, H, 64, 1, 1)


@pytest.mark.parametrize("T", [1, 2, 5, 31, 33, 70, 130])
@pytest.mark.parametrize("start", [0, 1, 3, 7, 8, 31, 32, 45, 63, 64, 100])
def test_append_places(T, start):
    append_case(frames(1, 1, 1, T, 0, 2), 2, [start])


@pytest.mark.parametrize("pairing", PAIRINGS)
@pytest.mark.parametrize("axes", [(0, 32, 32), (16, 24, 24), (64, 0, 0), (0, 0, 2), (20, 22, 14), (0, 0, 0)])
def test_append_pairings(pairing, axes):
    append_case(frames(2, 3, 3, 5, 2, 4), 2, [5, 60], pairing=pairing, axes=axes, kind="rms", base=10000.0, t0=-4)


@pytest.mark.parametrize("kind", ["none", "layer", "rms"])
@pytest.mark.parametrize("H, H_kv", [(1, 1), (3, 3), (5, 5), (8, 2), (9, 9), (16, 4), (33, 11)])
def test_append_heads_and_norms(H, H_kv, kind):
    append_case(frames(1, 2, 3, 3, 2, H), H_kv, [17], kind=kind, strided=True)


def test_append_ragged_and_out_of_range():
    """Tokens that do not exist, sequences that begin before the first row or end behind the last page, pages that are none."""
    append_case(frames(5, 1, 6, 7, 0, 2), 2, [0, 9, 64, 33, 200], [42, 0, 7, -1, 50])
    append_case(frames(4, 1, 6, 7, 0, 2), 2, [-10, -50, 100, 2 ** 31 - 1], None, max_pages=2)
    append_case(frames(3, 1, 6, 7, 0, 4), 2, [70, 110, 128], [42, 40, 3], max_pages=2, queries=False)
    append_case(frames(2, 1, 10, 10, 0, 2), 1, [3, 30], wild=True)


def test_append_given_positions_and_parts_left_out():
    append_case(frames(2, 1, 5, 5, 1, 4), 4, [1, 2], given=True, pairing=agg.AGG_ROPE_HEAD, axes=(16, 24, 24))
    append_case(frames(2, 1, 5, 5, 1, 4), 4, None, rope=False, kind="rms")
    append_case(frames(2, 1, 5, 5, 1, 4), 2, [62, 3], rope=False, kind="none", strided=True)


@pytest.mark.parametrize("pairing, axes", [(agg.AGG_ROPE_SECTIONS, (0, 32, 32)), (agg.AGG_ROPE_NEIGHBOURS, (16, 24, 24)),
                                           (agg.AGG_ROPE_SECTIONS, (20, 22, 14)), (agg.AGG_ROPE_HEAD, (0, 0, 0))])
def test_append_many_rows(pairing, axes):
    """More rows than pieces of 16 take: pieces of 32, beginning and ending inside one."""
    append_case(frames(3, 9, 37, 37, 5, 7), 7, [5, 49, 64], [12366, 5401, 9000], pairing=pairing, axes=axes, strided=True)
    append_case(frames(5, 8, 37, 37, 5, 6), 6, [1, 31, 4000, 0, 77], None, pairing=pairing, axes=axes, kind="rms", max_pages=200, queries=axes[1] != 24)
    append_case(frames(3, 2, 37, 37, 5, 3), 3, [5, 49, 64], [2748, 1401, 2000], pairing=pairing, axes=axes, strided=True)


def test_append_a_frame():
    append_case(frames(1, 1, 37, 37, 5, 16), 16, [1374 * 2 + 11])


def test_append_queries_in_place_are_those_of_the_rotary_call():
    """Queries come out as agg_rope_fwd turns them, also over their input."""
    say("append in place")
    g = gen(23)
    shape = frames(2, 2, 6, 5, 3, 8)
    q, k, v = bf16(g, 2, shape.NQ, 8, 64), bf16(g, 2, shape.NQ, 4, 64), bf16(g, 2, shape.NQ, 4, 64)
    rope = agg.make_rope(agg.AGG_ROPE_HEAD, 16, 24, 24, t0=9, patch0=2)
    n, _ = norm_of(g, "layer")
    want, _ = harness.rope_forward(shape, rope, q, None, n)
    pages, pool = pages_of(g, 2, 3)
    cache = agg.make_cache(*harness.make_pools(pool, 4, "cuda"), pages, 4)
    agg.agg_cache_append(cache, shape, rope, n, n, None, q, 0, k, 0, v, 0, None, None, None, q)
    torch.cuda.synchronize()
    assert same_bits(q, want)


# ---- as they are used ----------------------------------------------------------------------------
def test_a_stream_of_frames():
    """Frames arrive one after another: each is appended, its tokens attend to it and to all before it.  The same by one call
    over the whole clip, a frame being a sequence of its own length over the shared pages, and by the oracle."""
    say("stream")
    g = gen(31)
    N, H, H_kv = 6, 8, 4
    one, clip = frames(1, 1, 9, 11, 3, H), frames(1, N, 9, 11, 3, H)
    L = one.NQ
    q, k, v = bf16(g, 1, N * L, H, 64, scale=1.5), bf16(g, 1, N * L, H_kv, 64, scale=1.5), bf16(g, 1, N * L, H_kv, 64)
    (qn, _), (kn, _) = norm_of(g, "layer"), norm_of(g, "layer")
    entries = -(-N * L // 64)
    pages, pool = pages_of(g, 1, entries)
    pools = harness.make_pools(pool, H_kv, "cuda")
    cache = agg.make_cache(*pools, pages, H_kv)
    lens = [ints([0]), ints([0])]
    got, turned_q = [], []
    for f in range(N):
        rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 16, 24, 24, t0=f, patch0=1)
        part = slice(f * L, (f + 1) * L)
        qr = harness._buf((1, L, H, 64), torch.bfloat16, "cuda", "Qr")
        agg.agg_cache_append(cache, one, rope, qn, kn, None, q[:, part].contiguous(), 0, k[:, part].contiguous(), 0,
                             v[:, part].contiguous(), 0, lens[f % 2], None, lens[(f + 1) % 2], qr)
        cross = agg.make_cross(1, L, 64 * entries, H, H_kv, k_lens=lens[(f + 1) % 2])
        got.append(harness.cache_forward(cache, cross, qr))
        turned_q.append(qr)
    # the whole clip at once, into pages of its own
    other = harness.make_pools(pool, H_kv, "cuda")
    qr = harness._buf((1, N * L, H, 64), torch.bfloat16, "cuda", "Qr")
    rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 16, 24, 24, patch0=1)
    agg.agg_cache_append(agg.make_cache(*other, pages, H_kv), clip, rope, qn, kn, None, q, 0, k, 0, v, 0, None, None, None, qr)
    torch.cuda.synchronize()
    assert same_bits(qr, torch.cat(turned_q, 1))
    rows = [orc.rows_of(p, pages, place)[:, :N * L] for p, place in zip(other, (orc.k_place, orc.v_place))]
    for a, (p, place) in zip(rows, zip(pools, (orc.k_place, orc.v_place))):
        assert same_bits(a.contiguous(), orc.rows_of(p, pages, place)[:, :N * L].contiguous())
    by_frame = agg.make_cross(N, L, 64 * entries, H, H_kv, k_lens=ints([(f + 1) * L for f in range(N)]))
    shared = agg.make_cache(*other, pages.expand(N, entries).contiguous(), H_kv)
    at_once = harness.cache_forward(shared, by_frame, qr.view(N, L, H, 64))
    kk, vv = (r.expand(N, -1, -1, -1) for r in rows)
    check(by_frame, at_once, qr.view(N, L, H, 64), kk, vv, None, [(f + 1) * L for f in range(N)], "clip")
    for f in range(N):
        cross = agg.make_cross(1, L, N * L, H, H_kv)
        check(cross, got[f], turned_q[f], rows[0], rows[1], None, [(f + 1) * L], "frame %d" % f)


def test_streams_and_graphs():
    """A captured step of a stream, replayed with new inputs, starts and lengths; and two streams at once, each with a
    workspace of its own."""
    say("graphs")
    g = gen(32)
    H, NK = 4, 9000
    shape = frames(2, 1, 1, 6, 0, H)
    pages, pool = pages_of(g, 2, -(-NK // 64))
    pools = harness.make_pools(pool, H, "cuda", fill=0)
    for p in pools:
        p.copy_(bf16(g, *p.shape))
    cache = agg.make_cache(*pools, pages, H)
    rope = agg.make_rope(agg.AGG_ROPE_HEAD, 16, 24, 24)
    q, k, v = (bf16(g, 2, 6, H, 64) for _ in "qkv")
    many_q, mk, mv = bf16(g, 1, 600, H, 64), bf16(g, 1, 3000, H, 64), bf16(g, 1, 3000, H, 64)
    start, lens, pos = ints([0, 0]), ints([0, 0]), ints(np.zeros((2, 6, 3)).tolist())
    cross, many = agg.make_cross(2, 6, NK, H, k_lens=lens), agg.make_cross(1, 600, 3000, H)
    qr, o, om = torch.empty_like(q), torch.empty_like(q), torch.empty_like(many_q)
    lse, lm = torch.empty((2, H, 6), device="cuda"), torch.empty((1, H, 600), device="cuda")
    n, nm = agg.agg_cross_workspace_bytes(cross), agg.agg_cross_workspace_bytes(many)
    assert n > 0 and nm > 0
    ws = [torch.empty(x, dtype=torch.uint8, device="cuda") for x in (n, nm)]

    def run():
        agg.agg_cache_append(cache, shape, rope, None, None, pos, q, 0, k, 0, v, 0, start, None, lens, qr)
        agg.agg_cache_attn_fwd(cache, cross, qr, 0, o, lse, ws[0], n)
        agg.agg_cross_attn_fwd(many, many_q, 0, mk, 0, mv, 0, om, lm, ws[1], nm)

    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(4):
        for t in (q, k, v, many_q, mk):
            t.copy_(bf16(g, *t.shape))
        start.copy_(ints([100 * i, 8000 - 1500 * i]))
        pos.copy_(torch.randint(0, 1000, pos.shape, generator=g, device="cuda", dtype=torch.int32))
        kept = [p.clone() for p in pools]
        run()
        want = [t.clone() for t in (o, lse, qr, om, lm, *pools)]
        for p, b in zip(pools, kept):
            p.copy_(b)
        for t in (o, lse, qr, om, lm):
            t.zero_()
        lens.zero_()
        for w in ws:
            w.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((o, lse, qr, om, lm, *pools), want):
            assert same_bits(a, b), i
        assert lens.tolist() == [100 * i + 6, 8000 - 1500 * i + 6]
    # two streams
    streams = [torch.cuda.Stream() for _ in range(2)]
    want = harness.cross_forward(many, many_q, mk, mv)
    outs = [(torch.empty_like(om), torch.empty_like(lm), torch.empty(nm, dtype=torch.uint8, device="cuda")) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(3):
        for s, (a, b, w) in zip(streams, outs):
            with torch.cuda.stream(s):
                agg.agg_cross_attn_fwd(many, many_q, 0, mk, 0, mv, 0, a, b, w, nm)
    torch.cuda.synchronize()
    for a, b, _ in outs:
        assert same_bits(a, want[0]) and same_bits(b, want[1])


def test_results_repeat_to_the_bit():
    say("repeat")
    g = gen(33)
    for B, NQ, NK, H in ((1, 1, 30000, 3), (2, 50, 4000, 3), (1, 700, 5000, 3), (1, 1374, 9000, 16), (6, 65, 2000, 16)):
        q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H, 64), bf16(g, B, NK, H, 64)
        cross = agg.make_cross(B, NQ, NK, H)
        first = harness.cross_forward(cross, q, k, v)
        for _ in range(3):
            again = harness.cross_forward(cross, q, k, v)
            torch.cuda.synchronize()
            assert same_bits(first[0], again[0]) and same_bits(first[1], again[1])


# ---- sizes beyond 32 bits ------------------------------------------------------------------------
@pytest.mark.parametrize("NQ", [3, 200, 1500])
def test_offsets_beyond_32_bits(NQ):
    """A pool of 9 GiB whose used pages lie at its end, and rows 2 MiB apart."""
    say("far offsets", NQ)
    g = gen(34)
    H, NK = 16, 400
    n_pages = 73000
    pools = [torch.zeros((n_pages, H, 4096), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    pages = ints([[n_pages - 1 - 3 * i for i in range(7)]])
    q, k, v = bf16(g, 1, NQ, H, 64), bf16(g, 1, NK, H, 64), bf16(g, 1, NK, H, 64)
    cache = agg.make_cache(*pools, pages, H)
    lens = ints([0])
    agg.agg_cache_append(cache, frames(1, 1, 20, 20, 0, H), None, None, None, None, None, 0, k, 0, v, 0, None, None, lens)
    torch.cuda.synchronize()
    assert lens.tolist() == [NK]
    for p, t, place in zip(pools, (k, v), (orc.k_place, orc.v_place)):
        assert same_bits(orc.rows_of(p, pages, place)[:, :NK].contiguous(), t)
    cross = agg.make_cross(1, NQ, NK, H)
    check(cross, harness.cache_forward(cache, cross, q), q, k, v, what="far pages")
    del pools, cache
    stride = 1 << 20
    wide = torch.zeros(2 * NK * stride // 2 + stride, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(wide, (NK, H * 64), (stride, 1))
    beside = torch.as_strided(wide, (NK, H * 64), (stride, 1), H * 64)
    rows.copy_(k.view(NK, -1))
    beside.copy_(v.view(NK, -1))
    check(cross, harness.cross_forward(cross, q, wide, wide[H * 64:], 0, stride, stride), q, k, v, what="far rows")


def test_more_pairs_than_a_launch_counts():
    """2^22 (batch element, key head) pairs and some, of one query and two keys; joined results of as many rows."""
    say("many pairs")
    g = gen(35)
    B, H = (1 << 20) + 3, 5
    q, k, v = (bf16(g, B, n, H, 64) for n in (1, 2, 2))
    o, lse = harness.cross_forward(agg.make_cross(B, 1, 2, H), q, k, v)
    logit = (q.double() * k.double()).sum(-1) / 8  # [B, 2, H]
    p = torch.softmax(logit, 1)[..., None]
    want = (p * v.double()).sum(1)
    size = (p * v.double().abs()).sum(1)
    S = ((q.double() * k.double()).abs().sum(-1) / 8).amax(1)[..., None]
    tol = (2 * HALF + 2.0 ** -12 * (1 + S)) * size + HALF * want.abs()
    assert bool(((o[:, 0].double() - want).abs() <= tol).all())
    assert bool(((lse[:, :, 0].double() - torch.logsumexp(logit, 1)).abs() <= 2.0 ** -10 + 2.0 ** -16 * S[..., 0]).all())
