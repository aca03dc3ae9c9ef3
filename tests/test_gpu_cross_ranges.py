"""Attention to keys of another length where logits and values lie far apart, on the GPU, against float64.

Tolerances count roundings of the keys that carry weight, and of no others.  With p a key's probability, S the sum of |scale q k| over its
channels (S* that of the row's largest logit) and v its value:
  a logit is a sum of 64 exact products in float32: 64 * 2^-24 = 2^-18 of S, and so is the largest, which the others are taken relative to:
      d = 2^-18 (S + S*)
  O    a probability is rounded to bf16 on its way into the second product, 2^-8, and the sum may hold the rounded or the unrounded
       ones, 2^-8 more; float32 steps behind it 2^-12: sum of p (2^-7 + 2^-12 + d) |v|, by the sum |O| sum of p d, by the result's rounding 2^-8 |O|
  lse  sum of p d; 2^-16 (1 + |lse|) for the logarithm and the base; 2^-8 where the sum is that of rounded probabilities
Keys whose probability is zero in float64 count as nothing, whatever their logit.
That is first order in d.  Where d reaches 1/2 for a key within d of the row's largest logit (logits of 10^5 and more), float32 cannot tell which
keys weigh most: O has to be some mean of values, no further from the right one than twice the largest, and lse within the largest d.
"""
import math

import numpy as np
import pytest
import torch

from oracle import cache_oracle as orc
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import harness

from test_gpu_cross import bf16, both, check, gen, ints, norm_of, pages_of, put, same_bits, say

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8
DOT = 2.0 ** -18


def judge(cross, got, q, k, v, what):
    """O and lse of calls without lengths.  Where float64 has no number, O has to be none either."""
    torch.cuda.synchronize()
    o, lse = got
    scale, group = float(np.float32(cross.scale)), cross.H // cross.H_kv
    for b in range(cross.B):
        for h in range(cross.H):
            qh, kh, vh = (x.double() for x in (q[b, :, h], k[b, :, h // group], v[b, :, h // group]))
            logit = (qh @ kh.t().contiguous()) * scale
            p = torch.softmax(logit, -1)
            S = (qh.abs() @ kh.abs().t().contiguous()) * scale
            top = logit.argmax(1, keepdim=True)
            d = DOT * (S + S.gather(1, top))
            near = logit.gather(1, top) - logit <= d
            most = torch.where(near & torch.isfinite(d), d, torch.zeros_like(d)).amax(1, keepdim=True)
            d = torch.where(p > 0, d, torch.zeros_like(d))
            want = p @ vh
            pd = (p * d).sum(1, keepdim=True)
            tol = (p * (2 * HALF + 2.0 ** -12 + d)) @ vh.abs() + want.abs() * (pd + HALF)
            pd = torch.where(most < 0.5, pd, most)
            tol = torch.where(most < 0.5, tol, (2 + HALF) * vh.abs().amax(0))
            off = (o[b, :, h].double() - want).abs()
            none = torch.isnan(want)
            assert bool(torch.isnan(o[b, :, h])[none].all()), what + ": numbers where there are none"
            bad = ~(off <= tol) & ~none
            assert not bool(bad.any()), "%s, element %d head %d: %d of O off, worst %.3g of the tolerance" % (
                what, b, h, int(bad.sum()), float((off / tol)[~none].nan_to_num(1e9).max()))
            wl = torch.logsumexp(logit, -1)
            loff = (lse[b, h].double() - wl).abs()
            assert bool((lse[b, h][wl == -math.inf] == -math.inf).all()), what
            there = ~none[:, 0]
            lbad = there & ~(loff <= pd[:, 0] + HALF + 2.0 ** -16 * (1 + wl.abs()))
            assert not bool(lbad.any()), "%s, element %d head %d: %d of lse off, worst %.3g" % (
                what, b, h, int(lbad.sum()), float(loff[there].nan_to_num(1e9).max()))


def both_places(q, k, v, what):
    """The call with keys in place and out of a cache."""
    (B, NQ, H, _), (_, NK, H_kv, _) = q.shape, k.shape
    cross = agg.make_cross(B, NQ, NK, H, H_kv)
    say(what, "in place")
    judge(cross, harness.cross_forward(cross, q, k, v), q, k, v, what)
    pages, n = pages_of(gen(99), B, -(-NK // 64))
    pools = harness.make_pools(n, H_kv, "cuda")
    put(pools, pages, k, v)
    say(what, "paged")
    judge(cross, harness.cache_forward(agg.make_cache(*pools, pages, H_kv), cross, q), q, k, v, what + " paged")


# B, NQ, NK, H: every wide kernel, keys shared out or not, joined by one and by sixteen groups of lanes, and the kernel of few rows
KERNELS = [(20, 440, 100, 16), (6, 512, 400, 64), (20, 520, 130, 16), (1, 1374, 9000, 16), (1, 2816, 8000, 16), (2, 440, 5000, 12),
           (20, 100, 100, 4), (20, 100, 2000, 4), (24, 65, 1029, 4), (6, 65, 2000, 16), (1, 1374, 9000, 1), (2, 700, 9000, 2), (1, 700, 20000, 1),
           (1, 20, 7001, 2), (1, 1, 20001, 2)]


def spikes(q, k, u, at):
    """Every fiftieth query leaves the fast path's window by the keys `at`: logits of some 280."""
    q[:, ::50, :, 1:] = (6 * u[1:]).to(torch.bfloat16)
    k[:, at, :, 1:] = (6 * u[1:]).to(torch.bfloat16)


@pytest.mark.parametrize("B, NQ, NK, H", KERNELS)
def test_keys_hidden_by_value(B, NQ, NK, H):
    """A channel of the keys hides the first half of every tile of 64, the keys that any share of a sequence begins with: by a little, by much and
    by -infinity; the others at ordinary logits, and far below zero."""
    g = gen(41)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H, 64, scale=0.5), bf16(g, B, NK, H, 64)
    q[..., 0], k[..., 0] = 1.0, 0.0
    spikes(q, k, u, [NK - 1])
    hidden = torch.arange(NK, device="cuda") % 64 < 32
    hidden[NK - 1] = False
    for mask in (-8e4, -8e6, -8e9, -math.inf):
        for below in (0, -160):
            k2 = k.clone()
            k2[..., 0] = below * 8.0
            k2[:, hidden, :, 0] = mask
            both_places(q, k2, v, "hidden by %g, others at %d" % (mask, below))


# keys shared out, by the plan in 2 to 40: wide kernels alone and in halves, joined by one and by sixteen groups of lanes
SHARED = [(1, 1374, 9000, 16), (1, 2816, 8000, 16), (2, 440, 5000, 12), (20, 100, 2000, 4), (6, 65, 2000, 16), (1, 1374, 9000, 1),
          (2, 700, 9000, 2), (1, 700, 20000, 1), (1, 20, 7001, 2)]


@pytest.mark.parametrize("B, NQ, NK, H", SHARED)
def test_shares_of_the_keys_count_by_their_sums(B, NQ, NK, H):
    """The last share holds nearly all of a row's weight but begins with keys far below it, and is redone for another row's sake; the other
    shares are not.  Their references say nothing about their sums."""
    g = gen(42)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    q, k = bf16(g, B, NQ, H, 64, scale=0.1), bf16(g, B, NK, H, 64, scale=0.1)
    v = bf16(g, B, NK, H, 64, scale=0.2)
    q[..., 0], k[..., 0] = 8.0, -55.0
    key, tiles = torch.arange(NK, device="cuda"), -(-NK // 64)
    for shares in (2, 3, 4, 5, 10, 21, 40):
        last = key >= 64 * (tiles * (shares - 1) // shares)
        q2, k2, v2 = q.clone(), k.clone(), v.clone()
        k2[:, last, :, 0] = -42.0
        k2[:, last & (key % 64 < 32), :, 0] = -104.0
        v2[:, last] += 1
        v2[:, ~last] -= 1
        spikes(q2, k2, u, last & (key % 64 == 63))
        both_places(q2, k2, v2, "last of %d shares" % shares)


@pytest.mark.parametrize("B, NQ, NK, H", SHARED + [(1, 1, 20001, 2), (1, 30, 7001, 2), (1, 261, 16384, 2), (3, 5, 300, 2), (6, 512, 400, 64)])
def test_keys_at_minus_infinity(B, NQ, NK, H):
    """Keys whose logits are -infinity: whole shares of a sequence, all keys but one, and all of them, where O is no number and lse -infinity.
    The others lie at ordinary logits, and far below zero."""
    g = gen(43)
    q, k, v = bf16(g, B, NQ, H, 64, scale=0.3), bf16(g, B, NK, H, 64, scale=0.3), bf16(g, B, NK, H, 64)
    q[..., 0] = 8.0
    for below in (0.0, -150.0):
        for there in (slice(0, NK // 5), slice(4 * NK // 5, NK), slice(NK - 1, NK), slice(0, 1), slice(NK // 2, NK // 2 + 1), slice(0, 0)):
            k2 = k.clone()
            k2[..., 0] = -math.inf
            k2[:, there, :, 0] = below
            both_places(q, k2, v, "keys %s at %g" % (there, below))


@pytest.mark.parametrize("B, NQ, NK, H", KERNELS)
def test_values_of_any_size(B, NQ, NK, H):
    """Logits inside the fast path's window whose products with large or small values leave float32's, and rows that are redone relative to
    keys far below the others."""
    g = gen(44)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    q, k, v = bf16(g, B, NQ, H, 64, scale=0.3), bf16(g, B, NK, H, 64, scale=0.3), bf16(g, B, NK, H, 64)
    q[..., 0] = 8.0
    for at, size in ((45.0, 60), (45.0, -60), (-45.0, -90), (-45.0, 60), (0.0, 100), (0.0, -90)):
        k[..., 0] = at
        both_places(q, k, v * 2.0 ** size, "logits at %g, values 2^%d" % (at, size))
    k[..., 0] = 0.0
    k[:, torch.arange(NK, device="cuda") % 64 < 32, :, 0] = -45.0
    spikes(q, k, u, [NK - 1])
    for size in (60, 95, -90):
        both_places(q, k, v * 2.0 ** size, "redone, values 2^%d" % size)


@pytest.mark.parametrize("B, NQ, NK, H", KERNELS)
def test_logits_of_any_size(B, NQ, NK, H):
    """Logits of up to 10^37, where a step of float32 is many powers of two of a probability: of the first half of every tile, of all keys, and
    of all keys but the last, of either sign; rows that are redone among them."""
    g = gen(45)
    u = torch.sign(torch.randn(64, generator=g, device="cuda"))
    q, k, v = bf16(g, B, NQ, H, 64), bf16(g, B, NK, H, 64, scale=0.5), bf16(g, B, NK, H, 64)
    q[..., 0], k[..., 0] = 1.0, 0.0
    spikes(q, k, u, [NK - 1])
    key = torch.arange(NK, device="cuda")
    lowest = torch.finfo(torch.bfloat16).min
    for size in (-8e7, -8e10, -8e20, lowest, 8e10, -lowest):
        for where, there in (("half of every tile", (key % 64 < 32) & (key < NK - 1)), ("all", key >= 0), ("all but the last", key < NK - 1)):
            k2 = k.clone()
            k2[:, there, :, 0] = size
            both_places(q, k2, v, "%s at %g" % (where, size))


# ---- appending: the rotary call's numbers ---------------------------------------------------------------------
@pytest.mark.parametrize("pairing", [agg.AGG_ROPE_SECTIONS, agg.AGG_ROPE_NEIGHBOURS, agg.AGG_ROPE_HEAD])
@pytest.mark.parametrize("axes", [(0, 32, 32), (16, 24, 24), (20, 22, 14), (64, 0, 0)])
@pytest.mark.parametrize("kind, frames", [("none", 2), ("layer", 1), ("rms", 16)])
def test_appended_keys_and_queries_are_those_of_the_rotary_call(pairing, axes, kind, frames):
    """To the bit, in pieces of 16 rows and of 32, wherever a channel's other one lies."""
    say("as the rotary call", pairing, axes, kind)
    g = gen(55)
    H = 16
    shape = agg.make_shape(1, frames, 37, 37, 5, H, 64, 1, 1)
    T = shape.NQ
    q, k, v = (bf16(g, 1, T, H, 64) for _ in "qkv")
    rope, norm = agg.make_rope(pairing, *axes, base=1000.0, t0=3, patch0=1), norm_of(g, kind)[0]
    pages, pool = pages_of(g, 1, -(-(T + 21) // 64))
    pools = harness.make_pools(pool, H, "cuda")
    qr = torch.empty_like(q)
    agg.agg_cache_append(agg.make_cache(*pools, pages, H), shape, rope, norm, norm, None, q, 0, k, 0, v, 0, ints([21]), None, None, qr)
    want = harness.rope_forward(shape, rope, q, k, norm, norm)
    torch.cuda.synchronize()
    assert same_bits(qr, want[0])
    assert same_bits(orc.rows_of(pools[0], pages, orc.k_place)[:, 21:21 + T].contiguous(), want[1])


# ---- paths that only far or many things take ----------------------------------------------------------------
# ragged calls of every kernel, with and without shared out keys: B, NQ, NK, H, and whether queries end early too
RAGGED = [(2, 40, 100, 1, 0), (2, 40, 1000, 1, 0), (3, 65, 100, 32, 0), (2, 65, 5000, 16, 0), (3, 65, 9000, 4, 0), (5, 100, 1000, 16, 0),
          (3, 65, 1000, 32, 0), (2, 2816, 100, 32, 0), (5, 2816, 9000, 8, 0), (20, 520, 100, 16, 0), (5, 1374, 14000, 16, 0), (8, 700, 100, 32, 0),
          (5, 130, 14000, 32, 0), (2, 40, 100, 1, 1), (2, 40, 1000, 1, 1), (5, 100, 100, 16, 1), (5, 65, 5000, 8, 1), (5, 100, 9000, 2, 1),
          (3, 100, 1000, 32, 1), (5, 100, 1000, 16, 1), (5, 2816, 100, 16, 1), (5, 1000, 9000, 32, 1), (20, 520, 100, 32, 1),
          (8, 1374, 14000, 16, 1), (20, 700, 100, 16, 1), (8, 130, 14000, 32, 1)]


@pytest.mark.parametrize("B, NQ, NK, H, queries", RAGGED)
def test_ragged_calls_of_every_kernel(B, NQ, NK, H, queries):
    k_lens = ([NK, NK // 2, 0, NK - 1, 1, 65, NK + 3, -1] * 3)[:B]
    q_lens = ([NQ, NQ - 1, NQ, 1, NQ // 2, 0, NQ, 33] * 3)[:B] if queries else None
    both(B, NQ, NK, H, seed=51, q_lens=q_lens, k_lens=k_lens)


@pytest.mark.parametrize("NQ", [1, 20, 64, 300])
def test_rows_further_apart_than_wide_kernels_reach(NQ):
    say("far rows", NQ)
    g = gen(52)
    H, NK, stride = 2, 3, (1 << 23) + 8
    q, k, v = bf16(g, 2, NQ, H, 64), bf16(g, 2, NK, H, 64), bf16(g, 2, NK, H, 64)
    wide = torch.full((2 * NK * stride,), math.nan, dtype=torch.bfloat16, device="cuda")
    rows, beside = (torch.as_strided(wide, (2 * NK, H * 64), (stride, 1), at) for at in (0, H * 64))
    rows.copy_(k.view(2 * NK, -1))
    beside.copy_(v.view(2 * NK, -1))
    cross = agg.make_cross(2, NQ, NK, H, k_lens=ints([3, 2]))
    check(cross, harness.cross_forward(cross, q, wide, wide[H * 64:], 0, stride, stride), q, k, v, None, [3, 2], "far rows")


def test_a_batch_of_more_wide_workgroups_than_a_launch_takes():
    """2^22 sequences and five: two launches, in place and out of pages."""
    g = gen(53)
    B, H, NK = (1 << 22) + 5, 33, 2
    q = torch.randn((B, 1, H, 64), generator=g, device="cuda", dtype=torch.bfloat16)
    k, v = (torch.randn((B, NK, 1, 64), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    ql = torch.randint(0, 2, (B,), generator=g, device="cuda", dtype=torch.int32)
    kl = torch.randint(0, NK + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
    seen = torch.cat((torch.arange(20, device="cuda"), torch.arange((1 << 22) - 20, B, device="cuda"),
                      torch.randint(0, B, (100,), generator=g, device="cuda")))
    cross = agg.make_cross(B, 1, NK, H, 1, q_lens=ql, k_lens=kl)
    assert agg.agg_cross_workspace_bytes(cross) == 0
    pages = torch.randint(0, 50, (B, 1), generator=g, device="cuda", dtype=torch.int32)
    pools = [torch.randn((50, 1, 4096), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "kv"]
    o, lse = torch.empty_like(q), torch.empty((B, H, 1), device="cuda")
    some = agg.make_cross(len(seen), 1, NK, H, 1)
    for paged in (False, True):
        say("many wide workgroups", paged)
        o.view(torch.int16).fill_(0x7FC1)
        lse.fill_(math.nan)
        if paged:
            agg.agg_cache_attn_fwd(agg.make_cache(*pools, pages, 1), cross, q, 0, o, lse)
            ks, vs = (orc.rows_of(p, pages[seen], place)[:, :NK] for p, place in zip(pools, (orc.k_place, orc.v_place)))
        else:
            agg.agg_cross_attn_fwd(cross, q, 0, k, 0, v, 0, o, lse)
            ks, vs = k[seen], v[seen]
        check(some, (o[seen], lse[seen]), q[seen], ks, vs, ql[seen].tolist(), kl[seen].tolist(), "paged" if paged else "in place")
        for h in (0, H - 1):
            assert torch.equal(torch.isnan(o[:, 0, h, 5]), ql == 0) and torch.equal(torch.isnan(lse[:, h, 0]), ql == 0)


def test_more_pieces_of_new_tokens_than_a_launch_has_workgroups():
    """2^19 sequences and three of one token each, whose rows fill pages that they share: 2^20 pieces and six."""
    say("many pieces")
    g = gen(54)
    B = (1 << 19) + 3
    shape = agg.make_shape(B, 1, 1, 1, 0, 1, 64, 1, 1)
    k, v = bf16(g, B, 1, 1, 64), bf16(g, B, 1, 1, 64)
    number = torch.arange(B, device="cuda", dtype=torch.int32)
    pages, start = (number // 64).view(B, 1).contiguous(), number % 64
    pools = harness.make_pools(B // 64 + 1, 1, "cuda")
    lens = harness._buf((B,), torch.int32, "cuda", "lens")
    pos = torch.randint(0, 1000, (B, 1, 3), generator=g, device="cuda", dtype=torch.int32)
    rope, norm = agg.make_rope(agg.AGG_ROPE_SECTIONS, 0, 32, 32), agg.make_norm(agg.AGG_NORM_RMS, 1e-5)
    agg.agg_cache_append(agg.make_cache(*pools, pages, 1), shape, rope, None, norm, pos, None, 0, k, 0, v, 0, start, None, lens)
    _, turned = harness.rope_forward(shape, rope, None, k, None, norm, pos)
    torch.cuda.synchronize()
    assert torch.equal(lens, start + 1)
    table = torch.arange(B // 64 + 1, device="cuda", dtype=torch.int32).view(1, -1)
    for p, t, place in zip(pools, (turned, v), (orc.k_place, orc.v_place)):
        rows = orc.rows_of(p, table, place)[0]
        assert same_bits(rows[:B].contiguous(), t.view(B, 1, 64))
        assert bool((rows[B:].contiguous().view(torch.int16) == 0x7FC1).all())
