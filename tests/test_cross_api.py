"""Attention to keys of another length and the paged cache without a GPU: the oracle's pins, sizes, refusals and the
launch plan."""
import os
import re
import subprocess

import pytest
import torch

from oracle import cache_oracle as orc
from paper_2512_02541_amd import binding as agg
from paper_2512_02541_amd import build as b

N, S, U, A, W, O = (agg.AGG_ERR_NULL, agg.AGG_ERR_SHAPE, agg.AGG_ERR_UNSUPPORTED, agg.AGG_ERR_ALIGN, agg.AGG_ERR_WORKSPACE,
                    agg.AGG_ERR_OVERFLOW)
FAKE = 1 << 40  # addresses that no refused call touches


def at(i):
    return FAKE + (i << 34)


# ---- the oracle ----------------------------------------------------------------------------------
def test_oracle_attention_is_textbook_attention():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((2, n, h, 64), generator=g, dtype=torch.float64) for n, h in ((5, 4), (9, 2), (9, 2)))
    o, lse, size, _ = orc.attention(q, k, v, 0.125)
    kk, vv = (t.repeat_interleave(2, 2) for t in (k, v))
    want = torch.nn.functional.scaled_dot_product_attention(*(t.transpose(1, 2) for t in (q, kk, vv)), scale=0.125)
    assert torch.allclose(o, want.transpose(1, 2), atol=1e-13)
    logit = torch.einsum("bqhd,bkhd->bhqk", q, kk) / 8
    assert torch.allclose(lse, torch.logsumexp(logit, -1), atol=1e-13)
    assert bool((size >= o.abs() - 1e-13).all())
    short, sl, _, _ = orc.attention(q, k, v, 0.125, [5, 2], [0, 4])
    assert not bool(short[0].any()) and bool((sl[0] == -float("inf")).all()) and bool(torch.isnan(short[1, 2:]).all())
    alone, _, _, _ = orc.attention(q[1:, :2], k[1:, :4], v[1:, :4], 0.125)
    assert torch.equal(short[1:, :2], alone)


def test_oracle_pages_are_fragment_order_tiles():
    for place, offset in ((orc.k_place, agg.agg_kc_offset), (orc.v_place, agg.agg_vc_offset)):
        places = {place(r, d) for r in range(64) for d in range(64)}
        assert places == set(range(4096))
        assert all(place(r, d) == offset(r, d) for r in range(64) for d in range(64))


def test_oracle_pages_read_back():
    g = torch.Generator().manual_seed(2)
    pool = torch.zeros((5, 2, 4096))
    pages = torch.tensor([[3, 1], [0, 4]])
    rows = torch.randn((100, 2, 64), generator=g)
    for r in range(100):
        orc.store(pool, pages, orc.v_place, 1, r, rows[r])
    orc.store(pool, pages, orc.v_place, 1, 128, rows[0] + 1)
    orc.store(pool, pages, orc.v_place, 1, -1, rows[0] + 1)
    got = orc.rows_of(pool, pages, orc.v_place)
    assert torch.equal(got[1, :100], rows) and not bool(got[1, 100:].any()) and not bool(got[0].any())


# ---- sizes ---------------------------------------------------------------------------------------
def test_sizes():
    assert agg.agg_cache_bytes(agg.agg_cache(7, 3, 64, 2, 4, None, None, None)) == 7 * 3 * 8192
    assert agg.agg_cross_workspace_bytes(agg.make_cross(1, 1, 100, 16)) == 0
    few = agg.agg_cross_workspace_bytes(agg.make_cross(1, 1, 137400, 16))
    assert few > 0 and few % (16 * 66 * 4) == 0
    for bad in (agg.make_cross(0, 1, 1, 1), agg.make_cross(1, -1, 1, 1), agg.make_cross(1, 1, 1, 4, 3)):
        assert agg.agg_cross_workspace_bytes(bad) == 0
    with pytest.raises(agg.AggError) as e:
        agg.agg_cache_bytes(agg.agg_cache(0, 3, 64, 2, 4, None, None, None))
    assert e.value.status == S


def _status(call, *args):
    try:
        call(*args, stream=0)
    except agg.AggError as e:
        return e.status
    return 0


# ---- refusals: every one before anything is launched ------------------------------------------------
def _cross(B=2, NQ=10, NK=100, H=4, H_kv=2, D=64, scale=0.125, ql=None, kl=None, q=at(0), qs=0, k=at(1), ks=0, v=at(2), vs=0,
           o=at(3), lse=at(4), ws=None, n=0):
    c = agg.make_cross(B, NQ, NK, H, H_kv, D, scale, ql, kl)
    return _status(agg.agg_cross_attn_fwd, c, q, qs, k, ks, v, vs, o, lse, ws, n)


def test_cross_refusals():
    for bad in (dict(B=0), dict(NQ=-1), dict(NK=-1), dict(H=0), dict(H_kv=0), dict(H=4, H_kv=3), dict(D=0), dict(scale=0.0),
                dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert _cross(**bad) == S, bad
    assert _cross(D=32) == U
    assert _cross(NQ=0, q=None, k=None, v=None, o=None, lse=None) == N  # keys without an address
    assert _cross(NQ=0, NK=0, q=None, k=None, v=None, o=None, lse=None) == 0
    assert _cross(NQ=0) == 0
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(o=None)):
        assert _cross(**bad) == N, bad
    for bad in (dict(q=at(0) + 8), dict(k=at(1) + 2), dict(v=at(2) + 4), dict(o=at(3) + 8), dict(lse=at(4) + 2),
                dict(ql=at(5) + 1), dict(kl=at(5) + 2), dict(ws=at(6) + 8)):
        assert _cross(**bad) == A, bad
    for bad in (dict(qs=248), dict(qs=260), dict(qs=-256), dict(ks=120), dict(ks=132), dict(vs=64), dict(vs=129)):
        assert _cross(**bad) == S, bad
    assert _cross(qs=1 << 57) == O and _cross(ks=1 << 56) == O and _cross(vs=1 << 56) == O
    assert _cross(NK=2 ** 31 - 1) == O and _cross(NQ=2 ** 30, H=4, H_kv=1) == O and _cross(B=2 ** 30) == O
    assert _cross(B=2 ** 20, NK=2 ** 30, H=2) == O and _cross(H=2 ** 22 + 2) == O and _cached(H=2 ** 22 + 1) == O
    # split keys need a workspace
    c = dict(B=1, NQ=1, NK=100000, H=4, H_kv=4)
    need = agg.agg_cross_workspace_bytes(agg.make_cross(1, 1, 100000, 4))
    assert _cross(**c) == N and _cross(**c, ws=at(7), n=need - 1) == W


def test_outputs_of_attention_overlap_nothing():
    o_bytes, l_bytes, kv = 2 * 10 * 4 * 128, 2 * 10 * 4 * 4, 2 * 100 * 2 * 128
    for near in (at(3), at(3) + o_bytes - 16, at(3) - 16):
        for other in ("q", "k", "v"):
            assert _cross(**{other: near}) == S, (other, near - at(3))
        assert _cross(lse=near + (12 if near < at(3) else 0)) == S
    assert _cross(ql=at(3) + 4) == S and _cross(kl=at(4) + l_bytes - 4) == S and _cross(kl=at(4) - 4) == S
    assert _cross(lse=at(1) + kv - 4) == S and _cross(lse=at(2)) == S
    # a strided input's reach: the last token's row
    assert _cross(k=at(3) - 199 * 1024 * 2 - 256 + 16, ks=1024) == S
    c = dict(B=1, NQ=1, NK=100000, H=4, H_kv=4)
    need = agg.agg_cross_workspace_bytes(agg.make_cross(1, 1, 100000, 4))
    for other in ("q", "o", "lse"):
        assert _cross(**c, ws=at(8), n=need, **{other: at(8) + need - 16}) == S
    assert _cross(**c, ws=at(1) + 64, n=need) == S and _cross(**c, ws=at(8), n=need, kl=at(8) + 16) == S


def _cached(n_pages=9, H=2, D=64, cB=2, max_pages=2, kc=at(10), vc=at(11), pages=at(12), B=2, NQ=10, NK=100, HQ=4, H_kv=2, q=at(0), qs=0,
            o=at(3), lse=at(4), kl=None):
    cache = agg.agg_cache(n_pages, H, D, cB, max_pages, kc, vc, pages)
    return _status(agg.agg_cache_attn_fwd, cache, agg.make_cross(B, NQ, NK, HQ, H_kv, k_lens=kl), q, qs, o, lse)


def test_cache_attention_refusals():
    for bad in (dict(n_pages=0), dict(H=0), dict(D=-1), dict(cB=0), dict(max_pages=0), dict(B=3), dict(H_kv=4), dict(NK=129), dict(qs=8)):
        assert _cached(**bad) == S, bad
    assert _cached(D=128) == U
    for bad in (dict(kc=None), dict(vc=None), dict(pages=None), dict(q=None), dict(o=None)):
        assert _cached(**bad) == N, bad
    for bad in (dict(kc=at(10) + 8), dict(vc=at(11) + 2), dict(pages=at(12) + 2)):
        assert _cached(**bad) == A, bad
    assert _cached(max_pages=2 ** 26) == O and _cached(n_pages=2 ** 31 - 1, H=2 ** 17, H_kv=2 ** 17, HQ=2 ** 17) == O
    pool = 9 * 2 * 8192
    for near in (at(10), at(10) + pool - 16, at(11) + 64, at(12)):
        assert _cached(o=near) == S and _cached(lse=near) == S
    assert _cached(kl=at(3)) == S
    lib = agg.lib()
    assert lib.agg_cache_attn_fwd(None, agg.ctypes.byref(agg.make_cross(1, 1, 1, 1)), at(0), 0, at(1), None, None, 0, None) == N
    assert lib.agg_cross_attn_fwd(None, at(0), 0, at(1), 0, at(2), 0, at(3), None, None, 0, None) == N


def _append(n_pages=9, H=2, D=64, cB=2, max_pages=2, kc=at(10), vc=at(11), pages=at(12), shape=None, B=2, HQ=4, rope="plain", qn=None,
            kn=None, pos=None, q=at(0), qs=0, k=at(1), ks=0, v=at(2), vs=0, start=at(5), counts=at(6), lens=at(7), qr=at(3), **fields):
    cache = agg.agg_cache(n_pages, H, D, cB, max_pages, kc, vc, pages)
    shape = shape or agg.make_shape(B, 1, 4, 4, 1, HQ, 64, 1, 1)
    if rope == "plain":
        rope = agg.make_rope(agg.AGG_ROPE_SECTIONS, 0, 32, 32)
        for name, value in fields.items():
            setattr(rope, name, value)
    return _status(agg.agg_cache_append, cache, shape, rope, qn, kn, pos, q, qs, k, ks, v, vs, start, counts, lens, qr)


def test_append_refusals():
    for bad in (dict(n_pages=0), dict(max_pages=-1), dict(B=1), dict(HQ=3), dict(HQ=1), dict(pairing=5), dict(d_h=31), dict(d_t=2),
                dict(base=0.5), dict(qs=248), dict(ks=120), dict(ks=132), dict(vs=64), dict(qn=agg.make_norm(4)),
                dict(kn=agg.make_norm(agg.AGG_NORM_RMS, 0.0)), dict(shape=agg.make_shape(2, 0, 4, 4, 1, 4, 64, 1, 1))):
        assert _append(**bad) == S, bad
    assert _append(D=32) == U and _append(shape=agg.make_shape(2, 1, 4, 4, 1, 4, 32, 1, 1)) == U
    for bad in (dict(k=None), dict(v=None), dict(q=None), dict(qr=None), dict(kc=None), dict(vc=None), dict(pages=None)):
        assert _append(**bad) == N, bad
    for bad in (dict(q=at(0) + 8), dict(k=at(1) + 8), dict(v=at(2) + 8), dict(qr=at(3) + 8), dict(kc=at(10) + 8), dict(vc=at(11) + 8),
                dict(pages=at(12) + 2), dict(start=at(5) + 1), dict(counts=at(6) + 2), dict(lens=at(7) + 2), dict(pos=at(8) + 2),
                dict(kn=agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, FAKE + 4))):
        assert _append(**bad) == A, bad
    assert _append(t0=2 ** 31 - 1) == O and _append(patch0=2 ** 31 - 3) == O and _append(ks=1 << 56) == O
    assert _append(HQ=(1 << 22) + 2) == O
    lib = agg.lib()
    c = agg.agg_cache(9, 2, 64, 2, 2, at(10), at(11), at(12))
    assert lib.agg_cache_append(agg.ctypes.byref(c), None, None, None, None, None, None, 0, at(1), 0, at(2), 0, None, None, None, None,
                                None) == N
    assert lib.agg_cache_append(None, None, None, None, None, None, None, 0, at(1), 0, at(2), 0, None, None, None, None, None) == N


def test_outputs_of_appending_overlap_nothing():
    pool, T = 9 * 2 * 8192, 17
    for out, size in ((at(10), pool), (at(11), pool), (at(3), 2 * T * 4 * 128), (at(7), 8)):
        for near in (out, out + size - 4 & ~15, out - 4 & ~15):
            inside = near >= out
            for other in ("k", "v") + (() if out == at(3) else ("q",)):
                if inside or other != "q":
                    assert _append(**{other: near}) == S, (other, out)
        for other in ("start", "counts", "pages", "pos"):
            assert _append(**{other: out}) == S and _append(**{other: out + size - 4}) == S, other
        for n in (agg.make_norm(agg.AGG_NORM_LAYER, 1e-5, out & ~15), agg.make_norm(agg.AGG_NORM_RMS, 1e-5, None, out - 240)):
            assert _append(qn=n) == S and _append(kn=n) == S
    assert _append(vc=at(10) + 4096) == S and _append(qr=at(10)) == S and _append(lens=at(10) + 4) == S
    assert _append(qr=at(0) + 16) == S and _append(qr=at(0), qs=512) == S  # in place only whole and contiguous


# ---- the launch plan -------------------------------------------------------------------------------
DRIVER = r"""
#include <stdio.h>
#include "agg_cross_plan.h"
int main() {
  long long pairs, rows, keys;
  int ragged, fits, paged;
  while (scanf("%lld %lld %lld %d %d %d", &pairs, &rows, &keys, &ragged, &fits, &paged) == 6) {
    const agg::CrossPlan p = agg::plan_cross(pairs, rows, keys, ragged, fits, paged);
    printf("%d %d %d %lld %d\n", p.wide ? p.width : 16 * p.tiles, p.tail, p.halves, (long long)p.row_tiles, p.splits);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(DRIVER)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-Wno-unused-function", "-I", b.CSRC,
                           "-o", str(d / "plan"), str(d / "plan.cpp")])

    def ask(sizes):
        text = "".join("%d %d %d %d %d %d\n" % s for s in sizes)
        out = subprocess.run([str(d / "plan")], input=text, text=True, check=True, stdout=subprocess.PIPE).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]

    return ask


def test_every_row_has_a_workgroup_and_every_split_keys(plan):
    sizes = [(pairs, rows, keys, ragged, fits, paged) for pairs in (1, 3, 16, 100, 4096, 2 ** 31 - 1)
             for rows in (1, 16, 17, 33, 64, 65, 257, 400, 1374, 10992, 2 ** 30)
             for keys in (0, 1, 31, 64, 1000, 20000, 137400, 2 ** 31 - 600) for ragged in (0, 1) for fits in (0, 1) for paged in (0, 1)]
    for (pairs, rows, keys, ragged, fits, _), (width, tail, halves, row_tiles, splits) in zip(sizes, plan(sizes)):
        assert row_tiles * width >= rows > (row_tiles - 1) * width
        assert width in (16, 32, 128, 256) and (fits or width < 128)
        assert width < 128 or rows > 32
        assert tail in (0, 128, 192) and (tail == 0 or (width == 256 and 0 < rows % 256 <= tail))
        assert not halves or (width == 128 and (ragged or pairs * row_tiles * splits <= 256))
        assert 1 <= splits <= 64 and (splits == 1 or keys // splits >= (192 if width >= 128 else 1))


def test_parts_of_a_batch_share_out_no_keys(plan):
    """More workgroups than a launch takes: no splits, whose partial results a launch of its own could not find."""
    sizes = [(pairs, rows, 2 ** 31 - 600, ragged, 1, paged) for pairs in (2 ** 22, 2 ** 23 + 5, 2 ** 31 - 1) for rows in (65, 256, 1000)
             for ragged in (0, 1) for paged in (0, 1)]
    assert all(p[-1] == 1 for p in plan(sizes))


def test_sizes_reach_their_kernels(plan):
    """The GPU tests' sizes run every kernel, out of pages and in place, with and without shared out keys."""
    import test_gpu_cross as gpu

    for paged in (0, 1):
        def reached(sizes):
            asked = [(B * Hk, NQ * (H // Hk), NK, 0, 1, paged) for B, NQ, NK, H, Hk in sizes]
            return {(width, tail, halves, splits > 1) for width, tail, halves, _, splits in plan(asked)}

        got = reached([(B, NQ, NK, 2, 2) for B, NQ, NK in gpu.LENGTHS] + gpu.WIDE)
        for kernel in [(16, 0, 0), (32, 0, 0), (128, 0, 0), (128, 0, 1), (256, 0, 0), (256, 128, 0)]:
            assert kernel + (False,) in got and kernel + (True,) in got, (paged, kernel)
        assert (256, 192, 0, False) in got
        wide = {k[:3] for k in got if k[0] >= 128}
        behind = [(len(lens) * H, NQ, NK, len(lens) > 1, 1, paged) for NQ, H, NK, lens in gpu.BEHIND]
        assert {k[:3] for k in plan(behind) if k[0] >= 128} >= wide - {(256, 192, 0)}, paged
        assert {k for k in got if k[0] >= 128} == {k for k in reached([(B, NQ, NK, H, H) for B, NQ, NK, H in gpu.REDO]) if k[0] >= 128}, paged


# ---- the code that is built ----------------------------------------------------------------------------
@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "agg_cross.s"
    subprocess.check_call([b.HIPCC, *b.FLAGS, "-I", os.path.join(b.ROOT, "include"), "-I", b.CSRC, "-S", "--cuda-device-only",
                           os.path.join(b.CSRC, "agg_cross.hip"), "-o", str(out)], stderr=subprocess.DEVNULL)
    return out.read_text()


def test_kernels_leave_m0_to_their_copy_statements(assembly):
    """The copies into LDS set M0 inside assembly statements without declaring it (the compiler rejects it as a clobber),
    which is sound only while no instruction of the compiler's uses it."""
    inside, seen_copy, offenders = False, 0, []
    for line in assembly.splitlines():
        code = line.split(";")[0] if not line.lstrip().startswith(";;#") else line
        if "#ASMSTART" in line:
            inside = True
        elif "#ASMEND" in line:
            inside = False
        elif inside:
            seen_copy += "global_load_lds_dwordx4" in code
        elif re.search(r"\bm0\b", code):
            offenders.append(line.strip())
    assert seen_copy >= 4, "the copy statements were not found"
    assert not offenders, offenders[:5]


def metadata(text, kernels):
    """(name, fields) of the kernels whose mangled names hold `kernels`."""
    for kernel in re.split(r"^  - \.", text, flags=re.M):
        name = re.search(r"\.name: +\S*(%s\S*)" % kernels, kernel)
        if name:
            yield name.group(1), {f: int(re.search(r"\.%s: +(\d+)" % f, kernel).group(1))
                                  for f in ("vgpr_spill_count", "private_segment_fixed_size")}


def test_kernels_do_not_spill(assembly):
    """The wide kernels hold two paths' code: nothing of the second may lie in scratch memory while the first runs."""
    found = list(metadata(assembly, r"cross_\w+_kernel"))
    assert len(found) >= 14 and not [x for x in found if any(x[1].values())]


def test_append_kernels_do_not_spill(tmp_path):
    out = tmp_path / "agg_cache.s"
    subprocess.check_call([b.HIPCC, *b.FLAGS, "-I", os.path.join(b.ROOT, "include"), "-I", b.CSRC, "-S", "--cuda-device-only",
                           os.path.join(b.CSRC, "agg_cache.hip"), "-o", str(out)], stderr=subprocess.DEVNULL)
    text = out.read_text()
    found = list(metadata(text, "append_kernel"))
    assert len(found) == 8 and not [x for x in found if x[1]["vgpr_spill_count"]]
    assert "scratch_load" not in text and "scratch_store" not in text  # (scalar registers may spill, to lanes of a vector register)


# ---- what only looks like an operand in place ------------------------------------------------------------
def test_queries_in_place_are_nothing_else_of_the_call():
    """Qr may be Q; that Q is also the keys, the values, positions, lengths or pages does not make these writable."""
    for other in ("k", "v", "pos", "start", "counts", "pages"):
        assert _append(HQ=2, qr=at(0), **{other: at(0)}) == S, other
        assert _append(HQ=2, qr=at(0), **{other: at(0) + 16}) == S, other


# ---- more workgroups than a call counts --------------------------------------------------------------------
def test_calls_of_too_many_workgroups_are_sizes_beyond_the_index_range():
    far = [1 << (48 + i) for i in range(5)] + [(1 << 47) + (i << 40) for i in range(8)]
    # 2^22 wide workgroups of a batch element and some, rows in place and in pages
    c = agg.make_cross(1, 2 ** 26 + 256, 1000, 16)
    need = agg.agg_cross_workspace_bytes(c)
    assert need == 0
    assert _status(agg.agg_cross_attn_fwd, c, far[0], 0, far[1], 0, far[2], 0, far[3]) == O
    cache = agg.agg_cache(100, 16, 64, 1, 16, far[5], far[6], far[7])
    assert _status(agg.agg_cache_attn_fwd, cache, c, far[0], 0, far[3]) == O
    # 2^32 workgroups of 32 rows: distances that the wide kernels do not reach
    c = agg.make_cross(2 ** 20, 2 ** 19, 1, 1)
    assert _status(agg.agg_cross_attn_fwd, c, far[0], 0, far[1], 2 ** 23 + 8, far[2], 2 ** 23 + 8, far[3]) == O
    # 2^32 pieces of new tokens
    cache = agg.agg_cache(100, 1, 64, 2 ** 31 - 1, 1, far[5], far[6], far[4])
    shape = agg.make_shape(2 ** 31 - 1, 1, 1, 64, 0, 1, 64, 1, 1)
    assert _status(agg.agg_cache_append, cache, shape, None, None, None, None, None, 0, far[1], 0, far[2], 0) == O


# ---- the binding -------------------------------------------------------------------------------------------
def test_a_cache_has_the_pages_that_both_pools_hold():
    k, v = torch.zeros(5 * 2 * 4096, dtype=torch.bfloat16), torch.zeros(3 * 2 * 4096, dtype=torch.bfloat16)
    pages = torch.zeros((1, 1), dtype=torch.int32)
    assert agg.make_cache(k, v, pages, 2).n_pages == 3 and agg.make_cache(v, k, pages, 2).n_pages == 3
    assert agg.make_cache(k, k, pages, 2).n_pages == 5 and agg.make_cache(k, v, pages, 2, n_pages=2).n_pages == 2


# ---- the plan of ragged calls --------------------------------------------------------------------------------
def test_plans_of_queries_and_keys_that_end_early(plan):
    sizes = [(pairs, rows, keys, 2, fits, paged) for pairs in (1, 3, 16, 100, 4096, 2 ** 22, 2 ** 23 + 5, 2 ** 31 - 1)
             for rows in (1, 16, 17, 33, 64, 65, 257, 400, 1374, 10992, 2 ** 30)
             for keys in (0, 1, 31, 64, 1000, 20000, 137400, 2 ** 31 - 600) for fits in (0, 1) for paged in (0, 1)]
    for (pairs, rows, keys, _, fits, _), (width, tail, halves, row_tiles, splits) in zip(sizes, plan(sizes)):
        assert row_tiles * width >= rows > (row_tiles - 1) * width
        assert width in (16, 32, 128, 256) and (fits or width < 128) and (width < 128 or rows > 32)
        assert tail in (0, 128, 192) and (tail == 0 or (width == 256 and 0 < rows % 256 <= tail))
        assert not halves or width == 128
        assert 1 <= splits <= 64 and (splits == 1 or keys // splits >= (192 if width >= 128 else 1))
        assert splits == 1 or pairs * row_tiles * splits <= 4096


def test_ragged_sizes_reach_their_kernels(plan):
    import test_gpu_cross_ranges as gpu

    for ragged in (1, 2):
        for paged in (0, 1):
            asked = [(B * H, NQ, NK, ragged, 1, paged) for B, NQ, NK, H, queries in gpu.RAGGED if queries == ragged - 1]
            got = {(width, tail, halves, splits > 1) for width, tail, halves, _, splits in plan(asked)}
            want = {(w, t, 0, s) for w, t in ((32, 0), (128, 0), (256, 0), (256, 128), (256, 192)) for s in (False, True)} | {(128, 0, 1, False)}
            assert got >= want, (ragged, paged, want - got)


def test_far_and_hidden_sizes_reach_every_wide_kernel(plan):
    """The sizes whose logits lie far apart run every wide kernel, out of pages and in place, with and without shared out keys."""
    import test_gpu_cross_ranges as gpu

    for paged in (0, 1):
        got = {(width, tail, halves, splits > 1)
               for width, tail, halves, _, splits in plan([(B * H, NQ, NK, 0, 1, paged) for B, NQ, NK, H in gpu.KERNELS])}
        want = {(w, t, h, s) for w, t, h in ((128, 0, 0), (128, 0, 1), (256, 0, 0), (256, 128, 0), (256, 192, 0)) for s in (False, True)}
        assert got >= want, (paged, want - got)
