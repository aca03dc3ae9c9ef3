"""Timing and checking of attention to keys of another length and of the paged key/value cache.

  append   norm and rotary positions of new tokens' queries and keys; keys and values go to the cache
  cached   attention of queries to a cache's rows, found through its page table
  cross    attention of queries to another set's keys and values, read where they are

With ``own`` false a pass is computed in elementary torch operations in 32 bits, with ``own`` true by
the library's calls on buffers that exist before the call.  Token geometry is that of the package's
workloads: 37 x 37 patches and 5 special tokens a frame (1374 tokens), 16 heads of 64 channels; 28 x 37
patches with 12 heads; 16 x 16 patches for the smallest calls.
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 64
PAGE = 64                                 # rows of a page
EPS = 1e-5
FRAME = 37 * 37 + 5


def _append(N, grid, n_special, H, H_kv, start, B=1, axes=(0, 32, 32), pairing="sections", norm="layer", queries=True,
            given=False, ragged=False, fused=False, base=100.0, name=None):
    c = {"kind": "append", "B": B, "N": N, "n_h": grid[0], "n_w": grid[1], "n_special": n_special, "H": H, "H_kv": H_kv,
         "start": start, "d_t": axes[0], "d_h": axes[1], "d_w": axes[2], "pairing": pairing, "norm": norm,
         "queries": queries, "given": given, "ragged": ragged, "fused": fused, "base": base}
    return dict(c, name=name) if name else c


def _attend(kind, B, NQ, NK, H, H_kv=None, ragged=False, fused=False, name=None):
    c = {"kind": kind, "B": B, "NQ": NQ, "NK": NK, "H": H, "H_kv": H_kv or H, "ragged": ragged, "fused": fused}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token behind a short history (a camera token refined step by step): latency is all there is
        _append(1, (1, 1), 0, 16, 16, 261, given=True, name="append_1"),
        # a frame behind 99 others of a stream, straight out of a fused projection
        _append(1, (37, 37), 5, 16, 16, 99 * FRAME, fused=True, name="append_frame"),
        # clips of three streams whose frames end early, four key heads for twelve of queries, a time axis
        _append(8, (28, 37), 5, 12, 4, 1000, 3, (16, 24, 24), "head", "rms", given=True, ragged=True, base=10000.0,
                name="append_clips_3"),
        # a cache filled with a whole recording; its queries go another way
        _append(100, (37, 37), 5, 16, 16, 0, queries=False, name="append_100f"),
        # one query over a short history
        _attend("cached", 1, 1, 262, 16, name="cached_1_short"),
        # one token of each of eight streams of different lengths, grouped key heads
        _attend("cached", 8, 1, 20000, 16, 4, ragged=True, name="cached_8_streams"),
        # one token over a long recording
        _attend("cached", 1, 1, 100 * FRAME, 16, name="cached_1_100f"),
        # a frame over the recording it belongs to: a step of a stream
        _attend("cached", 1, FRAME, 100 * FRAME, 16, name="cached_frame_100f"),
        # one pose token per frame to the tokens of a small frame
        _attend("cross", 2, 1, 261, 8, name="cross_1"),
        # 512 tracked points to each of 24 frames
        _attend("cross", 24, 512, FRAME, 16, name="cross_points_24f"),
        # odd lengths, one of them zero, keys and values side by side in one projection's output
        _attend("cross", 4, 777, 1029, 12, ragged=True, fused=True, name="cross_odd"),
        # eight frames to forty others
        _attend("cross", 1, 8 * FRAME, 40 * FRAME, 16, name="cross_8f_40f"),
    ]


def _span(rng, low, high):
    return int(round(2 ** rng.uniform(math.log2(low), math.log2(high))))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        kind = most.setdefault(c["kind"], {"bytes": 0, "flops": 0})
        for key in kind:
            kind[key] = max(kind[key], w[key])
    while True:
        kind = rng.choice(("append", "cached", "cross"))
        H = rng.choice((16, 16, 12, 8, 20, 1, 33))
        H_kv = rng.choice([H, H] + [h for h in range(1, H) if H % h == 0])
        if kind == "append":
            pairing = rng.choice(("sections", "neighbours", "head"))
            axes = rng.choice(((0, 32, 32), (16, 24, 24), (32, 16, 16), (64, 0, 0), (8, 6, 10), (0, 0, 0)))
            one = rng.random() < 0.25
            grid, special = ((1, 1), 0) if one else (rng.choice(((37, 37), (28, 37), (16, 16), (rng.randint(9, 40), rng.randint(9, 40)))),
                                                     rng.choice((5, 1, 0)))
            c = _append(1 if one else _span(rng, 1, 100), grid, special, H, H_kv, rng.choice((0, _span(rng, 1, 100000))),
                        rng.choice((1, 1, 2, 5)), axes, pairing, rng.choice(("none", "layer", "rms")),
                        rng.choice((True, True, False)), rng.choice((False, True)), rng.choice((False, False, True)),
                        rng.choice((False, True)), rng.choice((100.0, 10000.0)))
        else:
            few = rng.random() < 0.4
            c = _attend(kind, rng.choice((1, 1, 2, 3, 8, 24)), rng.randint(1, 40) if few else _span(rng, 1, 10992),
                        _span(rng, 1, 137400), H, H_kv, rng.choice((False, False, True)), rng.choice((False, True)))
        w = work(c)
        if all(w[key] <= most[kind][key] for key in w):
            return c


def _tokens(c):
    return c["N"] * (c["n_h"] * c["n_w"] + c["n_special"])


def _shares(B):
    """Sixteenths of the longest length that the sequences of a ragged batch have; the second has nothing."""
    return [0 if b == 1 else 16 - 5 * b % 16 for b in range(B)]


def _lengths(c, most, gen):
    """int32 [B] on the GPU: each sequence's share of `most`, up to a page less; None where all are whole."""
    if not c["ragged"]:
        return None
    less = torch.randint(0, min(PAGE, most // 16 + 1), (c["B"],), generator=gen, device="cuda")
    share = torch.tensor(_shares(c["B"]), device="cuda")
    return (share * most // 16 - less).clamp(min=0).to(torch.int32)


def _queries_end_early(c):
    return c["ragged"] and c["NQ"] >= 256


def work(case):
    """Each input read once, each output written once."""
    c = case
    part = sum(_shares(c["B"])) / 16 / c["B"] if c["ragged"] else 1
    if c["kind"] == "append":
        n = c["B"] * _tokens(c) * part
        each = n * HEAD * (c["H_kv"] + c["H"] * c["queries"])
        return {"bytes": 2 * 2 * (each + n * HEAD * c["H_kv"]) + (12 * n if c["given"] else 0),
                "flops": each * (3 if c["norm"] == "none" else 9)}
    lens = [x / 16 for x in _shares(c["B"])] if c["ragged"] else [1] * c["B"]
    q_lens = lens if _queries_end_early(c) else [1] * c["B"]
    return {"bytes": 2 * 2 * HEAD * (sum(q_lens) * c["NQ"] * c["H"] + sum(lens) * c["NK"] * c["H_kv"]),
            "flops": 4 * HEAD * c["H"] * c["NQ"] * c["NK"] * sum(x * y for x, y in zip(lens, q_lens))}


# ---- inputs --------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _bf16(gen, *shape, scale=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16).mul_(scale)


def _affine(gen, norm):
    gamma = 1.0 + 0.2 * _normal(gen, HEAD)
    return gamma, (0.2 * _normal(gen, HEAD) if norm == "layer" else None)


def _pages(gen, B, rows):
    """A page table [B, pages] over a pool with a few pages to spare, handed out in no order."""
    each = -(-rows // PAGE)
    spare = B * each + 7
    return torch.randperm(spare, generator=gen, device="cuda")[:B * each].to(torch.int32).view(B, each), spare


def _side_by_side(gen, fused, B, N, heads, scales):
    """Tensors [B, N, h, 64] for h in `heads`, and their tokens' distance: slices of one projection's output, or each alone (0)."""
    if not fused:
        return [_bf16(gen, B, N, h, HEAD, scale=s) for h, s in zip(heads, scales)], 0
    whole = _bf16(gen, B, N, sum(heads), HEAD)
    parts = list(whole.split(list(heads), 2))
    for p, s in zip(parts, scales):
        p.mul_(s)
    return parts, sum(heads) * HEAD


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": c}
    B, H, H_kv = c["B"], c["H"], c["H_kv"]
    if c["kind"] == "append":
        n = _tokens(c)
        (q, k, v), st["stride"] = _side_by_side(gen, c["fused"], B, n, (H, H_kv, H_kv), (1.5, 2.0, 1.0))
        st.update(k=k, v=v, q=q if c["queries"] else None, qr=torch.zeros((B, n, H, HEAD), dtype=torch.bfloat16, device="cuda") if c["queries"] else None)
        less = torch.randint(0, PAGE, (B,), generator=gen, device="cuda", dtype=torch.int32)
        st["start"] = (c["start"] - less).clamp(min=0).to(torch.int32)
        st["counts"] = _lengths(c, n, gen)
        st["lens"] = torch.zeros((B,), dtype=torch.int32, device="cuda")
        st["pages"], pool = _pages(gen, B, c["start"] + n)
        for name in "qk":
            st[name + "_norm"] = _affine(gen, c["norm"])
        st["pos"] = None
        if c["given"]:  # frames taken from a longer recording, at another resolution
            pos = torch.stack(_grid_positions(c), -1).repeat(B, 1, 1)
            pos[..., 0] += torch.randint(0, 5000, (B, 1), generator=gen, device="cuda", dtype=torch.int32)
            pos[..., 1:] *= 2
            st["pos"] = pos.contiguous()
        st["pairs"] = _pairs(c)
    else:
        NQ, NK = c["NQ"], c["NK"]
        st["q"] = _bf16(gen, B, NQ, H, HEAD, scale=1.3)
        st["k_lens"] = _lengths(c, NK, gen)
        st["q_lens"] = _lengths(c, NQ, gen) if _queries_end_early(c) else None
        st["o"] = torch.zeros((B, NQ, H, HEAD), dtype=torch.bfloat16, device="cuda")
        if c["kind"] == "cross":
            (st["k"], st["v"]), st["stride"] = _side_by_side(gen, c["fused"], B, NK, (H_kv, H_kv), (1.0, 1.0))
        else:
            st["pages"], pool = _pages(gen, B, NK)
    if c["kind"] != "cross":  # what other sequences keep there, and what was there before
        st["kc"], st["vc"] = (_bf16(gen, pool, H_kv, PAGE * HEAD) for _ in "kv")
    if own:
        _plan(st)
    return st


# ---- the library's calls -------------------------------------------------------------------------
def _plan(st):
    from paper_2512_02541_amd import binding as agg

    c = st["case"]
    st["agg"] = agg
    if c["kind"] != "cross":
        st["cache"] = agg.make_cache(st["kc"], st["vc"], st["pages"], H=c["H_kv"])
    if c["kind"] == "append":
        kind = {"none": agg.AGG_NORM_NONE, "layer": agg.AGG_NORM_LAYER, "rms": agg.AGG_NORM_RMS}[c["norm"]]
        pairing = {"sections": agg.AGG_ROPE_SECTIONS, "neighbours": agg.AGG_ROPE_NEIGHBOURS, "head": agg.AGG_ROPE_HEAD}[c["pairing"]]
        st["shape"] = agg.make_shape(c["B"], c["N"], c["n_h"], c["n_w"], c["n_special"], c["H"], HEAD, 1, 1)
        st["rope"] = agg.make_rope(pairing, c["d_t"], c["d_h"], c["d_w"], base=c["base"], t0=7, patch0=1)
        st["norms"] = [agg.make_norm(kind, EPS, *st[n + "_norm"]) for n in "qk"]
    else:
        st["cross"] = agg.make_cross(c["B"], c["NQ"], c["NK"], c["H"], c["H_kv"], q_lens=st["q_lens"], k_lens=st["k_lens"])
        st["bytes"] = agg.agg_cross_workspace_bytes(st["cross"])
        st["space"] = torch.empty((max(st["bytes"], 16),), dtype=torch.uint8, device="cuda")


def _own(s):
    agg, c = s["agg"], s["case"]
    if c["kind"] == "append":
        agg.agg_cache_append(s["cache"], s["shape"], s["rope"], s["norms"][0], s["norms"][1], s["pos"],
                             s["q"], s["stride"], s["k"], s["stride"], s["v"], s["stride"],
                             s["start"], s["counts"], s["lens"], s["qr"])
        return {"kc": s["kc"], "vc": s["vc"], "lens": s["lens"], "q": s["qr"]}
    if c["kind"] == "cached":
        agg.agg_cache_attn_fwd(s["cache"], s["cross"], s["q"], 0, s["o"], None, s["space"], s["bytes"])
    else:
        agg.agg_cross_attn_fwd(s["cross"], s["q"], 0, s["k"], s["stride"], s["v"], s["stride"], s["o"], None, s["space"], s["bytes"])
    return {"o": s["o"]}


# ---- the plain form ------------------------------------------------------------------------------
def _grid_positions(c):
    """int32 [tokens] each: frame, row, column; special tokens are at row and column 0, patches begin at 1."""
    n_h, n_w, P = c["n_h"], c["n_w"], c["n_special"]
    slot = torch.arange(P + n_h * n_w, device="cuda")
    patch = slot >= P
    row = torch.where(patch, 1 + (slot - P) // n_w, 0).expand(c["N"], -1)
    col = torch.where(patch, 1 + (slot - P) % n_w, 0).expand(c["N"], -1)
    frame = torch.arange(c["N"], device="cuda")[:, None].expand_as(row)
    return 7 + frame.reshape(-1).to(torch.int32), row.reshape(-1).to(torch.int32), col.reshape(-1).to(torch.int32)


def _pairs(c):
    """For each pair of channels that turns: first channel, second channel, axis, frequency (64 bits)."""
    sizes = torch.tensor((c["d_t"], c["d_h"], c["d_w"]), device="cuda")
    turned = c["d_t"] + c["d_h"] + c["d_w"]
    axis = torch.repeat_interleave(torch.arange(3, device="cuda"), sizes // 2)
    i = torch.arange(turned // 2, device="cuda")
    d = sizes[axis]
    begin = (torch.cumsum(sizes, 0) - sizes)[axis]
    j = i - begin // 2
    if c["pairing"] == "head":
        first, second, e = i, i + turned // 2, 2.0 * i.double() / max(turned, 1)
    elif c["pairing"] == "sections":
        first, second, e = begin + j, begin + j + d // 2, 2.0 * j.double() / d
    else:
        first, second, e = begin + 2 * j, begin + 2 * j + 1, 2.0 * j.double() / d
    return first, second, axis, torch.pow(torch.tensor(c["base"], dtype=torch.float64, device="cuda"), -e)


def _turn(c, t, pos, pairs, affine):
    """Norm and rotation of t [B, N, h, 64], rounded once."""
    x = t.float()
    if c["norm"] != "none":
        if c["norm"] == "layer":
            x = x - x.mean(-1, keepdim=True)
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * affine[0]
        if c["norm"] == "layer":
            x = x + affine[1]
    a, b, axis, freq = pairs
    angle = pos[..., axis].double() * freq  # far positions: 64 bits
    cos, sin = angle.cos().float().unsqueeze(-2), angle.sin().float().unsqueeze(-2)
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    return y.to(torch.bfloat16)


def _k_rows(pool):
    """The keys' pool as [pages, 2, 32, heads, 4, 2, 8]: half of a page, row of it, head, and the channel in three parts."""
    n, h, _ = pool.shape
    return pool.view(n, h, 2, 4, 2, 32, 8).permute(0, 2, 5, 1, 3, 4, 6)


def _v_rows(pool):
    """The values' pool as [pages, 4, 2, 2, 4, heads, 64]: the row in four parts, head, channel."""
    n, h, _ = pool.shape
    return pool.view(n, h, 4, 2, HEAD, 2, 4).permute(0, 2, 5, 3, 6, 1, 4)


def _append_plain(s):
    c = s["case"]
    B, n = c["B"], _tokens(c)
    pos = torch.stack(_grid_positions(c), -1) if s["pos"] is None else s["pos"]
    t = torch.arange(n, device="cuda")
    count = torch.full_like(s["start"], n) if s["counts"] is None else s["counts"]
    here = t[None] < count[:, None]
    row = s["start"][:, None].long() + t
    page = torch.gather(s["pages"].long(), 1, row // PAGE)[here]
    at = (row % PAGE)[here]
    k = _turn(c, s["k"], pos, s["pairs"], s["k_norm"])
    _k_rows(s["kc"])[page, at // 32, at % 32] = k[here].view(-1, c["H_kv"], 4, 2, 8)
    _v_rows(s["vc"])[page, at // 16, at // 8 % 2, at // 4 % 2, at % 4] = s["v"][here]
    out = {"kc": s["kc"], "vc": s["vc"], "lens": (s["start"] + count).to(torch.int32), "q": None}
    if s["q"] is not None:
        out["q"] = torch.where(here[..., None, None], _turn(c, s["q"], pos, s["pairs"], s["q_norm"]), s["qr"])
    return out


def _softmax_of(q, k, v, k_lens, q_lens, old):
    """Attention of q [B, NQ, H, 64] to k and v [B, NK, H_kv, 64], in 32 bits."""
    H = q.shape[2]
    q, k, v = (x.transpose(1, 2).float() for x in (q, k, v))
    k = k.repeat_interleave(H // k.shape[1], 1).transpose(2, 3).contiguous()
    v = v.repeat_interleave(H // v.shape[1], 1).contiguous()
    s = torch.matmul(q.contiguous() * HEAD ** -0.5, k)
    if k_lens is not None:
        hidden = torch.arange(s.shape[-1], device="cuda") >= k_lens[:, None]
        s.masked_fill_(hidden[:, None, None], float("-inf"))
        v = v.masked_fill(hidden[:, None, :, None], 0.0)
    top = s.amax(-1, keepdim=True)
    s.sub_(torch.where(torch.isinf(top), 0.0, top)).exp_()
    total = s.sum(-1, keepdim=True)
    o = (torch.matmul(s, v) / torch.where(total == 0, 1.0, total)).to(torch.bfloat16).transpose(1, 2)
    if q_lens is None:
        return o.contiguous()
    inside = torch.arange(o.shape[1], device="cuda") < q_lens[:, None]
    return torch.where(inside[..., None, None], o, old)


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s)
    if c["kind"] == "append":
        return _append_plain(s)
    k, v = s.get("k"), s.get("v")
    if c["kind"] == "cached":
        pages = s["pages"].long()
        k = _k_rows(s["kc"])[pages].reshape(c["B"], -1, c["H_kv"], HEAD)[:, :c["NK"]]
        v = _v_rows(s["vc"])[pages].reshape(c["B"], -1, c["H_kv"], HEAD)[:, :c["NK"]]
    return {"o": _softmax_of(s["q"], k, v, s["k_lens"], s["q_lens"], s["o"])}


# ---- the same in 64 bits, from the definitions ---------------------------------------------------
def _norm64(x, kind, affine):
    if kind == "none":
        return x
    mean = x.sum(-1, keepdim=True) / HEAD if kind == "layer" else torch.zeros_like(x[..., :1])
    var = (x - mean).square().sum(-1, keepdim=True) / HEAD
    y = (x - mean) / (var + EPS).sqrt() * affine[0].double()
    return y + affine[1].double() if affine[1] is not None else y


def _turn64(c, t, pos, affine):
    """Each axis's channels as complex numbers, multiplied by exp(i * angle)."""
    out = _norm64(t.double(), c["norm"], affine)
    sizes = (c["d_t"], c["d_h"], c["d_w"])
    turned = sum(sizes)
    dev = t.device
    if c["pairing"] == "head":
        i = torch.arange(turned // 2, device=dev, dtype=torch.float64)
        axis = torch.repeat_interleave(torch.arange(3, device=dev), torch.tensor([d // 2 for d in sizes], device=dev))
        angle = pos.double()[..., axis] * torch.exp(-2 * i / max(turned, 1) * math.log(c["base"]))
        z = torch.complex(out[..., :turned // 2].contiguous(), out[..., turned // 2:turned].contiguous())
        z = z * torch.polar(torch.ones_like(angle), angle).unsqueeze(-2)
        return torch.cat((z.real, z.imag, out[..., turned:]), -1)
    parts, begin = [], 0
    for a, d in enumerate(sizes):
        x = out[..., begin:begin + d]
        begin += d
        j = torch.arange(d // 2, device=dev, dtype=torch.float64)
        angle = pos.double()[..., a:a + 1] * torch.exp(-2 * j / max(d, 1) * math.log(c["base"]))
        turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(-2)
        if c["pairing"] == "sections":
            z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
            parts += [z.real, z.imag]
        else:
            z = torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous()) * turn
            parts.append(torch.view_as_real(z).flatten(-2))
    return torch.cat(parts + [out[..., begin:]], -1)


def _places64(rows, values):
    """Where channel d of row m of a page's head lies in its 4096 elements: int64 [rows, 64]."""
    m, d = rows[:, None], torch.arange(HEAD, device=rows.device)
    if values:
        u = m % 16
        return ((m // 16 * 2 + u % 8 // 4) * HEAD + d) * 8 + u // 8 * 4 + u % 4
    return (((m // 32 * 4 + d // 16) * 2 + d % 16 // 8) * 32 + m % 32) * 8 + d % 8


def _append64(c, s):
    n, L, P, n_w = _tokens(c), c["n_h"] * c["n_w"] + c["n_special"], c["n_special"], c["n_w"]
    t = torch.arange(n, device="cuda")
    p = t % L - P
    place = torch.stack((t // L + 7, torch.where(p < 0, -1, p // n_w) + 1, torch.where(p < 0, -1, p % n_w) + 1), -1)
    kc, vc = s["kc"].double(), s["vc"].double()
    out = {"kc": kc, "vc": vc, "lens": None, "q": None if s["q"] is None else s["qr"].double()}
    for b in range(c["B"]):
        count = n if s["counts"] is None else int(s["counts"][b])
        pos = (place if s["pos"] is None else s["pos"][b])[None, :count]
        if s["q"] is not None:
            out["q"][b, :count] = _turn64(c, s["q"][b:b + 1, :count], pos, s["q_norm"])[0]
        rows = int(s["start"][b]) + t[:count]
        page = s["pages"][b][rows // PAGE].long()[:, None]
        k = _turn64(c, s["k"][b:b + 1, :count], pos, s["k_norm"])[0]
        for h in range(c["H_kv"]):
            kc[page, h, _places64(rows % PAGE, False)] = k[:, h]
            vc[page, h, _places64(rows % PAGE, True)] = s["v"][b, :count, h].double()
    return out


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _append64(c, s)
    out = s["o"].double()
    group = c["H"] // c["H_kv"]
    for b in range(c["B"]):
        keys = c["NK"] if s["k_lens"] is None else int(s["k_lens"][b])
        queries = c["NQ"] if s["q_lens"] is None else int(s["q_lens"][b])
        r = torch.arange(keys, device="cuda")
        for h in range(c["H"]):
            if keys == 0 or queries == 0:
                continue
            if c["kind"] == "cross":
                k, v = (s[n][b, :keys, h // group].double() for n in "kv")
            else:
                page = s["pages"][b][r // PAGE].long()[:, None]
                k = s["kc"][page, h // group, _places64(r % PAGE, False)].double()
                v = s["vc"][page, h // group, _places64(r % PAGE, True)].double()
            for at in range(0, queries, 2048):
                q = s["q"][b, at:min(at + 2048, queries), h].double()
                logit = q @ k.t().contiguous() / math.sqrt(HEAD)
                out[b, at:at + q.shape[0], h] = torch.softmax(logit, -1) @ v
    return {"o": out}
