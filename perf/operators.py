"""Timing and checking of the operators around a block's attention.

  rope        query/key normalisation and rotary positions on the axes time, height and width
  residual    a branch's norm, gate and residual scale, the residual sum and the next norm
  mx4         quantisation to microscaled 4-bit floats, and reading them back
  projection  quantisation of the activations and their product with 4-bit weights

With ``own`` false a pass is computed in elementary torch operations in 32 bits, with ``own`` true by
the library's calls on buffers that exist before the call.  Token geometry is that of the
package's workloads: 37 x 37 patches and 5 special tokens a frame, 16 heads of 64 channels, 1 to 100
frames; 16 x 16 patches for the smallest calls.
"""
from __future__ import annotations

import math

import torch

own = False

HEAD = 64
BLOCK = 32                                # channels that share a scale
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # magnitudes of a 4-bit float, by code
EPS = 1e-5


def _rope(N, grid, H, axes, pairing, norm, given=False, B=1, n_special=5, t0=0, base=100.0, name=None):
    c = {"kind": "rope", "B": B, "N": N, "n_h": grid[0], "n_w": grid[1], "n_special": n_special, "H": H,
         "d_t": axes[0], "d_h": axes[1], "d_w": axes[2], "pairing": pairing, "norm": norm,
         "given": given, "t0": t0, "base": base}
    return dict(c, name=name) if name else c


def _residual(rows, C, post="none", pre="layer", scale=True, gate_rows=0, name=None):
    c = {"kind": "residual", "rows": rows, "C": C, "post": post, "pre": pre, "scale": scale,
         "gate_rows": gate_rows}
    return dict(c, name=name) if name else c


def _mx4(rows, K, name=None):
    c = {"kind": "mx4", "rows": rows, "K": K}
    return dict(c, name=name) if name else c


def _projection(rows, K, N, count=1, residual=False, name=None):
    c = {"kind": "projection", "rows": rows, "K": K, "N": N, "count": count, "residual": residual}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one new small frame of a stream: launch and latency are all there is
        _rope(1, (16, 16), 8, (0, 32, 32), "sections", "layer", t0=17, name="rope_1f_16x16"),
        # the queries and keys of a short clip: rows and columns turn half a head each, behind a LayerNorm
        _rope(16, (37, 37), 16, (0, 32, 32), "sections", "layer", name="rope_16f"),
        # a long video with a time axis, one ladder of frequencies over the head, the caller's positions
        _rope(100, (37, 37), 16, (16, 24, 24), "head", "rms", given=True, base=10000.0, name="rope_video_100f"),
        # a single token behind a block (a camera token being refined)
        _residual(1, 1024, name="residual_1"),
        # the token stream of a short clip between attention and the next layer: layer scale, LayerNorm
        _residual(16 * 1374, 1024, name="residual_16f"),
        # norms on both sides of the branch and a gate per frame of 261 tokens, 33 heads wide, an odd number of rows
        _residual(8191, 2112, "rms", "rms", True, 261, name="residual_gated_33h"),
        # activations of two small frames to 4 bits and back
        _mx4(522, 1024, name="mx4_522"),
        # ... of 100 frames
        _mx4(137400, 1024, name="mx4_100f"),
        # a single token through a projection
        _projection(1, 1024, 1024, name="projection_1"),
        # queries, keys and values of two small frames
        _projection(522, 1024, 1024, 3, name="projection_qkv_522"),
        # the narrowing half of a token-wise network over a short clip, added to the stream
        _projection(16 * 1374, 4096, 1024, 1, True, name="projection_down_16f"),
        # queries, keys and values of 100 frames
        _projection(137400, 1024, 1024, 3, name="projection_qkv_100f"),
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
        kind = rng.choice(("rope", "residual", "mx4", "projection"))
        if kind == "rope":
            pairing = rng.choice(("sections", "neighbours", "head"))
            left, axes = HEAD, []
            for _ in range(2):
                axes.append(2 * rng.randint(0, min(16, left // 2)))
                left -= axes[-1]
            axes.append(rng.choice((left, 2 * rng.randint(0, left // 2))))
            if rng.random() < 0.5:
                axes = list(rng.choice(((0, 32, 32), (16, 24, 24), (32, 16, 16), (64, 0, 0))))
            c = _rope(_span(rng, 1, 100), rng.choice(((37, 37), (28, 37), (16, 16), (rng.randint(9, 40), rng.randint(9, 40)))),
                      rng.choice((16, 16, 8, 12, 20, 1, 33)), axes, pairing, rng.choice(("none", "layer", "rms")),
                      rng.choice((False, False, True)), rng.choice((1, 1, 2)), rng.choice((5, 1, 0)),
                      rng.choice((0, 0, 1000, 100000)), rng.choice((100.0, 10000.0)))
        elif kind == "residual":
            C = HEAD * rng.choice((16, 16, 12, 20, rng.randint(1, 64)))
            c = _residual(_span(rng, 1, 30000), C, rng.choice(("none", "none", "layer", "rms")),
                          rng.choice(("layer", "layer", "rms", "none")), rng.choice((True, False)),
                          rng.choice((0, 0, 261, 1374, 1)))
        elif kind == "mx4":
            c = _mx4(_span(rng, 1, 137400), rng.choice((1024, 1024, 4096, 32 * rng.randint(1, 128))))
        else:
            c = _projection(_span(rng, 1, 137400), rng.choice((1024, 1024, 4096, HEAD * rng.randint(1, 64))),
                            rng.choice((1024, 1024, 4096, HEAD * rng.randint(1, 64))), rng.choice((1, 1, 2, 3)),
                            rng.choice((False, True)))
            if c["count"] > 1:
                c["residual"] = False
        w = work(c)
        if all(w[key] <= most[kind][key] for key in w):
            return c


def _tokens(c):
    return c["N"] * (c["n_h"] * c["n_w"] + c["n_special"])


def work(case):
    """Each input read once, each output written once."""
    c = case
    if c["kind"] == "rope":
        n = c["B"] * _tokens(c)
        each = 2 * n * c["H"] * HEAD  # elements of queries and keys
        return {"bytes": 2 * 2 * each + (12 * n if c["given"] else 0), "flops": each * (3 if c["norm"] == "none" else 9)}
    if c["kind"] == "residual":
        n = c["rows"] * c["C"]
        tensors = 3 + (c["pre"] != "none")
        groups = -(-c["rows"] // c["gate_rows"]) if c["gate_rows"] else 0
        return {"bytes": 2 * (tensors * n + groups * c["C"]), "flops": n * (2 + 6 * (c["post"] != "none") + 6 * (c["pre"] != "none"))}
    rows, K = c["rows"], c["K"]
    held = K // 2 + -(-K // BLOCK)  # bytes of a row in 4 bits
    if c["kind"] == "mx4":
        return {"bytes": rows * (2 * K + held + 2 * K), "flops": 4 * rows * K}
    N, count = c["N"], c["count"]
    return {"bytes": rows * 2 * K + count * N * held + rows * N * 2 * (count + c["residual"]),
            "flops": 2 * rows * K * N * count}


# ---- inputs --------------------------------------------------------------------------------------
def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _stream(gen, rows, C):
    """Activations of a residual stream: unit noise, some channels an order of magnitude larger."""
    x = _normal(gen, rows, C)
    x *= torch.exp(0.7 * _normal(gen, C))
    return x.to(torch.bfloat16)


def _affine(gen, C, norm):
    gamma = 1.0 + 0.2 * _normal(gen, C)
    return gamma, (0.2 * _normal(gen, C) if norm == "layer" else None)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = {"case": c, "grid": _grid()}
    if c["kind"] == "rope":
        nq, H = _tokens(c), c["H"]
        q, k = (_normal(gen, c["B"], nq, H, HEAD).mul_(s).to(torch.bfloat16) for s in (1.5, 2.0))
        st.update(q=q, k=k, pos=None, qr=torch.empty_like(q), kr=torch.empty_like(k))
        for name in "qk":
            st[name + "_norm"] = _affine(gen, HEAD, c["norm"])
        if c["given"]:  # positions of frames taken from a longer recording, at another resolution
            pos = torch.stack(_grid_positions(c), -1).repeat(c["B"], 1, 1)
            pos[..., 0] += torch.randint(0, 5000, (c["B"], 1), generator=gen, device="cuda", dtype=torch.int32)
            pos[..., 1:] *= 2
            st["pos"] = pos.contiguous()
        if not own:
            pairs = list(zip(*_pairs(c))) or [(), (), (), ()]
            st["pairs"] = [torch.tensor(p, dtype=torch.int64, device="cuda") for p in pairs[:3]]
            st["freq"] = torch.tensor(pairs[3], dtype=torch.float64, device="cuda")
    elif c["kind"] == "residual":
        rows, C = c["rows"], c["C"]
        x, branch = _stream(gen, rows, C), _stream(gen, rows, C)
        st.update(x=x, branch=branch, scale=0.3 * _normal(gen, C) if c["scale"] else None, gate=None,
                  h=torch.empty_like(x), n=None if c["pre"] == "none" else torch.empty_like(x))
        if c["gate_rows"]:
            st["gate"] = _normal(gen, -(-rows // c["gate_rows"]), C).to(torch.bfloat16)
        st["post_norm"], st["pre_norm"] = _affine(gen, C, c["post"]), _affine(gen, C, c["pre"])
    else:
        rows, K = c["rows"], c["K"]
        st.update(x=_stream(gen, rows, K), **_held("x", rows, K))
        if c["kind"] == "mx4":
            st["back"] = torch.empty_like(st["x"])
        else:
            N = c["N"]
            st["w"] = []
            for _ in range(c["count"]):
                w = (_normal(gen, N, K) / math.sqrt(K)).to(torch.bfloat16)
                st["w"].append(_pack(*_quantize(w)))
            st["bias"] = [0.1 * _normal(gen, N) for _ in range(c["count"])]
            st["res"] = _stream(gen, rows, N) if c["residual"] else None
            st["res_scale"] = 0.3 * _normal(gen, N) if c["residual"] else None
            st["y"] = [torch.empty((rows, N), dtype=torch.bfloat16, device="cuda") for _ in range(c["count"])]
    if own:
        _plan(st)
    return st


def _held(name, rows, K):
    """Buffers of a matrix in 4 bits: rows of codes and of scales, padded to 128 and 16 bytes."""
    return {name + "_codes": torch.empty((rows, 128 * -(-K // 256)), dtype=torch.uint8, device="cuda"),
            name + "_scales": torch.empty((rows, 16 * -(-K // 512)), dtype=torch.uint8, device="cuda")}


# ---- the library's calls -------------------------------------------------------------------------
def _plan(st):
    from paper_2512_02541_amd import binding as agg

    c = st["case"]
    norms = {"none": agg.AGG_NORM_NONE, "layer": agg.AGG_NORM_LAYER, "rms": agg.AGG_NORM_RMS}

    def norm(kind, affine):
        return agg.make_norm(norms[kind], EPS, *affine)

    st["agg"] = agg
    if c["kind"] == "rope":
        pairing = {"sections": agg.AGG_ROPE_SECTIONS, "neighbours": agg.AGG_ROPE_NEIGHBOURS,
                   "head": agg.AGG_ROPE_HEAD}[c["pairing"]]
        st["shape"] = agg.make_shape(c["B"], c["N"], c["n_h"], c["n_w"], c["n_special"], c["H"], HEAD, 1, 1)
        st["rope"] = agg.make_rope(pairing, c["d_t"], c["d_h"], c["d_w"], base=c["base"], t0=c["t0"], patch0=1)
        st["norms"] = [norm(c["norm"], st[n + "_norm"]) for n in "qk"]
    elif c["kind"] == "residual":
        st["plan"] = agg.make_residual(post=norm(c["post"], st["post_norm"]), pre=norm(c["pre"], st["pre_norm"]),
                                       scale=st["scale"], gate=st["gate"], gate_rows=c["gate_rows"])
    elif c["kind"] == "projection":
        st["plan"] = agg.make_mx4_linear(st["w"], st["y"], st["bias"], residual=st["res"], res_scale=st["res_scale"])


def _own(s):
    agg, c = s["agg"], s["case"]
    if c["kind"] == "rope":
        agg.agg_rope_fwd(s["shape"], s["rope"], s["norms"][0], s["norms"][1], s["pos"], s["q"], 0, s["k"], 0,
                         s["qr"], s["kr"])
        return {"q": s["qr"], "k": s["kr"]}
    if c["kind"] == "residual":
        agg.agg_residual_norm_fwd(c["rows"], c["C"], s["plan"], s["x"], s["branch"], s["h"], s["n"])
        return {"h": s["h"]} if s["n"] is None else {"h": s["h"], "n": s["n"]}
    agg.agg_mx4_quantize(c["rows"], c["K"], s["x"], 0, s["x_codes"], s["x_scales"])
    if c["kind"] == "mx4":
        agg.agg_mx4_dequantize(c["rows"], c["K"], s["x_codes"], s["x_scales"], s["back"])
        return {"back": s["back"]}
    agg.agg_mx4_linear_fwd(c["rows"], c["N"], c["K"], s["plan"], s["x_codes"], s["x_scales"])
    return {"y%d" % i: y for i, y in enumerate(s["y"])}


# ---- the plain form ------------------------------------------------------------------------------
def _grid_positions(c):
    """int32 [tokens] each: frame, row, column; special tokens are at row and column 0, patches begin at 1."""
    n_h, n_w, P = c["n_h"], c["n_w"], c["n_special"]
    slot = torch.arange(P + n_h * n_w, device="cuda")
    patch = slot >= P
    row = torch.where(patch, 1 + (slot - P) // n_w, 0)
    col = torch.where(patch, 1 + (slot - P) % n_w, 0)
    frame = torch.arange(c["N"], device="cuda")[:, None].expand(-1, slot.numel())
    out = (c["t0"] + frame, row.expand(c["N"], -1), col.expand(c["N"], -1))
    return [t.reshape(-1).to(torch.int32) for t in out]


def _pairs(c):
    """For each pair of channels that turns: first channel, second channel, axis, frequency (64 bits)."""
    out, start = [], 0
    turned = c["d_t"] + c["d_h"] + c["d_w"]
    for axis, d in enumerate((c["d_t"], c["d_h"], c["d_w"])):
        for j in range(d // 2):
            if c["pairing"] == "head":
                i = start // 2 + j
                out.append((i, i + turned // 2, axis, c["base"] ** (-2.0 * i / turned)))
            elif c["pairing"] == "sections":
                out.append((start + j, start + j + d // 2, axis, c["base"] ** (-2.0 * j / d)))
            else:
                out.append((start + 2 * j, start + 2 * j + 1, axis, c["base"] ** (-2.0 * j / d)))
        start += d
    return out


def _norm(x, kind, affine):
    if kind == "none":
        return x
    if kind == "layer":
        x = x - x.mean(-1, keepdim=True)
    x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * affine[0]
    return x + affine[1] if kind == "layer" else x


def _turn(c, t, cos, sin, a, b, affine):
    x = _norm(t.float(), c["norm"], affine)
    first, second = x[..., a], x[..., b]
    y = x.clone()
    y[..., a] = first * cos - second * sin
    y[..., b] = second * cos + first * sin
    return y.to(torch.bfloat16)


def _quantize(x):
    """bf16 [rows, K] -> codes [rows, blocks * 32] and scale bytes [rows, blocks], K filled up with zeros."""
    rows, K = x.shape
    blocks = -(-K // BLOCK)
    v = torch.zeros((rows, blocks * BLOCK), dtype=torch.float32, device=x.device)
    v[:, :K] = x
    v = v.view(rows, blocks, BLOCK)
    most = v.abs().amax(-1)
    e = (torch.frexp(most).exponent - 3).clamp(-127, 127)
    e = torch.where(most == 0, -127, e)
    broken = ~torch.isfinite(most)
    v = torch.ldexp(v, -e[..., None])  # exact: a power of two, and below 8
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    m = (torch.round(m / step) * step).clamp(max=6.0)  # ties to the even code
    code = torch.where(m < 2, 2 * m, torch.where(m < 4, m + 2, m / 2 + 4))
    code = torch.where(broken[..., None], 0.0, code).to(torch.uint8)
    code += 8 * torch.signbit(v).to(torch.uint8)
    scale = torch.where(broken, 255, e + 127).to(torch.uint8)
    return code.view(rows, -1), scale


def _pack(code, scale):
    """The rows as they are held: two codes a byte, the earlier one low, padded with zeros."""
    rows, K = code.shape
    held = _held("m", rows, K)
    codes, scales = held["m_codes"].zero_(), held["m_scales"].zero_()
    codes[:, :K // 2] = code[:, 0::2] + 16 * code[:, 1::2]
    scales[:, :scale.shape[1]] = scale
    return codes, scales


def _grid():
    return torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float32, device="cuda")


def _values(code, scale, grid):
    s = torch.ldexp(torch.ones_like(scale, dtype=torch.float32), scale.to(torch.int32) - 127)
    s = torch.where(scale == 255, float("nan"), s)
    return (grid[code.long()].view(*scale.shape, BLOCK) * s[..., None]).view(code.shape[0], -1)


def _unpack(codes, scales, K, grid):
    code = torch.stack((codes & 15, codes >> 4), -1).view(codes.shape[0], -1)
    blocks = -(-K // BLOCK)
    return _values(code[:, :blocks * BLOCK], scales[:, :blocks], grid)[:, :K]


def run(state):
    s, c = state, state["case"]
    if own:
        return _own(s)
    if c["kind"] == "rope":
        first, second, axis = s["pairs"]
        pos = torch.stack(_grid_positions(c), -1) if s["pos"] is None else s["pos"]
        angle = pos[..., axis].double() * s["freq"]  # far positions: 64 bits
        cos, sin = angle.cos().float().unsqueeze(-2), angle.sin().float().unsqueeze(-2)
        return {n: _turn(c, s[n], cos, sin, first, second, s[n + "_norm"]) for n in "qk"}
    if c["kind"] == "residual":
        b = _norm(s["branch"].float(), c["post"], s["post_norm"])
        if s["scale"] is not None:
            b = b * s["scale"]
        if s["gate"] is not None:
            b = b * s["gate"].float().repeat_interleave(c["gate_rows"], 0)[:c["rows"]]
        h = s["x"].float() + b
        out = {"h": h.to(torch.bfloat16)}
        if c["pre"] != "none":
            out["n"] = _norm(h, c["pre"], s["pre_norm"]).to(torch.bfloat16)
        return out
    a = _values(*_quantize(s["x"]), s["grid"])[:, :c["K"]]
    if c["kind"] == "mx4":
        return {"back": a.to(torch.bfloat16)}
    out = {}
    for i, (codes, scales) in enumerate(s["w"]):
        y = a @ _unpack(codes, scales, c["K"], s["grid"]).t() + s["bias"][i]
        if s["res"] is not None:
            y = s["res"].float() + s["res_scale"] * y
        out["y%d" % i] = y.to(torch.bfloat16)
    return out


# ---- the same in 64 bits, from the definitions ---------------------------------------------------
def _norm64(x, kind, affine):
    if kind == "none":
        return x
    mean = x.sum(-1, keepdim=True) / x.shape[-1] if kind == "layer" else torch.zeros_like(x[..., :1])
    var = (x - mean).square().sum(-1, keepdim=True) / x.shape[-1]
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
    parts, start = [], 0
    for a, d in enumerate(sizes):
        x = out[..., start:start + d]
        start += d
        j = torch.arange(d // 2, device=dev, dtype=torch.float64)
        angle = pos.double()[..., a:a + 1] * torch.exp(-2 * j / max(d, 1) * math.log(c["base"]))
        turn = torch.polar(torch.ones_like(angle), angle).unsqueeze(-2)
        if c["pairing"] == "sections":
            z = torch.complex(x[..., :d // 2].contiguous(), x[..., d // 2:].contiguous()) * turn
            parts += [z.real, z.imag]
        else:
            z = torch.complex(x[..., 0::2].contiguous(), x[..., 1::2].contiguous()) * turn
            parts.append(torch.view_as_real(z).flatten(-2))
    return torch.cat(parts + [out[..., start:]], -1)


def _mx4_values64(x):
    """Nearest 4-bit float of every value over its block's scale, found among the fifteen themselves."""
    rows, K = x.shape
    v = torch.nn.functional.pad(x.double(), (0, -K % BLOCK)).view(rows, -1, BLOCK)
    most = v.abs().max(-1, keepdim=True).values
    e = torch.floor(torch.log2(most)) - 2
    # the logarithm of a value next to a power of two may round to it
    e = torch.where(torch.exp2(e + 2) > most, e - 1, e)
    e = torch.where(torch.exp2(e + 3) <= most, e + 1, e).clamp(min=-127.0)
    scale = torch.exp2(e)
    u = v.abs() / scale
    near = torch.zeros_like(u)
    for code in range(1, 8):
        low, high = GRID[code - 1], GRID[code]
        middle = (low + high) / 2
        # from the middle on the upper value, at the middle itself only if its code is even
        near = torch.where(u >= middle if code % 2 == 0 else u > middle, high, near)
    return (near * v.sign() * scale).view(rows, -1)[:, :K]


def _held64(codes, scales, K):
    low, high = (codes % 16).long(), (codes // 16).long()
    grid = torch.tensor(GRID, dtype=torch.float64, device=codes.device)
    v = torch.stack([grid[n % 8] * (1 - 2 * (n // 8)) for n in (low, high)], -1).flatten(1)[:, :K]
    return v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, 1)[:, :K]


def exact(case, seed):
    c = case
    s = prepare(c, seed)
    if c["kind"] == "rope":
        pos = s["pos"]
        if pos is None:
            P, n_w = c["n_special"], c["n_w"]
            t = torch.arange(_tokens(c), device="cuda")
            L = P + c["n_h"] * n_w
            p = t % L - P
            pos = torch.stack((t // L + c["t0"], torch.where(p < 0, -1, p // n_w) + 1, torch.where(p < 0, -1, p % n_w) + 1), -1)[None]
        return {n: torch.cat([_turn64(c, s[n][b:b + 1], pos[min(b, pos.shape[0] - 1)][None], s[n + "_norm"])
                              for b in range(c["B"])]) for n in "qk"}
    if c["kind"] == "residual":
        add = _norm64(s["branch"].double(), c["post"], s["post_norm"])
        if s["gate"] is not None:
            add = add * s["gate"].double()[torch.arange(c["rows"], device="cuda") // c["gate_rows"]]
        h = s["x"].double() + (add if s["scale"] is None else add * s["scale"].double())
        return {"h": h} if c["pre"] == "none" else {"h": h, "n": _norm64(h, c["pre"], s["pre_norm"])}
    a = _mx4_values64(s["x"])
    if c["kind"] == "mx4":
        return {"back": a}
    out = {}
    for i, held in enumerate(s["w"]):
        y = torch.addmm(s["bias"][i].double(), a, _held64(*held, c["K"]).t().contiguous())
        out["y%d" % i] = y if s["res"] is None else s["res"].double() + y * s["res_scale"].double()
    return out
