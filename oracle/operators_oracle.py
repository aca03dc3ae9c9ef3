"""CPU oracle for the operators around a block's attention (TEST INFRASTRUCTURE ONLY).

Everything is float64 numpy from the definitions: norms, rotary positions on three axes, the seam
between branches, microscaled 4-bit floats and products of matrices held so.  Nothing is rounded here
except where a format is the subject.

Pins (tests/test_operators_api.py): the norms against torch.nn.functional in float64; a rotation
against complex multiplication, against its inverse and against the dependence of <q, k> on the
difference of positions alone; the 4-bit rounding against a search over all fifteen values; reading
back what was quantised; the packed layout byte by byte.
"""
from __future__ import annotations

import math

import numpy as np

NONE, LAYER, RMS = 0, 1, 2
SECTIONS, NEIGHBOURS, HEAD = 0, 1, 2
GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def norm(x, kind, eps=1e-5, gamma=None, beta=None):
    """Over the last axis."""
    x = np.asarray(x, dtype=np.float64)
    if kind == NONE:
        return x
    if kind == LAYER:
        x = x - x.mean(axis=-1, keepdims=True)
    y = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    if gamma is not None:
        y = y * gamma
    return y if beta is None else y + beta


def rope_pairs(pairing, axes, base):
    """[(first channel, second channel, axis, angle per position)] for axes = (d_t, d_h, d_w)."""
    out, start = [], 0
    r = sum(axes)
    for axis, d in enumerate(axes):
        for j in range(d // 2):
            if pairing == HEAD:
                i = start // 2 + j
                out.append((i, i + r // 2, axis, base ** (-2.0 * i / r)))
            elif pairing == SECTIONS:
                out.append((start + j, start + j + d // 2, axis, base ** (-2.0 * j / d)))
            else:
                out.append((start + 2 * j, start + 2 * j + 1, axis, base ** (-2.0 * j / d)))
        start += d
    return out


def grid_positions(N, n_h, n_w, n_special, t0=0, patch0=0):
    """int64 [N*L, 3]: time, row, column of every token."""
    out = []
    for f in range(N):
        out += [(t0 + f, 0, 0)] * n_special
        out += [(t0 + f, patch0 + r, patch0 + c) for r in range(n_h) for c in range(n_w)]
    return np.array(out, dtype=np.int64)


def rope(x, pos, pairing, axes, base):
    """x: [tokens, H, D]; pos: [tokens, 3]."""
    x = np.asarray(x, dtype=np.float64)
    y = x.copy()
    for a, b, axis, freq in rope_pairs(pairing, axes, base):
        angle = pos[:, axis].astype(np.float64) * freq
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def seam(x, branch, post, pre, scale=None, gate=None, gate_rows=0):
    """post, pre: (kind, eps, gamma, beta).  Returns h and n (None without a norm)."""
    h = np.asarray(x, dtype=np.float64)
    if branch is not None:
        add = norm(branch, *post)
        if scale is not None:
            add = add * scale
        if gate is not None:
            add = add * gate[np.arange(len(h)) // gate_rows]
        h = h + add
    return h, (None if pre[0] == NONE else norm(h, *pre))


def quantize(x):
    """float64 [rows, K] -> codes [rows, blocks, 32], scale bytes [rows, blocks]; K filled with zeros."""
    rows, K = x.shape
    v = np.zeros((rows, -(-K // 32) * 32))
    v[:, :K] = x
    v = v.reshape(rows, -1, 32)
    most = np.abs(v).max(axis=-1)  # NaN wins
    bad = ~np.isfinite(most)
    # frexp: most = m 2^e with 0.5 <= m < 1, so floor(log2(most)) = e - 1
    e = np.frexp(np.where(bad, 1.0, most))[1] - 1 - 2
    s = np.where(most == 0, 0, np.maximum(e + 127, 0))
    u = np.abs(np.where(bad[..., None], 0.0, v)) * np.exp2(127.0 - s)[..., None]
    codes = np.zeros(u.shape, dtype=np.int64)
    for k in range(1, 8):
        middle = (GRID[k - 1] + GRID[k]) / 2
        codes = np.where(u >= middle if k % 2 == 0 else u > middle, k, codes)
    codes += 8 * (np.signbit(v) & ~bad[..., None])
    return codes, np.where(bad, 255, s)


def pack(codes, scales, code_stride, scale_stride):
    """uint8 [rows, code_stride] and [rows, scale_stride] as a matrix is held."""
    rows = codes.shape[0]
    flat = codes.reshape(rows, -1)
    c = np.zeros((rows, code_stride), dtype=np.uint8)
    c[:, :flat.shape[1] // 2] = flat[:, 0::2] | flat[:, 1::2] << 4
    s = np.zeros((rows, scale_stride), dtype=np.uint8)
    s[:, :scales.shape[1]] = scales
    return c, s


def values(c, s, K):
    """The float64 [rows, K] that packed codes and scales stand for."""
    k = np.arange(K)
    code = (c[:, k // 2] >> (4 * (k % 2)).astype(np.uint8)) & 15
    byte = s[:, k // 32].astype(np.int64)
    v = GRID[code & 7] * np.where(code & 8, -1.0, 1.0) * np.exp2(byte - 127.0)
    return np.where(byte == 255, math.nan, v)


def linear(a, w, bias=None, residual=None, res_scale=None):
    """a, w: values in float64.  Returns the result and the sum of the magnitudes that it is made of."""
    y, size = a @ w.T, np.abs(a) @ np.abs(w).T
    if bias is not None:
        y, size = y + bias, size + np.abs(bias)
    if residual is not None:
        if res_scale is not None:
            y, size = y * res_scale, size * np.abs(res_scale)
        y, size = residual + y, size + np.abs(residual)
    return y, size
