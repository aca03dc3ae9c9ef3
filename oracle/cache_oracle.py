"""Oracle for attention to keys of another length and the paged key/value cache (TEST INFRASTRUCTURE ONLY).

Float64 torch from the definitions, on whatever device the tensors lie.  Nothing is rounded here.

Pins (tests/test_cross_api.py): attention against torch.nn.functional.scaled_dot_product_attention in
float64; a page's layout against agg_kc_offset / agg_vc_offset element by element.
"""
from __future__ import annotations

import math

import torch


def attention(q, k, v, scale, q_lens=None, k_lens=None):
    """q [B, NQ, H, 64], k and v [B, NK, H_kv, 64].  Returns O [B, NQ, H, 64], lse [B, H, NQ], the sum of
    probability times |v| (what errors of probabilities multiply) and the largest sum of |q k| * scale of a row's
    keys [B, NQ, H, 1]; rows that do not exist hold NaN everywhere."""
    B, NQ, H, D = q.shape
    group = H // k.shape[2]
    o = torch.full((B, NQ, H, D), math.nan, dtype=torch.float64, device=q.device)
    size = o.clone()
    lse = torch.full((B, H, NQ), math.nan, dtype=torch.float64, device=q.device)
    dots = torch.full((B, NQ, H, 1), math.nan, dtype=torch.float64, device=q.device)
    for b in range(B):
        nq = NQ if q_lens is None else min(max(int(q_lens[b]), 0), NQ)
        nk = k.shape[1] if k_lens is None else min(max(int(k_lens[b]), 0), k.shape[1])
        for h in range(H):
            if nk == 0:
                o[b, :nq, h] = size[b, :nq, h] = 0.0
                dots[b, :nq, h] = 0.0
                lse[b, h, :nq] = -math.inf
                continue
            kh, vh = k[b, :nk, h // group].double(), v[b, :nk, h // group].double()
            for at in range(0, nq, 4096):
                part = slice(at, min(nq, at + 4096))
                qh = q[b, part, h].double()
                logit = (qh @ kh.t().contiguous()) * scale
                p = torch.softmax(logit, -1)
                o[b, part, h] = p @ vh
                size[b, part, h] = p @ vh.abs()
                lse[b, h, part] = torch.logsumexp(logit, -1)
                dots[b, part, h, 0] = (qh.abs() @ kh.abs().t().contiguous()).amax(-1) * scale
    return o, lse, size, dots


def k_place(row, d):
    """Element of channel d of a page's row in the keys' tile: chunks of eight channels, 32 rows beside each other."""
    half, r = divmod(row, 32)
    return ((half * 8 + d // 8) * 32 + r) * 8 + d % 8


def v_place(row, d):
    """... in the values' tile: chunks of eight rows of a channel: four, and the four that lie eight rows on."""
    sixteen, u = divmod(row, 16)
    return ((sixteen * 2 + (u % 8) // 4) * 64 + d) * 8 + (u // 8) * 4 + u % 4


def _places(place, device):
    return torch.tensor([[place(r, d) for d in range(64)] for r in range(64)], device=device)


def rows_of(pool, pages, place):
    """The rows [B, 64 * entries, H, 64] that a page table [B, entries] lists in a pool [n_pages, H, 4096]."""
    at = _places(place, pool.device)
    tiles = pool[pages.long().clamp(0, pool.shape[0] - 1)]           # [B, entries, H, 4096]
    return tiles[..., at].permute(0, 1, 3, 2, 4).reshape(pages.shape[0], -1, pool.shape[1], 64)


def store(pool, pages, place, b, row, values):
    """Row `row` of sequence b becomes `values` [H, 64]; nothing happens outside the table and the pool."""
    if not 0 <= row < 64 * pages.shape[1]:
        return
    page = int(pages[b, row // 64])
    if 0 <= page < pool.shape[0]:
        pool[page][:, _places(place, pool.device)[row % 64]] = values
