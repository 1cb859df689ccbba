"""Oracle of the operators for prompts and 8-bit rows on a paged cache (numpy, fp64, written from the definitions in
include/halo.h): the append with per-head norms, 8-bit rows and their way back, causal attention of packed chunks.

All inputs are float64 arrays that hold the values the GPU was given.
"""
from __future__ import annotations

import numpy as np

from oracle.attention_block_ref import rotate


def norm_turn(x, w, eps, pos, inv_freq, interleaved, turn_scale):
    """x [n_tok][heads][dh]: normed over dh with the gain w (None: not), the elements that the position turns times turn_scale."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    out = rotate(x, pos, inv_freq, interleaved)
    r = 0 if inv_freq is None else 2 * len(inv_freq)
    out[..., :r] *= turn_scale
    return out


def eight_rows(x):
    """(codes, scale bytes, values) of rows x [..., dh]: e the smallest whole number with amax <= 448 * 2^e in [-117, 119]."""
    flat = x.reshape(-1, x.shape[-1])
    codes, scales, values = np.zeros(flat.shape, np.uint8), np.zeros(len(flat), np.uint8), np.zeros(flat.shape)
    grid = np.array([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)])[:127]
    for i, row in enumerate(flat):
        if not np.isfinite(row).all():
            scales[i], values[i] = 255, np.nan
            continue
        amax, e = np.abs(row).max(), -117
        while amax > 448 * 2.0 ** e and e < 119:
            e += 1
        a = np.abs(row) / 2.0 ** e
        below = np.clip(np.searchsorted(grid, a, side="right") - 1, 0, 125)
        low, high = a - grid[below], grid[below + 1] - a
        code = below + ((high < low) | ((high == low) & (below % 2 == 1)))      # ties to the even code
        codes[i] = code + 128 * np.signbit(row)
        scales[i], values[i] = e + 127, np.copysign(grid[code], row) * 2.0 ** e
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1]), values.reshape(x.shape)


def prompt_mha(q, q_start, K, V, table, lens, scale, keep=None):
    """out, lse, the mean of |V| under the weights, the largest sum |q||k| scale of a row, which rows belong to a sequence, bad."""
    n_tok, H, dh = q.shape
    Hk, page_size, cap = K.shape[1], K.shape[2], table.shape[1] * K.shape[2]
    out, size = np.zeros((n_tok, H, dh)), np.zeros((n_tok, H, dh))
    lse, reach = np.full((n_tok, H), -np.inf), np.zeros((n_tok, H))
    mine, bad, end = np.zeros(n_tok, bool), False, 0
    for s in range(len(lens)):
        a, b, length = int(q_start[s]), int(q_start[s + 1]), int(lens[s])
        if not 0 <= length <= cap:
            bad, length = True, 0
        if not 0 <= a <= b <= n_tok or a < end:      # rows of two sequences belong to the first one
            bad, end = True, max(end, b) if 0 <= a <= b <= n_tok else end
            continue
        end = b
        mine[a:b] = True
        for t in range(a, b):
            for p_end in [length - (b - t) + 1]:
                places = [(int(table[s, p // page_size]), p % page_size) for p in range(max(p_end, 0))]
                good = [(g, o) for g, o in places if 0 <= g < K.shape[0]]
                bad |= (keep is None or bool(np.any(keep))) and len(good) != len(places)
                if not good:
                    continue
                pages, rows = np.array(good).T
                for h in range(H):
                    if keep is not None and not keep[h]:
                        continue
                    k, v = K[pages, h // (H // Hk), rows], V[pages, h // (H // Hk), rows]
                    score = k @ q[t, h] * scale
                    m = score.max()
                    if m == -np.inf:
                        continue
                    w = np.exp(score - m)
                    out[t, h], size[t, h] = w @ v / w.sum(), w @ np.abs(v) / w.sum()
                    lse[t, h] = m + np.log(w.sum())
                    reach[t, h] = (np.abs(k) @ np.abs(q[t, h])).max() * abs(scale)
    return out, lse, size, reach, mine, bad
