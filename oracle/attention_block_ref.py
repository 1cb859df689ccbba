"""Oracle of the batched attention-block operators (numpy, fp64, written from the definitions in include/halo.h):
paged K/V append, paged attention, the normalised residual, microscaled 4-bit rows.

All inputs are float64 arrays that hold the values the GPU was given; nothing here rounds to a narrower type.
"""
from __future__ import annotations

import numpy as np


def rotate(x: np.ndarray, pos: np.ndarray, inv_freq, interleaved: bool) -> np.ndarray:
    """x [n_tok][heads][dh] turned by pos [n_tok]; pairs (2i, 2i + 1) or (i, i + r / 2) of the first r = 2 * len(inv_freq)."""
    out = x.copy()
    r = 0 if inv_freq is None else 2 * len(inv_freq)
    for i in range(r // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
        angle = pos.astype(np.float64) * inv_freq[i]
        c, s = np.cos(angle)[:, None], np.sin(angle)[:, None]
        out[:, :, a] = x[:, :, a] * c - x[:, :, b] * s
        out[:, :, b] = x[:, :, a] * s + x[:, :, b] * c
    return out


def paged_append(q, k, v, pos, seq, table, inv_freq, interleaved, q_out, K, V):
    """Copies of q_out, K, V with every token of the call in its place, and whether a token was out of range."""
    q_out, K, V = (None if t is None else t.copy() for t in (q_out, K, V))
    page_size, bad = K.shape[2], False
    kr = rotate(k, pos, inv_freq, interleaved)
    qr = None if q is None else rotate(q, pos, inv_freq, interleaved)
    for t in range(k.shape[0]):
        p, s = int(pos[t]), t if seq is None else int(seq[t])
        if p < 0:
            continue
        if not (0 <= s < table.shape[0] and p // page_size < table.shape[1] and 0 <= table[s, p // page_size] < K.shape[0]):
            bad = True
            continue
        page = table[s, p // page_size]
        K[page, :, p % page_size] = kr[t]
        V[page, :, p % page_size] = v[t]
        if q is not None:
            q_out[t] = qr[t]
    return q_out, K, V, bad


def paged_mha(q, K, V, table, lens, scale, keep=None):
    """out, lse, the mean of |V| under the weights (error bounds need it), the largest sum |q||k| scale of a row, bad."""
    n, H, dh = q.shape
    Hk, page_size = K.shape[1], K.shape[2]
    out, size = np.zeros((n, H, dh)), np.zeros((n, H, dh))
    lse, reach, bad = np.full((n, H), -np.inf), np.zeros((n, H)), False
    for s in range(n):
        length = int(lens[s])
        if length < 0 or length > table.shape[1] * page_size:
            bad, length = True, 0
        places = [(int(table[s, p // page_size]), p % page_size) for p in range(length)]
        good = [(g, o) for g, o in places if 0 <= g < K.shape[0]]
        any_head = keep is None or np.any(keep)
        bad |= bool(any_head) and len(good) != len(places)
        if not good:
            continue
        pages, offs = np.array(good).T
        for h in range(H):
            if keep is not None and not keep[h]:
                continue
            Kh, Vh = K[pages, h // (H // Hk), offs], V[pages, h // (H // Hk), offs]
            score = Kh @ q[s, h] * scale
            reach[s, h] = (np.abs(Kh) @ np.abs(q[s, h])).max() * abs(scale)
            m = score.max()
            if m == -np.inf:
                continue
            w = np.exp(score - m)
            lse[s, h] = m + np.log(w.sum())
            w /= w.sum()
            out[s, h], size[s, h] = w @ Vh, w @ np.abs(Vh)
    return out, lse, size, reach, bad


def norm_glue(h, y, w_post, gate, res_scale, w_pre, eps):
    norm = lambda v: v / np.sqrt(np.mean(v * v, axis=-1, keepdims=True) + eps)  # noqa: E731
    if y is not None:
        u = norm(y) * w_post if w_post is not None else y
        h = h + res_scale * (u if gate is None else gate * u)
    x = norm(h)
    return h, x if w_pre is None else x * w_pre


MX4_VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mx4_quantize(W):
    """codes [n][d] (0..15) and scale bytes [n][d / 32]; an element at a time, nearest value, ties to the even code."""
    n, d = W.shape
    codes, scales = np.zeros((n, d), dtype=np.uint8), np.zeros((n, d // 32), dtype=np.uint8)
    for r in range(n):
        for b in range(d // 32):
            block = W[r, b * 32:(b + 1) * 32]
            if not np.all(np.isfinite(block)):
                scales[r, b] = 255
                continue
            top = np.abs(block).max()
            e = -127 if top == 0 else max(int(np.floor(np.log2(top))) - 2, -127)
            if top > 0 and e > -127:     # log2 of a value next to a power of two may round across it
                while top >= 2.0 ** (e + 3):
                    e += 1
                while e > -127 and top < 2.0 ** (e + 2):
                    e -= 1
            scales[r, b] = e + 127
            a = np.abs(block) / 2.0 ** e
            dist = np.abs(a[:, None] - MX4_VALUES[None])
            best = dist.min(axis=1)
            for i in range(32):
                near = np.flatnonzero(dist[i] == best[i])
                idx = near[0] if len(near) == 1 or near[0] % 2 == 0 else near[1]
                codes[r, b * 32 + i] = idx + (8 if np.signbit(block[i]) else 0)
    return codes, scales


def mx4_pack(codes, scales):
    """Code bytes [n][d / 2] and the scale blocks of 128 rows x 4."""
    n, nb = scales.shape
    S = np.zeros((n + 127) // 128 * (nb // 4) * 512, dtype=np.uint8)
    for r in range(n):
        for b in range(nb):
            S[((r // 128) * (nb // 4) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4] = scales[r, b]
    return codes[:, 0::2] | (codes[:, 1::2] << 4), S


def mx4_unpack(Q, S, n, d):
    """Values [n][d] of packed rows."""
    codes = np.empty((n, d), dtype=np.int64)
    codes[:, 0::2], codes[:, 1::2] = Q & 15, Q >> 4
    r, b = np.arange(n)[:, None], np.arange(d // 32)[None]
    byte = S[((r // 128) * (d // 128) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4].astype(np.float64)
    unit = np.where(byte == 255, np.nan, 2.0 ** (byte - 127))
    return np.where(codes > 7, -1.0, 1.0) * MX4_VALUES[codes & 7] * np.repeat(unit, 32, axis=1)
