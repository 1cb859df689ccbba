"""Pins of the oracle of prompts and 8-bit rows: known codes, the norm's length, causal rows one by one against one-token attention."""
import numpy as np

from oracle import attention_block_ref as A
from oracle import paged_prompt_ref as P


def test_eight_bit_codes_of_known_values():
    x = np.array([[448.0, -448.0, 1.0, 1.0625, 1.1875, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, 0.0, -0.0, 17.0, 19.0]])
    codes, scales, values = P.eight_rows(x)
    assert scales.tolist() == [127]
    # 1.0625 and 1.1875 lie between two codes: the even one; half the smallest number becomes 0, one and a half of it two
    assert codes[0].tolist() == [0x7e, 0xfe, 0x38, 0x38, 0x3a, 1, 0, 2, 0, 128, 0x58, 0x5a]
    assert values[0].tolist() == [448, -448, 1, 1, 1.25, 2.0 ** -9, 0, 2.0 ** -8, 0, 0, 16, 20]
    assert P.eight_rows(x * 2.0 ** -30)[1].tolist() == [97] and (P.eight_rows(x * 2.0 ** -30)[0] == codes).all()
    assert P.eight_rows(np.array([[448.1, 0.0]]))[1].tolist() == [128]                   # past the largest: the next power
    assert P.eight_rows(np.zeros((2, 4)))[1].tolist() == [10, 10]
    c, s, v = P.eight_rows(np.array([[1.0, np.nan], [np.inf, 1.0]]))
    assert s.tolist() == [255, 255] and (c == 0).all() and np.isnan(v).all()


def test_eight_bit_rows_are_off_by_half_a_step_at_most():
    x = np.random.default_rng(0).standard_normal((50, 64)) * 2.0 ** np.arange(-25, 25)[:, None]
    _, scales, v = P.eight_rows(x)
    unit = 2.0 ** (scales.astype(float) - 127)[:, None]
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, unit * 2.0 ** -10)).all()
    assert (np.abs(x).max(-1) <= 448 * unit[:, 0]).all() and (np.abs(x).max(-1) > 224 * unit[:, 0]).all()


def test_norm_and_turn():
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((3, 2, 8)), rng.standard_normal(8)
    y = P.norm_turn(x, w, 0.0, np.array([0, 5, 9]), np.array([1.0, 0.1]), True, 1.5)
    z = P.norm_turn(x, w, 0.0, np.array([0, 0, 0]), None, True, 1.5)
    assert np.allclose((z / w * z / w).mean(-1), 1)
    assert np.allclose(np.hypot(y[..., 0:4:2], y[..., 1:4:2]), 1.5 * np.hypot(z[..., 0:4:2], z[..., 1:4:2]))
    assert np.array_equal(y[..., 4:], z[..., 4:]) and np.allclose(y[0, :, :4], 1.5 * z[0, :, :4])


def test_rows_of_a_chunk_are_one_token_attentions():
    rng = np.random.default_rng(2)
    H, Hk, dh, page = 4, 2, 16, 3
    K, V = rng.standard_normal((8, Hk, page, dh)), rng.standard_normal((8, Hk, page, dh))
    table = np.array([[3, 1, 5], [0, 7, 99]])
    q, start, lens = rng.standard_normal((9, H, dh)), np.array([0, 4, 8]), np.array([7, 3])      # the second: its first row sees nothing
    out, lse, size, reach, mine, bad = P.prompt_mha(q, start, K, V, table, lens, 0.5)
    assert mine.tolist() == [True] * 8 + [False] and not bad and (lse[4] == -np.inf).all() and (out[4] == 0).all()
    for s in range(2):
        for t in range(start[s], start[s + 1]):
            n = max(lens[s] - (start[s + 1] - t) + 1, 0)
            one = A.paged_mha(q[t:t + 1], K, V, table[s:s + 1], np.array([n]), 0.5)
            assert np.allclose(out[t], one[0][0]) and np.allclose(lse[t], one[1][0]) and np.allclose(size[t], one[2][0])
    assert P.prompt_mha(q, start, K, V, table, np.array([7, 9]), 0.5)[5]         # a page out of range
    assert P.prompt_mha(q, np.array([0, 4, 2]), K, V, table, lens, 0.5)[5]
