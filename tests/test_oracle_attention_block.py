"""Pins of the attention-block oracle: values worked out by hand, dense forms, brute force."""
import numpy as np

from oracle import attention_block_ref as A


def test_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 9.0]]])
    quarter = np.array([np.pi / 2, np.pi])                        # angles at position 1
    got = A.rotate(x, np.array([1]), quarter, False)[0, 0]        # pairs (0, 2) and (1, 3); element 4 is copied
    assert np.allclose(got, [-3, -2, 1, -4, 9])
    got = A.rotate(x, np.array([1]), quarter, True)[0, 0]         # pairs (0, 1) and (2, 3)
    assert np.allclose(got, [-2, 1, -3, -4, 9])
    assert (A.rotate(x, np.array([0]), quarter, True) == x).all()
    # scores of turned rows depend on the difference of positions only
    rng = np.random.default_rng(0)
    q, k, f = rng.normal(size=(1, 1, 8)), rng.normal(size=(1, 1, 8)), 0.3 ** np.arange(4)
    dot = lambda a, b: float((A.rotate(q, np.array([a]), f, False) * A.rotate(k, np.array([b]), f, False)).sum())  # noqa: E731
    assert np.isclose(dot(7, 3), dot(104, 100))


def test_append_places_rows_and_skips_padding():
    K = np.zeros((4, 1, 2, 2))
    V = K.copy()
    k, v = np.arange(6.0).reshape(3, 1, 2) + 1, np.arange(6.0).reshape(3, 1, 2) + 11
    q_out, K2, V2, bad = A.paged_append(None, k, v, np.array([3, -1, 0]), np.array([0, 0, 1]), np.array([[2, 1], [3, 0]]),
                                        None, False, None, K, V)
    assert q_out is None and not bad
    assert (K2[1, 0, 1] == [1, 2]).all() and (K2[3, 0, 0] == [5, 6]).all() and (V2[3, 0, 0] == [15, 16]).all()
    assert np.count_nonzero(K2) == 4
    assert A.paged_append(None, k, v, np.array([4, -1, 0]), None, np.array([[2, 1]] * 3), None, False, None, K, V)[3]


def test_attention_against_a_dense_softmax_and_by_hand():
    rng = np.random.default_rng(1)
    K, V = rng.normal(size=(5, 2, 3, 4)), rng.normal(size=(5, 2, 3, 4))
    q, table = rng.normal(size=(1, 4, 4)), np.array([[4, 0, 2]])
    out, lse, _, _, bad = A.paged_mha(q, K, V, table, [7], 0.5)
    rows_k = np.concatenate([K[4], K[0], K[2]], axis=1)[:, :7]
    rows_v = np.concatenate([V[4], V[0], V[2]], axis=1)[:, :7]
    for h in range(4):
        e = np.exp(rows_k[h // 2] @ q[0, h] * 0.5)
        assert np.allclose(out[0, h], (e / e.sum()) @ rows_v[h // 2]) and np.isclose(lse[0, h], np.log(e.sum()))
    assert not bad
    out, lse, _, _, _ = A.paged_mha(q, K, V, table, [0], 0.5)
    assert (out == 0).all() and (lse == -np.inf).all()
    out, lse, _, _, _ = A.paged_mha(q, K, V, table, [1], 0.5)       # one position: its value
    assert np.allclose(out[0, 3], V[4, 1, 0])
    assert A.paged_mha(q, K, V, table, [10], 0.5)[4] and A.paged_mha(q, K, V, np.array([[4, 5, 2]]), [7], 0.5)[4]


def test_norm_glue_by_hand():
    h, x = A.norm_glue(np.array([[1.0, 1.0]]), np.array([[3.0, 4.0]]), None, None, 2.0, np.array([1.0, 10.0]), 0.0)
    assert np.allclose(h, [[7, 9]]) and np.allclose(x, [[7 / np.sqrt(65), 90 / np.sqrt(65)]])
    h, _ = A.norm_glue(np.zeros((1, 2)), np.array([[3.0, 4.0]]), np.array([2.0, 1.0]), np.array([[1.0, 0.5]]), 1.0, None, 0.0)
    assert np.allclose(h, [[6 / np.sqrt(12.5), 2 / np.sqrt(12.5)]])


def test_mx4_by_hand_and_by_search():
    w = np.zeros((1, 128))
    w[0, :8] = [6, 5, 2.5, 0.25, -0.75, -7.9, 0.2, -0.0]            # top 7.9: 2^2 <= 7.9, unit 1
    w[0, 32:35] = [1.0, 0.125, 0.1875]                              # unit 1/4: 4, 0.5, 0.75 -> tie to 1 (even code)
    codes, scales = A.mx4_quantize(w)
    assert codes[0, :8].tolist() == [7, 6, 4, 0, 8 + 2, 8 + 7, 0, 8]
    assert scales[0].tolist() == [127, 125, 0, 0] and codes[0, 32:35].tolist() == [6, 1, 2]
    Q, S = A.mx4_pack(codes, scales)
    assert Q[0, 0] == 7 | 6 << 4 and S[:4].tolist() == [127, 125, 0, 0] and len(S) == 512
    vals = A.mx4_unpack(Q, S, 1, 128)
    assert vals[0, :6].tolist() == [6, 4, 2, 0, -1, -6] and vals[0, 32:35].tolist() == [1.0, 0.125, 0.25]
    w[0, 40] = np.inf
    assert A.mx4_quantize(w)[1][0].tolist() == [127, 255, 0, 0]
    # values on the grid come back, and no other grid value is nearer
    rng = np.random.default_rng(2)
    w = rng.normal(size=(3, 256)) * 10.0 ** rng.integers(-6, 6, size=(3, 1))
    Q, S = A.mx4_pack(*A.mx4_quantize(w))
    v = A.mx4_unpack(Q, S, 3, 256)
    c2, s2 = A.mx4_quantize(v)
    assert (A.mx4_unpack(*A.mx4_pack(c2, s2), 3, 256) == v).all()
    unit = np.repeat(2.0 ** (A.mx4_quantize(w)[1].astype(float) - 127), 32, axis=1)
    grid = np.concatenate([A.MX4_VALUES, -A.MX4_VALUES])
    assert (np.abs(w - v) <= np.abs(w[..., None] - grid * unit[..., None]).min(-1) + 1e-15 * np.abs(w)).all()
