"""Paged K/V append, paged attention and the normalised residual against the fp64 oracle.

Bounds (u = half a rounding step of the type: 2^-8 bf16, 2^-24 fp32, relative to the value):
  append     |a cos - b sin| is formed in fp32 from sine and cosine within 4e-7: 6e-7 (|a| + |b|) + u |result|
  attention  S = the weighted mean of |V|.  Scores are off by at most e = (2^-21 + dh 2^-24) max_p sum|q k| scale + 2^-20
             max|score| (products, sums in fp32, the exponent's argument), a weight by 2 e relative; bf16 weights are
             rounded once more (2^-8): (2 e + 1e-5 + [2^-8]) S + u |out|.  lse: e + 1e-6 (1 + |lse|).
  norm       sums of squares of d positive terms in fp32, at most 2^-18 relative: 2^-18 |u| + 2^-23 |h|; x: that relative
             to the row's size + u |x|.
"""
import numpy as np
import pytest
import torch

from oracle import attention_block_ref as A
from paper_2601_11676_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, B.BF16, 2.0 ** -8), "f32": (torch.float32, B.F32, 2.0 ** -24)}


def host(t):
    return None if t is None else t.detach().double().cpu().numpy()


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, shape, t):
    return torch.randn(shape, generator=g, device=DEV).to(t)


def caches(g, t, n_pages, Hk, page, dh, interleaved):
    """K and V caches, dense or with a sequence's K and V pages side by side in one pool; and the page stride."""
    if not interleaved:
        return randn(g, (n_pages, Hk, page, dh), t), randn(g, (n_pages, Hk, page, dh), t), 0
    pool = randn(g, (n_pages, 2, Hk, page, dh), t)
    return pool[:, 0], pool[:, 1], 2 * Hk * page * dh


def block_table(g, lens, page, cols=None):
    need = [-(-max(n, 0) // page) for n in lens]
    cols = cols or max(max(need), 1)
    order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32).tolist()
    table = torch.full((len(lens), cols), -1, dtype=torch.int32)
    for s, n in enumerate(need):
        table[s, :n] = torch.tensor(order[:n], dtype=torch.int32)
        order = order[n:]
    return table.to(DEV), sum(need) + 2


def status():
    return torch.zeros(1, dtype=torch.int32, device=DEV)


# ---- append --------------------------------------------------------------------------------------------------------

APPEND = [
    # dtype, H, Hk, dh, page, rotary, interleaved pairs, positions, sequences, pool of K and V pages
    ("bf16", 4, 2, 64, 16, 64, False, [0], None, False),
    ("bf16", 32, 32, 128, 16, 128, False, [5, 17, 0, 4095, 16], None, False),
    ("bf16", 8, 2, 80, 16, 40, False, [3, -1, 18, 19, 20, -1, 7], [1, 0, 0, 0, 0, 0, 2], True),   # half of 20: no whole chunks
    ("bf16", 5, 1, 16, 7, 16, True, [6, 7, 8, 13], [0, 0, 0, 0], False),                      # pages of 7
    ("bf16", 4, 4, 256, 32, 128, True, [31, 32], None, True),
    ("bf16", 8, 8, 128, 16, 0, False, [1, 2, 3], [0, 0, 0], False),                           # no rotation
    ("f32", 8, 2, 64, 16, 64, False, [100000, 99999, 12], None, False),                      # far positions
    ("f32", 3, 1, 48, 16, 20, True, [1, 15, 16], None, True),
    ("f32", 4, 2, 32, 1, 24, False, [0, 1, 2, 3, 4], [0, 0, 0, 1, 1], False),                  # pages of one position
    ("f32", 2, 2, 64, 16, 10, False, [11, 33], None, False),
    ("bf16", 6, 3, 48, 48, 20, True, [47, 48, 95, 1], None, False),                           # a chunk ends behind the last pair
    ("bf16", 16, 2, 128, 16, 128, False, list(range(128)) * 6, [i // 128 for i in range(768)], True),   # more tokens than thread blocks at once
]


@pytest.mark.parametrize("case", range(len(APPEND)))
@pytest.mark.parametrize("with_q", [True, False])
def test_append_matches_oracle(case, with_q):
    dtype, H, Hk, dh, page, rotary, inter, pos, seq, pool = APPEND[case]
    t, code, u = TYPES[dtype]
    g, n = gen(case), len(pos)
    n_seq = n if seq is None else max(seq) + 1
    cols = max(pos) // page + 2
    n_pages = n_seq * 8
    # far positions: the table is long, its entries repeat 8 pages per sequence (the places written stay distinct)
    table = (torch.arange(cols, device=DEV)[None] % 8 + 8 * torch.arange(n_seq, device=DEV)[:, None]).to(torch.int32)
    K, V, stride = caches(g, t, n_pages, Hk, page, dh, pool)
    qkv = randn(g, (n, H + 2 * Hk, dh), t)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    inv = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device=DEV) / max(rotary, 1)) if rotary else None
    q_out = randn(g, (n, H, dh), t) if with_q else None
    p32 = torch.tensor(pos, dtype=torch.int32, device=DEV)
    s32 = None if seq is None else torch.tensor(seq, dtype=torch.int32, device=DEV)
    want = A.paged_append(host(q) if with_q else None, host(k), host(v), np.array(pos), seq, table.cpu().numpy(),
                          None if inv is None else host(inv), inter, host(q_out), host(K), host(V))
    before = [host(x) for x in (q_out, K, V)]
    st = status()
    sh = B.paged_shape(H, Hk, dh, page, n_pages, cols, code, stride)
    B.halo_paged_kv_append(sh, q if with_q else None, k, v, p32, s32, table, inv, inter, q_out, K, V, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and not want[3]
    size = 2 * max(float(k.abs().max()), float(q.abs().max()))      # |a| + |b| of any pair
    for got, ref, old in zip((q_out, K, V), want, before):
        if got is None:
            continue
        got = host(got)
        same = ref == old                                            # what the call does not touch keeps its bits
        assert (got[same] == old[same]).all()
        assert (np.abs(got - ref) <= 6e-7 * size + u * np.abs(ref)).all()
    # in place: the turned queries replace the projection's, padding rows stay
    if with_q:
        kept = q.clone()
        B.halo_paged_kv_append(sh, q, k, v, p32, s32, table, inv, inter, q, K, V, st)
        torch.cuda.synchronize()
        for i in range(n):
            assert torch.equal(q[i], q_out[i] if pos[i] >= 0 else kept[i])


def test_append_skips_tokens_that_are_out_of_range():
    t, code, _ = TYPES["bf16"]
    g = gen(3)
    K, V, _ = caches(g, t, 4, 2, 16, 64, False)
    K0, V0 = K.clone(), V.clone()
    table = torch.tensor([[0, 1], [2, 9], [-1, 3]], dtype=torch.int32, device=DEV)
    sh = B.paged_shape(2, 2, 64, 16, 4, 2, code)
    qkv = randn(g, (6, 3, 2, 64), t)
    q, k, v = qkv[:, 0], qkv[:, 1], qkv[:, 2]
    pos = torch.tensor([32, 16, 0, 3, 2, 5], dtype=torch.int32, device=DEV)    # behind the table; page 9; page -1; ok ...
    seq = torch.tensor([0, 1, 2, 0, 3, -1], dtype=torch.int32, device=DEV)     # ... ; sequences 3 and -1
    q_out, st = torch.full((6, 2, 64), 7.0, dtype=t, device=DEV), status()
    B.halo_paged_kv_append(sh, q, k, v, pos, seq, table, None, False, q_out, K, V, st)
    torch.cuda.synchronize()
    assert int(st.item()) == B.DEV_BAD_INDEX
    K0[0, :, 3], V0[0, :, 3] = k[3], v[3]
    assert torch.equal(K, K0) and torch.equal(V, V0)
    assert torch.equal(q_out[3], q[3]) and (q_out[[0, 1, 2, 4, 5]] == 7).all()


# ---- attention -----------------------------------------------------------------------------------------------------

def attend(sh, q, K, V, table, lens, scale, keep=None, want_lse=True, stream=None):
    n, H = q.shape[:2]
    t = q.dtype
    out = torch.full((n, H, sh.head_dim), float("nan"), dtype=t, device=DEV)
    lse = torch.full((n, H), float("nan"), dtype=torch.float32, device=DEV) if want_lse else None
    ws = torch.full((max(B.halo_paged_mha_workspace_bytes(sh, n), 16),), 255, dtype=torch.uint8, device=DEV)
    st = status()
    B.halo_paged_mha(sh, q, K, V, table, lens, scale, out, ws, keep, lse, st, stream)
    torch.cuda.synchronize()
    return out, lse, int(st.item())


def check_attention(q, K, V, table, lens, scale, out, lse, keep, u, bad):
    ref, ref_lse, size, reach, ref_bad = A.paged_mha(host(q), host(K), host(V), table.cpu().numpy(), lens.cpu().numpy(),
                                                     scale, None if keep is None else keep.cpu().numpy())
    dh = q.shape[2]
    e = (2.0 ** -21 + dh * 2.0 ** -24 + 2.0 ** -20) * reach
    rough = 2 * e + 1e-5 + (2.0 ** -8 if u > 1e-4 else 0.0)
    assert (np.abs(host(out) - ref) <= rough[..., None] * size + u * np.abs(ref)).all()
    if lse is not None:
        fine = np.isfinite(ref_lse)
        got = host(lse)
        assert (got[~fine] == ref_lse[~fine]).all()
        assert (np.abs(got[fine] - ref_lse[fine]) <= e[fine] + 1e-6 * (1 + np.abs(ref_lse[fine]))).all()
    assert (bad != 0) == ref_bad
    return ref


ATTENTION = [
    # dtype, H, Hk, dh, page, lengths, pool of K and V pages
    ("bf16", 1, 1, 16, 16, [1], False),
    ("bf16", 8, 8, 64, 16, [0, 1, 2, 15, 16, 17, 31], False),
    ("bf16", 32, 4, 64, 16, [700], False),
    ("bf16", 32, 4, 64, 7, [63, 64, 65, 127, 128, 129, 0, 200], True),       # pages that end inside a tile
    ("bf16", 8, 2, 80, 16, [33, 1, 0, 300], False),
    ("bf16", 5, 1, 128, 32, [1000, 3], True),
    ("bf16", 16, 1, 128, 64, [2049], False),
    ("bf16", 20, 1, 128, 16, [77, 500], False),                               # two blocks of query heads
    ("bf16", 40, 8, 128, 16, [5, 900, 64, 1, 333], False),
    ("bf16", 8, 2, 256, 16, [1, 48, 511], False),
    ("bf16", 2, 2, 160, 3, [100, 17], True),
    ("f32", 8, 8, 64, 16, [1, 0, 16, 17, 300], False),
    ("f32", 8, 2, 128, 16, [257, 4], True),
    ("f32", 6, 2, 48, 5, [64, 65, 31], False),
    ("f32", 17, 1, 256, 16, [129, 40], False),
    ("f32", 4, 4, 256, 128, [1030], False),
    ("bf16", 4, 2, 64, 48, [48, 49, 400, 0, 97], False),                      # whole runs, no power of two
    ("bf16", 2, 1, 64, 16, [i % 23 for i in range(700)], False),              # more sequences than thread blocks
    ("bf16", 32, 1, 128, 16, [130, 7], True),
    ("f32", 3, 3, 64, 16, [(i * 7) % 40 for i in range(400)], False),
    ("f32", 12, 2, 64, 24, [333, 20, 1], True),
]


@pytest.mark.parametrize("case", range(len(ATTENTION)))
def test_attention_matches_oracle(case):
    dtype, H, Hk, dh, page, lens, pool = ATTENTION[case]
    t, code, u = TYPES[dtype]
    g = gen(100 + case)
    table, n_pages = block_table(g, lens, page)
    K, V, stride = caches(g, t, n_pages, Hk, page, dh, pool)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code, stride)
    q = randn(g, (len(lens), H + 3, dh), t)[:, 2:2 + H] if dh % 8 == 0 else None      # rows inside wider rows
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    # what lies behind a length, and every page that no table names, is poison
    used = torch.zeros((n_pages, page), dtype=torch.bool, device=DEV)
    for s, length in enumerate(lens):
        for p in range(length):
            used[int(table[s, p // page]), p % page] = True
    K.copy_(torch.where(used[:, None, :, None], K, torch.full_like(K, float("nan"))))
    V.copy_(torch.where(used[:, None, :, None], V, torch.full_like(V, float("inf"))))
    for scale in (dh ** -0.5, -0.3):
        out, lse, bad = attend(sh, q, K, V, table, n, scale)
        check_attention(q, K, V, table, n, scale, out, lse, None, u, bad)
    again, lse2, _ = attend(sh, q, K, V, table, n, scale)
    assert torch.equal(again, out) and torch.equal(lse2, lse)                         # the same bits
    no_lse, _, _ = attend(sh, q, K, V, table, n, scale, want_lse=False)
    assert torch.equal(no_lse, out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_large_scores_and_lost_heads(dtype):
    """Scores of +-100 (a softmax without its maximum would overflow), then heads lost one by one and all of them."""
    t, code, u = TYPES[dtype]
    g, H, Hk, dh, page, lens = gen(7), 8, 2, 64, 16, [400, 3, 0, 90]
    table, n_pages = block_table(g, lens, page)
    K, V, _ = caches(g, t, n_pages, Hk, page, dh, False)
    q = randn(g, (len(lens), H, dh), t) * 4
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code)
    for keep in (None, [1, 0, 1, 1, 0, 0, 0, 1], [0] * 4 + [1] * 4, [0] * 8):
        k8 = None if keep is None else torch.tensor(keep, dtype=torch.uint8, device=DEV)
        out, lse, bad = attend(sh, q, K, V, table, n, 1.0, k8)
        check_attention(q, K, V, table, n, 1.0, out, lse, k8, u, bad)
        assert bad == 0
        for h in range(H):
            if keep is not None and not keep[h]:
                assert (out[:, h] == 0).all() and (lse[:, h] == -float("inf")).all()


def test_attention_follows_the_formula_for_infinite_and_lowest_scores():
    """bf16: a key of -inf scores takes no part, keys of the type's lowest value neither fault nor count, rows of nothing but
    -inf give zeros; a NaN value at a live position shows."""
    t, code, u = TYPES["bf16"]
    g, dh, page = gen(8), 64, 16
    table, n_pages = block_table(g, [70], page)
    K, V, _ = caches(g, t, n_pages, 1, page, dh, False)
    n = torch.tensor([70], dtype=torch.int32, device=DEV)
    sh = B.paged_shape(2, 1, dh, page, n_pages, table.shape[1], code)
    q = torch.rand((1, 2, dh), device=DEV, generator=g).to(t) + 0.5
    first = int(table[0, 0])
    K[first, 0, 3], K[first, 0, 5] = -float("inf"), torch.finfo(t).min
    out, lse, bad = attend(sh, q, K, V, table, n, 0.125)
    Kz = K.clone()
    Kz[first, 0, 3] = -1e30                                          # weight zero in the oracle too
    check_attention(q, Kz, V, table, n, 0.125, out, lse, None, u, bad)
    out, lse, _ = attend(sh, q, torch.full_like(K, -float("inf")), V, table, n, 0.125)
    assert (out == 0).all() and (lse == -float("inf")).all()
    V[first, 0, 4, 7] = float("nan")
    out, _, _ = attend(sh, q, Kz, V, table, n, 0.125)
    assert torch.isnan(out[..., 7]).all() and torch.isfinite(out[..., :7]).all() and torch.isfinite(out[..., 8:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_flags_bad_lengths_and_pages(dtype):
    t, code, u = TYPES[dtype]
    g, H, dh, page = gen(9), 4, 64, 16
    table, n_pages = block_table(g, [100, 64, 64, 64, 90], page)
    K, V, _ = caches(g, t, n_pages, 2, page, dh, False)
    sh = B.paged_shape(H, 2, dh, page, n_pages, table.shape[1], code)
    q = randn(g, (5, H, dh), t)
    ok = torch.tensor([100, 64, 64, 64, 90], dtype=torch.int32, device=DEV)
    for lens, spoil in (([100, -1, 64, 113, 90], []), ([100, 64, 64, 64, 90], [(0, 2, n_pages), (4, 0, -5), (4, 5, 1 << 30)]),
                        ([16, 64, 64, 64, 90], [(1, 0, -1), (1, 1, -1), (1, 2, -1), (1, 3, -1)])):
        tb, n = table.clone(), torch.tensor(lens, dtype=torch.int32, device=DEV)
        for s, c, page_id in spoil:
            tb[s, c] = page_id
        out, lse, bad = attend(sh, q, K, V, tb, n, 0.125)
        assert bad == B.DEV_BAD_INDEX
        check_attention(q, K, V, tb, n, 0.125, out, lse, None, u, bad)
    out, _, bad = attend(sh, q, K, V, table, ok, 0.125)
    assert bad == 0


@pytest.mark.parametrize("dtype,H,Hk,dh,page,lens", [
    ("bf16", 32, 8, 128, 16, [20000]), ("bf16", 8, 1, 64, 64, [30001, 5, 0, 12345]), ("f32", 4, 2, 64, 16, [9001, 1, 3000]),
    ("bf16", 16, 2, 256, 32, [7777, 64])])
def test_attention_split_over_long_caches(dtype, H, Hk, dh, page, lens):
    """Long axes cut over thread blocks and joined, against fp64 torch on the same tensors; the same bits every time."""
    t, code, u = TYPES[dtype]
    g = gen(11)
    table, n_pages = block_table(g, lens, page)
    K, V, stride = caches(g, t, n_pages, Hk, page, dh, True)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code, stride)
    q = randn(g, (len(lens), H, dh), t) * 2
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    out, lse, bad = attend(sh, q, K, V, table, n, dh ** -0.5)
    assert bad == 0
    for s, length in enumerate(lens):
        if length == 0:
            assert (out[s] == 0).all() and (lse[s] == -float("inf")).all()
            continue
        pages = table[s, : -(-length // page)].long()
        k = K[pages].transpose(0, 1).reshape(Hk, -1, dh)[:, :length].double().repeat_interleave(H // Hk, 0)
        v = V[pages].transpose(0, 1).reshape(Hk, -1, dh)[:, :length].double().repeat_interleave(H // Hk, 0)
        score = torch.einsum("hd,hpd->hp", q[s].double(), k) * dh ** -0.5
        reach = (torch.einsum("hd,hpd->hp", q[s].double().abs(), k.abs()) * dh ** -0.5).amax(-1, keepdim=True)
        w = torch.softmax(score, -1)
        ref, size = torch.einsum("hp,hpd->hd", w, v), torch.einsum("hp,hpd->hd", w, v.abs())
        e = (2.0 ** -21 + dh * 2.0 ** -24 + 2.0 ** -20) * reach
        rough = 2 * e + 1e-5 + (2.0 ** -8 if dtype == "bf16" else 0.0)
        assert ((out[s].double() - ref).abs() <= rough * size + u * ref.abs()).all()
        want = torch.logsumexp(score, -1)
        assert ((lse[s].double() - want).abs() <= e[:, 0] + 1e-6 * (1 + want.abs())).all()
    for _ in range(3):
        again, lse2, _ = attend(sh, q, K, V, table, n, dh ** -0.5)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


def test_attention_and_append_beyond_32_bit_offsets():
    """Pages whose first element lies past 2^32 elements (8.6 GB) of the pool, K and V side by side."""
    t, code, u = TYPES["bf16"]
    g, H, Hk, dh, page = gen(12), 4, 2, 128, 16
    stride = 1 << 29
    pool = torch.empty(9 * stride + 2 * Hk * page * dh, dtype=t, device=DEV)
    K = pool.as_strided((10, Hk, page, dh), (stride, page * dh, dh, 1))
    V = pool.as_strided((10, Hk, page, dh), (stride, page * dh, dh, 1), Hk * page * dh)
    for p in range(10):
        K[p], V[p] = randn(g, (Hk, page, dh), t), randn(g, (Hk, page, dh), t)
    table = torch.tensor([[9, 0, 8], [7, 9, 1]], dtype=torch.int32, device=DEV)
    sh = B.paged_shape(H, Hk, dh, page, 10, 3, code, stride)
    k, v, pos = randn(g, (2, Hk, dh), t), randn(g, (2, Hk, dh), t), torch.tensor([40, 5], dtype=torch.int32, device=DEV)
    st = status()
    B.halo_paged_kv_append(sh, None, k, v, pos, None, table, None, False, None, K, V, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0
    assert torch.equal(K[8, :, 8], k[0]) and torch.equal(V[8, :, 8], v[0]) and torch.equal(K[7, :, 5], k[1])
    q, n = randn(g, (2, H, dh), t), torch.tensor([41, 30], dtype=torch.int32, device=DEV)
    out, lse, bad = attend(sh, q, K, V, table, n, dh ** -0.5)
    small_K, small_V = torch.stack([K[p] for p in range(10)]), torch.stack([V[p] for p in range(10)])
    check_attention(q, small_K, small_V, table, n, dh ** -0.5, out, lse, None, u, bad)


def test_attention_captured_into_a_graph_and_on_another_stream():
    """One captured append + attention replayed for new tokens and lengths; the lengths are read on the device."""
    t, code, u = TYPES["bf16"]
    g, H, Hk, dh, page, n = gen(13), 8, 2, 64, 16, 3
    table, n_pages = block_table(g, [400, 400, 400], page)
    K, V, _ = caches(g, t, n_pages, Hk, page, dh, False)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code)
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    qkv = randn(g, (n, H + 2 * Hk, dh), t)
    q_out, out = torch.empty((n, H, dh), dtype=t, device=DEV), torch.empty((n, H, dh), dtype=t, device=DEV)
    pos, lens = torch.zeros(n, dtype=torch.int32, device=DEV), torch.ones(n, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(B.halo_paged_mha_workspace_bytes(sh, n), 16), dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()

    def step(stream=None):
        B.halo_paged_kv_append(sh, qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], pos, None, table, inv, False, q_out, K, V,
                               stream=stream)
        B.halo_paged_mha(sh, q_out, K, V, table, lens, 0.125, out, ws, stream=stream)

    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for places in ([3, 0, 399], [150, 17, 31], [64, 63, 62]):
        qkv.copy_(randn(g, qkv.shape, t))
        pos.copy_(torch.tensor(places, dtype=torch.int32))
        lens.copy_(pos + 1)
        graph.replay()
        torch.cuda.synchronize()
        replayed, K1 = out.clone(), K.clone()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        assert torch.equal(out, replayed) and torch.equal(K, K1)
        check_attention(q_out, K, V, table, lens, 0.125, out, None, None, u, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_on_two_streams_at_once_and_for_single_rows(dtype):
    """Two calls that overlap, each with its own workspace and outputs; then rows cut out of wider tensors, one at a time."""
    t, code, u = TYPES[dtype]
    g, H, Hk, dh, page, lens = gen(17), 8, 2, 64, 16, [3000, 12, 700]
    table, n_pages = block_table(g, lens, page)
    K, V, _ = caches(g, t, n_pages, Hk, page, dh, False)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code)
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    qs = [randn(g, (3, H, dh), t) for _ in range(2)]
    alone = [attend(sh, q, K, V, table, n, 0.125)[0] for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    outs = [torch.empty_like(q) for q in qs]
    ws = [torch.empty(B.halo_paged_mha_workspace_bytes(sh, 3) + 16, dtype=torch.uint8, device=DEV) for _ in qs]
    torch.cuda.synchronize()
    for _ in range(20):
        for q, o, w, st in zip(qs, outs, ws, streams):
            B.halo_paged_mha(sh, q, K, V, table, n, 0.125, o, w, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])
    wide = torch.zeros((1, H * dh + 5), dtype=t, device=DEV)
    wide[0, : H * dh] = qs[0][2].flatten()
    out = torch.empty((1, H, dh), dtype=t, device=DEV)
    B.halo_paged_mha(sh, wide[:, : H * dh], K, V, table[2:], n[2:], 0.125, out, ws[0])
    torch.cuda.synchronize()
    assert float((out - alone[0][2]).abs().max()) <= 2e-2


def test_the_largest_number_of_sequences():
    t, code, u = TYPES["bf16"]
    g, n_seq, page, dh = gen(18), 8192, 16, 16
    K, V, _ = caches(g, t, 64, 1, page, dh, False)
    table = torch.randint(0, 64, (n_seq, 2), dtype=torch.int32, device=DEV, generator=g)
    lens = torch.randint(0, 33, (n_seq,), dtype=torch.int32, device=DEV, generator=g)
    sh = B.paged_shape(1, 1, dh, page, 64, 2, code)
    q = randn(g, (n_seq, 1, dh), t)
    out, lse, bad = attend(sh, q, K, V, table, lens, 0.25)
    assert bad == 0
    k = K[table.long()].reshape(n_seq, 2 * page, dh).double()
    v = V[table.long()].reshape(n_seq, 2 * page, dh).double()
    there = torch.arange(2 * page, device=DEV)[None] < lens[:, None]
    score = torch.einsum("nd,npd->np", q[:, 0].double(), k) * 0.25
    w = torch.softmax(score.masked_fill(~there, -1e30), -1) * (lens > 0)[:, None]
    ref, size = torch.einsum("np,npd->nd", w, v), torch.einsum("np,npd->nd", w, v.abs())
    assert ((out[:, 0].double() - ref).abs() <= (2.0 ** -8 + 1e-4) * size + u * ref.abs()).all()
    assert torch.equal(torch.isinf(lse[:, 0]), lens == 0)


# ---- the residual between blocks ------------------------------------------------------------------------------------

GLUE = [(ty, tx, n, d, post, gate, pre)
        for (ty, tx) in (("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"))
        for (n, d, post, gate, pre) in ((1, 8, True, "full", True), (3, 4096, True, "row", True), (130, 264, False, "full", False),
                                        (5, 512, True, None, False), (7, 5120, False, None, True), (2, 16384, True, "wide", True),
                                        (33, 2048, False, "row", True), (9, 128, True, "wide", False), (37, 64, True, "full", True), (21, 40, True, "row", True),
                                        (13, 120, True, "wide", True), (1, 16, False, None, True))]


@pytest.mark.parametrize("case", range(len(GLUE)))
def test_norm_glue_matches_oracle(case):
    ty, tx, n, d, post, gate, pre = GLUE[case]
    yt, ycode, _ = TYPES[ty]
    xt, xcode, u = TYPES[tx]
    g = gen(300 + case)
    h, y = randn(g, (n, d), torch.float32) * 5, randn(g, (n, d), yt)
    w_post = randn(g, (d,), xt) if post else None
    w_pre = randn(g, (d,), xt) if pre else None
    gt = {None: lambda: None, "row": lambda: randn(g, (d,), xt), "full": lambda: randn(g, (n, d), xt),
          "wide": lambda: randn(g, (n, d + 64), xt)[:, 32:32 + d]}[gate]()
    if n > 3:
        y[1], h[2] = 0, 0
    eps, res = 1e-5, 0.37
    ref_h, ref_x = A.norm_glue(host(h), host(y), host(w_post), host(gt), res, host(w_pre), eps)
    add = np.abs(ref_h - host(h))
    sh = B.norm_shape(d, eps, ycode, xcode)
    h_out, x_out = torch.empty_like(h), torch.empty((n, d), dtype=xt, device=DEV)
    B.halo_norm_glue(sh, h, y, w_post, gt, res, w_pre, h_out, x_out)
    torch.cuda.synchronize()
    off = 2.0 ** -18 * add + 2.0 ** -23 * np.abs(ref_h) + 1e-30
    assert (np.abs(host(h_out) - ref_h) <= off).all()
    root = np.sqrt(np.mean(ref_h ** 2, axis=-1, keepdims=True) + eps)
    gain = 1.0 if w_pre is None else np.abs(host(w_pre))
    row = np.sqrt(np.sum(off ** 2, axis=-1, keepdims=True)) / np.sqrt(np.sum(ref_h ** 2, axis=-1, keepdims=True) + 1e-30)
    assert (np.abs(host(x_out) - ref_x) <= off / root * gain + (2.0 ** -18 + row + u) * np.abs(ref_x) + 1e-30).all()
    keep = h.clone()
    x2 = torch.empty_like(x_out)
    B.halo_norm_glue(sh, keep, y, w_post, gt, res, w_pre, keep, x2)                # in place, the same bits
    torch.cuda.synchronize()
    assert torch.equal(keep, h_out) and torch.equal(x2, x_out)
    B.halo_norm_glue(sh, h, None, None, None, res, w_pre, h_out, x_out)            # no block in front
    torch.cuda.synchronize()
    assert torch.equal(h_out, h)


def test_norm_glue_without_gains_is_halo_glue():
    """Where both exist they agree within rounding: no norm behind the block, no gains, no gate, scale 1, its epsilon."""
    g, n, d = gen(5), 6, 4096
    h, y = randn(g, (n, d), torch.float32), randn(g, (n, d), torch.float32)
    outs = [(torch.empty_like(h), torch.empty((n, d), dtype=torch.bfloat16, device=DEV)) for _ in range(2)]
    B.halo_norm_glue(B.norm_shape(d, 1e-5, B.F32, B.BF16), h, y, None, None, 1.0, None, *outs[0])
    B.halo_glue(d, n, B.BF16, h, y, *outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0])
    assert ((outs[0][1].float() - outs[1][1].float()).abs() <= 2.0 ** -7 * outs[1][1].float().abs()).all()


# ---- together -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("d,H,Hk,dh,lens", [(512, 8, 2, 64, [1, 40, 77]), (2048, 32, 4, 64, [300, 5, 0, 129, 64])])
def test_attention_block_of_a_token_step(d, H, Hk, dh, lens):
    """norm -> 4-bit q/k/v projection -> append with rotation -> attention of the heads that a selection kept -> 4-bit output
    projection -> gated residual and norm, each step against the oracle on what the GPU fed it.  Sequence 2 / 2 of the batch
    is a padding row (position -1, length 0)."""
    t, code, u = TYPES["bf16"]
    g, page, n = gen(d), 16, len(lens)
    lens = [max(x, 1) if i != 2 else 0 for i, x in enumerate(lens)]
    table, n_pages = block_table(g, lens, page)
    K, V, _ = caches(g, t, n_pages, Hk, page, dh, False)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], code)
    norm, glue = B.norm_shape(d, 1e-5, B.F32, B.BF16), B.norm_shape(d, 1e-5, B.BF16, B.BF16)
    rows = (H + 2 * Hk) * dh

    def packed(W):
        Q = torch.empty((W.shape[0], W.shape[1] // 2), dtype=torch.uint8, device=DEV)
        S = torch.empty(B.halo_mx4_scale_bytes(W.shape[1], W.shape[0]), dtype=torch.uint8, device=DEV)
        B.halo_quantize_rows_mx4(W.shape[1], W.shape[0], code, W, Q, S)
        return Q, S

    def project(x, W):
        Qx, Sx = packed(x)
        y, st = torch.empty((n, W[0].shape[0]), dtype=t, device=DEV), status()
        B.halo_product_mx4(x.shape[1], n, W[0].shape[0], Qx, Sx, *W, code, y, st)
        xv, wv = (A.mx4_unpack(q.cpu().numpy(), s.cpu().numpy(), q.shape[0], q.shape[1] * 2) for q, s in ((Qx, Sx), W))
        ref, size = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
        assert (np.abs(host(y) - ref) <= (x.shape[1] / 64 + 64) * 2.0 ** -23 * size + u * np.abs(ref)).all()
        assert int(st.item()) == 0
        return y

    Wqkv, Wo = packed(randn(g, (rows, d), t) * 0.05), packed(randn(g, (d, H * dh), t) * 0.05)
    w_in, w_post, w_next, gate = (torch.rand(d, device=DEV, generator=g).to(t) for _ in range(4))
    h = randn(g, (n, d), torch.float32)
    x = torch.empty((n, d), dtype=t, device=DEV)
    B.halo_norm_glue(norm, h, None, None, None, 1.0, w_in, h, x)
    qkv = project(x, Wqkv).view(n, H + 2 * Hk, dh)
    pos = torch.tensor([v - 1 for v in lens], dtype=torch.int32, device=DEV)
    n32 = torch.tensor(lens, dtype=torch.int32, device=DEV)
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    q_out = torch.zeros((n, H, dh), dtype=t, device=DEV)
    st = status()
    want = A.paged_append(host(qkv[:, :H]), host(qkv[:, H:H + Hk]), host(qkv[:, H + Hk:]), np.array([v - 1 for v in lens]), None,
                          table.cpu().numpy(), host(inv), False, host(q_out), host(K), host(V))
    B.halo_paged_kv_append(sh, qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], pos, None, table, inv, False, q_out, K, V, st)
    for got, ref in zip((q_out, K, V), want):
        assert (np.abs(host(got) - ref) <= 6e-7 * 2 * float(qkv.abs().max()) + u * np.abs(ref)).all()
    # heads are the neuron groups of an attention block: a selection decides which of them arrive
    plan = B.Plan(H, [0.3, 0.6], [1, 1], B.SEL_TOPK, H // 4, 0.0, 5)
    keep, kl, nk = (torch.zeros(k, dtype=dt, device=DEV) for k, dt in ((H, torch.uint8), (H, torch.int32), (1, torch.int32)))
    scores = torch.randn(H, generator=g, device=DEV)
    B.halo_select_groups(plan, scores, 1, 3, False, None, None, None, keep, kl, nk)
    torch.cuda.synchronize()
    assert 0 < int(keep.sum()) < H
    out, lse, bad = attend(sh, q_out, K, V, table, n32, dh ** -0.5, keep)
    check_attention(q_out, K, V, table, n32, dh ** -0.5, out, lse, keep, u, bad)
    assert bad == 0 and int(st.item()) == 0
    y = project(out.view(n, H * dh), Wo)
    assert (y[2] == 0).all()                                              # nothing attended, nothing projected
    ref_h, ref_x = A.norm_glue(host(h), host(y), host(w_post), host(gate), 0.5, host(w_next), 1e-5)
    h_before = host(h)
    B.halo_norm_glue(glue, h, y, w_post, gate, 0.5, w_next, h, x)
    torch.cuda.synchronize()
    assert (np.abs(host(h) - ref_h) <= 2.0 ** -18 * np.abs(ref_h - h_before) + 2.0 ** -23 * np.abs(ref_h)).all()
    assert np.abs(host(x) - ref_x).max() <= 2.0 ** -7 * np.abs(ref_x).max()


def test_paged_attention_agrees_with_group_mha_on_a_dense_cache():
    """A dense cache of halo_group_mha is a paged cache of one page; with the queries of its heads both give the same sum over
    heads of o_h Wo_h."""
    from paper_2601_11676_b200 import synth
    d, H, dh, L, pos = 512, 8, 64, 300, 270
    wl = synth.Workload("a", 1, d, 64, 16, 32, "bf16", (0.0,), (1,), 500, 1)
    Wq, _, _, Wo = synth.mha_matrices(wl, 0, H, DEV)
    g, t = gen(21), torch.bfloat16
    K, V = randn(g, (H, L, dh), t), randn(g, (H, L, dh), t)
    mh = B.mha_shape(d, H, dh, L, B.BF16)
    Wp = torch.empty((H, 2, dh, d), dtype=t, device=DEV)
    B.halo_pack_mha_weights(mh, Wq, Wo, Wp)
    x = randn(g, (1, d), t)
    P = torch.empty((1, d), dtype=torch.float32, device=DEV)
    ws = torch.empty(B.halo_group_mha_workspace_bytes(mh), dtype=torch.uint8, device=DEV)
    kl, nk = torch.arange(H, dtype=torch.int32, device=DEV), torch.tensor([H], dtype=torch.int32, device=DEV)
    B.halo_group_mha(mh, Wp, x, K, V, pos, kl, nk, None, 0, P, ws)
    q = (x.double() @ Wq.double().t()).to(t).view(1, H, dh)
    sh = B.paged_shape(H, H, dh, L, 1, 1, B.BF16)
    table, n = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.tensor([pos + 1], dtype=torch.int32, device=DEV)
    out, _, bad = attend(sh, q, K[None], V[None], table, n, dh ** -0.5)
    y = out.view(1, H * dh).double() @ Wo.double().t()
    assert bad == 0 and float((y - P.double()).abs().max()) <= 2e-2 * float(P.double().square().mean().sqrt())


@pytest.mark.parametrize("form", ["bf16", "i4"])
@pytest.mark.parametrize("kept", ["all", "none", "bad"])
def test_calls_behind_a_group_ffn_see_its_result_and_what_ran_before_it(form, kept):
    """norm_glue -> group FFN -> norm_glue on the partial slot, back to back without a wait, over and over in one buffer: a
    later call that started before an earlier one had ended would read the values of another turn.  The FFN kernels
    overlap with their neighbours on purpose, and with no (or no valid) group in the list they have nothing to wait for."""
    d, F, S, turns = 2048, 1024, 64, 40
    G, t = F // S, torch.bfloat16
    g = gen(31)
    sh = B.ffn_shape(d, F, S, B.BF16)
    W = randn(g, (G, 3, S, d), t) * 0.02
    Q, sc = torch.empty((G, 3, S, d // 2), dtype=torch.uint8, device=DEV), torch.empty((G, 3, S, d // 128), dtype=t, device=DEV)
    B.halo_quantize_weights_i4(sh, W, Q, sc)
    kl = torch.arange(G, dtype=torch.int32, device=DEV) + (1000 if kept == "bad" else 0)
    nk = torch.tensor([0 if kept == "none" else G], dtype=torch.int32, device=DEV)
    norm = B.norm_shape(d, 1e-5, B.F32, B.BF16)
    w = torch.rand((turns, d), device=DEV, generator=g).to(t)
    h0 = randn(g, (1, d), torch.float32)

    def run(wait):
        h, x, P = h0.clone(), torch.zeros((1, d), dtype=t, device=DEV), torch.full((1, 1, d), 1e30, device=DEV)
        st, seen = status(), torch.empty((turns, 2, d), dtype=t, device=DEV)
        for i in range(turns):
            B.halo_norm_glue(norm, h, None, None, None, 1.0, w[i], h, x)
            if wait:
                torch.cuda.synchronize()
            if form == "bf16":
                B.halo_group_ffn(sh, W, x, 1, kl, nk, None, 0, P, None, st)
            else:
                B.halo_group_ffn_i4(sh, Q, sc, x, 1, kl, nk, None, 0, P, st)
            if wait:
                torch.cuda.synchronize()
            B.halo_norm_glue(norm, h, P, None, None, 1.0, w[i], h, seen[i, 0:1])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return h, seen[:, 0].float(), int(st.item())

    h1, seen1, st1 = run(True)
    h2, seen2, st2 = run(False)
    assert st1 == st2 == (B.DEV_BAD_INDEX if kept == "bad" else 0)
    if kept != "all":
        assert torch.equal(h1, h0) and torch.equal(h2, h0) and torch.equal(seen1, seen2)
    else:   # atomic sums: the order of additions differs between runs
        assert float((h1 - h2).abs().max()) <= 1e-3 * float(h1.abs().max())
        assert float((seen1 - seen2).abs().max()) <= 0.02 * float(seen1.abs().max())
