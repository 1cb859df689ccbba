"""halo_paged_mha where sums are joined and where weights count: the fp64 oracle's definition with the bounds below.

S = the weighted mean of |V|, e as in test_gpu_attention_block (scores' error), u = half a rounding step of the output
(2^-8 bf16, 2^-24 fp32, relative).  A weight is off by 2 e relative, its fp32 sum by 1e-5; bf16: it meets the values as its upper
bits and their rest, which is below 2^-7 of it and rounded to 2^-8 of itself: 2^-15.  out: (2 e + 1e-5 + [2^-15]) S + u |out|.
"""
import numpy as np
import pytest
import torch

from oracle import attention_block_ref as A
from paper_2601_11676_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, B.BF16, 2.0 ** -8), "f32": (torch.float32, B.F32, 2.0 ** -24)}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, shape, t):
    return torch.randn(shape, generator=g, device=DEV).to(t)


def block_table(g, lens, page, cols=None):
    """Pages in a shuffled order; entries behind a sequence's last page name none."""
    need = [-(-n // page) for n in lens]
    order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32).cpu()
    table = torch.full((len(lens), cols or max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table.to(DEV), sum(need) + 2


def attend(sh, q, K, V, table, lens, scale, keep=None, ws=None):
    n, H = q.shape[:2]
    out = torch.full((n, H, sh.head_dim), float("nan"), dtype=q.dtype, device=DEV)
    lse = torch.full((n, H), float("nan"), dtype=torch.float32, device=DEV)
    if ws is None:
        ws = torch.full((max(B.halo_paged_mha_workspace_bytes(sh, n), 16),), 255, dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.halo_paged_mha(sh, q, K, V, table, lens, scale, out, ws, keep, lse, st)
    torch.cuda.synchronize()
    return out, lse, int(st.item())


def expected(q, K, V, table, lens, scale, keep=None):
    """The oracle's five results, in fp64 on the device, a sequence at a time."""
    n, H, dh = q.shape
    Hk, page, cap = K.shape[1], K.shape[2], table.shape[1] * K.shape[2]
    out, size = (torch.zeros((n, H, dh), dtype=torch.float64, device=DEV) for _ in range(2))
    lse = torch.full((n, H), -float("inf"), dtype=torch.float64, device=DEV)
    reach, bad = torch.zeros((n, H), dtype=torch.float64, device=DEV), False
    kept = torch.ones(H, dtype=torch.bool, device=DEV) if keep is None else keep != 0
    for s, length in enumerate(lens.tolist()):
        if length < 0 or length > cap:
            bad, length = True, 0
        p = torch.arange(length, device=DEV)
        pages = table[s].long()[p // page]
        there = (pages >= 0) & (pages < K.shape[0])
        bad |= bool(kept.any()) and not bool(there.all())
        pages, rows = pages[there], (p % page)[there]
        if len(pages) == 0:
            continue
        k, v = (c[pages, :, rows].double().transpose(0, 1).repeat_interleave(H // Hk, 0) for c in (K, V))   # [H][positions][dh]
        qs = q[s].double()[:, :, None]
        score = (k @ qs)[..., 0] * scale
        w = torch.softmax(score, -1)[:, None]
        out[s], size[s] = (w @ v)[:, 0], (w @ v.abs())[:, 0]
        lse[s], reach[s] = torch.logsumexp(score, -1), (k.abs() @ qs.abs())[..., 0].amax(-1) * abs(scale)
    out[:, ~kept], size[:, ~kept], lse[:, ~kept] = 0, 0, -float("inf")
    return out, lse, size, reach, bad


def check(dtype, q, K, V, table, lens, scale, keep=None, ws=None):
    u = TYPES[dtype][2]
    out, lse, bad = attend(B.paged_shape(q.shape[1], K.shape[1], K.shape[3], K.shape[2], K.shape[0], table.shape[1], TYPES[dtype][1]),
                           q, K, V, table, lens, scale, keep, ws)
    ref, ref_lse, size, reach, ref_bad = expected(q, K, V, table, lens, scale, keep)
    e = (2.0 ** -21 + q.shape[2] * 2.0 ** -24 + 2.0 ** -20) * reach
    rough = 2 * e + 1e-5 + (2.0 ** -15 if dtype == "bf16" else 0.0)
    assert ((out.double() - ref).abs() <= rough[..., None] * size + u * ref.abs()).all()
    fine = torch.isfinite(ref_lse)
    assert torch.equal(lse[~fine].double(), ref_lse[~fine])
    assert ((lse.double() - ref_lse).abs()[fine] <= (e + 1e-6 * (1 + ref_lse.abs()))[fine]).all()
    assert (bad != 0) == ref_bad
    return out, lse


@pytest.mark.parametrize("H,Hk,dh,lens", [(32, 4, 64, [700]), (8, 8, 64, [20, 1, 0, 33]), (32, 8, 128, [9, 40, 300]), (16, 1, 128, [50, 2049]),
                                          (20, 1, 80, [24, 77]), (8, 2, 256, [31, 5]), (12, 1, 256, [18, 200]), (8, 2, 128, [30000])])
def test_bf16_weights_are_not_what_the_output_is_off_by(H, Hk, dh, lens):
    """Elements that the values nearly cancel show the weights' own error: it stays far below the output's rounding."""
    t, g, page = torch.bfloat16, gen(H + dh), 16
    table, n_pages = block_table(g, lens, page)
    K, V = (randn(g, (n_pages, Hk, page, dh), t) for _ in range(2))
    n = torch.tensor(lens, dtype=torch.int32, device=DEV)
    check("bf16", randn(g, (len(lens), H, dh), t), K, V, table, n, dh ** -0.5)


@pytest.mark.parametrize("H,Hk", [(8, 2), (16, 1)])
def test_bf16_values_of_infinity_show_whatever_their_weight_is(H, Hk):
    """Weights that one bf16 number holds (1, 0.5, 2^-100) and others, each on a value of infinity: infinity, never NaN."""
    t, g, dh, page = torch.bfloat16, gen(1), 64, 16
    table, n_pages = block_table(g, [64], page)
    n = torch.tensor([64], dtype=torch.int32, device=DEV)
    K = torch.zeros((n_pages, Hk, page, dh), dtype=t, device=DEV)
    q = torch.zeros((1, H, dh), dtype=t, device=DEV)
    q[..., 0] = 1.0
    scores = torch.tensor([0.0, -1.0, -100.0, -0.3125, -17.5, -120.0, -125.0], device=DEV).to(t)     # powers of two
    for i in range(len(scores)):
        K[table[0].long(), :, :, 0] = -3.0
        K[table[0, 0].long(), :, : len(scores), 0] = scores[:, None].T.expand(Hk, -1)
        V = randn(g, (n_pages, Hk, page, dh), t)
        V[table[0, 0].long(), :, i, 5], V[table[0, 0].long(), :, i, 6] = float("inf"), -float("inf")
        out, _, bad = attend(B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], B.BF16), q, K, V, table, n, float(np.log(2.0)))
        assert bad == 0 and (out[..., 5] == float("inf")).all() and (out[..., 6] == -float("inf")).all()
        rest = torch.ones(dh, dtype=torch.bool)
        rest[5:7] = False
        assert torch.isfinite(out[..., rest]).all()


def test_the_bound_itself_follows_the_oracle():
    """`expected` above is the oracle's definition, vectorised: the same numbers on a small case."""
    t, g, H, Hk, dh, page, lens = torch.float32, gen(2), 6, 2, 16, 5, [0, 1, 12, 40, -1]
    table, n_pages = block_table(g, [0, 1, 12, 20, 5], page)
    table[2, 1] = n_pages
    K, V, q = randn(g, (n_pages, Hk, page, dh), t), randn(g, (n_pages, Hk, page, dh), t), randn(g, (5, H, dh), t)
    n, keep = torch.tensor(lens, dtype=torch.int32, device=DEV), torch.tensor([1, 0, 1, 1, 1, 0], dtype=torch.uint8, device=DEV)
    got = expected(q, K, V, table, n, 0.25, keep)
    want = A.paged_mha(*(x.double().cpu().numpy() for x in (q, K, V)), table.cpu().numpy(), np.array(lens), 0.25, keep.cpu().numpy())
    for i in (0, 1, 2):
        assert np.allclose(got[i].cpu().numpy(), want[i], rtol=1e-12, atol=1e-14)
    kept = keep.cpu().numpy() != 0
    assert np.allclose(got[3].cpu().numpy()[:, kept], want[3][:, kept], rtol=1e-12) and got[4] == want[4]


# ---- the line: items cut over thread blocks and joined --------------------------------------------------------------

def line_case(dtype, H, Hk, dh, page, lens, seed, cols=None):
    t, g = TYPES[dtype][0], gen(seed)
    table, n_pages = block_table(g, lens, page, cols)
    K, V = (randn(g, (n_pages, Hk, page, dh), t) for _ in range(2))
    q, n = randn(g, (len(lens), H, dh), t), torch.tensor(lens, dtype=torch.int32, device=DEV)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], TYPES[dtype][1])
    assert B.halo_paged_mha_workspace_bytes(sh, len(lens)) > 0      # no clusters: what is tested here is the line
    return sh, q, K, V, table, n


@pytest.mark.parametrize("dtype,lens", [("bf16", [20000]), ("bf16", [i * 31 % 3000 for i in range(100)]), ("f32", [9001, 3000])])
def test_a_workspace_is_aligned_to_16_bytes_and_no_more(dtype, lens):
    sh, q, K, V, table, n = line_case(dtype, 8, 2, 64, 16, lens, 3)
    need = B.halo_paged_mha_workspace_bytes(sh, len(lens))
    out, lse = check(dtype, q, K, V, table, n, 0.125)
    for offset in (16, 48):
        pool = torch.full((need + 128,), 255, dtype=torch.uint8, device=DEV)
        at = -pool.data_ptr() % 64 + offset
        ws = pool[at:at + need]
        assert ws.data_ptr() % 32 == 16
        again, lse2, _ = attend(sh, q, K, V, table, n, 0.125, ws=ws)
        assert torch.equal(again, out) and torch.equal(lse2, lse)
        assert (pool[:at] == 255).all() and (pool[at + need:] == 255).all()


# Many items of a few pieces each (the join by range) and few of many (by item); several blocks of query heads, pages that end
# inside a run, heads that are not as wide as their tiles, empty sequences between long ones.
LINE = [
    # dtype, H, Hk, dh, page, lengths
    ("bf16", 32, 8, 128, 16, [(i * 613) % 1500 for i in range(64)]),
    ("f32", 8, 1, 128, 16, [(i * 211) % 900 for i in range(40)]),
    ("bf16", 20, 1, 80, 7, [(i * 613) % 1500 for i in range(60)]),
    ("bf16", 8, 2, 256, 16, [(i * 389) % 900 for i in range(64)]),
    ("f32", 6, 2, 48, 5, [(i * 389) % 900 for i in range(80)]),
    ("f32", 17, 1, 256, 16, [(i * 127) % 300 for i in range(60)]),
    ("bf16", 40, 2, 64, 3, [(i * 523) % 1200 for i in range(150)]),
    ("bf16", 8, 8, 128, 48, [(i * 239) % 500 for i in range(64)]),
    ("f32", 5, 5, 128, 16, [(i * 311) % 700 for i in range(120)]),
    ("bf16", 20, 1, 80, 7, [7000, 0, 2500]),
    ("f32", 10, 2, 80, 16, [6000, 1, 0]),
    ("bf16", 32, 1, 128, 16, [9000]),
]


@pytest.mark.parametrize("case", range(len(LINE)))
@pytest.mark.parametrize("spoilt", [False, True])
def test_items_cut_over_thread_blocks(case, spoilt):
    """spoilt: lost heads (a whole block of query heads among them), pages out of range, lengths out of range."""
    dtype, H, Hk, dh, page, lens = LINE[case]
    sh, q, K, V, table, n = line_case(dtype, H, Hk, dh, page, lens, 50 + case)
    assert (B.halo_paged_mha_workspace_bytes(sh, len(lens)) > 0) and max(lens) > 64
    keep = None
    if spoilt:
        block, G = 16 if dtype == "bf16" else 4, H // Hk
        keep = torch.tensor([int(h % 3 != 1 and not (G > block and h % G < block)) for h in range(H)], dtype=torch.uint8, device=DEV)
        if not bool(keep.any()):
            keep[-1] = 1
        longest = int(n.argmax())
        table[longest, (max(lens) - 1) // page // 2] = sh.n_pages      # a page of a sequence that is cut
        table[longest, 0] = -7
        if len(lens) > 4:
            n[1], n[3] = -2, sh.max_pages * page + 1
    out, lse = check(dtype, q, K, V, table, n, dh ** -0.5, keep)
    for _ in range(2):
        again, lse2, _ = attend(sh, q, K, V, table, n, dh ** -0.5, keep)
        assert torch.equal(again, out) and torch.equal(lse2, lse)


@pytest.mark.parametrize("dtype,lens", [("bf16", [(i * 613) % 1500 for i in range(64)]), ("bf16", [20000, 5]), ("f32", [(i * 211) % 900 for i in range(40)])])
def test_joined_calls_on_two_streams_at_once(dtype, lens):
    """Two calls that overlap, each with its own workspace; then one workspace for calls in a row on one stream."""
    H, Hk = (32, 8) if dtype == "bf16" else (8, 1)
    sh, q, K, V, table, n = line_case(dtype, H, Hk, 128, 16, lens, 4)
    need = B.halo_paged_mha_workspace_bytes(sh, len(lens))
    qs = [q, randn(gen(5), q.shape, q.dtype)]
    alone = [check(dtype, x, K, V, table, n, 0.09) for x in qs]
    streams, outs = [torch.cuda.Stream() for _ in qs], [torch.empty_like(q) for _ in qs]
    lses = [torch.empty(q.shape[:2], dtype=torch.float32, device=DEV) for _ in qs]
    ws = [torch.empty(need, dtype=torch.uint8, device=DEV) for _ in qs]
    torch.cuda.synchronize()
    for _ in range(30):
        for x, o, l, w, st in zip(qs, outs, lses, ws, streams):
            B.halo_paged_mha(sh, x, K, V, table, n, 0.09, o, w, lse=l, stream=st)
    torch.cuda.synchronize()
    for (a, b), o, l in zip(alone, outs, lses):
        assert torch.equal(o, a) and torch.equal(l, b)
    for _ in range(10):
        for x, o, l in zip(qs, outs, lses):
            B.halo_paged_mha(sh, x, K, V, table, n, 0.09, o, ws[0], lse=l)
    torch.cuda.synchronize()
    for (a, b), o, l in zip(alone, outs, lses):
        assert torch.equal(o, a) and torch.equal(l, b)


@pytest.mark.parametrize("n_seq,cap", [(64, 1500), (2, 20000)])
def test_append_and_joined_attention_captured_into_a_graph(n_seq, cap):
    """One captured append + attention (line and join) replayed for new tokens and lengths, as on a side stream."""
    H, Hk, dh, page, t = 32, 8, 128, 16, torch.bfloat16
    sh, q, K, V, table, n = line_case("bf16", H, Hk, dh, page, [cap] * n_seq, 6)
    ws = torch.empty(B.halo_paged_mha_workspace_bytes(sh, n_seq), dtype=torch.uint8, device=DEV)
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    g = gen(7)
    qkv = randn(g, (n_seq, H + 2 * Hk, dh), t)
    pos = n - 1
    q_out, out = torch.empty_like(q), torch.empty_like(q)
    lse = torch.empty((n_seq, H), dtype=torch.float32, device=DEV)
    side = torch.cuda.Stream()

    def step(stream=None):
        B.halo_paged_kv_append(sh, qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:], pos, None, table, inv, False, q_out, K, V,
                               stream=stream)
        B.halo_paged_mha(sh, q_out, K, V, table, n, dh ** -0.5, out, ws, lse=lse, stream=stream)

    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(3):
        qkv.copy_(randn(g, qkv.shape, t))
        pos.copy_(torch.randint(0, cap, (n_seq,), generator=g, device=DEV))
        n.copy_(pos + 1)
        graph.replay()
        torch.cuda.synchronize()
        replayed, lse1 = out.clone(), lse.clone()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        assert torch.equal(out, replayed) and torch.equal(lse, lse1)
        again, _ = check("bf16", q_out, K, V, table, n, dh ** -0.5)
        assert torch.equal(again, replayed)


def test_short_sequences_under_a_wide_table():
    """A table as wide as the longest context that a server admits; what is in use is short."""
    for dtype, lens, cols in (("bf16", [700], 8192), ("bf16", [3, 0, 17, 200], 4096), ("f32", [40, 1], 2048)):
        sh, q, K, V, table, n = line_case(dtype, 32 if dtype == "bf16" else 4, 4, 64, 16, lens, 8, cols)
        check(dtype, q, K, V, table, n, 0.125)
