"""halo_paged_prompt_mha against the definition in 64 bits, at the sizes, masks and contents where it can go wrong.

S = the weighted mean of |V|, u = half a rounding step of the output (2^-8 bf16, 2^-24 fp32, relative).  Scores are fp32 sums of dh
products times a power of two's rounding: off by e = (2^-21 + dh 2^-24 + 2^-20) times the largest sum |q||k| scale of the row, as in
test_gpu_paged_attention.  A weight is off by 2 e relative, its fp32 sum by 1e-5, and bf16 and 8-bit caches round it to bf16: 2^-8.
out: (2 e + 1e-5 + [2^-8]) S + u |out|.  lse: e + 1e-6 (1 + |lse|) + 1e-5.
"""
import numpy as np
import pytest
import torch

from oracle import paged_prompt_ref as P
from paper_2601_11676_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, shape, t):
    return torch.randn(shape, generator=g, device=DEV).to(t)


def block_table(g, lens, page, cols=None):
    """Pages in a shuffled order; entries behind a sequence's last page name none."""
    need = [-(-max(n, 0) // page) for n in lens]
    order = torch.randperm(sum(need) + 2, generator=g, device=DEV).to(torch.int32).cpu()
    table = torch.full((len(lens), cols or max(max(need), 1)), -1, dtype=torch.int32)
    at = 0
    for s, n in enumerate(need):
        table[s, :n] = order[at:at + n]
        at += n
    return table.to(DEV), sum(need) + 2


def eight(x):
    """Codes, scale bytes and their values of 8-bit rows near x: inputs, not what a quantiser is compared with."""
    up = torch.ceil(torch.log2(x.float().abs().amax(-1).clamp(min=1e-20) / 448)).int()
    codes = torch.ldexp(x.float(), -up[..., None]).clamp(-448, 448).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), (up + 127).to(torch.uint8), torch.ldexp(codes.float().double(), up[..., None])


class Case:
    """A cache of one kind ("bf16", "f32", "8bit") and what an attention call over it needs."""

    def __init__(self, kind, H, Hk, dh, page, chunks, seed=0, cols=None, rows_behind=2, spread=1.0):
        g = gen(seed + H + dh)
        self.kind, self.t = kind, F32 if kind == "f32" else BF16
        new, past = zip(*chunks)
        lens = [a + b for a, b in chunks]
        self.table, n_pages = block_table(g, lens, page, cols)
        self.lens = torch.tensor(lens, dtype=torch.int32, device=DEV)
        self.start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=DEV)
        self.q = randn(g, (sum(new) + rows_behind, H, dh), self.t) * spread
        self.scale, self.keep, self.Ks, self.Vs = dh ** -0.5, None, None, None
        K, V = (randn(g, (n_pages, Hk, page, dh), self.t) for _ in range(2))
        if kind == "8bit":
            V = V * torch.exp2(torch.randint(-6, 7, (n_pages, Hk, page, 1), generator=g, device=DEV).float()).to(self.t)
            self.K, self.Ks, self.Kv = eight(K)
            self.V, self.Vs, self.Vv = eight(V)
        else:
            self.K, self.V = K, V
            self.refresh()

    def refresh(self):
        self.Kv, self.Vv = self.K.double(), self.V.double()

    def shape(self, stride=0):
        n_pages, Hk, page, dh = self.K.shape
        return B.paged_shape(self.q.shape[1], Hk, dh, page, n_pages, self.table.shape[1], B.F32 if self.t is F32 else B.BF16, stride)

    def workspace(self, fill=255):
        return torch.full((B.halo_paged_prompt_mha_workspace_bytes(self.shape(), self.q.shape[0], len(self.lens)),), fill,
                          dtype=torch.uint8, device=DEV)

    def buffers(self):
        n, H, dh = self.q.shape
        return torch.full((n, H, dh), 7.0, dtype=self.t, device=DEV), torch.full((n, H), 7.0, dtype=F32, device=DEV)

    def call(self, out, lse, ws, status=None, stream=None):
        B.halo_paged_prompt_mha(self.shape(), self.q, self.start, self.K, self.V, self.table, self.lens, self.scale, out, ws,
                                self.Ks, self.Vs, self.keep, lse, status, stream)

    def run(self):
        out, lse = self.buffers()
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        self.call(out, lse, self.workspace(), st)
        torch.cuda.synchronize()
        return out, lse, int(st.item())

    def expected(self):
        """The oracle's results in fp64 on the device, a sequence at a time."""
        n_tok, H, dh = self.q.shape
        n_pages, Hk, page = self.K.shape[:3]
        out, size = (torch.zeros((n_tok, H, dh), dtype=torch.float64, device=DEV) for _ in range(2))
        lse, reach = torch.full((n_tok, H), -INF, dtype=torch.float64, device=DEV), torch.zeros((n_tok, H), dtype=torch.float64, device=DEV)
        mine, bad = torch.zeros(n_tok, dtype=torch.bool, device=DEV), False
        kept = torch.ones(H, dtype=torch.bool, device=DEV) if self.keep is None else self.keep != 0
        start = self.start.tolist()
        for s, length in enumerate(self.lens.tolist()):
            a, b = start[s], start[s + 1]
            if not 0 <= length <= self.table.shape[1] * page:
                bad, length = True, 0
            if not 0 <= a <= b <= n_tok:
                bad = True
                continue
            mine[a:b] = True
            if a == b or length == 0:
                continue
            p = torch.arange(length, device=DEV)
            pages = self.table[s].long()[p // page]
            there = (pages >= 0) & (pages < n_pages)
            bad |= bool(kept.any()) and not bool(there.all())
            pages, rows, p = pages[there], (p % page)[there], p[there]
            seen = p[None] <= (length - (b - a) + torch.arange(b - a, device=DEV))[:, None]       # [rows][positions]
            for h in range(Hk):
                hs = slice(h * (H // Hk), (h + 1) * (H // Hk))
                k, v = self.Kv[pages, h, rows], self.Vv[pages, h, rows]
                q = self.q[a:b, hs].double().transpose(0, 1)
                score = torch.where(seen, q @ k.t() * self.scale, -INF)
                m = score.amax(-1, keepdim=True)
                w = torch.exp(score - torch.where(m == -INF, 0.0, m))
                l = w.sum(-1, keepdim=True)
                w = w / torch.where(l == 0, 1.0, l)
                # what a row does not see has no influence: weights of zero meet nothing
                fine = torch.isfinite(v)
                o = w @ torch.where(fine, v, 0.0)
                for j in torch.nonzero(~fine.all(-1))[:, 0].tolist():
                    o = o + torch.where(seen[None, :, j, None], torch.where(fine[j], 0.0, w[:, :, j, None] * v[j]), 0.0)
                out[a:b, hs], size[a:b, hs] = o.transpose(0, 1), (w @ torch.where(fine, v, 0.0).abs()).transpose(0, 1)
                lse[a:b, hs] = (m + torch.log(l))[..., 0].t()
                counts = seen & (score > m - 100)        # the others' weights are zero, however far off their scores are
                r = torch.where(counts, q.abs() @ torch.where(torch.isfinite(k), k, 0.0).abs().t(), 0.0).amax(-1) * abs(self.scale)
                reach[a:b, hs] = r.t()
        out[:, ~kept], size[:, ~kept], lse[:, ~kept] = 0, 0, -INF
        return out, lse, size, reach, mine, bad

    def check(self):
        out, lse, bad = self.run()
        self.compare(out, lse)
        assert (bad != 0) == self.expected()[5]
        return out, lse

    def compare(self, out, lse):
        ref, ref_lse, size, reach, mine, _ = self.expected()
        assert (out[~mine] == 7).all() and (lse[~mine] == 7).all()              # rows of no sequence stay as they were
        out, lse, ref, ref_lse, size, reach = (x[mine].double() for x in (out, lse, ref, ref_lse, size, reach))
        e = (2.0 ** -21 + self.q.shape[2] * 2.0 ** -24 + 2.0 ** -20) * reach
        rough = 2 * e + 1e-5 + (0.0 if self.kind == "f32" else 2.0 ** -8)
        fine = torch.isfinite(ref)
        assert torch.equal(torch.isnan(out), torch.isnan(ref))
        assert torch.equal(out[~fine & ~torch.isnan(ref)], ref[~fine & ~torch.isnan(ref)])
        off = (out - ref).abs() - (rough[..., None] * size + (2.0 ** -24 if self.t is F32 else 2.0 ** -8) * ref.abs())
        assert (off[fine] <= 0).all(), float(off[fine].max())
        fine = torch.isfinite(ref_lse)
        assert torch.equal(lse[~fine & ~torch.isnan(ref_lse)], ref_lse[~fine & ~torch.isnan(ref_lse)])
        assert ((lse - ref_lse).abs()[fine] <= (e + 1e-5 + 1e-6 * (1 + ref_lse.abs()))[fine]).all()


KINDS = ["f32", "bf16", "8bit"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,dh,page,chunks", [
    (4, 4, 64, 16, [(1, 0)]),                                          # one token, nothing before it
    (4, 1, 64, 16, [(3, 5), (1, 0), (0, 9), (17, 1)]),                 # a sequence without new tokens
    (8, 2, 128, 16, [(128, 0)]),
    (8, 2, 128, 16, [(64, 64), (65, 63), (63, 66)]),                   # rows and tiles that end on a border, and beside it
    (32, 8, 128, 16, [(257, 130), (1, 700), (40, 0)]),
    (5, 1, 80, 48, [(100, 3), (52, 200)]),                             # five heads on one: rows of a token in two items
    (40, 8, 80, 5, [(33, 20)]),                                        # pages that end inside everything
    (2, 2, 16, 1, [(9, 30)]),
    (4, 2, 256, 64, [(200, 100), (7, 500)]),
    (12, 1, 240, 32, [(31, 40)]),
    (3, 1, 112, 128, [(130, 260)]),
    (256, 1, 64, 16, [(3, 40)]),                                       # more heads on one than an item has rows
    (1024, 2, 32, 16, [(2, 20)]),
    (6, 3, 96, 24, [(64, 1000)]),
    (1, 1, 128, 16, [(600, 0), (1, 5), (300, 300)]),
])
def test_chunks(kind, H, Hk, dh, page, chunks):
    Case(kind, H, Hk, dh, page, chunks).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,dh,chunks", [
    (4, 1, 64, [(1, 9000)]), (4, 1, 128, [(5, 20000)]), (8, 8, 128, [(2, 3000), (1, 10), (3, 2500)]), (2, 1, 256, [(9, 4000)]),
    (32, 4, 128, [(100, 5000)]), (16, 2, 64, [(1200, 100)])])
def test_items_that_are_cut_and_joined(kind, H, Hk, dh, chunks):
    Case(kind, H, Hk, dh, 64, chunks).check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,dh", [(32, 32, 128), (32, 16, 64), (8, 8, 256)])
def test_long_and_short_items_in_turn(kind, H, Hk, dh):
    """A thread block goes from items of a few rows to items of many and back."""
    Case(kind, H, Hk, dh, 32, [(1, 345), (300, 200), (2, 700), (290, 10), (100, 600), (257, 3), (40, 900), (513, 0)]).check()


@pytest.mark.parametrize("kind", KINDS)
def test_many_sequences(kind):
    """More sequences than a thread block has threads; one-token chunks and empty ones among them."""
    n = np.random.default_rng(3).integers(0, 4, 700).tolist()
    past = np.random.default_rng(4).integers(0, 50, 700).tolist()
    Case(kind, 4, 2, 64, 16, list(zip(n, past))).check()


@pytest.mark.parametrize("kind", KINDS)
def test_large_scores(kind):
    """Scores over hundreds: running maxima move, most weights vanish."""
    Case(kind, 8, 2, 64, 16, [(150, 400), (20, 0)], spread=25.0).check()


@pytest.mark.parametrize("kind", KINDS)
def test_ascending_scores(kind):
    """Every tile's maximum is far above the one before it."""
    c = Case(kind, 4, 2, 64, 16, [(130, 900)])
    c.q = c.q.abs() + 0.5
    ramp = torch.arange(c.table.shape[1] * 16, device=DEV).float() / 64
    rows = torch.zeros_like(c.K, dtype=F32)
    rows[c.table[0].long()] = ramp.view(-1, 1, 16, 1).expand(-1, 2, -1, 64)[: c.table.shape[1]]
    if kind == "8bit":
        c.K, c.Ks, c.Kv = eight(rows)
    else:
        c.K = rows.to(c.t)
        c.refresh()
    c.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("keep", [[1, 0, 1, 1, 0, 0, 0, 1], [0] * 8, [0, 0, 0, 0, 1, 1, 1, 1]])
def test_lost_heads(kind, keep):
    c = Case(kind, 8, 2, 64, 16, [(70, 100), (3, 2000)])
    c.keep = torch.tensor(keep, dtype=torch.uint8, device=DEV)
    c.check()


@pytest.mark.parametrize("kind", KINDS)
def test_rows_that_see_nothing(kind):
    """More new tokens than the sequence is long: the first of them are in front of it."""
    c = Case(kind, 4, 2, 64, 16, [(90, 10), (5, 0), (300, 0)])
    c.lens = torch.tensor([40, 0, 200], dtype=torch.int32, device=DEV)
    out, lse = c.check()
    assert (out[:50] == 0).all() and (lse[:50] == -INF).all()


@pytest.mark.parametrize("kind", KINDS)
def test_bad_lengths_rows_and_pages(kind):
    c = Case(kind, 4, 2, 64, 16, [(20, 100), (7, 30), (9, 40), (5, 60), (3, 0)])
    c.lens[1], c.lens[2] = -1, c.table.shape[1] * 16 + 1
    c.table[0, 2], c.table[3, 1], c.table[3, 3] = -1, c.K.shape[0], 2 ** 31 - 1
    out, _ = c.check()
    assert (out[20:36] == 0).all()
    c.start = torch.tensor([0, 20, 27, 25, -3, 3], dtype=torch.int32, device=DEV)      # decreasing, negative
    c.check()
    c.start = torch.tensor([0, 5, 9, 11, 12, 10 ** 6], dtype=torch.int32, device=DEV)
    c.check()
    c.start = torch.zeros(6, dtype=torch.int32, device=DEV)                            # no rows at all
    out, lse, bad = c.run()
    assert (out == 7).all() and (lse == 7).all() and bad != 0


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
@pytest.mark.parametrize("dh", [64, 256])
def test_what_a_row_does_not_see_has_no_influence(kind, what, dh):
    """NaN and infinities in keys and values behind a row's position, and behind the sequence's end."""
    c = Case(kind, 8, 2, dh, 16, [(150, 37), (40, 300)])
    for s, p, col in [(0, 100, 3), (0, 150, 11), (0, 183, 0), (1, 310, dh - 1), (1, 339, 5)]:
        page = c.table[s, p // 16].long()
        c.V[page, :, p % 16, col] = what
        c.V[page, 0, p % 16, col - 1] = -what
        if p == 150 or p == 339:
            c.K[page, :, p % 16] = what
    for s in range(2):      # the rest of the last page
        n = int(c.lens[s])
        c.K[c.table[s, (n - 1) // 16].long(), :, n % 16:] = NAN
        c.V[c.table[s, (n - 1) // 16].long(), :, n % 16:] = NAN
    c.refresh()
    out, lse, _ = c.run()
    c.compare(out, lse)
    before = slice(0, 100 - 37)                  # rows in front of the first of them: those that it reached would not be finite
    assert torch.isfinite(out[before]).all() and torch.isfinite(lse[before]).all()
    c.K, c.V = torch.nan_to_num(c.K, 0.0, 0.0, 0.0), torch.nan_to_num(c.V, 0.0, 0.0, 0.0)
    c.refresh()
    clean, clean_lse, _ = c.run()
    c.compare(clean, clean_lse)                  # both within the bound of the same definition: sums may be formed in another order
    assert torch.equal(clean_lse[before], lse[before])


@pytest.mark.parametrize("dh", [64, 256])
def test_rows_of_nan_in_an_8_bit_cache(dh):
    c = Case("8bit", 8, 2, dh, 16, [(60, 37)])
    page = c.table[0, 80 // 16].long()
    c.Vs[page, 1, 0], c.Ks[page, 0, 0] = 255, 255
    out, lse, _ = c.run()
    sees = torch.arange(60, device=DEV) + 37 >= 80
    assert torch.isnan(out[:60][sees]).all() and torch.isfinite(out[:60][~sees]).all()
    assert torch.equal(torch.isnan(lse[:60]), sees[:, None] & (torch.arange(8, device=DEV) < 4))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_scores_of_minus_infinity_and_the_lowest_value(kind):
    c = Case(kind, 4, 2, 64, 16, [(100, 20)])
    c.q[..., 0], c.K[..., 0] = 1.0, 0.0
    at = lambda p: (c.table[0, p // 16].long(), slice(None), p % 16, 0)  # noqa: E731
    for p in list(range(30)) + [60, 77]:
        c.K[at(p)] = -INF
    for p in (40, 90):
        c.K[at(p)] = torch.finfo(c.t).min
    c.refresh()
    out, lse = c.check()
    assert (out[:10] == 0).all() and (lse[:10] == -INF).all()


@pytest.mark.parametrize("kind", KINDS)
def test_strides(kind):
    """Queries inside a projection's output; keys and values page by page beside one another."""
    c = Case(kind, 8, 2, 64, 16, [(70, 90), (3, 200)])
    n_pages = c.K.shape[0]
    wide = torch.full((c.q.shape[0], 12 * 64), NAN, dtype=c.t, device=DEV)
    wide[:, : 8 * 64] = c.q.flatten(1)
    c.q = wide[:, : 8 * 64].view(-1, 8, 64)
    both = torch.full((n_pages, 2, *c.K.shape[1:]), 127 if kind == "8bit" else NAN, dtype=c.K.dtype, device=DEV)
    both[:, 0], both[:, 1] = c.K, c.V
    c.K, c.V = both[:, 0], both[:, 1]
    shape = c.shape
    c.shape = lambda: shape(c.K.stride(0))
    c.check()


@pytest.mark.parametrize("kind", KINDS)
def test_workspace_contents_and_repetition_change_nothing(kind):
    c = Case(kind, 8, 2, 128, 16, [(3, 3000), (300, 100)])
    got = []
    for fill in (0, 255, 127):
        out, lse = c.buffers()
        c.call(out, lse, c.workspace(fill))
        got.append((out, lse))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got[1:] for a, b in zip(g, got[0]))


@pytest.mark.parametrize("kind", KINDS)
def test_two_streams_and_a_graph(kind):
    a, b = Case(kind, 8, 2, 128, 16, [(3, 3000), (300, 100)]), Case(kind, 8, 2, 128, 16, [(500, 700)], seed=9)
    want = [(*x.run()[:2],) for x in (a, b)]
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    bufs = [[x.buffers() for _ in range(4)] for x in (a, b)]
    ws = [x.workspace() for x in (a, b)]
    torch.cuda.synchronize()
    for i in range(4):
        for x, st, buf, w in zip((a, b), streams, bufs, ws):
            x.call(*buf[i], w, stream=st)
    torch.cuda.synchronize()
    for buf, w in zip(bufs, want):
        assert all(torch.equal(t, u) for pair in buf for t, u in zip(pair, w))
    out, lse = a.buffers()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a.call(out, lse, ws[0])
    other = Case(kind, 8, 2, 128, 16, [(296, 104), (7, 2996)], seed=5)       # as many rows, sequences and pages, other lengths
    for name in ("q", "K", "V", "Ks", "Vs", "table", "lens", "start"):
        if getattr(a, name) is not None:
            getattr(a, name).copy_(getattr(other, name))
    if kind == "8bit":
        a.Kv, a.Vv = other.Kv, other.Vv
    else:
        a.refresh()
    out.fill_(7.0)
    lse.fill_(7.0)
    graph.replay()
    torch.cuda.synchronize()
    a.compare(out, lse)
    eager = a.run()
    assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])


def test_the_bound_itself_follows_the_oracle():
    c = Case("f32", 6, 2, 16, 5, [(4, 3), (3, 9), (2, 0), (0, 4)])
    c.keep = torch.tensor([1, 0, 1, 1, 1, 0], dtype=torch.uint8, device=DEV)
    c.table[1, 1], c.lens[0] = c.K.shape[0], 2
    got = c.expected()
    want = P.prompt_mha(*(x.double().cpu().numpy() for x in (c.q,)), c.start.cpu().numpy(), *(x.double().cpu().numpy() for x in (c.K, c.V)),
                        c.table.cpu().numpy(), c.lens.cpu().numpy(), c.scale, c.keep.cpu().numpy())
    for i in range(3):
        assert np.allclose(got[i].cpu().numpy(), want[i], rtol=1e-12, atol=1e-14)
    kept = c.keep.cpu().numpy() != 0
    assert np.allclose(got[3].cpu().numpy()[:, kept], want[3][:, kept], rtol=1e-12)
    assert (got[4].cpu().numpy() == want[4]).all() and got[5] == want[5]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("what", [INF, NAN])
@pytest.mark.parametrize("chunks", [[(60, 100), (9, 300), (50, 90)], [(60, 100), (60, 220), (60, 340)], [(60, 100)], [(1, 127), (300, 500)]])
def test_pieces_of_an_item_that_some_rows_do_not_see(kind, what, chunks):
    """Rows in front of a tile that a thread block has on its own: their weights there are zero, whatever its values are."""
    c = Case(kind, 8, 2, 64, 16, chunks)
    for s, (new, past) in enumerate(chunks):
        p = past + new - 1                       # of the last key, which the sequence's last row alone sees
        page = c.table[s, p // 16].long()
        if kind == "8bit":
            c.Vs[page, :, p % 16] = 255          # a row of NaN
            c.Vv[page, :, p % 16] = NAN
        else:
            c.V[page, :, p % 16, 7] = what
            c.V[page, 1, p % 16, 8] = -what
    if kind != "8bit":
        c.refresh()
    out, lse, _ = c.run()
    c.compare(out, lse)
    last = c.start[1:].long() - 1
    seen = torch.ones(out.shape[0], dtype=torch.bool, device=DEV)
    seen[last], seen[int(c.start[-1]):] = False, False
    assert torch.isfinite(out[seen]).all() and not torch.isfinite(out[last]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("factor", [-1.0, 0.0, -8.0])
def test_scales_that_are_negative_or_zero(kind, factor):
    """The largest score is then the smallest product; under zero every key has the same weight."""
    c = Case(kind, 8, 2, 64, 16, [(150, 400), (20, 0)])
    c.scale *= factor
    c.check()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,page", [(128, 8), (64, 40), (128, 2), (256, 8)])
def test_page_sizes(kind, dh, page):
    Case(kind, 8, 2, dh, page, [(150, 300), (1, 7), (33, 0)]).check()


def far(c):
    """The caches with their pages so far apart that elements of the last one, which is in use, lie more than 2^31 behind the first."""
    n_pages = c.K.shape[0]
    stride = 2 ** 31 // (n_pages - 2) // 64 * 64
    assert (n_pages - 1) * stride > 2 ** 31
    last = c.table == c.table.max()
    for x in (c.Ks, c.Vs, c.Kv, c.Vv, c.K, c.V):
        if x is not None:
            x[n_pages - 1] = x[int(c.table.max())]
    c.table[last] = n_pages - 1
    for name in ("K", "V"):
        x = getattr(c, name)
        store = torch.empty((n_pages - 1) * stride + x[0].numel(), dtype=x.dtype, device=DEV)
        y = store.as_strided(x.shape, (stride, *x.stride()[1:]))
        y.copy_(x)
        setattr(c, name, y)
    shape = c.shape
    c.shape = lambda: shape(stride)


@pytest.mark.parametrize("kind", KINDS)
def test_pages_behind_31_bits(kind):
    c = Case(kind, 4, 2, 64, 16, [(20, 30), (3, 12)])
    far(c)
    c.check()
