"""The append with norms per head, 8-bit cache rows, their way back, and one-token attention over them, against the definitions in
64 bits.

Append, before the rounding: a sum of dh squares in fp32 is off by at most dh 2^-24 relative, its root by half of that, the factors of a
normed element by 2^-22 together; cosine and sine of an angle reduced in fp64 and rounded to fp32 are off by 2^-21 of a turn's
length.  d = (dh 2^-24 + 2^-20) (|a| + |b|) turn_scale for the pair (a, b), normed.  bf16: + 2^-8 of the value, fp32: + 2^-24.
8-bit rows: the nearest code is off by 2^-4 of the value, or by half the smallest step, 2^-10 of the row's power of two; that power is
the double where d carries the largest element past 448.

Attention: as test_gpu_paged_attention, a weight rounded to fp16 after it was multiplied with 2^9 and its position's power of two
relative to the largest: off by 2^-11 of itself or, below fp16's normal numbers, by half its smallest step, 2^-25 / 2^9 = 2^-34 relative
to a weight of 1 at the largest power, for each of n positions.
"""
import numpy as np
import pytest
import torch

from oracle import paged_prompt_ref as P
from paper_2601_11676_b200 import binding as B
from tests.test_gpu_paged_prompt import BF16, DEV, F32, INF, NAN, Case, block_table, eight, far, gen, randn

pytestmark = pytest.mark.gpu


def host(x):
    return None if x is None else x.double().cpu().numpy()


class Append:
    def __init__(self, kind, H, Hk, dh, page, n_tok, rotary, inter=False, norm="both", turn_scale=1.0, seed=0, n_seq=3):
        g = gen(seed + dh + n_tok)
        self.kind, self.t = kind, F32 if kind == "f32" else BF16
        lens = [n_tok + 40] * n_seq
        self.table, n_pages = block_table(g, lens, page)
        qkv = randn(g, (n_tok, H + 2 * Hk, dh), self.t)
        self.q, self.k, self.v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
        self.w_q, self.w_k = (randn(g, (dh,), self.t) if on else None for on in (norm in ("both", "queries"), norm in ("both", "keys")))
        places = torch.randperm(n_seq * (n_tok + 40), generator=g, device=DEV)[:n_tok]       # no place twice
        self.seq, self.pos = (places % n_seq).int(), (places // n_seq).int()
        self.inv = 10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64, device=DEV) / max(rotary, 1)) if rotary else None
        self.inter, self.turn_scale, self.eps = inter, turn_scale, 1e-6
        shape = (n_pages, Hk, page, dh)
        self.Ks = self.Vs = None
        if kind == "8bit":
            self.K, self.V = (torch.full(shape, 17, dtype=torch.uint8, device=DEV) for _ in range(2))
            self.Ks, self.Vs = (torch.full(shape[:3], 99, dtype=torch.uint8, device=DEV) for _ in range(2))
        else:
            self.K, self.V = (torch.full(shape, 7.0, dtype=self.t, device=DEV) for _ in range(2))
        self.q_out = torch.full((n_tok, H, dh), 7.0, dtype=self.t, device=DEV)
        self.sh = B.paged_shape(H, Hk, dh, page, n_pages, self.table.shape[1], B.F32 if self.t is F32 else B.BF16)

    def call(self):
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.halo_paged_norm_append(self.sh, self.q, self.k, self.v, self.w_q, self.w_k, self.eps, self.pos, self.seq, self.table, self.inv,
                                 self.inter, self.turn_scale, self.q_out, self.K, self.V, self.Ks, self.Vs, st)
        torch.cuda.synchronize()
        return int(st.item())

    def read(self):
        n, (_, Hk, _, dh) = self.k.shape[0], self.K.shape
        k, v = (torch.full((n, Hk, dh), 5.0, dtype=self.t, device=DEV) for _ in range(2))
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        B.halo_paged_kv_read(self.sh, self.pos, self.seq, self.table, self.K, self.V, k, v, self.Ks, self.Vs, st)
        torch.cuda.synchronize()
        return k, v, int(st.item())

    def places(self):
        p = self.pos.long()
        return self.table[self.seq.long(), p // self.K.shape[2]].long(), p % self.K.shape[2]

    def turned(self, x, w):
        """The turned rows before the rounding, and d."""
        inv, pos = host(self.inv), host(self.pos).astype(np.int64)
        y = P.norm_turn(host(x), host(w), self.eps, pos, inv, self.inter, self.turn_scale)
        n = P.norm_turn(host(x), host(w), self.eps, pos, None, self.inter, 1.0)
        r, dh = 0 if inv is None else 2 * len(inv), n.shape[-1]
        pair = np.abs(n).copy()
        for i in range(r // 2):
            a, b = (2 * i, 2 * i + 1) if self.inter else (i, i + r // 2)
            pair[..., a] = pair[..., b] = np.abs(n[..., a]) + np.abs(n[..., b])
        return y, (dh * 2.0 ** -24 + 2.0 ** -20) * pair * max(self.turn_scale, 1.0)

    def check_queries(self, rows=slice(None)):
        u = 2.0 ** -24 if self.t is F32 else 2.0 ** -8
        q, dq = (x[rows] for x in self.turned(self.q, self.w_q))
        assert (np.abs(host(self.q_out)[rows] - q) <= dq + u * (np.abs(q) + dq)).all()

    def check(self):
        assert self.call() == 0
        self.check_queries()
        u = 2.0 ** -24 if self.t is F32 else 2.0 ** -8
        k, dk = self.turned(self.k, self.w_k)
        got_k, got_v, bad = self.read()
        assert bad == 0
        if self.kind == "8bit":
            codes, scales, values = P.eight_rows(host(self.v))                   # values are stored as they are: bit for bit
            page, at = self.places()
            assert torch.equal(self.V[page, :, at].cpu(), torch.from_numpy(codes)) and torch.equal(self.Vs[page, :, at].cpu(), torch.from_numpy(scales))
            assert (host(got_v) == values).all()
            unit = 2.0 ** (P.eight_rows(k)[1].astype(float) - 127)[..., None]
            assert (np.abs(host(got_k) - k) <= np.maximum(2.0 ** -4 * (np.abs(k) + dk), 2.0 ** -9 * unit) + dk).all()
        else:
            assert (host(got_v) == host(self.v)).all()
            assert (np.abs(host(got_k) - k) <= dk + u * (np.abs(k) + dk)).all()
            page, at = self.places()
            assert torch.equal(self.K[page, :, at], got_k) and torch.equal(self.V[page, :, at], got_v)
        # every other place of the caches stays as it was
        rest = torch.ones(self.K.shape[0], self.K.shape[2], dtype=torch.bool, device=DEV)
        rest[self.places()] = False
        for c, was in ((self.K, 17 if self.kind == "8bit" else 7), (self.V, 17 if self.kind == "8bit" else 7), (self.Ks, 99), (self.Vs, 99)):
            if c is not None:
                assert (c.transpose(1, 2)[rest] == was).all()


@pytest.mark.parametrize("kind", ["f32", "bf16", "8bit"])
@pytest.mark.parametrize("H,Hk,dh,page,n_tok,rotary,inter,norm,ts", [
    (4, 2, 64, 16, 1, 64, False, "both", 1.0),
    (32, 8, 128, 16, 33, 128, False, "both", 1.25),
    (8, 8, 128, 16, 700, 64, True, "both", 1.0),
    (5, 1, 80, 48, 40, 80, False, "keys", 1.0),       # half of the pairs' distance inside a lane's elements
    (5, 1, 80, 5, 40, 40, False, "queries", 1.1),
    (3, 3, 96, 7, 20, 24, False, "both", 0.5),
    (2, 1, 16, 1, 9, 6, False, "both", 1.0),
    (2, 1, 16, 16, 9, 6, True, "none", 1.0),
    (16, 2, 256, 32, 50, 256, False, "both", 1.0),
    (4, 4, 240, 16, 12, 120, True, "both", 1.0),
    (40, 8, 128, 64, 3, 0, False, "both", 1.0),
    (1, 1, 48, 16, 2, 2, False, "none", 1.0),
])
def test_append_and_read(kind, H, Hk, dh, page, n_tok, rotary, inter, norm, ts):
    Append(kind, H, Hk, dh, page, n_tok, rotary, inter, norm, ts).check()


@pytest.mark.parametrize("kind", ["f32", "bf16", "8bit"])
def test_append_many_tokens(kind):
    Append(kind, 8, 2, 128, 16, 4000, 128).check()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_append_without_a_norm_is_the_append(kind):
    """No norm, turn_scale 1: the numbers of halo_paged_kv_append up to a rounding of each product (elements below 8) and of the result."""
    a = Append(kind, 8, 2, 64, 16, 50, 64, norm="none")
    a.call()
    K, V, q = torch.full_like(a.K, 7.0), torch.full_like(a.V, 7.0), torch.empty_like(a.q_out)
    B.halo_paged_kv_append(a.sh, a.q, a.k, a.v, a.pos, a.seq, a.table, a.inv, False, q, K, V)
    step = 2.0 ** -7 if kind == "bf16" else 2.0 ** -23
    assert torch.equal(V, a.V)
    for x, y in ((q, a.q_out), (K, a.K)):
        assert ((x.float() - y.float()).abs() <= step * x.float().abs() + 4 * 8 * 2.0 ** -24).all()


def test_8_bit_rows_are_exact_where_nothing_is_computed():
    """Ties, subnormal codes, zeros of both signs, the largest and smallest powers, NaN and infinities: bit for bit."""
    a = Append("8bit", 4, 2, 64, 16, 400, 0, norm="none")
    g = gen(3)
    k = torch.randint(-16, 17, a.k.shape, generator=g, device=DEV).float() / 16 * torch.exp2(torch.randint(-12, 3, a.k.shape, generator=g, device=DEV).float())
    k *= torch.exp2(torch.randint(-126, 120, (400, 2, 1), generator=g, device=DEV).float())
    k[0], k[1, :, ::2], k[2, 0, 5], k[3, 1, 6], k[4, 0, 7] = 0, -0.0, INF, -INF, NAN
    k[5], k[6], k[7] = 2.0 ** -133, torch.finfo(BF16).max, -448.0
    a.k = k.to(BF16)
    a.v = -a.k
    a.call()
    page, at = a.places()
    for x, codes, scales in ((a.k, a.K, a.Ks), (a.v, a.V, a.Vs)):
        c, s, v = P.eight_rows(host(x))
        assert torch.equal(scales[page, :, at].cpu(), torch.from_numpy(s))
        assert torch.equal(codes[page, :, at].cpu(), torch.from_numpy(c))
    k, v, _ = a.read()
    for got, x in ((k, a.k), (v, a.v)):
        assert np.array_equal(host(got), P.eight_rows(host(x))[2], equal_nan=True)


@pytest.mark.parametrize("kind", ["f32", "bf16", "8bit"])
def test_padding_bad_places_and_keys_alone(kind):
    a = Append(kind, 4, 2, 64, 16, 12, 64)
    a.pos[2], a.pos[5], a.seq[7], a.seq[8] = -1, 10 ** 6, -1, 3
    a.table[a.seq[9].long(), a.pos[9].long() // 16] = a.K.shape[0]
    skipped = [t for t in range(12) if t in (2, 5, 7, 8) or (a.seq[t] == a.seq[9] and a.pos[t] // 16 == a.pos[9] // 16)]
    ok = [t for t in range(12) if t not in skipped]
    assert 9 in skipped and len(ok) > 3 and a.call() != 0
    assert (a.q_out[skipped] == 7).all()
    a.check_queries(ok)
    k, v, bad = a.read()
    assert bad != 0 and (k[skipped] == 5).all() and (v[skipped] == 5).all()
    assert (np.abs(host(v)[ok] - host(a.v)[ok]) <= 2.0 ** -4 * np.abs(host(a.v)[ok]) + 2.0 ** -10).all()
    keys, full = (Append(kind, 4, 2, 64, 16, 12, 64) for _ in range(2))
    keys.q = keys.q_out = None
    assert keys.call() == 0 and full.call() == 0
    for x, y in ((keys.K, full.K), (keys.V, full.V), (keys.Ks, full.Ks), (keys.Vs, full.Vs)):
        assert x is None or torch.equal(x, y)


def test_append_in_place_and_without_sequences():
    a, b = (Append("8bit", 4, 2, 64, 16, 3, 64) for _ in range(2))
    for x in (a, b):
        x.seq = torch.arange(3, dtype=torch.int32, device=DEV)
    b.seq = None
    b.q = b.q.clone()
    b.q_out = b.q
    a.call(), b.call()
    assert torch.equal(a.q_out, b.q_out) and torch.equal(a.K, b.K) and torch.equal(a.Ks, b.Ks)
    assert all(torch.equal(x, y) for x, y in zip(a.read(), b.read()) if torch.is_tensor(x))


# ---- one token per sequence ---------------------------------------------------------------------------------------------------

def attend(c, q, ws=None, stream=None):
    n, H, dh = q.shape
    out = torch.full((n, H, dh), NAN, dtype=BF16, device=DEV)
    lse = torch.full((n, H), NAN, dtype=F32, device=DEV)
    sh = c.shape()
    if ws is None:
        ws = torch.full((max(B.halo_paged_mha_f8_workspace_bytes(sh, n), 16),), 255, dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.halo_paged_mha_f8(sh, q, c.K, c.V, c.Ks, c.Vs, c.table, c.lens, c.scale, out, ws, c.keep, lse, st, stream)
    torch.cuda.synchronize()
    return out, lse, int(st.item())


def one_token_case(H, Hk, dh, page, lens, **more):
    """A case of chunks of one token each: its expected rows are those of one-token attention; rows of empty sequences are zeros."""
    c = Case("8bit", H, Hk, dh, page, [(1, n - 1) for n in lens], rows_behind=0, **more)
    return c


def check_tokens(c):
    out, lse, bad = attend(c, c.q)
    ref, ref_lse, size, reach, _, ref_bad = c.expected()
    e = (2.0 ** -21 + c.q.shape[2] * 2.0 ** -24 + 2.0 ** -20) * reach
    top = 448 * torch.exp2(c.Vs[c.Vs != 255].double().max() - 127)
    rough = (2 * e + 1e-5 + 2.0 ** -11)[..., None] * size + (c.lens.clamp(min=0).double() * 2.0 ** -34 * top)[:, None, None]
    assert ((out.double() - ref).abs() <= rough + 2.0 ** -8 * ref.abs()).all()
    fine = torch.isfinite(ref_lse)
    assert torch.equal(lse[~fine].double(), ref_lse[~fine])
    assert ((lse.double() - ref_lse).abs()[fine] <= (e + 1e-6 * (1 + ref_lse.abs()))[fine]).all()
    assert (bad != 0) == ref_bad
    return out, lse


@pytest.mark.parametrize("H,Hk,dh,page,lens", [
    (4, 4, 64, 16, [1]), (32, 4, 64, 16, [700]), (8, 8, 64, 16, [20, 1, 33, 0]), (32, 8, 128, 16, [9, 40, 300, 1, 2500]),
    (16, 1, 128, 64, [50, 2049]), (20, 1, 80, 48, [24, 77]), (5, 1, 80, 5, [77, 8]), (8, 2, 256, 16, [31, 5]), (12, 1, 256, 32, [18, 200]),
    (64, 2, 240, 16, [100, 1000]), (2, 1, 16, 1, [40, 3]), (6, 3, 112, 7, [130]), (1024, 4, 32, 16, [50]), (8, 2, 128, 16, [30000])])
def test_one_token(H, Hk, dh, page, lens):
    check_tokens(one_token_case(H, Hk, dh, page, lens))


def test_one_token_under_a_wide_table_and_many_sequences():
    check_tokens(one_token_case(8, 2, 64, 16, [3, 900], cols=5000))
    check_tokens(one_token_case(8, 2, 128, 16, np.random.default_rng(0).integers(0, 300, 300).tolist()))


@pytest.mark.parametrize("spread", [2.0 ** -100, 2.0 ** -10, 30.0, 2.0 ** 60])
def test_queries_of_any_size(spread):
    """The queries' own power of two; scale makes up for it so that the scores stay."""
    c = one_token_case(8, 2, 64, 16, [200, 31])
    c.q = (c.q.float() * spread).to(BF16)
    c.scale = c.scale / spread
    check_tokens(c)


def test_values_of_very_different_size():
    """Rows whose powers of two differ by up to 2^60, in rising and falling order: what the largest leaves of the others counts."""
    c = one_token_case(8, 2, 64, 16, [300, 129])
    for s, order in ((0, 1), (1, -1)):
        n = int(c.lens[s])
        p = torch.arange(n, device=DEV)
        by = (order * (p - n // 2) * 60 // n).clamp(-30, 30) + 127
        c.Vs[c.table[s, p // 16].long(), :, p % 16] = by[:, None].to(torch.uint8)
    c.Vv = torch.from_numpy(np.ldexp(1.0, c.Vs.cpu().numpy().astype(int) - 127))[..., None].to(DEV) * c.V.view(torch.float8_e4m3fn).float().double()
    check_tokens(c)


def test_one_token_lost_heads_bad_pages_and_lengths():
    c = one_token_case(8, 2, 64, 16, [40, 300, 100, 17, 5])
    c.keep = torch.tensor([1, 0, 1, 1, 0, 0, 0, 0], dtype=torch.uint8, device=DEV)
    out, lse = check_tokens(c)
    assert (out[:, 1] == 0).all() and (lse[:, 4:] == -INF).all()
    c.keep = None
    c.lens[2], c.lens[3], c.table[1, 3], c.table[0, 0] = -4, 10 ** 6, -1, c.K.shape[0]
    check_tokens(c)


def test_one_token_rows_of_nan():
    c = one_token_case(8, 2, 64, 16, [100, 200])
    c.Vs[c.table[0, 2].long(), 0, 3], c.Ks[c.table[1, 5].long(), 1, 4] = 255, 255
    out, lse, _ = attend(c, c.q)
    nan = torch.zeros(2, 8, dtype=torch.bool, device=DEV)
    nan[0, :4] = nan[1, 4:] = True
    assert torch.equal(torch.isnan(out).all(-1), nan) and torch.equal(torch.isfinite(out).all(-1), ~nan)
    nan[0] = False
    assert torch.equal(torch.isnan(lse), nan)


def test_one_token_streams_and_a_graph():
    a, b = one_token_case(8, 2, 128, 16, [3000, 5, 900]), one_token_case(8, 2, 128, 16, [100, 4000], seed=3)
    want = [attend(x, x.q)[:2] for x in (a, b)]
    streams = [torch.cuda.Stream(DEV) for _ in range(2)]
    ws = [torch.empty(B.halo_paged_mha_f8_workspace_bytes(x.shape(), len(x.lens)), dtype=torch.uint8, device=DEV) for x in (a, b)]
    outs = [[torch.empty_like(x.q) for _ in range(6)] for x in (a, b)]
    torch.cuda.synchronize()
    for i in range(6):
        for x, st, w, o in zip((a, b), streams, ws, outs):
            B.halo_paged_mha_f8(x.shape(), x.q, x.K, x.V, x.Ks, x.Vs, x.table, x.lens, x.scale, o[i], w, stream=st)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(t, w[0]) for t in o)
    out, graph = torch.empty_like(a.q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.halo_paged_mha_f8(a.shape(), a.q, a.K, a.V, a.Ks, a.Vs, a.table, a.lens, a.scale, out, ws[0])
    a.lens.copy_(torch.tensor([10, 4, 899], dtype=torch.int32))
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, attend(a, a.q)[0])


# ---- a run of them together ---------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "bf16", "8bit"])
def test_a_prompt_in_chunks_then_tokens(kind):
    """A prompt appended and attended in two chunks and a token after it, against attention over all of it, read back from the cache."""
    H, Hk, dh, page, n = 8, 2, 64, 16, [150, 70, 1]
    g, t = gen(1), F32 if kind == "f32" else BF16
    table, n_pages = block_table(g, [sum(n), 5], page)
    sh = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], B.F32 if kind == "f32" else B.BF16)
    c = Case(kind, H, Hk, dh, page, [(sum(n), 0)], rows_behind=0)
    c.table, c.K = table[:1].contiguous(), torch.zeros((n_pages, Hk, page, dh), dtype=torch.uint8 if kind == "8bit" else t, device=DEV)
    c.V = torch.zeros_like(c.K)
    if kind == "8bit":
        c.Ks, c.Vs = (torch.zeros((n_pages, Hk, page), dtype=torch.uint8, device=DEV) for _ in range(2))
    qkv = randn(g, (sum(n), H + 2 * Hk, dh), t)
    w_q, w_k = randn(g, (dh,), t), randn(g, (dh,), t)
    inv = 10000.0 ** (-torch.arange(0, dh, 2, dtype=torch.float64, device=DEV) / dh)
    q = torch.empty((sum(n), H, dh), dtype=t, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((sum(n), H), 7.0, dtype=F32, device=DEV)
    at = 0
    for m in n:
        rows = slice(at, at + m)
        pos = torch.arange(at, at + m, dtype=torch.int32, device=DEV)
        x = qkv[rows]
        B.halo_paged_norm_append(sh, x[:, :H], x[:, H:H + Hk], x[:, H + Hk:], w_q, w_k, 1e-6, pos, torch.zeros_like(pos), table, inv, False,
                                 1.0, q[rows], c.K, c.V, c.Ks, c.Vs)
        lens = torch.tensor([at + m], dtype=torch.int32, device=DEV)
        args = (table[:1].contiguous(), lens, c.scale, out[rows])
        one = B.paged_shape(H, Hk, dh, page, n_pages, table.shape[1], B.F32 if kind == "f32" else B.BF16)
        if m > 1:
            ws = torch.empty(B.halo_paged_prompt_mha_workspace_bytes(one, m, 1), dtype=torch.uint8, device=DEV)
            B.halo_paged_prompt_mha(one, q[rows], torch.tensor([0, m], dtype=torch.int32, device=DEV), c.K, c.V, *args, ws, c.Ks, c.Vs,
                                    lse=lse[rows])
        elif kind == "8bit":
            ws = torch.empty(max(B.halo_paged_mha_f8_workspace_bytes(one, 1), 16), dtype=torch.uint8, device=DEV)
            B.halo_paged_mha_f8(one, q[rows], c.K, c.V, c.Ks, c.Vs, *args, ws, lse=lse[rows])
        else:
            ws = torch.empty(max(B.halo_paged_mha_workspace_bytes(one, 1), 16), dtype=torch.uint8, device=DEV)
            B.halo_paged_mha(one, q[rows], c.K, c.V, *args, ws, lse=lse[rows])
        at += m
    k, v = (torch.empty((sum(n), Hk, dh), dtype=t, device=DEV) for _ in range(2))
    pos = torch.arange(sum(n), dtype=torch.int32, device=DEV)
    B.halo_paged_kv_read(sh, pos, torch.zeros_like(pos), table, c.K, c.V, k, v, c.Ks, c.Vs)
    torch.cuda.synchronize()
    c.Kv, c.Vv = (torch.zeros((n_pages, Hk, page, dh), dtype=torch.float64, device=DEV) for _ in range(2))
    where = (table[0, pos.long() // page].long(), slice(None), pos.long() % page)
    c.Kv[where], c.Vv[where], c.q = k.double(), v.double(), q
    c.compare(out, lse)


@pytest.mark.parametrize("factor", [-1.0, 0.0, -8.0])
def test_one_token_under_scales_that_are_negative_or_zero(factor):
    c = one_token_case(8, 2, 64, 16, [200, 31, 1, 900])
    c.scale *= factor
    check_tokens(c)


def test_one_token_and_rows_in_pages_behind_31_bits():
    c = one_token_case(4, 2, 64, 16, [50, 15])
    far(c)
    check_tokens(c)
    pos = torch.arange(50, dtype=torch.int32, device=DEV)
    k, v = (torch.empty((50, 2, 64), dtype=BF16, device=DEV) for _ in range(2))
    B.halo_paged_kv_read(c.shape(), pos, torch.zeros_like(pos), c.table, c.K, c.V, k, v, c.Ks, c.Vs)
    where = (c.table[0, pos.long() // 16].long(), slice(None), pos.long() % 16)
    assert torch.equal(k.double(), c.Kv[where]) and torch.equal(v.double(), c.Vv[where])
    # and written there: the same rows again, which come back as they are
    q = torch.zeros((50, 4, 64), dtype=BF16, device=DEV)
    c.K[where], c.Ks[where], c.V[where], c.Vs[where] = 1, 1, 1, 1
    B.halo_paged_norm_append(c.shape(), q, k, v, None, None, 1e-6, pos, torch.zeros_like(pos), c.table, None, False, 1.0, q.clone(), c.K, c.V,
                             c.Ks, c.Vs)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    B.halo_paged_kv_read(c.shape(), pos, torch.zeros_like(pos), c.table, c.K, c.V, k2, v2, c.Ks, c.Vs)
    assert torch.equal(k, k2) and torch.equal(v, v2)
