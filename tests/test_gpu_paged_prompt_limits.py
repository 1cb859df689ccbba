"""halo_paged_prompt_mha and halo_paged_mha_f8 where contents are extreme: values that are infinite or NaN over long sequences and in all of
an item's last tiles, values near the largest number, queries of many powers of two, rows of two sequences or of none.  Against the
definition in 64 bits, with the bounds of test_gpu_paged_prompt and test_gpu_eight_bit_cache."""
import numpy as np
import pytest
import torch

from oracle import paged_prompt_ref as P
from tests.test_gpu_eight_bit_cache import attend, check_tokens, one_token_case
from tests.test_gpu_paged_prompt import BF16, DEV, INF, KINDS, NAN, Case, eight, gen

pytestmark = pytest.mark.gpu


def spoil(c, s, p, col, what, heads=slice(None)):
    """An infinite or NaN value at position p of sequence s; of an 8-bit cache the whole row is NaN."""
    page, at = c.table[s, p // c.K.shape[2]].long(), p % c.K.shape[2]
    if c.kind == "8bit":
        c.Vs[page, heads, at], c.Vv[page, heads, at] = 255, NAN
    else:
        c.V[page, heads, at, col] = what
        c.Vv[page, heads, at, col] = what


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh", [64, 128])
def test_values_that_are_not_finite_over_a_long_sequence(kind, dh):
    """One that every row sees, far in front, and one that some of the last tile's rows see; the sequence behind is untouched by both, and
    nothing runs out of time."""
    c = Case(kind, 4, 2, dh, 16, [(200, 40000), (150, 60)])
    spoil(c, 0, 5, 3, NAN, 0)
    spoil(c, 0, 40120, 7, INF, 1)
    out, lse, bad = c.run()
    assert bad == 0
    c.compare(out, lse)
    assert torch.isfinite(out[200:350]).all() and torch.isnan(out[:200, :2, 3]).all() and torch.isfinite(out[:120, 2:]).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,dh,page", [(2, 2, 64, 16), (2, 2, 128, 16), (2, 2, 256, 64), (2, 2, 144, 32), (8, 2, 128, 5), (5, 1, 80, 48), (12, 1, 64, 24)])
@pytest.mark.parametrize("chunks", [[(256, 300), (300, 5), (130, 0)], [(255, 129), (1, 400), (40, 990)]])
def test_last_tiles_full_of_values_that_are_not_finite(kind, H, Hk, dh, page, chunks):
    """Every row sees another part of them, in up to three tiles of an item, whole and cut."""
    c = Case(kind, H, Hk, dh, page, chunks)
    g = gen(11)
    kinds = [INF, -INF, NAN]
    for s, (new, past) in enumerate(chunks):
        for p in range(past + 1, past + new, 9):
            pick = torch.randint(0, 1 << 20, (3,), generator=g, device=DEV).tolist()
            spoil(c, s, p, pick[0] % dh, kinds[pick[1] % 3], pick[2] % Hk)
    out, lse, bad = c.run()
    assert bad == 0
    c.compare(out, lse)
    first = c.start[:-1].long()
    assert torch.isfinite(out[first]).all()


def rising(c, size):
    """Scores that rise by 18 powers of two from a sequence's first position to its last, over values of about `size` of one sign."""
    page, dh = c.K.shape[2], c.K.shape[3]
    c.q = torch.zeros_like(c.q)
    c.q[..., 0] = 1.0
    K, V = torch.zeros(c.K.shape, device=DEV), torch.full(c.V.shape, 0.0, device=DEV)
    g = gen(21)
    for s, n in enumerate(c.lens.tolist()):
        p = torch.arange(n, device=DEV)
        at = (c.table[s].long()[p // page], slice(None), p % page)
        K[at] = torch.nn.functional.pad((p * (18 * 0.6931 / c.scale) / max(n - 1, 1))[:, None, None], (0, dh - 1)).expand(-1, K.shape[1], -1)
        V[at] = (0.5 + 0.5 * torch.rand((n, K.shape[1], dh), generator=g, device=DEV)) * size
    if c.kind == "8bit":
        c.K, c.Ks, c.Kv = eight(K)
        c.V, c.Vs, c.Vv = eight(V)
    else:
        c.K, c.V = K.to(c.t), V.to(c.t)
        c.refresh()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dh,chunks", [(64, [(150, 400), (1, 0)]), (128, [(20, 3000), (300, 0)]), (256, [(9, 700)]), (128, [(5, 20000)])])
def test_values_near_the_largest_under_rising_scores(kind, dh, chunks):
    """fp32 caches: a plain sum of the values has to be finite."""
    c = Case(kind, 4, 2, dh, 16, chunks)
    rising(c, 1e34 if kind == "f32" else 3e38)
    out, _ = c.check()
    assert torch.isfinite(out[: int(c.start[-1])]).all()


@pytest.mark.parametrize("kind", ["bf16", "8bit"])
@pytest.mark.parametrize("size", [1e-15, 1e15])
def test_values_of_other_sizes(kind, size):
    c = Case(kind, 4, 2, 128, 16, [(150, 400), (3, 5000)])
    rising(c, size)
    c.check()


@pytest.mark.parametrize("H,Hk,dh,lens", [(8, 2, 64, [700]), (32, 8, 128, [9, 40, 300, 1, 2500]), (8, 2, 128, [30000]), (16, 1, 256, [64, 1000]), (8, 8, 64, [300] * 150)])
@pytest.mark.parametrize("size", [3e38, 1e-30])
def test_one_token_over_values_near_the_largest_and_small_ones(H, Hk, dh, lens, size):
    c = one_token_case(H, Hk, dh, 16, lens)
    rising(c, size)
    out, _ = check_tokens(c)
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("bits", [0, 30, 38, 45])
def test_queries_whose_elements_spread_over_many_powers_of_two(bits):
    """Small elements of a query meet large ones of the keys, so that all count.  An element is exact from 2^-31 of its row's largest on, and off
    by at most 2^-39 of that below."""
    c = one_token_case(8, 2, 64, 16, [200, 31])
    by = torch.exp2(-(torch.arange(64, device=DEV) * bits // 63).float())
    c.q = (c.q.float() * by).to(BF16)
    c.K, c.Ks, c.Kv = eight(torch.randn(c.K.shape, generator=gen(5), device=DEV) / by)
    out, lse, bad = attend(c, c.q)
    ref, ref_lse, size, reach, _, _ = c.expected()
    e = (2.0 ** -21 + 64 * 2.0 ** -24 + 2.0 ** -20) * reach
    # the largest lies in [2^14, 2^15) and fp16's smallest step is 2^-24: an element is off by 2^-25 at most, 2^-39 of the largest.  Elements
    # are 2^-bits times a normal number, so that with 30 bits too a few lie below 2^-31 of the largest
    e = e + 2.0 ** -39 * c.q.double().abs().amax(-1) * c.Kv.abs().sum(-1).max() * c.scale
    top = 448 * torch.exp2(c.Vs.double().max() - 127)
    rough = (2 * e + 1e-5 + 2.0 ** -11)[..., None] * size + (c.lens.double() * 2.0 ** -34 * top)[:, None, None]
    assert bad == 0 and ((out.double() - ref).abs() <= rough + 2.0 ** -8 * ref.abs()).all()
    assert ((lse.double() - ref_lse).abs() <= e + 1e-6 * (1 + ref_lse.abs())).all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("start,mine", [
    ([0, 20, 10, 30], [20, 0, 0]),                      # the third begins inside the first
    ([0, 20, 10, 30, 25, 40], [20, 0, 0, 0, 0]),        # the fifth inside the third, which is left out
    ([5, 3, 9, 9, 30, 12, 40, 40], [0, 6, 0, 21, 0, 0, 0]),
    ([0, 10, 10 ** 6, 10, 25], [10, 0, 0, 15]),         # what is out of range holds nothing
    ([30, 40, 0, 12, 8, 20, 39, 40], [10, 0, 0, 0, 0, 0, 0]),
])
def test_rows_that_two_sequences_claim(kind, start, mine):
    """They belong to the first one; the other is left out as a whole."""
    n = len(mine)
    c = Case(kind, 4, 2, 64, 16, [(40, 100 + 30 * s) for s in range(n)])
    c.q = c.q[:40].contiguous()
    for s in range(n):
        c.lens[s] -= 40 - max(start[s + 1] - start[s], 0) if start[s + 1] <= 40 else 0
    c.start = torch.tensor(start, dtype=torch.int32, device=DEV)
    out, lse, bad = c.run()
    assert bad != 0
    # the same calls with the others' rows taken away
    want, want_lse = c.buffers()
    for s, k in enumerate(mine):
        if k:
            one = Case(kind, 4, 2, 64, 16, [(40, 100 + 30 * i) for i in range(n)])
            one.q, one.table, one.lens = c.q[start[s]:start[s] + k].contiguous(), c.table[s:s + 1].contiguous(), c.lens[s:s + 1].contiguous()
            one.start = torch.tensor([0, k], dtype=torch.int32, device=DEV)
            one.compare(out[start[s]:start[s] + k], lse[start[s]:start[s] + k])
            want[start[s]:start[s] + k], want_lse[start[s]:start[s] + k] = out[start[s]:start[s] + k], lse[start[s]:start[s] + k]
    assert torch.equal(out, want) and torch.equal(lse, want_lse)          # the other rows stay as they were


def test_many_sequences_that_claim_rows_twice():
    """More of them than a thread block has threads."""
    starts, n = [0], 700
    g = np.random.default_rng(8)
    for i in range(n):
        starts.append(max(starts[-1] - 3, 0) if i % 50 == 20 else starts[-1] + int(g.integers(0, 3)))
    c = Case("bf16", 4, 2, 64, 16, [(2, int(g.integers(2, 60))) for _ in range(n)])
    c.q = c.q[: max(starts)].contiguous()
    c.start = torch.tensor(starts, dtype=torch.int32, device=DEV)
    out, lse, bad = c.run()
    ref, ref_lse, size, reach, mine, ref_bad = P.prompt_mha(c.q.double().cpu().numpy(), np.array(starts), c.Kv.cpu().numpy(), c.Vv.cpu().numpy(),
                                                            c.table.cpu().numpy(), c.lens.cpu().numpy(), c.scale)
    assert bad != 0 and ref_bad and not mine.all()
    out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (out[~mine] == 7).all() and (lse[~mine] == 7).all()
    e = (2.0 ** -21 + 64 * 2.0 ** -24 + 2.0 ** -20) * reach
    assert (np.abs(lse - ref_lse) <= e + 1e-5 + 1e-6 * (1 + np.abs(ref_lse)))[mine].all()
    assert (np.abs(out - ref) <= (2 * e + 1e-5 + 2.0 ** -8)[..., None] * size + 2.0 ** -8 * np.abs(ref))[mine].all()


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,Hk,dh", [(32, 8, 128), (8, 2, 64), (6, 2, 256)])
@pytest.mark.parametrize("what", [NAN, INF, 3e38])
def test_rows_of_no_sequence_have_no_influence(kind, H, Hk, dh, what):
    """A padded batch: whatever lies behind the last sequence's rows changes no bit of the others."""
    c = Case(kind, H, Hk, dh, 16, [(5, 300), (1, 900), (140, 200), (3, 40)], rows_behind=200)
    c.start = torch.tensor([0, 5, 6, 146, 149], dtype=torch.int32, device=DEV)
    got = []
    for fill in (0.0, what):
        c.q[149:] = fill
        out, lse = c.check()
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("past", [0, 300])
def test_a_value_of_nan_counts_however_small_its_weight(kind, past):
    """Weights that underflow: of the first keys, in tiles that every row sees and in an item's last ones."""
    c = Case(kind, 4, 2, 64, 16, [(100, past)])
    rising(c, 1.0)
    c.q[..., 0] = 40.0                                   # 720 powers of two from the first key to the last
    spoil(c, 0, past, 5, NAN)
    out, _, bad = c.run()
    assert bad == 0
    assert torch.isnan(out[:100, :, 5]).all()            # every row sees that position
    assert kind == "8bit" or torch.isfinite(out[:100, :, 6]).all()
