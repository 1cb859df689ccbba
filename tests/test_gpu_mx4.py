"""Microscaled 4-bit rows against the fp64 oracle: codes and scales bit for bit, products within the order of fp32 sums."""
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


def quantize(W):
    n, d = W.shape
    Q = torch.full((n, d // 2), 0xEE, dtype=torch.uint8, device=DEV)
    S = torch.full((B.halo_mx4_scale_bytes(d, n),), 0xEE, dtype=torch.uint8, device=DEV)
    B.halo_quantize_rows_mx4(d, n, B.F32 if W.dtype == torch.float32 else B.BF16, W, Q, S)
    return Q, S


def values(Q, S, n, d):
    """The same numbers as the oracle's mx4_unpack, on the device in fp64 (large cases)."""
    codes = torch.stack([Q & 15, Q >> 4], -1).view(n, d).long()
    size = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device=DEV)[codes & 7]
    r, b = torch.arange(n, device=DEV)[:, None], torch.arange(d // 32, device=DEV)[None]
    unit = torch.exp2(S[((r // 128) * (d // 128) + b // 4) * 512 + (r % 32) * 16 + (r % 128) // 32 * 4 + b % 4].double() - 127)
    return torch.where(codes > 7, -size, size) * unit.repeat_interleave(32, 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d", [(1, 128), (3, 384), (127, 128), (130, 256), (33, 2048), (5, 1152), (8191, 128), (8200, 384)])
def test_rows_match_oracle_bit_for_bit(dtype, n, d):
    t, code, _ = TYPES[dtype]
    g = gen(n + d)
    W = torch.randn((n, d), generator=g, device=DEV) * 10.0 ** torch.randint(-4, 4, (n, 1), generator=g, device=DEV)
    W = W.to(t)
    # ties, powers of two and what lies next to them, zeros, a zero block, tiny and huge blocks
    W[0, :16] = torch.tensor([6, 5, 3.5, 2.5, 1.75, 1.25, .75, .25, -5, -3.5, -2.5, -.25, 0, -0., 7.5, 4], device=DEV).to(t)
    W[0, 32:64] = 0
    W[0, 64:96] = torch.linspace(1, 32, 32, device=DEV).to(t) * 2.0 ** -130
    W[0, 96:128] = torch.linspace(-1, 1, 32, device=DEV).to(t) * 3e38
    if n > 2:
        W[1, :32], W[1, 32:64] = 2.0 ** -126, torch.finfo(t).max
        W[2, :32] = 1.0
        W[2, 0] = 8.0 * (1 - 2.0 ** -8)
    Q, S = quantize(W)
    codes, scales = A.mx4_quantize(W.double().cpu().numpy())
    Q_ref, S_ref = A.mx4_pack(codes, scales)
    assert (S.cpu().numpy() == S_ref).all()
    assert (Q.cpu().numpy() == Q_ref).all()
    ref = A.mx4_unpack(Q_ref, S_ref, n, d)
    for name in ("f32", "bf16"):
        out = torch.empty((n, d), dtype=TYPES[name][0], device=DEV)
        B.halo_dequantize_rows_mx4(d, n, TYPES[name][1], Q, S, out)
        assert (out.double().cpu().numpy() == ref).all()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_a_block_with_a_value_that_is_not_finite_reads_back_as_nan(what):
    W = torch.randn((2, 256), generator=gen(1), device=DEV)
    W[1, 77] = what
    Q, S = quantize(W)
    out = torch.empty_like(W)
    B.halo_dequantize_rows_mx4(256, 2, B.F32, Q, S, out)
    bad = torch.zeros_like(W, dtype=torch.bool)
    bad[1, 64:96] = True
    assert torch.equal(torch.isnan(out), bad)
    Qx, Sx = quantize(torch.ones((1, 256), device=DEV))
    y = torch.empty((1, 2), device=DEV)
    B.halo_product_mx4(256, 1, 2, Qx, Sx, Q, S, B.F32, y)
    assert torch.isfinite(y[0, 0]) and torch.isnan(y[0, 1])


PRODUCT = [(1, 1, 128), (1, 130, 256), (1, 8300, 256), (1, 8300, 2048), (1, 33001, 128), (2, 257, 384), (8, 128, 128), (15, 1000, 2048), (16, 64, 640), (17, 300, 256), (31, 90, 256), (32, 8300, 256), (33, 129, 512), (40, 8193, 128),
           (64, 1111, 1024), (65, 128, 128), (100, 333, 384), (129, 256, 4096), (256, 640, 1152), (257, 100, 256), (700, 1030, 512),
           (1, 32000, 4096), (5, 4096, 11008), (300, 4096, 4096), (1, 40, 65536), (3, 40, 65536), (70, 40, 65536),
           (300, 11008, 256), (1000, 9601, 256), (390, 9600, 384), (100, 20000, 2176)]   # a round of whole tiles and halves behind it


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,d", PRODUCT)
def test_product_matches_fp64(dtype, T, n, d):
    """The fp32 sum of d products: at most (d / 64 + 64) 2^-23 of the sum of their sizes, and one rounding of the result."""
    t, code, u = TYPES[dtype]
    g = gen(T * 7 + n + d)
    x = torch.randn((T, d), generator=g, device=DEV) * 2.0 ** torch.randint(-8, 8, (T, 1), generator=g, device=DEV)
    w = torch.randn((n, d), generator=g, device=DEV) * 2.0 ** torch.randint(-20, 3, (n, d // 32, 1), generator=g, device=DEV).expand(
        n, d // 32, 32).reshape(n, d)
    Qx, Sx = quantize(x)
    Qw, Sw = quantize(w)
    guard = torch.full((T * n + 64,), 7.0, dtype=t, device=DEV)      # behind the last output nothing is written
    y, st = guard[: T * n].view(T, n), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.halo_product_mx4(d, T, n, Qx, Sx, Qw, Sw, code, y, st)
    torch.cuda.synchronize()
    assert int(st.item()) == 0 and (guard[T * n:] == 7).all()
    xv, wv = values(Qx, Sx, T, d), values(Qw, Sw, n, d)
    ref, size = xv @ wv.t(), xv.abs() @ wv.abs().t()
    assert ((y.double() - ref).abs() <= (d / 64 + 64) * 2.0 ** -23 * size + u * ref.abs()).all()
    first = y.clone()
    B.halo_product_mx4(d, T, n, Qx, Sx, Qw, Sw, code, y, st)
    assert torch.equal(y, first)


def test_product_places_every_element_and_scale():
    """One element at a time: x has a single 1 at element e, so y reads column e of the weights with its own scale; rows'
    scales differ, so a scale of another row or run would show."""
    d, n, T = 512, 300, 40
    g = gen(4)
    w = torch.randint(-6, 7, (n, d // 32, 32), generator=g, device=DEV).float() * 2.0 ** (
        torch.arange(n, device=DEV)[:, None, None] % 11 - 3.0 * (torch.arange(d // 32, device=DEV)[None, :, None] % 5))
    Qw, Sw = quantize(w.view(n, d))
    wv = values(Qw, Sw, n, d)
    for e0 in range(0, d, T):
        T_ = min(T, d - e0)
        x = torch.zeros((T_, d), device=DEV)
        x[torch.arange(T_, device=DEV), e0 + torch.arange(T_, device=DEV)] = 2.0 ** (torch.arange(T_, device=DEV) % 7).float()
        Qx, Sx = quantize(x)
        y = torch.empty((T_, n), device=DEV)
        B.halo_product_mx4(d, T_, n, Qx, Sx, Qw, Sw, B.F32, y)
        assert torch.equal(y.double(), x.double() @ wv.t())


@pytest.mark.parametrize("T", [1, 7, 300])
def test_quantise_and_product_captured_into_a_graph_and_on_another_stream(T):
    """One captured pair of calls replayed on new activations; the same bits as calls on a side stream."""
    g, n, d = gen(9), 520, 1152
    Qw, Sw = quantize(torch.randn((n, d), generator=g, device=DEV))
    x = torch.randn((T, d), generator=g, device=DEV).bfloat16()
    Q, S = torch.empty((T, d // 2), dtype=torch.uint8, device=DEV), torch.empty(B.halo_mx4_scale_bytes(d, T), dtype=torch.uint8, device=DEV)
    y, side = torch.empty((T, n), dtype=torch.bfloat16, device=DEV), torch.cuda.Stream()

    def step(stream=None):
        B.halo_quantize_rows_mx4(d, T, B.BF16, x, Q, S, stream=stream)
        B.halo_product_mx4(d, T, n, Q, S, Qw, Sw, B.BF16, y, stream=stream)

    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.copy_(torch.randn((T, d), generator=g, device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        side.wait_stream(torch.cuda.current_stream())
        step(side)
        side.synchronize()
        assert torch.equal(got, y)
        ref = values(Q, S, T, d) @ values(Qw, Sw, n, d).t()
        assert ((got.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + 1e-4 * ref.abs().max()).all()


@pytest.mark.parametrize("big", [2.0 ** 123, 2.0 ** -120])
@pytest.mark.parametrize("T", [1, 2, 20, 40, 70])
def test_scales_at_both_ends_of_their_range_meet_in_range(T, big):
    """Tokens near one end of the fp32 range times weights near the other: the products are ordinary numbers, so no step in
    between may leave the range.  Small whole numbers times powers of two: every sum below is exact in 24 bits."""
    n, d = 70, 256
    g = gen(T)
    x = torch.randint(-6, 7, (T, d), generator=g, device=DEV).float().clamp(-4, 4)
    w = torch.randint(-4, 5, (n, d), generator=g, device=DEV).float()
    x[:, ::32] = 4.0
    w[:, ::32] = 4.0            # both sides' blocks keep the numbers 0..4 exactly
    Qx, Sx = quantize(x * big)
    Qw, Sw = quantize(w / big)
    y = torch.empty((T, n), device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.halo_product_mx4(d, T, n, Qx, Sx, Qw, Sw, B.F32, y, st)
    assert torch.equal(y.double(), x.double() @ w.double().T) and int(st) == 0
