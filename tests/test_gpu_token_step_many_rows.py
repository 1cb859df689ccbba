"""The forms that halo_norm_glue takes for many rows and halo_product_mx4 for few tokens through many long rows, against fp64.

Bounds as in test_gpu_attention_block (norms: sums of squares of d positive fp32 terms, 2^-18 relative) and test_gpu_mx4
(products: the order of d fp32 sums, (d / 64 + 64) 2^-23 of the sum of their sizes); u = half a rounding step of the output.
"""
import pytest
import torch

from paper_2601_11676_b200 import binding as B
from tests.test_gpu_mx4 import quantize, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = {"bf16": (torch.bfloat16, B.BF16, 2.0 ** -8), "f32": (torch.float32, B.F32, 2.0 ** -24)}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, shape, t):
    return torch.randn(shape, generator=g, device=DEV).to(t)


# 296 rows and more: two units of 8 per thread, in a warp per row up to 512 elements and in a thread block above; 264 and 520 leave
# the second unit of some lanes empty, 5120 fills 1.25 of them, 16384 and 8200 are the widest of either form
@pytest.mark.parametrize("n,d", [(301, 264), (300, 512), (297, 520), (300, 5120), (296, 2048), (295, 2056), (299, 8200), (296, 16384), (700, 256), (1001, 40)])
@pytest.mark.parametrize("ty,tx", [("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("gate", ["full", "wide", "row", None])
def test_norm_glue_of_many_rows(n, d, ty, tx, gate):
    yt, ycode, _ = TYPES[ty]
    xt, xcode, u = TYPES[tx]
    g = gen(n + d)
    h, y = randn(g, (n, d), torch.float32) * 5, randn(g, (n, d), yt)
    w_post, w_pre = randn(g, (d,), xt), randn(g, (d,), xt)
    gt = {None: lambda: None, "row": lambda: randn(g, (d,), xt), "full": lambda: randn(g, (n, d), xt),
          "wide": lambda: randn(g, (n, d + 64), xt)[:, 32:32 + d]}[gate]()
    y[1], h[2] = 0, 0
    eps, res = 1e-5, 0.37
    norm = lambda v: v / torch.sqrt(v.square().mean(-1, keepdim=True) + eps)  # noqa: E731
    guard = torch.full((n * d + 64,), 7.0, device=DEV)                        # behind the last row nothing is written
    guard_x = torch.full((n * d + 64,), 7.0, dtype=xt, device=DEV)
    h_out, x_out = guard[: n * d].view(n, d), guard_x[: n * d].view(n, d)
    for post in (w_post, None):
        add = norm(y.double()) * post.double() if post is not None else y.double()
        add = res * (add if gt is None else add * gt.double())
        ref_h = h.double() + add
        ref_x = norm(ref_h) * w_pre.double()
        B.halo_norm_glue(B.norm_shape(d, eps, ycode, xcode), h, y, post, gt, res, w_pre, h_out, x_out)
        off = 2.0 ** -18 * add.abs() + 2.0 ** -23 * ref_h.abs() + 1e-30
        assert ((h_out.double() - ref_h).abs() <= off).all()
        root = torch.sqrt(ref_h.square().mean(-1, keepdim=True) + eps)
        row = off.square().sum(-1, keepdim=True).sqrt() / (ref_h.square().sum(-1, keepdim=True).sqrt() + 1e-30)
        assert ((x_out.double() - ref_x).abs() <= off / root * w_pre.double().abs() + (2.0 ** -18 + row + u) * ref_x.abs() + 1e-30).all()
        assert (guard[n * d:] == 7).all() and (guard_x[n * d:] == 7).all()
    keep, x2 = h.clone(), torch.empty_like(x_out)
    B.halo_norm_glue(B.norm_shape(d, eps, ycode, xcode), keep, y, None, gt, res, w_pre, keep, x2)     # in place, the same bits
    assert torch.equal(keep, h_out) and torch.equal(x2, x_out)


# 2 to 32 tokens where the pairs of SMs take them (many long rows), next to the sizes where the line does
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,n,d", [(2, 5000, 2176), (16, 6144, 4096), (32, 4800, 2176), (17, 4737, 2176), (3, 18944, 4096), (9, 18945, 4096),
                                   (2, 18945, 4224), (32, 4736, 4096), (16, 4737, 2048), (33, 4737, 2048), (31, 11008, 11008)])
def test_products_of_few_tokens_through_many_long_rows(dtype, T, n, d):
    t, code, u = TYPES[dtype]
    g = gen(T + n + d)
    x = torch.randn((T, d), generator=g, device=DEV) * 2.0 ** torch.randint(-8, 8, (T, 1), generator=g, device=DEV)
    w = torch.randn((n, d), generator=g, device=DEV) * 2.0 ** torch.randint(-20, 3, (n, d // 32, 1), generator=g, device=DEV).expand(
        n, d // 32, 32).reshape(n, d)
    Qx, Sx = quantize(x)
    Qw, Sw = quantize(w)
    guard = torch.full((T * n + 64,), 7.0, dtype=t, device=DEV)
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
