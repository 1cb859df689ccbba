"""halo_paged_norm_append where elements or gains are large: the norm comes first, so that what is normed stays in range whatever it was.
Bounds of test_gpu_eight_bit_cache."""
import pytest
import torch

from tests.test_gpu_eight_bit_cache import Append

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["f32", "bf16", "8bit"])
@pytest.mark.parametrize("dh,rotary,inter", [(64, 64, False), (128, 64, True), (96, 24, False), (80, 80, False), (256, 256, False)])
@pytest.mark.parametrize("size,gain", [(1e15, 1e25), (1e18, 1e10), (1e19, 1.0), (1e25, 1.0), (5e37, 1.0), (1e-15, 1e20)])
def test_large_elements_and_gains(kind, dh, rotary, inter, size, gain):
    a = Append(kind, 4, 2, dh, 16, 25, rotary, inter, "both", 1.25)
    for x in (a.q, a.k):
        x *= size
    a.w_q, a.w_k = (a.w_q.float() * gain).to(a.t), (a.w_k.float() * gain).to(a.t)
    a.k[3], a.q[4, 1] = 0.0, 0.0
    a.check()
    assert torch.isfinite(a.q_out).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("dh,rotary", [(64, 64), (96, 24)])
def test_infinite_elements_leave_the_other_rows_alone(kind, dh, rotary):
    """x / infinity: NaN where x is infinite, and in what it is turned with, 0 elsewhere."""
    a, b = (Append(kind, 4, 2, dh, 16, 25, rotary, False, "both") for _ in range(2))
    a.k[7, 1, dh - 1] = float("inf")                 # behind the turned ones, or the second of a pair
    a.call(), b.call()
    k, _, _ = a.read()
    rest = torch.ones(25, 2, dtype=torch.bool, device=k.device)
    rest[7, 1] = False
    assert torch.equal(k[rest], b.read()[0][rest]) and torch.equal(a.q_out, b.q_out)
    row = k[7, 1]
    assert torch.isnan(row[dh - 1]) and int(torch.isnan(row).sum()) == (2 if rotary == dh else 1) and (row[~torch.isnan(row)] == 0).all()


@pytest.mark.parametrize("dh,rotary,inter", [(64, 64, False), (128, 64, True), (96, 24, False)])
@pytest.mark.parametrize("turn_scale", [1.0, 1.1386])
def test_cosines_and_sines_are_the_nearest(dh, rotary, inter, turn_scale):
    """Of pairs (1, 0) the turned ones are the cosine and the sine times turn_scale: rounded once, so equal to the 64-bit ones rounded but where
    the angle's own error (1e-10 for positions up to 10^5) meets a tie."""
    a = Append("f32", 4, 2, dh, 16, 200, rotary, inter, "none", turn_scale)
    a.q.zero_()
    first = slice(0, rotary, 2) if inter else slice(0, rotary // 2)
    second = slice(1, rotary, 2) if inter else slice(rotary // 2, rotary)
    a.q[..., first] = 1.0
    a.call()
    angle = a.pos.double()[:, None] * a.inv
    scale = torch.tensor(turn_scale, dtype=torch.float32).double().item()
    for part, want in ((first, torch.cos(angle) * scale), (second, torch.sin(angle) * scale)):
        got, want = a.q_out[..., part], want[:, None].expand(-1, 4, -1)
        assert ((got.double() - want).abs() <= 2.0 ** -24 * want.abs() + 1e-10).all()
        assert (got == want.float()).float().mean() > 0.99
