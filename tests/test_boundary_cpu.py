"""CPU-side checks of the C-ABI library: it loads, exports what include/halo.h declares, validates arguments on
the host, and its host-only Assignment phase agrees with the oracle's Algorithm 3."""
import ctypes
import os
import re

import numpy as np
import pytest

from oracle import halo_ref as R
from paper_2601_11676_b200 import binding as B
from paper_2601_11676_b200 import build as halo_build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    halo_build.build()
    return B.lib()


def _declared():
    text = open(os.path.join(ROOT, "include", "halo.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(halo_[a-z_0-9]+)\s*\(", text)))


def test_every_declared_symbol_is_exported(lib):
    names = _declared()
    assert len(names) >= 15
    for n in names:
        assert hasattr(lib, n), f"{n} declared in halo.h but not exported"
    assert sorted(B.EXPORTS) == names


def test_status_strings(lib):
    assert B.status_string(0) == "ok"
    assert "aligned" in B.status_string(-3)
    assert "index" in B.status_message(B.DEV_BAD_INDEX)
    assert B.status_message(0) == "clean"


def test_plan_matches_oracle_algorithm3(lib):
    rng = np.random.default_rng(0)
    for _ in range(200):
        n = int(rng.integers(0, 9))
        G = int(rng.integers(1, 300))
        M = int(rng.integers(0, G + 1))
        rho = rng.uniform(0, 1, n).round(2)
        w = rng.integers(0, 6, n)
        if n and w.sum() == 0:
            w[0] = 1
        plan = B.Plan(G, rho, w, B.SEL_TOPK, G - M, 0.0, 5)
        order, thr, bnd = plan.describe(M)
        o_ref, t_ref, b_ref = R.plan(rho, w, M)
        assert order == o_ref.tolist() and thr == [int(v) for v in t_ref] and bnd == b_ref.tolist()
        plan.close()


def test_plan_paper_example(lib):
    plan = B.Plan(8, [0.0, 0.5, 0.1], [4, 4, 2], B.SEL_TOPK, 0, 0.0, 0)
    order, thr, bnd = plan.describe(8)
    assert order == [0, 2, 1] and bnd == [0, 3, 5, 8]


def test_plan_rejects_bad_arguments(lib):
    for args in [
        (8, [1.5], [1]), (8, [-0.1], [1]), (8, [0.1, 0.2], [0, 0]), (0, [0.1], [1]), (B.MAX_GROUPS + 1, [0.1], [1]),
        (8, [0.0] * (B.MAX_DEVICES + 1), [1] * (B.MAX_DEVICES + 1)),
    ]:
        with pytest.raises(B.HaloError):
            B.Plan(*args)
    with pytest.raises(B.HaloError):
        B.Plan(8, [0.1], [1], B.SEL_TOPK, 9)
    with pytest.raises(B.HaloError):
        B.Plan(8, [0.1], [1], B.SEL_THRESHOLD, 0, float("nan"))


def test_host_side_argument_checks_launch_nothing(lib):
    # NULL pointers / bad shapes are rejected before any CUDA call, so this runs without a GPU
    sh = B.ffn_shape(256, 688, 16, B.F32)
    rc = lib.halo_group_ffn(ctypes.byref(sh), None, None, 1, None, None, None, 0, None, None, 0, None, None)
    assert rc == -1
    bad = B.ffn_shape(250, 688, 16, B.F32)
    rc = lib.halo_group_ffn(ctypes.byref(bad), 16, 16, 1, 16, 16, None, 0, 16, None, 0, None, None)
    assert rc == -2
    bad = B.ffn_shape(256, 690, 16, B.F32)
    assert lib.halo_pack_weights(ctypes.byref(bad), 16, 16, 16, 16, None) == -2
    bad = B.ffn_shape(256, 688, 16, 7)
    assert lib.halo_pack_weights(ctypes.byref(bad), 16, 16, 16, 16, None) == -4
    rc = lib.halo_group_ffn(ctypes.byref(sh), 24, 16, 1, 16, 16, None, 0, 16, None, 0, None, None)
    assert rc == -3  # W_packed not 16-byte aligned
    ps = B.pred_shape(256, 32, 43, B.F32)
    assert B.halo_predict_workspace_bytes(ps, 1) == 4 * (32 + 43)
    rc = lib.halo_predict_groups(ctypes.byref(ps), 16, 16, 16, 1, 0, 16, 16, 8, None, None)
    assert rc == -8  # workspace too small
    assert lib.halo_merge_partials(None, None, 1, 1, 8, None, None) == -1
    assert lib.halo_select_groups(None, None, 0, 0, 0, None, None, None, None, None, None, None, None) == -1


def test_int4_entry_points_check_their_arguments_on_the_host(lib):
    """The int4 calls reject NULL pointers, shapes outside the format (d_model % 128), misaligned arrays and other
    element types before anything is launched."""
    sh = B.ffn_shape(256, 688, 16, B.BF16)
    assert lib.halo_quantize_rows_i4(256, 10, B.BF16, None, 16, 16, None) == -1
    assert lib.halo_quantize_rows_i4(200, 10, B.BF16, 16, 16, 16, None) == -2          # not a multiple of 128
    assert lib.halo_quantize_rows_i4(256, 0, B.BF16, 16, 16, 16, None) == -2
    assert lib.halo_quantize_rows_i4(256, 10, 5, 16, 16, 16, None) == -4
    assert lib.halo_quantize_rows_i4(256, 10, B.BF16, 16, 24, 16, None) == -3
    assert lib.halo_dequantize_weights_i4(ctypes.byref(sh), None, 16, None, None, 16, None, None) == -1
    assert lib.halo_dequantize_weights_i4(ctypes.byref(sh), 16, 16, 16, None, 16, None, None) == -1   # list without a count
    assert lib.halo_dequantize_weights_i4(ctypes.byref(sh), 16, 16, None, None, 24, None, None) == -3
    bad = B.ffn_shape(192, 688, 16, B.BF16)
    assert lib.halo_dequantize_weights_i4(ctypes.byref(bad), 16, 16, None, None, 16, None, None) == -2
    lm = B.lm_shape(256, 100, 16, B.BF16)
    assert lib.halo_group_lm_head_i4(ctypes.byref(lm), 16, 16, 16, 1, None, None, 16, None, None) == -1   # no status word
    assert lib.halo_group_lm_head_i4(ctypes.byref(lm), 16, 16, 16, 1, 16, None, 16, 16, None) == -1       # list without a count
    assert lib.halo_group_lm_head_i4(ctypes.byref(B.lm_shape(200, 100, 16, B.BF16)), 16, 16, 16, 1, None, None, 16, 16, None) == -2
    assert lib.halo_group_lm_head_i4(ctypes.byref(lm), 16, 24, 16, 1, None, None, 16, 16, None) == -3
    mh = B.mha_shape(256, 4, 32, 64, B.BF16)
    ptrs = [16] * 9
    assert lib.halo_mha_block_i4(ctypes.byref(mh), None, *ptrs[1:], 0, 16, 16, None, 0, 16, None, None) == -1
    assert lib.halo_mha_block_i4(ctypes.byref(mh), *ptrs, 64, 16, 16, None, 0, 16, None, None) == -1       # pos beyond the cache
    assert lib.halo_mha_block_i4(ctypes.byref(B.mha_shape(256, 4, 32, 64, B.F32)), *ptrs, 0, 16, 16, None, 0, 16, None, None) == -4
    assert lib.halo_mha_block_i4(ctypes.byref(B.mha_shape(192, 4, 32, 64, B.BF16)), *ptrs, 0, 16, 16, None, 0, 16, None, None) == -2
    assert lib.halo_mha_block_i4(ctypes.byref(mh), 16, 24, *ptrs[2:], 0, 16, 16, None, 0, 16, None, None) == -3
    big = B.ffn_shape(512, 1024, 128, B.BF16)
    assert B.halo_group_ffn_i4_workspace_bytes(big, 8) == 0                      # too few tokens for the tensor cores
    need = B.halo_group_ffn_i4_workspace_bytes(big, 64)
    assert need >= 3 * 1024 * 512 * 2                                             # one bf16 block + the FFN's own
    assert B.halo_group_ffn_i4_workspace_bytes(B.ffn_shape(512, 1024, 32, B.BF16), 64) == 0   # group size not taken
    assert lib.halo_group_ffn_i4_prompt(ctypes.byref(big), 16, 16, 16, 64, 16, 16, None, 0, 16, None, 0, None, None) == -8
    assert lib.halo_group_ffn_i4_prompt(ctypes.byref(big), 16, 16, 16, 64, 16, 16, None, 0, 16, 16, need - 1, None, None) == -8
    assert lib.halo_group_ffn_i4_prompt(ctypes.byref(big), None, 16, 16, 64, 16, 16, None, 0, 16, 16, need, None, None) == -1
    assert lib.halo_group_ffn_i4_prompt(ctypes.byref(big), 16, 16, 16, 64, 16, 16, None, 0, 16, 24, need, None, None) == -3
    out = ctypes.c_void_p()
    assert lib.halo_block_stack_create_i4(ctypes.byref(out), ctypes.byref(sh), ctypes.byref(mh), None, None, None, 1, None,
                                          None, None, None) == -1


def test_schedulers_match_oracle_and_feed_the_plan(lib):
    rng = np.random.default_rng(3)
    for _ in range(200):
        n = int(rng.integers(1, 9))
        m = rng.uniform(0.3, 6.3, n).round(1)
        c = rng.uniform(0.6, 1.8, n).round(1)
        Mt = float(rng.uniform(0.2, 1.0) * m.sum())
        assert np.allclose(B.halo_schedule_comp_greedy(m, c, Mt), R.comp_greedy(m, c, Mt), atol=1e-12)
        # the library solves the min-max problem exactly, the oracle bisects as Algorithm 2 does: two different
        # routes, which must meet as the oracle's tolerance shrinks
        r_lib = np.array(B.halo_schedule_min_max(m, c, Mt, 1e-3))
        assert np.allclose(r_lib, R.min_max(m, c, Mt, 1e-10), atol=1e-7)
        assert np.abs(r_lib - R.min_max(m, c, Mt, 1e-3)).max() <= 2e-3
        # invariants of the problem itself: ratios sum to 1, the loads r * Mt fit every budget (the allocation holds
        # the model exactly), and no choice of "full" devices gives a smaller slowest-device time
        assert abs(r_lib.sum() - 1.0) <= 1e-12
        load = r_lib * Mt
        assert (load <= m * (1 + 1e-9)).all()
        best = np.inf
        for mask in range(1 << n):                       # brute force: which devices are filled to their budget
            full = np.array([(mask >> i) & 1 for i in range(n)], dtype=bool)
            if full.all():
                T = (m / c).max() if abs(m.sum() - Mt) <= 1e-9 * Mt else np.inf
            else:
                T = (Mt - m[full].sum()) / c[~full].sum()
            if T < 0 or not np.isfinite(T):
                continue
            if (T * c[~full] <= m[~full] * (1 + 1e-12)).all() and (m[full] <= T * c[full] * (1 + 1e-12)).all():
                best = min(best, T)
        assert np.isclose((load / c).max(), best, rtol=1e-9)
    # ratios -> integer share weights -> Algorithm 3: a device with ratio 0 gets an empty chunk
    r = B.halo_schedule_comp_greedy([4, 5, 3], [2.0, 1.0, 3.0], 6.0)
    w = B.halo_ratios_to_share_weights(r)
    assert w == [32768, 0, 32768]
    plan = B.Plan(20, [0.1, 0.0, 0.3], w, B.SEL_TOPK, 4, 0.0, 0)
    order, _, bnd = plan.describe(16)
    assert order == [1, 0, 2] and bnd == [0, 0, 8, 16]
    for bad in [([1, 1], [1.0, 1.0], 3.0), ([1, -1], [1.0, 1.0], 0.5), ([1, 1], [1.0, 0.0], 0.5)]:
        with pytest.raises(B.HaloError):
            B.halo_schedule_min_max(*bad)
        with pytest.raises(B.HaloError):
            B.halo_schedule_comp_greedy(*bad)


def test_late_devices_match_the_oracle_and_feed_the_plan(lib):
    rng = np.random.default_rng(11)
    for _ in range(200):
        n = int(rng.integers(1, 9))
        units = rng.integers(0, 60, size=n)
        comp = rng.uniform(0.2, 4.0, size=n)
        tau, tc, to = float(rng.uniform(0.05, 2.0)), float(rng.uniform(0.0, 1.0)), float(rng.uniform(1.0, 20.0))
        assert B.halo_late_devices(units, comp, tau, tc, to) == R.late_devices(units, comp, tau, tc, to).tolist()
    # chunks of a plan -> late devices -> a plan in which they never arrive and hold the least critical groups
    loss, w = [0.0, 0.2, 0.1], [2, 1, 1]
    plan = B.Plan(40, loss, w, B.SEL_TOPK, 8, 0.0, 0)
    order, _, bnd = plan.describe(32)
    chunk = [0] * 3
    for pos, dev in enumerate(order):
        chunk[dev] = bnd[pos + 1] - bnd[pos]
    assert chunk == [16, 8, 8]
    late = B.halo_late_devices(chunk, [1.0, 2.0, 0.5], 1.0, 0.0, 10.0)   # busy 16, 4, 16 -> devices 0 and 2 are late
    assert late == [1, 0, 1]
    plan2 = B.Plan(40, [1.0 if l else r for l, r in zip(late, loss)], w, B.SEL_TOPK, 8, 0.0, 0)
    order2, thresh2, _ = plan2.describe(32)
    assert order2[0] == 1 and thresh2[0] == 1 << 32 and thresh2[2] == 1 << 32 and thresh2[1] < 1 << 32
    for bad in [([1, 2], [1.0, 0.0], 1.0, 0.0, 1.0), ([1, -1], [1.0, 1.0], 1.0, 0.0, 1.0), ([1], [1.0], -1.0, 0.0, 1.0)]:
        with pytest.raises(B.HaloError):
            B.halo_late_devices(*bad)


def test_attention_block_entry_points_check_their_arguments_on_the_host(lib):
    """Paged append / attention, the normalised residual and the mx4 calls refuse bad shapes, NULL and misaligned pointers,
    strides, element types and workspaces before anything is launched."""
    ref = ctypes.byref
    ok = B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16)
    bad_shapes = [B.paged_shape(8, 3, 64, 16, 10, 4, B.BF16), B.paged_shape(0, 0, 64, 16, 10, 4, B.BF16),
                  B.paged_shape(8, 2, 60, 16, 10, 4, B.BF16), B.paged_shape(8, 2, 272, 16, 10, 4, B.BF16),
                  B.paged_shape(8, 2, 64, 0, 10, 4, B.BF16), B.paged_shape(8, 2, 64, 16, 0, 4, B.BF16),
                  B.paged_shape(8, 2, 64, 16, 10, 0, B.BF16), B.paged_shape(8, 2, 64, 1 << 16, 10, 1 << 15, B.BF16),
                  B.paged_shape(2048, 2, 64, 16, 10, 4, B.BF16), B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16, 2040),
                  B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16, 2052)]

    def append(sh=ok, n_tok=3, n_seq=3, q=16, qs=512, k=16, ks=128, v=16, vs=128, pos=16, seq=None, table=16, inv=16, rot=64,
               q_out=16, qos=512, K=16, V=16):
        return lib.halo_paged_kv_append(ref(sh), n_tok, n_seq, q, qs, k, ks, v, vs, pos, seq, table, inv, rot, 0, q_out, qos, K,
                                        V, None, None)

    def attend(sh=ok, n_seq=3, q=16, qs=512, K=16, V=16, table=16, lens=16, scale=1.0, out=16, ws=None, wb=0):
        return lib.halo_paged_mha(ref(sh), n_seq, q, qs, K, V, table, lens, None, scale, out, None, ws, wb, None, None)

    for sh in bad_shapes:
        assert append(sh) == -2 and attend(sh) == -2 and B.halo_paged_mha_workspace_bytes(sh, 3) == 0
    assert append(B.paged_shape(8, 2, 64, 16, 10, 4, 2)) == -4 and attend(B.paged_shape(8, 2, 64, 16, 10, 4, -1)) == -4
    for kw in (dict(k=None), dict(v=None), dict(pos=None), dict(table=None), dict(K=None), dict(V=None), dict(q=None),
               dict(q_out=None), dict(inv=None)):
        assert append(**kw) == -1, kw
    for kw in (dict(n_tok=0), dict(n_seq=0), dict(n_seq=2), dict(rot=63), dict(rot=66), dict(rot=-2), dict(qs=504), dict(ks=120),
               dict(vs=-128), dict(qos=0)):
        assert append(**kw) == -2, kw
    for kw in (dict(q=24), dict(k=8), dict(v=18), dict(q_out=20), dict(K=24), dict(V=24), dict(qs=513), dict(ks=132), dict(qos=514)):
        assert append(**kw) == -3, kw
    for kw in (dict(q=None), dict(K=None), dict(V=None), dict(table=None), dict(lens=None), dict(out=None),
               dict(scale=float("nan")), dict(scale=float("inf"))):
        assert attend(**kw) == -1, kw
    for kw in (dict(n_seq=0), dict(n_seq=8193), dict(qs=511)):
        assert attend(**kw) == -2, kw
    for kw in (dict(q=24), dict(K=24), dict(V=24), dict(out=8), dict(qs=513)):
        assert attend(**kw) == -3, kw
    long = B.paged_shape(8, 2, 64, 16, 10000, 8192, B.BF16)
    need = B.halo_paged_mha_workspace_bytes(long, 1)
    assert need > 0
    assert attend(long, n_seq=1) == -8 and attend(long, n_seq=1, ws=16, wb=need - 1) == -8
    assert attend(long, n_seq=1, ws=24, wb=need) == -3

    def glue(sh=B.norm_shape(256, 1e-5, B.F32, B.BF16), n=2, h=16, y=16, w1=16, gate=16, gs=256, res=1.0, w2=16, ho=16, xo=16):
        return lib.halo_norm_glue(ref(sh), n, h, y, w1, gate, gs, res, w2, ho, xo, None)

    for kw in (dict(h=None), dict(ho=None), dict(xo=None), dict(y=None), dict(res=float("inf"))):
        assert glue(**kw) == -1, kw
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        assert glue(B.norm_shape(256, eps, B.F32, B.BF16)) == -1
    assert glue(B.norm_shape(256, 1e-5, 2, B.BF16)) == -4 and glue(B.norm_shape(256, 1e-5, B.F32, 3)) == -4
    for sh in (B.norm_shape(0, 1e-5, B.F32, B.BF16), B.norm_shape(252, 1e-5, B.F32, B.BF16), B.norm_shape(16392, 1e-5, B.F32, B.BF16)):
        assert glue(sh) == -2
    assert glue(n=0) == -2 and glue(gs=128) == -2
    for kw in (dict(h=24), dict(y=24), dict(w1=24), dict(gate=24), dict(w2=24), dict(ho=24), dict(xo=24), dict(gs=260)):
        assert glue(**kw) == -3, kw

    assert B.halo_mx4_scale_bytes(256, 129) == 2 * 2 * 512 and B.halo_mx4_scale_bytes(200, 1) == 0
    for fn in (lib.halo_quantize_rows_mx4, lib.halo_dequantize_rows_mx4):
        assert fn(256, 10, B.BF16, None, 16, 16, None) == -1 and fn(256, 10, B.BF16, 16, 16, None, None) == -1
        assert fn(200, 10, B.BF16, 16, 16, 16, None) == -2 and fn(256, 0, B.BF16, 16, 16, 16, None) == -2
        assert fn(256, 10, 5, 16, 16, 16, None) == -4 and fn(256, 10, B.F32, 16, 24, 16, None) == -3
    product = lambda d=256, t=1, n=8, p=(16, 16, 16, 16), dt=B.BF16, y=16: lib.halo_product_mx4(d, t, n, *p, dt, y, None, None)  # noqa: E731
    assert product(d=192) == -2 and product(t=0) == -2 and product(n=0) == -2 and product(t=(1 << 20) + 1) == -2
    assert product(dt=2) == -4 and product(y=None) == -1 and product(y=24) == -3
    for i in range(4):
        ptrs = [16] * 4
        ptrs[i] = None
        assert product(p=ptrs) == -1
        ptrs[i] = 24
        assert product(p=ptrs) == -3


def test_attention_block_binding_checks_tensors(lib):
    """The Python layer compares tensors with the shape before any address is passed on (CPU tensors are enough to see it)."""
    import torch
    f, i = torch.bfloat16, torch.int32
    sh = B.paged_shape(4, 2, 16, 16, 3, 2, B.BF16)
    K = torch.zeros((3, 2, 16, 16), dtype=f)
    q, kv, pos, table = torch.zeros((2, 4, 16), dtype=f), torch.zeros((2, 2, 16), dtype=f), torch.zeros(2, dtype=i), torch.zeros((2, 2), dtype=i)
    good = dict(shape=sh, q=q, k=kv, v=kv, pos=pos, seq_of_tok=None, block_table=table, inv_freq=None, interleaved=False, q_out=q, K_cache=K,
                V_cache=K)
    for name, t in (("k", kv.float()), ("k", kv[:, :1]), ("v", kv[:1]), ("q", q.transpose(1, 2)), ("q_out", None), ("pos", pos.long()),
                    ("pos", pos[:1]), ("block_table", table[:, :1]), ("inv_freq", torch.zeros(8)), ("K_cache", K[:2]), ("V_cache", K.float()),
                    ("seq_of_tok", table)):
        with pytest.raises(ValueError):
            B.halo_paged_kv_append(**{**good, name: t})
    with pytest.raises(ValueError):
        B.halo_paged_kv_append(**good)                                   # not on a GPU
    out = torch.zeros((2, 4, 16), dtype=f)
    good = dict(shape=sh, q=q, K_cache=K, V_cache=K, block_table=table, seq_len=pos, scale=1.0, out=out, workspace=None)
    for name, t in (("out", out[:1]), ("seq_len", pos[:1]), ("K_cache", K.transpose(2, 3)), ("workspace", torch.zeros(4)),
                    ("keep", torch.zeros(3, dtype=torch.uint8)), ("lse", torch.zeros(8, dtype=f)), ("q", q.flatten())):
        with pytest.raises(ValueError):
            B.halo_paged_mha(**{**good, name: t})
    ns, h, x = B.norm_shape(64, 1e-5, B.F32, B.BF16), torch.zeros((2, 64)), torch.zeros((2, 64), dtype=f)
    for y, w, gate, xo in ((x, None, None, x), (h, h[0], None, x), (h, None, x[:, :32], x), (h, None, None, x[:1])):
        with pytest.raises(ValueError):
            B.halo_norm_glue(ns, h, y, w, gate, 1.0, None, h, xo)
    Q, S = torch.zeros((5, 64), dtype=torch.uint8), torch.zeros(512, dtype=torch.uint8)
    for args in ((128, 5, B.BF16, torch.zeros((5, 128)), Q, S), (128, 5, B.F32, torch.zeros((5, 128)), Q[:4], S),
                 (128, 5, B.F32, torch.zeros((5, 128)), Q, S[:511]), (100, 5, B.F32, torch.zeros((5, 100)), Q, S)):
        with pytest.raises(ValueError):
            B.halo_quantize_rows_mx4(*args)
    with pytest.raises(ValueError):
        B.halo_product_mx4(128, 5, 5, Q, S, Q, S, B.F32, torch.zeros((5, 4)))


def test_append_in_place_needs_one_stride(lib):
    """q_out = q with another stride would write a token's row over rows that are still to be read."""
    sh = B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16)

    def append(n_tok, qs, qos):
        return lib.halo_paged_kv_append(ctypes.byref(sh), n_tok, 3, 16, qs, 16, 128, 16, 128, 16, None, 16, 16, 64, 0, 16, qos, 16, 16,
                                        None, None)

    assert append(3, 512, 520) == -1 and append(2, 768, 512) == -1


def test_attention_block_binding_refuses_a_shape_of_another_kind(lib):
    """Other shapes have as many bytes: a head's {d, vocab, group, type} would pass for a norm's {d, eps, type, type}."""
    import torch
    h, x = torch.zeros((2, 64)), torch.zeros((2, 64), dtype=torch.bfloat16)
    for sh in (B.lm_shape(64, 1 << 23, B.F32, B.BF16), B.ffn_shape(64, 1 << 23, B.F32, B.BF16), None, b"0123456789abcdef"):
        with pytest.raises(ValueError, match="another type"):
            B.halo_norm_glue(sh, h, None, None, None, 1.0, None, h, x)
        with pytest.raises(ValueError, match="another type"):
            B.halo_paged_mha(sh, x, x, x, x, x, 1.0, x, None)
    with pytest.raises(ValueError, match="GPU"):
        B.halo_norm_glue(B.norm_shape(64, 1e-5, B.F32, B.BF16), h, None, None, None, 1.0, None, h, x)
