"""Refusals of the entry points for prompts and 8-bit rows: nothing is launched, so they run without a GPU."""
import ctypes

import pytest
import torch

from paper_2601_11676_b200 import binding as B
from paper_2601_11676_b200 import build as halo_build


@pytest.fixture(scope="module")
def lib():
    halo_build.build()
    return B.lib()


OK = B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16)
BAD = [B.paged_shape(8, 3, 64, 16, 10, 4, B.BF16), B.paged_shape(8, 2, 60, 16, 10, 4, B.BF16), B.paged_shape(8, 2, 64, 0, 10, 4, B.BF16),
       B.paged_shape(8, 2, 272, 16, 10, 4, B.BF16), B.paged_shape(8, 2, 64, 1 << 16, 10, 1 << 15, B.BF16)]
ref = ctypes.byref
ODD = 24     # an address off 16 bytes


def append(lib, sh=OK, n_tok=2, n_seq=2, q=16, qs=512, k=16, ks=128, v=16, vs=128, wq=16, wk=16, eps=1e-6, pos=16, seq=16, table=16,
           inv=16, rot=64, inter=0, ts=1.0, qo=32, qos=512, K=16, V=16, Ks=None, Vs=None):
    return lib.halo_paged_norm_append(ref(sh), n_tok, n_seq, q, qs, k, ks, v, vs, wq, wk, eps, pos, seq, table, inv, rot, inter, ts, qo,
                                      qos, K, V, Ks, Vs, None, None)


def read(lib, sh=OK, n_tok=2, n_seq=2, pos=16, seq=16, table=16, K=16, V=16, Ks=None, Vs=None, k=16, ks=128, v=16, vs=128):
    return lib.halo_paged_kv_read(ref(sh), n_tok, n_seq, pos, seq, table, K, V, Ks, Vs, k, ks, v, vs, None, None)


def token(lib, sh=OK, n_seq=2, q=16, qs=512, K=16, V=16, Ks=16, Vs=16, table=16, lens=16, scale=1.0, out=16, ws=16, wb=1 << 40):
    return lib.halo_paged_mha_f8(ref(sh), n_seq, q, qs, K, V, Ks, Vs, table, lens, None, scale, out, None, ws, wb, None, None)


def prompt(lib, sh=OK, n_tok=2, n_seq=2, q=16, qs=512, start=16, K=16, V=16, Ks=None, Vs=None, table=16, lens=16, scale=1.0, out=32,
           ws=16, wb=1 << 40):
    return lib.halo_paged_prompt_mha(ref(sh), n_tok, n_seq, q, qs, start, K, V, Ks, Vs, table, lens, None, scale, out, None, ws, wb, None,
                                     None)


def test_shapes_and_types(lib):
    for sh in BAD:
        assert append(lib, sh) == -2 and read(lib, sh) == -2 and token(lib, sh) == -2 and prompt(lib, sh) == -2
        assert B.halo_paged_mha_f8_workspace_bytes(sh, 2) == 0 and B.halo_paged_prompt_mha_workspace_bytes(sh, 2, 2) == 0
    for call in (append, read, token, prompt):
        assert call(lib, B.paged_shape(8, 2, 64, 16, 10, 4, 2)) == -4
    f32 = B.paged_shape(8, 2, 64, 16, 10, 4, B.F32)       # 8-bit rows go with bf16
    assert append(lib, f32, Ks=16, Vs=16) == -4 and read(lib, f32, Ks=16, Vs=16) == -4 and token(lib, f32) == -4
    assert prompt(lib, f32, Ks=16, Vs=16) == -4 and B.halo_paged_mha_f8_workspace_bytes(f32, 2) == 0
    odd_pages = B.paged_shape(8, 2, 64, 16, 10, 4, B.BF16, 2056)      # pages of 8-bit rows begin on 16 bytes
    assert append(lib, odd_pages, Ks=16, Vs=16) == -2 and token(lib, odd_pages) == -2 and prompt(lib, odd_pages, Ks=16, Vs=16) == -2


@pytest.mark.parametrize("call,needed", [
    (append, ["k", "v", "pos", "table", "K", "V", "inv", "q", "qo"]), (read, ["pos", "table", "K", "V", "k", "v"]),
    (token, ["q", "K", "V", "Ks", "Vs", "table", "lens", "out"]), (prompt, ["q", "start", "K", "V", "table", "lens", "out"])])
def test_missing_pointers(lib, call, needed):
    for name in needed:
        assert call(lib, **{name: None}) == -1, name


@pytest.mark.parametrize("call,aligned", [
    (append, ["q", "k", "v", "wq", "wk", "qo", "K", "V"]), (read, ["K", "V", "k", "v"]), (token, ["q", "K", "V", "Ks", "Vs", "out"]),
    (prompt, ["q", "K", "V", "out", "ws"])])
def test_alignment(lib, call, aligned):
    for name in aligned:
        assert call(lib, **{name: ODD}) == -3, name


def test_counts_strides_and_numbers(lib):
    for kw in (dict(n_tok=0), dict(n_tok=(1 << 24) + 1), dict(n_seq=0), dict(rot=63), dict(rot=66), dict(rot=-2), dict(qs=504),
               dict(ks=120), dict(vs=120), dict(qos=504), dict(seq=None, n_tok=3)):
        assert append(lib, **kw) == -2, kw
    for kw in (dict(qs=513), dict(ks=129), dict(qos=516)):
        assert append(lib, **kw) == -3, kw
    nan, inf = float("nan"), float("inf")
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=nan), dict(eps=inf), dict(ts=0.0), dict(ts=nan), dict(ts=inf), dict(ts=-1.0),
               dict(Ks=16), dict(Vs=16), dict(q=16, qo=16, qs=512, qos=520)):
        assert append(lib, **kw) == -1, kw
    assert append(lib, wq=None, wk=None, eps=0.0, n_tok=0) == -2      # eps is of no norm then: the count is what is refused
    assert read(lib, n_tok=0) == -2 and read(lib, ks=120) == -2 and read(lib, vs=129) == -3 and read(lib, Ks=16) == -1
    assert token(lib, n_seq=0) == -2 and token(lib, n_seq=8193) == -2 and token(lib, qs=504) == -2 and token(lib, scale=nan) == -1
    for kw in (dict(n_tok=0), dict(n_tok=(1 << 20) + 1), dict(n_seq=0), dict(n_seq=8193), dict(qs=504)):
        assert prompt(lib, **kw) == -2, kw
    assert prompt(lib, qs=516) == -3 and prompt(lib, scale=inf) == -1 and prompt(lib, Ks=16) == -1 and prompt(lib, Vs=16) == -1
    assert prompt(lib, out=16) == -1                                    # in place: other thread blocks still read the queries


def test_workspaces(lib):
    long = B.paged_shape(8, 2, 64, 16, 10000, 8192, B.BF16)
    need = B.halo_paged_mha_f8_workspace_bytes(long, 1)
    assert need > 0 and token(lib, long, n_seq=1, wb=need - 1) == -8 and token(lib, long, n_seq=1, ws=None) == -8
    for sh in (OK, long, B.paged_shape(8, 2, 64, 16, 10, 4, B.F32)):
        need = B.halo_paged_prompt_mha_workspace_bytes(sh, 5, 2)
        assert need > 0 and prompt(lib, sh, n_tok=5, wb=need - 1) == -8 and prompt(lib, sh, n_tok=5, ws=None) == -8
    assert B.halo_paged_prompt_mha_workspace_bytes(OK, 0, 2) == 0 and B.halo_paged_prompt_mha_workspace_bytes(OK, 2, 0) == 0


def test_tensors_that_do_not_fit_are_refused_by_name(lib):
    H, Hk, dh, page, n = 4, 2, 16, 16, 3
    sh = B.paged_shape(H, Hk, dh, page, n, 2, B.BF16)
    bf, u8, i32 = dict(dtype=torch.bfloat16), dict(dtype=torch.uint8), dict(dtype=torch.int32)
    cache, codes, scale = torch.zeros(n, Hk, page, dh, **bf), torch.zeros(n, Hk, page, dh, **u8), torch.zeros(n, Hk, page, **u8)
    q, k, table, lens, ws = torch.zeros(5, H, dh, **bf), torch.zeros(5, Hk, dh, **bf), torch.zeros(1, 2, **i32), torch.zeros(1, **i32), torch.zeros(64, **u8)
    pos, inv, w = torch.zeros(5, **i32), torch.zeros(8, dtype=torch.float64), torch.zeros(dh, **bf)
    good = dict(shape=sh, q=q, k=k, v=k, w_q=w, w_k=w, eps=1e-6, pos=pos, seq_of_tok=pos, block_table=table, inv_freq=inv, interleaved=False,
                turn_scale=1.0, q_out=q.clone(), K_cache=codes, V_cache=codes.clone(), K_scale=scale, V_scale=scale.clone())
    for name, t in dict(q=q.float(), k=k[:4], w_q=w[:8], w_k=w.float(), pos=pos.long(), block_table=table[:, :1].contiguous(),
                        inv_freq=inv.float(), K_cache=cache, V_cache=codes[:2], K_scale=scale[:2], V_scale=scale.int(), q_out=None,
                        shape=B.norm_shape(64, 1e-5, B.F32, B.BF16)).items():
        with pytest.raises(ValueError):
            B.halo_paged_norm_append(**{**good, name: t})
    with pytest.raises(ValueError, match="on a GPU"):
        B.halo_paged_norm_append(**good)
    with pytest.raises(ValueError):                                     # 8-bit caches without their scales
        B.halo_paged_norm_append(**{**good, "K_scale": None, "V_scale": None})
    good = dict(shape=sh, pos=pos, seq_of_tok=pos, block_table=table, K_cache=codes, V_cache=codes, k_out=k, v_out=k.clone(), K_scale=scale, V_scale=scale)
    for name, t in dict(pos=pos[:2], k_out=k.float(), v_out=k[:, :1], K_cache=cache, K_scale=scale.view(-1)[1:]).items():
        with pytest.raises(ValueError):
            B.halo_paged_kv_read(**{**good, name: t})
    one = torch.zeros(1, H, dh, **bf)
    good = dict(shape=sh, q=one, K_cache=codes, V_cache=codes, K_scale=scale, V_scale=scale, block_table=table, seq_len=lens, scale=1.0,
                out=one.clone(), workspace=ws)
    for name, t in dict(q=one.float(), K_cache=cache, V_scale=scale[:1], seq_len=lens.long(), out=q, workspace=ws.int()).items():
        with pytest.raises(ValueError):
            B.halo_paged_mha_f8(**{**good, name: t})
    good = dict(shape=sh, q=q, q_start=torch.zeros(2, **i32), K_cache=cache, V_cache=cache, block_table=table, seq_len=lens, scale=1.0,
                out=q.clone(), workspace=ws)
    for name, t in dict(q=q[:, :2], q_start=lens, K_cache=codes, V_cache=cache[:1], block_table=table.long(), seq_len=lens.float(),
                        out=q[:4], workspace=ws.int(), K_scale=scale, keep=lens, lse=torch.zeros(5, H, **bf)).items():
        with pytest.raises(ValueError):
            B.halo_paged_prompt_mha(**{**good, name: t})
    with pytest.raises(ValueError, match="on a GPU"):
        B.halo_paged_prompt_mha(**good)
