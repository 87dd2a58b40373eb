"""The token operators refuse what they cannot do, before any launch (CPU: the
C entry points see addresses that nothing reads)."""
import ctypes as C

import pytest
import torch

from paper_2608_11226_gb300 import build, pe

A = 0x10000  # a non-null, aligned address; no refused call touches it


@pytest.fixture(scope="module")
def L():
    build.build()
    return pe.lib()


def cache(**kw):
    d = dict(k=A, v=A, table=A, n_pages=8, page_stride=16 * 2 * 64, slot_stride=2 * 64, head_stride=64, table_stride=4,
             n_seqs=2, max_pages=4, page_size=16, n_heads=2, head_dim=64, dtype=pe.PE_BF16)
    d.update(kw)
    return pe.KVCacheDesc(**d)


def tokens(**kw):
    d = dict(pos=A, rot=A, q=A, q_out=A, k=A, v=A, n_tokens=3, max_pos=64, q_token_stride=256, q_head_stride=64,
             q_out_token_stride=256, q_out_head_stride=64, k_token_stride=128, k_head_stride=64, v_token_stride=128,
             v_head_stride=64, n_q_heads=4, rot_dim=64, interleaved=0)
    d.update(kw)
    return pe.KVTokens(**d)


BAD_CACHES = [dict(k=None), dict(v=None), dict(table=None), dict(k=A + 2), dict(v=A + 8), dict(n_pages=0),
              dict(n_pages=1 << 31), dict(page_stride=12), dict(slot_stride=-8), dict(head_stride=3), dict(table_stride=3),
              dict(n_seqs=-1), dict(max_pages=0), dict(max_pages=1 << 28), dict(page_size=0), dict(page_size=1 << 17),
              dict(n_heads=0), dict(head_dim=96), dict(head_dim=0), dict(dtype=pe.PE_F32), dict(dtype=3)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_cache_refused(L, bad):
    c = cache(**bad)
    assert L.pe_kv_append(C.byref(c), C.byref(tokens()), None) == pe.PE_EINVAL
    assert L.pe_last_error()
    assert L.pe_decode_attn_workspace_bytes(C.byref(c), 4) == -1
    assert L.pe_decode_attn(C.byref(c), A, 256, 64, 4, A, 1.0, 0, A, 256, 64, None, A, 1 << 40, None) == pe.PE_EINVAL


@pytest.mark.parametrize("bad", [dict(pos=None), dict(rot=None), dict(q_out=None), dict(k=None), dict(v=None),
                                 dict(n_tokens=-1), dict(n_tokens=1 << 31), dict(max_pos=0), dict(q_token_stride=4),
                                 dict(q_head_stride=-64), dict(q_out_token_stride=1), dict(k_head_stride=7),
                                 dict(v_token_stride=65), dict(n_q_heads=0), dict(rot_dim=24), dict(rot_dim=80),
                                 dict(rot_dim=-16), dict(q=A + 2), dict(k=A + 4), dict(rot=A + 4)])
def test_append_refused(L, bad):
    assert L.pe_kv_append(C.byref(cache()), C.byref(tokens(**bad)), None) == pe.PE_EINVAL
    assert L.pe_last_error()


def test_append_null_and_empty(L):
    assert L.pe_kv_append(None, C.byref(tokens()), None) == pe.PE_EINVAL
    assert L.pe_kv_append(C.byref(cache()), None, None) == pe.PE_EINVAL
    assert L.pe_kv_append(C.byref(cache()), C.byref(tokens(n_tokens=0)), None) == pe.PE_OK


DECODE = dict(q=A, qs=256, qh=64, hq=4, lens=A, scale=0.125, window=0, out=A, os=256, oh=64, lse=None, ws=A, nb=1 << 40)


@pytest.mark.parametrize("bad", [dict(q=None), dict(lens=None), dict(out=None), dict(qs=100), dict(qh=-8), dict(os=2),
                                 dict(oh=12), dict(hq=0), dict(hq=3), dict(scale=float("nan")),
                                 dict(scale=float("inf")), dict(window=-1), dict(q=A + 2), dict(out=A + 8)])
def test_decode_refused(L, bad):
    d = dict(DECODE, **bad)
    assert L.pe_decode_attn(C.byref(cache()), *d.values(), None) == pe.PE_EINVAL
    assert L.pe_last_error()


def test_decode_workspace_refused(L):
    c = cache()
    need = L.pe_decode_attn_workspace_bytes(C.byref(c), 4)
    assert need >= 0 and L.pe_decode_attn_workspace_bytes(C.byref(c), 3) == -1
    if need:
        for bad in (dict(ws=None), dict(nb=need - 1), dict(ws=A + 16)):
            d = dict(DECODE, **bad)
            assert L.pe_decode_attn(C.byref(c), *d.values(), None) == pe.PE_EINVAL
    empty = cache(n_seqs=0, table=None)
    assert L.pe_decode_attn(C.byref(empty), *DECODE.values(), None) == pe.PE_OK


LOGP = dict(x=A, dtype=pe.PE_BF16, n=3, V=100, rs=104, tok=A, scale=1.0, logp=A, ent=A, lse=A, k=5, tl=A, ti=A)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=A + 1), dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=1 << 31),
                                 dict(V=0), dict(V=(1 << 30) + 1), dict(rs=99), dict(tok=None), dict(scale=0.0),
                                 dict(scale=-1.0), dict(scale=float("nan")), dict(scale=1e5), dict(k=-1), dict(k=33),
                                 dict(V=4, k=5), dict(tl=None), dict(ti=None),
                                 dict(tok=None, logp=None, ent=None, lse=None, k=0)])
def test_logp_refused(L, bad):
    assert L.pe_token_logp(*dict(LOGP, **bad).values(), None) == pe.PE_EINVAL
    assert L.pe_last_error()


GRAD = dict(x=A, dtype=pe.PE_F32, n=3, V=100, rs=104, tok=A, scale=1.0, lse=A, ent=A, g=A, ge=A, dx=2 * A, ds=104)


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=A + 2), dict(dtype=7), dict(n=-2), dict(V=0), dict(rs=50),
                                 dict(tok=None), dict(scale=float("inf")), dict(lse=None), dict(ent=None),
                                 dict(g=None, ge=None), dict(dx=None), dict(dx=2 * A + 1), dict(ds=99),
                                 dict(dx=A, ds=108)])
def test_grad_refused(L, bad):
    assert L.pe_token_logp_grad(*dict(GRAD, **bad).values(), None) == pe.PE_EINVAL
    assert L.pe_last_error()


def test_no_rows_is_no_error(L):
    assert L.pe_token_logp(*dict(LOGP, n=0).values(), None) == pe.PE_OK
    assert L.pe_token_logp_grad(*dict(GRAD, n=0).values(), None) == pe.PE_OK


def test_binding_refuses_host_and_odd_tensors():
    k = torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        pe.KVCache(k, k.clone(), torch.zeros(2, 2, dtype=torch.int32))  # host memory
    with pytest.raises(ValueError):
        pe.token_logp(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32), torch.zeros(2))
    with pytest.raises(ValueError):
        pe.token_logp_grad(torch.zeros(2, 8), None, torch.zeros(2), torch.zeros(2, 8))


def test_rotation_table():
    t = pe.rot_table(5, 8, base=100.0, device="cpu")
    assert t.shape == (5, 8) and t.dtype == torch.float32
    f = 100.0 ** (-torch.arange(4, dtype=torch.float64) / 4)
    assert torch.equal(t[3], torch.cat([torch.cos(3 * f), torch.sin(3 * f)]).float())
