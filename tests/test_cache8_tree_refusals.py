"""The 8-bit cache's calls and those of drafted tokens refuse what they cannot
do, before any launch (CPU: the C entry points see addresses that nothing
reads; the binding sees host tensors that pass for device tensors)."""
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
             n_seqs=2, max_pages=4, page_size=16, n_heads=2, head_dim=64, dtype=pe.PE_E4M3)
    d.update(kw)
    return pe.KVCacheDesc(**d)


def scales(**kw):
    return pe.KVScales(**{**dict(k=A, v=A, page_stride=32, slot_stride=2, head_stride=1), **kw})


def tokens(**kw):
    d = dict(pos=A, rot=A, q=A, q_out=A, k=A, v=A, n_tokens=3, max_pos=64, q_token_stride=256, q_head_stride=64,
             q_out_token_stride=256, q_out_head_stride=64, k_token_stride=128, k_head_stride=64, v_token_stride=128,
             v_head_stride=64, n_q_heads=4, rot_dim=64, interleaved=0)
    d.update(kw)
    return pe.KVTokens(**d)


def tree(**kw):
    d = dict(q=A, out=A, lse=A, lens=A, mask=A, q_seq_stride=1024, q_node_stride=256, q_head_stride=64, out_seq_stride=1024,
             out_node_stride=256, out_head_stride=64, mask_stride=4, n_nodes=4, n_q_heads=4, dtype=pe.PE_BF16)
    d.update(kw)
    return pe.TreeQueries(**d)


def ref(x):
    return None if x is None else C.byref(x)


def calls(L, c, s, dtype=pe.PE_BF16):
    """Every call over the cache, with arguments that are otherwise in order."""
    return [L.pe_kv_append_at(ref(c), ref(s), ref(tokens()), A, dtype, None),
            L.pe_decode_attn8(ref(c), ref(s), dtype, A, 256, 64, 4, A, 0.125, 0, A, 256, 64, None, A, 1 << 40, None),
            L.pe_tree_attn(ref(c), ref(s), ref(tree(dtype=dtype)), 0.125, 0, A, 1 << 40, None),
            L.pe_kv_move(ref(c), ref(s), A, 4, A, 4, 4, None)]


BAD_CACHES = [dict(k=None), dict(v=None), dict(table=None), dict(k=A + 8), dict(n_pages=0), dict(n_pages=1 << 31),
              dict(page_stride=24), dict(slot_stride=8), dict(head_stride=40), dict(table_stride=3), dict(n_seqs=-1),
              dict(max_pages=0), dict(max_pages=1 << 28), dict(page_size=0), dict(n_heads=0), dict(head_dim=96),
              dict(dtype=pe.PE_F32), dict(dtype=4), dict(dtype=-1)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_cache_refused(L, bad):
    c = cache(**bad)
    assert calls(L, c, scales()) == [pe.PE_EINVAL] * 4
    assert L.pe_last_error()
    assert L.pe_decode_attn8_workspace_bytes(C.byref(c), 4) == -1
    assert L.pe_tree_attn_workspace_bytes(C.byref(c), 4, 4) == -1


@pytest.mark.parametrize("bad", [None, dict(k=None), dict(v=None), dict(page_stride=-1), dict(slot_stride=-2),
                                 dict(head_stride=1 << 50)])
def test_scales_refused(L, bad):
    assert calls(L, cache(), None if bad is None else scales(**bad)) == [pe.PE_EINVAL] * 4


def test_scales_of_a_16_bit_cache_refused(L):
    c = cache(dtype=pe.PE_BF16)
    assert calls(L, c, scales()) == [pe.PE_EINVAL] * 4
    assert calls(L, c, None, dtype=pe.PE_F16)[:3] == [pe.PE_EINVAL] * 3  # another type than the cache's
    assert L.pe_decode_attn8_workspace_bytes(C.byref(c), 4) == -1


@pytest.mark.parametrize("dtype", [pe.PE_F32, pe.PE_E4M3, 9])
def test_dtype_refused(L, dtype):
    assert calls(L, cache(), scales(), dtype=dtype)[:3] == [pe.PE_EINVAL] * 3


def test_the_16_bit_calls_refuse_codes(L):
    c = cache()
    assert L.pe_kv_append(C.byref(c), C.byref(tokens()), None) == pe.PE_EINVAL
    assert L.pe_decode_attn_workspace_bytes(C.byref(c), 4) == -1
    assert L.pe_decode_attn(C.byref(c), A, 256, 64, 4, A, 1.0, 0, A, 256, 64, None, A, 1 << 40, None) == pe.PE_EINVAL


@pytest.mark.parametrize("bad", [dict(pos=None), dict(rot=None), dict(q_out=None), dict(k=None), dict(n_tokens=-1),
                                 dict(max_pos=0), dict(q_token_stride=4), dict(v_token_stride=65), dict(n_q_heads=0),
                                 dict(rot_dim=24), dict(rot_dim=80), dict(k=A + 4)])
def test_append_refused(L, bad):
    assert L.pe_kv_append_at(C.byref(cache()), C.byref(scales()), C.byref(tokens(**bad)), A, pe.PE_BF16, None) == pe.PE_EINVAL
    assert L.pe_kv_append_at(C.byref(cache()), C.byref(scales()), None, A, pe.PE_BF16, None) == pe.PE_EINVAL


TREE_BAD = [dict(q=None), dict(out=None), dict(lens=None), dict(mask=None), dict(q=A + 2), dict(out=A + 8), dict(mask=A + 4),
            dict(q_seq_stride=4), dict(q_node_stride=-8), dict(q_head_stride=65), dict(out_seq_stride=1), dict(out_node_stride=12),
            dict(out_head_stride=-64), dict(mask_stride=-1), dict(n_nodes=-1), dict(n_nodes=65), dict(n_q_heads=0), dict(n_q_heads=3)]


@pytest.mark.parametrize("bad", TREE_BAD)
def test_tree_refused(L, bad):
    assert L.pe_tree_attn(C.byref(cache()), C.byref(scales()), C.byref(tree(**bad)), 0.125, 0, A, 1 << 40, None) == pe.PE_EINVAL
    assert L.pe_last_error()


@pytest.mark.parametrize("scale,window", [(float("nan"), 0), (float("inf"), 0), (1.0, -1), (1.0, 63)])
def test_tree_scale_and_window_refused(L, scale, window):
    assert L.pe_tree_attn(C.byref(cache()), C.byref(scales()), C.byref(tree()), scale, window, A, 1 << 40, None) == pe.PE_EINVAL


def test_workspaces(L):
    c, s = cache(), scales()
    assert L.pe_tree_attn_workspace_bytes(C.byref(c), 4, 3) == -1 and L.pe_tree_attn_workspace_bytes(C.byref(c), 65, 4) == -1
    need = L.pe_tree_attn_workspace_bytes(C.byref(c), 4, 4)
    need8 = L.pe_decode_attn8_workspace_bytes(C.byref(c), 4)
    assert need > 0 and need8 > 0
    for ws, more in ((None, 0), (A, -1), (A + 16, 0)):
        assert L.pe_tree_attn(C.byref(c), C.byref(s), C.byref(tree()), 1.0, 0, ws, need + more, None) == pe.PE_EINVAL
        assert L.pe_decode_attn8(C.byref(c), C.byref(s), pe.PE_BF16, A, 256, 64, 4, A, 1.0, 0, A, 256, 64, None, ws, need8 + more,
                                 None) == pe.PE_EINVAL


DECODE = dict(q=A, qs=256, qh=64, hq=4, lens=A, scale=0.125, window=0, out=A, os=256, oh=64, lse=None, ws=A, nb=1 << 40)


@pytest.mark.parametrize("bad", [dict(q=None), dict(lens=None), dict(out=None), dict(qs=100), dict(qh=-8), dict(os=2), dict(oh=12),
                                 dict(hq=0), dict(hq=3), dict(scale=float("nan")), dict(window=-1), dict(q=A + 2), dict(out=A + 8)])
def test_decode8_refused(L, bad):
    assert L.pe_decode_attn8(C.byref(cache()), C.byref(scales()), pe.PE_BF16, *dict(DECODE, **bad).values(), None) == pe.PE_EINVAL


@pytest.mark.parametrize("a", [(None, 4, A, 4, 4), (A, 4, None, 4, 4), (A, 3, A, 4, 4), (A, 4, A, 3, 4), (A, 4, A, 4, -1),
                               (A, 100, A, 100, 65)])
def test_move_refused(L, a):
    assert L.pe_kv_move(C.byref(cache()), C.byref(scales()), *a, None) == pe.PE_EINVAL


def test_nothing_to_do_is_no_error(L):
    empty, s = cache(n_seqs=0, table=None), scales()
    assert L.pe_kv_append_at(C.byref(cache()), C.byref(s), C.byref(tokens(n_tokens=0)), None, pe.PE_F16, None) == pe.PE_OK
    assert L.pe_tree_attn(C.byref(empty), C.byref(s), C.byref(tree()), 1.0, 0, A, 1 << 40, None) == pe.PE_OK
    assert L.pe_tree_attn(C.byref(cache()), C.byref(s), C.byref(tree(n_nodes=0)), 1.0, 0, A, 1 << 40, None) == pe.PE_OK
    assert L.pe_decode_attn8(C.byref(empty), C.byref(s), pe.PE_BF16, *DECODE.values(), None) == pe.PE_OK
    assert L.pe_kv_move(C.byref(empty), C.byref(s), A, 4, A, 4, 4, None) == pe.PE_OK
    assert L.pe_kv_move(C.byref(cache()), C.byref(s), None, 4, None, 4, 0, None) == pe.PE_OK


# ---------------------------------------------------------------------------
# the binding
# ---------------------------------------------------------------------------
class OnDevice(torch.Tensor):
    """A host tensor that says it is on device 0."""
    is_cuda = True

    def get_device(self):
        return 0


class Elsewhere(torch.Tensor):
    """A host tensor that says it is on device 1."""
    is_cuda = True

    def get_device(self):
        return 1


def z(*shape, dtype=torch.float32, on=OnDevice):
    return torch.zeros(shape, dtype=dtype).as_subclass(on)


BF, I32, I64, U8, E4M3 = torch.bfloat16, torch.int32, torch.int64, torch.uint8, torch.float8_e4m3fn


def parts(eight=True):
    d = dict(k=z(6, 4, 2, 64, dtype=E4M3 if eight else BF), v=z(6, 4, 2, 64, dtype=E4M3 if eight else BF), table=z(3, 2, dtype=I32))
    return dict(d, k_scale=z(6, 4, 2, dtype=U8), v_scale=z(6, 4, 2, dtype=U8)) if eight else d


@pytest.fixture
def on_device_0(monkeypatch):
    """Device 0 is current, and no C call is made."""
    class Library:
        def __getattr__(self, name):
            def call(*a):
                raise AssertionError("the C library was called")
            return call

    monkeypatch.setattr(pe, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(pe, "_stream_of", lambda *a: 0)
    monkeypatch.setattr(pe, "lib", Library)


def scale(shape=(6, 4, 2), dtype=U8):
    return z(*shape, dtype=dtype)


@pytest.mark.parametrize("bad", [dict(k_scale=None), dict(v_scale=None), dict(k_scale=scale((6, 4))),
                                 dict(k_scale=scale((6, 4, 3)), v_scale=scale((6, 4, 3))),
                                 dict(k_scale=scale(dtype=torch.float32), v_scale=scale(dtype=torch.float32)),
                                 dict(k_scale=scale(dtype=torch.int8)), dict(v_scale=scale((6, 2, 4)).transpose(1, 2)),
                                 dict(k_scale=scale((6, 4, 1)).expand(6, 4, 2), v_scale=scale((6, 4, 1)).expand(6, 4, 2)),
                                 dict(k_scale=z(6, 4, 2, dtype=U8, on=Elsewhere)), dict(k=z(6, 4, 2, 64, dtype=BF)),
                                 dict(k=z(6, 4, 2, 64, dtype=BF), v=z(6, 4, 2, 64, dtype=BF)),
                                 dict(k=z(6, 4, 2, 64, dtype=torch.float8_e5m2), v=z(6, 4, 2, 64, dtype=torch.float8_e5m2))])
def test_caches_that_are_refused(bad):
    with pytest.raises(ValueError):
        pe.KVCache(**dict(parts(), **bad))


def test_scales_of_either_type():
    e8 = dict(k_scale=scale(dtype=torch.float8_e8m0fnu), v_scale=scale(dtype=torch.float8_e8m0fnu))
    for more in ({}, e8, dict(k_scale=scale((6, 2, 4)).transpose(1, 2), v_scale=scale((6, 2, 4)).transpose(1, 2))):
        c = pe.KVCache(**dict(parts(), **more))
        assert c.eight and c._desc.dtype == pe.PE_E4M3
        assert (c._scale_desc.page_stride, c._scale_desc.slot_stride * c._scale_desc.head_stride) in ((8, 2), (8, 4))


CALLS = {
    "append": (lambda eight=True, **a: pe.kv_append(pe.KVCache(**parts(eight)), **a),
               lambda: dict(k=z(3, 2, 64, dtype=BF), v=z(3, 2, 64, dtype=BF), positions=z(3, dtype=I32), seqs=z(3, dtype=I32),
                            q=z(3, 4, 64, dtype=BF), q_out=z(3, 4, 64, dtype=BF), rot=z(8, 64), slots=z(3, dtype=I32))),
    "decode": (lambda eight=True, **a: pe.decode_attn(pe.KVCache(**parts(eight)), **a),
               lambda: dict(q=z(3, 4, 64, dtype=BF), lens=z(3, dtype=I32), out=z(3, 4, 64, dtype=BF), lse=z(3, 4),
                            workspace=z(64, dtype=U8))),
    "tree": (lambda eight=True, **a: pe.tree_attn(pe.KVCache(**parts(eight)), **a),
             lambda: dict(q=z(3, 5, 4, 64, dtype=BF), lens=z(3, dtype=I32), mask=z(3, 5, dtype=I64), out=z(3, 5, 4, 64, dtype=BF),
                          lse=z(3, 5, 4), workspace=z(64, dtype=U8))),
    "move": (lambda eight=True, **a: pe.kv_move(pe.KVCache(**parts(eight)), **a),
             lambda: dict(src=z(3, 2, dtype=I32), dst=z(3, 2, dtype=I32))),
}
ARGS = [(c, a) for c, (_, make) in CALLS.items() for a in make()]


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("eight", [False, True])
def test_calls_go_through(on_device_0, call, eight):
    f, make = CALLS[call]
    with pytest.raises(AssertionError, match="C library"):
        f(eight, **make())


@pytest.mark.parametrize("where", [Elsewhere, torch.Tensor], ids=["device_1", "host"])
@pytest.mark.parametrize("call,arg", ARGS)
def test_a_tensor_on_another_device_is_refused(on_device_0, call, arg, where):
    f, make = CALLS[call]
    a = make()
    a[arg] = a[arg].as_subclass(where)
    with pytest.raises(ValueError):
        f(**a)


@pytest.mark.parametrize("call", CALLS)
def test_a_device_that_is_not_current_is_refused(on_device_0, monkeypatch, call):
    f, make = CALLS[call]
    a = make()
    monkeypatch.setattr(pe, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError):
        f(**a)


@pytest.mark.parametrize("call,bad", [
    ("append", dict(k=z(3, 2, 64))), ("append", dict(v=z(3, 2, 64, dtype=torch.float16))), ("append", dict(slots=z(3, dtype=I64))),
    ("append", dict(slots=z(4, dtype=I32))), ("append", dict(q=z(3, 4, 64, dtype=E4M3))),
    ("decode", dict(q=z(3, 4, 64))), ("decode", dict(out=z(3, 4, 64, dtype=torch.float16))), ("decode", dict(window=2 ** 32)),
    ("tree", dict(q=z(3, 4, 64, dtype=BF))), ("tree", dict(mask=z(3, 4, dtype=I64))), ("tree", dict(mask=z(3, 5, dtype=I32))),
    ("tree", dict(mask=z(5, 3, dtype=I64).T)), ("tree", dict(out=z(3, 5, 4, 64))), ("tree", dict(lse=z(3, 5))),
    ("tree", dict(window=2 ** 31)), ("tree", dict(window=-2 ** 32)), ("tree", dict(lens=z(3, dtype=I64))),
    ("tree", dict(workspace=z(64, dtype=U8).expand(2, 64))),
    ("move", dict(src=z(3, 3, dtype=I32))), ("move", dict(dst=z(2, 3, dtype=I32).T)), ("move", dict(src=z(3, 2, dtype=I64))),
    ("move", dict(src=z(6, dtype=I32)))])
def test_the_binding_refuses(on_device_0, call, bad):
    f, make = CALLS[call]
    with pytest.raises(ValueError):
        f(**dict(make(), **bad))


def test_trees_and_moves_beyond_64_are_refused(on_device_0):
    f, make = CALLS["tree"]
    q = z(3, 65, 4, 64, dtype=BF)
    with pytest.raises(ValueError):
        f(**dict(make(), q=q, out=z(3, 65, 4, 64, dtype=BF), mask=z(3, 65, dtype=I64), lse=None))
    f, make = CALLS["move"]
    with pytest.raises(ValueError):
        f(src=z(3, 65, dtype=I32), dst=z(3, 65, dtype=I32))
