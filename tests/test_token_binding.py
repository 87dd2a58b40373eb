"""What the binding of the token operators makes of its arguments, before any
C call (CPU: host tensors that pass for device tensors; nothing is launched)."""
import pytest
import torch

from paper_2608_11226_gb300 import pe


class OnDevice(torch.Tensor):
    """A host tensor that says it is on device 0."""
    is_cuda = True

    def get_device(self):
        return 0


def dev(t):
    return t.as_subclass(OnDevice)


def pages(n=6, page=4, heads=2, D=64, dtype=torch.bfloat16):
    return dev(torch.zeros((n, page, heads, D), dtype=dtype))


def table(n_seqs=3, max_pages=2):
    return torch.arange(n_seqs * max_pages, dtype=torch.int32).view(n_seqs, max_pages)


@pytest.mark.parametrize("t", [
    table(1, 4).expand(3, -1),                                             # one row for all sequences
    torch.arange(9, dtype=torch.int32).as_strided((3, 4), (2, 1)),         # rows that overlap
    torch.zeros(1, dtype=torch.int32).expand(3, 1),                        # rows of one page
], ids=["expanded", "overlapping", "one_page"])
def test_table_rows_closer_than_their_length_are_refused(t):
    with pytest.raises(ValueError):
        pe.KVCache(pages(), pages(), dev(t))


@pytest.mark.parametrize("t,stride", [(table(), 2), (torch.zeros((3, 9), dtype=torch.int32)[:, 2:6], 9),
                                      (table(6)[::2], 4), (table(1, 5), 5), (table(1, 5).expand(1, -1), 5),
                                      (torch.zeros((8, 1), dtype=torch.int32)[::4], 4)])
def test_table_rows_are_as_far_apart_as_the_tensor_says(t, stride):
    d = pe.KVCache(pages(), pages(), dev(t))._desc
    assert (d.n_seqs, d.max_pages, d.table_stride) == (t.shape[0], t.shape[1], stride)
    last = (d.n_seqs - 1) * d.table_stride + d.max_pages  # entries that the kernels may read
    assert t.storage_offset() + last <= t.untyped_storage().nbytes() // 4


# ---------------------------------------------------------------------------
# devices and workspaces
# ---------------------------------------------------------------------------
class Elsewhere(torch.Tensor):
    """A host tensor that says it is on device 1."""
    is_cuda = True

    def get_device(self):
        return 1


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


def z(*shape, dtype=torch.float32):
    return dev(torch.zeros(shape, dtype=dtype))


BF, I32 = torch.bfloat16, torch.int32
CALLS = {
    "append": (lambda **a: pe.kv_append(pe.KVCache(pages(), pages(), dev(table())), **a),
               lambda: dict(k=z(3, 2, 64, dtype=BF), v=z(3, 2, 64, dtype=BF), positions=z(3, dtype=I32), seqs=z(3, dtype=I32),
                            q=z(3, 4, 64, dtype=BF), q_out=z(3, 4, 64, dtype=BF), rot=z(8, 64))),
    "decode": (lambda **a: pe.decode_attn(pe.KVCache(pages(), pages(), dev(table())), **a),
               lambda: dict(q=z(3, 4, 64, dtype=BF), lens=z(3, dtype=I32), out=z(3, 4, 64, dtype=BF), lse=z(3, 4),
                            workspace=z(64, dtype=torch.uint8))),
    "logp": (pe.token_logp,
             lambda: dict(logits=z(3, 9), tokens=z(3, dtype=I32), logp=z(3), entropy=z(3), lse=z(3), top_logp=z(3, 2),
                          top_id=z(3, 2, dtype=I32))),
    "grad": (pe.token_logp_grad,
             lambda: dict(logits=z(3, 9), tokens=z(3, dtype=I32), lse=z(3), dlogits=z(3, 9), g_logp=z(3), entropy=z(3),
                          g_entropy=z(3))),
}
ARGS = [(c, a) for c, (_, make) in CALLS.items() for a in make()]


@pytest.mark.parametrize("call", CALLS)
def test_calls_on_the_current_device_go_through(on_device_0, call):
    f, make = CALLS[call]
    with pytest.raises(AssertionError, match="C library"):
        f(**make())


@pytest.mark.parametrize("where", [Elsewhere, torch.Tensor], ids=["device_1", "host"])
@pytest.mark.parametrize("call,arg", ARGS)
def test_a_tensor_on_another_device_is_refused(on_device_0, call, arg, where):
    f, make = CALLS[call]
    a = make()
    a[arg] = a[arg].as_subclass(where)
    with pytest.raises(ValueError):
        f(**a)


@pytest.mark.parametrize("call", CALLS)
def test_tensors_that_share_a_device_that_is_not_current_are_refused(on_device_0, monkeypatch, call):
    f, make = CALLS[call]
    a = make()
    monkeypatch.setattr(pe, "_current_device", lambda: 1, raising=False)
    with pytest.raises(ValueError):
        f(**a)


@pytest.mark.parametrize("part", range(3))
@pytest.mark.parametrize("where", [Elsewhere, torch.Tensor], ids=["device_1", "host"])
def test_a_cache_lies_on_one_device(part, where):
    t = [pages(), pages(), dev(table())]
    t[part] = t[part].as_subclass(where)
    with pytest.raises(ValueError):
        pe.KVCache(*t)


@pytest.mark.parametrize("ws", [torch.zeros(1, dtype=torch.uint8).expand(1 << 20), torch.zeros(1 << 20, dtype=torch.uint8)[::2]],
                         ids=["expanded", "strided"])
def test_a_workspace_is_contiguous(on_device_0, ws):
    f, make = CALLS["decode"]
    with pytest.raises(ValueError):
        f(**dict(make(), workspace=dev(ws)))


# ---------------------------------------------------------------------------
# sizes that a 32-bit argument does not hold
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("window", [2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 63 - 1, -2 ** 32, -2 ** 32 + 5])
def test_a_window_that_passes_32_bits_is_refused(on_device_0, window):
    f, make = CALLS["decode"]
    with pytest.raises(ValueError):
        f(**make(), window=window)


@pytest.mark.parametrize("V", [2 ** 31, 2 ** 32 + 9])
@pytest.mark.parametrize("call", ["logp", "grad"])
def test_rows_that_pass_32_bits_are_refused(on_device_0, call, V):
    f, make = CALLS[call]
    a = {k: t[:0] for k, t in make().items()}
    a.update({k: z(0, V) for k in ("logits", "dlogits") if k in a})
    with pytest.raises(ValueError):
        f(**a)


def test_a_table_that_passes_32_bits_is_refused():
    with pytest.raises(ValueError):
        pe.KVCache(pages(), pages(), dev(torch.empty((0, 2 ** 32 + 2), dtype=I32)))
