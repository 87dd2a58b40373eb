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
