"""The bounded waits of the attention of drafted tokens: a wait that gives up
ends in a status, and what runs after it is not touched."""
import pytest
import torch

from paper_2608_11226_gb300 import pe


def test_refusals():
    L = pe.lib()
    for mode, limit, ws in ((-1, 2000, 256), (5, 2000, 256), (3, 999, 256), (4, 9 * 10 ** 9, 256), (3, 2000, None), (4, 2000, 128)):
        assert L.pe_wait_selftest(mode, limit, ws, None) == pe.PE_EINVAL, (mode, limit, ws)
    for mode, size in ((0, 15), (3, (1 << 26) - 1), (4, 16)):
        with pytest.raises(ValueError):
            pe.wait_selftest(mode, 2000, torch.empty(size, dtype=torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("mode,eight", [(3, False), (4, True)])
def test_tiles_that_never_come(mode, eight):
    import test_gpu_cache8_tree as base

    P = base.Pool(2, 12, 64, 1, 128, base.BF16, eight, "slot", 3)
    masks = base.tensor_of(base.tree_masks(2, 64, 5))
    lens = torch.tensor([700, 90], dtype=torch.int32, device="cuda")
    calls = []
    for heads in (1, 3):
        q = torch.randn((2, 64, heads, 128), generator=base.gen(heads), device="cuda").to(base.BF16)
        out = torch.empty_like(q)
        pe.tree_attn(P.cache, q, lens, masks, out)
        calls.append((q, out))
    pe.device_check()
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        with pytest.raises(pe.PEError) as e:
            pe.wait_selftest(mode, 20_000_000, ws)
        assert e.value.status == pe.PE_ETIMEOUT
        pe.device_check()  # reported once
        for q, out in calls:
            again = torch.full_like(out, float("nan"))
            pe.tree_attn(P.cache, q, lens, masks, again)
            assert torch.equal(again, out)
        pe.device_check()
