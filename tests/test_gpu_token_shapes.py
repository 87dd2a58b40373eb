"""The token operators at the shapes that choose their variants (GPU), against
the 64-bit evaluations of test_gpu_token_ops and within its tolerances."""
import pytest
import torch

import test_gpu_token_ops as ops
from paper_2608_11226_gb300 import pe

pytestmark = pytest.mark.gpu

BF16, F16, F32 = ops.BF16, ops.F16, ops.F32
NAN, INF = ops.NAN, ops.INF


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("n,V", [(3, 300), (2000, 900), (3, 9000), (1000, 9000), (3, 70000), (1, 200000)])
def test_logp_more_candidates_than_are_held(dtype, n, V):
    """Rows in which few to nearly all elements are as likely as the k-th alternative, in all warps at once: the
    warps of a row stop looking at different times."""
    g = ops.gen(n + V)
    x = torch.round(2 * torch.randn((n, V), generator=g, device="cuda")).clamp_(-6, 4)
    for i, share in enumerate((0.02, 0.06, 0.2, 0.6, 0.95)):  # of the row at its largest value
        rows = x[i::5]
        rows[torch.rand(rows.shape, generator=g, device="cuda") < share] = 4.0
    x[0, V // 2] = 5.0
    ops.check_logp(x.to(dtype), ops.targets(n, V, V), k=20)


@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 32, 2 ** 31 - 33])
@pytest.mark.parametrize("n", [40, 3000, 100003])
def test_decode_window_beyond_any_length(n, window):
    """A window that no length reaches is no window, bit for bit."""
    g = ops.gen(n)
    kc, vc, table = ops.make_cache([n, n // 3], 2, 64, 16, BF16, "slot", g)
    q = torch.randn((2, 8, 64), generator=g, device="cuda").to(BF16)
    lens = torch.tensor([n, n // 3], dtype=torch.int32, device="cuda")
    want, want_lse = ops.check_decode(kc, vc, table, q, lens)
    got, lse = ops.check_decode(kc, vc, table, q, lens, window=window)
    assert torch.equal(got, want) and torch.equal(lse, want_lse)
