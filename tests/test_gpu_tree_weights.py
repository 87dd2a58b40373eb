"""Drafted tokens' weights enter the sum of values with more bits than the result
has, whatever kernel the number of rows takes (GPU).

Tolerance: the result's rounding u (2^-8 bf16, 2^-11 fp16); a score off by
  ds = 2^-20 scale max_j sum_d |q_d k_jd|; weights as two 16-bit numbers, 2^-16 at
  most (bf16: 2^-9 of 2^-9, twice), or over 8 bits with bf16 queries one fp16 number,
  2^-12 (half a step); exponentials and sums 2^-14:
    |out - ref| <= u |ref| + (2 ds + w + 2^-14) sum_j p_j |v_j| + n 2^-30 max |v|.
  In the mean over a result the errors are independent roundings, so their 2-norm is
  held to 1.05 times that of the reference rounded once.
"""
import pytest
import torch

import test_gpu_cache8_tree as base
from paper_2608_11226_gb300 import pe

pytestmark = pytest.mark.gpu

BF16, F16 = base.BF16, base.F16

CASES = [  # dtype, 8 bits, D, nodes, heads a key head: few rows, tiles, wide blocks
    (BF16, False, 64, 24, 1), (BF16, False, 64, 25, 1), (BF16, False, 64, 43, 3), (BF16, False, 128, 16, 1), (BF16, False, 128, 32, 4),
    (BF16, False, 128, 50, 4), (BF16, False, 256, 8, 1), (BF16, False, 256, 32, 4), (F16, False, 64, 33, 2), (F16, False, 128, 25, 1),
    (F16, False, 128, 64, 4), (F16, False, 256, 17, 2), (F16, True, 64, 25, 2), (F16, True, 128, 20, 1), (F16, True, 128, 32, 4),
    (F16, True, 128, 50, 4), (F16, True, 256, 17, 2), (BF16, True, 128, 32, 4), (BF16, True, 128, 50, 4), (BF16, True, 64, 43, 3)]


@pytest.mark.parametrize("dtype,eight,D,N,G", CASES)
def test_weights(dtype, eight, D, N, G):
    n, page = 700, 16
    P = base.Pool(1, 50, page, 1, D, dtype, eight, "slot", D + N)
    masks = base.tree_masks(1, N, 2)
    q = torch.randn((1, N, G, D), generator=base.gen(N), device="cuda").to(dtype)
    out = torch.empty_like(q)
    pe.tree_attn(P.cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), base.tensor_of(masks), out)
    k, v, _, _, _ = P.rows(0, range(n + N))
    k, v = k[:, 0], v[:, 0]
    sees = torch.ones((N, n + N), dtype=torch.bool, device="cuda")
    for i, m in enumerate(masks[0]):
        for a in range(N):
            sees[i, n + a] = bool(m >> a & 1)
    z = (q[0].double() @ k.T) * D ** -0.5  # [N, G, positions]
    p = torch.softmax(z.masked_fill(~sees[:, None], -base.INF), -1)
    ref = p @ v
    u = base.U[dtype]
    w = 2.0 ** -12 if eight and dtype == BF16 else 2.0 ** -16
    ds = 2.0 ** -20 * D ** -0.5 * (q[0].double().abs() @ k.abs().T).amax(-1, keepdim=True)
    tol = u * ref.abs() + (2 * ds + w + 2.0 ** -14) * (p @ v.abs()) + (n + N) * 2.0 ** -30 * v.abs().max() + 2.0 ** -25
    base.close(out[0], ref, tol)
    error, least = (out[0].double() - ref).norm(), (ref.to(dtype).double() - ref).norm()
    assert error <= 1.05 * least, f"{(error / ref.norm()).item():.3g} for {(least / ref.norm()).item():.3g}"
