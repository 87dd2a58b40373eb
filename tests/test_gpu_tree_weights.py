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
    (BF16, False, 64, 33, 1), (BF16, False, 128, 17, 1), (F16, False, 128, 24, 1), (BF16, False, 64, 8, 4),
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


@pytest.mark.parametrize("dtype,eight,lens,N,max_pages,page,Hq,Hkv,layout", [
    (BF16, True, [900, 0, 31, 257], 8, 30, 32, 8, 2, "slot"), (F16, True, [64, 63, 65, 5], 29, 9, 13, 3, 3, "head"),
    (BF16, False, [3000], 4, 64, 48, 8, 1, "slot"), (F16, False, [500, 40, 7], 31, 40, 16, 2, 2, "head"),
    (BF16, True, [20, 8, -3], 32, 3, 8, 1, 1, "slot")])  # the last: nodes beyond the table
@pytest.mark.parametrize("window", [0, 64, 200])
def test_four_tiles_of_rows(dtype, eight, lens, N, max_pages, page, Hq, Hkv, layout, window):
    """25 to 32 rows of head_dim 64, in one warp."""
    base.test_tree(dtype, eight, lens, N, max_pages, page, Hq, Hkv, 64, layout, window)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("window", [0, 70])
def test_four_tiles_of_rows_and_values_that_are_no_numbers(eight, window):
    base.test_few_rows_and_values_that_are_no_numbers(eight, 8, 8, 64, 500, window)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,longest", [(90, 300), (3, 9000), (700, 2), (1, 20000)])
def test_four_tiles_of_rows_of_many_segments(eight, B, longest):
    base.test_many_segments(eight, 64, 4, 30, B, longest)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("lens,window", [([700, 3, 0], 0), ([9000, 40, 700], 0), ([9000, 40, 700], 1000)])
def test_one_token_of_32_heads(dtype, lens, window):
    base.test_decode8(dtype, True, lens, 150, 64, 60, 2, 64, "slot", window)
