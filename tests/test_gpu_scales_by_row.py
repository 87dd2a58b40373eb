"""Attention over an 8-bit cache whose rows have scales far apart (GPU): each row
counts by its own scale, whatever kernel the number of rows or heads takes.

Tolerance, from attended rows alone, each by its own scale (t_j that of value
row j, p_j its share of the weights):
  a score is a sum of fp32 products of codes, times powers of two: off by
    ds = 2^-20 scale max_j sum_d |q_d k_jd|; adding the value scale's exponent
    e_j and taking it out again rounds sums of up to 192 (|e| <= 120, |z| <= 72
    here) three times, 2^-17 each in powers of two;
  weights are rounded to fp16, 2^-11, and exponentials and sums are off by 2^-14;
    where a weight times its scale is below 2^-27 of the largest, 448 codes may be missing
    (fp16 keeps 2^-25 of numbers that start at 2^7; a tile's common factor may exceed a
    row's scale by 2^5):
    |out - ref| <= u |ref| + (2 ds + 2^-11 + 2^-14 + 3 * 2^-17) sum_j p_j |v_j|
                   + n 2^-27 448 max_j p_j t_j
    |lse - ref| <= ds + 3 * 2^-17 + 2^-18 (1 + |ref|)
"""
import pytest
import torch

import test_gpu_cache8_tree as base
from paper_2608_11226_gb300 import pe

pytestmark = pytest.mark.gpu

BF16, F16, U, NAN = base.BF16, base.F16, base.U, base.NAN


def attend(P, q, lens, scale, window, masks=None):
    """(out, lse, tolerances of both) in 64 bits; arguments as of the other evaluation."""
    B, N, Hq, _ = q.shape
    G = Hq // P.k.shape[2]
    cap = P.table.shape[1] * P.page
    out, lse = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.full(q.shape[:-1], -base.INF, dtype=torch.float64, device="cuda")
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n = lens[b]
        for i in range(N):
            if masks is None:
                where = list(range(max(0, n - window) if window else 0, n))
            else:
                nodes = [n + a for a in range(N) if masks[b][i] >> a & 1]
                if not nodes:
                    continue
                where = list(range(max(0, n + len(nodes) - window) if window else 0, n)) + [p for p in nodes if p < cap]
            k, v, _, vs, there = P.rows(b, where)
            assert bool(there.all())
            for h in range(P.k.shape[2]):
                hs = slice(h * G, (h + 1) * G)
                qs = q[b, i, hs].double()
                z = qs @ k[:, h].T * scale
                p = torch.softmax(z, -1)
                lse[b, i, hs], out[b, i, hs] = torch.logsumexp(z, -1), p @ v[:, h]
                ds = 2.0 ** -20 * abs(scale) * (qs.abs() @ k[:, h].abs().T).amax(-1)
                lost = len(where) * 2.0 ** -27 * 448 * (p * vs[:, h]).amax(-1)
                tol[b, i, hs] = (U[q.dtype] * out[b, i, hs].abs()
                                 + (2 * ds + 2.0 ** -11 + 2.0 ** -14 + 3 * 2.0 ** -17)[:, None] * (p @ v[:, h].abs()) + lost[:, None])
                ltol[b, i, hs] = ds + 3 * 2.0 ** -17 + 2.0 ** -18 * (1 + lse[b, i, hs].abs())
    return out, lse, tol + (2.0 ** -25 if q.dtype == F16 else 0.0), ltol


# nodes and heads a key head on either side of every choice of kernel and block
ROWS = [(64, 24, 1), (64, 32, 1), (64, 33, 1), (64, 43, 3), (128, 24, 1), (128, 25, 1), (128, 43, 3), (256, 16, 1), (256, 17, 1), (256, 43, 3)]


@pytest.mark.parametrize("D,N,G", ROWS)
@pytest.mark.parametrize("byte", [144, 200, 247])
@pytest.mark.parametrize("what", ["padding", "sibling", "ahead"])
@pytest.mark.parametrize("rows", ["keys", "values"])
def test_a_scale_that_a_row_does_not_see(D, N, G, byte, what, rows):
    """A large scale in a padding node's slot, in a node that some see, ahead of the deeper nodes' windows:
    no part in the results of those who do not attend there."""
    page, H, lens, window = 16, 2, [300, 65], 64 if what == "ahead" else 0
    P = base.Pool(2, 24, page, H, D, BF16, True, "slot", 5)
    masks = [[(1 << i + 1) - 1 for i in range(N)]] * 2 if what == "ahead" else base.tree_masks(2, N, 9)
    if what == "padding":
        masks = [[0 if i == N - 1 else m for i, m in enumerate(row)] for row in masks]
    if what == "ahead":
        at = [n + 1 - window + 10 for n in lens]
        sees = [[i <= 10 for i in range(N)]] * 2
    else:
        node = N - 1 if what == "padding" else 1
        at = [n + node for n in lens]
        sees = [[bool(m >> node & 1) for m in row] for row in masks]
    for b, p in enumerate(at):
        (P.ks if rows == "keys" else P.vs)[int(P.table[b, p // page]), p % page] = byte
    q = torch.randn((2, N, G * H, D), generator=base.gen(1), device="cuda").to(BF16)
    out, lse = torch.full_like(q, NAN), torch.full((2, N, G * H), NAN, device="cuda")
    pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), base.tensor_of(masks), out, window=window, lse=lse)
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, window, masks)
    blind = ~torch.tensor(sees, device="cuda")
    if rows == "values" and byte == 144:  # what the others see is ordinary too
        blind[:] = True
    assert blind.any(1).all()
    base.close(out[blind], ro[blind], to[blind])
    base.close(lse[blind], rl[blind], tl[blind])


CALLS = [  # nodes (0: one token), heads of a key head
    (64, 0, 24), (64, 0, 40), (128, 0, 24), (128, 0, 32), (256, 0, 16), (256, 0, 24),
    (64, 20, 1), (64, 30, 2), (64, 50, 4), (128, 20, 1), (128, 30, 2), (128, 50, 4), (256, 10, 1), (256, 30, 1), (256, 50, 4)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("D,N,G", CALLS)
@pytest.mark.parametrize("far", ["keys", "values", "values of nothing"])
def test_attended_rows_far_apart(dtype, D, N, G, far):
    """One attended row's scale is 2^30 times the others': a key at right angles to the queries, or values with next to
    no weight; or every value but one row's is zero, which is what the least scale stands for."""
    page, H, lens = 16, 2, [200, 40]
    P = base.Pool(2, 24, page, H, D, dtype, True, "slot", 6)
    at = 7  # a position of each sequence
    kb, vb = P.k.view(torch.uint8), P.v.view(torch.uint8)
    q = torch.randn((2, max(N, 1), G * H, D), generator=base.gen(1), device="cuda")
    q[..., 0], q[..., 1] = 8.0, 0.0
    q = q.to(dtype)
    for b in range(2):
        where = int(P.table[b, at // page]), at % page
        kb[where] = 0
        if far == "keys":
            kb[where[0], where[1], :, 1] = 0x7E  # 448, where queries are 0
            P.ks[where] = 119 + 30
        else:
            P.ks[where] = 127
            c = torch.tensor(-6.0 * D ** 0.5, device="cuda").to(base.E4M3).view(torch.uint8)  # a score of -48
            kb[where[0], where[1], :, 0] = c
            P.vs[where] = 119 + (30 if far == "values" else 0)
    if far == "values of nothing":
        sequence = torch.arange(40 + max(N, 1), device="cuda")
        for b in range(2):
            for p in sequence.tolist():
                if p != at:
                    where = int(P.table[b, p // page]), p % page
                    vb[where], P.vs[where] = 0, 63
    out, lse = torch.full_like(q, NAN), torch.full(q.shape[:-1], NAN, device="cuda")
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    if N:
        masks = base.tree_masks(2, N, 3)
        pe.tree_attn(P.cache, q, t, base.tensor_of(masks), out, lse=lse)
    else:
        masks = None
        pe.decode_attn(P.cache, q[:, 0], t, out[:, 0], lse=lse)
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, 0, masks)
    base.close(out, ro, to)
    base.close(lse, rl, tl)


@pytest.mark.parametrize("D,N,G", CALLS)
@pytest.mark.parametrize("power", [-50, 60, 114])
def test_large_keys_and_small_queries(D, N, G, power):
    """Keys 2^power times as large, queries as much smaller: the same scores, so the same bits."""
    page, H, n = 16, 2, 150
    P = base.Pool(1, 24, page, H, D, BF16, True, "slot", 6)
    q = 1.0 + torch.rand((1, max(N, 1), G * H, D), generator=base.gen(1), device="cuda")
    q *= torch.where(torch.rand(q.shape, generator=base.gen(2), device="cuda") < 0.5, -1.0, 1.0)
    t = torch.tensor([n], dtype=torch.int32, device="cuda")
    masks = base.tensor_of(base.tree_masks(1, max(N, 1), 3))
    got = []
    for k in (0, power):
        P.ks += k if k >= 0 else 256 + k  # (bytes wrap)
        x = (q.to(BF16).double() * 2.0 ** -k).to(BF16)
        out, lse = torch.full_like(x, NAN), torch.full(x.shape[:-1], NAN, device="cuda")
        if N:
            pe.tree_attn(P.cache, x, t, masks, out, lse=lse)
        else:
            pe.decode_attn(P.cache, x[:, 0], t, out[:, 0], lse=lse)
        got.append((out, lse))
    assert torch.isfinite(got[0][0].float()).all()
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("D,N,G", [c for c in CALLS if c[0] * c[2] > 64 or c[1] > 20])
@pytest.mark.parametrize("keys,values", [(0, 0), (5, 5), (14, 5), (15, 5), (14, 6), (15, 6), (3, 9)])
def test_spreads_of_scales(D, N, G, keys, values):
    """Scales within so many powers of two in every tile: either side of where a tile has one factor."""
    page, H, lens = 16, 2, [300, 129]
    P = base.Pool(2, 24, page, H, D, BF16, True, "slot", 6)
    for s, spread in ((P.ks, keys), (P.vs, values)):
        s.copy_(torch.randint(118 - spread // 2, 119 - spread // 2 + spread, s.shape, generator=base.gen(spread), device="cuda"))
        s[:, :: page - 1] = torch.tensor([118 - spread // 2, 118 - spread // 2 + spread], device="cuda")[:, None].to(torch.uint8)
    q = torch.randn((2, max(N, 1), G * H, D), generator=base.gen(1), device="cuda").to(BF16)
    out, lse = torch.full_like(q, NAN), torch.full(q.shape[:-1], NAN, device="cuda")
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    masks = base.tree_masks(2, N, 3) if N else None
    if N:
        pe.tree_attn(P.cache, q, t, base.tensor_of(masks), out, lse=lse)
    else:
        pe.decode_attn(P.cache, q[:, 0], t, out[:, 0], lse=lse)
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, 0, masks)
    base.close(out, ro, to)
    base.close(lse, rl, tl)
