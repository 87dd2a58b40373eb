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


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("n,spare", [(200, 0), (200, 9000), (9000, 0)])
@pytest.mark.parametrize("D,group", [(64, 2), (64, 20), (128, 12), (128, 40), (256, 3), (256, 40)])
def test_decode_nothing_but_minus_infinity(D, group, n, spare, dtype):
    """Every score -inf: zero and -inf, whatever the values are, in small batches and in the line of tiles."""
    g = ops.gen(n + D + group)
    kc, vc, table = ops.make_cache([n, n], 1, D, 16, dtype, "slot", g, slack=1 + spare // 16)
    at = table[0].long()[:-(-n // 16)]
    kc[at, :, 0, 0] = -INF
    vc[at[0], 3, 0, 5], vc[at[-1], 1, 0, 6], vc[at[2]] = INF, NAN, -INF
    q = torch.randn((2, group, D), generator=g, device="cuda").to(dtype)
    q[:, :, 0] = 1.0
    lens = torch.tensor([n, n], dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, NAN), torch.full((2, group), NAN, device="cuda")
    pe.decode_attn(pe.KVCache(kc, vc, table), q, lens, out, lse=lse)
    assert bool((out[0] == 0).all()) and bool((lse[0] == -INF).all())
    r, rl, ds, ab = (t[1] for t in ops.plain_decode(kc, vc, table, q, lens, D ** -0.5, 0))
    ds = ds * 2.0 ** -20
    ops.close(out[1], r, ops.U[dtype] * r.abs() + (2 * ds + 2.0 ** -14)[:, None] * ab + ops.TINY[dtype])
    ops.close(lse[1], rl, ds + 2.0 ** -18 + 2.0 ** -22 * rl.abs())


def wide_cache(lens, Hkv, D, page, dtype, capacity, g):
    """A cache whose table has room for `capacity` positions of each sequence, as a server's has for the model's
    context; the entries beyond a length name a page of NaN."""
    kc, vc, exact = ops.make_cache(lens, Hkv, D, page, dtype, "slot", g, slack=0, spare=1)
    unused = torch.ones(kc.shape[0], dtype=torch.bool, device="cuda")
    unused[exact.long().flatten()] = False
    table = torch.full((len(lens), capacity // page + 3), int(torch.nonzero(unused)[0]), dtype=torch.int32, device="cuda")
    for b, n in enumerate(lens):
        table[b, :-(-n // page)] = exact[b, :-(-n // page)]
    return kc, vc, table[:, :capacity // page]


# Every number of query heads at which a warp, or a team of warps, takes another number of them together, in the three
# ways in which sequences come: few and short (clusters), long ones in a line of tiles, more of them than CTAs.
@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("way", ["short", "long", "many"])
@pytest.mark.parametrize("group", [1, 8, 9, 16, 17, 24, 25, 32, 33, 64, 65])
@pytest.mark.parametrize("D", [64, 128, 256])
def test_decode_heads(D, group, way, dtype):
    g = ops.gen(D + group)
    lens, Hkv, capacity = {"short": ([37, 0, 300], 2, 304), "long": ([2100, 5, 700], 2, 16384),
                           "many": ([(i * 37) % 601 for i in range(44)], 8, 16384)}[way]
    kc, vc, table = wide_cache(lens, Hkv, D, 16, dtype, capacity, g)
    q = (2 * torch.randn((len(lens), Hkv * group, D), generator=g, device="cuda")).to(dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    for window in (0, 130):
        ops.check_decode(kc, vc, table, q, n, window=window)


def test_decode_on_two_streams_at_once():
    """Calls on two streams, each with a workspace of its own, over one cache."""
    g = ops.gen(40)
    lens = [9000, 1, 4000, 333]
    kc, vc, table = wide_cache(lens, 2, 128, 16, BF16, 16384, g)
    cache, n = pe.KVCache(kc, vc, table), torch.tensor(lens, dtype=torch.int32, device="cuda")
    qs = [torch.randn((4, 8, 128), generator=g, device="cuda").to(BF16) for _ in range(2)]
    want = [ops.check_decode(kc, vc, table, q, n)[0] for q in qs]
    streams = [torch.cuda.Stream() for _ in qs]
    ws = [pe.alloc_workspace(pe.decode_attn_workspace_bytes(cache, 8)) for _ in qs]
    outs = [[torch.full_like(q, NAN) for _ in range(20)] for q in qs]
    torch.cuda.synchronize()
    for i in range(20):
        for q, st, w, out in zip(qs, streams, ws, outs):
            pe.decode_attn(cache, q, n, out[i], workspace=w, stream=st)
    torch.cuda.synchronize()
    for out, r in zip(outs, want):
        assert all(torch.equal(o, r) for o in out)
