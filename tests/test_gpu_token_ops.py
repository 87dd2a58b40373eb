"""The token operators against plain evaluations in 64 bits (GPU).

Tolerances, from the arithmetic that include/pe.h states:
  u = 2^-8 (bf16), 2^-11 (fp16), 2^-24 (fp32): one rounding of the result, |x| u
  (for fp16 plus half the least subnormal, 2^-25).
  append: two products and a sum in fp32: 3 * 2^-24 (|a c| + |b s|).
  decode: a score is a sum of D fp32 products; its error is at most
    ds = 2^-20 scale max_j sum_d |q_d k_jd| (sixteen roundings of the whole sum, the
    tensor core's included), which moves every weight by a factor of at most
    e^ds; weights enter the second product with at least 16 significant bits
    and sums are fp32: |out - ref| <= u |ref| + (2 ds + 2^-14) sum_j p_j |v_j|.
  logp: fp32 differences, exponentials and sums: 2^-18 (1 + |ref|) and, for
    what the logits' own size costs (m = the row's largest), 2^-22 |m|.
  grad: u |ref| + p (|g_logp| + |g_entropy| (|ln p| + H)) scale (2^-18 + 2^-22 |lse|).
"""
import math

import pytest
import torch

from paper_2608_11226_gb300 import pe

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11, F32: 2.0 ** -24}
TINY = {BF16: 0.0, F16: 2.0 ** -25, F32: 0.0}
NAN, INF = float("nan"), float("inf")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def f32(x):
    """The fp32 value that an argument of the C call carries."""
    return torch.tensor(x, dtype=F32).item()


def close(got, ref, tol):
    """got against the 64-bit ref: equal where ref is not finite, within tol elsewhere."""
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf])
    ok = torch.isfinite(ref)
    bad = ok & ~((got - ref).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} values off, the worst by {((got - ref).abs() - tol)[ok].max().item():.3g}"


def storage(n_pages, page, heads, D, dtype, layout, fill=NAN):
    shape = (n_pages, page, heads, D) if layout == "slot" else (n_pages, heads, page, D)
    x = torch.full(shape, fill, dtype=dtype, device="cuda")
    return x if layout == "slot" else x.transpose(1, 2)


# ---------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------
def plain_append(k_cache, v_cache, table, k, v, pos, seqs, q, rot, inter, max_pos):
    """Token by token; returns (q, |q| terms, k_cache, |k| terms, v_cache) in 64 bits."""
    kc, vc = k_cache.double().clone(), v_cache.double().clone()
    ka = kc.abs()
    q_out, qa = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    page, rd = k_cache.shape[1], 0 if rot is None else rot.shape[1]
    half = rd // 2

    def turn(x, p):
        y, ab = x.double().clone(), x.double().abs()
        i = torch.arange(half, device="cuda")
        lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + half)
        c, s = (rot[p].double()[:half], rot[p].double()[half:]) if half else (1.0, 0.0)
        a, b = y[..., lo], y[..., hi]
        y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
        ab[..., lo], ab[..., hi] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
        return y, ab

    for t, p in enumerate(pos.tolist()):
        s = t if seqs is None else int(seqs[t])
        if p < 0 or (rd and p >= max_pos) or p >= table.shape[1] * page or not 0 <= s < table.shape[0]:
            continue
        q_out[t], qa[t] = turn(q[t], p)
        g = int(table[s, p // page])
        if 0 <= g < k_cache.shape[0]:
            kc[g, p % page], ka[g, p % page] = turn(k[t], p)
            vc[g, p % page] = v[t].double()
    return q_out, qa, kc, ka, vc


APPEND = [
    # dtype, T, n_seqs, Hq, Hkv, D, page, rot_dim, interleaved, layout, fused
    (BF16, 1, 1, 1, 1, 64, 16, 64, False, "slot", True),
    (BF16, 5, 5, 8, 2, 128, 16, 128, False, "slot", True),
    (F16, 37, 3, 6, 3, 64, 5, 32, True, "head", False),
    (BF16, 65, 2, 5, 1, 256, 24, 256, False, "head", True),
    (F16, 19, 4, 4, 4, 128, 1, 16, True, "slot", False),
    (BF16, 33, 2, 10, 2, 128, 64, 48, False, "slot", True),
    (BF16, 7, 7, 3, 3, 128, 16, 0, False, "slot", False),
    (F16, 300, 3, 40, 8, 128, 32, 128, False, "slot", True),
]


@pytest.mark.parametrize("dtype,T,n_seqs,Hq,Hkv,D,page,rd,inter,layout,fused", APPEND)
@pytest.mark.parametrize("in_place", [False, True])
def test_append(dtype, T, n_seqs, Hq, Hkv, D, page, rd, inter, layout, fused, in_place):
    g = gen(T + D)
    per = -(-T // n_seqs) + 3
    max_pages = -(-per // page)
    n_pages = n_seqs * max_pages + 1
    kc, vc = storage(n_pages, page, Hkv, D, dtype, layout, 3.0), storage(n_pages, page, Hkv, D, dtype, layout, -7.0)
    table = torch.randperm(n_pages, generator=g, device="cuda")[:n_seqs * max_pages].view(n_seqs, max_pages).to(torch.int32)
    if T == n_seqs:
        seqs, pos = None, torch.randint(0, per, (T,), generator=g, device="cuda").to(torch.int32)
    else:
        order = torch.randperm(T, generator=g, device="cuda")
        seqs, pos = (order % n_seqs).to(torch.int32), (order // n_seqs + 2).to(torch.int32)
    if T >= 7:  # padding, out-of-range tokens, a page that is not there
        pos[1], pos[2], pos[3] = -1, max_pages * page, 2 ** 31 - 1
        if seqs is not None:
            seqs[4], seqs[5] = -1, n_seqs
        table[-1, -1] = -1 if T % 2 else n_pages
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda").to(dtype)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    if not fused:
        q, k, v = (p.contiguous() for p in (q, k, v))
    max_pos = max(per - 1, 1)
    rot = pe.rot_table(max_pos, rd) if rd else None
    rq, qa, rk, ka, rv = plain_append(kc, vc, table, k, v, pos, seqs, q, rot, inter, max_pos)
    q_out = q if in_place else torch.full((T, Hq, D), NAN, dtype=dtype, device="cuda")
    cache = pe.KVCache(kc, vc, table)
    pe.kv_append(cache, k, v, pos, seqs=seqs, q=q, q_out=None if in_place else q_out, rot=rot, interleaved=inter)
    e = 3 * 2.0 ** -24
    close(q_out, rq, U[dtype] * rq.abs() + e * qa + TINY[dtype])
    close(kc, rk, U[dtype] * rk.abs() + e * ka + TINY[dtype])
    assert torch.equal(vc.double(), rv)
    if not in_place:  # without queries the cache gets the same
        k2, v2 = storage(n_pages, page, Hkv, D, dtype, layout, 3.0), storage(n_pages, page, Hkv, D, dtype, layout, -7.0)
        pe.kv_append(pe.KVCache(k2, v2, table), k, v, pos, seqs=seqs, rot=rot, interleaved=inter)
        assert torch.equal(k2, kc) and torch.equal(v2, vc)


def test_append_nothing():
    kc = storage(2, 16, 1, 64, BF16, "slot", 1.0)
    e = torch.empty((0, 1, 64), dtype=BF16, device="cuda")
    pe.kv_append(pe.KVCache(kc, kc.clone(), torch.zeros((1, 2), dtype=torch.int32, device="cuda")), e, e,
                 torch.empty(0, dtype=torch.int32, device="cuda"))
    assert bool((kc == 1.0).all())


# ---------------------------------------------------------------------------
# decode
# ---------------------------------------------------------------------------
def plain_decode(k_cache, v_cache, table, q, lens, scale, window):
    """(out, lse, score error unit, sum p |v|) of every sequence and head in 64 bits."""
    B, Hq, D = q.shape
    scale = f32(scale)
    n_pages, page, Hkv = k_cache.shape[:3]
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    ab, lse = torch.zeros_like(out), torch.full((B, Hq), -INF, dtype=torch.float64, device="cuda")
    ds = torch.zeros((B, Hq), dtype=torch.float64, device="cuda")
    for b in range(B):
        n = min(max(int(lens[b]), 0), table.shape[1] * page)
        j = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        g = table[b].long()[j // page]
        keep = (g >= 0) & (g < n_pages)
        j, g = j[keep], g[keep]
        if not len(j):
            continue
        k, v = k_cache[g, j % page].double(), v_cache[g, j % page].double()  # [n, Hkv, D]
        k, v = (t.repeat_interleave(Hq // Hkv, 1) for t in (k, v))
        z = torch.einsum("hd,jhd->hj", q[b].double(), k) * scale
        ds[b] = torch.einsum("hd,jhd->hj", q[b].double().abs(), k.abs()).amax(1) * abs(scale)
        m = z.amax(1, keepdim=True)
        p = torch.exp(z - torch.where(m == -INF, 0.0, m))
        l = p.sum(1, keepdim=True)
        lse[b] = (m + torch.log(l))[:, 0]
        p = torch.where(l == 0, 0.0, p / l)
        v = torch.where((p == 0).T[..., None], 0.0, v)
        out[b], ab[b] = torch.einsum("hj,jhd->hd", p, v), torch.einsum("hj,jhd->hd", p, v.abs())
    return out, lse, ds, ab


def check_decode(kc, vc, table, q, lens, scale=None, window=0, out=None, **kw):
    B, Hq, D = q.shape
    scale_ = D ** -0.5 if scale is None else scale
    out = torch.full((B, Hq, D), NAN, dtype=q.dtype, device="cuda") if out is None else out
    lse = torch.full((B, Hq), NAN, device="cuda")
    pe.decode_attn(pe.KVCache(kc, vc, table), q, lens, out, scale=scale, window=window, lse=lse, **kw)
    r, rl, ds, ab = plain_decode(kc, vc, table, q, lens, scale_, window)
    ds = ds * 2.0 ** -20
    close(out, r, U[q.dtype] * r.abs() + (2 * ds + 2.0 ** -14)[..., None] * ab + TINY[q.dtype])
    close(lse, rl, ds + 2.0 ** -18 + 2.0 ** -22 * torch.where(torch.isfinite(rl), rl.abs(), 0.0))
    return out, lse


def make_cache(lens, Hkv, D, page, dtype, layout, g, slack=1, spare=3):
    """A pool whose every element is NaN but the positions below lens."""
    B = len(lens)
    max_pages = max(1, -(-max(lens) // page)) + slack
    n_pages = B * max_pages + spare
    kc, vc = storage(n_pages, page, Hkv, D, dtype, layout), storage(n_pages, page, Hkv, D, dtype, layout)
    table = torch.randperm(n_pages, generator=g, device="cuda")[:B * max_pages].view(B, max_pages).to(torch.int32)
    for b, n in enumerate(lens):
        j = torch.arange(n, device="cuda")
        at = table[b].long()[j // page], j % page
        kc[at] = torch.randn((n, Hkv, D), generator=g, device="cuda").to(dtype)
        vc[at] = (1.0 + torch.randn((n, Hkv, D), generator=g, device="cuda")).to(dtype)
    return kc, vc, table


DECODE = [
    # dtype, lens, Hq, Hkv, D, page, window, layout
    (BF16, [1], 1, 1, 64, 16, 0, "slot"),
    (BF16, [0], 2, 1, 128, 16, 0, "slot"),
    (F16, [0, 1, 2, 15, 16, 17, 31, 33], 8, 2, 128, 16, 0, "slot"),
    (BF16, [63, 64, 65, 127, 128, 129, 0, 1000], 8, 8, 64, 24, 0, "head"),
    (BF16, [777, 3, 1500], 12, 4, 128, 7, 0, "slot"),
    (F16, [500, 1, 0, 129], 7, 1, 256, 1, 0, "head"),
    (BF16, [500, 90], 20, 1, 256, 100, 0, "slot"),
    (F16, [300, 41, 0], 24, 1, 64, 16, 0, "slot"),
    (BF16, [211], 64, 2, 128, 32, 0, "head"),
    (BF16, [5000, 17, 1], 10, 2, 128, 16, 0, "slot"),
    (BF16, [2000, 100, 0, 64, 65], 8, 2, 128, 16, 65, "slot"),
    (F16, [2000, 100, 1], 8, 2, 64, 24, 1, "head"),
    (BF16, [3000, 2999], 4, 4, 256, 48, 1000, "slot"),
    (BF16, [20011], 4, 1, 128, 16, 0, "slot"),
    (F16, [9000, 70000], 16, 2, 64, 64, 0, "head"),
    (BF16, [4097, 8193], 16, 2, 256, 256, 0, "slot"),
    # every number of query heads that one warp, or a team of warps, takes together
    (BF16, [700, 0, 33], 40, 1, 128, 16, 0, "slot"),
    (F16, [129, 5000], 33, 1, 256, 16, 0, "head"),
    (BF16, [300, 1, 9000], 130, 1, 64, 16, 0, "slot"),
    (BF16, [90, 2577], 24, 1, 256, 48, 0, "slot"),
    (F16, [1000, 3333], 32, 1, 64, 100, 0, "head"),
    (BF16, [4097, 100], 70, 1, 256, 16, 300, "slot"),
    (BF16, [5001, 6], 34, 2, 256, 16, 0, "slot"),
    (F16, [7000, 65], 46, 2, 128, 16, 0, "slot"),
]


@pytest.mark.parametrize("dtype,lens,Hq,Hkv,D,page,window,layout", DECODE)
def test_decode(dtype, lens, Hq, Hkv, D, page, window, layout):
    g = gen(sum(lens) + Hq)
    kc, vc, table = make_cache(lens, Hkv, D, page, dtype, layout, g)
    q = (2 * torch.randn((len(lens), Hq, D), generator=g, device="cuda")).to(dtype)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    check_decode(kc, vc, table, q, n, window=window)


def test_decode_many_sequences():
    """More sequences than SMs, most of them short; lengths in the hundreds of kinds."""
    g = gen(5)
    lens = [(i * 37) % 301 for i in range(700)]
    kc, vc, table = make_cache(lens, 2, 64, 16, BF16, "slot", g)
    q = torch.randn((700, 6, 64), generator=g, device="cuda").to(BF16)
    check_decode(kc, vc, table, q, torch.tensor(lens, dtype=torch.int32, device="cuda"))


def test_decode_rising_scores():
    """Scores that rise along the sequence by hundreds: the running maximum keeps moving, early sums vanish."""
    g = gen(6)
    n, D = 3001, 128
    kc, vc, table = make_cache([n], 1, D, 16, BF16, "slot", g)
    j = torch.arange(n, device="cuda")
    at = table[0].long()[j // 16], j % 16
    kc[at] = (j[:, None, None] / n).expand(n, 1, D).to(BF16)
    for sign in (1.0, -1.0):
        q = torch.full((1, 3, D), 4.0 * sign, device="cuda").to(BF16)
        check_decode(kc, vc, table, q, torch.tensor([n], dtype=torch.int32, device="cuda"), scale=1.0)


def test_decode_strided_scaled_clamped():
    """Queries inside a fused projection, outputs inside a wider buffer, a scale, lengths beyond the table."""
    g = gen(7)
    kc, vc, table = make_cache([160, 160, 160], 2, 128, 16, F16, "slot", g, slack=0)
    x = torch.randn((3, 12, 128), generator=g, device="cuda").to(F16)
    wide = torch.full((3, 10, 256), NAN, dtype=F16, device="cuda")
    lens = torch.tensor([2 ** 31 - 1, -5, 161], dtype=torch.int32, device="cuda")
    check_decode(kc, vc, table, x[:, 2:10], lens, scale=0.3, out=wide[:, 1:9, 128:])
    assert bool(torch.isnan(wide[:, :, :128]).all()) and bool(torch.isnan(wide[:, 0]).all())


def test_decode_absent_pages():
    """Page ids outside the pool take no part, a whole sequence of them included."""
    g = gen(8)
    lens = [900, 300, 64, 500]
    kc, vc, table = make_cache(lens, 2, 64, 24, BF16, "slot", g)
    table[0, 3], table[0, 4], table[0, 11], table[0, 37] = -1, kc.shape[0], 2 ** 31 - 1, -2 ** 31
    table[1] = -1
    q = torch.randn((4, 4, 64), generator=g, device="cuda").to(BF16)
    out, lse = check_decode(kc, vc, table, q, torch.tensor(lens, dtype=torch.int32, device="cuda"))
    assert bool((out[1] == 0).all()) and bool((lse[1] == -INF).all())


def test_decode_non_finite_positions():
    """Infinities and NaN that are attended to act as in the formula; a masked score of -inf has no weight."""
    g = gen(9)
    kc, vc, table = make_cache([200] * 4, 1, 64, 16, BF16, "slot", g)
    q = torch.randn((4, 2, 64), generator=g, device="cuda").to(BF16)
    q[:, :, 0] = 1.0
    kc[table[0, 3].long(), 5, 0, 0] = -INF    # one score -inf: no weight
    kc[table[1, 3].long(), 5, 0, 0] = NAN     # NaN anywhere attended: NaN
    vc[table[2, 0].long(), 1, 0, 7] = INF     # an infinite value: its column
    kc[table[3].long(), :, 0, 0] = -INF       # every score -inf: nothing attended
    out = torch.zeros((4, 2, 64), dtype=BF16, device="cuda")
    lse = torch.zeros((4, 2), device="cuda")
    n = torch.full((4,), 200, dtype=torch.int32, device="cuda")
    pe.decode_attn(pe.KVCache(kc, vc, table), q, n, out, lse=lse)
    r, rl, ds, ab = plain_decode(kc, vc, table, q, n, 0.125, 0)
    assert bool(torch.isfinite(out[0]).all())
    assert torch.allclose(out[0].double(), r[0], atol=2.0 ** -8 * 4) and torch.allclose(lse[0].double(), rl[0], atol=1e-4)
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(lse[1]).all())
    assert not bool(torch.isfinite(out[2, :, 7]).any()) and bool(torch.isfinite(out[2, :, :7]).all())
    assert bool((out[3] == 0).all()) and bool((lse[3] == -INF).all())


def test_offsets_past_32_bits():
    """A pool of more than 2^31 elements: pages at its far end are written and read."""
    page, D, Hkv = 64, 256, 8
    n_pages = 2 ** 31 // (page * D * Hkv) + 40
    kc = torch.empty((n_pages, page, Hkv, D), dtype=BF16, device="cuda")
    vc = torch.empty_like(kc)
    g = gen(10)
    table = torch.stack([torch.arange(n_pages - 6, n_pages - 3, device="cuda"), torch.arange(0, 3, device="cuda")]).to(torch.int32)
    n = 150
    k = torch.randn((2 * n, Hkv, D), generator=g, device="cuda").to(BF16)
    v = torch.randn((2 * n, Hkv, D), generator=g, device="cuda").to(BF16)
    seqs = (torch.arange(2 * n, device="cuda") // n).to(torch.int32)
    pos = (torch.arange(2 * n, device="cuda") % n).to(torch.int32)
    cache = pe.KVCache(kc, vc, table)
    pe.kv_append(cache, k, v, pos, seqs=seqs)
    at = table[seqs.long(), pos.long() // page].long(), pos.long() % page
    assert torch.equal(kc[at], k) and torch.equal(vc[at], v)
    q = torch.randn((2, 16, D), generator=g, device="cuda").to(BF16)
    check_decode(kc, vc, table, q, torch.tensor([n, n - 1], dtype=torch.int32, device="cuda"))


def test_decode_stream_workspace_and_repeat():
    """On a side stream, with a workspace full of NaN and without one, the same bits each time."""
    g = gen(11)
    lens = [6000, 1, 0, 900]
    kc, vc, table = make_cache(lens, 2, 128, 16, BF16, "slot", g)
    q = torch.randn((4, 8, 128), generator=g, device="cuda").to(BF16)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    a, la = check_decode(kc, vc, table, q, n)
    cache = pe.KVCache(kc, vc, table)
    ws = torch.full((pe.decode_attn_workspace_bytes(cache, 8) // 4 + 64,), NAN, device="cuda").view(torch.uint8)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    for w in (ws, None):
        out, lse = torch.full_like(a, NAN), torch.full_like(la, NAN)
        st.wait_stream(torch.cuda.current_stream())
        pe.decode_attn(cache, q, n, out, lse=lse, workspace=w, stream=st)
        st.synchronize()
        assert torch.equal(out, a) and torch.equal(lse, la)


def test_decode_graph_replay_with_growing_lengths():
    """A captured step follows lengths, pages and queries that change in place."""
    g = gen(12)
    kc, vc, table = make_cache([2500, 2500], 2, 64, 16, BF16, "slot", g)
    q = torch.randn((2, 4, 64), generator=g, device="cuda").to(BF16)
    n = torch.tensor([1, 2], dtype=torch.int32, device="cuda")
    cache = pe.KVCache(kc, vc, table)
    out = torch.zeros((2, 4, 64), dtype=BF16, device="cuda")
    ws = pe.alloc_workspace(pe.decode_attn_workspace_bytes(cache, 4))
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        pe.decode_attn(cache, q, n, out, workspace=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            pe.decode_attn(cache, q, n, out, workspace=ws)
    torch.cuda.synchronize()
    for lens in ([1, 2], [2500, 0], [77, 2499]):
        n.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        want = torch.empty_like(out)
        pe.decode_attn(cache, q, n, want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


# ---------------------------------------------------------------------------
# log-probabilities
# ---------------------------------------------------------------------------
def plain_logp(x, tokens, scale, k):
    scale = f32(scale)
    z = x.double() * scale
    m = z.amax(1, keepdim=True)
    empty = m == -INF
    d = torch.where(empty, -INF, z - torch.where(empty, 0.0, m))
    e = torch.exp(d)
    S = e.sum(1, keepdim=True)
    ln = torch.log(S)
    lp = torch.where(empty, -INF, d - ln)
    ent = torch.where(empty[:, 0], 0.0, (ln - (torch.where(d == -INF, 0.0, e * d)).sum(1, keepdim=True) / S)[:, 0])
    t = tokens.long()
    has = (t >= 0) & (t < x.shape[1])
    logp = torch.where(has, lp.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0], 0.0)
    lse = torch.where(empty, -INF, m + ln)[:, 0]
    ids = torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :k]
    return logp, ent, lse, lp.gather(1, ids), ids.to(torch.int32)


def check_logp(x, tokens, scale=1.0, k=0, stream=None):
    n = x.shape[0]
    logp, ent, lse = (torch.full((n,), NAN, device="cuda") for _ in range(3))
    tl = torch.full((n, k), NAN, device="cuda") if k else None
    ti = torch.full((n, k), -1, dtype=torch.int32, device="cuda") if k else None
    pe.token_logp(x, tokens, logp, entropy=ent, lse=lse, top_logp=tl, top_id=ti, scale=scale, stream=stream)
    r = plain_logp(x, tokens, scale, k)
    m = x.double().amax(1).abs() * scale
    m = torch.where(torch.isfinite(m), m, 0.0)
    for got, ref in zip((logp, ent, lse), r):
        close(got, ref, 2.0 ** -18 * (1 + torch.where(torch.isfinite(ref), ref.abs(), 0.0)) + 2.0 ** -22 * m)
    if k:
        assert torch.equal(ti, r[4])
        close(tl, r[3], 2.0 ** -18 * (1 + torch.where(torch.isfinite(r[3]), r[3].abs(), 0.0)) + 2.0 ** -22 * m[:, None])
    return logp, ent, lse


def logits(n, V, dtype, pad, seed, spread=3.0):
    """Rows inside a wider buffer whose padding is NaN."""
    x = torch.full((n, V + pad), NAN, device="cuda").to(dtype)
    x[:, :V] = (spread * torch.randn((n, V), generator=gen(seed), device="cuda")).to(dtype)
    return x[:, :V]


def targets(n, V, seed):
    t = torch.randint(0, V, (n,), generator=gen(seed + 1), device="cuda").to(torch.int32)
    if n > 2:
        t[1], t[2] = -1, V
    return t


LOGP = [(1, 1, 0, 1), (3, 2, 1, 2), (5, 7, 2, 5), (4, 31, 0, 31), (2, 33, 3, 32), (700, 16, 0, 4), (9, 255, 1, 20),
        (33, 1000, 0, 0), (3, 4097, 5, 32), (1, 32000, 0, 20), (400, 4099, 0, 7), (2, 50001, 3, 20), (1, 131072, 0, 20),
        (1, 262147, 0, 1), (12, 131071, 1, 0), (170, 65536, 8, 5), (2000, 700, 3, 3)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,V,pad,k", LOGP)
def test_logp(dtype, n, V, pad, k):
    x = logits(n, V, dtype, pad, n + V)
    check_logp(x, targets(n, V, V), k=k)
    if V in (33, 4097, 50001):
        check_logp(x, targets(n, V, V), k=k, scale=0.37)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("V", [5, 200, 4096, 40000])
def test_logp_hard_rows(dtype, V):
    """Ties, masks, lowest values, empty rows, rising and falling rows, non-finite rows."""
    g = gen(V)
    low = torch.finfo(dtype).min
    big = torch.finfo(dtype).max
    j = torch.arange(V, device="cuda", dtype=torch.float32)
    some = torch.rand(V, generator=g, device="cuda") < 0.5
    some[0], some[V - 1] = True, False
    r = torch.randn(V, generator=g, device="cuda")
    one = torch.full((V,), -INF, device="cuda")
    one[V - 1] = -3.0
    rows = [torch.full((V,), 1.5, device="cuda"),             # all equal
            torch.round(r),                                   # many ties
            torch.where(some, -INF, r),                       # masked by -inf
            torch.where(some, low, r),                        # masked by the lowest value
            torch.full((V,), -INF, device="cuda"),            # empty
            torch.full((V,), low, device="cuda"),             # all lowest: uniform
            torch.where(some, -INF, low),                     # lowest and -inf: uniform over the lowest
            j * (20.0 / V), -j * (20.0 / V),                  # rising, falling
            one,                                              # one token left
            r + 40.0 * (j == V // 2),                         # nearly certain
            torch.where(some, r, 0.0 * r) * 0.0,              # signed zeros
            torch.where(j == V // 3, INF, r),                 # +inf: NaN
            torch.where(j == V - 1, NAN, r),                  # NaN
            r * (big / 8.0),                                  # near the type's range
            1000.0 + r]
    x = torch.stack([t.to(dtype) for t in rows])
    t = torch.randint(0, V, (len(rows),), generator=g, device="cuda").to(torch.int32)
    logp, ent, lse = (torch.full((len(rows),), NAN, device="cuda") for _ in range(3))
    k = min(V, 32)
    tl, ti = torch.empty((len(rows), k), device="cuda"), torch.empty((len(rows), k), dtype=torch.int32, device="cuda")
    finite = [i for i in range(len(rows)) if i not in (12, 13)]
    check_logp(x[finite].contiguous(), t[finite].contiguous(), k=k)
    pe.token_logp(x, t, logp, entropy=ent, lse=lse, top_logp=tl, top_id=ti)
    assert bool(torch.isnan(torch.stack([logp, ent, lse])[:, 12:14]).all())
    want = torch.sort(x.float(), dim=1, descending=True, stable=True)[1][:, :k].to(torch.int32)
    assert torch.equal(ti, want)
    # a padding row of an empty or NaN distribution still has logp 0
    t[4] = t[13] = -1
    pe.token_logp(x, t, logp)
    assert float(logp[4]) == 0.0 and float(logp[13]) == 0.0


@pytest.mark.parametrize("n,V", [(3, 5000), (1, 100000), (300, 333)])
def test_logp_parts_and_streams(n, V):
    """Each output alone gives the bits of all together, on a side stream too."""
    x, t = logits(n, V, BF16, 3, 9), targets(n, V, 9)
    all_ = check_logp(x, t, k=4)
    st = torch.cuda.Stream()
    for i, name in enumerate(("logp", "entropy", "lse")):
        got = torch.full((n,), NAN, device="cuda")
        st.wait_stream(torch.cuda.current_stream())
        pe.token_logp(x, t if i == 0 else None, got if i == 0 else None, **({name: got} if i else {}), stream=st)
        st.synchronize()
        assert torch.equal(got, all_[i])


def test_logp_rows_past_32_bits():
    """Rows that lie more than 2^31 elements into the buffer."""
    n, V = 17, 1 << 27
    x = torch.empty((n, V), dtype=BF16, device="cuda")
    y = x[:, :3001]
    y.copy_(torch.randn(y.shape, generator=gen(3), device="cuda"))
    t = targets(n, 3001, 3)
    _, ent, lse = check_logp(y, t, k=3)
    d = torch.empty_like(x)[:, :3001]
    gl, ge = torch.randn(n, generator=gen(4), device="cuda"), torch.randn(n, generator=gen(5), device="cuda")
    check_grad(y, t, lse, ent, gl, ge, 1.0, d)


# ---------------------------------------------------------------------------
# gradient
# ---------------------------------------------------------------------------
def plain_grad(x, t, lse, ent, gl, ge, scale):
    """(gradient, size of its terms) of sum gl logp + ge entropy in 64 bits, from the lse and entropy that the
    operator is given."""
    scale = f32(scale)
    z = x.double() * scale
    lse = lse.double()[:, None]
    lnp = torch.where(lse == -INF, -INF, z - torch.where(lse == -INF, 0.0, lse))
    p = torch.exp(lnp)
    has = (t >= 0) & (t < x.shape[1])
    g = torch.where(has, gl.double(), 0.0)[:, None] if gl is not None else torch.zeros_like(lse)
    e = ge.double()[:, None] if ge is not None else torch.zeros_like(lse)
    H = ent.double()[:, None]
    lnp0 = torch.where(p == 0, 0.0, lnp)
    d = -p * g - e * p * (lnp0 + H)
    one = torch.zeros_like(d)
    rows = torch.arange(len(t), device="cuda")[has & (lse[:, 0] != -INF)]
    one[rows, t[rows].long()] = 1.0
    size = p * (g.abs() + e.abs() * (lnp0.abs() + H.abs()))
    return scale * (d + one * g), scale * size


def check_grad(x, t, lse, ent, gl, ge, scale, out):
    ref, size = plain_grad(x, t, lse, ent, gl, ge, scale)
    pe.token_logp_grad(x, t if gl is not None else None, lse, out, g_logp=gl, entropy=ent if ge is not None else None,
                       g_entropy=ge, scale=scale)
    l = torch.where(torch.isfinite(lse), lse.abs(), 0.0).double()[:, None]
    dt = out.dtype
    close(out, ref, U[dt] * ref.abs() + TINY[dt] + 2.0 ** -126 + size * (2.0 ** -18 + 2.0 ** -22 * l))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("n,V,pad", [(1, 1, 0), (3, 2, 1), (5, 33, 0), (4, 255, 3), (300, 16, 0), (2, 4099, 0),
                                     (3, 50001, 5), (1, 131072, 0), (64, 8192, 8), (1000, 700, 1)])
def test_grad(dtype, n, V, pad):
    x, t = logits(n, V, dtype, pad, n * V), targets(n, V, V)
    gl = torch.randn(n, generator=gen(1), device="cuda")
    ge = torch.randn(n, generator=gen(2), device="cuda")
    for scale in (1.0, 0.6):
        _, ent, lse = check_logp(x, t, scale=scale)
        wide = torch.full((n, V + pad), 5.0, dtype=dtype, device="cuda")
        check_grad(x, t, lse, ent, gl, ge, scale, wide[:, :V])
        assert bool((wide[:, V:] == 5.0).all())
        odd = torch.full((n * V + 1,), 5.0, dtype=dtype, device="cuda")[1:].view(n, V)  # other alignment than the logits'
        check_grad(x, t, lse, ent, gl, ge, scale, odd)
        assert torch.equal(odd, wide[:, :V])
        check_grad(x, t, lse, ent, gl, None, scale, odd)
        check_grad(x, t, lse, ent, None, ge, scale, odd)
        y = x.clone()
        pe.token_logp_grad(y, t, lse, y, g_logp=gl, entropy=ent, g_entropy=ge, scale=scale)
        assert torch.equal(y, wide[:, :V])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_grad_hard_rows(dtype):
    V = 1003
    g = gen(77)
    r = 3 * torch.randn(V, generator=g, device="cuda")
    some = torch.rand(V, generator=g, device="cuda") < 0.5
    one = torch.full((V,), -INF, device="cuda")
    one[11] = 2.0
    x = torch.stack([t.to(dtype) for t in (torch.full((V,), -INF, device="cuda"), torch.where(some, -INF, r),
                                           torch.where(some, torch.finfo(dtype).min, r), one,
                                           torch.full((V,), 0.25, device="cuda"), r + 30 * (torch.arange(V, device="cuda") == 5))])
    n = x.shape[0]
    t = torch.tensor([3, int(torch.nonzero(some)[0]), 7, 11, 0, 5], dtype=torch.int32, device="cuda")
    gl, ge = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
    _, ent, lse = check_logp(x, t)
    out = torch.empty_like(x)
    check_grad(x, t, lse, ent, gl, ge, 1.0, out)
    assert bool((out[0] == 0).all())


def test_grad_against_differences():
    """Central differences of the 64-bit objective at every coordinate of a few rows."""
    n, V, scale, h = 4, 23, 0.8, 1e-5
    x = logits(n, V, F32, 0, 13, spread=1.5)
    t = torch.tensor([3, -1, 22, 0], dtype=torch.int32, device="cuda")
    gl, ge = torch.randn(n, generator=gen(1), device="cuda"), torch.randn(n, generator=gen(2), device="cuda")
    _, ent, lse = check_logp(x, t, scale=scale)
    out = torch.empty_like(x)
    pe.token_logp_grad(x, t, lse, out, g_logp=gl, entropy=ent, g_entropy=ge, scale=scale)

    def objective(y):
        lp, e = plain_logp(y, t, scale, 0)[:2]
        return gl.double() * lp + ge.double() * e

    for j in range(V):
        d = torch.zeros((n, V), dtype=torch.float64, device="cuda")
        d[:, j] = h
        diff = (objective(x.double() + d) - objective(x.double() - d)) / (2 * h)
        # a third derivative of at most a few units times h^2, the subtraction's 2^-52 / h, and fp32
        assert float((out[:, j].double() - diff).abs().max()) < 1e-5


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
def test_generation_loop_matches_whole_sequence():
    """Twenty tokens appended one by one and attended to, against one causal evaluation in 64 bits."""
    B, Hq, Hkv, D, page, steps = 3, 4, 2, 64, 8, 20
    g = gen(21)
    max_pages = 3
    kc, vc = storage(B * max_pages, page, Hkv, D, BF16, "slot"), storage(B * max_pages, page, Hkv, D, BF16, "slot")
    table = torch.randperm(B * max_pages, generator=g, device="cuda").view(B, max_pages).to(torch.int32)
    cache, rot = pe.KVCache(kc, vc, table), pe.rot_table(steps, D)
    qkv = torch.randn((steps, B, Hq + 2 * Hkv, D), generator=g, device="cuda").to(BF16)
    outs, qs = [], []
    for i in range(steps):
        q, k, v = qkv[i, :, :Hq], qkv[i, :, Hq:Hq + Hkv], qkv[i, :, Hq + Hkv:]
        pos = torch.full((B,), i, dtype=torch.int32, device="cuda")
        q_out, out = torch.empty((B, Hq, D), dtype=BF16, device="cuda"), torch.empty((B, Hq, D), dtype=BF16, device="cuda")
        pe.kv_append(cache, k, v, pos, q=q, q_out=q_out, rot=rot)
        pe.decode_attn(cache, q_out, pos + 1, out)
        outs.append(out)
        qs.append(q_out)
    for i in range(steps):
        r, _, ds, ab = plain_decode(kc, vc, table, qs[i], torch.full((B,), i + 1), D ** -0.5, 0)
        close(outs[i], r, 2.0 ** -8 * r.abs() + (2.0 ** -19 * ds + 2.0 ** -14)[..., None] * ab)


def test_example_learns():
    """The example's loop: the log-probabilities of sampling and scoring agree, and the reward rises."""
    import importlib.util
    import os

    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "grpo_tokens.py")
    spec = importlib.util.spec_from_file_location("grpo_tokens", path)
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    rows = ex.main(batches=12, tokens=24)
    assert len({r["sequences"] for r in rows}) > 1
    assert all(r["drift"] < 0.05 and r["entropy"] >= 0.0 for r in rows)
    first, last = (sum(r["reward"] for r in x) / 3 for x in (rows[:3], rows[-3:]))
    assert last > first + 0.05, (first, last)


@pytest.mark.parametrize("n,V", [(3, 40000), (500, 1000), (64, 9001)])
def test_chain_of_calls_needs_no_wait(n, V):
    """Scoring and gradient in place, over and over, without a wait in between: each sees what the last one wrote."""
    def chain(wait):
        x, t = logits(n, V, F32, 3, 31, spread=1.0), targets(n, V, 31)
        logp, ent, lse = (torch.empty(n, device="cuda") for _ in range(3))
        gl, ge = torch.full((n,), 3.0, device="cuda"), torch.full((n,), 0.5, device="cuda")
        for _ in range(12):
            pe.token_logp(x, t, logp, entropy=ent, lse=lse)
            if wait:
                torch.cuda.synchronize()
            pe.token_logp_grad(x, t, lse, x, g_logp=gl, entropy=ent, g_entropy=ge)
            if wait:
                torch.cuda.synchronize()
        return x, logp, ent, lse

    a = chain(True)
    for _ in range(3):
        assert all(torch.equal(p, q) for p, q in zip(chain(False), a))
