"""The 8-bit cache and the operators of drafted tokens against plain evaluations
in 64 bits (GPU).

Tolerances, from the arithmetic that include/pe.h states:
  u = 2^-8 (bf16), 2^-11 (fp16): one rounding of the result, |x| u.
  append, 8 bits: a key's rotation is three fp32 roundings, er = 3 * 2^-24
    (|a c| + |b s|); the scale is the least power of two that brings the row
    within 448, for a row within er of what it is; a code is off by half a step,
    2^-4 of the element or 2^-10 of the scale.  Values have er = 0: their bytes
    are those of the definition.
  attention: a score's error is at most ds = 2^-20 scale max_j sum_d |q_d k_jd|
    (fp32 products and sums), and for an 8-bit cache what its fp16 form loses
    below 2^-24 of the largest scale, 2^-24 scale max_j s_j sum_d |q_d|, in the
    keys and 2^-24 max_j t_j in the values; weights and their sums are off by a
    factor e^(2 ds), by the rounding to 16 bits w (2^-8 in a bf16 cache, 2^-11 in
    the others), and by 2^-14 for exponentials and sums; in fp16 weights below
    2^-30 of the largest may be missing:
    |out - ref| <= u |ref| + (2 ds + w + 2^-14) sum_j p_j |v_j| + n 2^-30 max |v|.
    |lse - ref| <= ds + 2^-18 (1 + |ref|).
"""
import math

import pytest
import torch

from paper_2608_11226_gb300 import pe

pytestmark = pytest.mark.gpu

BF16, F16, E4M3 = torch.bfloat16, torch.float16, torch.float8_e4m3fn
U = {BF16: 2.0 ** -8, F16: 2.0 ** -11}
NAN, INF = float("nan"), float("inf")


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def close(got, ref, tol):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf])
    ok = torch.isfinite(ref)
    bad = ok & ~((got - ref).abs() <= tol)
    assert not bad.any(), f"{int(bad.sum())} values off, the worst by {((got - ref).abs() - tol)[ok].max().item():.3g}"


def laid(shape, layout, dtype, fill):
    """[pages, slots, heads, ...] storage, heads ahead of slots in memory where layout is "head"."""
    if layout == "head":
        shape = (shape[0], shape[2], shape[1], *shape[3:])
    x = torch.full(shape, fill, dtype=dtype, device="cuda")
    return x.transpose(1, 2) if layout == "head" else x


def scale_values(byte):
    f = torch.exp2(byte.double().clamp(63, 247) - 127.0)
    return torch.where(byte == 255, NAN, f)


def quantise64(x):
    """(codes' values, scale bytes) of 64-bit rows by the definition."""
    a = x.abs().amax(-1)
    e = torch.full(a.shape, -64, dtype=torch.int64, device=x.device)
    for k in range(-63, 121):
        e = torch.where(a > 448.0 * 2.0 ** (k - 1), k, e)
    y = x / torch.exp2(e.double())[..., None]
    step = torch.exp2((torch.frexp(y)[1] - 4).clamp(min=-9).double())
    codes = torch.round(y / step) * step
    bad = ~torch.isfinite(x).all(-1)
    return torch.where(bad[..., None], 0.0, codes), torch.where(bad, 255, e + 127)


class Pool:
    """A cache with everything around it: 16 bits of `dtype`, or 8 bits."""

    def __init__(self, n_seqs, max_pages, page, heads, D, dtype, eight, layout, seed, fill=None, spare=1):
        g = gen(seed)
        n = n_seqs * max_pages + spare
        self.page, self.D = page, D
        self.table = torch.randperm(n, generator=g, device="cuda")[:n_seqs * max_pages].view(n_seqs, max_pages).to(torch.int32)
        shape = (n, page, heads, D)
        if eight:
            codes, scales = [], []
            for _ in range(2):
                x = laid(shape, layout, torch.uint8, 0)
                x.copy_((torch.randn(shape, generator=g, device="cuda") * 60).clamp(-448, 448).to(E4M3).view(torch.uint8))
                sc = laid(shape[:3], layout, torch.uint8, 0)
                sc.copy_(torch.randint(118, 124, shape[:3], generator=g, device="cuda"))
                codes.append(x.view(E4M3))
                scales.append(sc)
            self.k, self.v = codes
            self.ks, self.vs = scales
            self.cache = pe.KVCache(self.k, self.v, self.table, self.ks, self.vs)
        else:
            self.ks = self.vs = None
            self.k, self.v = (laid(shape, layout, dtype, 0.0) for _ in range(2))
            for x in (self.k, self.v):
                x.copy_(torch.randn(shape, generator=g, device="cuda"))
            self.cache = pe.KVCache(self.k, self.v, self.table)

    def spoil(self, keep):
        """NaN in every slot that `keep` ([pages, slots] bool) does not name."""
        for x in (self.k, self.v):
            if self.ks is None:
                x[~keep] = NAN
            else:
                x.view(torch.uint8)[~keep] = 0x7F
        for s in (self.ks, self.vs):
            if s is not None:
                s[~keep] = 255

    def rows(self, b, positions):
        """64-bit keys and values [positions, heads, D] of a sequence, scales [positions, heads], and which are there."""
        p = torch.as_tensor(positions, device="cuda", dtype=torch.int64)
        page = self.table[b].long()[p // self.page]
        there = (page >= 0) & (page < self.k.shape[0])
        page, slot = page.clamp(0, self.k.shape[0] - 1), p % self.page
        out = []
        for x, s in ((self.k, self.ks), (self.v, self.vs)):
            if s is None:
                out += [x[page, slot].double(), None]
            else:
                f = scale_values(s[page, slot])
                out += [x.view(torch.uint8)[page, slot].view(E4M3).double() * f[..., None], f]
        return out[0], out[2], out[1], out[3], there


# ---------------------------------------------------------------------------
# append into 8 bits, and at slots
# ---------------------------------------------------------------------------
def turned(x, rot, pos, inter):
    """64-bit rotation of [T, heads, D] rows, and the sizes of its terms."""
    y, ab = x.double().clone(), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    if rot is None:
        return y, ab
    h = rot.shape[1] // 2
    i = torch.arange(h, device="cuda")
    lo, hi = (2 * i, 2 * i + 1) if inter else (i, i + h)
    r = rot.double()[pos.clamp(0, rot.shape[0] - 1).long()][:, None]
    c, s, a, b = r[..., :h], r[..., h:], y[..., lo], y[..., hi]
    y[..., lo], y[..., hi] = a * c - b * s, b * c + a * s
    ab[..., lo], ab[..., hi] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return y, ab


APPEND = [
    # dtype, T, n_seqs, Hq, Hkv, D, page, rot_dim, interleaved, layout
    (BF16, 1, 1, 1, 1, 64, 16, 64, False, "slot"),
    (BF16, 32, 32, 8, 2, 128, 16, 128, False, "slot"),
    (F16, 37, 3, 6, 3, 64, 5, 32, True, "head"),
    (BF16, 65, 2, 5, 1, 256, 24, 256, False, "head"),
    (F16, 19, 4, 4, 4, 128, 1, 16, True, "slot"),
    (BF16, 7, 7, 3, 3, 128, 16, 0, False, "slot"),
    (F16, 300, 3, 40, 8, 128, 32, 64, False, "slot"),
    (BF16, 2500, 5, 7, 5, 64, 100, 48, True, "head"),
]


@pytest.mark.parametrize("dtype,T,n_seqs,Hq,Hkv,D,page,rd,inter,layout", APPEND)
@pytest.mark.parametrize("at_slots", [False, True])
def test_append8(dtype, T, n_seqs, Hq, Hkv, D, page, rd, inter, layout, at_slots):
    g = gen(T + D)
    per = -(-T // n_seqs) + 5
    max_pages = -(-per // page)
    P = Pool(n_seqs, max_pages, page, Hkv, D, dtype, True, layout, T)
    before = [t.clone() for t in (P.k.view(torch.uint8), P.v.view(torch.uint8), P.ks, P.vs)]
    order = torch.randperm(T, generator=g, device="cuda")
    seqs, slots = (order % n_seqs).to(torch.int32), (order // n_seqs + 2).to(torch.int32)
    pos = torch.randint(0, 50, (T,), generator=g, device="cuda").to(torch.int32) if at_slots else slots.clone()
    if T >= 19:  # padding, out-of-range tokens, a page that is not there
        (slots if at_slots else pos)[1] = -1
        (slots if at_slots else pos)[2] = max_pages * page
        seqs[3], seqs[4] = -1, n_seqs
        P.table[-1, -1] = -1 if T % 2 else P.k.shape[0]
        if at_slots:
            pos[5] = -3
            if rd:
                pos[6] = 64
    rot = pe.rot_table(64 if at_slots else per + 1, rd) if rd else None
    x = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device="cuda")
    x *= torch.exp2(torch.randint(-12, 6, (T, Hq + 2 * Hkv, 1), generator=g, device="cuda").float())
    if dtype == BF16:
        x[0] *= 1e-22  # below the least scale
    x[T // 2, :, :] = 0.0
    x = x.to(dtype)
    if T >= 19:
        x[7, Hq, 3], x[8, Hq + Hkv, D - 1], x[9, Hq, 0] = NAN, INF, -INF
        x[10, Hq:, :2] = 448.0 if dtype == F16 else 1.75 * 2.0 ** 100  # a row whose largest is on the border
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    rq, qa = turned(q, rot, pos, inter)
    rk, ka = turned(k, rot, pos, inter)
    at = slots if at_slots else pos
    ok = (pos >= 0) & (at >= 0) & (at < max_pages * page) & (seqs >= 0) & (seqs < n_seqs)
    if rd:
        ok &= pos < rot.shape[0]
    q_out = torch.full((T, Hq, D), NAN, dtype=dtype, device="cuda")
    pe.kv_append(P.cache, k, v, pos, seqs=seqs, q=q, q_out=q_out, rot=rot, interleaved=inter, slots=slots if at_slots else None)
    rq[~ok], qa[~ok] = 0.0, 0.0
    close(q_out, rq, U[dtype] * rq.abs() + 3 * 2.0 ** -24 * qa + (2.0 ** -25 if dtype == F16 else 0.0))

    page_of = P.table[seqs.clamp(0, n_seqs - 1).long(), (at.clamp(0, max_pages * page - 1) // page).long()]
    live = ok & (page_of >= 0) & (page_of < P.k.shape[0])
    gp, gs = page_of[live].long(), (at[live] % page).long()
    # values: the bytes of the definition
    codes, byte = quantise64(v[live].double())
    assert torch.equal(P.vs[gp, gs].long(), byte)
    assert torch.equal(P.v.view(torch.uint8)[gp, gs].view(E4M3).double(), codes)
    # keys: within the rotation's rounding
    ref, er = rk[live], 3 * 2.0 ** -24 * ka[live]
    fine = torch.isfinite(ref).all(-1)
    gb = P.ks[gp, gs].long()
    assert torch.equal(gb == 255, ~fine)
    e = torch.exp2(gb.double() - 127.0)
    a, ae = ref.abs().amax(-1), er.amax(-1)
    assert ((a - ae <= 448.0 * e) & ((a + ae > 224.0 * e) | (gb == 63)))[fine].all()
    got = P.k.view(torch.uint8)[gp, gs].view(E4M3).double()
    assert (got[~fine] == 0).all()
    close((got * e[..., None])[fine], ref[fine], (torch.maximum(ref.abs() * 2.0 ** -4, e[..., None] * 2.0 ** -10) + er)[fine])
    # nothing else was written
    touched = torch.zeros(P.k.shape[:2], dtype=torch.bool, device="cuda")
    touched[gp, gs] = True
    for now, was in zip((P.k.view(torch.uint8), P.v.view(torch.uint8), P.ks, P.vs), before):
        assert torch.equal(now[~touched], was[~touched])


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_append_at_slots_of_a_16_bit_cache(dtype):
    """The rows of a plain append, at other places."""
    g = gen(3)
    T, H, D, page = 40, 3, 128, 16
    P, Q = (Pool(2, 4, page, H, D, dtype, False, "slot", 8) for _ in range(2))
    k, v, q = (torch.randn((T, H, D), generator=g, device="cuda").to(dtype) for _ in range(3))
    pos = torch.arange(T, dtype=torch.int32, device="cuda") // 2
    seqs = torch.arange(T, dtype=torch.int32, device="cuda") % 2
    slots = 50 - pos
    rot = pe.rot_table(64, D)
    q1, q2 = q.clone(), q.clone()
    pe.kv_append(P.cache, k, v, pos, seqs=seqs, q=q1, rot=rot)
    pe.kv_append(Q.cache, k, v, pos, seqs=seqs, q=q2, rot=rot, slots=slots)
    assert torch.equal(q1, q2)
    for b in range(2):
        for p in range(20):
            for x, y in ((P.k, Q.k), (P.v, Q.v)):
                assert torch.equal(x[P.table[b, p // page], p % page], y[Q.table[b, (50 - p) // page], (50 - p) % page])


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
def attend(P, q, lens, scale, window, masks=None):
    """(out, lse, tolerances of both) in 64 bits; q [B, N, Hq, D], masks [B, N] ints or None (one token that lens counts)."""
    B, N, Hq, D = q.shape
    Hkv, cap = P.k.shape[2], P.table.shape[1] * P.page
    G = Hq // Hkv
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(q.shape[:-1], -INF, dtype=torch.float64, device="cuda")
    tol, ltol = torch.zeros_like(out), torch.zeros_like(lse)
    u = U[q.dtype]
    w = u if P.ks is None else 2.0 ** -11
    for b in range(B):
        n = min(max(int(lens[b]), 0), cap)
        for i in range(N):
            if masks is None:
                lo, nodes = max(0, n - window) if window else 0, []
            else:
                m = masks[b][i] & ((1 << N) - 1)
                if not m:
                    continue
                nodes = [n + a for a in range(N) if m >> a & 1]
                lo = max(0, n + len(nodes) - window) if window else 0
                nodes = [p for p in nodes if p < cap]
            where = list(range(lo, n)) + nodes
            if not where:
                continue
            k, v, ks, vs, there = P.rows(b, where)
            k, v = k[there], v[there]
            if not len(k):
                continue
            for h in range(Hkv):
                qs = q[b, i, h * G:(h + 1) * G].double()
                z = qs @ k[:, h].T * scale
                hs = slice(h * G, (h + 1) * G)
                lse[b, i, hs] = torch.logsumexp(z, -1)
                p = torch.softmax(z, -1)
                none = (z == -INF).all(-1, keepdim=True)
                o = torch.where(p == 0, 0.0, p) @ v[:, h]
                out[b, i, hs] = torch.where(none, 0.0, o)
                ds = 2.0 ** -20 * abs(scale) * (qs.abs() @ k[:, h].abs().T).amax(-1)
                extra = 2.0 ** -30 * len(k) * v[:, h].abs().max() if w == 2.0 ** -11 else 0.0
                if ks is not None:
                    ds = ds + 2.0 ** -24 * abs(scale) * ks[there][:, h].max() * qs.abs().sum(-1)
                    extra = extra + 2.0 ** -24 * vs[there][:, h].max()
                tol[b, i, hs] = u * o.abs() + ((2 * ds + w + 2.0 ** -14)[:, None] * (p @ v[:, h].abs())) + extra
                ltol[b, i, hs] = ds + 2.0 ** -18 * (1 + lse[b, i, hs].abs())
    return out, lse, tol + (2.0 ** -25 if q.dtype == F16 else 0.0), ltol


def tree_masks(B, N, seed):
    """Trees as lists of ints: a node's ancestors and itself."""
    r = torch.Generator().manual_seed(seed)
    out = []
    for _ in range(B):
        row = [1]
        for i in range(1, N):
            row.append(row[int(torch.randint(0, i, (1,), generator=r))] | 1 << i)
        out.append(row)
    return out


def tensor_of(masks):
    return torch.tensor([[m - (1 << 64) if m >> 63 else m for m in row] for row in masks], dtype=torch.int64, device="cuda")


def kept(P, lens, N):
    """[pages, slots] that some new token may attend to."""
    keep = torch.zeros(P.k.shape[:2], dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        end = min(max(int(n), 0) + N, P.table.shape[1] * P.page)
        p = torch.arange(end, device="cuda")
        page = P.table[b].long()[p // P.page]
        ok = (page >= 0) & (page < keep.shape[0])
        keep[page[ok], (p % P.page)[ok]] = True
    return keep


SHAPES = [
    # dtype, eight, lens, max_pages, page, Hq, Hkv, D, layout
    (BF16, True, [1], 1, 16, 1, 1, 64, "slot"),
    (BF16, True, [700], 44, 16, 8, 2, 128, "slot"),
    (F16, True, [0, 5, 129, 1000], 90, 13, 15, 3, 64, "head"),
    (BF16, True, [33, 0, 257], 20, 24, 20, 1, 256, "slot"),
    (F16, True, [2500, 17], 40, 64, 16, 2, 128, "head"),
    (BF16, True, [127, 128, 129, 255, 256, 257, 1, 0], 5, 64, 32, 1, 128, "slot"),
    (BF16, True, [4000], 63, 64, 6, 6, 64, "head"),
    (F16, True, [1500, 40, 3], 17, 100, 64, 2, 256, "slot"),
    (BF16, True, [-4, 2 ** 31 - 1], 3, 8, 40, 1, 64, "slot"),
]


@pytest.mark.parametrize("dtype,eight,lens,max_pages,page,Hq,Hkv,D,layout", SHAPES)
@pytest.mark.parametrize("window", [0, 1, 100])
def test_decode8(dtype, eight, lens, max_pages, page, Hq, Hkv, D, layout, window):
    B = len(lens)
    P = Pool(B, max_pages, page, Hkv, D, dtype, eight, layout, sum(lens) % 1000 + D)
    P.spoil(kept(P, lens, 0))
    g = gen(D + B)
    q = (2 * torch.randn((B, Hq + 3, D), generator=g, device="cuda")).to(dtype)[:, 2:2 + Hq]
    out = torch.full((B, Hq, D), NAN, dtype=dtype, device="cuda")
    lse = torch.full((B, Hq), NAN, device="cuda")
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pe.decode_attn(P.cache, q, t, out, window=window, lse=lse)
    ro, rl, to, tl = attend(P, q[:, None], lens, D ** -0.5, window)
    close(out, ro[:, 0], to[:, 0])
    close(lse, rl[:, 0], tl[:, 0])
    again = torch.empty_like(out)
    pe.decode_attn(P.cache, q, t, again, window=window)
    assert torch.equal(out, again)


TREES = [
    # dtype, eight, lens, N, max_pages, page, Hq, Hkv, D, layout
    (BF16, False, [0], 1, 1, 16, 1, 1, 64, "slot"),
    (BF16, False, [700], 8, 45, 16, 8, 2, 128, "slot"),
    (F16, False, [0, 5, 129, 1000], 13, 90, 13, 15, 3, 64, "head"),
    (BF16, True, [33, 0, 257], 5, 20, 24, 20, 1, 256, "slot"),
    (F16, True, [2500, 17], 64, 42, 64, 16, 2, 128, "head"),
    (BF16, False, [127, 128, 64, 65, 1], 64, 5, 64, 8, 1, 128, "slot"),
    (BF16, True, [4000, 100], 33, 64, 64, 12, 6, 64, "head"),
    (F16, False, [1500, 40, 3], 37, 17, 100, 16, 2, 256, "slot"),
    (BF16, False, [300], 64, 6, 64, 20, 2, 128, "head"),
    (BF16, True, [600, 0, 90], 64, 11, 64, 8, 1, 128, "slot"),
    (F16, True, [250, 20], 64, 40, 8, 10, 1, 64, "slot"),
    (BF16, False, [200], 31, 8, 32, 16, 1, 256, "slot"),
    (BF16, False, [20, 8], 20, 3, 8, 4, 2, 128, "slot"),       # nodes beyond the table
    (F16, True, [-4, 2 ** 31 - 1, 7], 6, 3, 8, 40, 2, 64, "slot"),
]


@pytest.mark.parametrize("dtype,eight,lens,N,max_pages,page,Hq,Hkv,D,layout", TREES)
@pytest.mark.parametrize("window", [0, 100])
def test_tree(dtype, eight, lens, N, max_pages, page, Hq, Hkv, D, layout, window):
    B = len(lens)
    P = Pool(B, max_pages, page, Hkv, D, dtype, eight, layout, sum(lens) % 1000 + D)
    P.spoil(kept(P, lens, N))
    masks = tree_masks(B, N, N + B)
    if N > 4:  # padding, and bits of nodes that do not exist
        masks[0][-1] = masks[-1][N // 2] = 0
        if N < 64:
            masks[0][1] |= 1 << N
    g = gen(D + B)
    q = (2 * torch.randn((B, N, Hq + 3, D), generator=g, device="cuda")).to(dtype)[:, :, 2:2 + Hq]
    out = torch.full((B, N, Hq, D), NAN, dtype=dtype, device="cuda")
    lse = torch.full((B, N, Hq), NAN, device="cuda")
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pe.tree_attn(P.cache, q, t, tensor_of(masks), out, window=window, lse=lse)
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, window, masks)
    close(out, ro, to)
    close(lse, rl, tl)
    again = torch.empty_like(out)
    pe.tree_attn(P.cache, q, t, tensor_of(masks), again, window=window)
    assert torch.equal(out, again)


@pytest.mark.parametrize("eight,D,Hq,N", [(False, 64, 8, 3), (True, 64, 4, 2), (False, 128, 4, 9), (True, 128, 8, 35), (False, 256, 4, 2),
                                          (False, 128, 12, 50), (True, 256, 8, 40)])
@pytest.mark.parametrize("B,longest", [(90, 300), (3, 9000), (700, 2)])
def test_many_segments(eight, D, Hq, N, B, longest):
    """More tiles than CTAs, cut at every place: many short sequences, few long ones, nothing but trees."""
    H, page = 4, 32
    g = gen(B + D)
    lens = torch.randint(0, longest + 1, (B,), generator=g, device="cuda")
    P = Pool(B, -(-(longest + N) // page), page, H, D, BF16, eight, "slot", B)
    masks = tree_masks(1, N, 7) * B
    q = torch.randn((B, N, Hq, D), generator=g, device="cuda").to(BF16)
    out, lse = torch.full_like(q, NAN), torch.full((B, N, Hq), NAN, device="cuda")
    pe.tree_attn(P.cache, q, lens.to(torch.int32), tensor_of(masks), out, lse=lse)
    pe.device_check()
    some = torch.randperm(B, generator=g, device="cuda")[:6].tolist()  # the plain evaluation of a few, all rows
    whole = P.table
    for b in some:
        P.table = whole[b:b + 1]
        ro, rl, to, tl = attend(P, q[b:b + 1], [int(lens[b])], D ** -0.5, 0, masks[:1])
        close(out[b], ro[0], to[0])
        close(lse[b], rl[0], tl[0])
    assert torch.isfinite(out.float()).all() and torch.isfinite(lse).all()


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("Hq,N,D", [(2, 3, 64), (8, 7, 128), (8, 40, 128), (4, 20, 256), (16, 33, 64)])
def test_what_a_row_does_not_attend_to(eight, Hq, N, D):
    """NaN and infinite rows at absent pages, in the context and in the tree: only who attends sees them."""
    lens, page = [150, 60], 16
    P = Pool(2, 20, page, 2, D, BF16, eight, "slot", 5)
    P.table[0, 3] = -1
    P.table[1, 1] = P.k.shape[0]
    masks = tree_masks(2, N, 9)
    spoiled = min(2, N - 1)  # a node of sequence 0
    at = (int(P.table[0, (150 + spoiled) // page]), (150 + spoiled) % page)
    one = (int(P.table[1, 61 // page]), 61 % page)  # node 1 of sequence 1: an infinite value
    if eight:
        P.ks[at] = 255
        P.v.view(torch.uint8)[one[0], one[1], 1] = 0x7F
    else:
        P.k[at], P.v[at] = NAN, NAN
        P.v[one[0], one[1], 1] = INF
    q = torch.randn((2, N, Hq, D), generator=gen(1), device="cuda").to(BF16)
    out, lse = torch.empty_like(q), torch.empty((2, N, Hq), device="cuda")
    pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), tensor_of(masks), out, lse=lse)
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, 0, masks)
    sees0 = torch.tensor([bool(m >> spoiled & 1) for m in masks[0]], device="cuda")
    sees1 = torch.tensor([bool(m >> 1 & 1) for m in masks[1]], device="cuda")
    assert torch.isnan(out[0, sees0]).all() and torch.isnan(lse[0, sees0]).all()
    assert not torch.isfinite(out[1, sees1, Hq // 2:]).any()
    close(out[0, ~sees0], ro[0, ~sees0], to[0, ~sees0])
    close(lse[0, ~sees0], rl[0, ~sees0], tl[0, ~sees0])
    close(out[1, ~sees1], ro[1, ~sees1], to[1, ~sees1])
    close(out[1, :, :Hq // 2], ro[1, :, :Hq // 2], to[1, :, :Hq // 2])


@pytest.mark.parametrize("D", [64, 128, 256])
def test_window_over_nan(D):
    """A deeper node's window begins later: what lies ahead of it is not used by that node alone."""
    N, n, page, w = 40, 300, 16, 64
    P = Pool(1, 22, page, 1, D, BF16, False, "slot", 5)
    masks = [[(1 << i + 1) - 1 for i in range(N)]]  # a chain
    first = n + 1 - w  # of node 0; node i starts i later
    p = first + 10
    P.v[int(P.table[0, p // page]), p % page] = NAN
    q = torch.randn((1, N, 4, D), generator=gen(2), device="cuda").to(BF16)
    out = torch.empty_like(q)
    pe.tree_attn(P.cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), tensor_of(masks), out, window=w)
    ro, _, to, _ = attend(P, q, [n], D ** -0.5, w, masks)
    assert torch.isnan(out[0, :11]).all()
    close(out[0, 11:], ro[0, 11:], to[0, 11:])


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("Hq,D", [(1, 64), (16, 128), (16, 256)])
def test_large_scores(eight, Hq, D):
    """Scores of a few hundred, far apart, a scale other than the default, and rows of zeros."""
    lens, N = [500, 31], 9
    P = Pool(2, 9, 64, 1, D, F16, eight, "slot", 5)
    masks = tree_masks(2, N, 2)
    q = (30 * torch.randn((2, N, Hq, D), generator=gen(1), device="cuda")).to(F16)
    q[0, 1] = 0
    out, lse = torch.empty_like(q), torch.empty((2, N, Hq), device="cuda")
    for scale in (1.0, -0.3):
        pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), tensor_of(masks), out, scale=scale, lse=lse)
        scale = torch.tensor(scale, dtype=torch.float32).item()
        ro, rl, to, tl = attend(P, q, lens, scale, 0, masks)
        close(out, ro, to)
        close(lse, rl, tl)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_scales_far_apart(dtype):
    """Values of very different sizes in one tile, and bytes outside [63, 247]."""
    D, n = 128, 100
    P = Pool(1, 2, 64, 1, D, dtype, True, "slot", 6)
    P.vs[:] = torch.randint(110, 126, P.vs.shape, generator=gen(2), device="cuda").to(torch.uint8)
    P.ks[:] = torch.randint(110, 122, P.ks.shape, generator=gen(3), device="cuda").to(torch.uint8)
    P.ks[0, 0], P.vs[0, 1] = 0, 3  # as 63
    q = torch.randn((1, 4, D), generator=gen(1), device="cuda").to(dtype)
    out, lse = torch.empty_like(q), torch.empty((1, 4), device="cuda")
    pe.decode_attn(P.cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), out, lse=lse)
    ro, rl, to, tl = attend(P, q[:, None], [n], D ** -0.5, 0)
    close(out, ro[:, 0], to[:, 0])
    close(lse, rl[:, 0], tl[:, 0])
    P.vs[:], P.ks[:] = 20, 20  # everything as small as it gets
    pe.decode_attn(P.cache, q, torch.tensor([n], dtype=torch.int32, device="cuda"), out, lse=lse)
    ro, rl, to, tl = attend(P, q[:, None], [n], D ** -0.5, 0)
    close(out, ro[:, 0], to[:, 0])
    close(lse, rl[:, 0], tl[:, 0])


def test_one_tree_for_all_and_stream_and_graph():
    """An expanded mask, another stream, a captured call replayed on new inputs."""
    B, N, D = 5, 11, 128
    P = Pool(B, 10, 32, 2, D, BF16, False, "slot", 4)
    masks = tree_masks(1, N, 3)
    q = torch.randn((B, N, 8, D), generator=gen(1), device="cuda").to(BF16)
    lens = torch.tensor([0, 30, 100, 200, 300], dtype=torch.int32, device="cuda")
    out, lse = torch.empty_like(q), torch.empty((B, N, 8), device="cuda")
    work = pe.alloc_workspace(pe.tree_attn_workspace_bytes(P.cache, N, 8))
    mask = tensor_of(masks).expand(B, N)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    pe.tree_attn(P.cache, q, lens, mask, out, lse=lse, workspace=work, stream=st)
    st.synchronize()
    ro, _, to, _ = attend(P, q, lens.tolist(), D ** -0.5, 0, masks * B)
    close(out, ro, to)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pe.tree_attn(P.cache, q, lens, mask, out, lse=lse, workspace=work)
    for seed in (2, 3):
        q.copy_(torch.randn(q.shape, generator=gen(seed), device="cuda"))
        lens.copy_(torch.randint(0, 300, (B,), generator=gen(seed), device="cuda"))
        out.fill_(NAN)
        graph.replay()
        ro, _, to, _ = attend(P, q, lens.tolist(), D ** -0.5, 0, masks * B)
        close(out, ro, to)


@pytest.mark.parametrize("eight", [False, True])
def test_offsets_beyond_32_bits(eight):
    """A pool of more than 2^32 bytes, pages at its end."""
    D, page, H = 128, 64, 8
    n = (1 << 33) // (page * H * D * (1 if eight else 2)) // 2 + 40  # pages: over 2^32 bytes of keys
    dt = torch.uint8 if eight else BF16
    k, v = (torch.zeros((n, page, H, D), dtype=dt, device="cuda") for _ in range(2))
    ks, vs = (torch.full((n, page, H), 127, dtype=torch.uint8, device="cuda") for _ in range(2)) if eight else (None, None)
    table = torch.arange(n - 4, n, dtype=torch.int32, device="cuda").view(1, 4)
    cache = pe.KVCache(k.view(E4M3), v.view(E4M3), table, ks, vs) if eight else pe.KVCache(k, v, table)
    T, N = 200, 5
    x = torch.randn((T + N, 2 * H, D), generator=gen(1), device="cuda").to(BF16)
    pos = torch.arange(T + N, dtype=torch.int32, device="cuda")
    pe.kv_append(cache, x[:, :H], x[:, H:], pos, seqs=torch.zeros_like(pos))
    q = torch.randn((1, N, 16, D), generator=gen(2), device="cuda").to(BF16)
    out = torch.empty_like(q)
    masks = tree_masks(1, N, 1)
    lens = torch.tensor([T], dtype=torch.int32, device="cuda")
    P = Pool.__new__(Pool)
    P.k, P.v, P.ks, P.vs, P.table, P.page = (k.view(E4M3), v.view(E4M3), ks, vs, table, page) if eight else (k, v, None, None, table, page)
    pe.tree_attn(cache, q, lens, tensor_of(masks), out)
    ro, _, to, _ = attend(P, q, [T], D ** -0.5, 0, masks)
    close(out, ro, to)
    pe.kv_move(cache, torch.tensor([[T + 3]], dtype=torch.int32, device="cuda"), torch.tensor([[T + 1]], dtype=torch.int32, device="cuda"))
    a, b = (int(table[0, p // page]) for p in (T + 1, T + 3))
    assert torch.equal(k[a, (T + 1) % page], k[b, (T + 3) % page]) and torch.equal(v[a, (T + 1) % page], v[b, (T + 3) % page])


# ---------------------------------------------------------------------------
# moves
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("eight,dtype", [(False, BF16), (False, F16), (True, BF16)])
@pytest.mark.parametrize("B,n,H,D,page,layout", [(1, 1, 1, 64, 16, "slot"), (5, 7, 3, 128, 5, "head"), (3, 64, 2, 256, 24, "slot"),
                                                 (33, 16, 8, 128, 16, "head"), (2, 37, 1, 64, 1, "slot"), (4, 0, 2, 64, 8, "slot")])
def test_move(eight, dtype, B, n, H, D, page, layout):
    max_pages = -(-150 // page)
    P = Pool(B, max_pages, page, H, D, dtype, eight, layout, 7)
    g = gen(B + n)
    src = torch.stack([torch.randperm(140, generator=g, device="cuda")[:n] for _ in range(B)]).to(torch.int32)
    dst = torch.stack([torch.randperm(140, generator=g, device="cuda")[:n] for _ in range(B)]).to(torch.int32)
    if n >= 7:  # chains, a move to itself, moves out of range and from absent pages
        src[0, 1], dst[0, 0] = 148, 148
        src[0, 2] = dst[0, 2]
        src[0, 3], dst[0, 4], src[0, 5], dst[0, 6] = -1, max_pages * page, 2 ** 31 - 1, -7
        if B > 1:
            P.table[1, 0], P.table[1, -1] = -1, P.k.shape[0]
    # rows of a wider table of moves
    wide = torch.full((B, n + 3), -1, dtype=torch.int32, device="cuda")
    wide[:, 1:1 + n] = src
    was = [None if t is None else t.view(torch.uint8).clone() if eight else t.clone() for t in (P.k, P.v, P.ks, P.vs)]
    want = [None if t is None else t.clone() for t in was]
    for b in range(B):
        seen = set()
        for s, d in zip(src[b].tolist(), dst[b].tolist()):
            if not (0 <= s < max_pages * page and 0 <= d < max_pages * page):
                continue
            sp, dp = int(P.table[b, s // page]), int(P.table[b, d // page])
            if not (0 <= sp < P.k.shape[0] and 0 <= dp < P.k.shape[0]):
                continue
            assert d not in seen
            seen.add(d)
            for w, o in zip(want, was):
                if w is not None:
                    w[dp, d % page] = o[sp, s % page]
    pe.kv_move(P.cache, wide[:, 1:1 + n], dst)
    for t, w in zip((P.k, P.v, P.ks, P.vs), want):
        if w is not None:
            assert torch.equal(t.view(torch.uint8) if eight else t.view(torch.int16), w if eight else w.view(torch.int16))


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("graph", [False, True])
def test_a_drafted_step(eight, graph):
    """Append a tree, attend, keep a path, and attend again with the next token:
    the same as if the path alone had been appended."""
    B, N, Hq, H, D, page = 3, 6, 8, 2, 128, 16
    g = gen(11)
    rot = pe.rot_table(300, D)
    masks = [[0b1, 0b11, 0b101, 0b1011, 0b10101, 0b101011]] * B  # paths 0-1-3-5 and 0-2-4
    depth = torch.tensor([0, 1, 1, 2, 2, 3], dtype=torch.int32, device="cuda")
    path = [0, 1, 3, 5]
    lens = torch.tensor([0, 37, 200], dtype=torch.int32, device="cuda")
    P, Q = (Pool(B, 16, page, H, D, BF16, eight, "slot", 21) for _ in range(2))
    x = torch.randn((B * N, Hq + 2 * H, D), generator=g, device="cuda").to(BF16)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + H], x[:, Hq + H:]
    seqs = torch.arange(B, dtype=torch.int32, device="cuda").repeat_interleave(N)
    node = torch.arange(N, dtype=torch.int32, device="cuda").repeat(B)
    y = torch.randn((B, Hq, D), generator=g, device="cuda").to(BF16)
    q_out, out, end = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty((B, N, Hq, D), dtype=BF16, device="cuda"), torch.empty_like(y)
    src = lens[:, None] + torch.tensor(path, dtype=torch.int32, device="cuda")
    dst = lens[:, None] + torch.arange(4, dtype=torch.int32, device="cuda")
    mask = tensor_of(masks)
    base = lens[seqs.long()]
    pos, slots, after = base + depth[node.long()], base + node, lens + 4

    def step():
        pe.kv_append(P.cache, k, v, pos, seqs=seqs, q=q, q_out=q_out, rot=rot, slots=slots)
        pe.tree_attn(P.cache, q_out.view(B, N, Hq, D), lens, mask, out)
        pe.kv_move(P.cache, src, dst)
        pe.decode_attn(P.cache, y, after, end)

    if graph:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step()
        gr.replay()
    else:
        step()
    # the path alone, token by token
    xs = x.view(B, N, Hq + 2 * H, D)
    for i, a in enumerate(path):
        qa = torch.empty((B, Hq, D), dtype=BF16, device="cuda")
        pe.kv_append(Q.cache, xs[:, a, Hq:Hq + H], xs[:, a, Hq + H:], lens + i, q=xs[:, a, :Hq], q_out=qa, rot=rot)
        ro, _, to, _ = attend(Q, qa[:, None], (lens + i + 1).tolist(), D ** -0.5, 0)
        close(out[:, a], ro[:, 0], to[:, 0])
    last = torch.empty_like(y)
    pe.decode_attn(Q.cache, y, after, last)
    assert torch.equal(end, last)


# ---------------------------------------------------------------------------
# drafted nodes with few rows a key head, and calls that share what they use
# ---------------------------------------------------------------------------
FEW = [
    # dtype, eight, lens, N, max_pages, page, Hq, Hkv, D, layout
    (BF16, True, [900, 0, 31, 257], 4, 30, 32, 8, 2, 128, "slot"),
    (F16, True, [64, 63, 65, 5], 5, 6, 13, 8, 2, 128, "head"),
    (BF16, True, [3000], 24, 64, 48, 3, 3, 64, "slot"),
    (BF16, True, [500, 40], 23, 40, 16, 1, 1, 128, "head"),
    (F16, True, [77, 1400], 2, 60, 24, 24, 2, 64, "slot"),
    (BF16, True, [600, 3], 8, 40, 16, 2, 2, 256, "slot"),
    (F16, True, [129], 1, 20, 8, 16, 1, 128, "head"),
    (BF16, False, [900, 0, 31, 257], 4, 30, 32, 8, 2, 128, "slot"),
    (F16, False, [64, 63, 65, 5], 5, 6, 13, 6, 2, 128, "head"),
    (BF16, False, [3000], 16, 64, 48, 3, 3, 64, "slot"),
    (F16, False, [500, 40], 7, 40, 16, 4, 2, 64, "head"),
    (BF16, False, [600, 3], 8, 40, 16, 2, 2, 256, "slot"),
    (F16, False, [150, 9], 2, 20, 24, 4, 1, 256, "head"),
    (F16, True, [20, 8, -3], 20, 3, 8, 2, 2, 128, "slot"),  # nodes beyond the table
    (BF16, True, [600, 3, 0, 90], 5, 40, 16, 6, 2, 256, "slot"),
    (F16, True, [1000], 16, 90, 13, 1, 1, 256, "head"),
]


@pytest.mark.parametrize("dtype,eight,lens,N,max_pages,page,Hq,Hkv,D,layout", FEW)
@pytest.mark.parametrize("window", [0, 64, 200])
def test_few_rows(dtype, eight, lens, N, max_pages, page, Hq, Hkv, D, layout, window):
    test_tree(dtype, eight, lens, N, max_pages, page, Hq, Hkv, D, layout, window)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("Hq,N,D,n", [(2, 8, 64, 500), (4, 4, 128, 90), (4, 12, 128, 5000), (2, 7, 256, 300), (4, 7, 256, 300), (24, 1, 64, 40)])
@pytest.mark.parametrize("window", [0, 70])
def test_few_rows_and_values_that_are_no_numbers(eight, Hq, N, D, n, window):
    """A NaN in a node's values, and at the window's start: NaN in that element of the rows that attend to it, nowhere else."""
    page = 16
    P = Pool(2, -(-(n + N) // page), page, 2, D, BF16, eight, "slot", 5)
    masks = tree_masks(2, N, 9)
    q = torch.randn((2, N, Hq, D), generator=gen(1), device="cuda").to(BF16)
    lens = [n, n - 3]
    ro, rl, to, tl = attend(P, q, lens, D ** -0.5, window, masks)
    nan = torch.zeros(q.shape, dtype=torch.bool, device="cuda")
    G = Hq // 2

    def spoil(b, p, h, e):
        at = (int(P.table[b, p // page]), p % page, h, e)
        if eight:
            P.v.view(torch.uint8)[at] = 0xFF
        else:
            P.v[at] = NAN
        for i, m in enumerate(masks[b]):
            lo = max(0, lens[b] + bin(m).count("1") - window) if window else 0
            if (lo <= p < lens[b]) if p < lens[b] else (m >> (p - lens[b]) & 1):
                nan[b, i, h * G:(h + 1) * G, e] = True

    spoil(0, lens[0] + N // 2, 1, 0)
    spoil(0, lens[0], 0, D - 1)
    spoil(1, lens[1] + N - 1, 0, 21)
    spoil(1, max(0, lens[1] + 2 - window), 1, D // 2 + 8)
    spoil(1, lens[1] - 1, 1, 7)
    out, lse = torch.empty_like(q), torch.empty((2, N, Hq), device="cuda")
    pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), tensor_of(masks), out, window=window, lse=lse)
    close(out, torch.where(nan, NAN, ro), to)
    close(lse, rl, tl)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("B,longest", [(90, 300), (3, 9000), (700, 2), (1, 20000)])
@pytest.mark.parametrize("Hq,N,D", [(4, 8, 64), (12, 5, 128), (4, 6, 256), (8, 6, 256)])
def test_few_rows_of_many_segments(eight, Hq, N, D, B, longest):
    test_many_segments(eight, D, Hq, N, B, longest)


@pytest.mark.parametrize("eight", [False, True])
@pytest.mark.parametrize("Hq,N,D", [(20, 14, 128), (20, 14, 64), (32, 64, 128)])
def test_blocks_that_are_nearly_empty(eight, Hq, N, D):
    """Rows just beyond a block, with as many tiles in it as in the full one: a part of the CTA has nothing to do for long."""
    H, page, lens = 1, 64, [16000, 9000, 16001, 30, 12000, 7000]
    P = Pool(len(lens), -(-(max(lens) + N) // page), page, H, D, BF16, eight, "slot", 3)
    masks = tree_masks(1, N, 7) * len(lens)
    q = torch.randn((len(lens), N, Hq, D), generator=gen(4), device="cuda").to(BF16)
    out = torch.full_like(q, NAN)
    pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), tensor_of(masks), out)
    pe.device_check()
    whole = P.table
    for b in (0, 2, 3):
        P.table = whole[b:b + 1]
        ro, _, to, _ = attend(P, q[b:b + 1, :1], [lens[b]], D ** -0.5, 0, [[1]])  # node 0 attends to itself alone
        close(out[b, 0], ro[0, 0], to[0, 0])
    assert torch.isfinite(out.float()).all()
    # a node by itself, in a call of its own with the other nodes' rows left out
    alone = torch.full_like(q, NAN)
    only = [[m if i in (N // 2, N - 1) else 0 for i, m in enumerate(row)] for row in masks]
    P.table = whole
    pe.tree_attn(P.cache, q, torch.tensor(lens, dtype=torch.int32, device="cuda"), tensor_of(only), alone)
    for i in (N // 2, N - 1):
        assert torch.equal(alone[:, i], out[:, i])
    assert not alone[:, 0].any()


@pytest.mark.parametrize("eight", [False, True])
def test_calls_at_once_and_in_place(eight):
    """Two streams with workspaces of their own; two captured calls that share one; the output in the queries' place."""
    D, H, page, N, lens = 128, 4, 64, 9, [3000, 1700, 40, 2500]
    P = Pool(4, 48, page, H, D, BF16, eight, "slot", 3)
    t = torch.tensor(lens, dtype=torch.int32, device="cuda")
    calls = []
    for Hq, n in ((16, N), (8, 2), (16, 40), (32, 64)):
        masks = tensor_of(tree_masks(4, n, 5))
        q = torch.randn((4, n, Hq, D), generator=gen(Hq), device="cuda").to(BF16)
        ref = torch.empty_like(q)
        pe.tree_attn(P.cache, q, t, masks, ref)
        calls.append((q, masks, ref))
    token = torch.randn((4, 128, D), generator=gen(1), device="cuda").to(BF16)  # 32 heads a key head
    one = torch.empty_like(token)
    pe.decode_attn(P.cache, token, t, one)
    torch.cuda.synchronize()

    streams = [torch.cuda.Stream() for _ in range(5)]
    spaces = [torch.empty(pe.tree_attn_workspace_bytes(P.cache, q.shape[1], q.shape[2]), dtype=torch.uint8, device="cuda") for q, _, _ in calls]
    outs = [torch.full_like(q, NAN) for q, _, _ in calls]
    got = torch.full_like(token, NAN)
    space = torch.empty(pe.decode_attn_workspace_bytes(P.cache, 128), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    for _ in range(5):
        for s, (q, masks, _), o, w in zip(streams, calls, outs, spaces):
            pe.tree_attn(P.cache, q, t, masks, o, workspace=w, stream=s)
        pe.decode_attn(P.cache, token, t, got, workspace=space, stream=streams[4])
    torch.cuda.synchronize()
    for (_, _, ref), o in zip(calls, outs):
        assert torch.equal(o, ref)
    assert torch.equal(got, one)

    shared = torch.empty(max(w.numel() for w in spaces), dtype=torch.uint8, device="cuda")
    graphs = []
    for (q, masks, _), o in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pe.tree_attn(P.cache, q, t, masks, o, workspace=shared)
        graphs.append(g)
    for o in outs:
        o.fill_(NAN)
    shared.fill_(255)
    for _ in range(2):
        for g in graphs:
            g.replay()
    torch.cuda.synchronize()
    for (_, _, ref), o in zip(calls, outs):
        assert torch.equal(o, ref)
    for q, masks, ref in calls:
        pe.tree_attn(P.cache, q, t, masks, q)
        assert torch.equal(q, ref)
    pe.device_check()
