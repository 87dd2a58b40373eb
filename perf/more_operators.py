"""More token operators whose speed is measured: generation over a cache in 8
bits, and with drafted tokens.

  append  keys and values of new tokens into a paged cache of 8-bit codes with
          a power-of-two scale for each head's row, rotated on the way; drafted
          tokens go to slots of their own, siblings share a position
  decode  attention of one new token per sequence over that cache
  tree    attention of each sequence's tree of drafted tokens over the cache
          (8 or 16 bits) and over their ancestors in the tree
  move    the accepted drafts' rows to the positions that they end up at

Where ``own`` is true, ``run`` makes the calls of the public binding; where it
is false, the same operators in elementary torch operations in 32 bits,
rounded once at the end.  ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
E4M3 = torch.float8_e4m3fn
MOST_BYTES, MOST_FLOPS, MOST_SCORES = 2.3e9, 2.8e11, 5.5e8  # of a drawn case: what the largest listed ones cost


def listed():
    return [
        # one decode step of 32 running sequences into the 8-bit cache: latency counts
        dict(name="append_step", op="append", T=32, seqs=32, start=500, Hq=32, Hkv=8, D=128, page=16, dtype="bf16",
             cache="e4m3", rot=128, inter=False, layout="slot", nodes=0),
        # drafted trees of 24 tokens for 37 sequences, pages of 24: interleaved pairs, half of each head rotated
        dict(name="append_drafts_odd", op="append", T=37 * 24, seqs=37, start=900, Hq=16, Hkv=16, D=64, page=24,
             dtype="f16", cache="e4m3", rot=32, inter=True, layout="head", nodes=24),
        # a long prefill of many queries per key head, from one fused projection
        dict(name="append_prefill", op="append", T=32768, seqs=8, start=1000, Hq=64, Hkv=8, D=128, page=64,
             dtype="bf16", cache="e4m3", rot=128, inter=False, layout="slot", nodes=0),
        # one user, a short conversation: latency counts
        dict(name="decode_one", op="decode", B=1, len=700, lens="full", Hq=32, Hkv=8, D=128, page=16, dtype="bf16",
             cache="e4m3", window=0, layout="slot"),
        # the largest generation batch, at ragged lengths, one slot idle
        dict(name="decode_batch", op="decode", B=128, len=8192, lens="spread", Hq=64, Hkv=8, D=128, page=16,
             dtype="bf16", cache="e4m3", window=0, layout="slot"),
        # one very long context of half-precision queries: the split over the cache's length carries it
        dict(name="decode_long", op="decode", B=1, len=262143, lens="full", Hq=32, Hkv=8, D=128, page=64, dtype="f16",
             cache="e4m3", window=0, layout="head"),
        # one user's eight drafted tokens: latency counts
        dict(name="tree_one", op="tree", B=1, len=700, lens="full", N=8, Hq=32, Hkv=8, D=128, page=16, dtype="bf16",
             cache="same", window=0, layout="slot"),
        # a running batch that drafts 32 tokens a sequence, at ragged lengths, one slot idle: bound by the cache
        dict(name="tree_batch", op="tree", B=64, len=8192, lens="spread", N=32, Hq=32, Hkv=8, D=128, page=16,
             dtype="bf16", cache="same", window=0, layout="slot"),
        # the widest trees over the 8-bit cache, 512 rows of scores for each key head: bound by the products
        dict(name="tree_wide", op="tree", B=32, len=4096, lens="full", N=64, Hq=64, Hkv=8, D=128, page=64, dtype="bf16",
             cache="e4m3", window=0, layout="head"),
        # odd everything: 13 nodes, five queries a key head, odd pages, a sliding window
        dict(name="tree_odd_window", op="tree", B=7, len=20011, lens="spread", N=13, Hq=20, Hkv=4, D=64, page=24,
             dtype="f16", cache="same", window=8192, layout="slot"),
        # the accepted drafts of 32 sequences: latency counts
        dict(name="move_step", op="move", B=32, len=700, n=5, N=16, Hkv=8, D=128, page=16, dtype="bf16", cache="same",
             layout="slot"),
        # long accepted paths of a large batch in the 8-bit cache
        dict(name="move_batch", op="move", B=512, len=1000, n=16, N=64, Hkv=16, D=128, page=24, dtype="bf16",
             cache="e4m3", layout="head"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "append", "decode", "decode", "tree", "tree", "tree", "move"])
        D = rng.choice([64, 128, 128, 256])
        Hkv = rng.choice([1, 2, 4, 8, 8, 16])
        c = dict(op=op, Hq=Hkv * rng.choice([1, 2, 4, 5, 8, 8, 16, 20]), Hkv=Hkv, D=D,
                 page=rng.choice([8, 16, 16, 24, 64, 100, 256]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                 cache="e4m3", layout=rng.choice(["slot", "head"]))
        if c["Hq"] > 128:
            continue
        if op == "append":
            kind = rng.choice(["step", "prompt", "drafts"])
            T, nodes, seqs = _log(rng, 1, 32768), 0, rng.randint(1, 16)
            if kind == "step":
                T = seqs = min(T, 512)
            elif kind == "drafts":
                nodes, seqs = rng.randint(2, 64), _log(rng, 1, 512)
                T = seqs * nodes
                c["cache"] = rng.choice(["e4m3", "same"])
            c.update(T=T, seqs=min(T, seqs), start=_log(rng, 1, 1024), rot=rng.choice([D, D, D // 2]),
                     inter=rng.random() < 0.3, nodes=nodes)
        elif op == "move":
            N = rng.randint(1, 64)
            c.update(B=_log(rng, 1, 512), len=_log(rng, 1, 4096), N=N, n=rng.randint(1, min(N, 16)),
                     cache=rng.choice(["e4m3", "same"]))
            del c["Hq"]
            if 2 * c["B"] * (c["len"] + N) * Hkv * D > MOST_BYTES:
                continue
        else:
            c.update(B=_log(rng, 1, 256 if op == "decode" else 128), len=_log(rng, 16, 262144 if op == "decode" else 65536),
                     lens=rng.choice(["full", "spread", "spread"]), window=rng.choice([0, 0, 0, 1000, 4096]))
            if op == "tree":
                c.update(N=_log(rng, 1, 64), cache=rng.choice(["e4m3", "same"]))
            # the plain form gathers the whole table and holds every score: bound those, not only what is attended to
            span = c["B"] * (c["len"] + c.get("N", 0))
            if span * Hkv * D * 2 > MOST_BYTES or span * c["Hq"] * c.get("N", 1) > MOST_SCORES:
                continue
        w = work(c)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _lens(case):
    """Lengths of the sequences, the same for every seed (their order is not):
    all equal, or spread like the ages of a running batch, one slot idle."""
    B, L = case["B"], case["len"]
    if case["lens"] == "full":
        return [L] * B
    lens = [max(1, round(L * ((i + 1) / B) ** 1.5)) for i in range(B)]
    if B >= 8:
        lens[0] = 0
    return lens


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _quantise(x):
    """Codes (as bytes) and scale bytes of rows in fp32: the scale is the least
    power of two, 2^-64 at least, that brings the row within 448."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)
    e = torch.where(a > 0, e.int() - 9 + (m > 0.875).int(), -64).clamp(min=-64)
    e = torch.where(torch.isfinite(a), e, 128)
    inv = ((127 - e.clamp(max=120)) << 23).view(torch.float32)
    codes = torch.where(torch.isfinite(a)[..., None], x * inv[..., None], 0.0).to(E4M3)
    return codes.view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scale):
    """fp32 rows that codes and scale bytes stand for."""
    f = (scale.int() << 23).view(torch.float32)
    return codes.view(E4M3).float() * torch.where(scale == 255, float("nan"), f)[..., None]


def _storage(case, n_pages, fill, g):
    """Page storage of keys and of values, [pages, slots, heads, head_dim], and
    their scales ([pages, slots, heads], 8 bits only); the "head" layout keeps
    each head's slots of a page together in memory."""
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    dt = torch.uint8 if case["cache"] == "e4m3" else DTYPES[case["dtype"]]
    shape = (n_pages, page, Hkv) if case["layout"] == "slot" else (n_pages, Hkv, page)
    out = []
    for _ in range(2):
        x = torch.zeros((*shape, D), dtype=dt, device="cuda")
        sc = torch.full(shape, 63, dtype=torch.uint8, device="cuda") if case["cache"] == "e4m3" else None
        if fill:
            step = max(1, (1 << 27) // (page * Hkv * D))
            for a in range(0, n_pages, step):
                part = torch.randn((min(step, n_pages - a), *shape[1:], D), generator=g, device="cuda")
                if sc is None:
                    x[a:a + step] = part.to(dt)
                else:  # rows of different sizes, as a model's keys and values have
                    part *= torch.exp2(torch.randn(part.shape[:-1], generator=g, device="cuda"))[..., None].clamp(0.125, 2.0)
                    x[a:a + step], sc[a:a + step] = _quantise(part)
        out += [x, sc]
    if case["layout"] == "head":
        out = [None if t is None else t.transpose(1, 2) for t in out]
    return dict(zip(("k_cache", "k_scale", "v_cache", "v_scale"), out))


def _table(n_seqs, max_pages, g):
    """Each sequence's pages, scattered over the pool as a running server's are."""
    n = n_seqs * max_pages
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(n_seqs, max_pages)


def _trees(B, N, g):
    """Trees of drafted tokens in the order of drafting: (masks of a node's
    ancestors and itself [B, N] int64, depths [B, N])."""
    mask = torch.zeros((B, N), dtype=torch.int64, device="cuda")
    depth = torch.zeros((B, N), dtype=torch.int64, device="cuda")
    mask[:, 0] = 1
    for i in range(1, N):  # a recent node as the parent, more often than not: paths get long
        back = (torch.rand((B, 1), generator=g, device="cuda") ** 2 * i).long().clamp(max=i - 1)
        parent = i - 1 - back
        mask[:, i] = mask.gather(1, parent)[:, 0] | (1 << i if i < 63 else -2 ** 63)
        depth[:, i] = depth.gather(1, parent)[:, 0] + 1
    return mask, depth


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    op, Hkv, D, page = (case[k] for k in ("op", "Hkv", "D", "page"))
    dt = DTYPES[case["dtype"]]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(dt)

    if op == "append":
        T, S, Hq = case["T"], case["seqs"], case["Hq"]
        count = [T // S + (i < T % S) for i in range(S)]
        top = case["start"] + max(count)
        max_pages = -(-top // page)
        s.update(_storage(case, S * max_pages, False, g))
        s["table"] = _table(S, max_pages, g)
        first = torch.randint(0, case["start"] + 1, (S,), generator=g, device="cuda")
        cnt = torch.tensor(count, device="cuda")
        seq = torch.repeat_interleave(torch.arange(S, device="cuda"), cnt)
        within = torch.arange(T, device="cuda") - (torch.cumsum(cnt, 0) - cnt)[seq]
        slots = (first[seq] + within).to(torch.int32)
        if case["nodes"]:
            depth = _trees(S, case["nodes"], g)[1]
            s["positions"], s["slots"] = (first[:, None] + depth).view(-1).to(torch.int32), slots
        else:
            s["positions"], s["slots"] = slots, None
        s["seqs"] = None if T == S else seq.to(torch.int32)
        qkv = randn(T, Hq + 2 * Hkv, D)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        half = case["rot"] // 2
        ang = torch.arange(top, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        s["rot"] = torch.cat([torch.cos(ang), torch.sin(ang)], 1).float().cuda()
        s["q_out"] = torch.empty((T, Hq, D), dtype=dt, device="cuda")
    elif op == "move":
        B, N, n = case["B"], case["N"], case["n"]
        max_pages = -(-(case["len"] + N) // page)
        s.update(_storage(case, B * max_pages, True, g))
        s["table"] = _table(B, max_pages, g)
        base = torch.randint(0, case["len"] + 1, (B, 1), generator=g, device="cuda")
        # an accepted path: nodes in rising order from the tree's root on; the rest of the row is padding
        rest = torch.rand((B, N - 1), generator=g, device="cuda").argsort(1)[:, :n - 1].sort(1)[0] + 1
        path = torch.cat([torch.zeros((B, 1), dtype=torch.int64, device="cuda"), rest], 1)
        live = torch.arange(n, device="cuda") < torch.randint(1, n + 1, (B, 1), generator=g, device="cuda")
        s["src"] = torch.where(live, base + path, -1).to(torch.int32)
        s["dst"] = torch.where(live, base + torch.arange(n, device="cuda"), -1).to(torch.int32)
    else:
        B, Hq, N = case["B"], case["Hq"], case.get("N", 0)
        max_pages = -(-(case["len"] + N) // page)
        s.update(_storage(case, B * max_pages, True, g))
        s["table"] = _table(B, max_pages, g)
        order = torch.randperm(B, generator=g, device="cuda")
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order]
        shape = (B, N, Hq, D) if N else (B, Hq, D)
        # scores of a standard deviation of two: some positions matter, none alone
        s["q"] = 2.0 * randn(*shape)
        s["out"] = torch.empty(shape, dtype=dt, device="cuda")
        s["lse"] = torch.empty(shape[:-1], device="cuda")
        if N:
            mask, _ = _trees(B, N, g)
            if N >= 4:  # trees of different sizes: the rest of the row is padding
                size = torch.randint(N // 2, N + 1, (B, 1), generator=g, device="cuda")
                mask = torch.where(torch.arange(N, device="cuda") < size, mask, 0)
            s["mask"] = mask
    if own:
        from paper_2608_11226_gb300 import pe

        if case["cache"] == "e4m3":
            s["cache"] = pe.KVCache(s["k_cache"].view(E4M3), s["v_cache"].view(E4M3), s["table"], k_scale=s["k_scale"],
                                    v_scale=s["v_scale"])
        else:
            s["cache"] = pe.KVCache(s["k_cache"], s["v_cache"], s["table"])
        if op == "decode":
            s["workspace"] = pe.alloc_workspace(pe.decode_attn_workspace_bytes(s["cache"], case["Hq"]))
        elif op == "tree":
            s["workspace"] = pe.alloc_workspace(pe.tree_attn_workspace_bytes(s["cache"], case["N"], case["Hq"]))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _run_own(case["op"], s, case)
    return {"append": _plain_append, "decode": _plain_attn, "tree": _plain_attn, "move": _plain_move}[case["op"]](s, case)


def _caches(s):
    """The cache as outputs: codes as the 8-bit type that they are, scales as they are held."""
    if s["k_scale"] is None:
        return dict(k_cache=s["k_cache"], v_cache=s["v_cache"])
    return dict(k_cache=s["k_cache"].view(E4M3), v_cache=s["v_cache"].view(E4M3), k_scale=s["k_scale"], v_scale=s["v_scale"])


def _run_own(op, s, case):
    from paper_2608_11226_gb300 import pe

    if op == "append":
        pe.kv_append(s["cache"], s["k"], s["v"], s["positions"], seqs=s["seqs"], q=s["q"], q_out=s["q_out"],
                     rot=s["rot"], interleaved=case["inter"], slots=s["slots"])
        return dict(q=s["q_out"], **_caches(s))
    if op == "move":
        pe.kv_move(s["cache"], s["src"], s["dst"])
        return _caches(s)
    if op == "decode":
        pe.decode_attn(s["cache"], s["q"], s["lens"], s["out"], window=case["window"], lse=s["lse"],
                       workspace=s["workspace"])
    else:
        pe.tree_attn(s["cache"], s["q"], s["lens"], s["mask"], s["out"], window=case["window"], lse=s["lse"],
                     workspace=s["workspace"])
    return dict(out=s["out"], lse=s["lse"])


def _rotate(x, cs, rot, inter):
    x = x.float()
    half = rot // 2
    c, sn = cs[:, None, :half], cs[:, None, half:]
    if inter:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        y = torch.stack([a * c - b * sn, b * c + a * sn], -1).flatten(-2)
    else:
        a, b = x[..., :half], x[..., half:rot]
        y = torch.cat([a * c - b * sn, b * c + a * sn], -1)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(s, case):
    pos = s["positions"].long()
    at = pos if s["slots"] is None else s["slots"].long()
    seq = torch.arange(case["T"], device="cuda") if s["seqs"] is None else s["seqs"].long()
    cs = s["rot"][pos]
    q = _rotate(s["q"], cs, case["rot"], case["inter"]).to(s["q"].dtype)
    k, v = _rotate(s["k"], cs, case["rot"], case["inter"]), s["v"].float()
    pages, slot = s["table"][seq, at // case["page"]].long(), at % case["page"]
    for name, x in (("k", k), ("v", v)):
        if s["k_scale"] is None:
            s[name + "_cache"][pages, slot] = x.to(s["q"].dtype)
        else:
            s[name + "_cache"][pages, slot], s[name + "_scale"][pages, slot] = _quantise(x)
    return dict(q=q, **_caches(s))


def _plain_move(s, case):
    src, dst = s["src"].long(), s["dst"].long()
    b, i = torch.nonzero(src >= 0, as_tuple=True)
    src, dst, page = src[b, i], dst[b, i], case["page"]
    sp, dp = s["table"][b, src // page].long(), s["table"][b, dst // page].long()
    for name in ("k_cache", "v_cache", "k_scale", "v_scale"):
        if s[name] is not None:
            s[name][dp, dst % page] = s[name][sp, src % page]
    return _caches(s)


def _keep(s, case, span):
    """[B, rows or 1, span]: which positions a sequence's new tokens attend to."""
    j = torch.arange(span, device="cuda")
    n, w = s["lens"].long()[:, None, None], case["window"]
    if case["op"] == "decode":
        return (j < n) & (j >= n - w) if w else j < n
    mask, N = s["mask"], case["N"]
    bits = (mask[..., None] >> torch.arange(N, device="cuda")) & 1  # [B, N, N]
    keep = j < n
    if w:  # a node stands as many positions behind the context as it has ancestors
        keep = keep & (j > n + bits.sum(-1, keepdim=True) - 1 - w)
    own_j = j - n
    node = (own_j >= 0) & (own_j < N)
    in_tree = bits.gather(2, own_j.clamp(0, N - 1).expand(-1, N, -1)).bool() & node
    return (keep | in_tree) & (mask != 0)[..., None]


def _plain_attn(s, case):
    B, Hq, Hkv, D = (case[k] for k in ("B", "Hq", "Hkv", "D"))
    N, G = case.get("N", 1), Hq // Hkv
    t = s["table"].long()
    k, v = s["k_cache"][t].flatten(1, 2), s["v_cache"][t].flatten(1, 2)  # [B, positions, Hkv, D]
    if s["k_scale"] is None:
        k, v = k.float(), v.float()
    else:
        k, v = _values(k, s["k_scale"][t].flatten(1, 2)), _values(v, s["v_scale"][t].flatten(1, 2))
    q = s["q"].float().view(B, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, N * G, D)
    z = torch.matmul(q, k.permute(0, 2, 3, 1)) * D ** -0.5
    keep = _keep(s, case, z.shape[-1])  # [B, N or 1, positions]
    z = torch.where(keep[:, None, :, None], z.view(B, Hkv, N, G, -1), float("-inf"))
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(m > float("-inf"), m, 0.0))
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e.view(B, Hkv, N * G, -1), v.transpose(1, 2)).view(B, Hkv, N, G, D) / torch.where(l > 0, l, 1.0)
    shape = s["q"].shape
    return dict(out=o.transpose(1, 2).reshape(shape).to(s["q"].dtype),
                lse=(m + torch.log(l)).transpose(1, 2).reshape(shape[:-1]))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op, Hkv, D = case["op"], case["Hkv"], case["D"]
    row = D + 1 if case["cache"] == "e4m3" else 2 * D  # bytes of a head's row in the cache
    if op == "append":
        T, Hq = case["T"], case["Hq"]
        # every head's row in and out; positions, page ids; the rotation rows of the positions met, at most
        return dict(bytes=T * (4 * Hq * D + 2 * Hkv * (2 * D + row)) + 8 * T + min(T, case["start"] + T) * case["rot"] * 4,
                    flops=T * (3 * (Hq + Hkv) * case["rot"] + 4 * Hkv * D))
    if op == "move":
        return dict(bytes=4 * case["B"] * (case["n"] + 1) // 2 * Hkv * row + 8 * case["B"] * case["n"], flops=0)
    B, Hq, N, w = case["B"], case["Hq"], case.get("N", 1), case["window"]
    n = sum(min(x, w) if w else x for x in _lens(case))
    drafts = case.get("N", 0) * B
    near = round(N * (1 + math.log(N))) * B if drafts else 0  # ancestors, about
    return dict(bytes=2 * (n + drafts) * Hkv * row + B * N * Hq * (4 * D + 4) + 4 * n // case["page"] + 8 * drafts,
                flops=4 * (n * N + near) * Hq * D)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "decode": _exact_attn, "tree": _exact_attn, "move": _exact_move}[case["op"]](s, case)


def _exact_codes(x):
    """The codes' values: each element over the row's scale, to the nearest of
    the type's numbers (steps of 2^-3 of the power of two below, 2^-9 at least)."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a / 448.0)).clamp(min=-64.0)
    e = torch.where(a > 448.0 * torch.exp2(e), e + 1, torch.where((a <= 448.0 * torch.exp2(e - 1)) & (e > -64), e - 1, e))
    y = x / torch.exp2(e)
    step = torch.exp2((torch.frexp(y)[1] - 4).clamp(min=-9).double())
    return torch.round(y / step) * step


def _exact_append(s, case):
    D, rot, T = case["D"], case["rot"], case["T"]
    half = rot // 2
    angle = s["rot"].double()[s["positions"].long()]

    def turned(x):  # a pair as a complex number, turned by its angle
        x = x.double()
        lo = torch.arange(half, device="cuda") * 2 if case["inter"] else torch.arange(half, device="cuda")
        hi = lo + 1 if case["inter"] else lo + half
        w = torch.complex(x[..., lo], x[..., hi]) * torch.complex(angle[:, None, :half], angle[:, None, half:])
        y = x.clone()
        y[..., lo], y[..., hi] = w.real, w.imag
        return y

    seq = torch.arange(T, device="cuda") if s["seqs"] is None else s["seqs"].long()
    at = (s["positions"] if s["slots"] is None else s["slots"]).long()
    line = seq * s["table"].shape[1] * case["page"] + at  # the token's place, page after page of the table
    page = s["table"].reshape(-1).long()[line // case["page"]]
    place = page * case["page"] + line % case["page"]
    eight = s["k_scale"] is not None
    got = dict(q=turned(s["q"]))
    for name, x in (("k_cache", turned(s["k"])), ("v_cache", s["v"].double())):
        flat = torch.zeros((s["table"].numel() * case["page"], case["Hkv"], D), dtype=torch.float64, device="cuda")
        flat[place] = _exact_codes(x) if eight else x
        got[name] = flat.view(-1, case["page"], case["Hkv"], D)
    return dict(got, k_scale=None, v_scale=None) if eight else got


def _exact_move(s, case):
    """Row by row on the host's lists: what was at src before is at dst after."""
    page, table = case["page"], s["table"].cpu()
    eight = s["k_scale"] is not None
    moves = [(int(table[b, x // page]) * page + x % page, int(table[b, y // page]) * page + y % page)
             for b, (xs, ys) in enumerate(zip(s["src"].tolist(), s["dst"].tolist())) for x, y in zip(xs, ys) if x >= 0]
    frm, to = (torch.tensor(m, device="cuda") for m in zip(*moves))
    got = {}
    for name in ("k_cache", "v_cache"):
        x = s[name].view(E4M3) if eight else s[name]
        flat = x.double().reshape(-1, case["Hkv"], case["D"])
        got[name] = flat.index_copy(0, to, flat[frm]).view(x.shape)
    return dict(got, k_scale=None, v_scale=None) if eight else got


def _exact_attn(s, case):
    Hq, Hkv, D, page, w = (case[k] for k in ("Hq", "Hkv", "D", "page", "window"))
    tree, G = case["op"] == "tree", Hq // Hkv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:-1], float("-inf"), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        masks = s["mask"][b].tolist() if tree else [1]
        end = n + len(masks) if tree else n
        # (lowest position, nodes attended to) of each new token that is no padding
        rows = [(i, max(0, n + bin(x & (1 << 64) - 1).count("1") - w) if w else 0, [a for a in range(64) if x >> a & 1])
                for i, x in enumerate(masks) if x] if tree else [(0, max(0, n - w) if w else 0, [])] * (n > 0)
        if not rows:
            continue
        first = min(r[1] for r in rows)
        pages = s["table"][b, first // page:-(-end // page)].long()
        cut = slice(first - first // page * page, end - first // page * page)
        kv = []
        for name in ("k", "v"):
            x = s[name + "_cache"][pages].flatten(0, 1)[cut]
            if s["k_scale"] is not None:
                power = s[name + "_scale"][pages].flatten(0, 1)[cut].double() - 127.0
                x = x.view(E4M3).double() * torch.exp2(power)[..., None]
            kv.append(x)
        seen = torch.zeros((len(rows), end - first), dtype=torch.bool, device="cuda")
        for r, (_, low, nodes) in enumerate(rows):
            seen[r, max(0, low - first):max(0, n - first)] = True
            if nodes:
                seen[r, torch.tensor(nodes, device="cuda") + n - first] = True
        at = torch.tensor([r[0] for r in rows], device="cuda")
        for h in range(Hkv):
            heads = slice(h * G, (h + 1) * G)
            q = (s["q"][b, at][:, heads] if tree else s["q"][b, heads][None]).double()
            z = torch.einsum("rgd,pd->rgp", q, kv[0][:, h].double()) / math.sqrt(D)
            z = z.masked_fill(~seen[:, None], float("-inf"))
            o, ls = torch.softmax(z, -1) @ kv[1][:, h].double(), torch.logsumexp(z, -1)
            if tree:
                out[b, at, heads], lse[b, at, heads] = o, ls
            else:
                out[b, heads], lse[b, heads] = o[0], ls[0]
    return dict(out=out, lse=lse)
