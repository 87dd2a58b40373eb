"""The token operators whose speed is measured: the inner calls of the two
phases of the post-training that the controller governs.

  append  keys and values of new tokens into a paged cache, with the position
          rotation of queries and keys applied on the way (generation)
  decode  attention of one new token per sequence over that cache (generation)
  logp    log-probabilities of given tokens with entropy and the top
          alternatives of each row (scoring, and the record of a sampled token)
  grad    the gradient of log-probabilities and entropies in the logits (update)

Where ``own`` is true, ``run`` makes the calls of the public binding; where it
is false, the same operators in elementary torch operations in 32 bits,
rounded once at the end.  ``exact`` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
MOST_BYTES = 4.4e9  # of a drawn case: what the largest listed ones read and write


def listed():
    return [
        # one decode step of 32 running sequences, each at a position of its own: latency counts
        dict(name="append_step", op="append", T=32, seqs=32, start=500, Hq=32, Hkv=8, D=128, page=16, dtype="bf16",
             rot=128, inter=False, layout="slot", fused=True),
        # prompts of odd lengths entering a cache of odd pages: interleaved pairs, half of each head rotated
        dict(name="append_prompts_odd", op="append", T=4001, seqs=7, start=0, Hq=16, Hkv=16, D=64, page=24, dtype="f16",
             rot=32, inter=True, layout="head", fused=False),
        # a long prefill of many queries per key head, from one fused projection
        dict(name="append_prefill", op="append", T=32768, seqs=8, start=1000, Hq=64, Hkv=8, D=128, page=64,
             dtype="bf16", rot=128, inter=False, layout="slot", fused=True),
        # one user, a short conversation: latency counts
        dict(name="decode_one", op="decode", B=1, len=700, lens="full", Hq=32, Hkv=8, D=128, page=16, dtype="bf16",
             window=0, layout="slot"),
        # the largest generation batch, at ragged lengths, one slot idle
        dict(name="decode_batch", op="decode", B=128, len=8192, lens="spread", Hq=64, Hkv=8, D=128, page=16,
             dtype="bf16", window=0, layout="slot"),
        # one very long context: the split over the cache's length carries it
        dict(name="decode_long", op="decode", B=1, len=262143, lens="full", Hq=32, Hkv=8, D=128, page=64, dtype="f16",
             window=0, layout="head"),
        # one key head under many queries, wide heads, odd pages, a sliding window
        dict(name="decode_shared_window", op="decode", B=37, len=20011, lens="spread", Hq=20, Hkv=1, D=256, page=24,
             dtype="bf16", window=8192, layout="slot"),
        # the record of one sampled token: one row, its alternatives: latency counts
        dict(name="logp_one", op="logp", n=1, V=131072, dtype="bf16", top=20, scale=1.0, pad=0, masked=False),
        # odd rows of 32-bit logits under a temperature, some tokens forbidden by -inf
        dict(name="logp_odd", op="logp", n=777, V=50001, dtype="f32", top=5, scale=1.25, pad=3, masked=True),
        # the update phase's scoring of a batch of responses, and its gradient
        dict(name="logp_score", op="logp", n=8192, V=131072, dtype="bf16", top=0, scale=1.0, pad=0, masked=False),
        dict(name="grad_score", op="grad", n=8192, V=131072, dtype="bf16", scale=1.0, pad=0, masked=False),
        # the gradient at odd sizes, 32-bit logits under a temperature, some tokens forbidden
        dict(name="grad_odd", op="grad", n=333, V=32003, dtype="f32", scale=0.8, pad=5, masked=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        op = rng.choice(["append", "decode", "decode", "logp", "grad"])
        if op in ("append", "decode"):
            D = rng.choice([64, 128, 128, 256])
            Hkv = rng.choice([1, 2, 4, 8, 8, 16])
            c = dict(op=op, Hq=Hkv * rng.choice([1, 2, 4, 5, 8, 8, 16, 20]), Hkv=Hkv, D=D,
                     page=rng.choice([8, 16, 16, 24, 64, 100, 256]), dtype=rng.choice(["bf16", "bf16", "f16"]),
                     layout=rng.choice(["slot", "head"]))
            if c["Hq"] > 128:
                continue
        if op == "append":
            T = _log(rng, 1, 32768)
            step = rng.random() < 0.4
            c.update(T=min(T, 512) if step else T, seqs=min(T, 512) if step else min(T, rng.randint(1, 16)),
                     start=_log(rng, 1, 1024), rot=rng.choice([D, D, D // 2]), inter=rng.random() < 0.3,
                     fused=rng.random() < 0.7)
        elif op == "decode":
            c.update(B=_log(rng, 1, 256), len=_log(rng, 16, 262144), lens=rng.choice(["full", "spread", "spread"]),
                     window=rng.choice([0, 0, 0, 1000, 4096]))
            # the plain form gathers the whole table: bound that, not only what is attended to
            if c["B"] * c["len"] * Hkv * D * 4 > MOST_BYTES:
                continue
        else:
            c = dict(op=op, n=_log(rng, 1, 8192), V=_log(rng, 1000, 262144), dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                     scale=rng.choice([1.0, 1.0, 0.7, 1.25]), pad=rng.choice([0, 0, 1, 8, 61]), masked=rng.random() < 0.3)
            if op == "logp":
                c["top"] = rng.choice([0, 0, 1, 5, 20])
            if c["n"] * c["V"] > (2 ** 28 if c.get("top") else 2 ** 30):
                continue
        if work(c)["bytes"] <= MOST_BYTES:
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


def _attended(case):
    w = case["window"]
    return sum(min(n, w) if w else n for n in _lens(case))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(shape, g, dtype):
    if dtype == torch.float32:
        return torch.randn(shape, generator=g, device="cuda")
    x = torch.empty(shape, dtype=dtype, device="cuda")
    flat = x.view(-1)
    for a in range(0, flat.numel(), 1 << 28):
        b = min(flat.numel(), a + (1 << 28))
        flat[a:b] = torch.randn(b - a, generator=g, device="cuda", dtype=dtype)
    return x


def _storage(case, n_pages, fill, g):
    """Page storage of keys or values as [pages, slots, heads, head_dim]; the
    "head" layout keeps each head's slots of a page together in memory."""
    Hkv, D, page = case["Hkv"], case["D"], case["page"]
    dt = DTYPES[case["dtype"]]
    shape = (n_pages, page, Hkv, D) if case["layout"] == "slot" else (n_pages, Hkv, page, D)
    x = _randn(shape, g, dt) if fill else torch.zeros(shape, dtype=dt, device="cuda")
    return x if case["layout"] == "slot" else x.transpose(1, 2)


def _table(n_seqs, max_pages, g):
    """Each sequence's pages, scattered over the pool as a running server's are."""
    n = n_seqs * max_pages
    return torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(n_seqs, max_pages)


def prepare(case, seed):
    g = _gen(seed)
    s = dict(case=case)
    if case["op"] == "append":
        T, S, Hq, Hkv, D, page = (case[k] for k in ("T", "seqs", "Hq", "Hkv", "D", "page"))
        dt = DTYPES[case["dtype"]]
        count = [T // S + (i < T % S) for i in range(S)]
        top = case["start"] + max(count)
        max_pages = -(-top // page)
        s["k_cache"], s["v_cache"] = (_storage(case, S * max_pages, False, g) for _ in range(2))
        s["table"] = _table(S, max_pages, g)
        first = torch.randint(0, case["start"] + 1, (S,), generator=g, device="cuda")
        cnt = torch.tensor(count, device="cuda")
        seq = torch.repeat_interleave(torch.arange(S, device="cuda"), cnt)
        within = torch.arange(T, device="cuda") - (torch.cumsum(cnt, 0) - cnt)[seq]
        s["positions"] = (first[seq] + within).to(torch.int32)
        s["seqs"] = None if T == S else seq.to(torch.int32)
        qkv = _randn((T, Hq + 2 * Hkv, D), g, dt)
        parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["q"], s["k"], s["v"] = parts if case["fused"] else (p.contiguous() for p in parts)
        half = case["rot"] // 2
        ang = torch.arange(top, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)
        s["rot"] = torch.cat([torch.cos(ang), torch.sin(ang)], 1).float().cuda()
        s["q_out"] = torch.empty((T, Hq, D), dtype=dt, device="cuda")
    elif case["op"] == "decode":
        B, Hq, Hkv, D, page = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
        dt = DTYPES[case["dtype"]]
        max_pages = -(-case["len"] // page)
        s["k_cache"], s["v_cache"] = (_storage(case, B * max_pages, True, g) for _ in range(2))
        s["table"] = _table(B, max_pages, g)
        order = torch.randperm(B, generator=g, device="cuda")
        s["lens"] = torch.tensor(_lens(case), dtype=torch.int32, device="cuda")[order]
        # scores of a standard deviation of two: some positions matter, none alone
        s["q"] = 2.0 * _randn((B, Hq, D), g, dt)
        s["out"] = torch.empty((B, Hq, D), dtype=dt, device="cuda")
        s["lse"] = torch.empty((B, Hq), device="cuda")
    else:
        n, V = case["n"], case["V"]
        dt = DTYPES[case["dtype"]]
        rows = _randn((n, V + case["pad"]), g, dt)
        # a peaked model: a wide spread of logits, a few far above the rest
        rows *= 2.5
        at = torch.randint(0, V // 4, (n, 4), generator=g, device="cuda") + V // 4 * torch.arange(4, device="cuda")
        rows.scatter_(1, at, (12.0 + 1.5 * torch.randn(n, 4, generator=g, device="cuda")).to(dt))
        s["logits"] = rows[:, :V]
        if case["masked"]:
            for a in range(0, n, 1024):
                part = s["logits"][a:a + 1024]
                part.masked_fill_(torch.rand(part.shape, generator=g, device="cuda") < 0.3, float("-inf"))
        pick = torch.randint(0, 4, (n, 1), generator=g, device="cuda")
        s["tokens"] = at.gather(1, pick)[:, 0].to(torch.int32)
        if n >= 16:
            s["tokens"][::16] = -1  # padding of the batch: no target
        if case["op"] == "logp":
            s["logp"], s["entropy"], s["lse"] = (torch.empty(n, device="cuda") for _ in range(3))
            k = case["top"]
            s["top_logp"] = torch.empty((n, k), device="cuda") if k else None
            s["top_id"] = torch.empty((n, k), dtype=torch.int32, device="cuda") if k else None
        else:
            s["lse"], s["entropy"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            for a in range(0, n, 256):  # the forward's record, as the caller kept it
                z = s["logits"][a:a + 256].double() * case["scale"]
                lse = torch.logsumexp(z, 1)
                p = torch.exp(z - lse[:, None])
                s["lse"][a:a + 256] = lse.float()
                s["entropy"][a:a + 256] = (lse - (p * z.clamp(min=-1e30)).sum(1)).float()
            s["g_logp"] = torch.randn(n, generator=g, device="cuda") / n
            s["g_entropy"] = torch.full((n,), -0.01 / n, device="cuda")
            s["dlogits"] = torch.empty_like(rows)[:, :V]
    if own:
        from paper_2608_11226_gb300 import pe

        if case["op"] in ("append", "decode"):
            s["cache"] = pe.KVCache(s["k_cache"], s["v_cache"], s["table"])
        if case["op"] == "decode":
            s["workspace"] = pe.alloc_workspace(pe.decode_attn_workspace_bytes(s["cache"], case["Hq"]))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        return _run_own(case["op"], s, case)
    return {"append": _plain_append, "decode": _plain_decode, "logp": _plain_logp, "grad": _plain_grad}[case["op"]](s, case)


def _run_own(op, s, case):
    from paper_2608_11226_gb300 import pe

    if op == "append":
        pe.kv_append(s["cache"], s["k"], s["v"], s["positions"], seqs=s["seqs"], q=s["q"], q_out=s["q_out"],
                     rot=s["rot"], interleaved=case["inter"])
        return dict(q=s["q_out"], k_cache=s["k_cache"], v_cache=s["v_cache"])
    if op == "decode":
        pe.decode_attn(s["cache"], s["q"], s["lens"], s["out"], window=case["window"], lse=s["lse"],
                       workspace=s["workspace"])
        return dict(out=s["out"], lse=s["lse"])
    if op == "logp":
        pe.token_logp(s["logits"], s["tokens"], s["logp"], entropy=s["entropy"], lse=s["lse"], top_logp=s["top_logp"],
                      top_id=s["top_id"], scale=case["scale"])
        return dict(logp=s["logp"], entropy=s["entropy"], lse=s["lse"], top_logp=s["top_logp"], top_id=s["top_id"])
    pe.token_logp_grad(s["logits"], s["tokens"], s["lse"], s["dlogits"], g_logp=s["g_logp"], entropy=s["entropy"],
                       g_entropy=s["g_entropy"], scale=case["scale"])
    return dict(dlogits=s["dlogits"])


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
    seq = torch.arange(case["T"], device="cuda") if s["seqs"] is None else s["seqs"].long()
    cs = s["rot"][pos]
    q = _rotate(s["q"], cs, case["rot"], case["inter"]).to(s["q"].dtype)
    k = _rotate(s["k"], cs, case["rot"], case["inter"]).to(s["k"].dtype)
    pages = s["table"][seq, pos // case["page"]].long()
    s["k_cache"][pages, pos % case["page"]] = k
    s["v_cache"][pages, pos % case["page"]] = s["v"]
    return dict(q=q, k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_decode(s, case):
    B, Hq, Hkv, D, w = (case[k] for k in ("B", "Hq", "Hkv", "D", "window"))
    t = s["table"].long()
    k = s["k_cache"][t].flatten(1, 2).float().permute(0, 2, 3, 1)  # [B, Hkv, D, positions]
    v = s["v_cache"][t].flatten(1, 2).float().transpose(1, 2)      # [B, Hkv, positions, D]
    q = s["q"].float().view(B, Hkv, Hq // Hkv, D)
    z = torch.matmul(q, k) * D ** -0.5
    j = torch.arange(z.shape[-1], device="cuda")[None]
    n = s["lens"][:, None]
    keep = (j < n) if not w else (j < n) & (j >= n - w)
    z = torch.where(keep[:, None, None], z, float("-inf"))
    m = z.amax(-1, keepdim=True)
    e = torch.exp(z - torch.where(m > float("-inf"), m, 0.0))
    l = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(l > 0, l, 1.0)
    return dict(out=o.view(B, Hq, D).to(s["q"].dtype), lse=(m + torch.log(l)).view(B, Hq))


def _plain_logp(s, case):
    x, k, t = s["logits"], case["top"], s["tokens"].long()
    z = x.float() * case["scale"]
    m = z.amax(1, keepdim=True)
    d = z - torch.where(m > float("-inf"), m, 0.0)
    e = torch.exp(d)
    S = e.sum(1)
    ln = torch.log(S)
    lse = m[:, 0] + ln
    has = (t >= 0) & (t < case["V"])
    zt = z.gather(1, t.clamp(0, case["V"] - 1)[:, None])[:, 0]
    logp = torch.where(has, (zt - m[:, 0]) - ln, 0.0)
    entropy = ln - (e * d.clamp(min=-1e30)).sum(1) / S
    top_logp = top_id = None
    if k:
        top_id = torch.sort(x, dim=1, descending=True, stable=True)[1][:, :k].contiguous()
        top_logp = d.gather(1, top_id) - ln[:, None]
        top_id = top_id.to(torch.int32)
    return dict(logp=logp, entropy=entropy, lse=lse, top_logp=top_logp, top_id=top_id)


def _plain_grad(s, case):
    t = s["tokens"].long()
    lp = s["logits"].float() * case["scale"] - s["lse"][:, None]
    p = torch.exp(lp)
    has = (t >= 0) & (t < case["V"])
    g = torch.where(has, s["g_logp"], 0.0)
    d = -p * (g[:, None] + s["g_entropy"][:, None] * (lp.clamp(min=-1e30) + s["entropy"][:, None]))
    d.scatter_add_(1, t.clamp(0, case["V"] - 1)[:, None], g[:, None])
    return dict(dlogits=(d * case["scale"]).to(s["logits"].dtype))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    op, e = case["op"], SIZE[case["dtype"]]
    if op == "append":
        T, Hq, Hkv, D = (case[k] for k in ("T", "Hq", "Hkv", "D"))
        # every head's row in and out; positions, page ids; the rotation rows of the positions met, at most
        return dict(bytes=2 * T * (Hq + 2 * Hkv) * D * e + T * 8 + min(T, case["start"] + T) * case["rot"] * 4,
                    flops=3 * T * (Hq + Hkv) * case["rot"])
    if op == "decode":
        B, Hq, Hkv, D = (case[k] for k in ("B", "Hq", "Hkv", "D"))
        n = _attended(case)
        return dict(bytes=2 * n * Hkv * D * e + 2 * B * Hq * D * e + B * Hq * 4 + 4 * n // case["page"] + 4 * B,
                    flops=4 * n * Hq * D)
    n, V = case["n"], case["V"]
    if op == "logp":
        return dict(bytes=n * V * e + 16 * n + 8 * n * case["top"], flops=8 * n * V)
    return dict(bytes=2 * n * V * e + 20 * n, flops=8 * n * V)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "decode": _exact_decode, "logp": _exact_logp, "grad": _exact_grad}[case["op"]](s, case)


def _exact_append(s, case):
    D, rot, T = case["D"], case["rot"], case["T"]
    half = rot // 2
    table = s["rot"].double()[s["positions"].long()]

    def turned(x):  # a pair as a complex number, turned by its angle
        x = x.double()
        lo = torch.arange(half, device="cuda") * 2 if case["inter"] else torch.arange(half, device="cuda")
        hi = lo + 1 if case["inter"] else lo + half
        w = torch.complex(x[..., lo], x[..., hi]) * torch.complex(table[:, None, :half], table[:, None, half:])
        y = x.clone()
        y[..., lo], y[..., hi] = w.real, w.imag
        return y

    seq = torch.arange(T, device="cuda") if s["seqs"] is None else s["seqs"].long()
    line = seq * s["table"].shape[1] * case["page"] + s["positions"].long()  # the token's place, page after page of the table
    page = s["table"].reshape(-1).long()[line // case["page"]]
    at = page * case["page"] + line % case["page"]
    caches = []
    for x in (turned(s["k"]), s["v"].double()):
        flat = torch.zeros((s["table"].numel() * case["page"], case["Hkv"], D), dtype=torch.float64, device="cuda")
        flat[at] = x
        caches.append(flat.view(-1, case["page"], case["Hkv"], D))
    return dict(q=turned(s["q"]), k_cache=caches[0], v_cache=caches[1])


def _exact_decode(s, case):
    B, Hq, Hkv, D, page = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    out = torch.zeros((B, Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), float("-inf"), dtype=torch.float64, device="cuda")
    for b, n in enumerate(s["lens"].tolist()):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        pages = s["table"][b, first // page:-(-n // page)].long()
        cut = slice(first - first // page * page, n - first // page * page)
        k = s["k_cache"][pages].flatten(0, 1)[cut]
        v = s["v_cache"][pages].flatten(0, 1)[cut]
        for h in range(Hkv):
            heads = slice(h * (Hq // Hkv), (h + 1) * (Hq // Hkv))
            z = (k[:, h].double() @ s["q"][b, heads].double().T) / math.sqrt(D)  # [positions, heads]
            lse[b, heads] = torch.logsumexp(z, 0)
            out[b, heads] = torch.softmax(z, 0).T @ v[:, h].double()
    return dict(out=out, lse=lse)


def _exact_logp(s, case):
    n, k = case["n"], case["top"]
    got = dict(logp=[], entropy=[], lse=[], top_logp=[])
    for a in range(0, n, 512):
        z = s["logits"][a:a + 512].double() * case["scale"]
        t = s["tokens"][a:a + 512].long()
        lsm = torch.log_softmax(z, 1)
        got["lse"].append(torch.logsumexp(z, 1))
        got["entropy"].append(torch.special.entr(lsm.exp()).sum(1))
        got["logp"].append(torch.where(t >= 0, lsm.gather(1, t.clamp(min=0)[:, None])[:, 0], 0.0))
        if k:
            got["top_logp"].append(lsm.topk(k, 1)[0])
    return dict({m: torch.cat(v) if v else None for m, v in got.items()}, top_id=None)


def _exact_grad(s, case):
    n, V = case["n"], case["V"]
    d = torch.empty((n, V), dtype=torch.float64, device="cuda")
    for a in range(0, n, 512):
        z = s["logits"][a:a + 512].double() * case["scale"]
        t = s["tokens"][a:a + 512].long()
        lsm = torch.log_softmax(z, 1)
        p = lsm.exp()
        h = torch.special.entr(p)
        H = h.sum(1, keepdim=True)
        one = torch.zeros_like(p)
        rows = torch.arange(t.numel(), device="cuda")[t >= 0]
        one[rows, t[t >= 0]] = 1.0
        g = torch.where(t >= 0, s["g_logp"][a:a + 512].double(), 0.0)[:, None]
        d[a:a + 512] = case["scale"] * (g * (one - p) + s["g_entropy"][a:a + 512].double()[:, None] * (h - p * H))
    return dict(dlogits=d)
