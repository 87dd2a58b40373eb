"""Generation and update of a small policy under the power controller.

The controller (here the hysteresis rule over the 72B-shaped trace) sets the
generation concurrency, batch by batch, all of it from the replayed trace: the
power of the batches below does not flow back.  Each batch runs both phases of
group-relative policy optimisation on the same GPU:

  generation  per token: keys and values into a paged cache with the position
              rotation (pe.kv_append), attention over it (pe.decode_attn), a
              sampled token and its log-probability (pe.token_logp)
  update      the batch scored again, the clipped surrogate with an entropy
              bonus, and its gradient in the logits (pe.token_logp_grad),
              applied to the output layer

    python examples/grpo_tokens.py [--batches 12 --tokens 24]

The policy is one attention layer with random weights; its reward is the share
of tokens from the lower half of the vocabulary, so that a rising reward shows
the whole loop at work.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2608_11226_gb300 import pe  # noqa: E402
from paper_2608_11226_gb300 import workloads as W  # noqa: E402

VOCAB, WIDTH, HQ, HKV, D, PAGE = 4000, 512, 8, 2, 64, 16
BF16 = torch.bfloat16


class Policy:
    def __init__(self, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def w(*shape):
            return (torch.randn(shape, generator=g, device="cuda") * shape[0] ** -0.5).to(BF16)

        self.embed = torch.randn((VOCAB, WIDTH), generator=g, device="cuda").to(BF16)
        self.wqkv, self.wo = w(WIDTH, (HQ + 2 * HKV) * D), w(HQ * D, WIDTH)
        self.wu = w(WIDTH, VOCAB).float()  # fp32 master of the trained output layer


def controller_levels(batches: int):
    """Concurrency levels (0..15) that the hysteresis rule sets, one for each batch."""
    wl = W.make_72b(n_envs=1)
    env = pe.Env(wl.env, torch.from_numpy(wl.trace), torch.from_numpy(wl.phase))
    buf = pe.alloc_rule_rollout(wl.env, 32 * batches)
    pe.rollout_rule(env, W.hysteresis_rule(wl.env.budget_q), 32 * batches, 0, buf)
    levels = buf["act"][::32, 0].tolist()
    env.close()
    return levels


def generate(p: Policy, n: int, tokens: int, rot: torch.Tensor, g: torch.Generator):
    """n sequences of `tokens` sampled tokens: (states [tokens * n, WIDTH], tokens, logp)."""
    pages = -(-tokens // PAGE)
    kv = [torch.zeros((n * pages, PAGE, HKV, D), dtype=BF16, device="cuda") for _ in range(2)]
    table = torch.randperm(n * pages, generator=g, device="cuda").to(torch.int32).view(n, pages)
    cache = pe.KVCache(*kv, table)
    work = pe.alloc_workspace(pe.decode_attn_workspace_bytes(cache, HQ))
    states = torch.empty((tokens, n, WIDTH), dtype=BF16, device="cuda")
    ids = torch.empty((tokens, n), dtype=torch.int32, device="cuda")
    logp = torch.empty((tokens, n), device="cuda")
    out = torch.empty((n, HQ, D), dtype=BF16, device="cuda")
    pos = torch.zeros(n, dtype=torch.int32, device="cuda")
    token = torch.zeros(n, dtype=torch.int64, device="cuda")  # every sequence starts from token 0
    wu = p.wu.to(BF16)
    for t in range(tokens):
        x = p.embed[token]
        qkv = (x @ p.wqkv).view(n, HQ + 2 * HKV, D)
        q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
        pe.kv_append(cache, k, v, pos, q=q, rot=rot)  # q is rotated in place
        pos += 1
        pe.decode_attn(cache, q, pos, out, workspace=work)
        states[t] = x + out.view(n, HQ * D) @ p.wo
        logits = states[t] @ wu
        gumbel = -torch.log(-torch.log(torch.rand((n, VOCAB), generator=g, device="cuda").clamp_(1e-7, 1 - 1e-7)))
        token = (logits.float() + gumbel).argmax(1)
        ids[t] = token
        pe.token_logp(logits, ids[t], logp[t])
    return states.view(-1, WIDTH), ids, logp


def update(p: Policy, states, ids, logp_old, lr: float, epochs: int = 2, clip: float = 0.2, ent_coef: float = 1e-3):
    """Clipped surrogate on group-centred rewards, plus an entropy bonus; returns what it saw."""
    reward = (ids < VOCAB // 2).float().mean(0)              # of each sequence
    adv = ((reward - reward.mean()) / (reward.std() + 1e-6)).expand_as(logp_old).reshape(-1)
    tok, old = ids.view(-1), logp_old.view(-1)
    n = tok.numel()
    logp, entropy, lse = (torch.empty(n, device="cuda") for _ in range(3))
    seen = {}
    for e in range(epochs):
        logits = states @ p.wu.to(BF16)
        pe.token_logp(logits, tok, logp, entropy=entropy, lse=lse)
        ratio = torch.exp(logp - old)
        unclipped = torch.where(adv >= 0, ratio <= 1 + clip, ratio >= 1 - clip)
        g_logp = -adv * ratio * unclipped / n
        g_entropy = torch.full((n,), -ent_coef / n, device="cuda")
        pe.token_logp_grad(logits, tok, lse, logits, g_logp=g_logp, entropy=entropy, g_entropy=g_entropy)  # in place
        p.wu -= lr * (states.float().T @ logits.float())
        if e == 0:
            seen = dict(reward=float(reward.mean()), entropy=float(entropy.mean()), drift=float((logp - old).abs().max()))
    return seen


def main(batches: int = 12, tokens: int = 24, lr: float = 2.0, seed: int = 0):
    p, rot = Policy(seed), pe.rot_table(tokens, D)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    rows = []
    for i, level in enumerate(controller_levels(batches)):
        n = 8 * (level + 1)
        states, ids, logp = generate(p, n, tokens, rot, g)
        s = update(p, states, ids, logp, lr)
        rows.append(dict(batch=i, level=level, sequences=n, **s))
        print("batch {batch}: level {level}, {sequences} sequences, reward {reward:.3f}, entropy {entropy:.2f}, "
              "sampled against scored log-probability {drift:.1e}".format(**rows[-1]))
    return rows


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    a.add_argument("--batches", type=int, default=12)
    a.add_argument("--tokens", type=int, default=24)
    main(**vars(a.parse_args()))
