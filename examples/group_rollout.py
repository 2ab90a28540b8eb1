"""A policy update on groups of completions, from the prompt to the gradient.

    python examples/group_rollout.py [--steps 30] [--groups 4] [--completions 16] [--tokens 24]

A small random token model (embedding, one attention layer, output head) answers N prompts with G
completions each. Every token runs through

    rlcs_shared_prefix_attn   attention over the group's prompt, kept once, and the completion so far,
    rlcs_sample               the next token and the log-probability it was drawn with,

and every batch of completions through

    rlcs_gae_masked           advantages of the reward on each completion's last token, whitened over
                              the tokens up to it,
    rlcs_policy_loss          the clipped loss and its gradient by the logits.

The reward is the share of tokens in the upper half of the vocabulary; the output head is trained.
Prints the mean reward of each step; with random weights it starts near 0.5 and rises.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2608_17641_amd as rl  # noqa: E402


class Model:
    """Embedding, one attention layer with grouped heads, output head."""

    def __init__(self, vocab=512, width=256, heads=8, key_heads=2, head_dim=64, dtype=torch.bfloat16, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda a, b: (torch.randn(a, b, device="cuda", generator=g) / math.sqrt(a)).to(dtype)  # noqa: E731
        self.heads, self.key_heads, self.head_dim, self.vocab = heads, key_heads, head_dim, vocab
        self.embed = torch.randn(vocab, width, device="cuda", generator=g).to(dtype)
        self.wq, self.wo = w(width, heads * head_dim), w(heads * head_dim, width)
        self.wkv = w(width, 2 * key_heads * head_dim)
        self.head = w(width, vocab).float()  # trained, in float32

    def keys_values(self, x):
        kv = (x @ self.wkv).view(*x.shape[:-1], 2, self.key_heads, self.head_dim)
        return kv[..., 0, :, :], kv[..., 1, :, :]


def rollout(model, prompts, prompt_len, completions, tokens, temperature=1.0, generator=None):
    """Draws `tokens` tokens for `completions` completions of every prompt. Returns the hidden states
    [N, G, T, width] that the logits came from, the tokens and their log-probabilities [N, G, T]."""
    N, G, dev = prompts.shape[0], completions, prompts.device
    kp, vp = model.keys_values(model.embed[prompts.long()])  # the prompt's keys, once for the group
    shape = (N, G, tokens, model.key_heads, model.head_dim)
    ks, vs = (torch.empty(shape, dtype=kp.dtype, device=dev) for _ in range(2))
    last = prompts.gather(1, prompt_len.long()[:, None] - 1).expand(N, G)
    hidden, drawn, logps = [], [], []
    length = torch.zeros((N, G), dtype=torch.int32, device=dev)
    for t in range(tokens):
        x = model.embed[last.long()]
        if t > 0:  # (the prompt's last token is in the prefix already)
            ks[:, :, t - 1], vs[:, :, t - 1] = model.keys_values(x)
            length += 1
        q = (x @ model.wq).view(N, G, model.heads, model.head_dim)
        o, _ = rl.rlcs_shared_prefix_attn(q, kp, vp, ks, vs, prompt_len, length, want_lse=False)
        h = (x + o.view(N, G, -1) @ model.wo).float()
        h = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6)
        logits = h @ model.head
        noise = torch.empty_like(logits).exponential_(generator=generator)
        last, logp = rl.rlcs_sample(logits, noise, temperature=temperature)
        hidden.append(h)
        drawn.append(last)
        logps.append(logp)
    return torch.stack(hidden, 2), torch.stack(drawn, 2), torch.stack(logps, 2)


def advantages(reward, tokens):
    """Whitened advantages [B, T] of a reward [B] on each completion's last token."""
    B = reward.shape[0]
    r = torch.zeros((B, tokens), device=reward.device)
    r[:, -1] = reward
    term = torch.zeros((B, tokens), dtype=torch.uint8, device=reward.device)
    term[:, -1] = 1
    adv, _ = rl.rlcs_gae_masked(r, torch.zeros_like(r), None, term, gamma=1.0, lam=1.0, normalize=True, want_ret=False)
    return adv


def update(model, hidden, drawn, logp_old, adv, rate, epochs=2):
    """Steps of the clipped policy loss on the output head."""
    T = drawn.shape[-1]
    h, a = hidden.reshape(-1, T, hidden.shape[-1]), drawn.reshape(-1, T)
    weight = torch.full_like(adv, 1.0 / adv.numel())
    for _ in range(epochs):
        loss, grad, _, _ = rl.rlcs_policy_loss(h @ model.head, a, logp_old.reshape(-1, T), adv, weight, clip_low=0.2,
                                               clip_high=0.28, ent_coef=0.001)
        model.head -= rate * (h.reshape(-1, h.shape[-1]).t() @ grad.reshape(-1, grad.shape[-1]))
    return loss.sum()


def train(steps=30, groups=4, completions=16, tokens=24, prompt=200, rate=20.0, seed=0):
    """The mean reward of each step."""
    model = Model(seed=seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    rewards = []
    for _ in range(steps):
        prompts = torch.randint(0, model.vocab, (groups, prompt), device="cuda", generator=g, dtype=torch.int32)
        prompt_len = torch.randint(prompt // 2, prompt + 1, (groups,), device="cuda", generator=g, dtype=torch.int32)
        hidden, drawn, logp = rollout(model, prompts, prompt_len, completions, tokens, generator=g)
        reward = (drawn >= model.vocab // 2).float().mean(-1).reshape(-1)
        update(model, hidden, drawn, logp, advantages(reward, tokens), rate)
        rewards.append(float(reward.mean()))
    return rewards


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 30), ("groups", 4), ("completions", 16), ("tokens", 24)):
        p.add_argument(f"--{name}", type=int, default=value)
    args = p.parse_args()
    for i, r in enumerate(train(args.steps, args.groups, args.completions, args.tokens)):
        print(f"step {i}: mean reward {r:.3f}", flush=True)
