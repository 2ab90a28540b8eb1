"""Groups of completions drawn with a small drafting policy and checked against the target, over a paged cache.

    python examples/speculative_rollout.py [--steps 6] [--groups 3] [--completions 4] [--tokens 24] [--drafted 3]

Two random token models (embedding, one attention layer, output head), the target and a smaller draft of it, keep their
keys and values in pages of one cache, under one table. A step draws completions of new prompts:

    rlcs_pages_resize      pages for the prompts, for every round's new tokens, and back what fell,
    rlcs_pages_fork        every prompt's pages shared by its group,
    rlcs_pages_copy        the page that a prompt ends in, once a completion grows past it,
    rlcs_paged_write       keys and values of new tokens,
    rlcs_paged_attn        single drafted tokens (draft) and the round's whole chunk (target),
    rlcs_sample            the drafted tokens,
    rlcs_verify_draft      which of them stand, the token after them, log-probabilities under the target,

and then trains the draft's output head on the target's largest logits (rlcs_distill_loss). Prints each step's mean
number of tokens a round and the distillation loss.
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import paper_2608_17641_amd as rl  # noqa: E402

PAGE = 16


class Model:
    """Embedding, one attention layer with grouped heads, output head."""

    def __init__(self, vocab, width, heads, key_heads, head_dim, dtype, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        w = lambda a, b: (torch.randn(a, b, device="cuda", generator=g) / math.sqrt(a)).to(dtype)  # noqa: E731
        self.heads, self.key_heads, self.head_dim = heads, key_heads, head_dim
        self.embed = torch.randn(vocab, width, device="cuda", generator=g).to(dtype)
        self.wq, self.wo, self.wkv = w(width, heads * head_dim), w(heads * head_dim, width), w(width, 2 * key_heads * head_dim)
        self.head = 2.0 * w(width, vocab).float()

    def keys_values(self, tokens):
        kv = (self.embed[tokens.long()] @ self.wkv).view(-1, 2, self.key_heads, self.head_dim)
        return kv[:, 0], kv[:, 1]

    def hidden(self, tokens, cache, table, length, max_chunk):
        """What the head sees of each new token: all sequences have as many of them."""
        x = self.embed[tokens.long()]
        q = (x @ self.wq).view(-1, self.heads, self.head_dim)
        o, _ = rl.rlcs_paged_attn(q, cache[0], cache[1], table, length, max_chunk=max_chunk, want_lse=False)
        h = (x + o.view(o.shape[0], -1) @ self.wo).float()
        return h * torch.rsqrt((h * h).mean(-1, keepdim=True) + 1e-6)


class Rollout:
    """The two models, their caches ([4, pages, PAGE, heads, D]: the target's and the draft's keys and values) and the table."""

    def __init__(self, groups=3, completions=4, vocab=256, prompt=40, tokens=24, drafted=3, dtype=torch.bfloat16, seed=0):
        self.N, self.G, self.B, self.K, self.tokens, self.prompt, self.vocab = groups, completions, groups * completions, drafted, tokens, prompt, vocab
        self.target = Model(vocab, 128, 4, 2, 64, dtype, seed)
        self.draft = Model(vocab, 128, 4, 2, 64, dtype, seed)  # the target's layers, a head that is near its own
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.draft.head = self.draft.head + 0.05 * torch.randn(self.draft.head.shape, device="cuda", generator=g)
        self.generator = g
        width = (prompt + tokens + 2 * drafted + 2) // PAGE + 2
        pages = self.B * width
        self.cache = torch.zeros((4, pages, PAGE, 2, 64), dtype=dtype, device="cuda")
        self.table = torch.full((self.B, width), -1, dtype=torch.int32, device="cuda")
        self.length = torch.zeros(self.B, dtype=torch.int32, device="cuda")
        self.refs = torch.zeros(pages, dtype=torch.int32, device="cuda")

    def resize(self, length):
        self.table, self.length, self.refs, moves = rl.rlcs_pages_resize(self.table, self.length, self.refs, length, page=PAGE)
        rl.rlcs_pages_copy(self.cache, moves)

    def write(self, tokens, length, q_start=None):
        for i, model in ((0, self.target), (2, self.draft)):
            k, v = model.keys_values(tokens)
            rl.rlcs_paged_write(k, v, self.cache[i], self.cache[i + 1], self.table, length, q_start)

    def exponential(self, *shape):
        return torch.empty(shape, device="cuda").exponential_(generator=self.generator)

    def start(self, prompts, prompt_len):
        """The prompts (but for their last tokens, which the first round begins with) in the first slot of each group, then shared."""
        first = torch.arange(self.N, device="cuda") * self.G
        wanted = torch.zeros_like(self.length)
        wanted[first] = prompt_len - 1
        self.resize(wanted)
        begin = torch.zeros(self.B + 1, dtype=torch.int32, device="cuda")
        begin[1:] = torch.cumsum(wanted, 0)
        held = torch.arange(prompts.shape[1], device="cuda")[None] < (prompt_len - 1)[:, None]
        self.write(prompts[held], self.length, begin)
        parent = torch.arange(self.B, device="cuda") // self.G * self.G
        self.table, self.length, self.refs = rl.rlcs_pages_fork(self.table, self.length, self.refs, parent.to(torch.int32), page=PAGE)
        return prompts.gather(1, prompt_len.long()[:, None] - 1)[:, 0].repeat_interleave(self.G)

    def round(self, last):
        """Draws up to K + 1 tokens for every sequence. Returns them, how many, their log-probabilities, and what the draft is
        trained on: its head's inputs and the target's logits, [B, K + 1, ...]."""
        B, K = self.B, self.K
        base = self.length.clone()
        self.resize(base + K + 1)
        drafts, rows, token = [], [], last
        for i in range(K):
            k, v = self.draft.keys_values(token)
            rl.rlcs_paged_write(k, v, self.cache[2], self.cache[3], self.table, base + i + 1)
            rows.append(self.draft.hidden(token, self.cache[2:], self.table, base + i + 1, 1) @ self.draft.head)
            token, _ = rl.rlcs_sample(rows[-1], self.exponential(B, self.vocab), want_logp=False)
            drafts.append(token)
        chunk = torch.stack([last] + drafts, 1)
        self.write(chunk.reshape(-1), self.length)
        logits = (self.target.hidden(chunk.reshape(-1), self.cache, self.table, self.length, K + 1) @ self.target.head).view(B, K + 1, -1)
        h = self.draft.hidden(chunk.reshape(-1), self.cache[2:], self.table, self.length, K + 1).view(B, K + 1, -1)
        u = torch.rand((B, K), device="cuda", generator=self.generator)
        tokens, count, logp = rl.rlcs_verify_draft(logits, torch.stack(rows, 1), torch.stack(drafts, 1), u, self.exponential(B, self.vocab))
        self.resize(base + count)  # the keys of what fell go
        return tokens, count, logp, h, logits

    def draw(self, prompts, prompt_len):
        """Completions of at least `tokens` tokens: (tokens, log-probabilities, how many) [B, ...], tokens a round, and the rounds' rows."""
        last = self.start(prompts, prompt_len)
        room = self.tokens + self.K + 1
        out = torch.full((self.B, room), -1, dtype=torch.int32, device="cuda")
        logps = torch.zeros((self.B, room), device="cuda")
        have = torch.zeros(self.B, dtype=torch.int64, device="cuda")
        places, rounds, rows = torch.arange(self.K + 1, device="cuda"), 0, []
        while int(have.min()) < self.tokens:
            tokens, count, logp, h, logits = self.round(last)
            rows.append((h, logits))
            going = have < self.tokens
            at = have[:, None] + places
            some = going[:, None] & (places < count[:, None])
            seq = torch.arange(self.B, device="cuda")[:, None].expand_as(at)
            out[seq[some], at[some]] = tokens[some]
            logps[seq[some], at[some]] = logp[some]
            have += torch.where(going, count, 0)
            rounds += 1
            # sequences that are done stay where they are
            self.resize(torch.where(going, self.length, (self.length - count).to(torch.int32)))
            last = torch.where(going, tokens.gather(1, count.long()[:, None] - 1)[:, 0], last)
        return out, logps, have, float(have.float().mean()) / rounds, rows

    def distill(self, rows, listed=16, rate=1.0):
        """A step of the draft's head on the target's largest logits."""
        h, logits = (torch.cat([r[i] for r in rows]).flatten(0, 1) for i in range(2))
        top = torch.topk(torch.log_softmax(logits, -1), listed)
        weight = torch.full((h.shape[0],), 1.0 / h.shape[0], device="cuda")
        loss, grad = rl.rlcs_distill_loss(h @ self.draft.head, top.indices.to(torch.int32), top.values.contiguous(), weight, tail=True)
        self.draft.head -= rate * (h.t() @ grad)
        return loss.sum()

    def free(self):
        self.resize(torch.zeros_like(self.length))


def train(steps=6, seed=0, **sizes):
    """(tokens a round, loss) of each step."""
    r = Rollout(seed=seed, **sizes)
    g = torch.Generator(device="cuda").manual_seed(seed + 2)
    seen = []
    for _ in range(steps):
        prompts = torch.randint(0, r.vocab, (r.N, r.prompt), device="cuda", generator=g, dtype=torch.int32)
        prompt_len = torch.randint(r.prompt // 2, r.prompt + 1, (r.N,), device="cuda", generator=g, dtype=torch.int32)
        _, _, _, a_round, rows = r.draw(prompts, prompt_len)
        seen.append((a_round, float(r.distill(rows))))
        r.free()
    return seen


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("steps", 6), ("groups", 3), ("completions", 4), ("tokens", 24), ("drafted", 3)):
        p.add_argument(f"--{name}", type=int, default=value)
    args = p.parse_args()
    for i, (n, loss) in enumerate(train(args.steps, groups=args.groups, completions=args.completions, tokens=args.tokens, drafted=args.drafted)):
        print(f"step {i}: {n:.2f} tokens a round, distillation loss {loss:.4f}", flush=True)
