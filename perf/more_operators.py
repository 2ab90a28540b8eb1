"""What the operators of speculative group rollouts over a paged cache are measured on: attention of a
chunk of new tokens over the pages, writing the chunk's keys and values into them, the pages' own
life (fork, growth, copy, compaction), the check of drafted tokens against the target policy, and the
distillation of the drafting policy from the target's top logits.

With ``own`` false, ``run`` computes them in elementary torch operations; with ``own`` true it makes
the library's calls. Sizes are those of the benchmark's rollouts and of the group rollout's measurements
(32 heads on 8, 64 sequences, 4096 tokens, vocabularies of 32000, 50001 and 128000) or plain odd ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one decode step of eight short sequences of a small model: latency only
        dict(name="attn_8x1_300_f32", op="attn", B=8, T=1, L=300, Hq=8, Hkv=8, D=64, page=16, mixed=False, dtype="f32"),
        # a decode step of 64 long sequences, grouped heads: every key and value once
        dict(name="attn_64x1_8192_bf16", op="attn", B=64, T=1, L=8192, Hq=32, Hkv=8, D=128, page=64, mixed=False, dtype="bf16"),
        # the target's pass over one token and up to four drafted ones of 64 sequences, small pages
        dict(name="attn_64x5_4096_bf16", op="attn", B=64, T=5, L=4096, Hq=32, Hkv=8, D=128, page=16, mixed=False, dtype="bf16"),
        # tool outputs read into four long transcripts, a chunk each
        dict(name="attn_4x2048_16384_bf16", op="attn", B=4, T=2048, L=16384, Hq=32, Hkv=8, D=128, page=64, mixed=False, dtype="bf16"),
        # the new tokens of a decode step of 64 sequences, into small pages
        dict(name="write_64x5_f32", op="write", B=64, T=5, L=2048, Hkv=8, D=64, page=16, dtype="f32"),
        # two prompts of a layer, written as they are read
        dict(name="write_2x8192_bf16", op="write", B=2, T=8192, L=8192, Hkv=8, D=128, page=64, dtype="bf16"),
        # 16 completions forked from each of 4 prompts and grown by a few tokens: the shared last pages are copied
        dict(name="fork_4x16_2000_bf16", op="fork", N=4, G=16, L=2000, grow=8, page=16, pages=2048, layers=8, Hkv=8, D=128, dtype="bf16"),
        # half of a cache's pages, scattered, moved to its front
        dict(name="compact_8192_bf16", op="compact", B=64, pages=8192, used=0.5, page=64, layers=2, Hkv=8, D=128, dtype="bf16"),
        # eight sequences' four drafted tokens each: latency
        dict(name="verify_8x4_32000_f32", op="verify", B=8, K=4, V=32000, dtype="f32"),
        # a serving batch with a large vocabulary
        dict(name="verify_64x7_128000_bf16", op="verify", B=64, K=7, V=128000, dtype="bf16"),
        # a micro-batch of tokens against the teacher's 64 largest logits
        dict(name="distill_4096x32000_bf16", op="distill", M=4096, V=32000, K=64, tail=False, dtype="bf16"),
        # a large vocabulary, the mass outside the listed logits kept as a class of its own
        dict(name="distill_8192x128000_bf16", op="distill", M=8192, V=128000, K=128, tail=True, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "attn", "write", "fork", "compact", "verify", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    es = 4 if dtype == "f32" else 2
    if op == "attn":
        Hkv, D, B = rng.choice([1, 2, 4, 8]), rng.choice([64, 128]), _log_int(rng, 1, 64)
        Hq = Hkv * rng.choice([1, 2, 4, 7, 8])
        T, L = rng.choice([1, rng.randint(2, 8), _log_int(rng, 9, 2048)]), _log_int(rng, 16, 16384)
        # no more bytes of keys than the largest listed case of single tokens, nor more scores than the largest chunks'
        L = max(16, min(L, 64 * 8192 * 8 * 128 * 2 // (B * Hkv * D * es)))
        T = max(1, min(T, L, 4 * 32 * 2048 * 16384 // (B * Hq * L * (4 if dtype == "f32" else 1))))
        return dict(op=op, B=B, T=T, L=L, Hq=Hq, Hkv=Hkv, D=D, page=rng.choice([16, 32, 64, 256]), mixed=T > 8 and rng.random() < 0.4,
                    dtype=dtype)
    if op == "write":
        B, T = _log_int(rng, 1, 64), _log_int(rng, 1, 8192)
        T = max(1, min(T, 16384 // B))
        return dict(op=op, B=B, T=T, L=max(T, _log_int(rng, 16, 8192)), Hkv=rng.choice([1, 2, 4, 8]), D=rng.choice([64, 128]),
                    page=rng.choice([16, 32, 64, 256]), dtype=dtype)
    if op == "fork":
        N, G, page = _log_int(rng, 1, 8), _log_int(rng, 1, 32), rng.choice([16, 32])
        L, grow = _log_int(rng, 16, 4096), _log_int(rng, 1, 64)
        need = N * (-(-L // page)) + N * G * (grow // page + 2)
        return dict(op=op, N=N, G=G, L=L, grow=grow, page=page, pages=rng.randint(need, 2 * need), layers=rng.choice([2, 4, 8]),
                    Hkv=rng.choice([1, 2, 4]), D=rng.choice([64, 128]), dtype=dtype)
    if op == "compact":
        return dict(op=op, B=_log_int(rng, 1, 64), pages=_log_int(rng, 64, 8192), used=round(rng.uniform(0.1, 0.9), 2),
                    page=rng.choice([16, 32, 64]), layers=rng.choice([2, 4]) if dtype == "bf16" else 1, Hkv=rng.choice([1, 2, 4]),
                    D=rng.choice([64, 128]), dtype=dtype)
    V = _log_int(rng, 16, 128000)
    if op == "verify":
        K = rng.randint(1, 8)
        return dict(op=op, B=max(1, min(256, _log_int(rng, 1, max(2, (1 << 26) // (V * (2 * K + 3)))))), K=K, V=V, dtype=dtype)
    return dict(op=op, M=max(1, min(1 << 16, _log_int(rng, 16, max(17, (1 << 28) // V)))), V=V, K=min(V, _log_int(rng, 1, 128)),
                tail=rng.random() < 0.5, dtype=dtype)


# ---------------------------------------------------------------- inputs

def _tables(pages, counts, width, g):
    """A table of `width` page numbers a sequence, its first counts[b] scattered over all pages, the others -1."""
    perm = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    at = torch.arange(width, device="cuda")[None] + (torch.cumsum(counts, 0) - counts)[:, None]
    return torch.where(torch.arange(width, device="cuda")[None] < counts[:, None], perm[at.clamp(max=pages - 1)], -1).to(torch.int32)


def _references(table, pages):
    entries = torch.where(table >= 0, table, pages).reshape(-1).long()
    return torch.bincount(entries, minlength=pages + 1)[:pages].to(torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(shape, scale=1.0):
        t = torch.empty(shape, device="cuda", dtype=dt)
        return t.normal_(0.0, scale, generator=g)

    def below(n, shape):
        return torch.floor(torch.rand(shape, device="cuda", generator=g) * n).clamp_(max=n - 1).to(torch.int64)

    s = dict(case=case)
    op = case["op"]
    if op in ("attn", "write"):
        B, T, L, Hkv, D, page = (case[k] for k in ("B", "T", "L", "Hkv", "D", "page"))
        # the first sequence is the longest, with the longest chunk; the others' lengths go down to a
        # quarter. Chunks of drafted tokens have any number of them, longer ones at least half of the most; who
        # has which is drawn, how many tokens there are in all is the case's
        at = torch.arange(B, device="cuda")
        chunk = T - at % T if T <= 8 else T - at * 37 % max(1, T // 2)
        if case.get("mixed"):
            chunk = torch.where(at % 2 == 1, torch.ones_like(chunk), chunk)
        if B > 2:
            chunk = torch.cat([chunk[:1], chunk[1:][torch.randperm(B - 1, device="cuda", generator=g)]])
        length = L - below(3 * L // 4 + 1, (B,))
        length[0] = L
        length = torch.maximum(length, chunk)
        width = -(-L // page)
        counts = -(-length // page)
        pages = B * width + 3
        s["table"] = _tables(pages, counts, width, g)
        s["length"] = length.to(torch.int32)
        start = torch.zeros(B + 1, dtype=torch.int64, device="cuda")
        start[1:] = torch.cumsum(chunk, 0)
        s["q_start"] = start.to(torch.int32)
        s["tokens"] = int(start[-1])
        s["k_cache"], s["v_cache"] = normal((pages, page, Hkv, D)), normal((pages, page, Hkv, D))
        if op == "attn":
            s["q"] = normal((s["tokens"], case["Hq"], D))
            s["scale"] = 1.0 / math.sqrt(D)
        else:
            s["k"], s["v"] = normal((s["tokens"], Hkv, D)), normal((s["tokens"], Hkv, D))
        return s
    if op == "fork":
        N, G, L, page, pages = (case[k] for k in ("N", "G", "L", "page", "pages"))
        B = N * (G + 1)
        width = -(-(L + case["grow"]) // page)
        length = torch.zeros(B, dtype=torch.int64, device="cuda")
        length[:N] = (L - below(L // 4 + 1, (N,))).clamp(min=1)
        length[0] = L
        s["table"] = _tables(pages, -(-length // page), width, g)
        s["length"] = length.to(torch.int32)
        s["refs"] = _references(s["table"], pages)
        slots = torch.arange(B, device="cuda")
        s["parent"] = torch.where(slots < N, slots, (slots - N) // G).to(torch.int32)
        # completions grow by 1 to `grow` tokens; the prompts stay
        grown = length[s["parent"].long()] + torch.where(slots < N, 0, 1 + below(case["grow"], (B,)))
        s["new_length"] = grown.to(torch.int32)
        s["cache"] = normal((case["layers"], pages, page, case["Hkv"], case["D"]))
        return s
    if op == "compact":
        B, pages, page = case["B"], case["pages"], case["page"]
        used = max(B, int(pages * case["used"]))
        counts = used // B + (torch.arange(B, device="cuda") < used % B).long()
        s["table"] = _tables(pages, counts, used // B + 1, g)
        s["refs"] = _references(s["table"], pages)
        s["cache"] = normal((case["layers"], pages, page, case["Hkv"], case["D"]))
        return s
    if op == "verify":
        B, K, V = case["B"], case["K"], case["V"]
        s["target"] = normal((B, K + 1, V), 2.5)
        # a draft that is near the target: most of its tokens stand
        s["draft"] = (0.9 * s["target"][:, :K].float() + torch.randn((B, K, V), device="cuda", generator=g) * 0.8).to(dt)
        race = torch.empty((B, K, V), device="cuda").exponential_(generator=g)
        s["draft_tokens"] = torch.argmax(s["draft"].float() - torch.log(race), -1).to(torch.int32)
        s["u"] = torch.rand((B, K), device="cuda", generator=g)
        s["noise"] = torch.empty((B, V), device="cuda").exponential_(generator=g)
        s["n_draft"] = (K - below(K + 1, (B,)) // 2).to(torch.int32)
        return s
    M, V, K = case["M"], case["V"], case["K"]
    s["logits"] = normal((M, V), 2.5)
    s["top_ids"], s["top_logp"] = torch.empty((M, K), dtype=torch.int32, device="cuda"), torch.empty((M, K), device="cuda")
    step = max(1, (1 << 28) // V)
    for i in range(0, M, step):  # a teacher near the student
        x = s["logits"][i:i + step].float() * 0.9
        x = x + torch.randn(x.shape, device="cuda", generator=g)
        top = torch.topk(x, K)
        s["top_ids"][i:i + step] = top.indices.to(torch.int32)
        s["top_logp"][i:i + step] = top.values - torch.logsumexp(x, -1, keepdim=True)
    keep = (torch.rand((M,), device="cuda", generator=g) < 0.67).float()
    s["weight"] = keep / keep.sum().clamp_(min=1.0)
    return s


# ---------------------------------------------------------------- the plain forms

def _chunks(s):
    """Each sequence's number of new tokens, and every token's sequence and place in its chunk."""
    start = s["q_start"].long()
    token = torch.arange(s["tokens"], device=start.device)
    seq = torch.searchsorted(start[1:].contiguous(), token, right=True)
    return start[1:] - start[:-1], seq, token - start[seq]


def _plain_attn(s):
    c = s["case"]
    B, T, L, Hq, Hkv, D, page = (c[k] for k in ("B", "T", "L", "Hq", "Hkv", "D", "page"))
    r = Hq // Hkv
    chunk, seq, place = _chunks(s)
    length, dev = s["length"].long(), s["q"].device
    # sequences side by side, heads before tokens
    pages = s["table"].long().clamp(min=0)
    there = (torch.arange(L, device=dev)[None] < length[:, None])
    k = s["k_cache"][pages].reshape(B, -1, Hkv, D)[:, :L].float().permute(0, 2, 3, 1).contiguous()
    v = torch.where(there[..., None, None], s["v_cache"][pages].reshape(B, -1, Hkv, D)[:, :L].float(), 0.0)
    v = v.permute(0, 2, 1, 3).contiguous()
    q = torch.zeros((B, T, Hq, D), device=dev)
    q[seq, place] = s["q"].float()
    q = q.reshape(B, T, Hkv, r, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * r, D)
    a = torch.matmul(q, k).mul_(s["scale"]).view(B, Hkv, T, r, L)
    # token i of a chunk of n sees the keys up to its own: the first length - n + i + 1
    sees = (length - chunk)[:, None] + torch.arange(T, device=dev)[None] + 1
    hidden = torch.arange(L, device=dev)[None, None] >= sees[..., None]
    a.masked_fill_(hidden[:, None, :, None], -torch.inf)
    m = a.amax(-1, keepdim=True)
    m = torch.where(torch.isinf(m), 0.0, m)
    a.sub_(m).exp_()
    z = a.sum(-1)
    o = torch.matmul(a.view(B, Hkv, T * r, L), v).view(B, Hkv, T, r, D)
    o = torch.where(z[..., None] > 0, o / z[..., None], 0.0).permute(0, 2, 1, 3, 4).reshape(B, T, Hq, D)
    lse = (m[..., 0] + torch.log(z)).permute(0, 2, 1, 3).reshape(B, T, Hq)
    return o[seq, place].to(s["q"].dtype), lse[seq, place]


def _plain_write(s):
    page = s["case"]["page"]
    chunk, seq, place = _chunks(s)
    at = (s["length"].long() - chunk)[seq] + place
    number = s["table"].long()[seq, at // page]
    s["k_cache"][number, at % page] = s["k"]
    s["v_cache"][number, at % page] = s["v"]
    return s["k_cache"], s["v_cache"]


def _count(refs, entries, counted, by):
    """References with `by` added for each entry that is counted."""
    amount = torch.where(counted & (entries >= 0), by, 0).to(refs.dtype)
    return refs.index_add(0, entries.clamp(min=0).reshape(-1).long(), amount.reshape(-1))


def _plain_fork_pages(table, length, refs, parent, page):
    B, W = table.shape
    slots = torch.arange(B, device=table.device)
    par = torch.where((parent >= 0) & (parent < B), parent, slots).long()
    held = torch.arange(W, device=table.device)[None] < (-(-length // page))[:, None]
    old = torch.where(held, table, -1)
    new = old[par]
    moved = (par != slots)[:, None].expand(B, W)
    refs = _count(_count(refs, new, moved, 1), old, moved, -1)
    return new, length[par], refs


def _plain_resize_pages(table, length, refs, new_length, page):
    B, W = table.shape
    dev = table.device
    at, slots = torch.arange(W, device=dev)[None], torch.arange(B, device=dev)
    old = length.long()
    new = torch.where((new_length < 0) | (new_length > W * page), old, new_length.long())
    held, wanted = -(-old // page), -(-new // page)
    kept = torch.minimum(held, wanted)
    refs = _count(refs, table, (at >= kept[:, None]) & (at < held[:, None]), -1)
    table = torch.where(at < kept[:, None], table, -1)
    # a page that ends inside and is shared is left to the others: the sequence goes on in a copy
    edge = (old // page).clamp(max=W - 1)
    last = table.gather(1, edge[:, None])[:, 0]
    copies = (new > old) & (old % page != 0) & (last >= 0) & (refs[last.clamp(min=0).long()] > 1)
    need = torch.where(new > old, wanted - held + copies.long(), 0)
    free = torch.sort((refs > 0).to(torch.int8), stable=True).indices
    offset = torch.cumsum(need, 0) - need
    granted = (need == 0) | (offset + need <= (refs <= 0).sum())
    new = torch.where(granted, new, old)
    copies &= granted
    fresh = free[offset.clamp(max=free.numel() - 1)]
    moves = torch.where(copies[:, None], torch.stack([last.long(), fresh], 1), -1).to(torch.int32)
    fills = (at >= held[:, None]) & (at < wanted[:, None]) & granted[:, None]
    rank = (offset + copies)[:, None] + at - held[:, None]
    table = torch.where(fills, free[rank.clamp(0, free.numel() - 1)].to(torch.int32), table)
    swapped = copies[:, None] & (at == edge[:, None])
    table = torch.where(swapped, fresh[:, None].to(torch.int32), table)
    refs = _count(refs, table, fills | swapped, 1)
    refs = _count(refs, last, copies, -1)
    return table, new.to(torch.int32), refs, moves


def _plain_copy_pages(cache, moves):
    moves = moves[moves[:, 0] >= 0].long()
    cache[:, moves[:, 1]] = cache[:, moves[:, 0]]
    return cache


def _plain_compact_pages(table, refs):
    pages = refs.numel()
    number = torch.arange(pages, device=refs.device)
    used = refs > 0
    count = used.sum()
    moving, holes = used & (number >= count), ~used & (number < count)
    hole = torch.sort((~holes).to(torch.int8), stable=True).indices  # the holes first, from the lowest
    rank = torch.cumsum(moving, 0) - 1
    to = torch.where(moving, hole[rank.clamp(min=0)], number)
    at = torch.sort((~moving).to(torch.int8), stable=True).indices[:pages // 2]
    some = torch.arange(pages // 2, device=refs.device) < moving.sum()
    moves = torch.where(some[:, None], torch.stack([at, hole[:pages // 2]], 1), -1).to(torch.int32)
    live = (table >= 0) & used[table.clamp(min=0).long()]
    table = torch.where(live, to[table.clamp(min=0).long()].to(torch.int32), -1)
    refs = torch.zeros_like(refs).index_add(0, to, torch.where(used, refs, 0))
    return table, refs, moves, count.to(torch.int32).reshape(1)


def _plain_fork(s):
    page = s["case"]["page"]
    table, length, refs = _plain_fork_pages(s["table"], s["length"], s["refs"], s["parent"], page)
    table, length, refs, moves = _plain_resize_pages(table, length, refs, s["new_length"], page)
    return table, length, refs, moves, _plain_copy_pages(s["cache"], moves)


def _plain_compact(s):
    table, refs, moves, count = _plain_compact_pages(s["table"], s["refs"])
    return table, refs, moves, count, _plain_copy_pages(s["cache"], moves)


def _plain_verify(s):
    # in 64 bits: whether a token stands is a comparison, and the residual a difference
    x, B, K = s["target"].double(), s["case"]["B"], s["case"]["K"]
    dev = x.device
    e = torch.exp(x - x.amax(-1, keepdim=True))
    p = e / e.sum(-1, keepdim=True)
    y = s["draft"].double()
    e = torch.exp(y - y.amax(-1, keepdim=True))
    q = e / e.sum(-1, keepdim=True)
    at = s["draft_tokens"].long()[..., None]
    px, qx = p[:, :K].gather(2, at)[..., 0], q.gather(2, at)[..., 0]
    drafted = torch.arange(K, device=dev)[None] < s["n_draft"][:, None]
    stands = (s["u"].double() * qx < px) & drafted
    n = torch.cumprod(stands.long(), 1).sum(1)
    b = torch.arange(B, device=dev)
    left = p[b, n]
    left = torch.where((n < s["n_draft"])[:, None], (left - q[b, n.clamp(max=K - 1)]).clamp(min=0.0), left)
    left = torch.where((left > 0).any(-1, keepdim=True), left, p[b, n])
    token = torch.argmax(torch.log(left) - torch.log(s["noise"].double()), -1)
    place = torch.arange(K + 1, device=dev)[None]
    tokens = torch.cat([s["draft_tokens"].long(), token[:, None]], 1)
    tokens = torch.where(place < n[:, None], tokens, torch.where(place == n[:, None], token[:, None], -1))
    logp = torch.log(p.gather(2, tokens.clamp(min=0)[..., None])[..., 0])
    return tokens.to(torch.int32), (n + 1).to(torch.int32), torch.where(tokens >= 0, logp, 0.0).float()


def _plain_distill(s):
    x, ids = s["logits"].float(), s["top_ids"].long()
    part = (s["weight"] != 0)[:, None]
    w = s["weight"][:, None]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    p = e / z
    lt = s["top_logp"].double()
    if s["case"]["tail"]:
        t = torch.exp(lt)
        rest = (1.0 - t.sum(-1, keepdim=True)).clamp(min=0.0).float()
    else:
        lt = lt - lt.amax(-1, keepdim=True)
        lt = lt - torch.log(torch.exp(lt).sum(-1, keepdim=True))
        t = torch.exp(lt)
    lt, t = lt.float(), t.float()
    lp = x.gather(1, ids) - m - torch.log(z)
    loss = (t * (lt - lp)).sum(-1, keepdim=True)
    grad = p
    if s["case"]["tail"]:
        outside = torch.ones_like(p).scatter_(1, ids, 0.0)
        p_rest = (p * outside).sum(-1, keepdim=True)
        some = (p_rest > 0) & (rest > 0)
        loss = loss + torch.where(some, rest * (torch.log(rest) - torch.log(p_rest)), 0.0)
        # one class outside: the listed ones' gradient is p - t, the others share p_rest - rest
        grad = p * (1.0 - outside * torch.where(some, rest / p_rest, 0.0))
    grad = grad.scatter_add(1, ids, -t)
    return torch.where(part, loss * w, 0.0)[:, 0], torch.where(part, grad * w, 0.0).to(s["logits"].dtype)


# ---------------------------------------------------------------- one pass

_PLAIN = {"attn": _plain_attn, "write": _plain_write, "fork": _plain_fork, "compact": _plain_compact, "verify": _plain_verify,
          "distill": _plain_distill}


def run(s):
    op = s["case"]["op"]
    if not own:
        return _PLAIN[op](s)
    import paper_2608_17641_amd as rl
    if op == "attn":
        return rl.rlcs_paged_attn(s["q"], s["k_cache"], s["v_cache"], s["table"], s["length"], s["q_start"], scale=s["scale"],
                                  max_chunk=s["case"]["T"])
    if op == "write":
        rl.rlcs_paged_write(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["length"], s["q_start"])
        return s["k_cache"], s["v_cache"]
    if op == "fork":
        table, length, refs = rl.rlcs_pages_fork(s["table"], s["length"], s["refs"], s["parent"], page=s["case"]["page"])
        table, length, refs, moves = rl.rlcs_pages_resize(table, length, refs, s["new_length"], page=s["case"]["page"])
        rl.rlcs_pages_copy(s["cache"], moves)
        return table, length, refs, moves, s["cache"]
    if op == "compact":
        table, refs, moves, count = rl.rlcs_pages_compact(s["table"], s["refs"])
        rl.rlcs_pages_copy(s["cache"], moves)
        return table, refs, moves, count, s["cache"]
    if op == "verify":
        return rl.rlcs_verify_draft(s["target"], s["draft"], s["draft_tokens"], s["u"], s["noise"], s["n_draft"])
    return rl.rlcs_distill_loss(s["logits"], s["top_ids"], s["top_logp"], s["weight"], tail=s["case"]["tail"])


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    op = case["op"]
    if op in ("attn", "write"):
        B, T, L, Hkv, D = (case[k] for k in ("B", "T", "L", "Hkv", "D"))
        # mean chunks and lengths, as prepare() makes them
        chunk = (1 + T) / 2 if T <= 8 else T - min(37 * (B - 1), T // 2) / 2
        if case.get("mixed"):
            chunk = (chunk + 1) / 2
        chunk = (T + (B - 1) * chunk) / B
        length = max((L + (B - 1) * 0.625 * L) / B, chunk)
        if op == "write":
            return {"bytes": 4 * es * B * chunk * Hkv * D, "flops": B * chunk}
        Hq = case["Hq"]
        return {"bytes": es * B * (2 * length * Hkv * D + 2 * chunk * Hq * D) + 4 * B * chunk * Hq,
                "flops": 4.0 * D * Hq * B * chunk * (length - chunk / 2)}
    if op == "fork":
        N, G = case["N"], case["G"]
        page_bytes = case["layers"] * case["page"] * case["Hkv"] * case["D"] * es
        width = (case["L"] + case["grow"]) // case["page"] + 1
        return {"bytes": 2 * N * G * page_bytes + 4 * (2 * N * (G + 1) * width + 2 * case["pages"]), "flops": N * G * width}
    if op == "compact":
        page_bytes = case["layers"] * case["page"] * case["Hkv"] * case["D"] * es
        moved = case["pages"] * case["used"] * (1 - case["used"])
        return {"bytes": 2 * moved * page_bytes + 8 * case["pages"] * (1 + case["used"]), "flops": case["pages"]}
    V = case["V"]
    if op == "verify":
        # every row of both once (which of them count is known after reading them), one row of noise a sequence
        return {"bytes": case["B"] * V * (es * (2 * case["K"] + 1) + 4), "flops": 4.0 * case["B"] * V * (2 * case["K"] + 1)}
    # a third of the rows is left out: their logits need not be read
    M, K = case["M"], case["K"]
    return {"bytes": es * M * V * 1.67 + 8 * M * K * 0.67 + 8 * M, "flops": 8.0 * M * V * 0.67}


# ---------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return {"attn": _exact_attn, "write": _exact_write, "fork": _exact_fork, "compact": _exact_compact, "verify": _exact_verify,
            "distill": _exact_distill}[case["op"]](s)


def _exact_attn(s):
    """Sequence by sequence and key head by key head, keys gathered page by page."""
    q = s["q"].double()
    Hq, D = q.shape[1:]
    page, Hkv = s["k_cache"].shape[1:3]
    r = Hq // Hkv
    start, length = s["q_start"].tolist(), s["length"].tolist()
    o, lse = torch.zeros_like(q), torch.full(q.shape[:2], -torch.inf, dtype=torch.float64, device=q.device)
    for b, n in enumerate(length):
        i, j = start[b], start[b + 1]
        at = s["table"][b, :(n + page - 1) // page].long()
        last = torch.arange(n - (j - i), n, device=q.device)  # of the keys that each token sees
        for h in range(Hkv):
            k = s["k_cache"][at, :, h].reshape(-1, D)[:n].double()
            v = s["v_cache"][at, :, h].reshape(-1, D)[:n].double()
            for x in range(h * r, (h + 1) * r):
                a = torch.mm(q[i:j, x], k.t().contiguous()) * s["scale"]
                a = torch.where(torch.arange(n, device=q.device)[None] <= last[:, None], a, -torch.inf)
                lse[i:j, x] = torch.logsumexp(a, -1)
                o[i:j, x] = torch.mm(torch.softmax(a, -1), v)
    return o, lse


def _exact_write(s):
    page, start = s["case"]["page"], s["q_start"].tolist()
    for b, n in enumerate(s["length"].tolist()):
        i, first, row = start[b], n - (start[b + 1] - start[b]), s["table"][b].tolist()
        at = first
        while at < n:  # page by page
            some = min(n - at, page - at % page)
            for to, of in (("k_cache", "k"), ("v_cache", "v")):
                s[to][row[at // page], at % page:at % page + some] = s[of][i + at - first:i + at - first + some]
            at += some
    return s["k_cache"], s["v_cache"]


def _like(x, t):
    return torch.tensor(x, dtype=t.dtype, device=t.device).reshape(-1, *t.shape[1:])


def _exact_fork(s):
    """One sequence after the other."""
    page, table, length, refs = s["case"]["page"], s["table"].tolist(), s["length"].tolist(), s["refs"].tolist()
    W = len(table[0])
    rows = [[p for p in row if p >= 0] for row in table]
    was = list(length)
    forked = []
    for b, par in enumerate(s["parent"].tolist()):
        forked.append(list(rows[par]))
        length[b] = was[par]
        if par != b:
            for p in rows[par]:
                refs[p] += 1
            for p in rows[b]:
                refs[p] -= 1
    rows = forked
    free = [p for p, n in enumerate(refs) if n == 0]
    shared, before = {p for p, n in enumerate(refs) if n > 1}, 0
    moves = []
    for b, n in enumerate(s["new_length"].tolist()):
        copy = n > length[b] and length[b] % page != 0 and rows[b][-1] in shared
        need = -(-n // page) - len(rows[b]) + copy
        before += need
        moves.append([-1, -1])
        if before > len(free) and need:
            continue
        own_pages = free[before - need:before]
        if copy:
            moves[b] = [rows[b][-1], own_pages[0]]
            refs[rows[b][-1]] -= 1
            rows[b][-1] = own_pages.pop(0)
            refs[rows[b][-1]] = 1
        for p in own_pages:
            refs[p] = 1
        rows[b] += own_pages
        length[b] = n
    for src, dst in moves:
        if src >= 0:
            s["cache"][:, dst] = s["cache"][:, src]
    table = [row + [-1] * (W - len(row)) for row in rows]
    return _like(table, s["table"]), _like(length, s["length"]), _like(refs, s["refs"]), _like(moves, torch.empty((1, 2), dtype=torch.int32, device="cuda")), s["cache"]


def _exact_compact(s):
    refs = s["refs"].tolist()
    count = sum(n > 0 for n in refs)
    holes = (p for p in range(count) if refs[p] == 0)
    moves, to = [], {}
    for p in range(count, len(refs)):
        if refs[p] > 0:
            to[p] = next(holes)
            moves.append([p, to[p]])
            refs[to[p]], refs[p] = refs[p], 0
    table = [[to.get(p, p) for p in row] for row in s["table"].tolist()]
    for i in range(0, len(moves), 64):
        src, dst = zip(*moves[i:i + 64])
        s["cache"][:, list(dst)] = s["cache"][:, list(src)]
    moves += [[-1, -1]] * (len(refs) // 2 - len(moves))
    return (_like(table, s["table"]), _like(refs, s["refs"]), torch.tensor(moves, dtype=torch.int32, device="cuda").reshape(-1, 2),
            torch.tensor([count], dtype=torch.int32, device="cuda"), s["cache"])


def _exact_verify(s):
    """Sequence by sequence, token by token, until one falls."""
    B, K = s["case"]["B"], s["case"]["K"]
    tokens = torch.full((B, K + 1), -1, dtype=torch.int32, device="cuda")
    count, logp = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros((B, K + 1), dtype=torch.float64, device="cuda")
    drafts, drawn, u = s["n_draft"].tolist(), s["draft_tokens"].tolist(), s["u"].double().tolist()
    for b in range(B):
        i = 0
        while True:
            lp = torch.log_softmax(s["target"][b, i].double(), -1)
            if i == drafts[b]:
                score = lp
                break
            lq, a = torch.log_softmax(s["draft"][b, i].double(), -1), drawn[b][i]
            if u[b][i] >= math.exp(float(lp[a] - lq[a])):
                score = torch.log((lp.exp() - lq.exp()).clamp(min=0.0))
                break
            tokens[b, i], logp[b, i] = a, lp[a]
            i += 1
        a = int(torch.argmax(score - torch.log(s["noise"][b].double())))
        tokens[b, i], logp[b, i], count[b] = a, lp[a], i + 1
    return tokens, count, logp


def _exact_distill(s):
    M, V, tail = s["case"]["M"], s["case"]["V"], s["case"]["tail"]
    loss, grad = torch.zeros(M, dtype=torch.float64, device="cuda"), torch.zeros((M, V), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // V)
    for i in range(0, M, step):
        ids, w = s["top_ids"][i:i + step].long(), s["weight"][i:i + step].double()
        ls = torch.log_softmax(s["logits"][i:i + step].double(), -1)
        lt = s["top_logp"][i:i + step].double()
        if not tail:
            lt = torch.log_softmax(lt, -1)
        full = torch.zeros_like(ls)
        full.scatter_(1, ids, lt.exp())
        value = (lt.exp() * (lt - ls.gather(1, ids))).sum(-1)
        if tail:
            other = ls.exp().scatter(1, ids, 0.0)
            mass, rest = other.sum(-1), 1.0 - lt.exp().sum(-1)
            some = (mass > 0) & (rest > 0)
            value += torch.where(some, rest * torch.log(rest / mass), 0.0)
            # the teacher's rest, dealt out as the student deals out its own
            full += other * torch.where(some, rest / mass, 0.0)[:, None]
        loss[i:i + step] = w * value
        grad[i:i + step] = w[:, None] * (ls.exp() - full)
    return loss, grad
