"""What the operators around a group rollout are measured on: attention of a group of completions
over their shared prompt, sampling of the next token, and the policy loss on the sampled tokens.

With ``own`` false, ``run`` computes them in elementary torch operations in float32; with ``own``
true it makes the library's calls. Sizes are those of the benchmark's rollouts (8 x 128, 4096 and
64 x 4096 tokens, an 18-action space) or plain odd ones.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CLIP_LOW, CLIP_HIGH = 0.2, 0.28


def listed():
    return [
        # one decode step of a small group on a small model: latency only
        dict(name="attn_1x8_257+33_f32", op="attn", N=1, G=8, Hq=8, Hkv=8, D=64, P=257, S=33, dtype="f32", ragged=True),
        # a decode step of 16 completions of a 2k-token prompt, grouped heads
        dict(name="attn_1x16_2048+512_bf16", op="attn", N=1, G=16, Hq=32, Hkv=8, D=128, P=2048, S=512, dtype="bf16", ragged=True),
        # eight prompts of unequal length, 16 completions each
        dict(name="attn_8x16_4001+1000_bf16", op="attn", N=8, G=16, Hq=32, Hkv=8, D=128, P=4001, S=1000, dtype="bf16", ragged=True),
        # 64 completions of one long tool transcript, the suffix as long as the benchmark's token rows
        dict(name="attn_1x64_32768+4096_bf16", op="attn", N=1, G=64, Hq=32, Hkv=8, D=128, P=32768, S=4096, dtype="bf16", ragged=True),
        # actions of the benchmark's 4096 environments over 18 discrete actions, no filter
        dict(name="sample_4096x18_f32", op="sample", M=4096, V=18, dtype="f32", filters="none"),
        # a serving step of 64 rows, every filter on, each row with its own settings
        dict(name="sample_64x32000_bf16", op="sample", M=64, V=32000, dtype="bf16", filters="rows"),
        # a large rollout batch with nucleus sampling alone
        dict(name="sample_256x128000_f32", op="sample", M=256, V=128000, dtype="f32", filters="p"),
        # the same from the whole distribution, as on-policy rollouts are drawn
        dict(name="sample_512x128000_bf16", op="sample", M=512, V=128000, dtype="bf16", filters="none"),
        # the policy update of 4096 x 32 environment steps over 18 actions
        dict(name="policy_131072x18_f32", op="policy", M=131072, V=18, dtype="f32", grad=True),
        # log-probabilities and entropies alone (the reference policy, an off-policy ratio), an odd vocabulary
        dict(name="logp_2048x50001_f32", op="policy", M=2048, V=50001, dtype="f32", grad=False),
        # one micro-batch of token rows, loss and gradient, a third of the tokens masked
        dict(name="policy_4096x32000_bf16", op="policy", M=4096, V=32000, dtype="bf16", grad=True),
        # a large vocabulary
        dict(name="policy_8192x128000_bf16", op="policy", M=8192, V=128000, dtype="bf16", grad=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attn", "sample", "policy"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "attn":
        Hkv, D = rng.choice([1, 2, 4, 8]), rng.choice([64, 128])
        N, G = _log_int(rng, 1, 8), _log_int(rng, 1, 64)
        P, S = _log_int(rng, 16, 32768), _log_int(rng, 1, 4096)
        # no more bytes of keys than the largest listed case reads, nor more products
        most = 64 * 2048 * 8 * 128 // (2 * N * Hkv * D * (2 if dtype == "f32" else 1))
        S = max(1, min(S, most // G))
        P = max(1, min(P, most, 64 * 32 * 32768 * 128 // (N * G * 8 * Hkv * D)))
        return dict(op=op, N=N, G=G, Hq=Hkv * rng.choice([1, 2, 4, 7, 8]), Hkv=Hkv, D=D, P=P, S=S, dtype=dtype,
                    ragged=rng.random() < 0.7)
    V = _log_int(rng, 4, 128000)
    if op == "sample":
        return dict(op=op, M=max(1, min(8192, _log_int(rng, 1, max(2, (1 << 25) // V)))), V=V, dtype=dtype,
                    filters=rng.choice(["none", "k", "p", "rows", "rows"]))
    return dict(op=op, M=max(1, min(1 << 17, _log_int(rng, 16, max(17, (1 << 28) // V)))), V=V, dtype=dtype,
                grad=rng.random() < 0.7)


# ---------------------------------------------------------------- inputs

def _exponential(g, shape):
    return torch.empty(shape, device="cuda").exponential_(generator=g)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]

    def normal(shape, scale=1.0):
        return torch.randn(shape, device="cuda", generator=g, dtype=torch.float32).mul_(scale).to(dt)

    s = dict(case=case)
    if case["op"] == "attn":
        N, G, Hq, Hkv, D, P, S = (case[k] for k in ("N", "G", "Hq", "Hkv", "D", "P", "S"))
        s.update(q=normal((N, G, Hq, D)), kp=normal((N, P, Hkv, D)), vp=normal((N, P, Hkv, D)),
                 ks=normal((N, G, S, Hkv, D)), vs=normal((N, G, S, Hkv, D)), scale=1.0 / math.sqrt(D),
                 prefix_len=None, suffix_len=None)
        if case["ragged"]:
            # prompts of the longest length or up to a quarter shorter; completions at any length
            s["prefix_len"] = (P - (torch.rand((N,), device="cuda", generator=g) * (P // 4 + 1)).floor()).to(torch.int32)
            s["prefix_len"][0] = P
            s["suffix_len"] = (torch.rand((N, G), device="cuda", generator=g) * (S + 1)).floor().clamp_(max=S).to(torch.int32)
            s["suffix_len"][0, 0] = S
        return s
    M, V = case["M"], case["V"]
    s["logits"] = normal((M, V), 2.5)
    if case["op"] == "sample":
        f = case["filters"]
        s["noise"] = _exponential(g, (M, V))
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = 1.0, 0, 1.0, 0.0
        if f == "k":
            s["temperature"], s["top_k"] = 0.7, min(50, V)
        elif f == "p":
            s["temperature"], s["top_p"] = 0.8, 0.95
        elif f == "rows":
            # each request's own: temperatures around 0.8, top-k of 20 to 100 or off, top-p of 0.8
            # to 1, min-p of 0 to 0.1
            u = torch.rand((4, M), device="cuda", generator=g)
            s["temperature"] = 0.4 + 0.8 * u[0]
            s["top_k"] = torch.where(u[1] < 0.25, 0, 20 + torch.floor(80 * u[1])).to(torch.int32)
            s["top_p"] = 0.8 + 0.2 * u[2]
            s["min_p"] = torch.clamp(0.15 * u[3] - 0.05, min=0.0)
        return s
    # tokens drawn from the policy, behaviour log-probabilities near its own, whitened advantages,
    # weights of a mean over the tokens that take part
    lead = torch.empty((M,), dtype=torch.int64, device="cuda")
    lp = torch.empty((M,), device="cuda")
    step = max(1, (1 << 28) // V)
    for i in range(0, M, step):
        x = s["logits"][i:i + step].float()
        lead[i:i + step] = torch.argmax(x - torch.log(_exponential(g, x.shape)), dim=-1)
        lp[i:i + step] = x.gather(1, lead[i:i + step, None])[:, 0] - torch.logsumexp(x, -1)
    s["tokens"] = lead.to(torch.int32)
    s["logp_old"] = lp + 0.1 * torch.randn((M,), device="cuda", generator=g)
    s["adv"] = torch.randn((M,), device="cuda", generator=g)
    keep = (torch.rand((M,), device="cuda", generator=g) < 0.67).float()
    s["weight"] = keep / keep.sum().clamp_(min=1.0)
    return s


# ---------------------------------------------------------------- the plain forms

def _plain_attn(s):
    q, kp, vp, ks, vs = (s[k].float() for k in ("q", "kp", "vp", "ks", "vs"))
    N, G, Hq, D = q.shape
    P, Hkv, S = kp.shape[1], kp.shape[2], ks.shape[2]
    r = Hq // Hkv
    at = lambda n, most: torch.arange(most, device=q.device) < n[..., None]  # noqa: E731
    seen_p = at(s["prefix_len"], P) if s["prefix_len"] is not None else torch.ones((N, P), dtype=torch.bool, device=q.device)
    seen_s = at(s["suffix_len"], S) if s["suffix_len"] is not None else torch.ones((N, G, S), dtype=torch.bool, device=q.device)
    # heads before rows: the prefix is one product for all rows of the group
    qp = q.reshape(N, G, Hkv, r, D).permute(0, 2, 1, 3, 4).reshape(N, Hkv, G * r, D).contiguous()
    sp = torch.matmul(qp, kp.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    sp = torch.where(seen_p[:, None, None, :], sp, -torch.inf).reshape(N, Hkv, G, r, P).permute(0, 2, 1, 3, 4)
    ss = torch.matmul(q.reshape(N, G, Hkv, r, D), ks.permute(0, 1, 3, 4, 2).contiguous()) * s["scale"]
    ss = torch.where(seen_s[:, :, None, None, :], ss, -torch.inf)
    m = torch.maximum(sp.amax(-1), ss.amax(-1))[..., None]
    m = torch.where(torch.isinf(m), 0.0, m)
    ep, es = torch.exp(sp - m), torch.exp(ss - m)
    z = ep.sum(-1) + es.sum(-1)
    vp = torch.where(seen_p[:, :, None, None], vp, 0.0)
    vs = torch.where(seen_s[..., None, None], vs, 0.0)
    op = torch.matmul(ep.permute(0, 2, 1, 3, 4).reshape(N, Hkv, G * r, P), vp.permute(0, 2, 1, 3).contiguous())
    os_ = torch.matmul(es, vs.permute(0, 1, 3, 2, 4).contiguous())
    o = op.reshape(N, Hkv, G, r, D).permute(0, 2, 1, 3, 4) + os_
    o = torch.where(z[..., None] > 0, o / z[..., None], 0.0).reshape(N, G, Hq, D)
    lse = (m[..., 0] + torch.log(z)).reshape(N, G, Hq)
    return o.to(s["q"].dtype), lse


def _plain_sample(s):
    x, M, V = s["logits"].float(), s["case"]["M"], s["case"]["V"]
    row = lambda v, dt: v.to(dt) if torch.is_tensor(v) else torch.full((M,), v, dtype=dt, device=x.device)  # noqa: E731
    y = x / row(s["temperature"], torch.float32)[:, None]
    keep = None
    if s["case"]["filters"] != "none":
        k, p, mp = row(s["top_k"], torch.int64), row(s["top_p"], torch.float32), row(s["min_p"], torch.float32)
        k = torch.where(k > 0, k, V)
        ys, order = torch.sort(y, dim=-1, descending=True, stable=True)
        w = torch.exp(ys - ys[:, :1])
        kept = torch.arange(V, device=x.device)[None] < k[:, None]
        w = torch.where(kept, w, 0.0)
        before = torch.cumsum(w, -1) - w
        kept = kept & ((before < p[:, None] * w.sum(-1, keepdim=True)) | (p[:, None] >= 1.0)) & (w >= mp[:, None])
        keep = torch.zeros((M, V), dtype=torch.bool, device=x.device).scatter_(1, order, kept)
        y = torch.where(keep, y, -torch.inf)
    tokens = torch.argmax(y - torch.log(s["noise"]), dim=-1)
    m = y.amax(-1, keepdim=True)
    lse = m[:, 0] + torch.log(torch.exp(y - m).sum(-1))
    return tokens.to(torch.int32), y.gather(1, tokens[:, None])[:, 0] - lse


def _plain_policy(s):
    x = s["logits"].float()
    a = s["tokens"].long()[:, None]
    m = x.amax(-1, keepdim=True)
    e = torch.exp(x - m)
    z = e.sum(-1, keepdim=True)
    p = e / z
    lp_all = x - m - torch.log(z)
    logp = lp_all.gather(1, a)[:, 0]
    ent = -(p * lp_all).sum(-1)
    if not s["case"]["grad"]:
        return logp, ent
    rho = torch.exp(logp - s["logp_old"])
    free, held = rho * s["adv"], rho.clamp(1.0 - CLIP_LOW, 1.0 + CLIP_HIGH) * s["adv"]
    w = s["weight"]
    loss = w * (-torch.minimum(free, held) - 0.01 * ent)
    dlogp = torch.where(free <= held, -w * free, 0.0)
    grad = p * ((w * 0.01)[:, None] * (lp_all + ent[:, None]) - dlogp[:, None])
    grad.scatter_add_(1, a, dlogp[:, None])
    part = w != 0  # tokens of no weight are left out
    return loss, grad.to(s["logits"].dtype), torch.where(part, logp, 0.0), torch.where(part, ent, 0.0)


# ---------------------------------------------------------------- one pass

def run(s):
    op = s["case"]["op"]
    if not own:
        return {"attn": _plain_attn, "sample": _plain_sample, "policy": _plain_policy}[op](s)
    import paper_2608_17641_amd as rl
    if op == "attn":
        return rl.rlcs_shared_prefix_attn(s["q"], s["kp"], s["vp"], s["ks"], s["vs"], s["prefix_len"], s["suffix_len"],
                                          scale=s["scale"])
    if op == "sample":
        return rl.rlcs_sample(s["logits"], s["noise"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                              min_p=s["min_p"])
    if not s["case"]["grad"]:
        return rl.rlcs_token_logp(s["logits"], s["tokens"])
    return rl.rlcs_policy_loss(s["logits"], s["tokens"], s["logp_old"], s["adv"], s["weight"], clip_low=CLIP_LOW,
                               clip_high=CLIP_HIGH, ent_coef=0.01)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "attn":
        N, G, Hq, Hkv, D, P, S = (case[k] for k in ("N", "G", "Hq", "Hkv", "D", "P", "S"))
        # mean lengths of the ragged ones
        p, c = (P * 0.875 + P * 0.125 / N, S * 0.5 + S * 0.5 / (N * G)) if case["ragged"] else (P, S)
        return {"bytes": 2 * es * N * Hkv * D * (p + G * c) + 2 * es * N * G * Hq * D + 4 * N * G * Hq,
                "flops": 4.0 * D * N * G * Hq * (p + c)}
    M, V = case["M"], case["V"]
    if case["op"] == "sample":
        # the noise of the kept tokens only: a few dozen of a filtered row
        noise = 4 * M * V if case["filters"] == "none" else 0
        return {"bytes": es * M * V + noise + 8 * M, "flops": 4.0 * M * V}
    if not case["grad"]:
        return {"bytes": es * M * V + 12 * M, "flops": 5.0 * M * V}
    # a third of the tokens is left out: their logits need not be read
    return {"bytes": es * M * V * 1.67 + 28 * M, "flops": 10.0 * M * V * 0.67}


# ---------------------------------------------------------------- the same in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attn":
        return _exact_attn(s)
    if case["op"] == "sample":
        return _exact_sample(s)
    return _exact_policy(s)


def _exact_attn(s):
    """Group by group and head by head, keys cut to their lengths."""
    q = s["q"].double()
    N, G, Hq, D = q.shape
    P, Hkv, S = s["kp"].shape[1], s["kp"].shape[2], s["ks"].shape[2]
    r = Hq // Hkv
    o, lse = torch.zeros_like(q), torch.empty((N, G, Hq), dtype=torch.float64, device=q.device)
    plen = [P] * N if s["prefix_len"] is None else s["prefix_len"].tolist()
    slen = [[S] * G] * N if s["suffix_len"] is None else s["suffix_len"].tolist()
    for n in range(N):
        kp, vp = s["kp"][n, :plen[n]].double().transpose(0, 1).contiguous(), s["vp"][n, :plen[n]].double().transpose(0, 1).contiguous()
        for i in range(G):
            c = slen[n][i]
            k = torch.cat([kp, s["ks"][n, i, :c].double().transpose(0, 1)], 1)
            v = torch.cat([vp, s["vs"][n, i, :c].double().transpose(0, 1)], 1)
            if k.shape[1] == 0:
                lse[n, i] = -torch.inf
                continue
            a = torch.bmm(q[n, i].reshape(Hkv, r, D), k.transpose(1, 2).contiguous()) * s["scale"]
            z = torch.logsumexp(a, -1)
            o[n, i] = torch.bmm(torch.exp(a - z[..., None]), v).reshape(Hq, D)
            lse[n, i] = z.reshape(Hq)
    return o, lse


def _exact_sample(s):
    M, V = s["case"]["M"], s["case"]["V"]

    def each(v, i, n):
        return v[i:i + n].double() if torch.is_tensor(v) else torch.full((n,), float(torch.tensor(v, dtype=torch.float32)), dtype=torch.float64, device="cuda")

    tokens, logp = torch.empty((M,), dtype=torch.int32, device="cuda"), torch.empty((M,), dtype=torch.float64, device="cuda")
    step = max(1, (1 << 26) // V)
    for i in range(0, M, step):
        x = s["logits"][i:i + step].double()
        n = x.shape[0]
        x = x / each(s["temperature"], i, n)[:, None]
        if s["case"]["filters"] != "none":
            x0, at = torch.sort(x, dim=-1, descending=True, stable=True)
            pr = torch.softmax(x0, -1)
            k = each(s["top_k"], i, n)
            alive = (torch.arange(V, device="cuda") < k[:, None]) | (k[:, None] <= 0)
            pr = pr * alive
            pr = pr / pr.sum(-1, keepdim=True)
            top_p = each(s["top_p"], i, n)[:, None]
            alive &= (torch.cat([torch.zeros_like(pr[:, :1]), torch.cumsum(pr, -1)[:, :-1]], -1) < top_p) | (top_p >= 1.0)
            alive &= pr >= each(s["min_p"], i, n)[:, None] * pr[:, :1]
            dead = torch.empty_like(alive)
            dead.scatter_(1, at, ~alive)
            x = x.masked_fill(dead, -torch.inf)
        t = torch.argmax(x - torch.log(s["noise"][i:i + step].double()), -1)
        tokens[i:i + step] = t.to(torch.int32)
        logp[i:i + step] = torch.log_softmax(x, -1).gather(1, t[:, None])[:, 0]
    return tokens, logp


def _exact_policy(s):
    M, V, grad = s["case"]["M"], s["case"]["V"], s["case"]["grad"]
    logp, ent, loss = (torch.empty((M,), dtype=torch.float64, device="cuda") for _ in range(3))
    dx = torch.empty((M, V), dtype=torch.float64, device="cuda") if grad else None
    lo, hi, c = (float(torch.tensor(v, dtype=torch.float32)) for v in (CLIP_LOW, CLIP_HIGH, 0.01))
    step = max(1, (1 << 26) // V)
    for i in range(0, M, step):
        x = s["logits"][i:i + step].double()
        a = s["tokens"][i:i + step].long()
        rows = torch.arange(x.shape[0], device="cuda")
        lsm = torch.log_softmax(x, -1)
        h = -(lsm.exp() * lsm).sum(-1)
        logp[i:i + step], ent[i:i + step] = lsm[rows, a], h
        if grad:
            A, w = s["adv"][i:i + step].double(), s["weight"][i:i + step].double()
            ratio = torch.exp(lsm[rows, a] - s["logp_old"][i:i + step].double())
            edge = torch.where(A >= 0, 1.0 + hi, 1.0 - lo)
            clipped = torch.where(A >= 0, ratio > edge, ratio < edge)
            loss[i:i + step] = -w * A * torch.where(clipped, edge, ratio) - w * c * h
            d = torch.where(clipped, 0.0, -w * A * ratio)
            g = lsm.exp() * (w * c)[:, None] * (lsm + h[:, None]) - lsm.exp() * d[:, None]
            g[rows, a] += d
            dx[i:i + step] = g
            logp[i:i + step] *= w != 0
            ent[i:i + step] *= w != 0
    return (loss, dx, logp, ent) if grad else (logp, ent)
