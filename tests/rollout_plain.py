"""Plain 64-bit forms of the operators around a group rollout, on the CPU, written from their
formulas: the oracle of tests/test_gpu_attn.py, test_gpu_sample.py and test_gpu_policy.py."""
import math

import torch


def policy(logits, tokens, logp_old, adv, weight, clip_low, clip_high, ent_coef, temperature):
    """(loss, dlogits, logp, ent), float64. logits [M, V] already float64."""
    M, V = logits.shape
    y = logits / temperature
    loss, logp, ent = (torch.zeros(M, dtype=torch.float64) for _ in range(3))
    grad = torch.zeros((M, V), dtype=torch.float64)
    for i in range(M):
        a, w = int(tokens[i]), float(weight[i])
        if not 0 <= a < V or w == 0.0:
            continue
        if not bool((y[i] > -math.inf).any()):
            logp[i], ent[i], p, lp = -math.inf, 0.0, torch.zeros(V, dtype=torch.float64), None
        else:
            lp = y[i] - y[i].max()  # (first: 64 bits do not hold both 1e38 and its rest)
            lp = lp - torch.logsumexp(lp, 0)
            p = torch.exp(lp)
            logp[i] = lp[a]
            ent[i] = -torch.where(p > 0, p * lp, 0.0).sum()
        rho = math.exp(min(float(logp[i] - logp_old[i]), 700.0))
        A = float(adv[i])
        free, held = rho * A, min(max(rho, 1 - clip_low), 1 + clip_high) * A
        loss[i] = w * (-min(free, held) - ent_coef * float(ent[i]))
        g = -w * A * rho if free <= held else 0.0
        row = -g * p
        if lp is not None:
            row = row + w * ent_coef * torch.where(p > 0, p * (lp + ent[i]), 0.0)
        row[a] += g
        grad[i] = row / temperature
    return loss, grad, logp, ent


def sample_row(x, noise, T, k, p, min_p):
    """(token, logp, margin of the race): x [V] float64."""
    V = x.numel()
    x = torch.where(torch.isnan(x), -math.inf, x)
    if not bool((x > -math.inf).any()):
        return -1, -math.inf, math.inf
    if not T > 0:
        return int(torch.argmax(x)), 0.0, math.inf
    y = (x - x.max()) / T
    order = torch.sort(x, descending=True, stable=True).indices
    order = order[x[order] > -math.inf]
    if 0 < k < V:
        order = order[:k]
    if p < 1:
        w = torch.exp(y[order])
        before = torch.cumsum(w, 0) - w
        kept = before < p * w.sum()
        kept[0] = True
        order = order[kept]
    if min_p > 0:
        kept = torch.exp(y[order] - y[order[0]]) >= min(min_p, 1.0)
        kept[0] = True
        order = order[kept]
    order = torch.sort(order).values
    yk = y[order]
    score = yk - torch.log(noise[order]) if noise is not None else yk
    best = int(torch.argmax(score))
    rest = torch.cat([score[:best], score[best + 1:]])
    margin = float(score[best] - rest.max()) if rest.numel() and noise is not None else math.inf
    return int(order[best]), float(yk[best] - torch.logsumexp(yk, 0)), margin


def attention(q, kp, vp, ks, vs, plen, slen, scale):
    """(o, lse), float64, from float64 inputs; lengths as nested lists."""
    N, G, Hq, D = q.shape
    Hkv = kp.shape[2]
    r = Hq // Hkv
    o, lse = torch.zeros_like(q), torch.full((N, G, Hq), -math.inf, dtype=torch.float64)
    for n in range(N):
        for g in range(G):
            k, v = kp[n, :plen[n]], vp[n, :plen[n]]
            if ks is not None:
                k, v = torch.cat([k, ks[n, g, :slen[n][g]]]), torch.cat([v, vs[n, g, :slen[n][g]]])
            if k.shape[0] == 0:
                continue
            for h in range(Hq):
                s = (k[:, h // r] * q[n, g, h]).sum(-1) * scale
                lse[n, g, h] = torch.logsumexp(s, 0)
                o[n, g, h] = (torch.exp(s - lse[n, g, h])[:, None] * v[:, h // r]).sum(0)
    return o, lse
