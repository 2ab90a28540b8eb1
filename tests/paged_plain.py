"""Plain 64-bit forms of the operators of speculative rollouts over a paged cache, on the CPU, written from
their formulas: the oracle of tests/test_gpu_paged.py, test_gpu_pages.py, test_gpu_verify.py and
test_gpu_distill.py."""
import math

import torch


# ---------------------------------------------------------------- a paged cache

def slots(table_row, length, pages, page):
    """(page, place) of every token of a sequence, None where its entry is no page."""
    out = []
    for t in range(length):
        p = table_row[t // page]
        out.append((p, t % page) if 0 <= p < pages else None)
    return out


def paged_attention(q, k_cache, v_cache, table, length, start, scale):
    """(o, lse), float64; rows of no sequence NaN. table, length, start as lists."""
    n, Hq, D = q.shape
    pages, page, Hkv = k_cache.shape[:3]
    r = Hq // Hkv
    o, lse = torch.full((n, Hq, D), math.nan, dtype=torch.float64), torch.full((n, Hq), math.nan, dtype=torch.float64)
    for b, row in enumerate(table):
        L = max(0, min(length[b], len(row) * page)) if pages else 0
        at = slots(row, L, pages, page)
        T = start[b + 1] - start[b]
        keys = [i for i, s in enumerate(at) if s is not None]
        k = torch.stack([k_cache[at[i]] for i in keys]) if keys else torch.zeros((0, Hkv, D), dtype=torch.float64)
        v = torch.stack([v_cache[at[i]] for i in keys]) if keys else torch.zeros((0, Hkv, D), dtype=torch.float64)
        seen = torch.tensor(keys, dtype=torch.int64)
        for i in range(T):
            t, pos = start[b] + i, L - T + i
            m = int((seen <= pos).sum())
            if m == 0:
                o[t], lse[t] = 0.0, -math.inf
                continue
            s = torch.matmul(k[:m].permute(1, 0, 2), q[t].reshape(Hkv, r, D).transpose(1, 2)) * scale  # [Hkv, m, r]
            z = torch.logsumexp(s, 1)
            lse[t] = z.reshape(Hq)
            o[t] = torch.matmul(torch.exp(s - z[:, None]).transpose(1, 2), v[:m].permute(1, 0, 2)).reshape(Hq, D)
    return o, lse


def paged_write(k, v, k_cache, v_cache, table, length, start):
    pages, page = k_cache.shape[:2]
    for b, row in enumerate(table):
        L = max(0, min(length[b], len(row) * page))
        T = start[b + 1] - start[b]
        for i in range(T):
            pos = L - T + i
            if pos < 0 or not 0 <= row[pos // page] < pages:
                continue
            k_cache[row[pos // page], pos % page] = k[start[b] + i]
            v_cache[row[pos // page], pos % page] = v[start[b] + i]


# ---------------------------------------------------------------- pages

class Cache:
    """Tables as lists of lists, one entry after the other."""

    def __init__(self, table, length, refs, page):
        self.W, self.page, self.pages = len(table[0]) if table else 0, page, len(refs)
        self.length = [max(0, min(n, self.W * page)) for n in length]
        self.refs = list(refs)
        self.rows = [row[:self.held(n)] for row, n in zip(table, self.length)]

    def held(self, n):
        return (n + self.page - 1) // self.page

    def count(self, p, by):
        if 0 <= p < self.pages:
            self.refs[p] += by

    def table(self):
        return [row + [-1] * (self.W - len(row)) for row in self.rows]

    def fork(self, parent):
        rows, length = [list(r) for r in self.rows], list(self.length)
        for b, p in enumerate(parent):
            if not 0 <= p < len(rows) or p == b:
                continue
            for x in rows[p]:
                self.count(x, 1)
            for x in rows[b]:
                self.count(x, -1)
            self.rows[b], self.length[b] = list(rows[p]), length[p]

    def resize(self, new):
        most = self.W * self.page
        new = [old if n < 0 or n > most else n for n, old in zip(new, self.length)]
        for b, n in enumerate(new):
            if n < self.length[b]:
                for x in self.rows[b][self.held(n):]:
                    self.count(x, -1)
                self.rows[b] = self.rows[b][:self.held(n)]
                self.length[b] = n
        free = [p for p in range(self.pages) if self.refs[p] <= 0]
        shared = {p for p in range(self.pages) if self.refs[p] > 1}
        moves, used = [], 0
        for b, n in enumerate(new):
            moves.append([-1, -1])
            if n <= self.length[b]:
                continue
            copy = self.length[b] % self.page != 0 and self.rows[b][-1] in shared
            need = self.held(n) - len(self.rows[b]) + copy
            used += need
            if need and used > len(free):
                continue
            fresh = free[used - need:used]
            if copy:
                moves[b] = [self.rows[b][-1], fresh[0]]
                self.refs[self.rows[b][-1]] -= 1
                self.rows[b] = self.rows[b][:-1]
            for p in fresh:
                self.refs[p] = 1
            self.rows[b] = self.rows[b] + fresh
            self.length[b] = n
        return moves

    def compact(self, table):
        """(table, moves, count): all entries of the table, whatever the lengths."""
        used = [p for p in range(self.pages) if self.refs[p] > 0]
        U = len(used)
        holes = [p for p in range(U) if self.refs[p] <= 0]
        to = dict(zip([p for p in used if p >= U], holes))
        refs = [0] * self.pages
        for p in used:
            refs[to.get(p, p)] = self.refs[p]
        out = [[to.get(p, p) if 0 <= p < self.pages and self.refs[p] > 0 else -1 for p in row] for row in table]
        self.refs = refs
        moves = [[a, b] for a, b in to.items()]
        return out, moves + [[-1, -1]] * (self.pages // 2 - len(moves)), U


# ---------------------------------------------------------------- drafted tokens

def softmax_row(x, T):
    """Probabilities of a float64 row as the check counts them, None where all are masked."""
    x = torch.where(torch.isnan(x), -math.inf, x)
    if not bool((x > -math.inf).any()):
        return None
    if T <= 0:
        p = torch.zeros_like(x)
        p[int(torch.argmax(x))] = 1.0
        return p
    y = (x - x.max()) / T if T < math.inf else torch.where(x > -math.inf, 0.0, -math.inf)
    return torch.softmax(y, 0)


def verify(target, draft, drawn, u, noise, n_draft, T, Td):
    """One sequence: (tokens, logp, margin), target [K + 1, V] and draft [K, V] (or None) float64. margin: how far the nearest
    decision is from the other way, relative for a comparison, in the score for a race."""
    K, V = target.shape[0] - 1, target.shape[1]
    tokens, logp, margin, i = [], [], math.inf, 0
    while True:
        p = softmax_row(target[i], T)
        fell = False
        if i < n_draft:
            x = int(drawn[i])
            if draft is None:
                q = torch.zeros(V, dtype=torch.float64)
                if 0 <= x < V:
                    q[x] = 1.0
            else:
                q = softmax_row(draft[i], Td)
                q = torch.zeros(V, dtype=torch.float64) if q is None else q
            px = float(p[x]) if p is not None and 0 <= x < V else 0.0
            uq = float(u[i]) * (float(q[x]) if 0 <= x < V else 1.0)
            if px > 0:
                margin = min(margin, abs(uq - px) / max(uq, px))
            if 0 <= x < V and uq < px:
                tokens.append(x)
                logp.append(math.log(px))
                i += 1
                continue
            fell = True
        if p is None:
            return tokens + [-1], logp + [-math.inf], margin
        left = p
        if fell:
            rest = (p - q).clamp(min=0.0)
            rest[rest < 1e-7 * p] = 0.0  # (what rounding alone may leave)
            left = rest if bool((rest > 0).any()) else p
        score = torch.log(left) - torch.log(noise)
        best = int(torch.argmax(score))
        others = torch.cat([score[:best], score[best + 1:]])
        if T > 0 and others.numel() and bool((others > -math.inf).any()):
            margin = min(margin, float(score[best] - others.max()))
        return tokens + [best], logp + [math.log(float(p[best])) if float(p[best]) > 0 else -math.inf], margin


# ---------------------------------------------------------------- distillation

def distill(x, ids, top, weight, T, tail):
    """(loss, gradient) of float64 rows x [M, V]."""
    M, V = x.shape
    loss, grad = torch.zeros(M, dtype=torch.float64), torch.zeros((M, V), dtype=torch.float64)
    for m in range(M):
        w = float(weight[m])
        if w == 0.0:
            continue
        ok = (ids[m] >= 0) & (ids[m] < V) & (top[m] != -math.inf)
        at, lt = ids[m][ok].long(), top[m][ok].double()
        if not tail:
            if at.numel() == 0:
                continue
            lt = lt - lt.max()
            lt = lt - torch.logsumexp(lt, 0)
        t = torch.exp(lt)
        y = x[m] / T
        if bool((y > -math.inf).any()):
            lp = y - y.max()
            lp = lp - torch.logsumexp(lp, 0)
        else:
            lp = torch.full((V,), -math.inf, dtype=torch.float64)
        p = torch.exp(lp)
        total = float((t * (lt - lp[at])).sum())
        share = torch.zeros(V, dtype=torch.float64).index_add(0, at, t)
        g = p - share
        if tail:
            listed = torch.zeros(V, dtype=torch.bool)
            listed[ids[m][(ids[m] >= 0) & (ids[m] < V)].long()] = True
            rest, p_rest = max(0.0, 1.0 - float(t.sum())), float(p[~listed].sum())
            if rest > 0 and p_rest > 0:
                total += rest * (math.log(rest) - math.log(p_rest))
                g = torch.where(listed, g, p * (1.0 - rest / p_rest))
        loss[m] = w * total
        grad[m] = w / T * g
    return loss, grad
