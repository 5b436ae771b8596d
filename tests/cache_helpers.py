"""Plain restatements of the paged cache for the tests: the bookkeeping one page at
a time on the host, norms, rotation and attention in float64."""
import math

import torch


class CacheModel:
    """Table, lengths and reference counts as the calls' rules give them."""

    def __init__(self, n_pages, max_seqs, max_pages, page):
        self.page, self.max_pages = page, max_pages
        self.own = [[] for _ in range(max_seqs)]
        self.len, self.base, self.ref = [0] * max_seqs, [0] * max_seqs, [0] * n_pages

    def step(self, seq, q):
        """Pages to copy as (from, to), or None when the step does not fit."""
        before = list(self.ref)
        free = [p for p, r in enumerate(before) if r == 0]
        plan, at = [], 0
        for s, m in zip(seq, q):
            cow = bool(m and self.len[s] % self.page and before[self.own[s][-1]] > 1)
            need = -(-(self.len[s] + m) // self.page)
            if need > self.max_pages:
                return None
            take = need - len(self.own[s]) + cow
            plan.append((cow, free[at:at + take]))
            at += take
        if at > len(free):
            return None
        copies = []
        for s, m, (cow, new) in zip(seq, q, plan):
            if cow:
                copies.append((self.own[s][-1], new[0]))
                self.ref[self.own[s][-1]] -= 1
                self.own[s].pop()
            self.own[s] += new
            for p in new:
                self.ref[p] = 1
            self.base[s], self.len[s] = self.len[s], self.len[s] + m
        return copies

    def fork(self, src, dst):
        for s, d in zip(src, dst):
            for p in self.own[d]:
                self.ref[p] -= 1
        for s, d in zip(src, dst):
            self.own[d], self.len[d], self.base[d] = list(self.own[s]), self.len[s], self.len[s]
            for p in self.own[d]:
                self.ref[p] += 1

    def truncate(self, seq, to):
        for s, n in zip(seq, to):
            n = min(n, self.len[s])
            while len(self.own[s]) > -(-n // self.page):
                self.ref[self.own[s].pop()] -= 1
            self.len[s], self.base[s] = n, min(self.base[s], n)

    def row(self, s, p):
        return self.own[s][p // self.page], p % self.page

    def accept(self, seq, n_acc, path):
        """Moved rows as (page, place) -> (page, place), or None for a sequence left alone."""
        moves = []
        for s, n, p in zip(seq, n_acc, path):
            drafts = self.len[s] - self.base[s]
            ok = 0 <= n <= min(drafts, 64, len(p))
            ok = ok and all(0 <= x < drafts for x in p[:n]) and all(a < b for a, b in zip(p, p[1:n]))
            ok = ok and all(self.ref[self.row(s, self.base[s] + e)[0]] == 1 for e in range(n))
            if not ok:
                moves.append(None)
                continue
            moves.append([(self.row(s, self.base[s] + p[e]), self.row(s, self.base[s] + e)) for e in range(n)])
            to = self.base[s] + n
            self.truncate([s], [to])
            self.base[s] = to
        return moves

    def compact(self):
        live = sum(r > 0 for r in self.ref)
        to = dict(zip([p for p in range(live, len(self.ref)) if self.ref[p] > 0],
                      [p for p in range(live) if self.ref[p] == 0]))
        for a, b in to.items():
            self.ref[b], self.ref[a] = self.ref[a], 0
        self.own = [[to.get(p, p) for p in r] for r in self.own]
        return to

    def table(self):
        return torch.tensor([r + [-1] * (self.max_pages - len(r)) for r in self.own], dtype=torch.int32)


def rows_of(pool, model, s, n):
    """Positions 0..n of sequence s in one layer's pool: [kv_heads][n][head_dim]."""
    ids = torch.tensor(model.own[s][:-(-n // model.page)], dtype=torch.long, device=pool.device)
    return pool[ids].transpose(0, 1).reshape(pool.shape[1], -1, pool.shape[3])[:, :n]


def attend_ref(q, k, v, seen, scale):
    """q [m][Hq][D], k and v [Hkv][n][D], seen [m][n] -> (result, sum of p |v|, each [m][Hq][D]), float64; masked
    keys and values are not touched, rows that see nothing are zero."""
    m, hq, dh = q.shape
    rep = hq // k.shape[0]
    k = k.double().repeat_interleave(rep, 0)
    v = v.double().repeat_interleave(rep, 0)
    out, mag = torch.zeros(m, hq, dh, dtype=torch.float64, device=q.device), torch.zeros(m, hq, dh, dtype=torch.float64,
                                                                                         device=q.device)
    for i in range(m):
        at = seen[i].nonzero()[:, 0]
        if len(at):
            w = torch.softmax(torch.einsum("hd,hnd->hn", q[i].double(), k[:, at]) * scale, -1)
            out[i] = torch.einsum("hn,hnd->hd", w, v[:, at])
            mag[i] = torch.einsum("hn,hnd->hd", w, v[:, at].abs())
    return out, mag


def attend_tol(out, mag):
    """The result is rounded to bf16 (8 significant bits: at most 2^-8 relative), and so is every probability as an
    operand; exponentials and fp32 sums of scores are good to 2^-12 of sum p |v| at these sizes."""
    return out.abs() * 2.0 ** -8 + mag * (2.0 ** -8 + 2.0 ** -12) + 1e-30


def rope_ref(x, pos, gamma, eps, theta):
    """x [T][H][D] -> normed (gamma) and rotated (theta), float64."""
    x = x.double()
    dh = x.shape[-1]
    if gamma is not None:
        x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps) * gamma.double()
    if theta:
        ang = pos.double()[:, None] * theta ** (-2.0 * torch.arange(dh // 2, device=x.device, dtype=torch.float64) / dh)
        c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
        a, b = x[..., :dh // 2], x[..., dh // 2:]
        x = torch.cat([a * c - b * s, b * c + a * s], -1)
    return x


def scale_of(dh):
    return 1.0 / math.sqrt(dh)
