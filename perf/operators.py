"""The paged key/value cache and the attention that reads it, timed through ``binding.PagedCache``.

A serving program keeps one cache: pages of keys and values for every layer,
a page table and a length per sequence, a reference count per page, all on the
GPU.  Four kinds of calls are timed:

* ``append``: norms of each query and key head, rotary positions, and the keys
  and values of a step's new tokens written into their pages, in one pass;
* ``prompt``: causal grouped-query attention of packed prompts of different
  lengths (or chunks of prompts that follow a cached prefix);
* ``tree``: attention of single tokens, or of a tree of drafted tokens, over
  each sequence's cache;
* ``fork`` and ``accept``: page bookkeeping.  ``fork`` branches a prompt into
  several continuations that share its pages and makes the shared last page of
  each its own for the first token; ``accept`` rolls a sequence back, makes room
  for a draft tree, and keeps one path of it, moved to the front.

Head counts are those of the repository's model families
(``workload.ATTN_SHAPES``).  In the plain form everything is elementary torch
operations in 32 bits, rounded once.
"""
import heapq
import math

import torch

own = False

# Query heads, key/value heads, head dimension of the model families.
SHAPES = {"switch": (12, 12, 64), "qwen": (16, 16, 128), "mixtral": (32, 8, 128)}
THETA = 1.0e6
EPS = 1.0e-6


def _case(name, op, family, seqs, ctx, q, page=64, layers=2, width=1, norm=True):
    """seqs sequences with between ctx[0] and ctx[1] cached tokens and between q[0] and q[1] new ones.
    width: parallel chains of a draft tree.  fork: q[0] tokens for each of seqs continuations of one prompt."""
    c = dict(op=op, family=family, seqs=seqs, ctx_lo=ctx[0], ctx_hi=ctx[1], q_lo=q[0], q_hi=q[1], page=page,
             layers=layers, width=width, norm=norm)
    return dict(c, name=name) if name else c


def listed():
    return [
        # One decode step of an odd batch: latency counts.
        _case("append_decode_113", "append", "mixtral", 113, (40, 2500), (1, 1)),
        # A full prefill batch of ragged prompts without cached prefix.
        _case("append_prompt_16384", "append", "mixtral", 9, (0, 0), (1100, 2541)),
        # A short prompt of the small model.
        _case("prompt_switch_777", "prompt", "switch", 1, (0, 0), (777, 777), page=32),
        # A batch of ragged prompts, as many key/value heads as query heads.
        _case("prompt_qwen_ragged", "prompt", "qwen", 11, (0, 0), (333, 1200)),
        # Chunks of long prompts behind cached prefixes.
        _case("prompt_mixtral_chunk", "prompt", "mixtral", 3, (2000, 9001), (500, 1033), page=128),
        # The longest prompt.
        _case("prompt_mixtral_16384", "prompt", "mixtral", 1, (0, 0), (16384, 16384)),
        # One sequence's next token: the smallest call.
        _case("decode_mixtral_1", "tree", "mixtral", 1, (1500, 1500), (1, 1)),
        # A decode batch over small pages.
        _case("decode_qwen_64", "tree", "qwen", 64, (300, 4000), (1, 1), page=16),
        # Long contexts.
        _case("decode_mixtral_long", "tree", "mixtral", 7, (30000, 65000), (1, 1)),
        # Verification of drafted trees: six chains, five deep, one of them cut.
        _case("tree_mixtral_24", "tree", "mixtral", 24, (1000, 8000), (29, 29), width=6),
        # A prompt branched into 24 continuations.
        _case("fork_mixtral_24", "fork", "mixtral", 24, (6001, 6001), (1, 1), layers=32),
        # Accepted paths of drafted trees.
        _case("accept_qwen_40", "accept", "qwen", 40, (100, 1500), (29, 29), width=6, layers=24),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "prompt", "prompt", "tree", "tree", "tree", "fork", "accept"])
    family = rng.choice(["switch", "qwen", "mixtral"])
    hq, hkv, dh = SHAPES[family]
    page = rng.choice([16, 32, 64, 128])
    if op == "append":
        if rng.random() < 0.5:
            return _case(None, op, family, _log_int(rng, 1, 256), (0, _log_int(rng, 16, 4000)), (1, 1), page,
                         norm=rng.random() < 0.7)
        seqs = _log_int(rng, 1, 12)
        mean = _log_int(rng, 64, 16384 // seqs)
        return _case(None, op, family, seqs, (0, rng.choice([0, 500])), (max(1, mean // 2), mean), page,
                     norm=rng.random() < 0.7)
    if op == "prompt":
        seqs = _log_int(rng, 1, 12)
        while True:
            top = _log_int(rng, 65, 12000)
            ctx = rng.choice([0, 0, _log_int(rng, 10, 8000)])
            if seqs * hq * top * (top + ctx) <= 32 * 12000 * 12000:
                return _case(None, op, family, seqs, (ctx // 2, ctx), (max(1, top // 3), top), page)
    if op == "tree":
        seqs = _log_int(rng, 1, 128)
        top = _log_int(rng, 30, max(60, min(40000, 250000 // seqs)))
        q = rng.choice([1, 1, _log_int(rng, 2, 64)])
        return _case(None, op, family, seqs, (top // 4, top), (q, q), page, width=rng.randint(1, 8) if q > 1 else 1)
    if op == "fork":
        return _case(None, op, family, _log_int(rng, 2, 24), (c := _log_int(rng, 20, 6000), c), (1, 1), page,
                     layers=rng.randint(4, 24))
    width = rng.randint(2, 8)
    q = rng.randint(3 * width, 64)
    return _case(None, op, family, _log_int(rng, 1, 40), (20, _log_int(rng, 40, 1500)), (q, q), page,
                 layers=rng.randint(4, 24), width=width)


def _spread(lo, hi, n, step):
    return [lo + int((hi - lo + 1) * ((i + 1) * step % 1.0)) if hi > lo else lo for i in range(n)]


def _lengths(case):
    """Cached and new tokens of each sequence of the step (fork: of each continuation)."""
    n = case["seqs"]
    return _spread(case["ctx_lo"], case["ctx_hi"], n, 0.6180339887), _spread(case["q_lo"], case["q_hi"], n, 0.7548776662)


def _inputs(case, seed):
    """Cache state before the step and the call's tensors, by the seed alone."""
    hq, hkv, dh = SHAPES[case["family"]]
    page, layers, op = case["page"], case["layers"], case["op"]
    ctx, q = _lengths(case)
    n = case["seqs"]
    pages = [-(-c // page) for c in ctx]
    if op == "fork":            # row 0 the prompt, rows 1..n the continuations (each the fork before the last's)
        held = [pages[0]] + [0] * n
        total = pages[0] + 3 * n
    else:
        held = pages
        total = sum(-(-(c + m) // page) for c, m in zip(ctx, q))
    rows, n_pages = len(held), total + 5 + total // 16
    max_pages = max(-(-(c + m) // page) for c, m in zip(ctx, q)) + 2
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 9176 + 11)
    dev = "cuda"
    ids = torch.randperm(n_pages, generator=g, device=dev)[:sum(held)].to(torch.int32)
    at = torch.arange(max_pages, device=dev)[None, :] < torch.tensor(held, device=dev)[:, None]
    table = torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev)
    table[at] = ids
    ref = torch.zeros(n_pages, dtype=torch.int32, device=dev)
    ref[ids.long()] = 1
    s = dict(case=case, page=page, table=table, ref=ref, heads=(hq, hkv, dh), ctx=ctx, q_len=q,
             length=torch.tensor(([ctx[0]] + [0] * n) if op == "fork" else ctx, dtype=torch.int32, device=dev),
             seq=list(range(1, n + 1)) if op == "fork" else list(range(n)),
             k=torch.empty((layers, n_pages, hkv, page, dh), dtype=torch.bfloat16, device=dev).normal_(generator=g),
             v=torch.empty((layers, n_pages, hkv, page, dh), dtype=torch.bfloat16, device=dev).normal_(generator=g))
    T = sum(q)
    if op == "append":
        s["qkv"] = torch.empty((T, (hq + 2 * hkv) * dh), dtype=torch.bfloat16, device=dev).normal_(generator=g)
        for name in ("gamma_q", "gamma_k"):
            w = 1 + 0.1 * torch.randn(dh, generator=g, device=dev)
            s[name] = w.to(torch.bfloat16) if case["norm"] else None
    elif op in ("prompt", "tree"):
        s["x"] = torch.empty((T, hq * dh), dtype=torch.bfloat16, device=dev).normal_(0.0, 1.3, generator=g)
    if op == "tree" and q[0] > 1:
        # Token i of a draft is at depth i // width of chain i % width and reads its chain's earlier tokens.
        words = []
        for i in range(q[0]):
            w = sum(1 << j for j in range(i % case["width"], i + 1, case["width"]))
            words.append(w - (1 << 64) if w >= 1 << 63 else w)
        s["tree"] = torch.tensor(words * n, dtype=torch.int64, device=dev)
    if op == "accept":
        # Chain c's first `kept` tokens, with c >= kept.
        w, deep = case["width"], q[0] // case["width"]
        kept = torch.randint(1, min(deep, w - 1) + 1, (n,), generator=g, device=dev) if w > 1 else torch.ones(n, device=dev)
        kept = kept.to(torch.int32)
        chain = kept + (torch.rand(n, generator=g, device=dev) * (w - kept)).to(torch.int32)
        s["kept"] = kept
        s["path"] = chain[:, None] + w * torch.arange(deep, device=dev, dtype=torch.int32)[None, :]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    hq = s["heads"][0]
    if own:
        from paper_2608_00573_gb300 import binding as B
        s["cache"] = B.PagedCache(s["k"], s["v"], s["table"], s["length"], s["ref"], q_heads=hq,
                                  T_max=max(1, sum(s["q_len"])))
        if case["op"] in ("append", "prompt", "tree"):
            s["cache"].step(s["seq"], s["q_len"])
    elif case["op"] in ("append", "prompt", "tree"):
        _plain_step(s, s["seq"], s["q_len"])
    return s


def run(s):
    case, op = s["case"], s["case"]["op"]
    if not own:
        return {"append": _plain_append, "prompt": _plain_attend, "tree": _plain_attend, "fork": _plain_fork,
                "accept": _plain_accept}[op](s)
    c = s["cache"]
    if op == "append":
        q = c.append(1, s["qkv"], gamma_q=s["gamma_q"], gamma_k=s["gamma_k"], eps=EPS, theta=THETA)
        return q, s["k"], s["v"]
    if op in ("prompt", "tree"):
        return c.attend(1, s["x"], tree=s.get("tree"))
    if op == "fork":
        c.fork([0] * case["seqs"], s["seq"])
        c.step(s["seq"], s["q_len"])
    else:
        c.truncate(s["seq"], s["ctx"])
        c.step(s["seq"], s["q_len"])
        c.accept(s["seq"], s["kept"], s["path"])
    return s["k"], s["v"], s["table"], s["length"], s["ref"]


# ------------------------------------------------------------- plain form

def _dev(s, values):
    return torch.tensor(values, device=s["k"].device)


def _count(s, ids, by):
    """ref[id] += by for every id >= 0."""
    ids = ids.reshape(-1).long()
    s["ref"].index_add_(0, ids.clamp(min=0), ((ids >= 0) * by).to(torch.int32))


def _plain_step(s, seq, q_len):
    """Room for q_len new tokens of each sequence: the lowest free pages, in the order of the sequences; a shared last
    page that would be written is copied."""
    page, rows = s["page"], _dev(s, seq)
    length = s["length"][rows].long()
    after = length + _dev(s, q_len)
    t = s["table"][rows]
    had, need = (length + page - 1) // page, (after + page - 1) // page
    last = t.gather(1, (had - 1).clamp(min=0)[:, None])[:, 0].long()
    copied = (length % page != 0) & (after > length) & (s["ref"][last.clamp(min=0)] > 1)
    j = torch.arange(t.shape[1], device=t.device)[None, :]
    fresh = ((j >= had[:, None]) & (j < need[:, None])) | ((j == had[:, None] - 1) & copied[:, None])
    free = torch.argsort((s["ref"] > 0).to(torch.int32), stable=True)
    rank = fresh.reshape(-1).cumsum(0).reshape(t.shape) - 1
    _count(s, torch.where(fresh & (t >= 0), t, -1), -1)
    t = torch.where(fresh, free[rank.clamp(min=0)].to(torch.int32), t)
    _count(s, torch.where(fresh, t, -1), 1)
    i = copied.nonzero()[:, 0]
    to = t.gather(1, (had - 1).clamp(min=0)[:, None])[:, 0].long()
    for pool in (s["k"], s["v"]):
        pool[:, to[i]] = pool[:, last[i]]
    s["table"][rows] = t
    s["length"][rows] = after.to(torch.int32)


def _slots(s, rows, pos):
    """Page and place in it of position pos[i] of sequence rows[i]."""
    return s["table"][rows, pos // s["page"]].long(), pos % s["page"]


def _plain_append(s):
    hq, hkv, dh = s["heads"]
    x = s["qkv"].float().view(-1, hq + 2 * hkv, dh)
    q_len = _dev(s, s["q_len"])
    rows = torch.repeat_interleave(_dev(s, s["seq"]), q_len, output_size=x.shape[0])
    first = torch.repeat_interleave(q_len.cumsum(0) - q_len - _dev(s, s["ctx"]), q_len, output_size=x.shape[0])
    pos = torch.arange(x.shape[0], device=x.device) - first
    qk = x[:, :hq + hkv]
    if s["gamma_q"] is not None:
        qk = qk * torch.rsqrt(qk.square().mean(-1, keepdim=True) + EPS)
        qk = qk * torch.cat([s["gamma_q"].float().expand(hq, dh), s["gamma_k"].float().expand(hkv, dh)])
    turn = pos.float()[:, None] * torch.pow(THETA, -torch.arange(0, dh, 2, device=x.device).float() / dh)[None, :]
    cos, sin = turn.cos()[:, None, :], turn.sin()[:, None, :]
    a, b = qk[..., :dh // 2], qk[..., dh // 2:]
    qk = torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(torch.bfloat16)
    where, place = _slots(s, rows, pos)
    s["k"][1][where, :, place] = qk[:, hq:]
    s["v"][1][where, :, place] = s["qkv"].view(-1, hq + 2 * hkv, dh)[:, hq + hkv:]
    return qk[:, :hq].reshape(-1, hq * dh), s["k"], s["v"]


def _plain_attend(s):
    hq, hkv, dh = s["heads"]
    n, q_len, ctx = len(s["q_len"]), _dev(s, s["q_len"]), _dev(s, s["ctx"])
    m, T = max(s["q_len"]), s["x"].shape[0]
    longest = max(a + b for a, b in zip(s["ctx"], s["q_len"]))
    pages = -(-longest // s["page"])
    at = s["table"][_dev(s, s["seq"]), :pages].clamp(min=0).long()
    k, v = (p[1][at].permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, dh)[:, :, :longest].float() for p in (s["k"], s["v"]))
    i = torch.arange(m, device=k.device)
    new = i[None, :] < q_len[:, None]                                   # [n][m] tokens that are there
    x = torch.zeros((n, m, hq * dh), device=k.device)
    x[new] = s["x"].float()
    x = x.view(n, m, hkv, hq // hkv, dh).permute(0, 2, 3, 1, 4).reshape(n, hkv, -1, dh)
    key = torch.arange(longest, device=k.device)[None, None, :]
    if s.get("tree") is not None:
        word = s["tree"].view(n, m)[:, :, None]
        draft = key - ctx[:, None, None]
        seen = (draft < 0) | ((draft < m) & ((word >> draft.clamp(0, 63)) & 1 == 1))
    else:
        seen = key <= (ctx[:, None] + i[None, :])[:, :, None]           # [n][m][keys]
    w = torch.matmul(x, k.transpose(2, 3)).view(n, hkv, hq // hkv, m, longest)
    w.mul_(1.0 / math.sqrt(dh)).masked_fill_(~seen[:, None, None], -math.inf)
    top = w.amax(-1, keepdim=True)
    w.sub_(top.masked_fill(top == -math.inf, 0.0)).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(n, hkv, -1, longest), v).view(n, hkv, hq // hkv, m, dh)
    o = o / total.masked_fill(total == 0, 1.0)
    return o.permute(0, 3, 1, 2, 4).reshape(n, m, hq * dh)[new].to(torch.bfloat16).view(T, hq * dh)


def _plain_fork(s):
    rows = _dev(s, s["seq"])
    _count(s, s["table"][rows], -1)
    s["table"][rows] = s["table"][0].clone()
    s["length"][rows] = s["length"][0].clone()
    _count(s, s["table"][rows], 1)
    _plain_step(s, s["seq"], s["q_len"])
    return s["k"], s["v"], s["table"], s["length"], s["ref"]


def _plain_truncate(s, seq, to):
    rows = _dev(s, seq)
    to = torch.minimum(to, s["length"][rows].long())
    t = s["table"][rows]
    over = torch.arange(t.shape[1], device=t.device)[None, :] >= ((to + s["page"] - 1) // s["page"])[:, None]
    _count(s, torch.where(over, t, -1), -1)
    s["table"][rows] = torch.where(over, -1, t)
    s["length"][rows] = to.to(torch.int32)


def _plain_accept(s):
    base = _dev(s, s["ctx"])
    _plain_truncate(s, s["seq"], base)
    _plain_step(s, s["seq"], s["q_len"])
    rows = _dev(s, s["seq"])[:, None].expand_as(s["path"])
    i = torch.arange(s["path"].shape[1], device=base.device)[None, :]
    to = (base[:, None] + i)
    frm = torch.where(i < s["kept"][:, None], base[:, None] + s["path"], to)
    a, x = _slots(s, rows.reshape(-1), frm.reshape(-1).long())
    b, y = _slots(s, rows.reshape(-1), to.reshape(-1).long())
    for pool in (s["k"], s["v"]):
        pool[:, b, :, y] = pool[:, a, :, x]
    _plain_truncate(s, s["seq"], base + s["kept"])
    return s["k"], s["v"], s["table"], s["length"], s["ref"]


# ----------------------------------------------------- work and exact values

def work(case):
    hq, hkv, dh = SHAPES[case["family"]]
    ctx, q = _lengths(case)
    T, row = sum(q), 2 * hkv * dh * 2                       # K and V bytes of one token and layer
    table = 4 * sum(-(-(c + m) // case["page"]) for c, m in zip(ctx, q))
    if case["op"] == "append":
        return {"bytes": T * (hq + 2 * hkv) * dh * 4, "flops": T * (hq + hkv) * dh * 7}
    if case["op"] in ("prompt", "tree"):
        if case["op"] == "tree" and q[0] > 1:
            seen = [q[0] * c + sum(i // case["width"] + 1 for i in range(q[0])) for c in ctx]
        else:
            seen = [m * c + m * (m + 1) // 2 for c, m in zip(ctx, q)]
        return {"bytes": sum((c + m) * row for c, m in zip(ctx, q)) + 2 * T * hq * dh * 2 + table,
                "flops": 4 * dh * hq * sum(seen)}
    if case["op"] == "fork":
        copied = case["seqs"] * (1 if ctx[0] % case["page"] else 0)
        return {"bytes": 2 * copied * case["page"] * row * case["layers"] + 3 * table, "flops": 0}
    kept = case["seqs"] * (1 + min(q[0] // case["width"], max(1, case["width"] - 1))) / 2
    return {"bytes": 2 * kept * row * case["layers"] + 3 * table, "flops": 0}


class _Pages:
    """The cache's bookkeeping on the host, one sequence and page at a time."""

    def __init__(self, s):
        self.page = s["page"]
        self.len = s["length"].tolist()
        self.own = [[p for p in r if p >= 0] for r in s["table"].tolist()]
        self.ref = s["ref"].tolist()

    def drop(self, p):
        self.ref[p] -= 1

    def step(self, seq, q):
        free = [p for p, r in enumerate(self.ref) if r == 0]
        heapq.heapify(free)
        before, copies = list(self.ref), []
        for r, m in zip(seq, q):
            mine = self.own[r]
            if m and self.len[r] % self.page and before[mine[-1]] > 1:
                p = heapq.heappop(free)
                copies.append((mine[-1], p))
                self.drop(mine[-1])
                mine[-1] = p
                self.ref[p] = 1
            self.len[r] += m
            while len(mine) * self.page < self.len[r]:
                mine.append(heapq.heappop(free))
                self.ref[mine[-1]] = 1
        return copies

    def cut(self, r, to):
        while (len(self.own[r]) - 1) * self.page >= to and self.own[r]:
            self.drop(self.own[r].pop())
        self.len[r] = to

    def tensors(self, s):
        width = s["table"].shape[1]
        return [torch.tensor(x, dtype=torch.int32) for x in
                ([r + [-1] * (width - len(r)) for r in self.own], self.len, self.ref)]


def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, dh = s["heads"]
    page, ctx, q = s["page"], s["ctx"], s["q_len"]
    b = _Pages(s)
    if case["op"] == "fork":
        for r in s["seq"]:
            b.own[r], b.len[r] = list(b.own[0]), b.len[0]
            for p in b.own[r]:
                b.ref[p] += 1
        copies = b.step(s["seq"], q)
        k, v = s["k"].double(), s["v"].double()
        for frm, to in copies:
            k[:, to], v[:, to] = k[:, frm].clone(), v[:, frm].clone()
        return (k, v, *b.tensors(s))
    b.step(s["seq"], q)
    if case["op"] == "accept":
        k, v = s["k"].double(), s["v"].double()
        for r, (c, kept, path) in enumerate(zip(ctx, s["kept"].tolist(), s["path"].tolist())):
            for i in range(kept):
                a, z = c + path[i], c + i
                for pool in (k, v):
                    pool[:, b.own[r][z // page], :, z % page] = pool[:, b.own[r][a // page], :, a % page].clone()
            b.cut(r, c + kept)
        return (k, v, *b.tensors(s))
    if case["op"] == "append":
        x = s["qkv"].double().view(-1, hq + 2 * hkv, dh)
        k, v = s["k"].double(), s["v"].double()
        out, t = [], 0
        rate = THETA ** (-2.0 * torch.arange(dh // 2, device=x.device, dtype=torch.float64) / dh)
        for r, (c, m) in enumerate(zip(ctx, q)):
            y = x[t:t + m]
            pos = torch.arange(c, c + m, device=x.device)
            both = []
            for part, w in ((y[:, :hq], s["gamma_q"]), (y[:, hq:hq + hkv], s["gamma_k"])):
                if w is not None:
                    part = part / torch.sqrt(part.pow(2).sum(-1, keepdim=True) / dh + EPS) * w.double()
                z = torch.complex(part[..., :dh // 2], part[..., dh // 2:])
                z = z * torch.polar(torch.ones_like(rate), pos.double()[:, None] * rate)[:, None, :]
                both.append(torch.cat([z.real, z.imag], -1))
            own_pages = torch.tensor(b.own[r], device=x.device)
            k[1, own_pages[pos // page], :, pos % page] = both[1]
            v[1, own_pages[pos // page], :, pos % page] = y[:, hq + hkv:]
            out.append(both[0].reshape(m, hq * dh))
            t += m
        return torch.cat(out), k, v
    out, t = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda"), 0
    rep = hq // hkv
    for r, (c, m) in enumerate(zip(ctx, q)):
        n = c + m
        pages = torch.tensor(b.own[r], device="cuda")
        k, v = (p[1, pages].transpose(0, 1).reshape(hkv, -1, dh)[:, :n].double() for p in (s["k"], s["v"]))
        for lo in range(0, m, 1024):
            hi = min(m, lo + 1024)
            keys = n if s.get("tree") is not None else c + hi
            ok = torch.arange(keys, device="cuda")[None, :] <= torch.arange(c + lo, c + hi, device="cuda")[:, None]
            if s.get("tree") is not None:
                for i in range(lo, hi):
                    bits = int(s["tree"][t + i]) & ((1 << 64) - 1)
                    ok[i - lo, c:] = torch.tensor([bool(bits >> j & 1) for j in range(m)], device="cuda")
            for h in range(hq):
                x = s["x"][t + lo:t + hi, h * dh:(h + 1) * dh].double()
                w = (x @ k[h // rep, :keys].T) / math.sqrt(dh)
                out[t + lo:t + hi, h * dh:(h + 1) * dh] = w.masked_fill(~ok, -math.inf).softmax(-1) @ v[h // rep, :keys]
        t += m
    return out
