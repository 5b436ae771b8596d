"""Attention over a paged cache that does not read all of it for every sequence, timed through ``binding.PagedCache``.

Two ways to read less, and what the second one needs:

* ``shared``: sequences that were forked from one prompt hold the same pages for it.  ``cache.share`` tells a step
  which of its sequences belong together, and ``cache.attend`` then reads their common pages once for all of
  them, each sequence's own pages for itself.
* ``blocks``: each query attends to a few pages ("blocks") of its sequence's past, a list per token and
  key/value head, and to the positions from the step's first page on.
* ``select``: writes such lists.  The score of a block bounds the scores of its keys from above: with the least and
  the largest value of each key column, lo and hi, it is sum_d max(q_d lo_d, q_d hi_d), the largest over the query
  heads that share the key/value head.  lo and hi are held in 8 bits, rounded outwards, with one power of two per
  block and head, and queries are rounded to 8 bits likewise, so every sum is a whole number times a power of
  two: exact in 32 bits, and equal scores go to the lower block.
* ``bounds``: lo and hi of the pages that a step's new tokens filled.

Head counts are those of the repository's model families (``workload.ATTN_SHAPES``).  In the plain form everything is
elementary torch operations in 32 bits, rounded once.
"""
import math

import torch

own = False

# Query heads, key/value heads, head dimension of the model families.
SHAPES = {"switch": (12, 12, 64), "qwen": (16, 16, 128), "mixtral": (32, 8, 128)}


def _case(name, op, family, seqs, ctx, q, page=64, layers=2, width=1, n=0, groups=0, prefix=(0, 0)):
    """seqs sequences with between ctx[0] and ctx[1] cached tokens and between q[0] and q[1] new ones; width:
    parallel chains of a draft tree (1: causal); n: blocks per list.  shared: `groups` groups of between seqs[0] and
    seqs[1] sequences, with a common prefix of between prefix[0] and prefix[1] tokens before the ctx of their own."""
    few, many = seqs if isinstance(seqs, tuple) else (seqs, seqs)
    c = dict(op=op, family=family, seqs_lo=few, seqs_hi=many, ctx_lo=ctx[0], ctx_hi=ctx[1], q_lo=q[0], q_hi=q[1],
             page=page, layers=layers, width=width, n=n, groups=groups, prefix_lo=prefix[0], prefix_hi=prefix[1])
    return dict(c, name=name) if name else c


def listed():
    return [
        # Four samples of a short prompt, a token each: latency counts.
        _case("shared_mixtral_4", "shared", "mixtral", 4, (3, 60), (1, 1), groups=1, prefix=(700, 700)),
        # Many samples of one long prompt.
        _case("shared_mixtral_64", "shared", "mixtral", 64, (0, 900), (1, 1), groups=1, prefix=(8200, 8200)),
        # A decode batch of several system prompts, few or many sequences behind each; small pages.
        _case("shared_qwen_groups", "shared", "qwen", (1, 24), (0, 500), (1, 1), page=16, groups=5, prefix=(300, 6000)),
        # Drafted trees behind a long common document; large pages.
        _case("shared_mixtral_tree", "shared", "mixtral", 12, (100, 2000), (29, 29), page=128, width=6, groups=1,
              prefix=(12001, 12001)),
        # One long sequence's next token.
        _case("blocks_mixtral_1", "blocks", "mixtral", 1, (20011, 20011), (1, 1), n=32),
        # A decode batch over small pages.
        _case("blocks_qwen_48", "blocks", "qwen", 48, (2000, 12000), (1, 1), page=16, n=96),
        # Chunks of prompts behind long contexts, each token with lists of its own.
        _case("blocks_mixtral_chunk", "blocks", "mixtral", 3, (6000, 15000), (200, 333), n=24),
        # The lists of one long sequence's next token.
        _case("select_mixtral_1", "select", "mixtral", 1, (20011, 20011), (1, 1), n=32),
        # Those of a decode batch of long contexts.
        _case("select_mixtral_48", "select", "mixtral", 48, (4000, 40000), (1, 1), page=32, layers=1, n=64),
        # Those of chunks of prompts, small heads.
        _case("select_switch_chunk", "select", "switch", 3, (6000, 15000), (200, 333), page=32, n=40),
        # A decode step: few sequences fill a page.
        _case("bounds_decode_113", "bounds", "mixtral", 113, (40, 2500), (1, 1), page=16),
        # A full prefill batch of ragged prompts.
        _case("bounds_prompt_16384", "bounds", "mixtral", 9, (0, 0), (1100, 2541)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """No costlier than the largest listed case of its kind; some block is left out of a list, some page is filled."""
    op = rng.choice(["shared", "shared", "shared", "blocks", "blocks", "blocks", "select", "select", "bounds"])
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        case = _draw(rng, op)
        w = work(case)
        idle = max(_lengths(case)[2]) // case["page"] < case["n"] + 3 if op == "select" else w["flops"] == 0
        if not idle and all(w[k] <= max(m[k] for m in most) for k in w):
            return case


def _draw(rng, op):
    family, page = rng.choice(list(SHAPES)), rng.choice([16, 32, 64, 128])
    if op == "shared":
        groups = rng.choice([1, 1, 2, rng.randint(3, 6)])
        few, many = sorted((_log_int(rng, 1, 64), _log_int(rng, 2, 64)))
        lo, hi = sorted((_log_int(rng, 50, 12000), _log_int(rng, 100, 12000)))
        ctx = _log_int(rng, 1, 2000)
        q = rng.choice([1, 1, rng.randint(2, 40)])
        return _case(None, op, family, (few, many), (ctx // 4, ctx), (q, q), page,
                     width=rng.randint(1, 6) if q > 1 else 1, groups=groups, prefix=(lo, hi))
    if op == "bounds":
        if rng.random() < 0.5:
            return _case(None, op, family, _log_int(rng, 1, 256), (0, _log_int(rng, 16, 4000)), (1, 1), page)
        seqs = _log_int(rng, 1, 12)
        mean = _log_int(rng, 64, 16384 // seqs)
        return _case(None, op, family, seqs, (0, rng.choice([0, 500])), (max(1, mean // 2), mean), page)
    n = max(4, _log_int(rng, 128, 2048) // page)
    if rng.random() < 0.6:
        seqs = _log_int(rng, 1, 64)
        top = _log_int(rng, 60, max(100, min(40000, 500000 // seqs)))
        return _case(None, op, family, seqs, (top // 4, top), (1, 1), page, n=n)
    seqs, m, top = _log_int(rng, 1, 4), _log_int(rng, 2, 300), _log_int(rng, 60, 15000)
    if op == "blocks" and m <= 64 and rng.random() < 0.5:
        return _case(None, op, family, seqs, (top // 4, top), (m, m), page, n=n, width=rng.randint(1, 6))
    return _case(None, op, family, seqs, (top // 4, top), (max(1, m // 2), m), page, n=n)


def _spread(lo, hi, n, step):
    return [lo + int((hi - lo + 1) * ((i + 1) * step % 1.0)) if hi > lo else lo for i in range(n)]


def _lengths(case):
    """Per group: sequences and common tokens; per sequence: cached and new tokens."""
    if case["op"] == "shared":
        sizes = _spread(case["seqs_lo"], case["seqs_hi"], case["groups"], 0.4142135624)
        prefix = _spread(case["prefix_lo"], case["prefix_hi"], case["groups"], 0.7320508076)
    else:
        sizes, prefix = [1] * case["seqs_hi"], [0] * case["seqs_hi"]
    n = sum(sizes)
    common = [p for p, m in zip(prefix, sizes) for _ in range(m)]
    ctx = [p + c for p, c in zip(common, _spread(case["ctx_lo"], case["ctx_hi"], n, 0.6180339887))]
    return sizes, prefix, ctx, _spread(case["q_lo"], case["q_hi"], n, 0.7548776662)


def _inputs(case, seed):
    """Cache state before the step and the call's tensors, by the seed alone."""
    hq, hkv, dh = SHAPES[case["family"]]
    page, layers, op, dev = case["page"], case["layers"], case["op"], "cuda"
    sizes, prefix, ctx, q = _lengths(case)
    rows = len(ctx)
    shared = [p // page if m > 1 else 0 for p, m in zip(prefix, sizes)]          # whole pages that a group holds together
    total = sum(shared) + sum(-(-(c + m) // page) for c, m in zip(ctx, q))
    n_pages, max_pages = total + 5 + total // 16, max(-(-(c + m) // page) for c, m in zip(ctx, q)) + 2
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 7919 + 23)
    ids = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32).cpu()
    table, ref = torch.full((rows, max_pages), -1, dtype=torch.int32), torch.zeros(n_pages, dtype=torch.int32)
    at = r = 0
    for size, common in zip(sizes, shared):
        front = ids[at:at + common]
        at += common
        ref[front.long()] = size
        for _ in range(size):
            held = -(-ctx[r] // page) - common
            table[r, :common] = front
            table[r, common:common + held] = ids[at:at + held]
            ref[ids[at:at + held].long()] = 1
            at += held
            r += 1
    s = dict(case=case, page=page, table=table.to(dev), ref=ref.to(dev), heads=(hq, hkv, dh), ctx=ctx, q_len=q,
             seq=list(range(rows)), sizes=sizes, shared=shared, layer=layers - 1,
             length=torch.tensor(ctx, dtype=torch.int32, device=dev),
             k=torch.empty((layers, n_pages, hkv, page, dh), dtype=torch.bfloat16, device=dev).normal_(generator=g),
             v=torch.empty((layers, n_pages, hkv, page, dh), dtype=torch.bfloat16, device=dev).normal_(generator=g))
    if op in ("blocks", "select"):
        # Neighbouring keys are alike, or no block would stand out.
        k = s["k"][s["layer"]]
        k.mul_(0.7).add_(torch.empty((n_pages, hkv, 1, dh), dtype=torch.bfloat16, device=dev).normal_(0.0, 0.7, generator=g))
    if op == "bounds":
        s["codes"] = torch.zeros((layers, n_pages, hkv, 2, dh), dtype=torch.int8, device=dev)
        s["scales"] = torch.zeros((layers, n_pages, hkv), device=dev)
    else:
        s["x"] = torch.empty((sum(q), hq * dh), dtype=torch.bfloat16, device=dev).normal_(0.0, 1.3, generator=g)
    if case["width"] > 1:
        # Token i of a draft is at depth i // width of chain i % width and reads its chain's earlier tokens.
        words = []
        for i in range(q[0]):
            w = sum(1 << j for j in range(i % case["width"], i + 1, case["width"]))
            words.append(w - (1 << 64) if w >= 1 << 63 else w)
        s["tree"] = torch.tensor(words * rows, dtype=torch.int64, device=dev)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op, layer = case["op"], s["layer"]
    if op in ("blocks", "select"):
        codes, scales = _plain_bounds_of(s["k"][layer])
        s["codes"], s["scales"] = (torch.zeros((case["layers"],) + t.shape, dtype=t.dtype, device=t.device)
                                   for t in (codes, scales))
        s["codes"][layer], s["scales"][layer] = codes, scales
    if own:
        from paper_2608_00573_gb300 import binding as B
        bounds = (s["codes"], s["scales"]) if "codes" in s else None
        s["cache"] = B.PagedCache(s["k"], s["v"], s["table"], s["length"], s["ref"], q_heads=s["heads"][0],
                                  T_max=max(1, sum(s["q_len"])), bounds=bounds)
        s["cache"].step(s["seq"], s["q_len"])
        if op == "shared":
            s["cache"].share(s["sizes"])
    else:
        _plain_step(s)
    if op == "blocks":
        s["blocks"] = _plain_select(s)
    return s


def run(s):
    op, layer = s["case"]["op"], s["layer"]
    if not own:
        if op == "bounds":
            return _plain_bounds(s)
        return {"shared": _plain_shared, "blocks": _plain_blocks, "select": _plain_select}[op](s)
    c = s["cache"]
    if op == "shared":
        return c.attend(layer, s["x"], tree=s.get("tree"))
    if op == "blocks":
        return c.attend_blocks(layer, s["x"], s["blocks"], tree=s.get("tree"))
    if op == "select":
        return c.select(layer, s["x"], s["case"]["n"])
    c.summarize(layer)
    return _bounds_values(s)


def _bounds_values(s):
    """The bounds that the 8-bit codes of the layer stand for, and the scales."""
    codes, scales = s["codes"][s["layer"]], s["scales"][s["layer"]]
    return codes.float() * scales[..., None, None], scales


# ------------------------------------------------------------- plain form

def _dev(s, values):
    return torch.tensor(values, device=s["k"].device)


def _plain_step(s):
    """Room for the new tokens: the lowest free pages, in the order of the sequences (no last page is shared here)."""
    had = _dev(s, [-(-c // s["page"]) for c in s["ctx"]])[:, None]
    need = _dev(s, [-(-(c + m) // s["page"]) for c, m in zip(s["ctx"], s["q_len"])])[:, None]
    j = torch.arange(s["table"].shape[1], device=had.device)[None, :]
    fresh = (j >= had) & (j < need)
    free = (s["ref"] == 0).nonzero()[:, 0][:int(fresh.sum())]
    s["table"][fresh] = free.to(torch.int32)
    s["ref"][free] = 1
    s["length"] += _dev(s, s["q_len"]).to(torch.int32)


def _token_rows(s):
    """Of each new token: its sequence, its place among the sequence's new tokens, the positions before the step."""
    q, ctx = _dev(s, s["q_len"]), _dev(s, s["ctx"])
    T = sum(s["q_len"])
    rows = torch.repeat_interleave(torch.arange(len(s["q_len"]), device=q.device), q, output_size=T)
    return rows, torch.arange(T, device=q.device) - (q.cumsum(0) - q)[rows], ctx[rows]


def _grid(amax):
    """The least power of two of which amax is at most 127 times (at least 2^-126)."""
    m, e = torch.frexp(amax)
    e = torch.where(m * 128 <= 127, e - 7, e - 6).masked_fill(amax == 0, -126).clamp(min=-126)
    return ((e + 127) << 23).view(torch.float32)                        # 2^e


def _plain_bounds_of(k):
    """Codes [..][2][dh] and scale of each block and head of keys [..][page][dh]."""
    lo, hi = k.float().amin(-2), k.float().amax(-2)
    scale = _grid(torch.maximum(lo.abs(), hi.abs()).amax(-1))
    return torch.stack([(lo / scale[..., None]).floor(), (hi / scale[..., None]).ceil()], -2).to(torch.int8), scale


def _plain_bounds(s):
    page, layer = s["page"], s["layer"]
    first = _dev(s, [c // page for c in s["ctx"]])[:, None]
    end = _dev(s, [(c + m) // page for c, m in zip(s["ctx"], s["q_len"])])[:, None]
    j = torch.arange(s["table"].shape[1], device=end.device)[None, :]
    ids = s["table"][(j >= first) & (j < end)].long()
    codes, scales = _plain_bounds_of(s["k"][layer][ids])
    s["codes"][layer][ids] = codes
    s["scales"][layer][ids] = scales
    return _bounds_values(s)


def _plain_select(s):
    hq, hkv, dh = s["heads"]
    n, page, layer = s["case"]["n"], s["page"], s["layer"]
    rows, _, ctx = _token_rows(s)
    full = ctx // page                                                  # whole blocks before the step
    most = max(1, max(s["ctx"]) // page)
    x = s["x"].float().view(-1, hkv, hq // hkv, dh)
    grid = _grid(x.abs().amax(-1, keepdim=True))
    x = (x / grid).round()                                              # half to even
    col = torch.arange(most, device=x.device)
    out = torch.full((x.shape[0], hkv, n), -1, dtype=torch.int32, device=x.device)
    for r in range(len(s["ctx"])):
        mine = (rows == r).nonzero()[:, 0]
        f = s["ctx"][r] // page
        if not f:
            continue
        ids = s["table"][r, :f].long()
        lo, hi = s["codes"][layer][ids].float().permute(2, 1, 3, 0)     # [hkv][dh][f]
        y = x[mine].permute(1, 0, 2, 3).reshape(hkv, -1, dh)
        score = torch.matmul(y.clamp(min=0), hi) + torch.matmul(y.clamp(max=0), lo)
        score = score.view(hkv, len(mine), -1, f) * grid[mine].permute(1, 0, 2, 3)
        score = score.amax(2) * s["scales"][layer][ids].t()[:, None, :]
        score[..., 0] = score[..., f - 1] = math.inf                    # the first and the last one always
        best = torch.sort(score, dim=-1, descending=True, stable=True)[1][..., :n].sort(-1)[0]
        out[mine, :, :best.shape[-1]] = best.permute(1, 0, 2).to(torch.int32)
    return out


def _plain_blocks(s):
    hq, hkv, dh = s["heads"]
    page, layer, rep = s["page"], s["layer"], hq // hkv
    rows, place, ctx = _token_rows(s)
    first = ctx // page * page                                          # the step's own pages begin here
    tail = torch.arange(max((c % page + m - 1) // page for c, m in zip(s["ctx"], s["q_len"])) + 1, device=rows.device)
    off = torch.arange(page, device=rows.device)
    head = torch.arange(hkv, device=rows.device)
    scale, out = 1.0 / math.sqrt(dh), []
    step = max(1, (1 << 28) // (hkv * dh * page * (s["blocks"].shape[2] + len(tail))))
    for a in range(0, len(rows), step):
        t = slice(a, a + step)
        col = torch.cat([s["blocks"][t], (first[t, None] // page + tail)[:, None, :].expand(-1, hkv, -1)], 2).long()
        own_page = torch.arange(col.shape[2], device=rows.device) >= s["blocks"].shape[2]
        pos = col[..., None] * page + off                               # [m][hkv][columns][page]
        if s.get("tree") is not None:
            draft = pos - ctx[t, None, None, None]
            bit = (s["tree"][t, None, None, None] >> draft.clamp(0, 63)) & 1 == 1
            late = (draft < 0) | ((draft < 64) & bit)
        else:
            late = pos <= (ctx + place)[t, None, None, None]
        seen = torch.where(own_page[:, None], late, col[..., None] >= 0).flatten(2)
        id = s["table"][rows[t, None, None], col.clamp(0, s["table"].shape[1] - 1)].clamp(min=0).long()
        k, v = (p[layer][id, head[:, None]].float().flatten(2, 3) for p in (s["k"], s["v"]))
        w = torch.matmul(s["x"][t].float().view(-1, hkv, rep, dh), k.transpose(2, 3)) * scale
        w = w.masked_fill(~seen[:, :, None], -math.inf)
        top = w.amax(-1, keepdim=True)
        w = (w - top.masked_fill(top == -math.inf, 0.0)).exp()
        total = w.sum(-1, keepdim=True)
        o = torch.matmul(w, v) / total.masked_fill(total == 0, 1.0)
        out.append(o.reshape(-1, hq * dh).to(torch.bfloat16))
    return torch.cat(out)


def _plain_shared(s):
    hq, hkv, dh = s["heads"]
    page, layer, rep = s["page"], s["layer"], hq // hkv
    scale, out, a, t = 1.0 / math.sqrt(dh), [], 0, 0
    for size, common in zip(s["sizes"], s["shared"]):
        q_len, ctx = s["q_len"][a:a + size], s["ctx"][a:a + size]
        T, m, longest = sum(q_len), max(q_len), max(c + n for c, n in zip(ctx, q_len))
        first, x = common * page, s["x"][t:t + T].float()
        # The common pages once, for all rows of the group.
        id = s["table"][a, :common].long()
        k, v = (p[layer][id].transpose(0, 1).reshape(hkv, first, dh).float() for p in (s["k"], s["v"]))
        y = x.view(T, hkv, rep, dh).transpose(0, 1).reshape(hkv, -1, dh)
        wc = (torch.matmul(y, k.transpose(1, 2)) * scale).view(hkv, T, rep, first).transpose(0, 1)
        # Each sequence's own ones.
        lens, base = _dev(s, q_len), _dev(s, ctx)
        i = torch.arange(m, device=x.device)
        new = i[None, :] < lens[:, None]
        z = torch.zeros((size, m, hq * dh), device=x.device)
        z[new] = x
        z = z.view(size, m, hkv, rep, dh).permute(0, 2, 3, 1, 4).reshape(size, hkv, -1, dh)
        id = s["table"][a:a + size, common:-(-longest // page)].clamp(min=0).long()
        ko, vo = (p[layer][id].permute(0, 2, 1, 3, 4).reshape(size, hkv, -1, dh).float() for p in (s["k"], s["v"]))
        key = first + torch.arange(ko.shape[2], device=x.device)[None, None, :]
        if s.get("tree") is not None:
            draft = key - base[:, None, None]
            word = s["tree"][t:t + T].view(size, m)[:, :, None]
            seen = (draft < 0) | ((draft < m) & ((word >> draft.clamp(0, 63)) & 1 == 1))
        else:
            seen = key <= (base[:, None] + i[None, :])[:, :, None]
        wo = (torch.matmul(z, ko.transpose(2, 3)) * scale).view(size, hkv, rep, m, -1)
        wo = wo.masked_fill(~seen[:, None, None], -math.inf).permute(0, 3, 1, 2, 4)[new]     # [T][hkv][rep][keys]
        w = torch.cat([wc, wo], -1)
        top = w.amax(-1, keepdim=True)
        w = (w - top.masked_fill(top == -math.inf, 0.0)).exp()
        total = w.sum(-1, keepdim=True)
        wc, wo = w[..., :first], w[..., first:]
        oc = torch.matmul(wc.transpose(0, 1).reshape(hkv, T * rep, first), v).view(hkv, T, rep, dh).transpose(0, 1)
        z = torch.zeros((size, m) + wo.shape[1:], device=x.device)
        z[new] = wo
        z = z.permute(0, 2, 3, 1, 4).reshape(size, hkv, rep * m, -1)
        oo = torch.matmul(z, vo).view(size, hkv, rep, m, dh).permute(0, 3, 1, 2, 4)[new]
        o = (oc + oo) / total.masked_fill(total == 0, 1.0)
        out.append(o.reshape(T, hq * dh).to(torch.bfloat16))
        a, t = a + size, t + T
    return torch.cat(out)


# ----------------------------------------------------- work and exact values

def work(case):
    hq, hkv, dh = SHAPES[case["family"]]
    page, n, op, width = case["page"], case["n"], case["op"], case["width"]
    sizes, prefix, ctx, q = _lengths(case)
    T, row = sum(q), 2 * hkv * dh * 2                       # K and V bytes of one position
    table = 4 * sum(-(-(c + m) // page) for c, m in zip(ctx, q))
    if op == "bounds":
        pages = sum((c + m) // page - c // page for c, m in zip(ctx, q))
        return {"bytes": pages * hkv * (page * dh * 2 + 2 * dh + 4) + 4 * pages, "flops": pages * hkv * page * dh * 2}
    if op == "select":
        blocks = [c // page for c in ctx]
        return {"bytes": sum(blocks) * hkv * (2 * dh + 4) + T * hq * dh * 2 + T * hkv * n * 4 + table,
                "flops": 4 * dh * hq * sum(b * m for b, m in zip(blocks, q))}
    drafts = [[i // width + 1 if width > 1 else i + 1 for i in range(m)] for m in q]     # new tokens that each one sees
    if op == "shared":
        common = [p // page * page if m > 1 else 0 for p, m in zip(prefix, sizes)]
        each = [p for p, m in zip(common, sizes) for _ in range(m)]
        keys = sum(common) + sum(c - p + m for c, p, m in zip(ctx, each, q))
        seen = sum(m * c + sum(d) for c, m, d in zip(ctx, q, drafts))
        return {"bytes": keys * row + 2 * T * hq * dh * 2 + table, "flops": 4 * dh * hq * seen}
    # Lists of one sequence's tokens may overlap: each of its blocks is needed once.
    keys = seen = 0
    for c, m, d in zip(ctx, q, drafts):
        listed_ = min(n, c // page)
        keys += min(c // page, listed_ * m) * page + c % page + m
        seen += m * (listed_ * page + c % page) + sum(d)
    return {"bytes": keys * row + 2 * T * hq * dh * 2 + T * hkv * n * 4 + table, "flops": 4 * dh * hq * seen}


def _pages_after(s):
    """Pages of each sequence behind the step, on the host."""
    own_pages = [[p for p in r if p >= 0] for r in s["table"].tolist()]
    free = iter([p for p, n in enumerate(s["ref"].tolist()) if n == 0])
    for mine, c, m in zip(own_pages, s["ctx"], s["q_len"]):
        while len(mine) * s["page"] < c + m:
            mine.append(next(free))
    return own_pages


def _two_to(e):
    """2^e in 64 bits, from its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _unit_exact(biggest):
    """The unit of 8-bit values up to `biggest`: 127 of it reach that far, 127 of half of it do not."""
    e = torch.ceil(torch.log2((biggest / 127).clamp(min=2.0 ** -126)))
    e = torch.where(127 * _two_to(e - 1) >= biggest, e - 1, e)
    return _two_to(torch.where(127 * _two_to(e) < biggest, e + 1, e).clamp(min=-126))


def _bounds_exact(keys):
    """lo and hi of keys [h][page][dh] on their grid, and the grid, in 64 bits."""
    k = keys.double()
    unit = _unit_exact(k.abs().flatten(1).max(1)[0])[:, None]
    return torch.floor(k.min(1)[0] / unit) * unit, torch.ceil(k.max(1)[0] / unit) * unit, unit[:, 0]


def _select_exact(s, own_pages):
    """Lists [T][hkv][n] by sorting every block's score."""
    hq, hkv, dh = s["heads"]
    n, page, k = s["case"]["n"], s["page"], s["k"][s["layer"]]
    out, t = torch.full((s["x"].shape[0], hkv, n), -1, dtype=torch.int32), 0
    for r, (c, m) in enumerate(zip(s["ctx"], s["q_len"])):
        f = c // page
        q = s["x"][t:t + m].double().view(m, hq, dh)
        if f:
            lo, hi, _ = _bounds_exact(k[torch.tensor(own_pages[r][:f], device=k.device)].flatten(0, 1))
            lo, hi = lo.view(f, hkv, dh), hi.view(f, hkv, dh)
            unit = _unit_exact(q.abs().max(-1, keepdim=True)[0])
            q = torch.round(q / unit) * unit
            best = torch.full((m, hkv, f), -math.inf, dtype=torch.float64, device=q.device)
            for h in range(hq):
                g = h // (hq // hkv)
                got = torch.where(q[:, h] > 0, q[:, h], 0) @ hi[:, g].T + torch.where(q[:, h] < 0, q[:, h], 0) @ lo[:, g].T
                best[:, g] = torch.maximum(best[:, g], got)
            best[..., [0, f - 1]] = math.inf
            rank = torch.argsort(-best, dim=-1, stable=True)[..., :n]
            out[t:t + m, :, :rank.shape[-1]] = torch.sort(rank, -1)[0].int().cpu()
        t += m
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, dh = s["heads"]
    page, ctx, q, layer, op = s["page"], s["ctx"], s["q_len"], s["layer"], case["op"]
    own_pages = _pages_after(s)
    if op == "bounds":
        values = torch.zeros((s["k"].shape[1], hkv, 2, dh), dtype=torch.float64, device="cuda")
        scales = torch.zeros(values.shape[:2], dtype=torch.float64, device="cuda")
        for mine, c, m in zip(own_pages, ctx, q):
            for p in mine[c // page:(c + m) // page]:
                values[p, :, 0], values[p, :, 1], scales[p] = _bounds_exact(s["k"][layer, p])
        return values, scales
    if op == "select":
        return _select_exact(s, own_pages)
    lists = _select_exact(s, own_pages) if op == "blocks" else None
    out, t = torch.empty(s["x"].shape, dtype=torch.float64, device="cuda"), 0
    rep = hq // hkv
    for r, (c, m) in enumerate(zip(ctx, q)):
        pages = torch.tensor(own_pages[r], device="cuda")
        k, v = (p[layer, pages].transpose(0, 1).reshape(hkv, -1, dh)[:, :c + m].double() for p in (s["k"], s["v"]))
        for lo in range(0, m, 256):
            hi = min(m, lo + 256)
            ok = torch.arange(c + m, device="cuda")[None, :] <= torch.arange(c + lo, c + hi, device="cuda")[:, None]
            if s.get("tree") is not None:
                for i in range(lo, hi):
                    bits = int(s["tree"][t + i]) & ((1 << 64) - 1)
                    ok[i - lo, c:] = torch.tensor([bool(bits >> j & 1) for j in range(m)], device="cuda")
            for g in range(hkv):
                seen = ok
                if lists is not None:                       # blocks before the step: the listed ones alone
                    mask = torch.zeros((hi - lo, c // page + 1), dtype=torch.bool)
                    mask.scatter_(1, lists[t + lo:t + hi, g].long() % (c // page + 1), True)
                    mask[:, -1] = False
                    old = c // page * page
                    seen = ok.clone()
                    seen[:, :old] &= mask[:, :-1].repeat_interleave(page, 1).cuda()
                for h in range(g * rep, (g + 1) * rep):
                    x = s["x"][t + lo:t + hi, h * dh:(h + 1) * dh].double()
                    w = (x @ k[g].T) / math.sqrt(dh)
                    out[t + lo:t + hi, h * dh:(h + 1) * dh] = w.masked_fill(~seen, -math.inf).softmax(-1) @ v[g]
        t += m
    return out
