"""Paged key/value cache and its attention (GPU) against plain restatements in float64."""
import random

import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.cache_helpers import CacheModel, attend_ref, attend_tol, rope_ref, rows_of, scale_of

pytestmark = pytest.mark.gpu

DEV = "cuda"


def filled(shapes, page, ctx, q, layers=2, seed=0, poison=True, spare=7, width=2):
    """A cache whose sequence i holds ctx[i] positions on shuffled pages and has begun a step of q[i] more, with
    random keys and values everywhere (those of the step included); places that no position uses hold NaN."""
    hq, hkv, dh = shapes
    g = torch.Generator(device=DEV).manual_seed(seed)
    n = len(ctx)
    need = [-(-(c + m) // page) for c, m in zip(ctx, q)]
    n_pages = sum(need) + spare
    m = CacheModel(n_pages, n + 1, max(need) + width, page)
    order = torch.randperm(n_pages, generator=g, device=DEV).tolist()
    for s in range(n):
        m.own[s] = [order.pop() for _ in range(-(-ctx[s] // page))]
        m.len[s] = m.base[s] = ctx[s]
        for p in m.own[s]:
            m.ref[p] = 1
    shape = (layers, n_pages, hkv, page, dh)
    k = torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV)
    v = k.clone()
    cache = B.PagedCache(k, v, m.table().to(DEV), torch.tensor(m.len, dtype=torch.int32, device=DEV),
                         torch.tensor(m.ref, dtype=torch.int32, device=DEV), q_heads=hq, T_max=max(1, sum(q)))
    cache.step(range(n), q)
    assert m.step(range(n), q) == []
    for s in range(n):
        for p0 in range(0, m.len[s], page):
            e = min(page, m.len[s] - p0)
            for pool in (k, v):
                pool[:, m.own[s][p0 // page], :, :e] = torch.randn((layers, hkv, e, dh), generator=g, device=DEV).to(
                    torch.bfloat16)
    if not poison:
        k.nan_to_num_(), v.nan_to_num_()
    x = (torch.randn((sum(q), hq * dh), generator=g, device=DEV) * 1.4).to(torch.bfloat16)
    return cache, m, x


def check_attend(cache, m, x, q, out, layer, tree=None, scale=None):
    hq, dh = cache.q_heads, cache.head_dim
    at = 0
    for s, n in enumerate(q):
        kv = m.len[s]
        if n == 0:
            continue
        key = torch.arange(kv, device=DEV)
        if tree is None:
            seen = key[None, :] <= (kv - n + torch.arange(n, device=DEV))[:, None]
        else:
            seen = torch.zeros((n, kv), dtype=torch.bool, device=DEV)
            seen[:, :kv - n] = True
            for i in range(n):
                w = int(tree[at + i])
                for j in range(n):
                    seen[i, kv - n + j] = bool(w >> j & 1)
        rows = random.Random(n).sample(range(n), min(n, 40)) if n > 48 else list(range(n))
        ref, mag = attend_ref(x[at:at + n].view(n, hq, dh)[rows], rows_of(cache.k[layer], m, s, kv),
                              rows_of(cache.v[layer], m, s, kv), seen[rows], scale or scale_of(dh))
        got = out[at:at + n].view(n, hq, dh)[rows].double()
        assert torch.equal(torch.isnan(got), torch.isnan(ref)), s
        fine = torch.isfinite(ref)
        err = torch.where(fine, (got - ref).abs() - attend_tol(ref, mag), -1.0)
        assert float(err.max()) <= 0, (s, float(err.max()), float((got - ref).abs()[fine].max()))
        at += n


CASES = {
    # one token over one, a page, a tile, and around their edges
    "one_token": ((8, 2, 128), 16, [0, 1, 15, 16, 17, 126, 127, 128, 129, 255, 256, 700], [1] * 12),
    "one_token_d64": ((12, 12, 64), 32, [0, 31, 127, 128, 500], [1] * 5),
    "one_sequence_long": ((4, 1, 128), 64, [20000], [1]),
    "one_sequence_long_d64": ((2, 1, 64), 128, [9001], [1]),
    "shared_heads_5": ((10, 2, 128), 64, [300, 0, 77], [3, 30, 25]),
    "shared_heads_7_d64": ((7, 1, 64), 16, [1, 128], [40, 19]),
    "shared_heads_128": ((128, 1, 64), 64, [200, 3], [1, 3]),
    "prompts": ((8, 2, 128), 64, [0, 0, 0, 0], [1, 129, 64, 300]),
    "prompts_mha": ((3, 3, 64), 32, [0, 0, 0], [257, 128, 127]),
    "prompt_behind_prefix": ((8, 2, 128), 128, [1000, 127, 128, 5], [200, 65, 64, 1]),
    "prompt_long": ((4, 2, 128), 64, [0], [2500]),
    "mixed": ((8, 2, 64), 16, [400, 0, 900, 33], [1, 700, 1, 8]),
    "some_without_tokens": ((8, 2, 128), 64, [100, 50, 0, 64], [1, 0, 0, 130]),
    "many": ((4, 4, 64), 16, [(i * 37) % 300 for i in range(200)], [1 + (i % 3 == 0) for i in range(200)]),
}


@pytest.mark.parametrize("name", CASES)
def test_attend(name):
    shapes, page, ctx, q = CASES[name]
    cache, m, x = filled(shapes, page, ctx, q)
    for layer in (0, 1):
        out = cache.attend(layer, x)
        check_attend(cache, m, x, q, out, layer)
    assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page", [((8, 2, 128), 64), ((6, 6, 64), 16), ((40, 5, 128), 32)])
def test_attend_tree(shapes, page):
    ctx, q = [0, 127, 300, 100, 64, 1000], [17, 64, 1, 40, 64, 33]
    cache, m, x = filled(shapes, page, ctx, q, seed=3)
    rng = random.Random(5)
    words = []
    for n in q:
        parent = [rng.randint(-1, i - 1) if i else -1 for i in range(n)]
        for i in range(n):
            w, j = 0, i
            while j >= 0:
                w |= 1 << j
                j = parent[j]
            words.append(w)
    words[2] = 0                                   # first sequence, no prefix: sees nothing
    words[5] = 1 << 9                              # only a later token
    words[sum(q[:3])] = (1 << 64) - 1              # bits past the drafts
    words[sum(q[:4])] = 0                          # the prefix alone
    tree = torch.tensor([w - (1 << 64) if w >> 63 else w for w in words], dtype=torch.int64, device=DEV)
    out = cache.attend(1, x, tree=tree)
    check_attend(cache, m, x, q, out, 1, tree=words)
    assert torch.count_nonzero(out[2]) == 0


@pytest.mark.parametrize("shapes", [(8, 2, 128), (4, 4, 64)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_masked_places_may_hold_anything(shapes, bad):
    """Keys and values of later tokens and of other branches: not finite, results as without them."""
    page, ctx, q = 32, [100, 0, 500], [150, 140, 9]
    cache, m, x = filled(shapes, page, ctx, q, seed=7)
    for s, p in ((0, 200), (1, 100), (2, 505)):
        a, b = m.row(s, p)
        cache.v[1, a, :, b, 3:] = bad
        cache.k[1, a, :, b] = bad
    out = cache.attend(1, x)
    at = 0
    for s, n in enumerate(q):
        own = {0: 200, 1: 100, 2: 505}[s] - ctx[s]
        assert torch.isfinite(out[at:at + own].float()).all(), s          # tokens before it
        at += n
    early = [own for own in (100, 100, 5)]
    at = 0
    for s, n in enumerate(q):
        kv = ctx[s] + early[s]
        ref, mag = attend_ref(x[at:at + early[s]].view(early[s], *shapes[::2]), rows_of(cache.k[1], m, s, kv),
                              rows_of(cache.v[1], m, s, kv),
                              torch.arange(kv, device=DEV)[None] <= (ctx[s] + torch.arange(early[s], device=DEV))[:, None],
                              scale_of(shapes[2]))
        got = out[at:at + early[s]].view(early[s], *shapes[::2]).double()
        assert ((got - ref).abs() <= attend_tol(ref, mag)).all(), s
        at += n


def test_unmasked_infinity_reaches_its_rows_only():
    cache, m, x = filled((4, 2, 64), 16, [10], [40], seed=9)
    a, b = m.row(0, 30)
    cache.v[0, a, 0, b, 5] = float("inf")
    out = cache.attend(0, x).view(40, 4, 64).float()
    hit = ~torch.isfinite(out)
    want = torch.zeros_like(hit)
    want[20:, :2, 5] = True
    assert torch.equal(hit, want)


def test_scale_strides_and_side_stream():
    q = [5, 130]
    cache, m, x = filled((8, 2, 128), 64, [60, 200], q, seed=11)
    wide = torch.full((135, 1024 + 40), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:1032] = x
    out = torch.full((135, 2048), 7.0, dtype=torch.bfloat16, device=DEV)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    res = cache.attend(0, wide[:, 8:1032], out=out[:, 512:1536], scale=0.05, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert res.data_ptr() == out[:, 512:].data_ptr()
    check_attend(cache, m, x, q, out[:, 512:1536], 0, scale=0.05)
    assert (out[:, :512] == 7).all() and (out[:, 1536:] == 7).all()


def test_repeated_calls_are_bitwise_equal():
    q = [1, 400, 1, 64]
    cache, m, x = filled((8, 2, 128), 16, [9000, 100, 3333, 2000], q, seed=13)
    first = cache.attend(0, x)
    for _ in range(3):
        assert torch.equal(cache.attend(0, x), first)


def test_extreme_scores():
    """Scores far apart (the running maximum grows by more than 2^8) and a row whose first keys are negligible."""
    cache, m, x = filled((4, 1, 128), 64, [700], [130], seed=15)
    cache.k *= (1 + 30 * torch.rand(cache.k.shape[:4], device=DEV))[..., None].to(torch.bfloat16)
    out = cache.attend(1, x)
    # scores up to ~500: fp32 sums of 128 products are off by up to 2^-17 of them, so p by 2^-8
    at, n, kv = 0, 130, 830
    seen = torch.arange(kv, device=DEV)[None] <= (700 + torch.arange(n, device=DEV))[:, None]
    ref, mag = attend_ref(x.view(n, 4, 128), rows_of(cache.k[1], m, 0, kv), rows_of(cache.v[1], m, 0, kv), seen,
                          scale_of(128))
    assert ((out.view(n, 4, 128).double() - ref).abs() <= attend_tol(ref, mag) + mag * 2.0 ** -8).all()


@pytest.mark.parametrize("shapes", [(8, 2, 128), (12, 12, 64), (5, 1, 128), (7, 7, 64)])
@pytest.mark.parametrize("norm,theta,given", [(True, 1e6, False), (False, 1e4, False), (True, 0.0, False),
                                              (False, 0.0, False), (True, 1e6, True)])
def test_append(shapes, norm, theta, given):
    hq, hkv, dh = shapes
    q = [1, 0, 130, 7]
    cache, m, x = filled(shapes, 16, [33, 5, 0, 4000], q, seed=17)
    T, H = sum(q), hq + 2 * hkv
    wide = torch.randn((T, H * dh + 24), device=DEV).to(torch.bfloat16)
    qkv = wide[:, 16:16 + H * dh]
    gq, gk = ((1 + 0.2 * torch.randn(dh, device=DEV)).to(torch.bfloat16) for _ in range(2)) if norm else (None, None)
    place = torch.cat([torch.arange(c, c + n) for c, n in zip([33, 5, 0, 4000], q)]).to(DEV)
    pos = torch.randint(0, 1 << 30, (T,), device=DEV, dtype=torch.int32) if given else None
    k0, v0 = cache.k.clone(), cache.v.clone()
    src = qkv.clone()
    out = cache.append(1, qkv, gamma_q=gq, gamma_k=gk, eps=1e-5, theta=theta, pos=pos)
    y = src.view(T, H, dh)
    at = place if pos is None else pos
    want_q = rope_ref(y[:, :hq], at, gq, 1e-5, theta).view(T, hq * dh)
    want_k = rope_ref(y[:, hq:hq + hkv], at, gk, 1e-5, theta)
    # rounding to bf16 once (2^-8), fp32 norm and rotation of two terms (2^-20 of the pair)
    size = y[:, :hq].double().abs().amax() * (2 if norm else 1)
    assert ((out.double() - want_q).abs() <= want_q.abs() * 2.0 ** -8 + size * 2.0 ** -19).all()
    t = 0
    for s, n in enumerate(q):
        for i in range(n):
            a, b = m.row(s, m.len[s] - n + i)
            assert ((cache.k[1, a, :, b].double() - want_k[t]).abs() <= want_k[t].abs() * 2.0 ** -8 + size * 2.0 ** -19).all()
            assert torch.equal(cache.v[1, a, :, b], y[t, hq + hkv:])
            k0[1, a, :, b], v0[1, a, :, b] = cache.k[1, a, :, b], cache.v[1, a, :, b]
            t += 1
    bits = lambda z: z.view(torch.int16)                               # noqa: E731
    assert torch.equal(bits(cache.k), bits(k0)) and torch.equal(bits(cache.v), bits(v0))   # nothing else written
    # in place
    cache.append(1, qkv, q_out=qkv[:, :hq * dh], gamma_q=gq, gamma_k=gk, eps=1e-5, theta=theta, pos=pos)
    assert torch.equal(qkv[:, :hq * dh], out) and torch.equal(qkv[:, hq * dh:], src[:, hq * dh:])


@pytest.mark.parametrize("page,dh,seed", [(16, 64, 1), (64, 128, 2), (32, 128, 3), (128, 64, 4)])
def test_bookkeeping_of_random_programs(page, dh, seed):
    """Steps, forks, cuts, accepted drafts and compaction in random order: tables, lengths, counts and every stored row
    as the plain model gives them, refused calls included."""
    rng = random.Random(seed)
    layers, hkv, n_pages, seqs, max_pages = 3, 2, 61, 9, 20
    c = B.PagedCache.empty(layers, n_pages, 2 * hkv, hkv, dh, page, seqs, max_pages, T_max=4000)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    k, v = c.k.cpu(), c.v.cpu()
    m = CacheModel(n_pages, seqs, max_pages, page)
    refused = 0
    for _ in range(120):
        what = rng.choice(["step", "step", "step", "fork", "cut", "accept", "compact"])
        some = rng.sample(range(seqs), rng.randint(1, seqs))
        if what == "step":
            q = [rng.choice([0, 1, 1, 7, page, 3 * page + 1]) for _ in some]
            c.step(some, q)
            copies = m.step(some, q)
            if copies is None:
                refused += 1
                st = c.stats(reset=True)
                assert st["device_error"] == 8 and st["status"] == -7
            else:
                for a, b in copies:
                    k[:, b], v[:, b] = k[:, a], v[:, a]
        elif what == "fork" and len(some) > 1:
            src = [rng.choice(some[:1]) for _ in some[1:]]
            c.fork(src, some[1:])
            m.fork(src, some[1:])
        elif what == "cut":
            to = [rng.choice([0, m.len[s] // 2, m.len[s], m.len[s] + 5]) for s in some]
            c.truncate(some, to)
            m.truncate(some, to)
        elif what == "accept":
            depth = rng.randint(1, 9)
            n_acc, path = [], []
            for s in some:
                d = m.len[s] - m.base[s]
                n = rng.randint(0, min(depth, d)) if d else 0
                p = sorted(rng.sample(range(d), n)) + [-1] * (depth - n)
                if rng.random() < 0.1:
                    n, p = depth, [d + 3] * depth
                n_acc.append(n)
                path.append(p)
            c.accept(some, torch.tensor(n_acc, dtype=torch.int32, device=DEV),
                     torch.tensor(path, dtype=torch.int32, device=DEV))
            moves = m.accept(some, n_acc, path)
            for mv in moves:
                for a, b in mv or []:
                    k[:, b[0], :, b[1]], v[:, b[0], :, b[1]] = k[:, a[0], :, a[1]], v[:, a[0], :, a[1]]
            if None in moves:
                refused += 1
                assert c.stats(reset=True)["device_error"] == 10
        elif what == "compact":
            c.compact()
            for a, b in m.compact().items():
                k[:, b], v[:, b] = k[:, a], v[:, a]
        assert torch.equal(c.table.cpu(), m.table()), what
        assert c.length.tolist() == m.len and c.ref.tolist() == m.ref, what
    assert torch.equal(c.k.cpu(), k) and torch.equal(c.v.cpu(), v)
    st = c.stats()
    assert st["status"] == 0 and st["free_pages"] == sum(r == 0 for r in m.ref) and refused


def test_refused_step_leaves_everything():
    c = B.PagedCache.empty(1, 4, 2, 1, 64, 16, 3, 8, T_max=200)
    c.step([0, 1], [20, 20])
    c.append(0, torch.ones((40, 256), dtype=torch.bfloat16, device=DEV))
    x = torch.ones((90, 128), dtype=torch.bfloat16, device=DEV)
    c.step([2, 0], [60, 30])                        # 7 pages wanted, none free
    out = torch.full((90, 128), 3.0, dtype=torch.bfloat16, device=DEV)
    c.attend(0, x, out=out)
    c.append(0, torch.ones((90, 256), dtype=torch.bfloat16, device=DEV), q_out=out)
    assert c.length.tolist() == [20, 20, 0] and c.ref.tolist() == [1] * 4 and (out == 3).all()
    st = c.stats(reset=True)
    assert st["device_error"] == 8
    c.truncate([1], [0])
    c.step([0], [12])
    c.append(0, torch.ones((12, 256), dtype=torch.bfloat16, device=DEV))
    assert torch.isfinite(c.attend(0, x[:12]).float()).all() and c.stats()["status"] == 0


def test_pool_past_32_bit_offsets():
    """Pages whose element offsets pass 2^31 and 2^32 in the pool."""
    layers, n_pages, hkv, page, dh = 2, 21000, 8, 128, 128
    k = torch.zeros((layers, n_pages, hkv, page, dh), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    assert k[0].numel() > 1 << 31 and k.numel() > 1 << 32
    table = torch.full((2, 4), -1, dtype=torch.int32, device=DEV)
    ids = [20999, 16500, 3]
    table[0, :3] = torch.tensor(ids, dtype=torch.int32)
    ref = torch.ones(n_pages, dtype=torch.int32, device=DEV)
    ref[20000] = 0
    length = torch.tensor([300, 0], dtype=torch.int32, device=DEV)
    c = B.PagedCache(k, v, table, length, ref, q_heads=8, T_max=200)
    for i in ids + [20000]:
        k[1, i] = torch.randn((hkv, page, dh), device=DEV).to(torch.bfloat16)
        v[1, i] = torch.randn((hkv, page, dh), device=DEV).to(torch.bfloat16)
    c.step([0], [130])                              # 84 on the last page, 46 on page 20000
    qkv = torch.randn((130, 24 * dh), device=DEV).to(torch.bfloat16)
    x = c.append(1, qkv, theta=0.0)
    m = CacheModel(n_pages, 2, 4, page)
    m.own[0], m.len = ids + [20000], [430, 0]
    assert torch.equal(v[1, 20000, :, 45], qkv[129, 16 * dh:].view(8, dh))
    out = c.attend(1, x)
    check_attend(c, m, x, [130], out, 1)
    ref[16500] += 1                                 # a shared last page of another sequence
    c.truncate([0], [200])
    c.step([0], [1])
    assert ref[16500] == 1 and int(table[0, 1]) in (3, 20000, 20999)
    to = int(table[0, 1])
    assert torch.equal(k[1, to], k[1, 16500]) and torch.equal(v[1, to], v[1, 16500])
    assert c.stats()["status"] == 0


def test_graph_replays_follow_the_lengths():
    """A captured step + append + attend, replayed: every replay sees one more token."""
    hq, hkv, dh = 8, 2, 128
    c = B.PagedCache.empty(1, 40, hq, hkv, dh, 16, 3, 20, T_max=300)
    c.k.fill_(float("nan"))
    c.v.fill_(float("nan"))
    m = CacheModel(40, 3, 20, 16)
    c.step([0, 1, 2], [50, 1, 120])
    m.step([0, 1, 2], [50, 1, 120])
    c.append(0, torch.randn((171, 12 * dh), device=DEV).to(torch.bfloat16))
    qkv = torch.zeros((3, 12 * dh), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros((3, hq * dh), dtype=torch.bfloat16, device=DEV)
    x = torch.zeros_like(out)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        c.step([0, 1, 2], [1, 1, 1])
        c.append(0, qkv, q_out=x)
        c.attend(0, x, out=out)
    for _ in range(20):
        qkv.copy_(torch.randn(qkv.shape, device=DEV))
        graph.replay()
        m.step([0, 1, 2], [1, 1, 1])
        check_attend(c, m, x, [1, 1, 1], out, 0)
    assert c.length.tolist() == m.len and c.stats()["status"] == 0


def test_refusals():
    mk = lambda **o: B.PagedCache.empty(**{**dict(layers=1, n_pages=8, q_heads=4, kv_heads=2, head_dim=64, page=16,  # noqa: E731
                                                  max_seqs=3, max_pages=4, T_max=100), **o})
    for bad, status in ((dict(q_heads=5), -1), (dict(head_dim=96), -2), (dict(page=48), -2), (dict(page=256), -2),
                        (dict(max_seqs=1025), -2), (dict(q_heads=258), -2), (dict(T_max=0), -1)):
        with pytest.raises(B.TrimmoeError) as e:
            mk(**bad)
        assert e.value.status == status, bad
    c = mk()
    x = torch.zeros((10, 256), dtype=torch.bfloat16, device=DEV)
    with pytest.raises(B.TrimmoeError, match="no step"):
        c.attend(0, x[:0])
    for args in (([3], [1]), ([-1], [1]), ([0, 0], [1, 1]), ([0], [-1]), ([0], [101]), ([0, 1], [1]),
                 ([0, 1, 2, 0], [1] * 4)):
        with pytest.raises(B.TrimmoeError):
            c.step(*args)
    c.step([0, 2], [4, 6])
    ok = dict(layer=0, q=x)
    for bad in (dict(layer=1), dict(layer=-1), dict(q=x[:9]), dict(q=x.float()), dict(q=x.cpu()), dict(scale=-1.0),
                dict(scale=float("nan")), dict(q=torch.zeros((10, 257), dtype=torch.bfloat16, device=DEV)[:, 1:]),
                dict(tree=torch.zeros(9, dtype=torch.int64, device=DEV)),
                dict(tree=torch.zeros(10, dtype=torch.int32, device=DEV)), dict(out=x.t())):
        with pytest.raises(B.TrimmoeError):
            c.attend(**{**ok, **bad})
    qkv = torch.zeros((10, 512), dtype=torch.bfloat16, device=DEV)
    g = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    for bad in (dict(layer=1), dict(gamma_q=g), dict(gamma_q=g, gamma_k=g, eps=-1.0), dict(theta=0.5),
                dict(theta=float("inf")), dict(gamma_q=g[:32], gamma_k=g), dict(qkv=qkv[:, :511]),
                dict(pos=torch.zeros(10, dtype=torch.int64, device=DEV))):
        with pytest.raises(B.TrimmoeError):
            c.append(**{**dict(layer=0, qkv=qkv), **bad})
    for src, dst in (([0], [0]), ([0, 1], [1, 2]), ([0, 0], [1, 1]), ([5], [1]), ([0], [7])):
        with pytest.raises(B.TrimmoeError):
            c.fork(src, dst)
    with pytest.raises(B.TrimmoeError):
        c.truncate([0], [-1])
    with pytest.raises(B.TrimmoeError):
        c.accept([0], torch.zeros(2, dtype=torch.int32, device=DEV), torch.zeros((1, 1), dtype=torch.int32, device=DEV))
    c.step([1], [70 - 6])                          # 64 tokens fit a tree, one page more does not fit the row
    c.attend(0, torch.zeros((64, 256), dtype=torch.bfloat16, device=DEV),
             tree=torch.zeros(64, dtype=torch.int64, device=DEV))
    assert c.stats()["status"] == 0
    c.truncate([1], [0])
    c2 = mk(max_pages=8)
    c2.step([0], [65])
    with pytest.raises(B.TrimmoeError, match="64 tokens"):
        c2.attend(0, torch.zeros((65, 256), dtype=torch.bfloat16, device=DEV),
                  tree=torch.zeros(65, dtype=torch.int64, device=DEV))
    c.step([0], [0])
    c.step([1], [10])
    c.fork([0], [1])                               # ends the step
    with pytest.raises(B.TrimmoeError, match="no step"):
        c.attend(0, x)


def test_nothing_to_do():
    c = B.PagedCache.empty(1, 8, 4, 2, 64, 16, 3, 4, T_max=10)
    c.step([], [])
    e = lambda n: torch.zeros((0, n), dtype=torch.bfloat16, device=DEV)        # noqa: E731
    assert c.append(0, e(512)).shape == (0, 256) and c.attend(0, e(256)).shape == (0, 256)
    c.step([0, 1], [0, 0])
    assert c.attend(0, e(256)).shape == (0, 256)
    c.fork([], [])
    c.truncate([], [])
    c.compact()
    assert c.length.tolist() == [0, 0, 0] and c.stats() == dict(status=0, device_error=0, free_pages=8,
                                                                launches=c.stats()["launches"])


def test_serving_example():
    """The example's loop: drafted rounds leave the cache that the accepted texts alone would, and attention over it gives
    what a fresh prefill of the same text gives."""
    from examples.paged_serving import run
    r = run(rounds=4, verbose=False)
    c, text = r["cache"], r["text"]
    assert r["stats"]["status"] == 0 and r["engine"].stats()["device_error"] == 0
    assert c.length.tolist() == [len(t) - 1 for t in text]       # all but the last token is in the cache
    assert r["accepted"] > 0
    held = sum(-(-n // c.page) for n in c.length.tolist()) - 200 // c.page    # full pages of the forked prompt are shared
    assert r["stats"]["free_pages"] == c.n_pages - held
    # The first layer's keys depend on tokens and positions only: those of sequence 1, written round by round, equal a
    # fresh prefill's up to the rounding of another batch's projection.
    n = int(c.length[1])
    got = c.k[0][c.table[1, :-(-n // c.page)].long()].transpose(0, 1).reshape(c.kv_heads, -1, c.head_dim)[:, :n].clone()
    c.truncate([1], [0])
    c.step([1], [n])
    r["model"](torch.tensor(text[1][:n], device=DEV))
    want = c.k[0][c.table[1, :-(-n // c.page)].long()].transpose(0, 1).reshape(c.kv_heads, -1, c.head_dim)[:, :n]
    assert ((got.float() - want.float()).abs() <= 2.0 ** -6 * want.float().abs().amax()).all()


def test_append_without_rotation_keeps_infinities():
    c = B.PagedCache.empty(1, 4, 2, 1, 64, 16, 1, 4, T_max=4)
    c.step([0], [3])
    qkv = torch.randn((3, 256), device=DEV).to(torch.bfloat16)
    qkv[1, 5], qkv[2, 130] = float("inf"), float("-inf")
    out = c.append(0, qkv, theta=0.0)
    assert torch.equal(out, qkv[:, :128])
    assert torch.equal(c.k[0, int(c.table[0, 0]), 0, :3], qkv[:, 128:192])


def test_calls_follow_the_given_stream():
    """Work queued on a stream of its own sees what that stream did before it."""
    c = B.PagedCache.empty(1, 64, 4, 2, 64, 16, 2, 32, T_max=300)
    c.k.zero_(), c.v.zero_()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        big = torch.randn((4096, 4096), device=DEV)
        for _ in range(20):
            big = big @ big * 1e-3
        qkv = torch.randn((300, 512), device=DEV).to(torch.bfloat16) + (big.sum() * 0).to(torch.bfloat16)
        c.step([0, 1], [200, 100])
        x = c.append(0, qkv)
        out = c.attend(0, x)
    m = CacheModel(64, 2, 32, 16)
    m.step([0, 1], [200, 100])
    torch.cuda.current_stream().wait_stream(st)
    check_attend(c, m, x, [200, 100], out, 0)


def test_groups_that_end_before_their_sequence():
    """Short steps count key tiles to the sequence's end; where a group's own tokens end a tile earlier, a CTA's share may
    hold nothing but that tile."""
    shapes, page = (16, 1, 64), 16                       # 8 tokens a query tile, groups of 16 tokens
    for ctx in ([128 * k - 33 for k in range(1, 12)], [128 * k - 20 for k in range(1, 40, 3)]):
        q = [64 - (i % 3) for i in range(len(ctx))]
        cache, m, x = filled(shapes, page, ctx, q, seed=len(ctx))
        out = cache.attend(0, x)
        check_attend(cache, m, x, q, out, 0)
        assert cache.stats()["device_error"] == 0


@pytest.mark.parametrize("shapes,page", [((32, 8, 128), 64), ((12, 12, 64), 16), ((8, 1, 64), 128)])
def test_a_single_seen_key_gives_its_value(shapes, page):
    """The only key's probability is 1, which bf16 holds, so the value comes back bit for bit: first tokens of prompts,
    single tokens without context, drafts that see only themselves."""
    hq, hkv, dh = shapes
    for q, tree in (([1, 300, 1, 5, 1], False), ([1, 64, 3], True)):
        cache, m, x = filled(shapes, page, [0] * len(q), q, seed=sum(q))
        mask = torch.tensor([1 << j for n in q for j in range(n)], dtype=torch.uint64).view(torch.int64) if tree else None
        out = cache.attend(0, x * 3, tree=None if mask is None else mask.to(DEV))
        at = 0
        for s, n in enumerate(q):
            rows = n if tree else 1
            v = rows_of(cache.v[0], m, s, rows).transpose(0, 1).repeat_interleave(hq // hkv, 1)
            assert torch.equal(out[at:at + rows].view(rows, hq, dh), v), (s, tree)
            at += n
        assert cache.stats()["device_error"] == 0
