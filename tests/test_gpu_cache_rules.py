"""What the paged cache promises beyond single calls: references held from outside, refused steps, inputs on other
streams, rows of any stride."""
import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.test_gpu_cache import DEV, filled

pytestmark = pytest.mark.gpu


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def rows(c, s):
    """Keys and values of sequence s, all layers."""
    ids = c.table[s, :-(-int(c.length[s]) // c.page)].long()
    return torch.stack([p[:, ids].transpose(1, 2).flatten(2, 3)[:, :, :int(c.length[s])] for p in (c.k, c.v)])


@pytest.mark.parametrize("page,dh", [(16, 64), (64, 128)])
def test_compaction_leaves_pages_held_from_outside(page, dh):
    """ref above the holders in table keeps a page alive where it is: its holder knows it by its index."""
    c = B.PagedCache.empty(2, 40, 4, 2, dh, page, 5, 9, T_max=2000)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    c.step([0, 2], [8 * page, 7 * page + 2])       # pages 0..7, 8..15
    c.fork([2], [3])
    c.step([4], [3 * page])                        # 16..18
    c.step([1], [5 * page - 3])                    # 19..23
    alone = c.table[1, 3:5].clone().long()         # 22, 23: of a sequence that goes
    c.ref[alone] += 1
    c.ref[14] += 2                                 # a page of 2 and 3 too
    c.ref[17] += 1                                 # one of 4 too
    c.truncate([0, 1, 2], [page, 0, 7 * page])     # free: 1..7 and 19..21; 22 and 23 held by the outside alone
    kept = rows(c, 0), rows(c, 2), rows(c, 3), rows(c, 4)
    pool = torch.stack([c.k, c.v])
    held = [14, 17, *alone.tolist()]
    ref = c.ref.clone()
    c.compact()
    st = c.stats()
    assert st["status"] == 0
    assert c.ref[held].tolist() == ref[held].tolist() and int((c.ref > 0).sum()) == int((ref > 0).sum())
    assert torch.equal(torch.stack([c.k, c.v])[:, :, held], pool[:, :, held])
    for s, want in zip((0, 2, 3, 4), kept):
        assert torch.equal(rows(c, s), want), s
    assert (c.table == 14).sum() == 2 and (c.table == 17).sum() == 1
    in_use = (c.ref > 0).nonzero()[:, 0].tolist()                  # the others took the lowest free places
    live = len(in_use)
    assert live == 14 and [p for p in in_use if p >= live] == held
    # released: the next compaction leaves no gap
    c.ref[alone] -= 1
    c.ref[14] -= 2
    c.ref[17] -= 1
    c.compact()
    live = int((c.ref > 0).sum())
    assert (c.ref[:live] > 0).all() and (c.ref[live:] == 0).all()
    for s, want in zip((0, 2, 3, 4), kept):
        assert torch.equal(rows(c, s), want), s
    holders = torch.bincount(c.table[c.table >= 0].long(), minlength=40)
    assert torch.equal(holders.to(torch.int32), c.ref) and c.stats()["status"] == 0


def test_accept_behind_a_refused_step_keeps_the_sequence():
    """A step for drafts that finds no room adds none: an accept queued behind it must not take the tokens of the step
    before (a prompt) for drafts and cut the sequence to a few of them."""
    c = B.PagedCache.empty(2, 10, 4, 2, 64, 16, 3, 7, T_max=200)
    c.k.copy_(torch.randn(c.k.shape, device=DEV))
    c.v.copy_(torch.randn(c.v.shape, device=DEV))
    c.step([0, 1], [100, 20])                      # 7 and 2 of the 10 pages
    k, v, table, length, ref = (t.clone() for t in (c.k, c.v, c.table, c.length, c.ref))
    path = ints([[0, 2, 5], [0, 1, 2]])
    c.step([0, 1], [29, 29])                       # more than max_pages
    c.accept([0, 1], ints([3, 3]), path)
    for now, was in zip((c.k, c.v, c.table, c.length, c.ref), (k, v, table, length, ref)):
        assert torch.equal(now, was)
    # A step that succeeds ends this, for all sequences.
    c.step([2], [5])
    c.accept([2, 1], ints([2, 20]), ints([[1, 4] + [0] * 18, list(range(20))]))
    assert c.length.tolist() == [100, 20, 2]
    st = c.stats(reset=True)
    assert st["status"] == -7 and st["device_error"] == 8
    # So does having been told: the last step that added tokens is the prompt's again.
    c.step([0], [29])
    c.accept([0], ints([2]), path[:1])
    assert c.length.tolist() == [100, 20, 2] and c.stats(reset=True)["device_error"] == 8
    c.accept([0], ints([2]), path[:1])
    assert c.length.tolist() == [2, 20, 2] and c.stats()["status"] == 0


def _busy(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(60_000_000)              # some 30 ms


def test_inputs_live_until_another_stream_has_read_them():
    """Tensors given to a call on another stream may be dropped by the caller right behind it."""
    cache, m, x = filled((8, 2, 64), 16, [100, 300], [40, 50], seed=31, poison=False)
    words = torch.tensor([(1 << i + 1) - 1 for n in (40, 50) for i in range(n)], dtype=torch.int64, device=DEV)
    want = cache.attend(0, x, tree=words)
    qkv = torch.randn((90, 12 * 64), device=DEV).to(torch.bfloat16)
    gammas = [(1 + torch.rand(64, device=DEV)).to(torch.bfloat16) for _ in range(2)]
    pos = torch.arange(90, dtype=torch.int32, device=DEV)
    want_q = cache.append(1, qkv, gamma_q=gammas[0], gamma_k=gammas[1], pos=pos)
    want_k = cache.k.clone()
    st = torch.cuda.Stream()
    torch.cuda.synchronize()

    def dropped(call, *inputs):
        """call on copies that are freed, and whose memory is written again, before the stream gets to it."""
        copies = [t.clone() for t in inputs]
        torch.cuda.synchronize()
        _busy(st)
        result = call(*copies)
        sizes = [(t.shape, t.dtype) for t in copies]
        del copies
        again = [torch.full(shape, 1, dtype=dtype, device=DEV) for shape, dtype in sizes]
        torch.cuda.synchronize()
        del again
        return result

    assert torch.equal(dropped(lambda q, t: cache.attend(0, q, tree=t, stream=st), x, words), want)
    cache.k[1].fill_(0.0)
    got = dropped(lambda a, b, c, d: cache.append(1, a, gamma_q=b, gamma_k=c, pos=d, stream=st), qkv, *gammas, pos)
    assert torch.equal(got, want_q)
    written = cache.k[1] != 0
    assert torch.equal(cache.k[1][written], want_k[1][written]) and int(written.sum()) > 90 * 2 * 60
    before = cache.length.tolist()
    dropped(lambda a, b: cache.accept([0, 1], a, b, stream=st), ints([2, 3]), ints([[0, 4, 9], [1, 2, 7]]))
    assert cache.length.tolist() == [before[0] - 38, before[1] - 47, 0] and cache.stats()["status"] == 0
    cache.step([0, 1], [2, 3])
    out = torch.zeros((5, 512), dtype=torch.bfloat16, device=DEV)      # a result given by the caller
    torch.cuda.synchronize()
    _busy(st)
    cache.attend(0, x[:5], out=out, stream=st)
    at = out.data_ptr()
    del out
    other = torch.full((5, 512), 3.0, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    assert (other == 3).all() and other.data_ptr() != at


def test_the_stride_of_a_single_row_means_nothing():
    """One token's row cut out of a wider buffer, whatever the buffer's width."""
    cache, m, _ = filled((4, 2, 64), 16, [37], [1], seed=33, poison=False)
    wide = torch.randn((3, 1031), device=DEV).to(torch.bfloat16)
    q, qkv = wide[:1, :256], wide[:1, 512:1024]
    assert q.stride(0) == 1031 and q.data_ptr() % 16 == 0
    want = cache.attend(0, q.contiguous())
    assert torch.equal(cache.attend(0, q), want)
    out = torch.zeros((2, 259), dtype=torch.bfloat16, device=DEV)
    cache.attend(0, q, out=out[:1, :256])
    assert torch.equal(out[:1, :256], want) and (out[0, 256:] == 0).all() and (out[1] == 0).all()
    want = cache.append(0, qkv.contiguous())
    assert torch.equal(cache.append(0, qkv), want)
    cache.append(0, qkv, q_out=qkv[:, :256])       # in place
    assert torch.equal(qkv[:, :256], want)
