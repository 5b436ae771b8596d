"""What the paged cache's header promises beyond single calls: references held from outside, refused steps, inputs on
other streams."""
import pytest
import torch

from paper_2608_00573_gb300 import binding as B
from tests.test_gpu_cache import DEV

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
