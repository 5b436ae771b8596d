"""The serving example with a common prompt read once and with attention over chosen pages."""
import pytest
import torch

from examples.paged_serving import run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("options", [dict(share=True), dict(blocks=4), dict(blocks=3, share=True)])
def test_runs(options):
    r = run(rounds=4, prompts=(400, 37, 130), verbose=False, **options)
    cache, text = r["cache"], r["text"]
    assert r["stats"]["status"] == 0 and len(text) == 4
    # The last token of each text is not in the cache yet.
    assert cache.length.tolist() == [len(t) - 1 for t in text]
    assert text[0][:400] == text[3][:400] and text[0][400] != text[3][400]
    holders = torch.bincount(cache.table[cache.table >= 0].long(), minlength=cache.n_pages)
    assert torch.equal(holders.to(torch.int32), cache.ref)


def test_all_pages_chosen_is_attention():
    """As many blocks as there are pages: the accepted texts are those of plain attention, but for roundings at a
    threshold (which a round's drafts may tip once; the first round's answers stand on the same prompts)."""
    plain, chosen = run(rounds=1, verbose=False), run(rounds=1, verbose=False, blocks=64)
    same = [a[:200] == b[:200] for a, b in zip(plain["text"], chosen["text"])]
    assert all(same) and chosen["stats"]["status"] == 0
