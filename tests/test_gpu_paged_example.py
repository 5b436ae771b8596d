"""The serving example's model keeps the rules of the adaptive-depth block: who attends, what a token leaves with, and
that its decisions do not hang on its place in the step."""
import numpy as np
import pytest
import torch

from examples.paged_serving import Model
from paper_2608_00573_gb300 import binding as B
from paper_2608_00573_gb300 import workload as W

pytestmark = pytest.mark.gpu

SEQS = (200, 70, 131)


def small_model(seed=5):
    """A model whose tokens exit (half of those asked at a layer) and skip."""
    cfg = W.WorkloadConfig(name="paged", N=5, d=512, E=8, k=2, F=256, C=1, M=6, H=3, act=W.ACT_SWIGLU, T=512, seed=seed)
    calib = dict(exit_bias=[2.2] * cfg.N, theta=[0.45] * cfg.N)
    small = W.make_small_weights(cfg, calib=calib)
    engine = B.Engine(cfg, W.make_tables(cfg, small["W_r"], calib=calib), small, W.make_expert_weights_host(cfg), T_max=512)
    cache = B.PagedCache.empty(cfg.N, 64, 8, 2, 64, 16, len(SEQS), 20, T_max=512)
    return Model(cfg, 8, 2, 64, 200, cache, engine, seed)


class Watched:
    """Stands before the model's cache and engine and keeps the states that enter and leave each layer."""

    def __init__(self, model):
        self.cache, self.engine, self.layers = model.cache, model.engine, []
        model.cache = model.engine = self

    def tokens_to_device(self, tok):
        self.tok = self.engine.tokens_to_device(tok)
        return self.tok

    def state(self):
        return self.tok["hidden"].clone(), self.tok["alive"].bool()

    def append(self, *a, **kw):
        self.layers.append([self.state()])
        return self.cache.append(*a, **kw)

    def attend(self, *a, **kw):
        return self.cache.attend(*a, **kw)

    def layer_step(self, *a, **kw):
        self.engine.layer_step(*a, **kw)


def test_exited_tokens_keep_their_state():
    """Attention runs for live tokens; a token that exits at a layer leaves with the state that entered it."""
    m = small_model()
    w = Watched(m)
    w.cache.step(range(len(SEQS)), SEQS)
    m(torch.from_numpy(np.random.default_rng(3).integers(0, 200, sum(SEQS))).cuda())
    after = [entry[0] for entry in w.layers[1:]] + [w.state()]
    gone = 0
    for (before, live), (hidden, alive) in zip((entry[0] for entry in w.layers), after):
        assert not (alive & ~live).any()
        gone += int((~alive).sum())
        assert torch.equal(hidden[~alive], before[~alive])
        assert (hidden[alive] != before[alive]).any(1).all()
    assert 0 < int((~w.state()[1]).sum()) < sum(SEQS) and gone > 100
    assert w.cache.stats()["status"] == 0


def test_decisions_do_not_depend_on_the_place_in_the_step():
    """The same prompts listed in another order: every token starts from its own sequence's access server, so exits,
    substitutions and next tokens are the same, but for roundings at a threshold (scores, gates and confidences
    move by 2^-8 of themselves in each of five layers; a tenth of the tokens is far more than can sit that close)."""
    m = small_model()
    w = Watched(m)
    rng = np.random.default_rng(3)
    text, servers = [rng.integers(0, 200, n) for n in SEQS], [1, 4, 2]
    found = []
    for order in ([0, 1, 2], [2, 0, 1]):
        w.cache.truncate(order, [0] * 3)
        w.cache.step(order, [SEQS[s] for s in order])
        following = m(torch.from_numpy(np.concatenate([text[s] for s in order])).cuda(),
                      server=torch.tensor(np.repeat([servers[s] for s in order], [SEQS[s] for s in order])).cuda())
        parts = [torch.stack([following, w.tok["exit_layer"].long(), w.tok["s"].long()]).split([SEQS[s] for s in order], 1)]
        found.append({s: p for s, p in zip(order, parts[0])})
    same = torch.cat([(found[0][s] == found[1][s]).all(0) for s in range(3)])
    assert float(same.float().mean()) >= 0.9, float(same.float().mean())
