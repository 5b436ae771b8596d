"""The serving example's model keeps the rules of the adaptive-depth block: who attends, and what a token leaves with."""
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
