"""The example that runs the cache's operators together with the linear layers, and the property its caches have to have:
what the cache serves step by step is what one pass over the whole stream computes."""
import importlib.util
import os

import pytest
import torch

import paper_2503_13565_b200 as mxq

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("cached_speculation", os.path.join(ROOT, "examples", "cached_speculation.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    return mod


def test_the_example_runs(example):
    stream, tally, shared, path = example.main(40)
    assert len(stream) >= 40 and all(0 <= t < example.VOCAB for t in stream)
    assert tally.proposed[0] == 4 * tally.steps[0] and len(stream) == tally.accepted[0] + tally.steps[0]
    assert shared >= 1 and len(path) >= 2        # the first branch starts with the model's own token


def test_step_by_step_equals_one_pass(example):
    """Twelve tokens one by one, in blocks with a rollback in between, and in one pass of twelve rows: the same hidden states up
    to what the order of the sums and BF16's rounding of the activations may change, and the same bytes in layer 0 of the cache
    (whose K and V do not depend on attention) wherever the projection's BF16 outputs agree."""
    w = example.Weights(3)
    toks = [5, 900, 17, 44, 1234, 8, 8, 1999, 0, 77, 321, 6]
    one, step, roll = (example.CachedModel(w, example.LAYERS) for _ in range(3))
    one.resize(0, len(toks))
    whole = one.forward(toks).float()
    rows = []
    for i, t in enumerate(toks):
        step.resize(0, i + 1)
        rows.append(step.forward([t]).float())
    steps = torch.cat(rows)
    roll.resize(0, 5)
    roll.forward(toks[:5])
    roll.resize(0, 9)
    roll.forward([1, 2, 3, 4])                     # four rows that are not kept
    roll.resize(0, 5)
    roll.resize(0, len(toks))
    back = roll.forward(toks[5:]).float()
    # a BF16 activation carries 2^-9 of itself per rounding; some tens of roundings on the way through three layers
    scale = whole.abs().max()
    assert (steps - whole).abs().max() <= 2.0 ** -4 * scale and (back - whole[5:]).abs().max() <= 2.0 ** -4 * scale
    k1, v1 = mxq.mxq_kv_read(one.cache, 0, one.tables[:1], one.lens[:1], len(toks))
    k2, v2 = mxq.mxq_kv_read(step.cache, 0, step.tables[:1], step.lens[:1], len(toks))
    for x, y in ((k1, k2), (v1, v2)):
        same = (x == y).float().mean()
        assert same > 0.98 and (x.float() - y.float()).abs().max() <= 0.5 * x.float().abs().max()
