"""Attention of chunks over sequences whose pages have left from the middle (trr_evict), were moved (trr_compact), and went on:
against the definition over what is still stored."""
import numpy as np
import pytest
import torch

from _shared import model_evict, snapshot
from test_gpu_chunk import LAYOUTS, check, fill, holder

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    torch.cuda.set_device(0)


def evict(h, seqs, keep_from, sinks):
    """Evicts on the GPU and takes the tokens that leave, by the model, from what the sequences should hold."""
    gone = model_evict(snapshot(h), h, seqs, keep_from, sinks)
    h.gpu.evict(h.ints(seqs), h.ints(keep_from), sinks)
    assert h.gpu.status() == 0
    for (layer, s), positions in gone.items():
        for p in positions:
            del h.tokens[layer][s][p]
    return gone


@pytest.mark.parametrize("lay", LAYOUTS)
@pytest.mark.parametrize("sinks", [0, 3, 40])
def test_local_and_full_queries_after_evictions(lay, sinks):
    """A stream: evicted twice, appended to between and after, closed up; windows that end before, in and behind the gap, and
    full queries that see what is left on both sides of it."""
    rng = np.random.default_rng([1, sinks])
    h = holder(lay, S=3, maxctx=1200)
    for s, n in ((0, 700), (2, 500)):
        fill(h, rng, 0, s, n)
    fill(h, rng, 0, 1, 300)
    assert evict(h, [0, 2], [430, 300], sinks) or lay["P"] == 64  # (whose pages may all reach out of the gap)
    new = 120

    def chunks(ends):
        n = 3 * new
        check(h, rng, [0, 2, 1], [e - new for e in ends], [new] * 3, rng.choice(3, n, p=[0.1, 0.5, 0.4]), rng.integers(1, 400, n), sinks)

    chunks([700, 500, 300])
    h.append(rng, 0, 0, np.arange(700, 840))
    chunks([840, 500, 300])
    assert evict(h, [0], [690], sinks) or lay["P"] == 64
    h.gpu.compact()
    assert h.gpu.status() == 0
    chunks([840, 500, 300])
    h.append(rng, 0, 0, np.arange(840, 1001))
    h.append(rng, 0, 2, np.arange(500, 533))
    chunks([1001, 533, 300])


@pytest.mark.parametrize("lay", [LAYOUTS[0], LAYOUTS[2]])
def test_queries_within_the_gap(lay):
    """Chunks whose own positions have been evicted, with sinks kept and without: what is left below them, or nothing."""
    rng = np.random.default_rng(2)
    for sinks in (0, 5):
        h = holder(lay, S=2, maxctx=900)
        fill(h, rng, 0, 1, 800)
        evict(h, [1], [760], sinks)
        n = 300
        check(h, rng, [1, 1], [100, 600], [100, 200], rng.choice(3, n), rng.integers(1, 300, n), sinks)
