"""What the generator over pages refuses on the host (no GPU)."""
from types import SimpleNamespace

import numpy as np
import pytest

torch = pytest.importorskip("torch")
from paper_2607_24841_amd import generate as G  # noqa: E402


def bare(n=3, block=8, limit=100, max_rows=256, ctx=(), live=()):
    """A generator's host state; a plan that is asked for ends the test."""
    g = G.PagedGenerator.__new__(G.PagedGenerator)
    g.block, g.n, g.limit, g.n_sel = block, n, limit, -1
    g.ctx, g.live = np.zeros(n, dtype=np.int32), np.zeros(n, dtype=bool)
    g.ctx[:len(ctx)], g.live[:len(live)] = ctx, live
    g.pages, g.prompt_pages = SimpleNamespace(max_rows=n * block), SimpleNamespace(max_rows=max_rows)

    def plan(pages, new):
        raise AssertionError("planned")
    g._plan = plan
    return g


def test_requests_past_their_last_position():
    ids = lambda n: np.ones(n, np.int32)  # noqa: E731
    with pytest.raises(ValueError, match="request 1"):
        bare().admit({0: ids(100), 1: ids(101)})
    with pytest.raises(AssertionError, match="planned"):
        bare().admit({0: ids(100), 1: ids(100)})
    with pytest.raises(ValueError, match="request 2"):
        bare(ctx=(92, 0, 93), live=(1, 0, 1)).run_block(1, 1)
    for live in ((1, 0, 0), (1, 1, 0)):      # up to the last one; released requests do not count
        with pytest.raises(AssertionError, match="planned"):
            bare(ctx=(92, 92, 93), live=live).run_block(1, 1)


@pytest.mark.parametrize("block", [-1, 0, 4097])
def test_blocks_that_a_step_cannot_unmask(block):
    with pytest.raises(ValueError, match="block"):
        G.PagedGenerator(SimpleNamespace(max_pos=1 << 20), 1, block, max_len=1 << 14, pool=256)
