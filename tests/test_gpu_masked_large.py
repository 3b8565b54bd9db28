"""Masked attention of many rows: tiles of 32 rows whose workgroups go to the dies in turn,
against the oracle, bit for bit.  And the greedy rounds of a drafted generator, token
by token, so that what is accepted is pinned."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from tests import _masked as K
from tests._gpu import need_gpu
from tests.test_gpu_drafted import generator, model
from tests.test_gpu_masked import check

pytestmark = pytest.mark.gpu


def in_turn(M, H, tile):
    """Workgroups go to the dies in turn from 64 tiles of groups of up to eight heads on."""
    return -(-M // tile) * -(-H // 8) >= 64


def mixed(M, J, seed):
    """Documents, rows behind a prefix, first keys and a window, any ranges, rows of none."""
    rng = np.random.default_rng([17, seed])
    r, pos = K.docs_mask([700, 1, 63], M - 764)
    i = np.arange(764, 1400)
    r[i], pos[i] = np.stack([0 * i, i, 0 * i, 0 * i], 1), i
    i = np.arange(1400, 1790)
    r[i], pos[i] = np.stack([0 * i, 0 * i + 4, i - 130, i + 1], 1), i
    r[1790:1900], pos[1790:1900] = K.random_mask(rng, 110, J)
    i = np.arange(1950, M)                       # 1900 to 1950: rows of none
    r[i], pos[i] = np.stack([0 * i, 0 * i + J, 0 * i, 0 * i], 1), i
    return r, pos


@pytest.mark.parametrize("T, H, dh, max_dist", [(2, 16, 64, None), (2, 16, 128, 40), (2, 9, 128, None), (3, 9, 64, 7),
                                                (4, 5, 128, 300), (1, 17, 64, None)])
@pytest.mark.parametrize("M", [2048, 2055])
def test_tiles_of_32_rows_in_turn(M, T, H, dh, max_dist):
    J = M + 77
    r = K.route(T, M, J, H)
    assert (r.tile, r.heads) == (32, False) and in_turn(M, H, 32)
    ranges, pos = mixed(M, J, H)
    check(K.make_case(H, ranges, pos, J, T=T, H=H, dh=dh, max_dist=max_dist))


@pytest.mark.parametrize("H, M", [(1, 1287), (5, 1287), (9, 1607), (16, 1607)])
def test_the_route_of_many_tiles(H, M):
    """Of the calls of one timestep over as many rows in documents: tiles of 16, in turn."""
    r = K.route(1, M, M, H)
    assert (r.tile, r.heads) == (16, False) and in_turn(M, H, 16)


@pytest.mark.parametrize("seed, draft, more", [(72, 2, 10), (70, 2, 4), (82, 1, 4), (75, "own", 0)])
def test_greedy_rounds_accept_what_the_oracle_accepts(seed, draft, more):
    """Each round's tokens; `more`: drafts that stand in the oracle's rounds, at the least."""
    torch, B = need_gpu()
    m, other = model(seed), model(seed + 100, n_layers=1)
    want = O.drafted(m, other if draft == "own" else None, None if draft == "own" else draft, [3, 4, 5], 10, 4, 0.0, 0.0,
                     lambda *shape: np.zeros(shape, np.float32))
    assert sum(len(x) for x in want) >= 10 + more
    g = generator(B, m, other if draft == "own" else draft, 128, 4, 0.0)
    g.start([3, 4, 5])
    assert [g.round() for _ in range(10)] == want
