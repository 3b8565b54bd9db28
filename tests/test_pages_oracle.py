"""The oracle of the paged caches on cases worked by hand, and against the
contiguous attention."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O

from . import _pages as P


def test_plan_by_hand():
    # pool of 6; the ring holds pages 4, 1, 3 from index 5 on (wrapping)
    ring = [1, 3, 9, 9, 9, 4]
    table = [[0, -1, -1], [2, 5, -1], [-1, -1, -1]]
    p = O.page_plan([60, 100, 0], [10, -1, 65], table, [1, 2, 0], ring, [5, 3], 80)
    assert p["table"].tolist() == [[0, 4, -1], [2, 5, -1], [1, 3, -1]]
    assert p["held"].tolist() == [2, 0, 2]
    assert p["ring"].tolist() == [1, 3, 2, 5, 9, 4]            # 2 and 5 behind the old ring
    assert p["ring_state"] == [2, 2]                            # and they are all that is free
    assert p["cu_rows"].tolist() == [0, 10, 10, 75]
    assert p["slot"][:10].tolist() == [60, 61, 62, 63] + [4 * 64 + i for i in range(6)]
    assert p["slot"][10] == 64 and p["slot"][74] == 3 * 64 and (p["slot"][75:] == -1).all()
    assert p["pos"][9] == 69 and p["pos"][74] == 64 and p["status"] == 0


def test_plan_refuses():
    table = np.full((5, 2), -1)
    table[3, 0] = 0
    # the second lacks pages that the ring (1 free) does not have: it and the third are
    # refused, the fourth needs none, the fifth lies outside its table
    p = O.page_plan([0, 0, 0, 10, 0], [64, 65, 1, 20, 129], table, [0, 0, 0, 1, 0], [1, 0], [0, 1], 400)
    assert p["ok"].tolist() == [True, False, False, True, False]
    assert p["status"] == O.PAGES_SHORT | O.BAD_REQUEST
    assert p["cu_rows"].tolist() == [0, 64, 129, 130, 150, 279]
    assert (p["slot"][64:130] == -1).all() and p["slot"][130] == 10 and (p["slot"][150:] == -1).all()
    assert p["ring_state"] == [1, 0] and p["held"].tolist() == [1, 0, 0, 1, 0]
    # rows past the last packed row; a context beyond the held pages
    p = O.page_plan([0, 0], [5, 4], np.full((2, 1), -1), [0, 0], [0, 1], [0, 2], 8)
    assert p["ok"].tolist() == [True, False] and p["cu_rows"].tolist() == [0, 5, 8]
    p = O.page_plan([65], [1], [[0, -1]], [1], [1, 0], [0, 1], 8)
    assert p["status"] == O.BAD_REQUEST


def test_selection_by_hand():
    Q = np.zeros((1, 2, 1, 64), dtype=np.uint8)
    Q[0, 0, 0, :2] = 1                      # row 0 asks for channels 0 and 1; row 1 for none
    counts = np.zeros((5, 1, 1, 64), dtype=np.int64)
    counts[:, 0, 0, 0] = [3, 1, 0, 3, 9]
    counts[:, 0, 0, 1] = [0, 4, 0, 0, 9]
    counts[:, 0, 0, 2] = 50
    sel = O.page_select(Q, counts, 4, 5, 2)  # scores 3 5 0 3: page 1, then 0 before 3
    assert sel[0, 0].tolist() == [1, 1, 0, 0, 1]
    assert sel[1, 0].tolist() == [1, 1, 0, 0, 1]                # no score: the lowest pages
    assert O.page_select(Q, counts, 4, 5, 0)[0, 0].tolist() == [0, 0, 0, 0, 1]
    assert O.page_select(Q, counts, 4, 5, 9).all()


def test_counts_score_is_the_sum_of_the_scores():
    c = P.make_case(1, [130], [7], T=2, H=2, dh=64)
    p = P.plan(c)
    ids = P.pages_of(c, p, 0)[:2]
    for m in range(7):
        for h in range(2):
            want = sum(int((c.q[t, m, h] & c.k_pages[i, h, t]).sum()) for t in range(2) for i in ids)
            got = int((c.counts[ids, h] * c.q[:, m, h]).sum())
            assert got == want


@pytest.mark.parametrize("J,M", [(1, 1), (64, 3), (131, 9)])
def test_all_pages_is_the_contiguous_attention(J, M):
    rng = np.random.default_rng(J)
    T, H, dh = 3, 2, 64
    Q, K, V = (rng.random((T, r, H * dh)) < 0.3 for r in (M, J, J))
    lut = rng.integers(1, 256, size=256)
    split = lambda x: x.reshape(T, -1, H, dh)  # noqa: E731
    cache = lambda x: split(x).transpose(2, 0, 1, 3)  # noqa: E731
    a = O.paged_attention(split(Q), cache(K), cache(V), lut, np.ones((M, H, J), dtype=np.uint8))
    assert np.array_equal(a, O.bbm_attention(Q, K, V, J, H, lut))
    none = O.paged_attention(split(Q), cache(K), cache(V), lut, np.zeros((M, H, J), dtype=np.uint8))
    assert not none.any()


def test_store_counts_up_to_the_last_row():
    c = P.make_case(2, [10, 64], [5, 1], T=1, H=1)
    p = P.plan(c)
    k0 = c.k_pages.copy()
    O.page_store(c.k, c.v, p["slot"], c.k_pages, c.v_pages, c.counts)
    pg = p["table"][0, 0]
    assert np.array_equal(c.k_pages[pg, 0, 0, 10:15], c.k[0, :5, 0])
    assert np.array_equal(c.k_pages[pg, 0, 0, 15:], k0[pg, 0, 0, 15:])
    assert np.array_equal(c.counts[pg, 0, 0], c.k_pages[pg, 0, 0, :15].sum(0))
    assert np.array_equal(c.counts[p["table"][1, 1], 0, 0], c.k[0, 5, 0])
