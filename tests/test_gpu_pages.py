"""GPU parity of the paged caches (plan, store, selection, attention) against
the oracle: integers, so every comparison is equality."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O

from . import _pages as P
from ._gpu import assert_same, need_gpu

pytestmark = pytest.mark.gpu


def device(c):
    torch, B = need_gpu()
    return P.Device(torch, B, c)


def sync():
    import torch
    torch.cuda.synchronize()


def check_plan(d, p, status=None):
    pg = d.pages
    for name in ("table", "held", "ring", "ring_state", "cu_rows", "slot", "pos"):
        assert_same(getattr(pg, name).cpu().numpy(), np.asarray(p[name]), name)
    assert int(d.status) == (p["status"] if status is None else status)


def store_oracle(c, p):
    O.page_store(c.k, c.v, p["slot"], c.k_pages, c.v_pages, c.counts)


def check_store(d, c):
    assert_same(d.bits(d.k_pages, c.dh), c.k_pages, "key pages")
    assert_same(d.values(), c.v_pages, "value pages")
    assert_same(d.counts.cpu().numpy(), c.counts, "key counts")


# --------------------------------------------------------------------------
# plan
# --------------------------------------------------------------------------
LENGTHS = {
    "one_token": ([0], [1]),
    "one_page": ([0], [64]),
    "page_and_one": ([64, 63, 65, 128], [1, 1, 1, 64]),
    "idle_and_ended": ([100, 64, 0, 640, 5], [0, -1, 7, -1, 16]),
    "all_idle": ([3, 0], [0, 0]),
    "ended_only": ([3, 200], [-1, -1]),
    "mixed": ([0, 1, 63, 64, 127, 500, 2000, 33], [1, 63, 2, 64, 300, 1, -1, 70]),
}


@pytest.mark.parametrize("name", LENGTHS)
def test_plan(name):
    c = P.make_case(3, *LENGTHS[name], T=1, H=1)
    d = device(c)
    d.plan()
    sync()
    p = P.plan(c)
    check_plan(d, p)
    if name != "idle_and_ended":
        return
    # the same lengths again: nothing more is taken (ended requests hold nothing now)
    d.plan()
    sync()
    p2 = O.page_plan(c.ctx, c.new, p["table"], p["held"], p["ring"], p["ring_state"], c.max_rows)
    assert p2["ring_state"] == p["ring_state"]
    check_plan(d, p2)


@pytest.mark.parametrize("n,hi,seed", [(1, 5000, 0), (37, 40, 1), (300, 12, 2), (1024, 3, 3), (1025, 200, 4),
                                       (3000, 30, 5), (700, 0, 6), (16384, 9, 7)])
def test_plan_many(n, hi, seed):
    """One launch and two, more requests than a chunk of the sums, and the ring
    running out."""
    rng = np.random.default_rng(seed)
    ctx = rng.integers(0, 400, size=n)
    new = rng.integers(-1, hi + 1, size=n)
    new[rng.random(n) < 0.1] = -1
    for short in (False, True):
        c = P.make_case(seed, ctx, new, T=1, H=1, spare_rows=70)
        if short:  # the last of the free pages are not there
            c.ring_state[1] = max(c.ring_state[1] - 7, 0) // 2
        d = device(c)
        d.plan()
        sync()
        check_plan(d, P.plan(c))


def test_plan_refuses():
    """Lengths outside the bounds, each beside requests that are served."""
    import torch

    c = P.make_case(5, [10, 100, 64, 0, 70, 10, 0], [5, 30, 1, 9, 3, 64, 20], T=1, H=1, spare_rows=60)
    big = 2 ** 31 - 1
    changes = [dict(ctx={1: -1}), dict(ctx={1: 129}), dict(ctx={4: big}), dict(new={3: -2}), dict(new={3: -big}),
               dict(new={3: big}), dict(new={0: c.max_rows + 1}), dict(new={0: c.max_rows}),
               dict(new={6: 64 * c.max_pages + 1}), dict(held={2: -1}), dict(held={2: big}),
               dict(held={4: c.max_pages + 1}, new={4: -1}), dict(table={(2, 0): c.pool}),
               dict(table={(2, 0): -5}), dict(new={1: -1, 4: -1}, table={(1, 0): -3})]
    for ch in changes:
        e = P.make_case(5, c.ctx, c.new, T=1, H=1, spare_rows=60)
        for name, sub in ch.items():
            for i, v in sub.items():
                getattr(e, name)[i] = v
        d = device(e)
        d.plan()
        sync()
        check_plan(d, P.plan(e))
    # the status word keeps other bits; none is needed
    e = P.make_case(5, c.ctx, c.new, T=1, H=1)
    e.ctx[1] = -1
    d = device(e)
    d.status.fill_(1)
    d.plan()
    d.B.nmdlm_page_plan(d.pages, d.ctx, d.new)
    torch.cuda.synchronize()
    assert int(d.status) == 1 | O.BAD_REQUEST


def test_plan_over_steps():
    """Requests come, grow block by block and end; the pages they hold are
    disjoint and none is lost."""
    import torch

    rng = np.random.default_rng(9)
    n = 20
    c = P.make_case(6, [0] * n, [0] * n, T=1, H=1, spare_rows=400, spare_pages=8, spare_pool=40)
    d = device(c)
    st = dict(table=c.table, held=c.held, ring=c.ring, ring_state=c.ring_state)
    ctx = np.zeros(n, dtype=np.int64)
    for step in range(25):
        new = np.where(ctx == 0, rng.integers(0, 120, n), rng.integers(0, 33, n))
        new = np.where((ctx > 200) | (rng.random(n) < 0.1), -1, new)
        p = O.page_plan(ctx, new, *st.values(), c.max_rows)
        d.ctx.copy_(torch.from_numpy(ctx))
        d.new.copy_(torch.from_numpy(new))
        d.status.zero_()
        d.plan()
        sync()
        check_plan(d, p)
        st = {k: p[k] for k in st}
        ctx = np.where(new == -1, 0, np.where(p["ok"], ctx + new, ctx))
        own = [int(x) for s in range(n) for x in p["table"][s, :p["held"][s]]]
        head, free = p["ring_state"]
        own += [int(p["ring"][(head + i) % c.pool]) for i in range(free)]
        assert sorted(own) == list(range(c.pool))


# --------------------------------------------------------------------------
# store
# --------------------------------------------------------------------------
@pytest.mark.parametrize("T,H,dh", [(1, 1, 64), (4, 2, 128), (3, 5, 64), (8, 3, 128)])
def test_store(T, H, dh):
    c = P.make_case(T, [0, 5, 63, 64, 100, 0, 30, 200], [1, 40, 1, 64, 130, 0, -1, 7], T=T, H=H, dh=dh)
    d = device(c)
    d.plan()
    d.store()
    sync()
    store_oracle(c, P.plan(c))
    check_store(d, c)


def test_store_skips_refused_rows():
    c = P.make_case(8, [0, 0, 40], [70, 70, 3], T=2, H=2, spare_rows=0)
    c.ring_state[1] = 2                       # one request's pages
    c.table[2, 0] = c.pool + 4                # and a page that does not exist
    d = device(c)
    d.plan()
    d.store()
    sync()
    p = P.plan(c)
    assert p["status"] == O.PAGES_SHORT and (p["slot"][70:] == -1).all()
    store_oracle(c, p)
    check_store(d, c)


# --------------------------------------------------------------------------
# selection
# --------------------------------------------------------------------------
@pytest.mark.parametrize("T,H,dh,n_sel", [(1, 1, 64, 1), (4, 3, 128, 3), (3, 2, 64, 0), (8, 2, 128, 7),
                                          (2, 4, 64, 1000)])
def test_select(T, H, dh, n_sel):
    c = P.make_case(T + 10, [0, 64, 63, 700, 1200, 640, 4200, 70], [3, 1, 2, 17, 33, 0, 5, -1], T=T, H=H, dh=dh)
    d = device(c)
    d.plan()
    d.select(n_sel)
    sync()
    assert_same(d.selection(), P.select(c, P.plan(c), n_sel), "selected pages")


@pytest.mark.parametrize("rate", [0.0, 1.0])
def test_select_ties(rate):
    """Equal scores everywhere: zero, and the largest there is (8 x 128 x 64)."""
    c = P.make_case(21, [64 * 70 + 3], [18], T=8, H=1, dh=128, rate=rate)
    d = device(c)
    d.plan()
    d.select(65)
    sync()
    sel = d.selection()
    assert_same(sel, P.select(c, P.plan(c), 65), "selected pages")
    assert sel[0, 0].sum() == 65 + 1 and sel[0, 0, :65].all()


def test_select_long():
    """More pages than a wave keeps in registers, and a page that is not there."""
    c = P.make_case(22, [64 * 2500, 64 * 300 + 1], [2, 20], T=1, H=1)
    c.table[1, 7] = -1
    d = device(c)
    d.plan()
    d.select(40)
    sync()
    assert_same(d.selection(), P.select(c, P.plan(c), 40), "selected pages")


@pytest.mark.parametrize("T,H,dh,n_sel", [(4, 4, 64, 3), (1, 4, 128, 1), (8, 4, 128, 20), (3, 4, 64, 0)])
def test_select_one_kernel(T, H, dh, n_sel):
    """Requests enough for scores and choice in one kernel."""
    rng = np.random.default_rng(T)
    ctx, new = rng.integers(0, 900, size=70), rng.integers(1, 20, size=70)
    ctx[0], new[0], new[1] = 64 * 126, 17, 0
    c = P.make_case(T + 24, ctx, new, T=T, H=H, dh=dh, spare_pages=0)
    assert P.case_route(c).fused
    d = device(c)
    d.plan()
    d.select(n_sel)
    sync()
    assert_same(d.selection(), P.select(c, P.plan(c), n_sel), "selected pages")


@pytest.mark.parametrize("n_sel", [1, 64, 600])
def test_select_widths(n_sel):
    """Contexts in every class of the choice: up to 64, 128, 512 and 2048 pages and more."""
    pages = [64, 65, 128, 129, 512, 513, 700, 2048, 2049]
    c = P.make_case(25, [64 * p for p in pages], [1] * len(pages), T=1, H=1)
    assert not P.case_route(c).fused
    d = device(c)
    d.plan()
    d.select(n_sel)
    sync()
    assert_same(d.selection(), P.select(c, P.plan(c), n_sel), "selected pages")


# --------------------------------------------------------------------------
# attention
# --------------------------------------------------------------------------
SHAPES = {
    "one_token": ([0], [1]),
    "tokens": ([0, 63, 64, 65, 700, 1, 2000], [1] * 7),
    "blocks": ([0, 100, 640, 5], [16, 16, 0, 16]),
    "ragged": ([0, 50, 64, 1300, 9, 0, 300], [1, 40, 64, 3, 17, 5, -1]),
    "prompts": ([0, 0, 10], [130, 70, 33]),
}


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("T,H,dh", [(1, 1, 64), (2, 3, 128), (3, 2, 64), (4, 2, 128), (5, 1, 128), (7, 2, 64),
                                    (8, 1, 64)])
def test_attention(name, T, H, dh):
    c = P.make_case(T + H, *SHAPES[name], T=T, H=H, dh=dh)
    d = device(c)
    d.plan()
    d.attention()
    sync()
    cur, spk = P.attention(c, P.plan(c))
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


def some_selection(c, p, seed, share):
    rng = np.random.default_rng(seed)
    return (rng.random((c.max_rows, c.H, -(-c.max_pages // 64) * 64)) < share).astype(np.uint8)


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("T,H,dh,share", [(1, 2, 64, 0.3), (4, 2, 128, 0.05), (3, 1, 128, 0.6), (8, 2, 64, 0.1)])
def test_attention_selected(name, T, H, dh, share):
    """Random selections: rows that see no page among them, bits past the last page."""
    c = P.make_case(T + H + 30, *SHAPES[name], T=T, H=H, dh=dh)
    d = device(c)
    d.plan()
    p = P.plan(c)
    sel = some_selection(c, p, T, share)
    sel[0] = 0
    d.attention(sel=d.put_selection(sel))
    sync()
    cur, spk = P.attention(c, p, sel)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("new", [(3, 2), (14, 9)])
@pytest.mark.parametrize("dh,share", [(64, None), (128, None), (64, 0.4), (128, 0.02)])
def test_attention_long(new, dh, share):
    """Contexts from 65536 keys on (sums beyond 24 bits) beside a short one, by
    rows and by tiles."""
    c = P.make_case(40, [64 * 1200 + 7, 30], new, T=1, H=1, dh=dh)
    assert P.case_route(c).token == (new == (3, 2))
    c.lut[:] = 255
    d = device(c)
    d.plan()
    p = P.plan(c)
    sel = None if share is None else some_selection(c, p, 1, share)
    d.attention(sel=None if sel is None else d.put_selection(sel))
    sync()
    cur, spk = P.attention(c, p, sel)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("share", [None, 0.02])
def test_attention_long_tiles(share):
    """Tiles of rows over more pages than the kernel lists at once."""
    c = P.make_case(41, [64 * 270 + 9], [500], T=1, H=32, dh=64)
    d = device(c)
    d.plan()
    p = P.plan(c)
    sel = None if share is None else some_selection(c, p, 1, share)
    d.attention(sel=None if sel is None else d.put_selection(sel))
    sync()
    cur, spk = P.attention(c, p, sel)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("T,H,dh,sel", [(4, 16, 64, False), (4, 16, 128, True), (1, 16, 128, False)])
def test_attention_wide_tiles(T, H, dh, sel):
    """Enough rows for 32 queries a wave."""
    c = P.make_case(50, [0, 200, 64], [700, 517, 390], T=T, H=H, dh=dh)
    d = device(c)
    d.plan()
    p = P.plan(c)
    s = some_selection(c, p, 2, 0.2) if sel else None
    d.attention(sel=d.put_selection(s) if sel else None)
    sync()
    cur, spk = P.attention(c, p, s)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("T,H,dh,share", [(1, 64, 64, None), (2, 20, 128, 0.3), (8, 5, 128, None)])
def test_attention_wide_tiles_other_timesteps(T, H, dh, share):
    c = P.make_case(51, [100, 0], [600, 333], T=T, H=H, dh=dh)
    assert P.case_route(c).groups == 2
    d = device(c)
    d.plan()
    p = P.plan(c)
    s = None if share is None else some_selection(c, p, 3, share)
    d.attention(sel=None if s is None else d.put_selection(s))
    sync()
    cur, spk = P.attention(c, p, s)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("new,splits", [(1, 20), (20, 20)])
@pytest.mark.parametrize("share", [None, 0.1, 0.0])
def test_attention_many_splits(new, splits, share):
    """Rows and tiles over a context in many splits, whole, selected and with
    nothing selected; a short request beside it in one."""
    c = P.make_case(52, [64 * 160, 40], [new, new], T=3, H=1, dh=128)
    r = P.case_route(c)
    assert r.token == (new == 1) and r.splits == splits
    d = device(c)
    d.plan()
    p = P.plan(c)
    s = None if share is None else some_selection(c, p, 3, share)
    d.attention(sel=None if s is None else d.put_selection(s))
    sync()
    cur, spk = P.attention(c, p, s)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


def test_attention_one_output():
    c = P.make_case(60, [90, 7], [20, 3], T=4, H=2, dh=64)
    cur, spk = P.attention(c, P.plan(c))
    for want_cur, want_spk in ((True, False), (False, True)):
        d = device(c)
        d.plan()
        d.attention(cur=want_cur, spk=want_spk)
        sync()
        if want_cur:
            assert_same(d.cur.cpu().numpy(), cur, "currents")
            assert int((d.spk != -1).sum()) == 0
        else:
            assert_same(d.spikes(), spk, "spikes")
            assert int((d.cur != -9).sum()) == 0


def test_attention_zero_weights():
    """A table of zeros: no weight anywhere, currents 0."""
    c = P.make_case(61, [90], [20], T=2, H=1, dh=128)
    c.lut[:] = 0
    d = device(c)
    d.plan()
    d.attention()
    sync()
    assert int(d.cur[:, :20].abs().sum()) == 0 and int((d.spk[:, :20] != 0).sum()) == 0


def test_attention_misaligned_currents():
    c = P.make_case(62, [90, 3], [20, 5], T=2, H=1, dh=64)
    d = device(c)
    import torch
    buf = torch.full((d.cur.numel() + 1,), -9, dtype=torch.int32, device="cuda")
    d.cur = buf[1:].view(d.cur.shape)
    d.plan()
    d.attention()
    sync()
    assert_same(d.cur.cpu().numpy(), P.attention(c, P.plan(c))[0], "currents")


def test_attention_pages_not_there():
    """Table entries outside the pool count as pages without keys."""
    c = P.make_case(63, [500, 200], [20, 1], T=2, H=2, dh=64)
    c.table[0, 3], c.table[1, 0] = c.pool, -2
    d = device(c)
    d.plan()
    d.attention()
    sync()
    p = P.plan(c)
    sel = np.ones((c.max_rows, c.H, -(-c.max_pages // 64) * 64), dtype=np.uint8)
    sel[:20, :, 3] = 0
    sel[20:21, :, 0] = 0
    p["table"][0, 3] = p["table"][1, 0] = 0
    cur, spk = P.attention(c, p, sel)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


# --------------------------------------------------------------------------
# together
# --------------------------------------------------------------------------
def run_all(d, n_sel, **kw):
    d.plan(**kw)
    d.store(**kw)
    d.select(n_sel, **kw)
    d.attention(sel=d.sel, **kw)


def check_all(d, c, n_sel):
    p = P.plan(c)
    store_oracle(c, p)
    sel = P.select(c, p, n_sel)
    cur, spk = P.attention(c, p, sel)
    check_plan(d, p)
    check_store(d, c)
    assert_same(d.selection(), sel, "selected pages")
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("T,H,dh", [(4, 2, 64), (8, 2, 128), (1, 3, 128)])
def test_together(T, H, dh):
    c = P.make_case(70, [0, 100, 640, 5, 1000, 77], [16, 16, 0, 16, 16, -1], T=T, H=H, dh=dh)
    d = device(c)
    run_all(d, 3)
    sync()
    check_all(d, c, 3)


@pytest.mark.parametrize("new", [20, 1])
def test_refused_requests_between_others(new):
    """Rows of refused requests are neither selected for nor attended, whichever
    kernel takes the rows."""
    c = P.make_case(72, [100, 0, 70, 0, 200], [new, new, new, 70 if new > 1 else 1, new], T=2, H=2, dh=64, spare_rows=0)
    assert P.case_route(c).token == (new == 1)
    c.ctx[2] = 129                            # beyond its pages
    c.ring_state[1] = 1                       # the second takes the only page
    d = device(c)
    run_all(d, 1)
    sync()
    p = P.plan(c)
    assert p["ok"].tolist() == [True, True, False, False, True]
    check_all(d, c, 1)


def test_nothing_to_do():
    """Idle and ended requests only: no row, nothing written."""
    c = P.make_case(73, [100, 0, 70], [0, 0, -1], T=2, H=2, dh=64)
    d = device(c)
    run_all(d, 1)
    sync()
    check_all(d, c, 1)


def test_a_pool_beyond_32_bits():
    """Pages whose words lie past 2^32 of the pool's first."""
    import torch

    c = P.make_case(74, [64 * 9, 30], [9, 1], T=8, H=16, dh=128)
    d = device(c)
    words = 16 * 8 * 128                     # of a page's keys, and of its values
    pool, shift = 2 ** 32 // words + 40 + c.pool, 2 ** 32 // words + 40
    free, _ = torch.cuda.mem_get_info()
    if free < 2 * 8 * pool * words + pool * words + (8 << 30):
        pytest.skip("not enough memory")
    n = P.Device.__new__(P.Device)
    n.__dict__.update(d.__dict__)
    n.pages = d.B.Pages(c.n, c.max_rows, c.max_pages, pool)
    move = lambda x: torch.where(x >= 0, x + shift, x)  # noqa: E731
    ring = torch.zeros(pool, dtype=torch.int32, device="cuda")
    head, k = c.ring_state
    ring[:k] = torch.from_numpy(c.ring[(head + np.arange(k)) % c.pool].astype(np.int32)).cuda() + shift
    n.pages.set_state(move(d.pages.table), d.pages.held, ring, torch.tensor([0, k], dtype=torch.int32))
    n.k_pages, n.v_pages, n.counts = n.pages.pools(8, 16, 128)
    for big, small in ((n.k_pages, d.k_pages), (n.v_pages, d.v_pages), (n.counts, d.counts)):
        big[shift:] = small
    run_all(n, 3)
    sync()
    n.k_pages, n.v_pages, n.counts = (x[shift:].clone() for x in (n.k_pages, n.v_pages, n.counts))
    p = P.plan(c)
    store_oracle(c, p)
    check_store(n, c)
    sel = P.select(c, p, 3)
    cur, spk = P.attention(c, p, sel)
    assert_same(n.selection(), sel, "selected pages")
    assert_same(n.cur.cpu().numpy(), cur, "currents")
    assert_same(n.spikes(), spk, "spikes")


def test_on_another_stream_and_in_a_graph():
    """The four calls on a stream of the caller's, then captured and replayed
    with eager work between the replays."""
    import torch

    c = P.make_case(71, [30, 100, 640, 5, 1000], [16, 16, 0, 16, -1], T=4, H=2, dh=128)
    d = device(c)
    first = d.pages.state.clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        run_all(d, 2)
    s.synchronize()
    want = [x.clone() for x in (d.pages.state, d.k_pages, d.v_pages, d.counts, d.sel, d.cur, d.spk)]
    check_all(d, c, 2)
    g = torch.cuda.CUDAGraph()
    d.pages.state.copy_(first)
    with torch.cuda.graph(g):
        run_all(d, 2)
    for _ in range(3):
        d.pages.state.copy_(first)
        d.cur.fill_(-9)
        d.spk.fill_(-1)
        d.sel.fill_(-1)
        d.ws_att.fill_(7)
        d.ws_sel.fill_(7)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for got, ref in zip((d.pages.state, d.k_pages, d.v_pages, d.counts, d.sel, d.cur, d.spk), want):
            assert torch.equal(got, ref)


def test_two_calls_at_once():
    """Two requests' sets on two streams, each with its own plan and workspaces."""
    import torch

    cs = [P.make_case(80 + i, [64 * 20 + i, 300], [9 + i, 20], T=4, H=2, dh=128) for i in range(2)]
    ds = [device(c) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    for d, s in zip(ds, streams):
        run_all(d, 4, stream=s)
    torch.cuda.synchronize()
    for d, c in zip(ds, cs):
        check_all(d, c, 4)


@pytest.mark.parametrize("H,heads", [(7, 4), (3, 3)])
def test_select_by_groups_of_heads(H, heads):
    """A plan of so many rows that the scores of its heads are held in turn (four
    and three of them, or all three): a few of its rows are there, with a context
    of several hundred pages."""
    c = P.make_case(26, [64 * 300 + 5, 700], [20, 3], T=1, H=H, dh=64, spare_rows=64000, spare_pages=700)
    d = device(c)
    assert d.ws_sel.numel() == -(-c.max_rows * heads * -(-c.max_pages // 16) * 16 * 4 // 256) * 256
    d.plan()
    d.select(9)
    sync()
    assert_same(d.selection(), P.select(c, P.plan(c), 9), "selected pages")


def run_attention(c, share, seed=4):
    d = device(c)
    d.plan()
    p = P.plan(c)
    sel = None if share is None else some_selection(c, p, seed, share)
    d.attention(sel=None if sel is None else d.put_selection(sel))
    sync()
    cur, spk = P.attention(c, p, sel)
    assert_same(d.cur.cpu().numpy(), cur, "currents")
    assert_same(d.spikes(), spk, "spikes")


@pytest.mark.parametrize("T,dh", [(1, 64), (4, 128)])
@pytest.mark.parametrize("share", [None, 0.3, 0.9, 0.0])
def test_attention_rows_over_many_lists(T, dh, share):
    """Single rows whose one workgroup lists its pages in three pieces (256, 256
    and the rest), beside short requests."""
    n, H = 70, 8
    c = P.make_case(90, [64 * 531 + 5] + [20 + 3 * i for i in range(n - 1)], [1] * n, T=T, H=H, dh=dh, spare_pages=0)
    r = P.case_route(c)
    assert r.token and r.splits == 1 and c.max_pages > 512
    run_attention(c, share)


@pytest.mark.parametrize("pages", [256, 257, 512, 513])
def test_attention_rows_at_the_list_end(pages):
    n = 70
    c = P.make_case(91, [64 * pages - 1] + [9] * (n - 1), [1] * n, T=2, H=8, dh=64, spare_pages=0)
    r = P.case_route(c)
    assert r.token and r.splits == 1 and c.max_pages == pages
    run_attention(c, None)
    run_attention(c, 0.5)


@pytest.mark.parametrize("share", [None, 0.2, 0.005])
def test_attention_wide_tiles_over_many_lists(share):
    """Tiles of 32 rows over more pages than are listed at once."""
    c = P.make_case(92, [64 * 300 + 30] + [0] * 7, [37] + [32] * 7, T=8, H=8, dh=64, spare_rows=0, spare_pages=0)
    r = P.case_route(c)
    assert r.groups == 2 and c.max_pages > 256
    run_attention(c, share)


@pytest.mark.parametrize("name", SHAPES)
@pytest.mark.parametrize("share", [None, 0.3])
def test_attention_six_timesteps(name, share):
    run_attention(P.make_case(93, *SHAPES[name], T=6, H=2, dh=128), share)


def test_attention_single_rows_six_timesteps():
    """Two parts a timestep: twelve waves."""
    c = P.make_case(94, [1000 + i for i in range(16)], [2] * 16, T=6, H=4, dh=128)
    r = P.case_route(c)
    assert r.token and r.parts == 2
    run_attention(c, None)
    run_attention(c, 0.3)
