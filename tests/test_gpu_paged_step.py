"""The block step over pages against the oracle: requests of different lengths
admitted, advanced and released over one pool, a step over selected pages, and
the step in a graph."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from workloads import synth

from ._gpu import assert_same, need_gpu

pytestmark = pytest.mark.gpu


def small_model(seed=5, n_layers=2, d=128, H=2, F=192, V=304, T=4, max_pos=512):
    return synth.make_mdlm(seed, n_layers, d=d, H=H, F=F, V=V, T=T, max_pos=max_pos)


def device_model(B, m, blocked=False):
    return B.DeviceModel.from_mdlm(m, 64, blocked=blocked)


def prompts_of(lens, V, seed=0):
    return [synth.random_tokens(seed + i, n, V) for i, n in enumerate(lens)]


@pytest.mark.parametrize("T,H,blocked", [(4, 2, False), (4, 1, True), (8, 2, True)])
def test_requests_of_different_lengths(T, H, blocked):
    """Three requests at once, one ends and gives its pages to a fourth that the
    pool would not have held beside the three."""
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model(T=T, H=H)
    Bk, steps, k = 8, 3, 3
    lens = [70, 1, 131, 150]
    ps = prompts_of(lens, m.V)
    want = [O.generate(m, p, 2, Bk, steps, k) for p in ps]
    # 70 + 16 -> 2 pages, 17 -> 1, 147 -> 3 and 166 -> 3 once the first has gone
    g = PagedGenerator(device_model(B, m, blocked), 3, Bk, max_len=192, pool=7, max_prompt_rows=210)
    g.admit({0: ps[0], 1: ps[1]})
    log = []
    out = {0: [], 1: [], 2: []}
    for i, x in g.run_block(steps, k, log).items():
        out[i].append(x)
    g.admit({2: ps[2]})                       # the others stand one block further
    first = g.run_block(steps, k)
    for i, x in first.items():
        out[i].append(x)
    last = g.run_block(steps, k)              # the third request's second block
    out[2].append(last[2])
    for i in range(3):
        assert_same(torch.cat(out[i][:2]).cpu().numpy(), want[i][0], f"request {i}")
    for j in range(steps):
        for i in range(2):
            w = list(want[i][1][j])           # the oracle lists those that were there to choose
            assert_same(log[j][i].cpu().numpy(), w + [-1] * (k - len(w)), f"chosen {i}, step {j}")
        assert (log[j][2] == -1).all()
    with pytest.raises(ValueError):
        g.admit({0: ps[3]})
    g.release([0])
    g.admit({0: ps[3]})
    a = g.run_block(steps, k)[0]
    g.release([1, 2])
    b = g.run_block(steps, k)[0]
    assert_same(torch.cat([a, b]).cpu().numpy(), want[3][0], "the fourth request")
    g.release([0])
    assert g.pages.ring_state.tolist()[1] == 7 and sorted(g.pages.ring.tolist()) == list(range(7))


def test_pool_runs_out():
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model()
    g = PagedGenerator(device_model(B, m), 2, 8, max_len=192, pool=3, max_prompt_rows=210)
    ps = prompts_of([100, 100], m.V)
    g.admit({0: ps[0]})
    with pytest.raises(RuntimeError, match="too few pages"):
        g.admit({1: ps[1]})
    assert g.pages.ring_state.tolist()[1] == 1 and g.pages.held.tolist() == [2, 0]
    with pytest.raises(ValueError):
        g.admit({1: np.zeros(0, np.int32)})
    g.release([0])
    with pytest.raises(RuntimeError, match="too few pages"):
        g.admit({0: ps[0], 1: ps[1]})         # the first's pages go back with the refusal
    assert g.pages.ring_state.tolist()[1] == 3 and g.pages.held.tolist() == [0, 0]
    g.admit({0: ps[0]})
    # and it goes on by itself
    want = O.generate(m, ps[0], 1, 8, 2, 4)[0]
    assert_same(g.run_block(2, 4)[0].cpu().numpy(), want, "ids")


def paged_layer(X, L, ctx, n_sel, K, V, c0):
    """One layer of one request over selected pages: X [T][M][d], K and V 0/1
    [T][>= c0 + M][d] hold the context and take the rows."""
    T, M, d = X.shape
    H, dh, J = L.H, L.d // L.H, c0 + M
    I = O.qbsm(X, L.W_qkv)
    q, k, v = (O.if_neuron(I[..., i * d:(i + 1) * d], L.theta[n])[0] for i, n in enumerate("qkv"))
    K[:, c0:J], V[:, c0:J] = k, v
    nP = -(-J // 64)
    heads = lambda x: x.reshape(T, -1, H, dh)  # noqa: E731
    pad = np.zeros((T, nP * 64, d), dtype=bool)
    pad[:, :J] = K[:, :J]
    counts = pad.reshape(T, nP, 64, H, dh).sum(2).transpose(1, 2, 0, 3)
    sel = O.page_select(heads(q), counts, c0 // 64, nP, n_sel)
    see = np.repeat(sel, 64, axis=2)[:, :, :J]
    cache = lambda x: heads(x[:, :J]).transpose(2, 0, 1, 3)  # noqa: E731
    a = O.paged_attention(heads(q), cache(K), cache(V), L.lut_att, see)
    A = O.if_neuron(a, L.theta["a"])[0]
    X1 = O.if_neuron(O.qbsm(A, L.W_o), L.theta["o"], resid=X)[0]
    U = O.qnl_lut(O.qbsm(X1, L.W_up), L.s_up, L.lut_act)
    Hs = O.if_neuron(U, L.theta["up"])[0]
    return O.if_neuron(O.qbsm(Hs, L.W_dn), L.theta["dn"], resid=X1)[0]


def run_paged(torch, B, m, lens, M, n_sel, spare=3):
    """Prompts of the given lengths, then one step of M rows each; returns the
    step's rows on the GPU and the oracle's, and what is needed to run again."""
    n = len(lens)
    dm = device_model(B, m)
    pages = B.Pages(n, n * M + spare, 6, 40)
    pre = pages.view(sum(lens) + 5)
    pm = B.PagedModel(dm, pages)
    pmv = pm.view(pre, head=False)
    rng = np.random.default_rng(len(lens))
    Xc = rng.random((m.T, pre.max_rows, m.d)) < 0.15
    Xb = rng.random((m.T, pages.max_rows, m.d)) < 0.15
    dev = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    B.nmdlm_page_plan(pre, dev([0] * n), dev(lens))
    ws = B.workspace(max(B.nmdlm_block_step_paged_workspace_size(pm, B.NMDLM_NO_HEAD),
                         B.nmdlm_block_step_paged_workspace_size(pmv, B.NMDLM_NO_HEAD)))
    xc, xb = (B.to_dev_bits(synth.pack_bits(x)) for x in (Xc, Xb))
    B.nmdlm_block_step_paged(pmv, B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, x_in=xc), ws, n_sel=n_sel)
    B.nmdlm_page_plan(pages, dev(lens), dev([M] * n))
    y = torch.zeros(m.T, pages.max_rows, m.d // 64, dtype=torch.int64, device="cuda")
    io = B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, x_in=xb, y_out=y)
    step = lambda **kw: B.nmdlm_block_step_paged(pm, io, ws, n_sel=n_sel, **kw)  # noqa: E731
    want = []
    r = 0
    for s, P in enumerate(lens):
        x, xs = Xc[:, r:r + P], Xb[:, s * M:(s + 1) * M]
        r += P
        K, V = ([np.zeros((m.T, P + M, m.d), dtype=bool) for _ in m.layers] for _ in range(2))
        for l, L in enumerate(m.layers):
            x = paged_layer(x, L, 0, n_sel, K[l], V[l], 0)
        for l, L in enumerate(m.layers):
            xs = paged_layer(xs, L, P, n_sel, K[l], V[l], P)
        want.append(xs)
    return step, y, np.concatenate(want, axis=1), (dm, pages, pre, pm, pmv, ws, xb)


@pytest.mark.parametrize("T,M,n_sel", [(4, 16, 1), (4, 1, 2), (3, 5, 0), (8, 4, 100)])
def test_step_over_selected_pages(T, M, n_sel):
    torch, B = need_gpu()
    m = small_model(T=T)
    step, y, want, keep = run_paged(torch, B, m, [200, 64, 30, 129], M, n_sel)
    step()
    torch.cuda.synchronize()
    got = synth.unpack_bits(B.from_dev_bits(y), m.d)[:, :want.shape[1]]
    assert_same(got, want, "spikes")


def test_step_in_a_graph():
    """Captured once, replayed with eager work between."""
    torch, B = need_gpu()
    m = small_model()
    step, y, want, keep = run_paged(torch, B, m, [100, 65], 8, 1)
    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        y.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = synth.unpack_bits(B.from_dev_bits(y), m.d)[:, :want.shape[1]]
        assert_same(got, want, "spikes")


def test_positions_past_the_table_and_ids_outside_it():
    torch, B = need_gpu()
    m = small_model(max_pos=70)
    dm = device_model(B, m)
    pages = B.Pages(1, 90, 2, 2)
    pm = B.PagedModel(dm, pages, head=False)
    dev = lambda a: torch.as_tensor(a, dtype=torch.int32).cuda()  # noqa: E731
    B.nmdlm_page_plan(pages, dev([0]), dev([80]))
    ws = B.workspace(B.nmdlm_block_step_paged_workspace_size(pm, B.NMDLM_NO_HEAD))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    tokens = torch.zeros(90, dtype=torch.int32, device="cuda")
    tokens[3] = m.V + 9
    B.nmdlm_block_step_paged(pm, B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, tokens=tokens, status=status), ws)
    torch.cuda.synchronize()
    assert int(status) == B.NMDLM_STATUS_TOKEN_CLAMPED | B.NMDLM_STATUS_BAD_REQUEST


@pytest.mark.parametrize("max_len,max_pos", [(192, 70), (70, 512)])
def test_generator_stops_at_the_last_position(max_len, max_pos):
    """70 positions, by the position table or by the caller's word (pages hold
    more): no block begins past them, and what the others get is unchanged."""
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model(max_pos=max_pos)
    g = PagedGenerator(device_model(B, m), 2, 8, max_len=max_len, pool=6, max_prompt_rows=128)
    ps = prompts_of([62, 40], m.V)
    with pytest.raises(ValueError, match="request 0"):
        g.admit({0: synth.random_tokens(9, 71, m.V)})
    g.admit({0: ps[0], 1: ps[1]})
    a = g.run_block(2, 4)
    free = g.pages.ring_state.tolist()
    with pytest.raises(ValueError, match="request 0"):
        g.run_block(2, 4)
    assert g.pages.ring_state.tolist() == free and g.ctx.tolist() == [70, 48]
    g.release([0])
    b = g.run_block(2, 4)
    assert_same(a[0].cpu().numpy(), O.generate(m, ps[0], 1, 8, 2, 4)[0], "up to the last position")
    assert_same(torch.cat([a[1], b[1]]).cpu().numpy(), O.generate(m, ps[1], 2, 8, 2, 4)[0], "the other")


@pytest.mark.parametrize("bad", [-1, 305, 2 ** 32 + 5])
def test_generator_refuses_ids_outside_the_table(bad):
    """None of the prompts is admitted, their pages go back, and the request
    that runs beside them goes on as before."""
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model()
    g = PagedGenerator(device_model(B, m), 3, 8, max_len=192, pool=6, max_prompt_rows=200)
    ps = prompts_of([30, 70, 40], m.V)
    g.admit({0: ps[0]})
    wrong = ps[1].astype(np.int64)
    wrong[69] = bad
    with pytest.raises(ValueError, match="ids"):
        g.admit({1: wrong, 2: ps[2]})
    assert g.live.tolist() == [True, False, False] and g.ctx.tolist() == [30, 0, 0]
    assert g.pages.held.tolist() == [1, 0, 0] and g.pages.ring_state.tolist()[1] == 5
    a = g.run_block(2, 4)
    assert_same(a[0].cpu().numpy(), O.generate(m, ps[0], 1, 8, 2, 4)[0], "the first")
    g.admit({1: ps[1]})
    b = g.run_block(2, 4)
    assert_same(b[1].cpu().numpy(), O.generate(m, ps[1], 1, 8, 2, 4)[0], "the second")


def test_workspace_of_a_step_without_a_selection():
    """As large as such a step needs: what lies behind is left alone, and the
    spikes are those of a step that selects every page."""
    torch, B = need_gpu()
    m = small_model()
    step, y, want, (dm, pages, pre, pm, pmv, ws, xb) = run_paged(torch, B, m, [200, 64, 30, 129], 16, 100)
    need = B.nmdlm_block_step_paged_workspace_size(pm, B.NMDLM_NO_HEAD | B.NMDLM_ALL_PAGES)
    assert need < B.nmdlm_block_step_paged_workspace_size(pm, B.NMDLM_NO_HEAD)
    room = torch.full((need + 4096,), 85, dtype=torch.uint8, device="cuda")
    room[:need] = 0
    io = B.step_io(0, 0, flags=B.NMDLM_NO_HEAD | B.NMDLM_ALL_PAGES, x_in=xb, y_out=y)
    B.nmdlm_block_step_paged(pm, io, room[:need])
    torch.cuda.synchronize()
    assert (room[need:] == 85).all()
    got = synth.unpack_bits(B.from_dev_bits(y), m.d)[:, :want.shape[1]]
    assert_same(got, want, "spikes")


def test_generator_with_a_selection():
    """A context of more pages than are selected: prompts see all of theirs, a
    block's rows choose.  Taking every page is the generator without selection."""
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model()
    ps = prompts_of([200, 70], m.V)
    ids = {}
    for n_sel in (None, 3, 1):
        g = PagedGenerator(device_model(B, m), 2, 8, max_len=320, pool=9, n_sel=n_sel)
        g.admit({0: ps[0], 1: ps[1]})
        keys = [k.clone() for k, _, _ in g.model.pools]
        out = g.run_block(2, 4)
        ids[n_sel] = out[0], out[1], keys
    assert_same(ids[None][0].cpu().numpy(), O.generate(m, ps[0], 1, 8, 2, 4)[0], "all pages")
    assert_same(ids[None][1].cpu().numpy(), O.generate(m, ps[1], 1, 8, 2, 4)[0], "the other")
    assert torch.equal(ids[3][0], ids[None][0]) and torch.equal(ids[3][1], ids[None][1])
    for n_sel in (3, 1):
        for a, b in zip(ids[n_sel][2], ids[None][2]):
            assert torch.equal(a, b)


def test_generator_over_a_view_of_a_model():
    """Some of a model's layers, with its tables and head."""
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import PagedGenerator

    m = small_model(n_layers=3)
    dm = device_model(B, m)
    ps = prompts_of([70], m.V)
    g = PagedGenerator(dm.view(0, 2, head=True), 1, 8, max_len=128, pool=2)
    g.admit({0: ps[0]})
    m.layers = m.layers[:2]
    assert_same(g.run_block(2, 4)[0].cpu().numpy(), O.generate(m, ps[0], 1, 8, 2, 4)[0], "ids")
