"""Masked attention on the GPU against the oracle: integers, so equal bit for
bit."""
import numpy as np
import pytest

from tests import _masked as K
from tests._gpu import assert_same, need_gpu

pytestmark = pytest.mark.gpu


def check(c, **kw):
    torch, B = need_gpu()
    dev = K.Device(torch, B, c)
    dev.run(**kw)
    torch.cuda.synchronize()
    a, s = K.attention(c)
    if kw.get("cur", True):
        assert_same(dev.cur.cpu().numpy(), a, "currents")
    if kw.get("spk", True):
        assert_same(dev.spikes(), s, "spikes")
    return dev


@pytest.mark.parametrize("T", [1, 2, 3, 4, 5, 8])
@pytest.mark.parametrize("dh", [64, 128])
def test_drafted_rows(T, dh):
    r, pos = K.draft_mask(70, 5)
    check(K.make_case(T, r, pos, 82, T=T, H=2, dh=dh))


@pytest.mark.parametrize("M, ctx", [(1, 0), (1, 63), (1, 64), (1, 3000), (2, 130), (3, 61), (15, 600), (17, 2000),
                                    (33, 100), (64, 0), (65, 40)])
@pytest.mark.parametrize("max_dist", [None, 0, 20, 1024])
def test_causal_rows(M, ctx, max_dist):
    pos = ctx + np.arange(M)
    r = np.stack([0 * pos, pos + 1, 0 * pos, 0 * pos], 1)
    check(K.make_case(M + ctx, r, pos, ctx + M, H=3, max_dist=max_dist))


@pytest.mark.parametrize("seed", range(12))
def test_any_ranges(seed):
    """Empty, reversed, overlapping and out-of-bounds ranges, positions in any order."""
    rng = np.random.default_rng([5, seed])
    M, J = int(rng.integers(1, 90)), int(rng.integers(1, 700))
    r, pos = K.random_mask(rng, M, J)
    check(K.make_case(seed, r, pos, J, T=int(rng.integers(1, 9)), H=int(rng.integers(1, 6)),
                      dh=int(rng.choice([64, 128])), max_dist=[None, 7, 300][seed % 3],
                      k_pos=rng.integers(0, 2 * J, size=J)))


@pytest.mark.parametrize("S", [1, 7, 32, 200])
def test_blocks(S):
    r, pos = K.blocks_mask(150, S)
    check(K.make_case(S, r, pos, 300, T=3, H=2, dh=128, max_dist=30, k_pos=pos))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("max_dist", [None, 20])
def test_tiles_of_32_rows(dh, max_dist):
    """Rows enough for 32 a wave: drafted, ragged, empty and unordered ones."""
    rng = np.random.default_rng(dh)
    r, pos = K.docs_mask([100, 3, 77], 93)
    r[150:200], pos[150:200] = K.random_mask(rng, 50, 400)
    assert K.route(8, len(r), 400, 16).tile == 32
    check(K.make_case(dh, r, pos, 400, T=8, H=16, dh=dh, max_dist=max_dist))


@pytest.mark.parametrize("H", [1, 5, 9, 16])
def test_many_tiles(H):
    """Tiles enough to go to the dies in turn, with heads in groups of unequal size."""
    r, pos = K.docs_mask([40] * (40 if H > 8 else 32), 7)
    check(K.make_case(H, r, pos, len(r), T=1, H=H, max_dist=5, k_pos=pos))


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("max_dist", [None, 33])
@pytest.mark.parametrize("T, M, n_keys, H, tile, heads", [(4, 1, 300, 2, 1, False), (4, 2, 3000, 2, 1, True),
                                                          (4, 3, 300, 2, 16, False), (2, 12, 5000, 1, 16, True),
                                                          (3, 30, 3000, 11, 32, True), (4, 40, 3500, 9, 32, True),
                                                          (2, 1, 9000, 13, 1, True), (8, 70, 2600, 3, 32, True)])
def test_routes_of_small_calls(T, M, n_keys, H, tile, heads, max_dist, dh):
    """The kernels that the sizes of these tests reach, heads that do not fill a workgroup."""
    r = K.route(T, M, n_keys, H)
    assert (r.tile, r.heads) == (tile, heads)
    pos = n_keys - M + np.arange(M)
    ranges = np.stack([0 * pos, pos + 1, 0 * pos, 0 * pos], 1)
    ranges[M // 2] = 0   # sees nothing
    ranges[-1] = 70, 70 + n_keys // 3, n_keys - 5, n_keys
    check(K.make_case(M, ranges, pos, n_keys, T=T, H=H, dh=dh, max_dist=max_dist))


def test_one_split_of_several():
    """A route of several splits whose rows see too little for more than one, or nothing."""
    assert K.route(4, 20, 4000, 2).splits > 4
    for r in ((0, 0, 0, 0), (100, 130, 3900, 3990), (0, 4000, 0, 0)):
        check(K.make_case(1, np.tile([r], (20, 1)), np.full(20, 4000), 4000, max_dist=8))


def test_documents_and_rows_of_none():
    r, pos = K.docs_mask([1, 64, 63, 65, 2, 130, 7], 20)
    c = K.make_case(1, r, pos, len(r), H=5, max_dist=10, k_pos=pos)
    dev = check(c)
    assert not dev.spk[:, -20:].any() and not dev.cur[:, -20:].any()


def test_window_and_first_keys():
    r, pos = K.window_mask(1000, 40, 90)
    check(K.make_case(2, r, pos, 1040, dh=128))


def test_nothing_seen_at_all():
    check(K.make_case(3, np.zeros((21, 4)), np.zeros(21), 500, max_dist=3))


def test_ranges_at_the_ends_of_int32():
    big = 2 ** 31 - 1
    r = np.array([[-big - 1, big, 5, 4], [big, -big - 1, -7, big], [3, 9, big, big], [0, 1, -big, 1]])
    pos = np.array([-big - 1, big, 0, big])
    check(K.make_case(4, r, pos, 130, max_dist=9, k_pos=np.linspace(-big, big, 130).astype(np.int64)))


@pytest.mark.parametrize("cur, spk", [(True, False), (False, True)])
def test_one_output(cur, spk):
    r, pos = K.draft_mask(500, 9)
    dev = check(K.make_case(5, r, pos, 520), cur=cur, spk=spk)
    assert (dev.spk == -1).all() if not spk else (dev.cur == -9).all()


def test_zero_weights_and_full_weights():
    """Tables of 0 (no current) and of 255 alone (plain means)."""
    r, pos = K.draft_mask(300, 9)
    for v in (0, 255):
        c = K.make_case(6, r, pos, 320)
        c.lut = np.full(256, v, np.uint8)
        check(c)


def test_all_spikes():
    r, pos = K.draft_mask(300, 9)
    c = K.make_case(7, r, pos, 320, dh=128, rate=1.0, max_dist=40)
    check(c)


def test_long_context():
    """More than 65535 keys: sums beyond 24 bits, and many splits."""
    for M in (1, 18):
        pos = 70000 + np.arange(M)
        r = np.stack([0 * pos, pos + 1, 0 * pos, 0 * pos], 1)
        check(K.make_case(8, r, pos, 70000 + M, T=2, H=1, rate=0.5, max_dist=64))


def test_same_as_plain_attention():
    """All rows see all keys: nmdlm_bbm_attn."""
    torch, B = need_gpu()
    r = np.tile([[0, 333, 0, 0]], (33, 1))
    c = K.make_case(9, r, np.zeros(33), 333, H=4)
    dev = check(c)
    spk = torch.zeros_like(dev.spk)
    ws = B.workspace(B.nmdlm_bbm_attn_workspace_size(c.T, c.M, c.H, c.dh))
    B.nmdlm_bbm_attn(dev.q, dev.k, dev.v, c.cap, c.T, c.M, 300, c.H, c.dh, dev.lut, theta_a=c.theta, s_out=spk, ws=ws)
    assert torch.equal(spk, dev.spk)


def test_captured_and_replayed():
    """A captured call reads the mask anew at each replay, between eager calls."""
    torch, B = need_gpu()
    r, pos = K.draft_mask(600, 7)
    c = K.make_case(10, r, pos, 616, max_dist=16)
    dev = K.Device(torch, B, c)
    dev.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            dev.run()
    for k in (0, 1, 2):
        c.ranges = np.maximum(c.ranges - 40 * k, 0)
        dev.mask.ranges.copy_(torch.from_numpy(c.ranges))
        g.replay()
        torch.cuda.synchronize()
        a, s = K.attention(c)
        assert_same(dev.cur.cpu().numpy(), a, f"replay {k}")
        assert_same(dev.spikes(), s, f"replay {k}")
        dev.run()
        torch.cuda.synchronize()
        assert_same(dev.spikes(), s, f"eager {k}")


def test_two_streams():
    """Two calls at once with workspaces of their own."""
    torch, B = need_gpu()
    cases = []
    for i in (0, 1):
        r, pos = K.draft_mask(2000 + i, 6)
        cases.append(K.make_case(20 + i, r, pos, 2014 + i))
    devs = [K.Device(torch, B, c) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in devs]
    for _ in range(5):
        for d, s in zip(devs, streams):
            d.run(stream=s)
    torch.cuda.synchronize()
    for c, d in zip(cases, devs):
        assert_same(d.spikes(), K.attention(c)[1], "spikes")


def test_rejects_foreign_tensors():
    torch, B = need_gpu()
    r, pos = K.draft_mask(50, 3)
    c = K.make_case(30, r, pos, 58, max_dist=4)
    dev = K.Device(torch, B, c)
    for name in ("q", "k", "v", "lut", "bias", "cur", "spk"):
        keep = getattr(dev, name)
        setattr(dev, name, keep.cpu())
        with pytest.raises(B.NmdlmError):
            dev.run()
        setattr(dev, name, keep)
    dev.run()
