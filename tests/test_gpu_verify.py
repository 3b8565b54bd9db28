"""Tokens drawn from logits and verification of drafts on the GPU against the
oracle: ids equal, confidences to 1e-12 (sums of at most 2^17 weights in float64,
each of a few units of 2^-53 off, in another order: 2^17 * 2^-53 = 1.5e-11 at the
very most, and 2^-53 sqrt(2^17) = 4e-14 for independent roundings)."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from tests import _masked as K
from tests._gpu import assert_same, need_gpu

pytestmark = pytest.mark.gpu
CONF = 1e-12


def sample(l, tau, u):
    torch, B = need_gpu()
    M, V = l.shape
    tok = torch.full((M,), -7, dtype=torch.int32, device="cuda")
    conf = torch.full((M,), -7.0, dtype=torch.float64, device="cuda")
    B.nmdlm_token_sample(torch.from_numpy(l).cuda(), M, V, tau,
                         None if u is None else torch.from_numpy(u).cuda(), tok, conf=conf)
    return tok.cpu().numpy(), conf.cpu().numpy()


def same(got, want):
    assert_same(got[0], want[0], "tokens")
    np.testing.assert_allclose(got[1], want[1], rtol=CONF, atol=0)


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 255, 1000, 4097, 32000, 32767, 32769, 70001, 131072])
@pytest.mark.parametrize("tau", [0.0, 0.7, 1.0])
def test_sample(V, tau):
    rng = np.random.default_rng([1, V])
    l, u = K.logits(rng, 9, V), rng.random(9, dtype=np.float32)
    same(sample(l, tau, u), O.token_sample(l, tau, u))


def test_sample_covers_the_row():
    """u over its whole range: the first id at 0, the last just below 1, and
    borders between equal weights."""
    l = np.zeros((9, 8), np.float32)
    u = (np.arange(9) / 8).astype(np.float32)
    u[8] = np.float32(1) - np.float32(2 ** -24)
    tok, conf = sample(l, 1.0, u)
    assert list(tok) == [0, 1, 2, 3, 4, 5, 6, 7, 7]
    assert (conf == 0.125).all()


def test_sample_of_odd_values():
    """Infinities, NaN, rows that rule out everything, far logits, u out of range."""
    rng = np.random.default_rng(3)
    V = 777
    l = K.logits(rng, 12, V)
    l[0, :] = -np.inf
    l[1, :] = np.nan
    l[2, 5:] = -np.inf
    l[3, rng.random(V) < 0.5] = np.nan
    l[4, [9, 700]] = np.inf
    l[5, 400] = 3e38
    l[6, :] = -3e38
    l[7, :776] = -np.inf
    l[8] *= 1e4
    l[9] = -np.inf
    l[9, 12] = np.nan
    u = rng.random(12, dtype=np.float32)
    u[10], u[11] = 1.0, np.float32(0)
    for tau in (0.0, 0.5, 1e-3, 1e3):
        same(sample(l, tau, u), O.token_sample(l, tau, u))


def test_sample_without_numbers_at_temperature_0():
    rng = np.random.default_rng(4)
    l = K.logits(rng, 40, 500, spread=3)   # many equal largest: the first
    same(sample(l, 0.0, None), O.token_sample(l, 0.0, None))


def test_sample_follows_the_distribution():
    """Over a grid of u the counts of each id are its probability's."""
    rng = np.random.default_rng(5)
    n = 4096
    row = K.logits(rng, 1, 50)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)
    tok, _ = sample(np.repeat(row, n, 0), 1.0, u)
    w = O.token_weights(row[0], 1.0)[0]
    # an interval of length L holds L n - 1 to L n + 1 grid points
    assert (np.abs(np.bincount(tok, minlength=50) - n * w / w.sum()) <= 1 + 1e-6).all()


def verify(l, ql, draft, u, tau, dtau, cu, chain, counts=True, conf=True):
    torch, B = need_gpu()
    M, V = l.shape
    dev = lambda a, t=None: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    tok = torch.full((M,), -9, dtype=torch.int32, device="cuda")
    acc = torch.full((M,), 9, dtype=torch.uint8, device="cuda")
    cf = torch.full((M,), -9.0, dtype=torch.float64, device="cuda") if conf else None
    n = torch.full((len(cu) - 1,), -9, dtype=torch.int32, device="cuda") if counts else None
    B.nmdlm_draft_verify(dev(l), dev(ql), M, V, dev(draft.astype(np.int32)), dev(u), tau, dtau, tok, acc,
                         cu_rows=dev(np.asarray(cu, np.int32)), n_seq=len(cu) - 1, n_accepted=n, conf=cf, chain=chain)
    return tok.cpu().numpy(), acc.cpu().numpy(), cf.cpu().numpy() if conf else None, n.cpu().numpy() if counts else None


def same4(got, want):
    for g, w, name in zip(got, want, ("tokens", "accepted", "conf", "n_accepted")):
        if g is None:
            continue
        if name == "conf":
            np.testing.assert_allclose(g, w, rtol=CONF, atol=0)
        else:
            assert_same(g, w, name)


def make(seed, rows, V, tau=0.8, near=0.6, spare=(2, 3)):
    """Requests of `rows` rows, the last of some without a draft, rows before and behind."""
    rng = np.random.default_rng([7, seed])
    cu = spare[0] + np.concatenate([[0], np.cumsum(rows)])
    M = int(cu[-1]) + spare[1]
    l = K.logits(rng, M, V)
    ql = (l + rng.normal(size=l.shape) * near).astype(np.float32)
    draft = K.drafts(rng, ql, tau)
    for s in range(len(rows)):
        if s % 3 != 2 and rows[s]:
            draft[cu[s + 1] - 1] = [-1, V, 2 ** 31 - 1][s % 3]
    return l, ql, draft, rng.random((M, 2), dtype=np.float32), cu


@pytest.mark.parametrize("V", [1, 7, 64, 1000, 5003, 32000, 32771, 70001])
@pytest.mark.parametrize("chain", [True, False])
@pytest.mark.parametrize("certain", [False, True])
def test_verify(V, chain, certain):
    l, ql, draft, u, cu = make(V, [1, 5, 0, 9, 3], V)
    ql = None if certain else ql
    want = O.draft_verify(l, ql, draft, u, 0.8, 0.9, cu, chain)
    same4(verify(l, ql, draft, u, 0.8, 0.9, cu, chain), want)


@pytest.mark.parametrize("tau, dtau", [(0.0, 0.8), (0.8, 0.0), (0.0, 0.0), (1.3, 0.2)])
@pytest.mark.parametrize("certain", [False, True])
def test_verify_temperatures(tau, dtau, certain):
    l, ql, draft, u, cu = make(3, [4, 8, 8, 2], 900, tau=dtau, near=0.2)
    want = O.draft_verify(l, None if certain else ql, draft, u, tau, dtau, cu, True)
    same4(verify(l, None if certain else ql, draft, u, tau, dtau, cu, True), want)
    assert want[3].sum() > 0


def test_verify_long_requests():
    """More rows than a wave has lanes, refusals in any part."""
    l, ql, draft, u, cu = make(4, [70, 130, 64, 63, 1], 40, near=0.02)
    u[:, 0] **= 0.1
    for chain in (True, False):
        same4(verify(l, ql, draft, u, 0.8, 0.8, cu, chain), O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, chain))
    u[:, 0] = 0
    draft[draft < 0] = 0
    draft[draft >= 40] = 39
    got = verify(l, ql, draft, u, 0.8, 0.8, cu, True)
    assert list(got[3]) == [70, 130, 64, 63, 1]


def test_verify_same_distributions_take_all():
    l, _, draft, u, cu = make(5, [6, 6, 6], 3000)
    draft[:] = np.abs(draft) % 3000
    u[:, 0] = 1 - 2.0 ** -24
    got = verify(l, l, draft, u, 0.8, 0.8, cu, True)
    assert list(got[3]) == [6, 6, 6]


def test_verify_odd_values():
    """Ids that the draft or the target rules out, empty rows, NaN."""
    V = 300
    l, ql, draft, u, cu = make(6, [5, 5, 5, 5, 5], V)
    rng = np.random.default_rng(8)
    draft[:] = rng.integers(0, V, len(draft))
    l[2:7][:, rng.random(V) < 0.5] = -np.inf
    ql[7:12][:, rng.random(V) < 0.5] = -np.inf
    ql[9, draft[9]] = -np.inf
    l[12] = -np.inf
    ql[13] = -np.inf
    l[14], ql[14] = np.nan, np.nan
    l[15, 3] = np.inf
    ql[16, 9] = np.nan
    for chain in (True, False):
        for q in (ql, None):
            same4(verify(l, q, draft, u, 0.8, 0.8, cu, chain), O.draft_verify(l, q, draft, u, 0.8, 0.8, cu, chain))


def test_verify_of_one_request_without_offsets():
    torch, B = need_gpu()
    l, ql, draft, u, cu = make(9, [7], 500, spare=(0, 0))
    want = O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, True)
    tok = torch.zeros(7, dtype=torch.int32, device="cuda")
    acc = torch.zeros(7, dtype=torch.uint8, device="cuda")
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    B.nmdlm_draft_verify(g(l), g(ql), 7, 500, g(draft.astype(np.int32)), g(u), 0.8, 0.8, tok, acc)
    assert_same(tok.cpu().numpy(), want[0], "tokens")
    assert_same(acc.cpu().numpy(), want[1], "accepted")


@pytest.mark.parametrize("counts, conf", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("chain", [True, False])
def test_verify_optional_outputs(counts, conf, chain):
    l, ql, draft, u, cu = make(10, [4, 6], 128)
    same4(verify(l, ql, draft, u, 0.8, 0.8, cu, chain, counts, conf),
          O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, chain))


@pytest.mark.parametrize("off, qoff", [(0, 1), (1, 0), (2, 3), (3, 3)])
@pytest.mark.parametrize("V", [64, 1001, 33001])
def test_verify_logits_at_any_address(V, off, qoff):
    """Rows that begin at any float, the target's and the draft's at different ones."""
    torch, B = need_gpu()
    l, ql, draft, u, cu = make(14, [3, 4], V, spare=(0, 0))
    M = len(l)

    def put(a, o):
        t = torch.full((a.size + 8,), float("nan"), device="cuda")
        t[o:o + a.size] = torch.from_numpy(a.ravel()).cuda()
        return t[o:o + a.size].view(a.shape)

    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    tok = torch.zeros(M, dtype=torch.int32, device="cuda")
    acc = torch.zeros(M, dtype=torch.uint8, device="cuda")
    B.nmdlm_draft_verify(put(l, off), put(ql, qoff), M, V, g(draft.astype(np.int32)), g(u), 0.8, 0.8, tok, acc,
                         cu_rows=g(cu.astype(np.int32)), n_seq=2)
    want = O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, True)
    assert_same(tok.cpu().numpy(), want[0], "tokens")
    assert_same(acc.cpu().numpy(), want[1], "accepted")
    one = torch.zeros(M, dtype=torch.int32, device="cuda")
    B.nmdlm_token_sample(put(l, off), M, V, 0.8, g(u[:, 0]), one)
    assert_same(one.cpu().numpy(), O.token_sample(l, 0.8, u[:, 0])[0], "drawn")


def test_verified_tokens_follow_the_target():
    """Over many pairs of numbers a token comes as often as the target says,
    whatever the draft: counts within 6 standard deviations."""
    rng = np.random.default_rng(11)
    n, V = 20000, 12
    l = np.repeat(K.logits(rng, 1, V), n, 0)
    ql = np.repeat(K.logits(rng, 1, V), n, 0)
    draft = K.drafts(rng, ql, 1.0)
    u = rng.random((n, 2), dtype=np.float32)
    tok = verify(l, ql, draft, u, 1.0, 1.0, [0, n], False)[0]
    w = O.token_weights(l[0], 1.0)[0]
    p = w / w.sum()
    assert (np.abs(np.bincount(tok, minlength=V) - n * p) <= 6 * np.sqrt(n * p * (1 - p)) + 1).all()


def test_verify_captured_and_replayed():
    torch, B = need_gpu()
    l, ql, draft, u, cu = make(12, [5, 3, 9], 2000, spare=(0, 0))
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    t = dict(l=g(l), ql=g(ql), draft=g(draft.astype(np.int32)), u=g(u), cu=g(cu.astype(np.int32)))
    M = len(l)
    out = dict(tok=torch.zeros(M, dtype=torch.int32, device="cuda"), acc=torch.zeros(M, dtype=torch.uint8, device="cuda"),
               n=torch.zeros(3, dtype=torch.int32, device="cuda"), cf=torch.zeros(M, dtype=torch.float64, device="cuda"))

    def call():
        B.nmdlm_draft_verify(t["l"], t["ql"], M, 2000, t["draft"], t["u"], 0.8, 0.8, out["tok"], out["acc"],
                             cu_rows=t["cu"], n_seq=3, n_accepted=out["n"], conf=out["cf"])

    call()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            call()
    rng = np.random.default_rng(13)
    for _ in range(3):
        u = rng.random(u.shape, dtype=np.float32)
        t["u"].copy_(g(u))
        want = O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, True)
        for how in (graph.replay, call):
            for x in out.values():
                x.zero_()
            how()
            torch.cuda.synchronize()
            same4([out[k].cpu().numpy() for k in ("tok", "acc", "cf", "n")], want)


def test_workspace_on_another_stream():
    """Memory that the current stream's waiting work still reads is not taken for a call
    on another stream."""
    torch, B = need_gpu()
    l, ql, draft, u, cu = make(15, [4] * 40, 9000, spare=(0, 0))
    M, V = l.shape
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    t = [g(l), g(ql), g(draft.astype(np.int32)), g(u), g(cu.astype(np.int32)), g(u[:, 0])]
    tok, acc = torch.zeros(M, dtype=torch.int32, device="cuda"), torch.zeros(M, dtype=torch.uint8, device="cuda")
    cf, drawn = torch.zeros(M, dtype=torch.float64, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    calls = [(B.nmdlm_draft_verify_workspace_size(M, V),
              lambda: B.nmdlm_draft_verify(t[0], t[1], M, V, t[2], t[3], 0.8, 0.8, tok, acc, cu_rows=t[4],
                                           n_seq=len(cu) - 1, conf=cf, stream=side)),
             (B.nmdlm_token_sample_workspace_size(M, V),
              lambda: B.nmdlm_token_sample(t[0], M, V, 0.8, t[5], drawn, stream=side))]
    for size, call in calls:
        for _ in range(3):
            x = torch.full((size,), 7, dtype=torch.uint8, device="cuda")
            y = torch.zeros_like(x)
            torch.cuda.synchronize()
            torch.cuda._sleep(2_000_000)
            y.copy_(x)
            del x
            call()
            torch.cuda.synchronize()
            assert bool((y == 7).all())
    same4((tok.cpu().numpy(), acc.cpu().numpy(), cf.cpu().numpy(), None),
          O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, True))
    assert_same(drawn.cpu().numpy(), O.token_sample(l, 0.8, u[:, 0])[0], "drawn")


def test_two_calls_at_once():
    """On two streams, and two captured graphs."""
    torch, B = need_gpu()
    g = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    jobs = []
    for i in (0, 1):
        l, ql, draft, u, cu = make(16 + i, [6, 2, 30], 7000, spare=(0, 0))
        M = len(l)
        t = [g(l), g(ql), g(draft.astype(np.int32)), g(u), g(cu.astype(np.int32))]
        tok, acc = torch.zeros(M, dtype=torch.int32, device="cuda"), torch.zeros(M, dtype=torch.uint8, device="cuda")
        jobs.append((M, t, tok, acc, torch.cuda.Stream(), O.draft_verify(l, ql, draft, u, 0.7, 0.9, cu, True)))

    def call(job, stream=None):
        M, t, tok, acc = job[:4]
        B.nmdlm_draft_verify(t[0], t[1], M, 7000, t[2], t[3], 0.7, 0.9, tok, acc, cu_rows=t[4], n_seq=3, stream=stream)

    def check():
        torch.cuda.synchronize()
        for _, _, tok, acc, _, want in jobs:
            same4((tok.cpu().numpy(), acc.cpu().numpy(), None, None), want)
            tok.zero_(), acc.zero_()
        torch.cuda.synchronize()

    for _ in range(5):
        for job in jobs:
            call(job, job[4])
    check()
    graphs = []
    for job in jobs:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(job)
    for _ in range(3):
        for gr, job in zip(graphs, jobs):
            with torch.cuda.stream(job[4]):
                gr.replay()
        check()


def test_sample_of_many_rows():
    rng = np.random.default_rng(17)
    l, u = K.logits(rng, 65535, 5), rng.random(65535, dtype=np.float32)
    same(sample(l, 1.0, u), O.token_sample(l, 1.0, u))


@pytest.mark.parametrize("V", [1 << 20, 1100003])
def test_sample_of_a_long_list(V):
    """2^20 weights: 2^-53 sqrt(2^20) = 1.1e-13 for independent roundings."""
    rng = np.random.default_rng(18)
    l, u = K.logits(rng, 3, V), rng.random(3, dtype=np.float32)
    same(sample(l, 1.0, u), O.token_sample(l, 1.0, u))


def test_rejects_foreign_tensors():
    torch, B = need_gpu()
    l, u = torch.zeros(4, 10, device="cuda"), torch.zeros(4, device="cuda")
    tok = torch.zeros(4, dtype=torch.int32, device="cuda")
    for bad in (dict(logits=l.cpu()), dict(logits=l.double()), dict(logits=l.t()), dict(u=u[:3]), dict(u=u.cpu()),
                dict(tokens=tok.long()), dict(tokens=tok.cpu()), dict(temperature=-1.0), dict(temperature=float("nan")),
                dict(temperature=float("inf")), dict(u=None)):
        a = dict(logits=l, u=u, tokens=tok, temperature=1.0)
        a.update(bad)
        with pytest.raises(B.NmdlmError):
            B.nmdlm_token_sample(a["logits"], 4, 10, a["temperature"], a["u"], a["tokens"])
