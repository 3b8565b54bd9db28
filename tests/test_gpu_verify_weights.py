"""Weights of tokens on the GPU: logits whose rounding is many exponents wide, the
exponentials' accuracy, equal distributions, draft logits that end with the drafts.  Ids
equal the oracle's, confidences to the tolerance of the other tests where no other is
derived."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from tests._gpu import assert_same, need_gpu
from tests.test_gpu_verify import make, same, same4, sample, verify

pytestmark = pytest.mark.gpu

# the largest logit, floats below it, temperature: exponents of -763, -954, -781, -1024 and
# -1024, where a float has no room for "700 temperatures below the largest"
NEAR = [(40.0, 2, 1e-8), (20.0, 1, 2e-9), (20000.0, 4, 1e-5), (2.0 ** 33 + 1024, 1, 1.0), (-2.0 ** 33, 1, 1.0)]


def near_equal(rng, M, V, top, steps):
    """Rows of the largest logit and the one `steps` floats below alone."""
    low = np.float32(top)
    for _ in range(steps):
        low = np.nextafter(low, np.float32(-np.inf))
    l = np.where(rng.random((M, V)) < 0.5, np.float32(top), low)
    l[:, 0] = top
    return l


@pytest.mark.parametrize("top, steps, tau", NEAR)
@pytest.mark.parametrize("V", [3000, 4099])
def test_sample_among_near_equal_logits(V, top, steps, tau):
    """Whole parts of ids whose exponents are 0 or below -700."""
    rng = np.random.default_rng([1, V])
    l, u = near_equal(rng, 8, V, top, steps), rng.random(8, dtype=np.float32)
    l[1, 1:] = l[1].min()                 # one id alone
    l[2, :2048], l[2, 2100] = l[2].min(), top   # parts without a largest one
    for t in (tau, 0.0):
        same(sample(l, t, u), O.token_sample(l, t, u))


@pytest.mark.parametrize("top, steps, tau", NEAR)
@pytest.mark.parametrize("chain", [True, False])
def test_verify_among_near_equal_logits(chain, top, steps, tau):
    rng = np.random.default_rng([2, steps])
    V, M = 4099, 12
    l, ql = near_equal(rng, M, V, top, steps), near_equal(rng, M, V, top, steps)
    draft, u = rng.integers(0, V, M), rng.random((M, 2), dtype=np.float32)
    cu = [0, 5, 6, 12]
    for q, taus in ((ql, (tau, tau)), (None, (tau, tau)), (ql, (1e30 * tau, tau)), (ql, (tau, 0.0))):
        same4(verify(l, q, draft, u, *taus, cu, chain), O.draft_verify(l, q, draft, u, *taus, cu, chain))


@pytest.mark.parametrize("V", [300, 32000])
@pytest.mark.parametrize("n", [1, 8])
def test_draft_logits_end_with_the_drafts(n, V):
    """Logits of the drafted rows alone through the C entry: the row behind them has none."""
    import ctypes as C

    torch, B = need_gpu()
    l, ql, draft, u, cu = make(n, [n + 1], V, spare=(0, 0))
    draft[n] = -1
    want = O.draft_verify(l, ql, draft, u, 0.8, 0.8, cu, True)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    t = [dev(l), dev(ql[:n]), dev(draft.astype(np.int32)), dev(u)]
    tok, acc = torch.zeros(n + 1, dtype=torch.int32, device="cuda"), torch.zeros(n + 1, dtype=torch.uint8, device="cuda")
    ws = B.workspace(B.nmdlm_draft_verify_workspace_size(n + 1, V))
    p = lambda x: C.c_void_p(x.data_ptr())  # noqa: E731
    for _ in range(2):
        assert B.load().nmdlm_draft_verify(p(t[0]), p(t[1]), n + 1, V, p(t[2]), p(t[3]), 0.8, 0.8, None, 1, 0, p(tok), p(acc),
                                           None, None, p(ws), ws.numel(), None) == B.NMDLM_OK
        torch.cuda.synchronize()
        assert_same(tok.cpu().numpy(), want[0], "tokens")
        assert_same(acc.cpu().numpy(), want[1], "accepted")


@pytest.mark.parametrize("tau", [0.1, 0.8, 1.0, 7.3, 250.0])
def test_weights_are_exponentials_in_float64(tau):
    """Two ids, the second drafted and taken (u = 0): its probability is e^x / (1 + e^x), x the
    exponent.  A weight errs by 4.6e-16 + 1.2e-16 |x|, the sum, the division and float64 of the
    reference by 2^-53 each.  The reference, in 64 bits of mantissa, adds |x| 2^-63."""
    M = 4000
    rng = np.random.default_rng(int(tau * 10))
    l = np.zeros((M, 2), np.float32)
    l[:, 0] = rng.normal(size=M) * tau
    l[:, 1] = l[:, 0] - (tau * np.concatenate([rng.random(M // 2) * 3, np.linspace(0, 680, M - M // 2)])).astype(np.float32)
    tok, acc, conf, _ = verify(l, None, np.ones(M, int), np.zeros((M, 2), np.float32), tau, tau, [0, M], False)
    assert (acc == 1).all() and (tok == 1).all()
    x = (l[:, 1].astype(np.longdouble) - l[:, 0]) / np.longdouble(tau)
    w = np.exp(x)
    want = w / (1 + w)
    bound = 4.6e-16 + 1.2e-16 * np.abs(x) + 3 * 2.0 ** -53 + np.abs(x) * 2.0 ** -63
    off = np.abs(conf / want - 1)
    assert (off <= bound).all(), (float((off / bound).max()), float(off.max()))


@pytest.mark.parametrize("V", [500, 33001])
def test_nothing_is_left_of_equal_distributions(V):
    """p is q and the draft an id that both rule out: the token is drawn from p."""
    rng = np.random.default_rng(V)
    l, _, draft, u, cu = make(21, [9, 8], V)
    draft[:] = rng.integers(0, V, len(draft))
    l[np.arange(len(l)), draft] = -np.inf
    for tau in (0.0, 0.3, 0.8):
        got = verify(l, l, draft, u, tau, tau, cu, False)
        want = O.draft_verify(l, l, draft, u, tau, tau, cu, False)
        same4(got, want)
        rows = slice(cu[0], cu[-1])
        assert_same(got[0][rows], O.token_sample(l[rows], tau, u[rows, 1])[0], "drawn")
