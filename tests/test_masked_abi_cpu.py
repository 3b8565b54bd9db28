"""Refusals of the masked attention, of drawing tokens and of verifying drafts:
before any HIP call, so without a GPU; and the oracle's own pins."""
import ctypes as C
import os

import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from tests import _masked as K

torch = pytest.importorskip("torch")
from paper_2607_24841_amd import binding as B  # noqa: E402

FAKE = 1 << 40   # never dereferenced: every call below fails validation first
INVALID, UNSUPPORTED, WORKSPACE = B.NMDLM_ERR_INVALID_ARG, B.NMDLM_ERR_UNSUPPORTED, B.NMDLM_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        pytest.skip("libnmdlm.so not built")
    return B.load()


def attn(lib, ranges=FAKE, q_pos=FAKE, k_pos=FAKE, max_dist=8, no_mask=False, **kw):
    a = dict(q=FAKE, k=FAKE, v=FAKE, cap=4096, T=4, M=1, n_keys=4000, H=2, dh=64, lut=FAKE, bias=FAKE,
             a_out=FAKE, theta=100, s_out=FAKE, ws=None, nb=0)
    a.update(kw)
    m = B.MaskC(ranges, q_pos, k_pos, max_dist)
    return lib.nmdlm_bbm_attn_masked(a["q"], a["k"], a["v"], a["cap"], a["T"], a["M"], a["n_keys"], a["H"], a["dh"],
                                     a["lut"], None if no_mask else C.byref(m), a["bias"], a["a_out"], a["theta"],
                                     a["s_out"], a["ws"], a["nb"], None)


def test_attention_refusals(lib):
    for bad in (dict(q=None), dict(k=None), dict(v=None), dict(lut=None), dict(q=FAKE + 4), dict(k=FAKE + 4),
                dict(v=FAKE + 4), dict(a_out=FAKE + 2), dict(s_out=FAKE + 4), dict(a_out=None, s_out=None),
                dict(theta=0), dict(T=0), dict(M=0), dict(M=-1), dict(n_keys=0), dict(H=0), dict(dh=0),
                dict(no_mask=True), dict(ranges=None), dict(ranges=FAKE + 8), dict(q_pos=None), dict(k_pos=None),
                dict(q_pos=FAKE + 2), dict(max_dist=-1), dict(max_dist=B.NMDLM_MAX_DIST + 1), dict(n_keys=4097),
                dict(cap=4095, n_keys=4000)):
        assert attn(lib, **bad) == INVALID, bad
    for bad in (dict(T=9), dict(dh=96), dict(H=1025), dict(M=(1 << 17) + 1),
                dict(n_keys=(1 << 23) + 1, cap=1 << 24), dict(cap=64 * 2 ** 31)):
        assert attn(lib, **bad) == UNSUPPORTED, bad
    # a call of one row over 4000 keys is split: it needs its workspace
    need = lib.nmdlm_bbm_attn_masked_workspace_size(4, 1, 4000, 2, 64)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None, nb=need), dict(ws=FAKE + 8, nb=need), dict(ws=FAKE, nb=need - 1)):
        assert attn(lib, **bad) == WORKSPACE, bad


def test_attention_workspace_sizes(lib):
    f = lib.nmdlm_bbm_attn_masked_workspace_size
    assert f(4, 4096, 4096, 16, 128) == 0       # rows enough without splits
    for bad in ((0, 1, 1, 1, 64), (9, 1, 1, 1, 64), (4, 0, 1, 1, 64), (4, 1, 0, 1, 64), (4, 1, 1, 0, 64),
                (4, 1, 1, 1, 96), (4, 1 << 18, 1, 1, 64), (4, 1, (1 << 23) + 1, 1, 64)):
        assert f(*bad) == 0, bad


def test_sample_refusals(lib):
    def call(l=FAKE, M=4, V=100, tau=1.0, u=FAKE, tok=FAKE, conf=None, ws=FAKE, nb=1 << 20):
        return lib.nmdlm_token_sample(l, M, V, tau, u, tok, conf, ws, nb, None)
    for bad in (dict(l=None), dict(tok=None), dict(u=None), dict(M=0), dict(V=0), dict(tau=-0.5),
                dict(tau=float("nan")), dict(tau=float("inf")), dict(l=FAKE + 2), dict(u=FAKE + 1),
                dict(tok=FAKE + 2), dict(conf=FAKE + 4)):
        assert call(**bad) == INVALID, bad
    assert call(V=B.NMDLM_MAX_SAMPLE_V + 1) == UNSUPPORTED
    assert call(M=B.NMDLM_MAX_SAMPLE_M + 1) == UNSUPPORTED
    need = lib.nmdlm_token_sample_workspace_size(4, 100)
    assert need > 0 and need % 256 == 0
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(nb=need - 1)):
        assert call(**bad) == WORKSPACE, bad
    for f in (lib.nmdlm_token_sample_workspace_size, lib.nmdlm_draft_verify_workspace_size):
        for bad in ((0, 5), (5, 0), (-1, 5), (1 << 16, 5), (5, (1 << 24) + 1)):
            assert f(*bad) == 0


def test_verify_refusals(lib):
    def call(l=FAKE, q=FAKE, M=4, V=100, draft=FAKE, u=FAKE, tau=1.0, dtau=1.0, cu=FAKE, n=2, flags=0, tok=FAKE,
             acc=FAKE, n_acc=None, conf=None, ws=FAKE, nb=1 << 20):
        return lib.nmdlm_draft_verify(l, q, M, V, draft, u, tau, dtau, cu, n, flags, tok, acc, n_acc, conf, ws, nb,
                                      None)
    for bad in (dict(l=None), dict(draft=None), dict(u=None), dict(tok=None), dict(acc=None), dict(M=0), dict(V=0),
                dict(n=0), dict(cu=None, n=2), dict(flags=2), dict(tau=-1.0), dict(dtau=-1.0),
                dict(dtau=float("nan")), dict(l=FAKE + 1), dict(q=FAKE + 2), dict(draft=FAKE + 2), dict(u=FAKE + 2),
                dict(cu=FAKE + 2), dict(tok=FAKE + 1), dict(n_acc=FAKE + 1), dict(conf=FAKE + 4)):
        assert call(**bad) == INVALID, bad
    assert call(V=B.NMDLM_MAX_SAMPLE_V + 1) == UNSUPPORTED
    assert call(n=B.NMDLM_MAX_PLAN_ROWS + 1) == UNSUPPORTED
    need = lib.nmdlm_draft_verify_workspace_size(4, 100)
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(nb=need - 1)):
        assert call(**bad) == WORKSPACE, bad


def test_binding_refuses_host_tensors_and_wrong_masks():
    z = torch.zeros
    with pytest.raises(B.NmdlmError):
        B.nmdlm_token_sample(z(2, 5), 2, 5, 1.0, z(2), z(2, dtype=torch.int32))
    with pytest.raises(B.NmdlmError):
        B.Mask(z(3, 2, dtype=torch.int32))
    with pytest.raises(B.NmdlmError):
        B.Mask(z(3, 4, dtype=torch.int64))
    with pytest.raises(B.NmdlmError):
        B.Mask(z(3, 4, dtype=torch.int32), q_pos=z(2, dtype=torch.int32))
    m = B.Mask(z(3, 4, dtype=torch.int32), q_pos=z(3, dtype=torch.int32))
    for M, biased in ((4, False), (3, True)):
        with pytest.raises(B.NmdlmError):
            m.check("x", M, 10, biased)


def test_oracle_of_the_mask():
    """All keys: the plain attention; a document alone: that attention over its keys."""
    rng = np.random.default_rng(0)
    Q, Kc, V = (rng.random((2, n, 128)) < 0.3 for n in (6, 50, 50))
    lut = np.sort(rng.integers(1, 256, 256))
    full = O.masked_attention(Q, Kc, V, 2, lut, [[0, 50, 0, 0]] * 6)
    assert (full == O.bbm_attention(Q, Kc, V, 50, 2, lut)).all()
    two = O.masked_attention(Q, Kc, V, 2, lut, [[0, 20, 30, 50]] * 6)
    both = np.r_[0:20, 30:50]
    assert (two == O.bbm_attention(Q, Kc[:, both], V[:, both], 40, 2, lut)).all()
    assert not O.masked_attention(Q, Kc, V, 2, lut, [[9, 9, 5, 2]] * 6).any()
    # a bias of a distance that no pair has changes nothing; a shift of the table is a constant bias
    b = np.full((2, 3), 5)
    pos = np.zeros(50, int)
    shifted = np.r_[lut[5:], np.full(5, lut[-1])]
    assert (O.masked_attention(Q, Kc, V, 2, lut, [[0, 50, 0, 0]] * 6, b, pos[:6], pos, 1)
            == O.bbm_attention(Q, Kc, V, 50, 2, shifted)).all()


def test_oracle_of_the_draw():
    """The draw over all numbers has the distribution's lengths, and drafts that are
    verified come out as the target's."""
    rng = np.random.default_rng(1)
    l = K.logits(rng, 1, 20)[0]
    w = O.token_weights(l, 0.9)[0]
    p = w / w.sum()
    u = (np.arange(4000) + 0.5) / 4000
    got = np.bincount([O.draw_token(w, x) for x in u], minlength=20)
    assert (np.abs(got - 4000 * p) <= 1 + 1e-9).all()
    ql = K.logits(rng, 1, 20)[0]
    wq = O.token_weights(ql, 1.0)[0]
    q = wq / wq.sum()
    # the sum over drafts of q(x) P(out = v | x) is p(v): the acceptances and the residual in closed form
    take = np.minimum(1.0, p / q)
    left = np.maximum(p - q, 0)
    assert np.allclose(q * take + (q * (1 - take)).sum() * left / left.sum(), p)


def test_masked_step_refusals(lib):
    layers = (B.Layer * 1)(B.Layer(FAKE, FAKE, FAKE, FAKE, 200, 200, 200, 200, 200, 200, 200, 4, FAKE, FAKE, FAKE, FAKE))

    def call(flags=B.NMDLM_NO_HEAD, M=16, C_=512, ranges=FAKE, q_pos=FAKE, k_pos=FAKE, dist=4, bias=None, nb=1 << 30,
             ws=FAKE, no_mask=False, emb=FAKE, **io):
        m = B.Model(1, 1024, 16, 4096, 32000, 4, 576, 64, layers, emb, FAKE, None, None)
        step = B.step_io(M, C_, flags=flags, tokens=FAKE, **io)
        mask = B.MaskC(ranges, q_pos, k_pos, dist)
        table = (C.c_void_p * 1)(bias) if bias else None
        return lib.nmdlm_block_step_masked(C.byref(m), None if no_mask else C.byref(mask), table, C.byref(step), ws, nb, None)
    for bad in (dict(no_mask=True), dict(ranges=None), dict(ranges=FAKE + 4), dict(q_pos=None), dict(emb=None),
                dict(bias=FAKE, k_pos=None), dict(bias=FAKE, dist=-1), dict(bias=FAKE, dist=2000), dict(M=0),
                dict(C_=-1), dict(C_=561), dict(flags=0), dict(n_seq=-1)):
        assert call(**bad) == INVALID, bad
    assert call(n_seq=2) == UNSUPPORTED
    assert call(M=1 << 18) == UNSUPPORTED
    m = B.Model(1, 1024, 16, 4096, 32000, 4, 576, 64, layers, FAKE, FAKE, None, None)
    f = lambda M, n: lib.nmdlm_block_step_masked_workspace_size(C.byref(m), M, n, B.NMDLM_NO_HEAD)  # noqa: E731
    need = f(16, 528)
    assert need > 0
    for bad in (dict(ws=None), dict(ws=FAKE + 8), dict(nb=need - 1)):
        assert call(**bad) == WORKSPACE, bad
    assert f(0, 5) == f(5, 4) == f(5, 0) == 0
    sizes = [f(16, n) for n in range(16, 40000, 97)]
    assert sizes == sorted(sizes)     # does not fall as the keys grow


def test_masked_step_refuses_misaligned_buffers(lib):
    layers = (B.Layer * 1)(B.Layer(FAKE, FAKE, FAKE, FAKE, 200, 200, 200, 200, 200, 200, 200, 4, FAKE, FAKE, FAKE, FAKE))
    m = B.Model(1, 1024, 16, 4096, 32000, 4, 576, 64, layers, FAKE, FAKE, None, None)
    mask = B.MaskC(FAKE, FAKE, FAKE, 4)
    for name, off in [("tokens", 2), ("logits", 2), ("pred", 1), ("unmasked_pos", 2), ("status", 1), ("x_in", 4),
                      ("y_out", 4), ("conf", 4), ("stats", 4)]:
        io = B.step_io(16, 512, flags=B.NMDLM_NO_HEAD, **{"tokens": FAKE, name: FAKE + off})
        assert lib.nmdlm_block_step_masked(C.byref(m), C.byref(mask), None, C.byref(io), FAKE, 1 << 30, None) == INVALID, name
