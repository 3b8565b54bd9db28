"""A step whose rows see the keys of a mask, and generation with drafted blocks,
against the oracle."""
import numpy as np
import pytest

from oracle import nmdlm_oracle as O
from tests import _masked as K
from tests._gpu import assert_same, need_gpu
from workloads import synth

pytestmark = pytest.mark.gpu


def model(seed, n_layers=2, T=4, H=2, d=128, V=64, max_pos=256):
    return synth.make_mdlm(seed, n_layers, d=d, H=H, F=256, V=V, T=T, max_pos=max_pos)


def caches(dm, l, n):
    """Keys and values of the first n cache rows of layer l, 0/1 [T][n][d]."""
    from paper_2607_24841_amd import binding as B

    layer = dm.layers[l]
    k = synth.unpack_bits(B.from_dev_bits(layer.k_cache), dm.d)[:, :n]
    v = synth.unpack_bits(B.from_dev_bits(layer.vt_cache.unsqueeze(-1)), 64)
    return k, v.transpose(0, 1, 3, 2).reshape(dm.T, -1, dm.d)[:, :n]


@pytest.mark.parametrize("T, H, d, C, n_docs, biased", [(4, 2, 128, 37, 0, False), (4, 2, 256, 64, 0, True),
                                                         (3, 3, 192, 0, 4, True), (8, 1, 128, 5, 3, False)])
def test_step_matches_oracle(T, H, d, C, n_docs, biased):
    """A step behind a context: drafted rows, or documents and rows of none."""
    torch, B = need_gpu()
    m = model(50 + C, T=T, H=H, d=d)
    rng = np.random.default_rng(C)
    if n_docs:
        r, pos = K.docs_mask([1, 9, 70, 20][:n_docs], 3)
        r[:, :2] += np.where(r[:, 1:2] > 0, C, 0)
    else:
        r, pos = K.draft_mask(C, 6)
    M, J = len(r), C + len(r)
    dm = B.DeviceModel.from_mdlm(m, J)
    emb = O.unpack_model_emb(m)
    kc, vc = O.new_caches(m.n_layers, T, dm.cache_cap, d)
    prompt = rng.integers(0, m.V, C)
    if C:
        O.prefill(O.block_input(prompt, np.arange(C), emb, m.pos_ch), m.layers, kc, vc)
        ids = torch.as_tensor(prompt.astype(np.int32)).cuda()   # the io holds addresses only
        B.nmdlm_block_step(dm, B.step_io(C, 0, flags=B.NMDLM_NO_HEAD, tokens=ids),
                           B.workspace(B.nmdlm_block_step_workspace_size(dm, C, B.NMDLM_NO_HEAD)))
    D = 5
    bias = [rng.integers(-60, 60, (H, 2 * D + 1)).astype(np.int8), None] if biased else None
    k_pos = np.concatenate([np.arange(C), pos])
    tokens, masked = rng.integers(0, m.V, M), rng.random(M) < 0.4
    dev = lambda a, t=np.int32: torch.from_numpy(np.ascontiguousarray(a.astype(t))).cuda()  # noqa: E731
    mask = B.Mask(dev(r), dev(pos), dev(k_pos), D)
    y = torch.zeros(T, M, d // 64, dtype=torch.int64, device="cuda")
    logits, pred = torch.zeros(M, m.V, device="cuda"), torch.zeros(M, dtype=torch.int32, device="cuda")
    tok, msk, chosen = dev(tokens), dev(masked, np.uint8), torch.zeros(5, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = B.workspace(B.nmdlm_block_step_masked_workspace_size(dm, M, J))
    tables = None if bias is None else [None if b is None else dev(b, np.int8) for b in bias]
    io = B.step_io(M, C, tokens=tok, masked=msk, k_unmask=5, y_out=y, logits=logits, pred=pred, unmasked_pos=chosen,
                   status=status)
    B.nmdlm_block_step_masked(dm, io, mask, ws, bias=tables)
    torch.cuda.synchronize()
    X = O.block_input(np.where(masked, m.mask_id, tokens), pos, emb, m.pos_ch)
    Y = O.masked_stack(X, m.layers, kc, vc, C, r, bias, pos, k_pos, D)
    assert_same(synth.unpack_bits(B.from_dev_bits(y), d), Y, "spikes")
    for l in range(m.n_layers):
        k, v = caches(dm, l, J)
        assert_same(k, kc[l][:, :J], f"keys of layer {l}")
        assert_same(v, vc[l][:, :J], f"values of layer {l}")
    want = O.head_logits(Y, m.W_head, m.scale)
    assert_same(logits.cpu().numpy(), want, "logits")
    p, conf = O.confidence(want)
    assert_same(pred.cpu().numpy(), p, "pred")
    t2, m2, ch = O.unmask(tokens, masked, p, conf, 5)
    assert_same(tok.cpu().numpy(), t2, "tokens")
    assert_same(msk.cpu().numpy().astype(bool), m2, "masked")
    assert int(status) == 0


def test_step_where_all_see_all_is_the_plain_step():
    torch, B = need_gpu()
    m = model(60)
    out = []
    for masked in (False, True):
        dm = B.DeviceModel.from_mdlm(m, 40)
        tok = torch.arange(40, dtype=torch.int32, device="cuda")
        y = torch.zeros(m.T, 40, m.d // 64, dtype=torch.int64, device="cuda")
        io = B.step_io(40, 0, flags=B.NMDLM_NO_HEAD, tokens=tok, y_out=y)
        if masked:
            mask = B.Mask(torch.tensor([[0, 40, 0, 0]] * 40, dtype=torch.int32, device="cuda"),
                          torch.arange(40, dtype=torch.int32, device="cuda"))
            ws = B.workspace(B.nmdlm_block_step_masked_workspace_size(dm, 40, 40, B.NMDLM_NO_HEAD))
            B.nmdlm_block_step_masked(dm, io, mask, ws)
        else:
            B.nmdlm_block_step(dm, io, B.workspace(B.nmdlm_block_step_workspace_size(dm, 40, B.NMDLM_NO_HEAD)))
        out.append((y, dm.layers[1].k_cache.clone(), dm.layers[1].vt_cache.clone()))
    for a, b in zip(*out):
        assert torch.equal(a, b)


def test_documents_of_one_step_are_those_of_steps_by_themselves():
    torch, B = need_gpu()
    m = model(61)
    rng = np.random.default_rng(1)
    docs = [rng.integers(0, m.V, n).astype(np.int32) for n in (30, 1, 65)]
    r, pos = K.docs_mask([len(x) for x in docs], 0)
    dm = B.DeviceModel.from_mdlm(m, len(r))
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a.astype(np.int32))).cuda()  # noqa: E731
    y = torch.zeros(m.T, len(r), m.d // 64, dtype=torch.int64, device="cuda")
    ws = B.workspace(B.nmdlm_block_step_masked_workspace_size(dm, len(r), len(r), B.NMDLM_NO_HEAD))
    ids = [dev(x) for x in [np.concatenate(docs)] + docs]
    B.nmdlm_block_step_masked(dm, B.step_io(len(r), 0, flags=B.NMDLM_NO_HEAD, tokens=ids[0], y_out=y),
                              B.Mask(dev(r), dev(pos)), ws)
    at = 0
    for x, t in zip(docs, ids[1:]):
        one = B.DeviceModel.from_mdlm(m, len(x))
        yo = torch.zeros(m.T, len(x), m.d // 64, dtype=torch.int64, device="cuda")
        B.nmdlm_block_step(one, B.step_io(len(x), 0, flags=B.NMDLM_NO_HEAD, tokens=t, y_out=yo),
                           B.workspace(B.nmdlm_block_step_workspace_size(one, len(x), B.NMDLM_NO_HEAD)))
        assert torch.equal(y[:, at:at + len(x)], yo)
        at += len(x)


def test_step_captured_and_replayed():
    """Every replay takes the ranges, positions and tokens that are there then."""
    torch, B = need_gpu()
    m = model(64)
    r, pos = K.draft_mask(0, 6)
    M = len(r)
    dm = B.DeviceModel.from_mdlm(m, M)
    rng = np.random.default_rng(5)
    emb = O.unpack_model_emb(m)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a.astype(np.int32))).cuda()  # noqa: E731
    mask, ids = B.Mask(dev(r), dev(pos)), dev(rng.integers(0, m.V, M))
    y = torch.zeros(m.T, M, m.d // 64, dtype=torch.int64, device="cuda")
    ws = B.workspace(B.nmdlm_block_step_masked_workspace_size(dm, M, M, B.NMDLM_NO_HEAD))
    io = B.step_io(M, 0, flags=B.NMDLM_NO_HEAD, tokens=ids, y_out=y)
    B.nmdlm_block_step_masked(dm, io, mask, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.nmdlm_block_step_masked(dm, io, mask, ws)
    for k in range(4):
        r2 = r.copy()
        if k:
            r2[:, 1] = np.maximum(r[:, 1] - k, 0)
        toks = rng.integers(0, m.V, M)
        mask.ranges.copy_(dev(r2).view(mask.ranges.shape))
        ids.copy_(dev(toks))
        kc, vc = O.new_caches(m.n_layers, m.T, dm.cache_cap, m.d)
        want = O.masked_stack(O.block_input(toks, pos, emb, m.pos_ch), m.layers, kc, vc, 0, r2, None, pos, pos, 0)
        for how in (graph.replay, lambda: B.nmdlm_block_step_masked(dm, io, mask, ws)):
            y.zero_()
            how()
            torch.cuda.synchronize()
            assert_same(synth.unpack_bits(B.from_dev_bits(y), m.d), want, f"replay {k}")


def test_positions_outside_the_table():
    torch, B = need_gpu()
    m = model(62, max_pos=64)
    dm = B.DeviceModel.from_mdlm(m, 4)
    i32 = dict(dtype=torch.int32, device="cuda")
    for pos, bad in (([0, 1, 2, 63], 0), ([0, 64, 2, 3], 1), ([0, 1, -1, 3], 1), ([2 ** 31 - 1, 1, 2, 3], 1)):
        status = torch.zeros(1, **i32)
        mask = B.Mask(torch.tensor([[0, 4, 0, 0]] * 4, **i32), torch.tensor(pos, **i32))
        ws = B.workspace(B.nmdlm_block_step_masked_workspace_size(dm, 4, 4, B.NMDLM_NO_HEAD))
        ids = torch.zeros(4, **i32)
        B.nmdlm_block_step_masked(dm, B.step_io(4, 0, flags=B.NMDLM_NO_HEAD, tokens=ids, status=status), mask, ws)
        assert int(status) == (B.NMDLM_STATUS_BAD_REQUEST if bad else 0), pos


def generator(B, m, draft, cap, block, tau, **kw):
    from paper_2607_24841_amd.generate import DraftedGenerator

    dm = B.DeviceModel.from_mdlm(m, cap)
    d = dm.view(0, draft, head=True) if isinstance(draft, int) else B.DeviceModel.from_mdlm(draft, cap)
    return DraftedGenerator(dm, d, block, tau, **kw)


def record(g, seed):
    """Numbers that the oracle can be given too."""
    import torch

    rng = np.random.default_rng(seed)
    log = []

    def numbers(*shape):
        log.append(rng.random(shape, dtype=np.float32))
        return torch.from_numpy(log[-1]).cuda()

    g.numbers = numbers
    return log


@pytest.mark.parametrize("draft", [1, 2, "own"])
@pytest.mark.parametrize("block, P", [(1, 1), (3, 2), (6, 11)])
def test_greedy_generation_is_left_to_right(draft, block, P):
    """At temperature 0 drafts change nothing: one token at a time gives the same."""
    torch, B = need_gpu()
    m = model(70)
    prompt = np.random.default_rng(P).integers(0, m.V, P)
    g = generator(B, m, model(71, n_layers=1) if draft == "own" else draft, 128, block, 0.0)
    assert g.run(prompt, 12) == O.left_to_right(m, prompt, 12)


def test_the_model_drafts_for_itself_with_success():
    """A draft that is the model accepts more than chance would."""
    torch, B = need_gpu()
    m = model(72)
    g = generator(B, m, 2, 256, 4, 0.0)
    g.start([3, 4, 5])
    found = sum(len(g.round()) for _ in range(10))
    assert found >= 10 and g.ctx == 2 + found and len(g.seq) == 3 + found


@pytest.mark.parametrize("draft, T", [(1, 4), ("own", 4), (2, 3)])
@pytest.mark.parametrize("tau, dtau", [(1.0, 1.0), (0.7, 1.2), (0.5, 0.0)])
def test_drawn_generation_matches_oracle(draft, T, tau, dtau):
    """The same numbers, the same rounds."""
    torch, B = need_gpu()
    m, other = model(73, T=T), model(74, n_layers=1, T=T)
    prompt = np.random.default_rng(T).integers(0, m.V, 7)
    block, rounds = 4, 5
    g = generator(B, m, other if draft == "own" else draft, 128, block, tau, draft_temperature=dtau)
    log = record(g, T)
    g.start(prompt)
    got = [g.round() for _ in range(rounds)]
    it = iter(log)
    want = O.drafted(m, other if draft == "own" else None, None if draft == "own" else draft, prompt, rounds, block,
                     tau, dtau, lambda *shape: next(it))
    assert got == want
    if tau == dtau == 1.0:   # where both kinds of round are likely
        assert any(len(x) > 1 for x in got) and any(len(x) <= block for x in got)


def test_same_seed_same_text():
    torch, B = need_gpu()
    m = model(75)
    a, b, c = (generator(B, m, 1, 128, 3, 1.0, seed=s).run([1, 2], 15) for s in (5, 5, 6))
    assert a == b != c


def test_generator_refuses():
    torch, B = need_gpu()
    from paper_2607_24841_amd.generate import DraftedGenerator

    m = model(76, n_layers=3, max_pos=64)
    dm = B.DeviceModel.from_mdlm(m, 64)
    for bad in (dict(block=0), dict(block=B.NMDLM_MAX_HEAD_M // 2), dict(draft=dm.view(1, 1, head=True)),
                dict(draft=B.DeviceModel.from_mdlm(model(77, V=65), 64))):
        with pytest.raises(ValueError):
            DraftedGenerator(dm, **{**dict(draft=dm.view(0, 1, head=True), block=4), **bad})
    g = DraftedGenerator(dm, dm.view(0, 1, head=True), 4, 0.0)
    with pytest.raises(ValueError):
        g.round()
    for prompt in ([], [64], [-1], np.zeros(60, int)):
        with pytest.raises(ValueError):
            g.start(prompt)
    with pytest.raises(ValueError):
        g.run([1], 200)
    assert g.run([1], 6) == O.left_to_right(m, [1], 6)   # and it goes on
    with pytest.raises(B.NmdlmError):
        B.nmdlm_block_step_masked(dm, B.step_io(11, 0, tokens=g.tokens, masked=g.masked), g.mask, g.ws)
    with pytest.raises(B.NmdlmError):
        B.nmdlm_block_step_masked(dm, B.step_io(4, 0, tokens=g.tokens, masked=g.masked), g.mask, g.ws, bias=[None])
