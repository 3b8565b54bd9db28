"""Refusals of the paged calls, before any HIP call (no GPU)."""
import ctypes as C
import os

import pytest

torch = pytest.importorskip("torch")
from paper_2607_24841_amd import binding as B  # noqa: E402

FAKE = 1 << 40
pytestmark = pytest.mark.skipif(not os.path.exists(B.LIB_PATH), reason="libnmdlm.so not built")
INVALID, UNSUPPORTED, WORKSPACE = B.NMDLM_ERR_INVALID_ARG, B.NMDLM_ERR_UNSUPPORTED, B.NMDLM_ERR_WORKSPACE


def pages(**kw):
    a = dict(n_seq=3, max_rows=40, max_pages=5, pool=9, table=FAKE, held=FAKE, ring=FAKE, ring_state=FAKE,
             cu_rows=FAKE, slot=FAKE, pos=FAKE, index=FAKE, index_bytes=1 << 40)
    a.update(kw)
    return B.PagesC(*[a[n] for n, _ in B.PagesC._fields_])


def plan(p=None, ctx=FAKE, new=FAKE):
    return B.load().nmdlm_page_plan(C.byref(p if p is not None else pages()), ctx, new, None, None)


def store(p=None, **kw):
    a = dict(k=FAKE, v=FAKE, T=4, H=2, dh=64, kp=FAKE, vp=FAKE, cnt=FAKE)
    a.update(kw)
    return B.load().nmdlm_page_store(C.byref(p if p is not None else pages()), *a.values(), None)


def select(p=None, **kw):
    a = dict(q=FAKE, T=4, H=2, dh=64, cnt=FAKE, n_sel=2, sel=FAKE, ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return B.load().nmdlm_page_select(C.byref(p if p is not None else pages()), *a.values(), None)


def attn(p=None, **kw):
    a = dict(q=FAKE, T=4, H=2, dh=64, kp=FAKE, vp=FAKE, lut=FAKE, sel=None, a_out=FAKE, theta=100, s_out=FAKE,
             ws=FAKE, ws_bytes=1 << 40)
    a.update(kw)
    return B.load().nmdlm_bbm_attn_paged(C.byref(p if p is not None else pages()), *a.values(), None)


CALLS = [plan, store, select, attn]


@pytest.mark.parametrize("call", CALLS)
def test_plan_arguments(call):
    for name in ("n_seq", "max_rows", "max_pages", "pool"):
        assert call(pages(**{name: 0})) == INVALID, name
        assert call(pages(**{name: -5})) == INVALID, name
    for name in ("table", "held", "ring", "ring_state", "cu_rows", "slot", "pos", "index"):
        assert call(pages(**{name: None})) == INVALID, name
    assert call(pages(slot=FAKE + 4)) == INVALID
    assert call(pages(index=FAKE + 8)) == INVALID
    assert call(pages(table=FAKE + 2)) == INVALID
    assert call(pages(n_seq=B.NMDLM_MAX_REQUESTS + 1)) == UNSUPPORTED
    assert call(pages(max_rows=B.NMDLM_MAX_PLAN_ROWS + 1)) == UNSUPPORTED
    assert call(pages(max_pages=B.NMDLM_MAX_PAGES + 1)) == UNSUPPORTED
    assert call(pages(pool=B.NMDLM_MAX_POOL + 1)) == UNSUPPORTED
    need = B.load().nmdlm_page_index_bytes(3, 40)
    assert call(pages(index_bytes=need - 1)) == WORKSPACE


def test_null_plan():
    assert B.load().nmdlm_page_plan(None, FAKE, FAKE, None, None) == INVALID
    assert plan(ctx=None) == INVALID
    assert plan(new=None) == INVALID


@pytest.mark.parametrize("call", CALLS[1:])
def test_sizes(call):
    for name in ("T", "H", "dh"):
        assert call(**{name: 0}) == INVALID, name
    assert call(T=9) == UNSUPPORTED
    assert call(dh=96) == UNSUPPORTED
    assert call(H=1025) == UNSUPPORTED                       # H*dh beyond 65536
    assert call(pages(max_rows=(1 << 17) + 1)) == UNSUPPORTED  # T*max_rows beyond 2^19


def test_pointers():
    for name in ("k", "v", "kp", "vp", "cnt"):
        assert store(**{name: None}) == INVALID, name
        assert store(**{name: FAKE + 8}) == INVALID, name
    for name in ("q", "cnt"):
        assert select(**{name: None}) == INVALID, name
        assert select(**{name: FAKE + 8}) == INVALID, name
    assert select(sel=None) == INVALID
    assert select(n_sel=-1) == INVALID
    wide = pages(max_pages=2000)
    need = B.load().nmdlm_page_select_workspace_size(C.byref(wide), 4, 2, 64)
    assert need > 0
    assert select(wide, ws=None) == WORKSPACE
    assert select(wide, ws=FAKE + 16) == WORKSPACE
    assert select(wide, ws_bytes=need - 1) == WORKSPACE
    for name in ("q", "kp", "vp"):
        assert attn(**{name: None}) == INVALID, name
        assert attn(**{name: FAKE + 8}) == INVALID, name
    assert attn(lut=None) == INVALID
    assert attn(a_out=None, s_out=None) == INVALID
    assert attn(theta=0) == INVALID
    need = B.load().nmdlm_bbm_attn_paged_workspace_size(C.byref(pages(max_pages=500)), 4, 2, 64)
    assert need > 0
    assert attn(pages(max_pages=500), ws_bytes=need - 1) == WORKSPACE
    assert attn(pages(max_pages=500), ws=None) == WORKSPACE


def test_sizes_of_invalid_calls_are_zero():
    lib = B.load()
    assert lib.nmdlm_page_index_bytes(0, 4) == 0
    assert lib.nmdlm_page_index_bytes(4, 0) == 0
    assert lib.nmdlm_page_index_bytes(B.NMDLM_MAX_REQUESTS + 1, 4) == 0
    assert lib.nmdlm_page_index_bytes(4, B.NMDLM_MAX_PLAN_ROWS + 1) == 0
    for f in (lib.nmdlm_page_select_workspace_size, lib.nmdlm_bbm_attn_paged_workspace_size):
        assert f(C.byref(pages()), 9, 2, 64) == 0
        assert f(C.byref(pages()), 4, 2, 32) == 0
        assert f(None, 4, 2, 64) == 0


def test_binding_checks_its_tensors():
    p = B.Pages(2, 10, 3, 7, device="cpu")
    assert p.ring.tolist() == list(range(7)) and p.ring_state.tolist() == [0, 7] and p.table.shape == (2, 3)
    k = torch.zeros(4, 10, 2, dtype=torch.int64)
    kp, vp, cnt = p.pools(4, 2, 64)
    ok = dict(k=k, v=k, T=4, H=2, dh=64, k_pages=kp, v_pages=vp, key_counts=cnt)
    for bad in (dict(k=k[:3]), dict(v=k.int()), dict(k_pages=kp[:-1]), dict(v_pages=vp.transpose(1, 2)),
                dict(key_counts=cnt[1:])):
        with pytest.raises(B.NmdlmError, match=next(iter(bad))):
            B.nmdlm_page_store(p, **{**ok, **bad})
    with pytest.raises(B.NmdlmError, match="ctx"):
        B.nmdlm_page_plan(p, torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(B.NmdlmError, match="not on a GPU"):
        B.nmdlm_page_store(p, **ok)
    with pytest.raises(B.NmdlmError):
        B.Pages(0, 10, 3, 7, device="cpu")


def test_step_over_pages_argument_errors():
    lib = B.load()
    layer = [FAKE] * 4 + [200] * 7 + [4] + [FAKE] * 4

    def model(n=1, d=128, H=2, T=4, layers=layer, head=None, pos=FAKE):
        arr = (B.Layer * 1)(B.Layer(*layers))
        return B.Model(n, d, H, 256, 300, T, 0, 10, arr, FAKE, pos, head, head)

    def call(m=None, p=None, counts=FAKE, io=None, ws=FAKE, less=0):
        m, p = m or model(), p or pages()
        arr = None if counts is None else (C.c_void_p * 1)(counts or None)
        io = io or B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, tokens=FAKE)
        need = lib.nmdlm_block_step_paged_workspace_size(C.byref(m), C.byref(p), io.flags)
        return lib.nmdlm_block_step_paged(C.byref(m), C.byref(p), arr, 2, C.byref(io), ws, max(need - less, 0), None)
    assert call(counts=None) == INVALID
    assert call(counts=0) == INVALID
    assert call(counts=FAKE + 8) == INVALID
    assert call(m=model(layers=layer[:12] + [FAKE, FAKE, FAKE + 8, FAKE])) == INVALID   # key pages
    assert call(m=model(layers=layer[:12] + [FAKE, FAKE, FAKE, None])) == INVALID
    assert call(m=model(layers=layer[:5] + [0] + layer[6:])) == INVALID                 # a threshold of 0
    assert call(m=model(d=192, H=2)) == UNSUPPORTED                                     # heads of 96
    assert call(m=model(T=9)) == UNSUPPORTED
    assert call(p=pages(pool=0)) == INVALID
    assert call(p=pages(max_rows=(1 << 17) + 1)) == UNSUPPORTED
    assert call(m=model(pos=None)) == INVALID                                           # no token tables
    assert call(io=B.step_io(0, 0, flags=B.NMDLM_NO_HEAD)) == INVALID                   # and no input
    assert call(io=B.step_io(0, 0, tokens=FAKE, masked=FAKE)) == INVALID                # a head without weights
    assert call(m=model(head=FAKE), io=B.step_io(0, 0, tokens=FAKE, masked=FAKE, k_unmask=-1)) == INVALID
    assert call(ws=None) == WORKSPACE
    assert call(less=1) == WORKSPACE
    assert lib.nmdlm_block_step_paged_workspace_size(None, C.byref(pages()), 0) == 0
    assert lib.nmdlm_block_step_paged_workspace_size(C.byref(model(T=9)), C.byref(pages()), 0) == 0
    assert lib.nmdlm_block_step_paged_workspace_size(C.byref(model()), C.byref(pages(pool=0)), 0) == 0


def test_routes():
    from ._pages import route

    # rows by themselves up to two a request
    assert route(64, 64, 70, 4, 16).token and route(64, 136, 70, 4, 16).token
    assert not route(64, 137, 70, 4, 16).token and not route(1, 16, 70, 4, 16).token
    # 32 rows a wave from 1024 such waves on, of requests that fill them
    assert route(1, 480, 20, 4, 16).groups == 2 and route(1, 479, 20, 4, 16).groups == 1
    assert route(20, 639, 20, 4, 16).groups == 1
    # splits: as many as fill the chip, of eight pages at least, none beside wide tiles
    assert route(1, 16, 2000, 4, 16).splits == 16 and route(1, 16, 20, 4, 16).splits == 2
    assert route(1, 16, 7, 4, 16).splits == 1 and route(16, 256, 500, 4, 16).splits == 1
    assert route(1, 1, 2000, 4, 16).splits == 32 and route(1, 1, 2000, 1, 1).splits == 64
    assert route(1, 2000, 2000, 4, 16).splits == 1
    for T in range(1, 9):
        for r in (route(2, 60, 9, T, 1), route(1, 4000, 9, T, 64)):
            assert 1 <= r.parts and T * r.parts <= 8
        assert 1 <= route(1, 1, 9, T, 1).parts <= 4 and T * route(1, 1, 9, T, 1).parts <= 12
    assert route(64, 64, 128, 4, 4).fused and not route(63, 64, 128, 4, 4).fused
    assert not route(64, 64, 129, 4, 16).fused


def test_constants_match_the_header():
    import re

    text = open(os.path.join(os.path.dirname(B.PKG), "include", "nmdlm.h")).read()
    for name in ("NMDLM_PAGE", "NMDLM_MAX_REQUESTS", "NMDLM_MAX_PLAN_ROWS", "NMDLM_MAX_PAGES",
                 "NMDLM_MAX_POOL", "NMDLM_STATUS_PAGES_SHORT", "NMDLM_STATUS_BAD_REQUEST"):
        m = re.search(r"#define\s+%s\s+([0-9xXa-fA-F]+)" % name, text)
        assert getattr(B, name) == int(m.group(1), 0), name


def step_sizes(rows, ctx_pages, flags, T=4, d=2048, H=16):
    """Bytes of a step over pages without the head's outputs, and of the
    contiguous step over as many rows."""
    m = B.Model(2, d, H, 4 * d, 300, T, 0, 10, None, FAKE, FAKE, None, None)
    p = pages(n_seq=2, max_rows=rows, max_pages=ctx_pages, pool=ctx_pages)
    lib = B.load()
    return (lib.nmdlm_block_step_paged_workspace_size(C.byref(m), C.byref(p), flags),
            lib.nmdlm_block_step_workspace_size(C.byref(m), rows, flags))


@pytest.mark.parametrize("rows", [32, 4096])
def test_step_over_pages_holds_no_currents(rows):
    """Over pages the rows' keys and values and, for 64 pages, a word and 64
    scores a row and head come to a contiguous step's needs; the currents of
    its attention (4 bytes a row, timestep and channel) do not."""
    T, d, H = 4, 2048, 16
    paged, contiguous = step_sizes(rows, 64, B.NMDLM_NO_HEAD, T, d, H)
    more = 2 * T * rows * d // 8 + rows * H * (8 + 64 * 4)
    more += B.load().nmdlm_bbm_attn_paged_workspace_size(C.byref(pages(n_seq=2, max_rows=rows, max_pages=64)),
                                                         T, H, d // H)
    assert paged <= contiguous + more - 4 * T * rows * d + 8 * 256


def test_steps_without_a_selection_need_no_room_for_one():
    rows, ctx_pages, H, flags = 4096, 512, 16, B.NMDLM_NO_HEAD
    with_sel, _ = step_sizes(rows, ctx_pages, flags)
    without, _ = step_sizes(rows, ctx_pages, flags | B.NMDLM_ALL_PAGES)
    p = pages(n_seq=2, max_rows=rows, max_pages=ctx_pages)
    scores = B.load().nmdlm_page_select_workspace_size(C.byref(p), 4, H, 128)
    assert with_sel - without >= scores + rows * H * ctx_pages // 8

    lib = B.load()
    arr = (B.Layer * 1)(B.Layer(*([FAKE] * 4 + [200] * 7 + [4] + [FAKE] * 4)))
    m = B.Model(1, 128, 2, 256, 300, 4, 0, 10, arr, FAKE, FAKE, None, None)
    counts = (C.c_void_p * 1)(FAKE)
    size = lambda fl: lib.nmdlm_block_step_paged_workspace_size(C.byref(m), C.byref(pages()), fl)  # noqa: E731

    def call(n_sel, fl, nbytes):
        io = B.step_io(0, 0, flags=fl, tokens=FAKE)
        return lib.nmdlm_block_step_paged(C.byref(m), C.byref(pages()), counts, n_sel, C.byref(io), FAKE, nbytes, None)
    less = size(flags | B.NMDLM_ALL_PAGES)
    assert less < size(flags)
    assert call(2, flags, less) == WORKSPACE                          # a selection needs its room
    assert call(-1, flags, less - 1) == WORKSPACE
    assert call(-1, flags | B.NMDLM_ALL_PAGES, less - 1) == WORKSPACE
    assert call(2, flags | B.NMDLM_ALL_PAGES, 1 << 40) == INVALID


def test_scores_of_a_selection_are_bounded():
    """1 GiB, or the scores of one head where those are more."""
    size = lambda rows, ctx_pages, H: B.load().nmdlm_page_select_workspace_size(  # noqa: E731
        C.byref(pages(n_seq=8, max_rows=rows, max_pages=ctx_pages)), 4, H, 128)
    assert size(32, 2047, 16) == 32 * 16 * 2048 * 4
    assert size(8192, 2048, 16) == 1 << 30
    for rows, ctx_pages, H in ((8193, 2048, 16), (8192, 8192, 16), (32768, 2048, 16)):
        assert size(rows, ctx_pages, H) <= 1 << 30
    assert size(131072, 4096, 16) == 131072 * 4096 * 4


def test_misaligned_outputs():
    """A status word is written by an atomic, which faults between words."""
    run = lambda ctx, new, status: B.load().nmdlm_page_plan(C.byref(pages()), ctx, new, status, None)  # noqa: E731
    for i in range(3):
        for off in (1, 2):
            assert run(*[FAKE + off * (j == i) for j in range(3)]) == INVALID, (i, off)
    assert select(sel=FAKE + 4) == INVALID
    for name, off in (("sel", 4), ("a_out", 2), ("s_out", 4)):
        assert attn(**{name: FAKE + off}) == INVALID, name
    arr = (B.Layer * 1)(B.Layer(*([FAKE] * 4 + [200] * 7 + [4] + [FAKE] * 4)))
    m = B.Model(1, 128, 2, 256, 300, 4, 0, 10, arr, FAKE, FAKE, None, None)
    for kw in (dict(status=FAKE + 2), dict(unmasked_pos=FAKE + 1)):
        io = B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, tokens=FAKE, **kw)
        assert B.load().nmdlm_block_step_paged(C.byref(m), C.byref(pages()), (C.c_void_p * 1)(FAKE), 2, C.byref(io),
                                               FAKE, 1 << 40, None) == INVALID, kw


def test_a_model_and_a_plan_that_do_not_fit():
    """The step reads no tensor's size: pools of fewer pages than the plan's, or
    of other types or layers, and layers elsewhere are refused beforehand."""
    from types import SimpleNamespace as S

    layer = S(w_qkv=torch.zeros(1, dtype=torch.int8), c=B.Layer())
    parent = S(T=4, H=2, d=128, layers=[layer], c=B.Model())
    p, wider = (B.Pages(2, 10, 3, n, device="cpu") for n in (7, 8))
    pm = B.PagedModel(parent, p)
    assert pm.view(p.view(20), head=False).pools is pm.pools
    k, v, counts = pm.pools[0]
    with pytest.raises(B.NmdlmError, match="k_pages"):
        pm.view(wider, head=False)
    for bad, name in (([(k.int(), v, counts)], "k_pages"), ([(k, v[:6], counts)], "v_pages"),
                      ([(k, v, counts.transpose(1, 2))], "key_counts"), ([(k, v, counts)] * 2, "layers")):
        with pytest.raises(B.NmdlmError, match=name):
            B.PagedModel(parent, p, pools=bad)
    parent.layers = [S(w_qkv=S(get_device=lambda: 1), c=B.Layer())]
    with pytest.raises(B.NmdlmError, match="layers"):
        B.PagedModel(parent, p)
