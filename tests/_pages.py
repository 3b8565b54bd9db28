"""Cases of the paged caches: lengths, a page state that holds the contexts,
pools and rows, and the same on the GPU."""
from types import SimpleNamespace

import numpy as np

from oracle import nmdlm_oracle as O
from workloads import synth

PAGE = O.PAGE


def make_case(seed, ctx, new, T=4, H=2, dh=64, spare_rows=3, spare_pages=2, spare_pool=5, rate=0.3):
    """Requests of the given contexts and new rows (0 idle, -1 ended) over a
    pool in random order, its ring wrapping; unheld pages are random too."""
    rng = np.random.default_rng([77, seed])
    ctx, new = np.array(ctx, dtype=np.int64), np.array(new, dtype=np.int64)
    n = len(ctx)
    held = -(-ctx // PAGE)
    need = np.maximum(-(-(ctx + new.clip(0)) // PAGE) - held, 0)
    max_pages = int((held + need).max()) + spare_pages
    pool = max(int(held.sum() + need.sum()) + spare_pool, 1)
    rows = int(new.clip(0).sum())
    ids = rng.permutation(pool)
    table = np.full((n, max_pages), -1)
    at = 0
    for s in range(n):
        table[s, :held[s]] = ids[at:at + held[s]]
        at += held[s]
    head, free = int(rng.integers(pool)), pool - at
    ring = np.zeros(pool, dtype=np.int64)
    ring[(head + np.arange(free)) % pool] = ids[at:]
    c = SimpleNamespace(n=n, ctx=ctx, new=new, T=T, H=H, dh=dh, rows=rows, max_rows=max(rows + spare_rows, 1),
                        max_pages=max_pages, pool=pool, table=table, held=held, ring=ring,
                        ring_state=[head, free], theta=150)
    R = c.max_rows
    c.k, c.v, c.q = (synth.bernoulli(rng, rate, (T, R, H, dh)) for _ in range(3))
    c.k_pages, c.v_pages = (synth.bernoulli(rng, rate, (pool, H, T, PAGE, dh)) for _ in range(2))
    c.counts = c.k_pages.sum(3)
    c.lut = synth.sorted_lut_u8(rng)
    return c


def plan(c, **kw):
    a = dict(ctx=c.ctx, new=c.new, table=c.table, held=c.held, ring=c.ring, ring_state=c.ring_state,
             max_rows=c.max_rows)
    a.update(kw)
    return O.page_plan(**a)


def pages_of(c, p, s):
    return p["table"][s, :-(-int(c.ctx[s] + c.new[s]) // PAGE)]


def live(c, p):
    """(request, first row, rows) of the requests whose rows have pages."""
    return [(s, int(p["cu_rows"][s]), int(c.new[s])) for s in range(c.n) if p["ok"][s] and c.new[s] > 0]


def select(c, p, n_sel):
    """0/1 [rows][H][64 * words], rows without a page all ones."""
    words = -(-c.max_pages // 64)
    out = np.ones((c.max_rows, c.H, words * 64), dtype=np.uint8)
    counts = np.concatenate([c.counts, np.zeros_like(c.counts[:1])])  # a page that is not there
    for s, r0, M in live(c, p):
        ids = pages_of(c, p, s)
        ids = np.where((ids >= 0) & (ids < c.pool), ids, c.pool)
        out[r0:r0 + M] = 0
        out[r0:r0 + M, :, :len(ids)] = O.page_select(c.q[:, r0:r0 + M], counts[ids], int(c.ctx[s]) // PAGE,
                                                     len(ids), n_sel)
    return out


def attention(c, p, sel=None):
    """Currents [T][rows][H*dh] (-9 for rows without a page) and spikes."""
    cur = np.full((c.T, c.max_rows, c.H * c.dh), -9, dtype=np.int64)
    spk = np.ones((c.T, c.max_rows, c.H * c.dh), dtype=bool)
    for s, r0, M in live(c, p):
        ids, J = pages_of(c, p, s), int(c.ctx[s]) + M
        K, V = (x[ids].transpose(1, 2, 0, 3, 4).reshape(c.H, c.T, -1, c.dh)[:, :, :J]
                for x in (c.k_pages, c.v_pages))
        see = np.ones((M, c.H, J), dtype=np.uint8)
        if sel is not None:
            see = np.repeat(sel[r0:r0 + M, :, :len(ids)], PAGE, axis=2)[:, :, :J]
        a = O.paged_attention(c.q[:, r0:r0 + M], K, V, c.lut, see)
        cur[:, r0:r0 + M] = a
        spk[:, r0:r0 + M] = O.if_neuron(a, c.theta)[0]
    return cur, spk


def route(n_seq, max_rows, max_pages, T, H):
    """The kernels a call takes (a host-side query): by rows, 16-row groups of a
    wave, waves per timestep, most splits, selection in one kernel."""
    import ctypes as C

    from paper_2607_24841_amd import binding as B

    out = (C.c_int32 * 5)()
    B.load().nmdlm_internal_paged_route(n_seq, max_rows, max_pages, T, H, out)
    return SimpleNamespace(token=bool(out[0]), groups=out[1], parts=out[2], splits=out[3], fused=bool(out[4]))


def case_route(c):
    return route(c.n, c.max_rows, c.max_pages, c.T, c.H)


class Device:
    """The case on the GPU."""

    def __init__(self, torch, B, c, device="cuda"):
        self.torch, self.B, self.c = torch, B, c
        self.pages = B.Pages(c.n, c.max_rows, c.max_pages, c.pool, device)
        self.pages.set_state(*(torch.from_numpy(np.asarray(x, dtype=np.int32))
                               for x in (c.table, c.held, c.ring, c.ring_state)))
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        self.ctx, self.new = dev(c.ctx.astype(np.int32)), dev(c.new.astype(np.int32))
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        flat = lambda x: synth.pack_bits(x.reshape(c.T, c.max_rows, -1))  # noqa: E731
        self.q, self.k, self.v = (B.to_dev_bits(flat(x), device) for x in (c.q, c.k, c.v))
        self.k_pages = B.to_dev_bits(synth.pack_bits(c.k_pages), device)
        self.v_pages = B.to_dev_bits(synth.pack_bits(c.v_pages.transpose(0, 1, 2, 4, 3))[..., 0], device)
        self.counts = dev(c.counts.astype(np.uint8))
        self.lut = dev(c.lut)
        self.sel = torch.full((c.max_rows, c.H, -(-c.max_pages // 64)), -1, dtype=torch.int64, device=device)
        shape = (c.T, c.max_rows, c.H * c.dh)
        self.cur = torch.full(shape, -9, dtype=torch.int32, device=device)
        self.spk = torch.full((c.T, c.max_rows, c.H * c.dh // 64), -1, dtype=torch.int64, device=device)
        self.hd = (c.T, c.H, c.dh)
        self.ws_sel = B.workspace(B.nmdlm_page_select_workspace_size(self.pages, *self.hd), device)
        self.ws_att = B.workspace(B.nmdlm_bbm_attn_paged_workspace_size(self.pages, *self.hd), device)

    def plan(self, **kw):
        self.B.nmdlm_page_plan(self.pages, self.ctx, self.new, status=self.status, **kw)

    def store(self, **kw):
        self.B.nmdlm_page_store(self.pages, self.k, self.v, *self.hd, self.k_pages, self.v_pages, self.counts, **kw)

    def select(self, n_sel, **kw):
        self.B.nmdlm_page_select(self.pages, self.q, *self.hd, self.counts, n_sel, self.sel, ws=self.ws_sel, **kw)

    def attention(self, sel=None, cur=True, spk=True, **kw):
        self.B.nmdlm_bbm_attn_paged(self.pages, self.q, *self.hd, self.k_pages, self.v_pages, self.lut,
                                    a_out=self.cur if cur else None, theta_a=self.c.theta if spk else 0,
                                    s_out=self.spk if spk else None, sel=sel, ws=self.ws_att, **kw)

    # results on the host
    def bits(self, t, n):
        return synth.unpack_bits(self.B.from_dev_bits(t), n)

    def spikes(self):
        return self.bits(self.spk, self.c.H * self.c.dh)

    def selection(self):
        return self.bits(self.sel, self.sel.shape[2] * 64).astype(np.uint8)

    def values(self):
        return self.bits(self.v_pages.unsqueeze(-1), PAGE).transpose(0, 1, 2, 4, 3)

    def put_selection(self, sel):
        self.sel.copy_(self.B.to_dev_bits(synth.pack_bits(sel)))
        return self.sel
