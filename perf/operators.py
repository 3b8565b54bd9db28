"""Timed calls of the paged spike cache: requests of different lengths that
share one pool of 64-position pages.

Kinds of case
  plan    block tables, slots and row positions from the request lengths
  store   keys and values of packed rows into the pages, with the pages' spike counts
  select  for each query and head, the context pages of the highest score
  attn    attention of packed rows over their pages, all of them or the selected ones
  serve   the four, one after the other, as a layer of a serving step makes them

Layouts.  A page holds 64 positions:
  k_pages [pool][H][T][64][dh/64] words, bit c%64 of word c/64 = channel c of a position
  v_pages [pool][H][T][dh] words, bit j = position j of the page
  counts  [pool][H][T][dh] bytes, the page's keys that spike in a channel
Packed rows (queries, new keys and values): [T][max_rows][H dh/64] words, the
requests one after the other.  Logical page p of request s is pool page table[s][p].
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
PAGE = 64


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _c(kind, n, ctx, new, T=4, H=16, dh=128, **kw):
    c = dict(kind=kind, n=n, ctx_lo=ctx[0], ctx_hi=ctx[1], new_lo=new[0], new_hi=new[1], T=T, H=H,
             dh=dh, idle=0.0, sel=0, cur=False, short=False, mix=1)
    c.update(kw)
    return c


def listed():
    return [
        # a denoising block of 16 tokens begins for 128 requests, some idle, some finished
        _c("plan", 128, (0, 4096), (16, 16), idle=0.2, name="plan_blocks"),
        # a wave of admissions: prompts of very different lengths, more than the pool takes
        _c("plan", 1000, (0, 200), (1, 900), idle=0.3, short=True, name="plan_prompts"),
        # the new keys and values of one step of 64 requests (8 timesteps, 512 channels)
        _c("store", 64, (0, 700), (4, 4), T=8, H=8, dh=64, name="store_blocks"),
        # keys and values of whole prompts of the 24-layer model
        _c("store", 6, (0, 0), (300, 2048), name="store_prompts"),
        # page scores of one block over a very long context
        _c("select", 1, (131000, 131000), (32, 32), sel=64, name="select_long"),
        # page scores of many short blocks over middling contexts
        _c("select", 48, (1000, 9000), (3, 16), T=8, H=8, dh=64, sel=12, name="select_batch"),
        # one token a request over all of its context
        _c("attn", 64, (1, 4000), (1, 1), name="attn_tokens"),
        # few requests of odd lengths, three timesteps, currents asked for
        _c("attn", 5, (0, 700), (1, 75), T=3, H=5, dh=64, cur=True, name="attn_ragged"),
        # whole prompts over themselves
        _c("attn", 3, (0, 0), (700, 2048), name="attn_prompts"),
        # one block over the selected pages of a very long context
        _c("attn", 1, (131000, 131000), (32, 32), sel=64, name="attn_long_selected"),
        # blocks of a batch over selected pages
        _c("attn", 32, (2000, 12000), (16, 16), sel=24, name="attn_batch_selected"),
        # a layer's four calls in a serving step: blocks of 16, idle and finished requests
        _c("serve", 48, (64, 4000), (16, 16), H=16, dh=64, idle=0.15, sel=16, name="serve_layer"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, below the largest listed one's cost."""
    kind = rng.choice(["plan", "store", "select", "attn", "attn", "attn", "serve"])
    T, dh = rng.choice([1, 2, 3, 4, 4, 6, 8]), rng.choice([64, 128])
    H = rng.choice([2, 4, 5, 8, 12, 16])
    mix = rng.randrange(1, 1 << 20)
    if kind == "plan":
        n = _log(rng, 1, 1000)
        hi = _log(rng, 1, max(1, min(2048, 400000 // n)))
        return _c("plan", n, (0, _log(rng, 1, 4096)), (rng.randrange(1, hi + 1), hi),
                  idle=rng.choice([0.0, 0.2, 0.5]), short=rng.random() < 0.3, mix=mix)
    if kind == "store":
        n = _log(rng, 1, 96)
        hi = _log(rng, 1, max(1, min(2048, 8000 // n)))
        return _c("store", n, (0, _log(rng, 1, 900)), (rng.randrange(1, hi + 1), hi), T=T, H=H, dh=dh,
                  mix=mix)
    if kind == "attn" and rng.random() < 0.3:  # prompts
        n = rng.randrange(1, 4)
        hi = _log(rng, 64, 1500)
        return _c("attn", n, (0, 0), (rng.randrange(1, hi + 1), hi), T=T, H=H, dh=dh,
                  cur=rng.random() < 0.3, mix=mix)
    n, M = _log(rng, 1, 64), _log(rng, 1, 48)
    ctx = _log(rng, 1, min(100000, 250000 // n))
    ctx = max(1, min(ctx, int(3.2e10) // (n * M * T * H * dh)))
    lo = rng.randrange(0, ctx)
    sel = 0 if kind == "attn" and rng.random() < 0.5 else _log(rng, 1, 96)
    if kind == "select":  # contexts of more pages than are selected
        ctx = max(ctx, 600)
        lo = rng.randrange(300, ctx)
        sel = _log(rng, 1, min(96, lo // 128))
    return _c(kind, n, (lo, ctx), (rng.randrange(1, M + 1), M), T=T, H=H, dh=dh,
              sel=sel, cur=kind == "attn" and rng.random() < 0.3,
              idle=0.0 if kind == "attn" else rng.choice([0.0, 0.2]), mix=mix)


# ----------------------------------------------------------------------------
# inputs, from the seed alone (the lengths from the case: they set the sizes)
# ----------------------------------------------------------------------------
def _lengths(c):
    """Context and new rows of each request; -1 new rows: the request has
    ended (0: idle).  Held pages: those of the context."""
    rng = np.random.default_rng([c["mix"], c["n"], c["ctx_hi"], c["new_hi"]])
    ctx = rng.integers(c["ctx_lo"], c["ctx_hi"] + 1, size=c["n"])
    lo, hi = math.log(c["new_lo"]), math.log(c["new_hi"] + 1)
    new = np.exp(rng.uniform(lo, hi, size=c["n"])).astype(np.int64).clip(c["new_lo"], c["new_hi"])
    u = rng.random(c["n"])
    new = np.where(u < c["idle"] / 2, 0, np.where(u < c["idle"], -1, new))
    if not (new > 0).any():
        new[0] = c["new_hi"]
    return ctx, new, -(-ctx // PAGE)


def _gen(seed, *path):
    s = 1469598103934665603
    for v in (seed, *path):
        s = ((s ^ (int(v) + 1)) * 1099511628211) % (1 << 63)
    return torch.Generator(device=DEV).manual_seed(s)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).to(DEV)


def _pack(bits):
    w = torch.tensor([1, 2, 4, 8, 16, 32, 64, 128], dtype=torch.uint8, device=bits.device)
    by = (bits.reshape(-1, 8).to(torch.uint8) * w).sum(-1, dtype=torch.uint8)
    return by.view(torch.int64).reshape(*bits.shape[:-1], bits.shape[-1] // 64)


def _unpack(words):
    by = words.contiguous().view(torch.uint8)
    sh = torch.arange(8, dtype=torch.uint8, device=words.device)
    b = (by.unsqueeze(-1) >> sh) & 1
    return b.reshape(*words.shape[:-1], words.shape[-1] * 64)


def _sizes(c):
    ctx, new, held = _lengths(c)
    rows = int(new.clip(0).sum())
    need = (-(-(ctx + new.clip(0)) // PAGE) - held).clip(0)
    total = int(held.sum() + need.sum())
    return SimpleNamespace(ctx=ctx, new=new, held=held, need=need, rows=rows,
                           max_rows=-(-rows // 16) * 16 + 5,
                           max_pages=int((held + need).max()) + 3,
                           pool=max(total + 7, 1) - (int(need.sum()) // 5 if c["short"] else 0))


def _state(c, seed, z):
    """The page state before a step: tables of the held pages, the ring of the
    free ones (its first at `head`) and where it stands."""
    rng = np.random.default_rng([seed, 11])
    ids = rng.permutation(z.pool)
    n_held = int(z.held.sum())
    table = np.full((c["n"], z.max_pages), -1)
    at = 0
    for s in range(c["n"]):
        table[s, :z.held[s]] = ids[at:at + z.held[s]]
        at += z.held[s]
    head, free = int(rng.integers(0, z.pool)), z.pool - n_held
    ring = np.zeros(z.pool, np.int64)
    ring[(head + np.arange(free)) % z.pool] = ids[n_held:]
    return _dev(table), _dev(z.held), _dev(ring), _dev([head, free])


def _topics(c, seed):
    """Spike rates of 16 topics; keys of a page and queries of a request follow one."""
    rng = np.random.default_rng([seed, 12])
    r = np.clip(rng.beta(0.6, 2.0, size=(16, c["T"] * c["H"] * c["dh"])) * 1.2, 0.0, 0.95)
    return _dev(r, torch.float32).reshape(16, c["H"], c["T"], c["dh"])


def _pool(c, seed, z, rates):
    """Random pages in the layouts above."""
    H, T, dh = c["H"], c["T"], c["dh"]
    g = _gen(seed, 13)
    topic = torch.randint(0, 16, (z.pool,), device=DEV, generator=g)
    value_rate = torch.rand(H, T, dh, 1, device=DEV, generator=g)  # of a channel
    k = torch.empty(z.pool, H, T, PAGE, dh // 64, dtype=torch.int64, device=DEV)
    v = torch.empty(z.pool, H, T, dh, dtype=torch.int64, device=DEV)
    cnt = torch.empty(z.pool, H, T, dh, dtype=torch.uint8, device=DEV)
    for p in range(0, z.pool, 128):
        r = rates[topic[p:p + 128]]
        b = torch.rand(*r.shape[:3], PAGE, dh, device=DEV, generator=g) < r.unsqueeze(3)
        k[p:p + 128] = _pack(b)
        cnt[p:p + 128] = b.sum(3, dtype=torch.uint8)
        b = torch.rand(*r.shape, PAGE, device=DEV, generator=g) < value_rate
        v[p:p + 128] = _pack(b).squeeze(-1)
    return k, v, cnt


def _rows(c, seed, z, rates, *path):
    """Spikes of the packed rows, by request; rows past the last are spikes too."""
    g = _gen(seed, *path)
    topic = torch.randint(0, 16, (c["n"],), device=DEV, generator=g)
    own_t = topic[torch.repeat_interleave(torch.arange(c["n"], device=DEV), _dev(z.new.clip(0)))]
    own_t = torch.nn.functional.pad(own_t, (0, z.max_rows - z.rows))
    out = torch.empty(c["T"], z.max_rows, c["H"] * c["dh"] // 64, dtype=torch.int64, device=DEV)
    for m in range(0, z.max_rows, 2048):
        r = rates[own_t[m:m + 2048]].permute(2, 0, 1, 3)  # [T][rows][H][dh]
        b = torch.rand(*r.shape, device=DEV, generator=g) < r
        out[:, m:m + 2048] = _pack(b.reshape(c["T"], r.shape[1], -1))
    return out


def _inputs(c, seed):
    s = SimpleNamespace(c=c, z=_sizes(c))
    z = s.z
    s.table, s.held, s.ring, s.ring_state = _state(c, seed, z)
    s.ctx, s.new = _dev(z.ctx), _dev(z.new)
    if c["kind"] == "plan":
        return s
    rates = _topics(c, seed)
    s.k_pages, s.v_pages, s.counts = _pool(c, seed, z, rates)
    if c["kind"] in ("store", "serve"):
        s.k, s.v = _rows(c, seed, z, rates, 14), _rows(c, seed, z, rates, 15)
    if c["kind"] != "store":
        s.q = _rows(c, seed, z, rates, 16)
        s.lut = torch.randint(1, 256, (256,), device=DEV, generator=_gen(seed, 17)).sort().values.to(torch.uint8)
        s.theta = 160
    return s


def _words(c, z):
    return torch.zeros(z.max_rows, c["H"], -(-z.max_pages // 64), dtype=torch.int64, device=DEV)


def _prepare(c, seed):
    s = _inputs(c, seed)
    z = s.z
    if c["kind"] in ("plan", "serve"):
        s.keep = [x.clone() for x in (s.table, s.held, s.ring, s.ring_state)]
    else:  # the pages of the new rows are there already
        s.table, s.held, s.ring, s.ring_state, s.cu, s.slot, s.pos = _plan_plain(
            c, z, s.ctx, s.new, s.table, s.held, s.ring, s.ring_state)
    if c["kind"] == "attn" and c["sel"]:
        s.sel = _words(c, z)
        _select_plain(s, s.cu, s.table, s.sel)
    if c["kind"] in ("select", "serve"):
        s.sel = _words(c, z)
    if c["kind"] in ("store", "serve"):
        s.runs = _runs(z)
    if c["kind"] in ("attn", "serve"):
        d = c["H"] * c["dh"]
        s.a = torch.zeros(c["T"], z.max_rows, d, dtype=torch.int32, device=DEV) if c["cur"] else None
        s.spk = torch.zeros(c["T"], z.max_rows, d // 64, dtype=torch.int64, device=DEV)
    return s


def prepare(case, seed):
    c = case
    s = _prepare(c, seed)
    if not own:
        return s
    from paper_2607_24841_amd import binding as B

    z = s.z
    s.pages = B.Pages(c["n"], z.max_rows, z.max_pages, z.pool)
    s.pages.set_state(s.table, s.held, s.ring, s.ring_state)
    if c["kind"] in ("plan", "serve"):
        s.first = s.pages.state.clone()
    else:
        B.nmdlm_page_plan(s.pages, s.ctx, s.new)
    T, H, dh = c["T"], c["H"], c["dh"]
    if c["kind"] in ("select", "serve"):
        s.ws_sel = B.workspace(B.nmdlm_page_select_workspace_size(s.pages, T, H, dh))
    if c["kind"] in ("attn", "serve"):
        s.ws_att = B.workspace(B.nmdlm_bbm_attn_paged_workspace_size(s.pages, T, H, dh))
    return s


# ----------------------------------------------------------------------------
# the calls
# ----------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2607_24841_amd import binding as B

    c, p = s.c, s.pages
    T, H, dh = c["T"], c["H"], c["dh"]
    out = []
    if c["kind"] in ("plan", "serve"):
        p.state.copy_(s.first)  # a step starts from the tables of the one before
        B.nmdlm_page_plan(p, s.ctx, s.new)
        out += [p.table, p.held, p.ring, p.ring_state, p.cu_rows, p.slot, p.pos]
    if c["kind"] in ("store", "serve"):
        B.nmdlm_page_store(p, s.k, s.v, T, H, dh, s.k_pages, s.v_pages, s.counts)
        out += [s.k_pages, s.v_pages, s.counts]
    if c["kind"] in ("select", "serve"):
        B.nmdlm_page_select(p, s.q, T, H, dh, s.counts, c["sel"], s.sel, ws=s.ws_sel)
        out.append(s.sel)
    if c["kind"] in ("attn", "serve"):
        B.nmdlm_bbm_attn_paged(p, s.q, T, H, dh, s.k_pages, s.v_pages, s.lut, a_out=s.a,
                               theta_a=s.theta, s_out=s.spk, sel=s.sel if c["sel"] else None,
                               ws=s.ws_att)
        out += [s.a, s.spk]
    return out


def _run_plain(s):
    c, z = s.c, s.z
    out = []
    if c["kind"] in ("plan", "serve"):
        st = _plan_plain(c, z, s.ctx, s.new, *s.keep)
        out += st
        table, cu, slot = st[0], st[4], st[5]
    else:
        table, cu, slot = s.table, s.cu, s.slot
    if c["kind"] in ("store", "serve"):
        _store_plain(s, slot)
        out += [s.k_pages, s.v_pages, s.counts]
    if c["kind"] in ("select", "serve"):
        _select_plain(s, cu, table, s.sel)
        out.append(s.sel)
    if c["kind"] in ("attn", "serve"):
        _attn_plain(s, table)
        out += [s.a, s.spk]
    return out


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------
def _plan_plain(c, z, ctx, new, table, held, ring, ring_state):
    """Requests in order: one that ends gives its pages back, one with new rows
    is given the pages it lacks, in order, while the ring has them.  Rows of a
    request without its pages have slot -1, as the rows past the last."""
    ctx, new, table, held, ring = ctx.long(), new.long(), table.long(), held.long(), ring.long()
    head, free = ring_state[0].long(), ring_state[1].long()
    end = ctx + new
    rows = torch.where((new > 0) & (new <= z.max_rows), new, 0)
    row_end = torch.cumsum(rows, 0)
    ok = ((new >= 0) & (ctx >= 0) & (held >= 0) & (held <= z.max_pages) & (ctx <= held * PAGE)
          & (end <= z.max_pages * PAGE) & (row_end <= z.max_rows))
    need = torch.where(ok, ((end + PAGE - 1) // PAGE - held).clamp(min=0), 0)
    need_end = torch.cumsum(need, 0)
    ok = ok & ((need == 0) | (need_end <= free))
    gone = (new == -1) & (held >= 0) & (held <= z.max_pages)
    back = torch.where(gone, held, 0)
    back_start = torch.cumsum(back, 0) - back
    granted = torch.where(ok, need, 0).sum()
    cu = torch.nn.functional.pad(row_end.clamp(max=z.max_rows), (1, 0))
    # rows
    m = torch.arange(z.max_rows, device=DEV)
    s = torch.searchsorted(cu[1:].contiguous(), m, right=True)
    valid = s < c["n"]
    s = s.clamp(max=c["n"] - 1)
    pos = ctx[s] + m - cu[s]
    lp = (pos // PAGE).clamp(0, z.max_pages - 1)
    fresh = valid & ok[s] & (lp >= held[s])
    from_ring = ring[(head + (need_end - need)[s] + lp - held[s]) % z.pool]
    page = torch.where(fresh, from_ring, table[s, lp])
    good = valid & ok[s] & (page >= 0) & (page < z.pool)
    slot = torch.where(good, page * PAGE + pos % PAGE, -1)
    pos = torch.where(valid & ok[s], pos, 0)
    # tables: the rows' new pages (rows of one page write the same)
    t2 = torch.cat([table.reshape(-1), table.new_zeros(1)])
    t2[torch.where(fresh, s * z.max_pages + lp, c["n"] * z.max_pages)] = from_ring
    # the ring takes the pages of ended requests behind its last
    k = torch.arange(z.max_pages, device=DEV)
    put = gone[:, None] & (k[None] < held[:, None])
    r2 = torch.cat([ring, ring.new_zeros(1)])
    r2[torch.where(put, (head + free + back_start[:, None] + k[None]) % z.pool, z.pool)] = table
    held2 = torch.where(gone, 0, torch.where(ok, torch.maximum(held, (end + PAGE - 1) // PAGE), held))
    state = torch.stack([(head + granted) % z.pool, free - granted + back.sum()])
    return [t2[:-1].reshape(table.shape).int(), held2.int(), r2[:-1].int(), state.int(), cu.int(), slot,
            pos.int()]


def _runs(z):
    """Run of each row (consecutive rows of one page), the rows that begin one
    and the page positions filled after it."""
    run_of, first, end = [], [], []
    for ctx, new in zip(z.ctx, z.new):
        pos = np.arange(ctx, ctx + max(new, 0))
        pg = pos // PAGE
        st = np.flatnonzero(np.diff(pg, prepend=-1))
        first += list(len(run_of) + st)
        end += list(pos[np.append(st[1:], len(pos)) - 1] % PAGE + 1) if len(pos) else []
        run_of += list(len(first) - len(st) + np.cumsum(np.isin(np.arange(len(pos)), st)) - 1)
    return _dev(run_of, torch.int64), _dev(first, torch.int64), _dev(end, torch.int64)


def _store_plain(s, slot):
    c, z = s.c, s.z
    T, H, dh, R = c["T"], c["H"], c["dh"], z.rows
    run_of, first, end = s.runs
    page, off = slot[:R] // PAGE, slot[:R] % PAGE
    k = s.k[:, :R].reshape(T, R, H, dh // 64).permute(1, 2, 0, 3)
    s.k_pages.permute(0, 3, 1, 2, 4)[page, off] = k
    v = _unpack(s.v[:, :R]).reshape(T, R, H, dh).permute(1, 2, 0, 3)
    bit = torch.ones_like(off) << off
    acc = torch.zeros(len(first), H, T, dh, dtype=torch.int64, device=DEV)
    for h in range(H):
        acc[:, h].index_add_(0, run_of, v[:, h].long() << off[:, None, None])
    mask = torch.zeros(len(first), dtype=torch.int64, device=DEV).index_add_(0, run_of, bit)
    rp = page[first]
    m = mask[:, None, None, None]
    s.v_pages[rp] = (s.v_pages[rp] & ~m) | acc
    there = torch.arange(PAGE, device=DEV)[None] < end[:, None]
    for i in range(0, len(first), 64):
        b = _unpack(s.k_pages[rp[i:i + 64]]) * there[i:i + 64, None, None, :, None]
        s.counts[rp[i:i + 64]] = b.sum(3, dtype=torch.uint8)


def _select_plain(s, cu, table, sel):
    """The sel pages of the highest score among the context's full pages (ties:
    the lower page), and every page from the context's last position on."""
    c, z = s.c, s.z
    row = 0
    for r in range(c["n"]):
        ctx, M = int(z.ctx[r]), int(max(z.new[r], 0))
        if M == 0:
            continue
        P, nP = ctx // PAGE, -(-(ctx + M) // PAGE)
        chosen = torch.zeros(c["H"], M, sel.shape[2] * 64, dtype=torch.bool, device=DEV)
        chosen[:, :, P:nP] = True
        n = min(c["sel"], P)
        if n > 0:
            q = _unpack(s.q[:, row:row + M]).reshape(c["T"], M, c["H"], c["dh"])
            q = q.permute(2, 1, 0, 3).reshape(c["H"], M, -1).float()
            ct = s.counts[table[r, :P].long()].reshape(P, c["H"], -1).permute(1, 2, 0).float()
            score = (q @ ct.contiguous()).long()
            key = score * P + (P - 1 - torch.arange(P, device=DEV))
            chosen.scatter_(2, key.topk(n, dim=2).indices, True)
        sel[row:row + M] = _pack(chosen).permute(1, 0, 2)
        row += M


def _attn_plain(s, table):
    c, z = s.c, s.z
    T, H, dh = c["T"], c["H"], c["dh"]
    lut, row = s.lut.float(), 0
    for r in range(c["n"]):
        M = int(max(z.new[r], 0))
        if M == 0:
            continue
        J = int(z.ctx[r]) + M
        nP = -(-J // PAGE)
        q = _unpack(s.q[:, row:row + M]).reshape(T, M, H, dh).permute(2, 0, 1, 3).float().contiguous()
        num = torch.zeros(H, T, M, dh, dtype=torch.float64, device=DEV)
        den = torch.zeros(H, T, M, 1, dtype=torch.float64, device=DEV)
        step = 256  # pages a product: the sums of the table's weights stay below 2^24
        for p0 in range(0, nP, step):
            ids = table[r, p0:min(p0 + step, nP)].long()
            n = len(ids) * PAGE
            k = _unpack(s.k_pages[ids]).permute(1, 2, 4, 0, 3).reshape(H, T, dh, n).float()
            p = lut[(q @ k).to(torch.int32)]
            keep = torch.arange(p0 * PAGE, p0 * PAGE + n, device=DEV) < J
            if c["sel"]:
                b = _unpack(s.sel[row:row + M])[:, :, p0:p0 + len(ids)].permute(1, 0, 2)
                keep = keep & b.bool().repeat_interleave(PAGE, 2).unsqueeze(1)
            p = p * keep
            v = _unpack(s.v_pages[ids].unsqueeze(-1)).permute(1, 2, 0, 4, 3).reshape(H, T, n, dh).float()
            num += p @ v
            den += p.sum(3, keepdim=True, dtype=torch.float64)
        a = torch.where(den > 0, (256 * num.long()) // den.long().clamp(min=1), 0)
        a = a.permute(1, 2, 0, 3).reshape(T, M, H * dh)
        if s.a is not None:
            s.a[:, row:row + M] = a.int()
        V = torch.zeros_like(a[0])
        for t in range(T):
            V = V + a[t]
            f = V >= s.theta
            V = V - s.theta * f
            s.spk[t, row:row + M] = _pack(f)
        row += M


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    c = case
    z = _sizes(c)
    T, d, H = c["T"], c["H"] * c["dh"], c["H"]
    live = z.new > 0
    M, J = z.new[live], (z.ctx + z.new)[live]
    P, nP = z.ctx[live] // PAGE, -(-J // PAGE)
    runs = float((nP - P).sum())
    by = fl = 0.0
    if c["kind"] in ("plan", "serve"):
        by += 16 * c["n"] + 12 * z.rows + 8 * float(z.need.sum()) + 4 * runs
        fl += 4 * z.rows
    if c["kind"] in ("store", "serve"):
        by += 4 * T * z.rows * d / 8 + runs * T * d
        fl += T * runs * d * PAGE
    if c["kind"] in ("select", "serve"):
        by += float(P.sum()) * T * d + T * z.rows * d / 8 + z.rows * H * -(-z.max_pages // 64) * 8
        fl += 2 * T * d * float((M * P).sum())
    if c["kind"] in ("attn", "serve"):
        seen = np.minimum(P, c["sel"]) + nP - P if c["sel"] else nP  # pages a query sees
        by += 2 * T * d * 8 * float(seen.sum()) + 2 * T * z.rows * d / 8 + 4 * T * z.rows * d * c["cur"]
        fl += 4 * T * d * float((M * np.minimum(seen * PAGE, J)).sum())
    return dict(bytes=by, flops=fl)


# ----------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    z = s.z
    T, H, dh, n = c["T"], c["H"], c["dh"], c["n"]
    # the requests one by one, on the host
    table, held = s.table.cpu().numpy().copy(), s.held.cpu().numpy().copy()
    ring, (head, free) = s.ring.cpu().numpy().copy(), [int(x) for x in s.ring_state.cpu()]
    slot, pos = np.full(z.max_rows, -1, np.int64), np.zeros(z.max_rows, np.int32)
    cu, given, asked, back = [0], 0, 0, []
    for r in range(n):
        ctx, new = int(z.ctx[r]), int(z.new[r])
        cu.append(cu[-1] + max(new, 0))
        if new == -1:
            back += list(table[r, :held[r]])
            held[r] = 0
            continue
        lack = max(0, -(-(ctx + new) // PAGE) - int(held[r]))
        asked += lack
        if lack and asked > free:
            continue
        for i in range(lack):
            table[r, held[r]] = ring[(head + given) % z.pool]
            held[r] += 1
            given += 1
        at = np.arange(ctx, ctx + new)
        slot[cu[r]:cu[r + 1]] = table[r, at // PAGE].astype(np.int64) * PAGE + at % PAGE
        pos[cu[r]:cu[r + 1]] = at
    for i, p in enumerate(back):
        ring[(head + free + i) % z.pool] = p
    out = []
    if c["kind"] in ("plan", "serve"):
        out += [_dev(table), _dev(held), _dev(ring), _dev([(head + given) % z.pool, free - given + len(back)]),
                _dev(cu), _dev(slot, torch.int64), _dev(pos)]
    if c["kind"] in ("store", "serve"):
        for r in range(n):
            a, b = cu[r], cu[r + 1]
            while a < b:  # page by page, as bits
                pg, off = divmod(int(slot[a]), PAGE)
                m = min(PAGE - off, b - a)
                k = _unpack(s.k[:, a:a + m]).reshape(T, m, H, dh).permute(2, 0, 1, 3)
                v = _unpack(s.v[:, a:a + m]).reshape(T, m, H, dh).permute(2, 0, 3, 1)
                s.k_pages[pg, :, :, off:off + m] = _pack(k)
                vb = _unpack(s.v_pages[pg].unsqueeze(-1))
                vb[..., off:off + m] = v
                s.v_pages[pg] = _pack(vb).squeeze(-1)
                s.counts[pg] = _unpack(s.k_pages[pg, :, :, :off + m]).sum(2).to(torch.uint8)
                a += m
        out += [s.k_pages, s.v_pages, s.counts]
    if c["kind"] in ("plan", "store"):
        return out
    q = _unpack(s.q).reshape(T, z.max_rows, H, dh).double()
    spk = torch.zeros(T, z.max_rows, H * dh // 64, dtype=torch.int64, device=DEV)
    cur = torch.zeros(T, z.max_rows, H * dh, dtype=torch.int32, device=DEV)
    sel = _words(c, z)
    for r in range(n):
        lo, hi = cu[r], cu[r + 1]
        if hi == lo:
            continue
        ctx, M = int(z.ctx[r]), hi - lo
        J, P = ctx + M, ctx // PAGE
        ids = _dev(table[r, :-(-J // PAGE)], torch.int64)
        chosen = torch.zeros(M, H, sel.shape[2] * 64, dtype=torch.bool, device=DEV)
        chosen[:, :, P:len(ids)] = True
        for h in range(H):
            if c["sel"] and P:
                score = sum(q[t, lo:hi, h] @ s.counts[ids[:P], h, t].double().T.contiguous() for t in range(T))
                order = torch.sort(score, dim=1, descending=True, stable=True).indices
                chosen[:, h].scatter_(1, order[:, :min(c["sel"], P)], True)
            if c["kind"] == "select":
                continue
            see = (chosen[:, h, :len(ids)].repeat_interleave(PAGE, 1)[:, :J] if c["sel"]
                   else torch.ones(M, J, dtype=torch.bool, device=DEV))
            V = torch.zeros(M, dh, dtype=torch.int64, device=DEV)
            for t in range(T):
                k = _unpack(s.k_pages[ids, h, t]).reshape(-1, dh)[:J].double()
                sc = (q[t, lo:hi, h] @ k.T.contiguous()).long()
                p = s.lut.double()[sc] * see
                v = _unpack(s.v_pages[ids, h, t].unsqueeze(-1)).transpose(1, 2).reshape(-1, dh)[:J].double()
                num, den = (p @ v).long(), p.sum(1, keepdim=True).long()
                a = torch.where(den > 0, (256 * num) // den.clamp(min=1), 0)
                cur[t, lo:hi, h * dh:(h + 1) * dh] = a.int()
                V = V + a
                f = V >= s.theta
                V = V - s.theta * f.long()
                spk[t, lo:hi, h * dh // 64:(h + 1) * dh // 64] = _pack(f)
        sel[lo:hi] = _pack(chosen)
    if c["kind"] in ("select", "serve"):
        out.append(sel)
    if c["kind"] in ("attn", "serve"):
        out += [cur if c["cur"] else None, spk]
    return out
