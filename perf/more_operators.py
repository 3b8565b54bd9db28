"""Timed calls of drafted decoding: spike attention whose rows see different
keys, tokens drawn from the head's logits, and verification of drafted tokens.

Kinds of case
  attn    spike attention of M rows over a contiguous cache; a row sees the
          cache rows of two ranges, [r0, r1) and [r2, r3), and the scores may
          get a bias by the distance of the positions
  sample  a token of each row of logits at a temperature, from given numbers
  verify  drafted tokens against the target's probabilities, from given numbers

Masks of the attn cases
  draft   the pass that verifies B drafted tokens: a pending token and the drafts,
          each seeing what is before it, then B + 1 masked rows, each seeing the
          tokens before its position and itself (M = 2 B + 2)
  blocks  a sequence scored in one pass: its L tokens, block-causal, then L masked
          rows, each seeing the blocks before its own and its own block's masked
          rows (M = 2 L)
  docs    documents one after the other, each seeing itself alone; the last
          rows belong to none and see nothing
  prefix  the first `span` rows see each other, the others what is before them
  window  the first four keys and the last `span` ones

Layouts.  Spikes are bits: q [T][M][d/64] words, keys [T][cap][d/64], values
[T][cap/64][d] with bit j%64 of word (t, j/64, c) for position j.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
DEV = "cuda"
THETA = 160
FLOOR = -700.0  # exponents below weigh nothing


# ----------------------------------------------------------------------------
# cases
# ----------------------------------------------------------------------------
def _attn(mask, M, ctx, T=4, H=16, dh=128, **kw):
    c = dict(kind="attn", mask=mask, M=M, ctx=ctx, T=T, H=H, dh=dh, span=0, dist=-1, cur=False, mix=1)
    c.update(kw)
    return c


def _sample(M, V, **kw):
    return dict(dict(kind="sample", M=M, V=V, temp=0.8, ban=0.0, mix=1), **kw)


def _verify(n, drafts, V, **kw):
    return dict(dict(kind="verify", n=n, drafts=drafts, V=V, temp=0.8, dtemp=0.8, near=0.5, ban=0.0,
                     bonus=True, sure=False, chain=True, mix=1), **kw)


def listed():
    return [
        # one token of a short chat, a small head layout: latency
        _attn("prefix", 1, 300, H=8, dh=64, name="token_short"),
        # one token over a very long context, scores falling with the distance
        _attn("prefix", 1, 130000, dist=64, name="token_long"),
        # the target's pass over 16 drafted tokens behind a usual context
        _attn("draft", 34, 1024, name="draft_block"),
        # 8 drafted tokens behind a long context, with a distance bias
        _attn("draft", 18, 65000, dist=128, name="draft_long"),
        # a document of 1024 tokens scored block by block in one pass
        _attn("blocks", 2048, 0, span=32, name="score_blocks"),
        # prompts of many lengths in one prefill, odd heads, rows to spare; currents asked for
        _attn("docs", 1501, 0, T=3, H=5, dh=64, span=300, cur=True, name="docs_ragged"),
        # a whole prompt, causal behind a prefix, with a distance bias
        _attn("prefix", 2048, 0, span=100, dist=128, name="prompt_bias"),
        # a denoising step draws a token for each masked row
        _sample(32, 32000, name="sample_step"),
        # the steps of many sequences at once
        _sample(1000, 32000, temp=1.0, ban=0.1, name="sample_wave"),
        # one request: 8 drafted tokens and the one that follows them
        _verify(1, 8, 32000, name="verify_one"),
        # a batch of requests
        _verify(64, 8, 32000, ban=0.05, name="verify_wave"),
        # rows by themselves, drafts taken as certain, an odd vocabulary
        _verify(90, 5, 5003, bonus=False, sure=True, chain=False, name="verify_each"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Another case of the same ranges, below the largest listed one's cost."""
    kind = rng.choice(["attn", "attn", "attn", "sample", "verify"])
    mix = rng.randrange(1, 1 << 20)
    if kind == "sample":
        V = _log(rng, 50, 130000)
        M = _log(rng, 1, max(1, min(1000, 32000000 // V)))
        return _sample(M, V, temp=rng.choice([0.0, 0.5, 0.8, 1.0, 1.3]), ban=rng.choice([0.0, 0.0, 0.3]), mix=mix)
    if kind == "verify":
        V = _log(rng, 50, 130000)
        drafts = rng.randrange(1, 17)
        n = _log(rng, 1, max(1, min(96, 16000000 // (V * (drafts + 1)))))
        return _verify(n, drafts, V, temp=rng.choice([0.0, 0.6, 0.8, 1.0]), dtemp=rng.choice([0.6, 0.8, 1.0]),
                       near=rng.choice([0.2, 0.5, 1.0]), ban=rng.choice([0.0, 0.2]), bonus=rng.random() < 0.7,
                       sure=rng.random() < 0.3, chain=rng.random() < 0.7, mix=mix)
    T, dh = rng.choice([1, 2, 3, 4, 4, 6, 8]), rng.choice([64, 128])
    H = rng.choice([1, 2, 4, 5, 8, 12, 16])
    dist = rng.choice([-1, -1, 0, 8, 64, 128, 1000])
    cur = rng.random() < 0.3
    mask = rng.choice(["draft", "draft", "blocks", "docs", "prefix", "prefix", "window"])
    most = int(1.5e10) // (T * H * dh)  # rows times keys
    if mask == "blocks":
        L = _log(rng, 8, max(9, min(1024, int(math.sqrt(most / 4)))))
        return _attn(mask, 2 * L, 0, T, H, dh, span=_log(rng, 1, 64), dist=dist, cur=cur, mix=mix)
    if mask == "docs":
        M = _log(rng, 8, max(9, min(2048, int(math.sqrt(most)))))
        return _attn(mask, M, 0, T, H, dh, span=_log(rng, 2, 900), dist=dist, cur=cur, mix=mix)
    if mask == "draft":
        M = 2 * _log(rng, 1, 32) + 2
    else:
        M = rng.choice([1, 1, 2, _log(rng, 1, 1500)])
    ctx = _log(rng, 1, max(2, min(100000, most // M)))
    return _attn(mask, M, ctx - 1, T, H, dh, span=_log(rng, 1, 2000), dist=dist, cur=cur, mix=mix)


# ----------------------------------------------------------------------------
# inputs: from the seed alone (lengths and masks from the case)
# ----------------------------------------------------------------------------
def _mask(c):
    """Ranges [M][4] and positions of the rows, positions of the keys."""
    M, ctx, span = c["M"], c["ctx"], c["span"]
    i = np.arange(M)
    r = np.zeros((M, 4), np.int64)
    pos = ctx + i
    if c["mask"] == "draft":
        B = M // 2 - 1
        step = i % (B + 1)
        late = i > B
        pos = ctx + step + late
        r[:, 1] = ctx + step + 1
        r[late, 2] = (ctx + i)[late]
        r[late, 3] = (ctx + i + 1)[late]
    elif c["mask"] == "blocks":
        L = M // 2
        pos = i % L
        b0 = pos // span * span
        b1 = np.minimum(b0 + span, L)
        late = i >= L
        r[:, 1] = np.where(late, b0, b1)
        r[late, 2] = (L + b0)[late]
        r[late, 3] = (L + b1)[late]
    elif c["mask"] == "docs":
        rng = np.random.default_rng([c["mix"], M, span])
        at = 0
        while at < M - M // 20:
            n = min(int(math.exp(rng.uniform(0, math.log(span + 1)))) + 1, M - M // 20 - at)
            r[at:at + n, :2] = at, at + n
            pos[at:at + n] = np.arange(n)
            at += n
    elif c["mask"] == "prefix":
        r[:, 1] = np.maximum(pos + 1, min(ctx + span, ctx + M) if span else 0)
    else:
        r[:, 1] = np.minimum(pos + 1, 4)
        r[:, 2] = np.maximum(pos + 1 - span, r[:, 1])
        r[:, 3] = pos + 1
    return r, pos, np.concatenate([np.arange(ctx), pos])


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


def _spikes(g, rate, T, rows):
    """Words [T][rows][d/64] of spikes at the channels' rates [T][d]."""
    out = [_pack(torch.rand(T, min(4096, rows - m), rate.shape[1], device=DEV, generator=g) < rate[:, None])
           for m in range(0, rows, 4096)]
    return torch.cat(out, 1)


def _attn_inputs(c, seed):
    s = SimpleNamespace(c=c)
    T, H, dh, M = c["T"], c["H"], c["dh"], c["M"]
    d = H * dh
    ranges, pos, k_pos = _mask(c)
    s.n_keys = len(k_pos)
    s.cap = -(-s.n_keys // 64) * 64 + 64
    s.ranges, s.q_pos, s.k_pos = _dev(ranges), _dev(pos), _dev(k_pos)
    g = _gen(seed, 21)
    rate = (torch.rand(T, d, device=DEV, generator=g) ** 3).clamp(0.01, 0.9)
    s.q = _spikes(g, rate, T, M)
    s.k = _spikes(g, rate, T, s.cap)
    v = torch.rand(T, d, device=DEV, generator=g)
    s.v = torch.empty(T, s.cap // 64, d, dtype=torch.int64, device=DEV)
    for p in range(0, s.cap // 64, 256):
        n = min(256, s.cap // 64 - p)
        s.v[:, p:p + n] = _pack(torch.rand(T, n, d, 64, device=DEV, generator=g) < v[:, None, :, None]).squeeze(-1)
    s.lut = torch.randint(1, 256, (256,), device=DEV, generator=g).sort().values.to(torch.uint8)
    s.bias = None
    if c["dist"] >= 0:  # falls with the distance, by the head, with some noise
        D = c["dist"]
        off = torch.arange(-D, D + 1, device=DEV).abs()
        slope = 30.0 * 2.0 ** (-torch.arange(H, device=DEV) % 8).float()
        b = 12 - slope[:, None] * off / (D + 1) + torch.randn(H, 2 * D + 1, device=DEV, generator=g)
        s.bias = b.round().clamp(-128, 127).to(torch.int8)
    return s


def _logits(g, M, V, ban):
    """As the head makes them: an integer sum times a scale of the id; some ids
    are ruled out."""
    scale = (torch.rand(V, device=DEV, generator=g) + 0.5) * 2.0 ** -10
    acc = (torch.randn(M, V, device=DEV, generator=g) * 2500).round()
    acc.scatter_add_(1, torch.randint(0, V, (M, 8), device=DEV, generator=g),
                     (torch.rand(M, 8, device=DEV, generator=g) * 9000).round())
    x = acc * scale
    if ban:
        x = x.masked_fill(torch.rand(V, device=DEV, generator=g) < ban, -math.inf)
    return x


def _verify_inputs(c, seed):
    s = SimpleNamespace(c=c)
    rng = np.random.default_rng([c["mix"], c["n"], c["drafts"], c["V"]])
    rows = rng.integers(1, c["drafts"] + 1, size=c["n"]) if c["n"] > 1 else np.array([c["drafts"]])
    rows = rows + int(c["bonus"])
    s.cu = _dev(np.concatenate([[0], np.cumsum(rows)]))
    s.used = int(rows.sum())
    s.R = s.used + 3  # rows behind the last request
    g = _gen(seed, 31)
    V = c["V"]
    s.p = _logits(g, s.R, V, c["ban"])
    s.qd = None if c["sure"] else s.p + torch.randn(s.R, V, device=DEV, generator=g) * c["near"]
    # drafts: drawn from the draft's distribution
    x = (s.p if c["sure"] else s.qd) / c["dtemp"]
    e = -torch.log(torch.rand(s.R, V, device=DEV, generator=g) + 1e-20)
    s.draft = (x - torch.log(e + 1e-20)).argmax(1).to(torch.int32)
    if c["bonus"]:
        s.draft[s.cu[1:].long() - 1] = -1
    s.u = torch.rand(s.R, 2, device=DEV, generator=g)
    return s


def _inputs(c, seed):
    if c["kind"] == "attn":
        return _attn_inputs(c, seed)
    if c["kind"] == "verify":
        return _verify_inputs(c, seed)
    s = SimpleNamespace(c=c)
    g = _gen(seed, 41)
    s.logits = _logits(g, c["M"], c["V"], c["ban"])
    s.u = torch.rand(c["M"], device=DEV, generator=g)
    return s


def prepare(case, seed):
    c = case
    s = _inputs(c, seed)
    i32 = dict(dtype=torch.int32, device=DEV)
    if c["kind"] == "attn":
        T, H, dh, M = c["T"], c["H"], c["dh"], c["M"]
        s.a = torch.zeros(T, M, H * dh, **i32) if c["cur"] else None
        s.spk = torch.zeros(T, M, H * dh // 64, dtype=torch.int64, device=DEV)
        if own:
            from paper_2607_24841_amd import binding as B

            s.mask = B.Mask(s.ranges, q_pos=s.q_pos, k_pos=s.k_pos, max_dist=max(c["dist"], 0))
            s.ws = B.workspace(B.nmdlm_bbm_attn_masked_workspace_size(T, M, s.n_keys, H, dh))
    elif c["kind"] == "sample":
        s.tokens = torch.zeros(c["M"], **i32)
        s.conf = torch.zeros(c["M"], dtype=torch.float64, device=DEV)
    else:
        s.tokens = torch.zeros(s.R, **i32)
        s.accepted = torch.zeros(s.R, dtype=torch.uint8, device=DEV)
        s.n_acc = torch.zeros(c["n"], **i32)
        s.conf = torch.zeros(s.R, dtype=torch.float64, device=DEV)
    return s


# ----------------------------------------------------------------------------
# the calls
# ----------------------------------------------------------------------------
def run(s):
    c = s.c
    if own:
        from paper_2607_24841_amd import binding as B

        if c["kind"] == "attn":
            B.nmdlm_bbm_attn_masked(s.q, s.k, s.v, s.cap, c["T"], c["M"], s.n_keys, c["H"], c["dh"], s.lut,
                                    s.mask, bias=s.bias, a_out=s.a, theta_a=THETA, s_out=s.spk, ws=s.ws)
        elif c["kind"] == "sample":
            B.nmdlm_token_sample(s.logits, c["M"], c["V"], c["temp"], s.u, s.tokens, conf=s.conf)
        else:
            B.nmdlm_draft_verify(s.p, s.qd, s.R, c["V"], s.draft, s.u, c["temp"], c["dtemp"], s.tokens,
                                 s.accepted, cu_rows=s.cu, n_seq=c["n"], n_accepted=s.n_acc, conf=s.conf,
                                 chain=c["chain"])
    elif c["kind"] == "attn":
        _attn_plain(s)
    elif c["kind"] == "sample":
        _sample_plain(s)
    else:
        _verify_plain(s)
    if c["kind"] == "attn":
        return [s.a, s.spk]
    if c["kind"] == "sample":
        return [s.tokens, s.conf]
    return [s.tokens, s.accepted, s.n_acc, s.conf]


# ----------------------------------------------------------------------------
# plain forms
# ----------------------------------------------------------------------------
def _attn_plain(s):
    c = s.c
    T, H, dh, M, J = c["T"], c["H"], c["dh"], c["M"], s.n_keys
    lut = s.lut.float()
    q = _unpack(s.q).reshape(T, M, H, dh).permute(0, 2, 1, 3).float().contiguous()
    num = torch.zeros(T, H, M, dh, dtype=torch.float64, device=DEV)
    den = torch.zeros(T, H, M, 1, dtype=torch.float64, device=DEV)
    # keys a product: the sums of the table's weights stay below 2^24 and the scores fit
    step = max(64, min(16384, (1 << 28) // (T * H * M * 64) * 64))
    for j in range(0, J, step):
        n = min(step, J - j)
        key = torch.arange(j, j + n, device=DEV)
        k = _unpack(s.k[:, j:j + n]).reshape(T, n, H, dh).permute(0, 2, 3, 1).float().contiguous()
        idx = (q @ k).to(torch.int32)
        if s.bias is not None:
            off = (s.q_pos[:, None] - s.k_pos[None, j:j + n]).clamp(-c["dist"], c["dist"]) + c["dist"]
            idx = (idx + s.bias.int()[:, off]).clamp(0, 255)
        r = s.ranges[:, :, None]
        see = ((key >= r[:, 0]) & (key < r[:, 1])) | ((key >= r[:, 2]) & (key < r[:, 3]))
        p = lut[idx] * see
        w0, w1 = j // 64, -(-(j + n) // 64)
        v = _unpack(s.v[:, w0:w1].unsqueeze(-1)).permute(0, 2, 1, 3).reshape(T, H, dh, -1)[..., :n]
        num += p @ v.transpose(2, 3).float().contiguous()
        den += p.sum(3, keepdim=True, dtype=torch.float64)
    a = torch.where(den > 0, (256 * num.long()) // den.long().clamp(min=1), 0)
    a = a.permute(0, 2, 1, 3).reshape(T, M, H * dh)
    if s.a is not None:
        s.a.copy_(a)
    V = torch.zeros_like(a[0])
    for t in range(T):
        V = V + a[t]
        f = V >= THETA
        V = V - THETA * f
        s.spk[t] = _pack(f)


def _weights(logits, temp):
    """exp((l - max) / temp) in 64 bits (at temperature 0: 1 at the first of the
    largest), its largest logits' mask and whether the row has any."""
    x = logits.double().nan_to_num(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    top = x.amax(1, keepdim=True)
    some = top > -math.inf
    x = torch.where(x == top, 0.0, (x - top) * (1.0 / (temp if temp else 1.0)))
    w = torch.where(x >= FLOOR, x.exp(), 0.0) * some
    first = torch.where(x == 0, torch.arange(x.shape[1], device=DEV), x.shape[1]).amin(1, keepdim=True)
    return w, first, some


def _pick(w, u):
    """First id whose running sum exceeds u times the sum (the last of positive
    weight when none does)."""
    cs = w.cumsum(1)
    at = torch.searchsorted(cs, (u.double()[:, None] * cs[:, -1:]), right=True)
    last = torch.where(w > 0, torch.arange(w.shape[1], device=DEV), 0).amax(1, keepdim=True)
    return torch.minimum(at, last)


def _sample_plain(s):
    c = s.c
    w, first, some = _weights(s.logits, c["temp"])
    at = first if c["temp"] == 0 else _pick(w, s.u)
    s.conf.copy_((w.gather(1, at) / w.sum(1, keepdim=True)).where(some, 0.0)[:, 0])
    s.tokens.copy_(at.where(some, -1)[:, 0])


def _verify_plain(s):
    c = s.c
    n, V = s.used, c["V"]
    w, first, some = _weights(s.p[:n], c["temp"])
    p = conf = torch.where(some, w / w.sum(1, keepdim=True), 0.0)
    if c["temp"] == 0:
        p = torch.zeros_like(w).scatter_(1, first, 1.0) * some
    x = s.draft[:n].long()[:, None]
    real = (x >= 0) & (x < V)
    x = x.clamp(0, V - 1)
    if s.qd is None:
        q = torch.zeros_like(p).scatter_(1, x, 1.0)
    else:
        wq, firstq, someq = _weights(s.qd[:n], c["dtemp"])
        q = torch.where(someq, wq / wq.sum(1, keepdim=True), 0.0)
        if c["dtemp"] == 0:
            q = torch.zeros_like(wq).scatter_(1, firstq, 1.0) * someq
    take = real & (s.u[:n, :1].double() * q.gather(1, x) < p.gather(1, x))
    r = torch.where(real, (p - q).clamp(min=0), p)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    tok = torch.where(take, x, torch.where(some, _pick(r, s.u[:n, 1]), -1))
    pr = conf.gather(1, tok.clamp(min=0)).where(tok >= 0, 0.0)
    tok, pr, take = tok[:, 0], pr[:, 0], take[:, 0]
    cu = s.cu.long()
    of = torch.searchsorted(cu[1:].contiguous(), torch.arange(n, device=DEV), right=True)
    if c["chain"]:
        over = torch.nn.functional.pad((~take).long().cumsum(0), (1, 0))  # refusals before a row
        alive = over[:n] == over[cu[of]]
        tok, pr, take = tok.where(alive, -1), pr.where(alive, 0.0), take & alive
    s.tokens[:n] = tok.int()
    s.accepted[:n] = take.to(torch.uint8)
    s.conf[:n] = pr
    s.n_acc.copy_(torch.zeros(c["n"], dtype=torch.int64, device=DEV).index_add_(0, of, take.long()))


# ----------------------------------------------------------------------------
# what a pass cannot do without
# ----------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "sample":
        return dict(bytes=c["M"] * (4.0 * c["V"] + 16), flops=4.0 * c["M"] * c["V"])
    if c["kind"] == "verify":
        s = np.random.default_rng([c["mix"], c["n"], c["drafts"], c["V"]])
        rows = s.integers(1, c["drafts"] + 1, size=c["n"]) if c["n"] > 1 else np.array([c["drafts"]])
        rows = float(rows.sum())
        extra = c["n"] * float(c["bonus"])  # a row without a draft needs the target's logits alone
        by = rows * (4.0 if c["sure"] else 8.0) * c["V"] + extra * 4.0 * c["V"] + 25 * (rows + extra)
        return dict(bytes=by, flops=8.0 * (rows + extra) * c["V"])
    T, H, d, M = c["T"], c["H"], c["H"] * c["dh"], c["M"]
    r, pos, k_pos = _mask(c)
    seen = np.zeros(len(k_pos) + 1, np.int64)
    np.add.at(seen, r[:, 0], 1)
    np.add.at(seen, r[:, 1], -1)
    np.add.at(seen, r[:, 2], 1)
    np.add.at(seen, r[:, 3], -1)
    keys = float((np.cumsum(seen)[:-1] > 0).sum())
    pairs = float((r[:, 1] - r[:, 0] + r[:, 3] - r[:, 2]).sum())
    by = 2 * T * d * keys / 8 + 2 * T * M * d / 8 + 16 * M + 4 * T * M * d * c["cur"]
    if c["dist"] >= 0:
        by += 4 * (M + keys) + H * (2 * c["dist"] + 1)
    return dict(bytes=by, flops=4 * T * d * pairs)


# ----------------------------------------------------------------------------
# the same from the definitions in 64 bits
# ----------------------------------------------------------------------------
def exact(case, seed):
    c = case
    s = _inputs(c, seed)
    if c["kind"] == "attn":
        return _attn_exact(s)
    if c["kind"] == "sample":
        tok, conf = np.zeros(c["M"], np.int32), np.zeros(c["M"])
        u = s.u.cpu().numpy().astype(np.float64)
        for m, l in enumerate(s.logits.cpu().numpy().astype(np.float64)):
            p, p1 = _probabilities(l, c["temp"])
            tok[m] = _draw_id(p, u[m])
            conf[m] = p1[tok[m]] if tok[m] >= 0 else 0.0
        return [_dev(tok), _dev(conf, torch.float64)]
    R, V = s.R, c["V"]
    tok, acc, conf, n_acc = np.zeros(R, np.int32), np.zeros(R, np.uint8), np.zeros(R), np.zeros(c["n"], np.int32)
    cu, draft, u = s.cu.cpu().numpy(), s.draft.cpu().numpy(), s.u.cpu().numpy().astype(np.float64)
    for r in range(c["n"]):
        ended = False
        for m in range(cu[r], cu[r + 1]):
            if ended:
                tok[m] = -1
                continue
            p, p1 = _probabilities(s.p[m].cpu().numpy().astype(np.float64), c["temp"])
            x = int(draft[m])
            left = p
            if 0 <= x < V:
                if s.qd is None:
                    q = np.zeros(V)
                    q[x] = 1.0
                else:
                    q = _probabilities(s.qd[m].cpu().numpy().astype(np.float64), c["dtemp"])[0]
                if u[m, 0] * q[x] < p[x]:
                    tok[m], acc[m], conf[m] = x, 1, p1[x]
                    n_acc[r] += 1
                    continue
                left = np.maximum(p - q, 0.0)
                left = left if left.sum() > 0 else p
            tok[m] = _draw_id(left, u[m, 1])
            conf[m] = p1[tok[m]] if tok[m] >= 0 else 0.0
            ended = c["chain"]
    return [_dev(tok), _dev(acc, torch.uint8), _dev(n_acc), _dev(conf, torch.float64)]


def _probabilities(l, temp):
    """Softmax of a row at the temperature (0: all on the first of the largest),
    and the one that confidences are taken from."""
    l = np.where(np.isnan(l), -np.inf, l)
    top = l.max()
    if top == -np.inf:
        return np.zeros(len(l)), np.zeros(len(l))
    with np.errstate(invalid="ignore"):
        e = np.where(l == top, 0.0, (l - top) / (temp or 1.0))
    w = np.where(e >= FLOOR, np.exp(e), 0.0)
    p1 = w / math.fsum(w)
    if temp:
        return p1, p1
    p = np.zeros(len(l))
    p[int(np.argmax(l == top))] = 1.0
    return p, p1


def _draw_id(p, u):
    if not p.any():
        return -1
    cs = np.cumsum(p)
    return min(int(np.searchsorted(cs, u * cs[-1], side="right")), int(np.flatnonzero(p)[-1]))


def _attn_exact(s):
    c = s.c
    T, H, dh, M, J = c["T"], c["H"], c["dh"], c["M"], s.n_keys
    r, pos, k_pos = (torch.as_tensor(x, device=DEV) for x in _mask(c))
    key = torch.arange(J, device=DEV)
    out = torch.zeros(T, M, H * dh, dtype=torch.int32, device=DEV)
    spk = torch.zeros(T, M, H * dh // 64, dtype=torch.int64, device=DEV)
    for m in range(0, M, 512):
        rm = r[m:m + 512, :, None]
        first, second = (key >= rm[:, 0]) & (key < rm[:, 1]), (key >= rm[:, 2]) & (key < rm[:, 3])
        see = (first | second).double()
        off = (pos[m:m + 512, None] - k_pos[None]).clamp(-max(c["dist"], 0), max(c["dist"], 0)) + max(c["dist"], 0)
        for h in range(H):
            w = slice(h * dh // 64, (h + 1) * dh // 64)
            b = s.bias[h].long()[off] if s.bias is not None else 0
            V = torch.zeros(see.shape[0], dh, dtype=torch.int64, device=DEV)
            for t in range(T):
                q = _unpack(s.q[t, m:m + 512, w]).double()
                k = _unpack(s.k[t, :J, w]).double()
                p = s.lut.double()[((q @ k.T.contiguous()).long() + b).clamp(0, 255)] * see
                v = _unpack(s.v[t, :, h * dh:(h + 1) * dh].unsqueeze(-1)).transpose(1, 2).reshape(-1, dh)[:J]
                num, den = (p @ v.double()).long(), p.sum(1, keepdim=True).long()
                a = torch.where(den > 0, (256 * num) // den.clamp(min=1), 0)
                out[t, m:m + 512, h * dh:(h + 1) * dh] = a.int()
                V = V + a
                f = V >= THETA
                V = V - THETA * f.long()
                spk[t, m:m + 512, w] = _pack(f)
    return [out if c["cur"] else None, spk]
