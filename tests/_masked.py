"""Cases of the masked attention and of the verification of drafts: masks,
inputs, and the same on the GPU."""
from types import SimpleNamespace

import numpy as np

from oracle import nmdlm_oracle as O
from workloads import synth


def draft_mask(ctx, B):
    """A pending token and B drafts behind ctx keys, then B + 1 masked rows."""
    r, pos = [], []
    for i in range(B + 1):
        r.append((0, ctx + i + 1, 0, 0))
        pos.append(ctx + i)
    for i in range(B + 1):
        r.append((0, ctx + i + 1, ctx + B + 1 + i, ctx + B + 2 + i))
        pos.append(ctx + i + 1)
    return np.array(r), np.array(pos)


def blocks_mask(L, S):
    i = np.arange(L)
    b0, b1, z = i // S * S, np.minimum(i // S * S + S, L), np.zeros(L, int)
    return np.concatenate([np.stack([z, b1, z, z], 1), np.stack([z, b0, L + b0, L + b1], 1)]), np.concatenate([i, i])


def docs_mask(lengths, spare):
    r, pos, at = [], [], 0
    for n in lengths:
        r += [(at, at + n, 0, 0)] * n
        pos += list(range(n))
        at += n
    return np.array(r + [(0, 0, 0, 0)] * spare), np.array(pos + [0] * spare)


def window_mask(ctx, M, W):
    i = ctx + np.arange(M)
    return np.stack([0 * i, np.minimum(i + 1, 4), np.maximum(i + 1 - W, 0), i + 1], 1), i


def random_mask(rng, M, J):
    """Any ranges: empty, overlapping, reversed, past the keys."""
    return rng.integers(-20, J + 40, size=(M, 4)), rng.integers(0, 2 * J, size=M)


def make_case(seed, ranges, q_pos, n_keys, T=4, H=2, dh=64, max_dist=None, rate=0.3, theta=150, k_pos=None):
    rng = np.random.default_rng([91, seed])
    M, d = len(ranges), H * dh
    c = SimpleNamespace(T=T, M=M, H=H, dh=dh, d=d, n_keys=n_keys, theta=theta, max_dist=max_dist or 0)
    c.cap = -(-n_keys // 64) * 64 + 64
    c.ranges, c.q_pos = np.asarray(ranges, np.int32), np.asarray(q_pos, np.int32)
    c.k_pos = np.asarray(k_pos if k_pos is not None else np.arange(n_keys), np.int32)
    c.q = synth.bernoulli(rng, rate, (T, M, d))
    c.k, c.v = (synth.bernoulli(rng, rate, (T, c.cap, d)) for _ in range(2))
    c.lut = synth.sorted_lut_u8(rng)
    c.bias = None
    if max_dist is not None:
        c.bias = rng.integers(-128, 128, size=(H, 2 * max_dist + 1)).astype(np.int8)
    return c


def route(T, M, n_keys, H):
    """The kernel a call takes (a host-side query): rows of a workgroup (1: the row
    kernel), waves per timestep, most splits, whether workgroups take several heads."""
    import ctypes as C

    from paper_2607_24841_amd import binding as B

    out = (C.c_int32 * 4)()
    B.load().nmdlm_internal_masked_route(T, M, n_keys, H, out)
    return SimpleNamespace(tile=out[0], parts=out[1], splits=out[2], heads=bool(out[3]))


def attention(c):
    a = O.masked_attention(c.q, c.k[:, :c.n_keys], c.v[:, :c.n_keys], c.H, c.lut, np.clip(c.ranges, 0, c.n_keys),
                           c.bias, c.q_pos, c.k_pos, c.max_dist)
    return a, O.if_neuron(a, c.theta)[0]


class Device:
    """The case on the GPU; outputs begin at -9 and all ones."""

    def __init__(self, torch, B, c, device="cuda"):
        self.torch, self.B, self.c, self.device = torch, B, c, device
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(device)  # noqa: E731
        self.q, self.k = (B.to_dev_bits(synth.pack_bits(x), device) for x in (c.q, c.k))
        v = c.v.reshape(c.T, c.cap // 64, 64, c.d).transpose(0, 1, 3, 2)
        self.v = B.to_dev_bits(synth.pack_bits(v)[..., 0], device)
        self.lut = dev(c.lut)
        self.bias = None if c.bias is None else dev(c.bias)
        self.mask = B.Mask(dev(c.ranges), dev(c.q_pos), dev(c.k_pos), c.max_dist)
        self.cur = torch.full((c.T, c.M, c.d), -9, dtype=torch.int32, device=device)
        self.spk = torch.full((c.T, c.M, c.d // 64), -1, dtype=torch.int64, device=device)
        self.ws = B.workspace(B.nmdlm_bbm_attn_masked_workspace_size(c.T, c.M, c.n_keys, c.H, c.dh), device)

    def run(self, cur=True, spk=True, **kw):
        c = self.c
        self.B.nmdlm_bbm_attn_masked(self.q, self.k, self.v, c.cap, c.T, c.M, c.n_keys, c.H, c.dh, self.lut,
                                     self.mask, bias=self.bias, a_out=self.cur if cur else None,
                                     theta_a=c.theta if spk else 0, s_out=self.spk if spk else None,
                                     ws=self.ws, **kw)

    def spikes(self):
        return synth.unpack_bits(self.B.from_dev_bits(self.spk), self.c.d)


# ----------------------------------------------------------------------------
def logits(rng, M, V, spread=1500):
    """As the head makes them: an integer times a scale of the id."""
    scale = ((rng.random(V) + 0.5) * 2.0 ** -10).astype(np.float32)
    return np.rint(rng.normal(size=(M, V)) * spread).astype(np.float32) * scale


def drafts(rng, draft_logits, tau):
    """Drafts drawn from their distribution."""
    return O.token_sample(draft_logits, tau, rng.random(len(draft_logits)))[0]
