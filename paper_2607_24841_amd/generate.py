"""Block-diffusion generation driver (Eq. (2)): prompt prefill, then per block
``steps`` calls of nmdlm_block_step that reveal ``k_unmask`` tokens each; a
finished block's keys/values stay in the caches as context.  The host only
loops and marshals; every step runs in libnmdlm's kernels and the token
state stays on the device until the end.  Several sequences (prompts of
one length) advance together, one batched step per denoising step; requests
of different lengths share pools of pages (PagedGenerator).  DraftedGenerator
goes left to right: a cheaper model drafts a block in one step, one masked step of
the model checks all of it."""
from __future__ import annotations

import numpy as np
import torch

from . import binding as B


class Generator:
    def __init__(self, dm: B.DeviceModel, prompt_len: int, block: int, n_seq: int = 1):
        self.dm = dm
        self.B = block
        self.n = n_seq
        nb = max(B.nmdlm_block_step_workspace_size(dm, n_seq * prompt_len, B.NMDLM_NO_HEAD),
                 B.nmdlm_block_step_workspace_size(dm, n_seq * block, 0))
        self.ws = B.workspace(nb)
        self.tokens = torch.zeros(n_seq * block, dtype=torch.int32, device="cuda")
        self.masked = torch.ones(n_seq * block, dtype=torch.uint8, device="cuda")
        self.chosen = torch.zeros((n_seq, block), dtype=torch.int32, device="cuda")

    def prefill(self, prompt_ids: torch.Tensor) -> int:
        """prompt_ids: the n_seq prompts one after the other."""
        P = int(prompt_ids.numel()) // self.n
        masked = torch.zeros(self.n * P, dtype=torch.uint8, device="cuda")
        io = B.step_io(P, 0, pos0=0, flags=B.NMDLM_NO_HEAD, tokens=prompt_ids, masked=masked,
                       n_seq=self.n)
        B.nmdlm_block_step(self.dm, io, self.ws)
        return P

    def run_block(self, C: int, steps: int, k_unmask: int, log: list | None = None) -> torch.Tensor:
        self.tokens.zero_()
        self.masked.fill_(1)
        # chosen positions: [n_seq][k_unmask] packed at the front of the buffer
        chosen_k = self.chosen.view(-1)[:self.n * k_unmask].view(self.n, k_unmask)
        for _ in range(steps):
            io = B.step_io(self.B, C, pos0=C, flags=0, tokens=self.tokens, masked=self.masked,
                           k_unmask=k_unmask, unmasked_pos=self.chosen, n_seq=self.n)
            B.nmdlm_block_step(self.dm, io, self.ws)
            if log is not None:
                log.append(chosen_k.clone())
        return self.tokens.view(self.n, self.B).clone()

    def run(self, prompt_ids: torch.Tensor, n_blocks: int, steps: int, k_unmask: int,
            log: list | None = None) -> torch.Tensor:
        """Generated ids [n_seq][n_blocks * block]."""
        C = self.prefill(prompt_ids)
        out = []
        for _ in range(n_blocks):
            out.append(self.run_block(C, steps, k_unmask, log))
            C += self.B
        return torch.cat(out, dim=1)


def generate(dm: B.DeviceModel, prompt: np.ndarray, n_blocks: int, block: int, steps: int,
             k_unmask: int):
    """Returns (generated ids [n_blocks*block], per-step chosen positions)."""
    ids, log = generate_batch(dm, np.asarray(prompt)[None, :], n_blocks, block, steps, k_unmask)
    return ids[0], [c[0] for c in log]


def generate_batch(dm: B.DeviceModel, prompts: np.ndarray, n_blocks: int, block: int, steps: int,
                   k_unmask: int):
    """prompts [n_seq][P] advanced together (one batched step per denoising
    step).  Returns (generated ids [n_seq][n_blocks*block], per-step chosen
    positions [n_seq][k_unmask])."""
    prompts = np.asarray(prompts, dtype=np.int32)
    n, P = prompts.shape
    g = Generator(dm, P, block, n_seq=n)
    log: list = []
    ids = torch.from_numpy(np.ascontiguousarray(prompts).reshape(-1)).cuda()
    out = g.run(ids, n_blocks, steps, k_unmask, log)
    torch.cuda.synchronize()
    return out.cpu().numpy(), [c.cpu().numpy() for c in log]


class PagedGenerator:
    """Block diffusion for up to n_seq requests of different lengths at once.

    Their keys and values live in one pool of pages a layer, `pool` pages of 64
    positions for all requests, at most max_len positions for one (and no more
    than the model's position table has: `limit`).  A request is admitted with
    its prompt, advances by one block a call of run_block and gives its pages
    back when it is released.  n_sel: context pages that a row and head attends
    to besides its block's own (None: all).

    admit and run_block raise ValueError before anything is taken when a request
    would pass its limit; run_block goes on once that request is released.  A
    block has at most NMDLM_MAX_HEAD_M rows, all that a step can unmask."""

    def __init__(self, dm: B.DeviceModel, n_seq: int, block: int, max_len: int, pool: int,
                 max_prompt_rows: int | None = None, n_sel: int | None = None):
        if not 1 <= block <= B.NMDLM_MAX_HEAD_M:
            raise ValueError(f"a block of {block} rows: 1 to {B.NMDLM_MAX_HEAD_M}")
        self.block, self.n, self.n_sel = block, n_seq, -1 if n_sel is None else int(n_sel)
        self.limit = min(max_len, dm.c.max_pos)         # positions of a request
        max_pages = -(-max_len // B.NMDLM_PAGE)
        # prompts go through a plan of their own over the same tables: a step's
        # rows are as many as its plan has room for
        self.pages = B.Pages(n_seq, n_seq * block, max_pages, pool)
        self.prompt_pages = self.pages.view(max_prompt_rows or max_len)
        self.model = B.PagedModel(dm, self.pages)
        self.prompt_model = self.model.view(self.prompt_pages, head=False)
        # a prompt has no context pages to choose from: its step sees all there are
        self.ws = B.workspace(max(
            B.nmdlm_block_step_paged_workspace_size(self.model, 0 if self.n_sel >= 0 else B.NMDLM_ALL_PAGES),
            B.nmdlm_block_step_paged_workspace_size(self.prompt_model, B.NMDLM_NO_HEAD | B.NMDLM_ALL_PAGES)))
        self.ctx = np.zeros(n_seq, dtype=np.int32)      # positions that a request holds
        self.live = np.zeros(n_seq, dtype=bool)
        rows = n_seq * block
        self.tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        self.masked = torch.ones(rows, dtype=torch.uint8, device="cuda")
        self.chosen = torch.zeros(n_seq, block, dtype=torch.int32, device="cuda")
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def _check_lengths(self, new: np.ndarray) -> None:
        """A step has no position spike to give past the position table, so no
        request is taken there."""
        for s in np.flatnonzero((new > 0) & (self.ctx + new > self.limit)):
            raise ValueError(f"request {s}: {self.ctx[s]} positions and {new[s]} new ones, of at most {self.limit}")

    def _plan(self, pages: B.Pages, new: np.ndarray) -> None:
        """Makes the step's plan; raises when a request does not get its pages."""
        self.status.zero_()
        B.nmdlm_page_plan(pages, torch.from_numpy(self.ctx).cuda(),
                          torch.from_numpy(new.astype(np.int32)).cuda(), status=self.status)
        self._check_status()

    def _check_status(self) -> None:
        """Raises for what the plan, or the steps since, have set."""
        bits = int(self.status)
        if bits & B.NMDLM_STATUS_TOKEN_CLAMPED:
            raise ValueError("token ids outside the model's table")
        if bits:
            raise RuntimeError("the pool has too few pages" if bits == B.NMDLM_STATUS_PAGES_SHORT
                               else f"a request is longer than the plan holds (status {bits})")

    def admit(self, prompts: dict[int, np.ndarray]) -> None:
        """Prefills the prompts (request number -> ids of the model's table) in
        one step; when it raises, none of them is admitted."""
        new = np.zeros(self.n, dtype=np.int64)
        for s, ids in prompts.items():
            if not 0 <= s < self.n or self.live[s]:
                raise ValueError(f"request {s}: running, or not one of {self.n}")
            new[s] = len(ids)
        rows = int(new.sum())
        if rows > self.prompt_pages.max_rows or any(n < 1 for n in new[list(prompts)]):
            raise ValueError(f"prompts of {rows} tokens in all: 1 to {self.prompt_pages.max_rows}")
        self._check_lengths(new)
        ids = np.zeros(self.prompt_pages.max_rows, dtype=np.int32)
        # ids beyond 32 bits stay outside the table
        ids[:rows] = np.clip(np.concatenate([np.asarray(prompts[s]) for s in sorted(prompts)]), -1, 2**31 - 1)
        try:
            self._plan(self.prompt_pages, new)
            tokens = torch.from_numpy(ids).cuda()
            io = B.step_io(0, 0, flags=B.NMDLM_NO_HEAD, tokens=tokens, status=self.status)
            B.nmdlm_block_step_paged(self.prompt_model, io, self.ws)
            self._check_status()
        except (RuntimeError, ValueError):   # what they were given goes back
            B.nmdlm_page_plan(self.prompt_pages, torch.from_numpy(self.ctx).cuda(),
                              torch.from_numpy(np.where(new > 0, -1, 0).astype(np.int32)).cuda())
            raise
        for s in prompts:
            self.ctx[s], self.live[s] = new[s], True

    def run_block(self, steps: int, k_unmask: int, log: list | None = None) -> dict[int, torch.Tensor]:
        """One block for every running request: request number -> its ids."""
        order = np.flatnonzero(self.live)
        new = np.where(self.live, self.block, 0)
        self._check_lengths(new)
        self._plan(self.pages, new)
        self.tokens.zero_()
        self.masked.fill_(1)
        chosen = self.chosen.view(-1)[:self.n * k_unmask].view(self.n, k_unmask)
        io = B.step_io(0, 0, tokens=self.tokens, masked=self.masked, k_unmask=k_unmask,
                       unmasked_pos=self.chosen, status=self.status)
        for _ in range(steps):
            B.nmdlm_block_step_paged(self.model, io, self.ws, n_sel=self.n_sel)
            if log is not None:
                log.append(chosen.clone())
        self._check_status()
        self.ctx += new.astype(np.int32)
        out = self.tokens[:len(order) * self.block].view(len(order), self.block).clone()
        return {int(s): out[i] for i, s in enumerate(order)}

    def release(self, requests) -> None:
        """Gives the pages of the requests back."""
        new = np.zeros(self.n, dtype=np.int64)
        for s in requests:
            if not 0 <= s < self.n:
                raise ValueError(f"request {s}: not one of {self.n}")
            new[s] = -1
        self._plan(self.pages, new)
        for s in requests:
            self.ctx[s], self.live[s] = 0, False


class DraftedGenerator:
    """Left-to-right generation of one sequence with drafted blocks.

    A token is distributed as the model `dm` has it at a masked row that sees the
    tokens before (at temperature 0 it is the most likely one).  Each round `draft`,
    a cheaper model, fills a block of `block` masked tokens in one step, and one
    masked step of `dm` computes the distributions behind the pending token and
    behind each draft at once; nmdlm_draft_verify keeps the drafts that stand and
    draws the token that follows them, so a round yields 1 to block + 1 tokens.

    draft: the first layers of dm (dm.view(0, n, head=True)), which share dm's keys and
    values, or another model over the same vocabulary with caches of its own.
    Prompts are read as prefixes whose tokens see each other."""

    def __init__(self, dm: B.DeviceModel, draft, block: int, temperature: float = 1.0,
                 draft_temperature: float | None = None, seed: int = 0):
        if not 1 <= block <= B.NMDLM_MAX_HEAD_M // 2 - 1:
            raise ValueError(f"a block of {block} drafts: 1 to {B.NMDLM_MAX_HEAD_M // 2 - 1}")
        if draft.V != dm.V:
            raise ValueError(f"vocabularies of {dm.V} and {draft.V} tokens")
        n = len(draft.layers)
        self.shared = n > 0 and all(a is b for a, b in zip(draft.layers, dm.layers)) and n <= len(dm.layers)
        if not self.shared and any(a is b for a in draft.layers for b in dm.layers):
            raise ValueError("a draft of the model's own layers takes the first ones")
        self.dm, self.draft, self.block = dm, draft, block
        self.temperature = float(temperature)
        self.draft_temperature = self.temperature if draft_temperature is None else float(draft_temperature)
        self.rng = torch.Generator(device="cuda").manual_seed(seed)
        # rows: the pending token and the drafts, then a masked row behind each of them
        late, i = np.arange(block + 1), np.arange(2 * block + 2)
        rows = np.zeros((2 * block + 2, 4), np.int32)
        rows[:, 1] = i % (block + 1) + 1
        rows[block + 1:, 2], rows[block + 1:, 3] = block + 1 + late, block + 2 + late
        moves = (rows > 0).astype(np.int32)   # ends that go with the context
        i32 = dict(dtype=torch.int32, device="cuda")
        dev = lambda a: torch.as_tensor(a, **i32)  # noqa: E731
        self._rows, self._moves = dev(rows), dev(moves)
        self._pos = dev(np.concatenate([late, late + 1]))
        self.mask = B.Mask(torch.zeros_like(self._rows), q_pos=torch.zeros_like(self._pos))
        self.tokens = torch.zeros(2 * block + 2, **i32)
        self.masked = dev((i > block)).to(torch.uint8)
        self.logits = torch.empty(2 * block + 2, dm.V, device="cuda")
        # the draft's rows: tokens that it has not seen, then the block
        most = block + 1 + block
        self.d_mask = B.Mask(torch.zeros(most, 4, **i32), q_pos=torch.zeros(most, **i32))
        self.d_tokens = torch.zeros(most, **i32)
        self.d_masked = torch.zeros(most, dtype=torch.uint8, device="cuda")
        self.d_logits = torch.empty(most + 1, dm.V, device="cuda")
        self.drafts = torch.full((block + 1,), -1, **i32)   # the last row has none
        self.out = torch.zeros(block + 1, **i32)
        self.accepted = torch.zeros(block + 1, dtype=torch.uint8, device="cuda")
        self.n_accepted = torch.zeros(1, **i32)
        size = B.nmdlm_block_step_masked_workspace_size
        self.ws = B.workspace(max(
            [size(dm, 2 * block + 2, dm.cache_cap)]
            + [size(draft, m, draft.cache_cap) for m in range(block + 1, most + 1) if m <= draft.cache_cap]))
        self.seq: list[int] = []   # all tokens; the last is pending: in no cache
        self.ctx = self.d_ctx = 0  # tokens in the caches of dm and of the draft

    def numbers(self, *shape: int) -> torch.Tensor:
        """The uniform numbers of a round: [block] for the drafts, then [block + 1][2]."""
        return torch.rand(*shape, generator=self.rng, device="cuda")

    def start(self, prompt) -> None:
        """Prefills the prompt, all but its last token."""
        ids = np.asarray(prompt).reshape(-1)
        if len(ids) < 1 or ids.min() < 0 or ids.max() >= self.dm.V:
            raise ValueError(f"a prompt of {len(ids)} tokens: at least one, of ids below {self.dm.V}")
        self._check_room(len(ids) - 1, len(ids) - 1)
        P = len(ids) - 1
        if P > 0:
            t = torch.as_tensor(ids[:P].astype(np.int32)).cuda()
            io = B.step_io(P, 0, flags=B.NMDLM_NO_HEAD, tokens=t)
            for m in [self.dm] + ([] if self.shared else [self.draft]):
                B.nmdlm_block_step(m, io, B.workspace(B.nmdlm_block_step_workspace_size(m, P, B.NMDLM_NO_HEAD)))
        self.seq = [int(x) for x in ids]
        self.ctx = self.d_ctx = P

    def _check_room(self, ctx: int, d_ctx: int) -> None:
        """A round's rows have places in the caches and in the position tables."""
        rows, last = 2 * self.block + 2, ctx + self.block + 1
        if ctx + rows > self.dm.cache_cap or last >= self.dm.c.max_pos:
            raise ValueError(f"{ctx} tokens and {rows} rows: at most {self.dm.cache_cap} in the caches, "
                             f"{self.dm.c.max_pos} positions")
        if ctx + 1 + self.block > self.draft.cache_cap or last > self.draft.c.max_pos:
            raise ValueError(f"{ctx} tokens and a block: at most {self.draft.cache_cap} in the draft's caches")

    def round(self) -> list[int]:
        """The tokens of one round: the drafts that stand and the one that follows them."""
        if not self.seq:
            raise ValueError("no prompt")
        self._check_room(self.ctx, self.d_ctx)
        n, C, D = self.block, self.ctx, self.d_ctx
        # the draft: tokens that its caches lack, then the block
        new = self.seq[D:]
        k, rows = len(new), len(new) + n
        r = np.zeros((rows, 4), np.int32)
        r[:, 1] = np.minimum(D + np.arange(rows) + 1, D + rows)
        r[k:, 1] = D + rows
        self.d_mask.ranges[:rows].copy_(torch.from_numpy(r))
        torch.arange(D, D + rows, out=self.d_mask.q_pos[:rows])
        self.d_tokens[:k].copy_(torch.tensor(new, dtype=torch.int32))
        self.d_masked[:k].zero_()
        self.d_masked[k:rows].fill_(1)
        io = B.step_io(rows, D, tokens=self.d_tokens, masked=self.d_masked, logits=self.d_logits)
        B.nmdlm_block_step_masked(self.draft, io, self.d_mask, self.ws)
        B.nmdlm_token_sample(self.d_logits[k:], n, self.dm.V, self.draft_temperature, self.numbers(n), self.drafts)
        # the model: the pending token, the drafts, and the rows behind them
        torch.add(self._rows, self._moves, alpha=C, out=self.mask.ranges)
        torch.add(self._pos, C, out=self.mask.q_pos)
        self.tokens[:1].fill_(self.seq[-1])
        self.tokens[1:n + 1].copy_(self.drafts[:n])
        io = B.step_io(2 * n + 2, C, tokens=self.tokens, masked=self.masked, logits=self.logits)
        B.nmdlm_block_step_masked(self.dm, io, self.mask, self.ws)
        B.nmdlm_draft_verify(self.logits[n + 1:], self.d_logits[k:], n + 1, self.dm.V, self.drafts,
                             self.numbers(n + 1, 2), self.temperature, self.draft_temperature, self.out,
                             self.accepted, n_accepted=self.n_accepted)
        got = self.out[:int(self.n_accepted) + 1].tolist()
        # dm has the pending token and the drafts that stand; the draft what it was given
        self.ctx = C + len(got)
        self.d_ctx = self.ctx if self.shared else D + k
        self.seq += got
        return got

    def run(self, prompt, n_tokens: int) -> list[int]:
        """n_tokens ids that follow the prompt (the last round may find more)."""
        self.start(prompt)
        out: list[int] = []
        while len(out) < n_tokens:
            out += self.round()
        return out[:n_tokens]
