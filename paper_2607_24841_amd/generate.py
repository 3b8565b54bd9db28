"""Block-diffusion generation driver (Eq. (2)): prompt prefill, then per block
``steps`` calls of nmdlm_block_step that reveal ``k_unmask`` tokens each; a
finished block's keys/values stay in the caches as context.  The host only
loops and marshals; every step runs in libnmdlm's kernels and the token
state stays on the device until the end.  Several sequences (prompts of
one length) advance together, one batched step per denoising step; requests
of different lengths share pools of pages (PagedGenerator)."""
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
