"""Beam search over a paged cache: the selection of each step, the beams' pages, and
what is kept per beam."""
from __future__ import annotations

from typing import List, Sequence

from . import DecodeProblem, PagePools, PageTable, beam_reorder, beam_select, pages_copy


class BeamSearch:
    """The beams of a batch of requests.

    ``prompts`` are sequences of ``table`` (one per request) whose keys and values
    are in the pages already, in all of ``pools``: cartridges by reference, and the
    prompt behind them. Every request has ``beams`` beams, forks of its prompt;
    what they have in common stays in pages that they share. A decoding loop:

        search = BeamSearch(table, pools, prompts, beams, end_token, max_tokens)
        tokens = search.step(logits)             # [batch, 1, vocab], of the prompts' last tokens
        while not search.done:
            problem = search.problem(num_kv_heads, group_size, head_dim, softmax_scale)
            # one row per beam: for each layer paged_append and paged_chunk_fwd (or paged_decode_fwd) with the problem
            tokens = search.step(logits)         # [batch, beams, vocab]
        histories, scores = search.results()

    A beam that has chosen ``end_token`` keeps its score; its pages are free at
    once but one, in which its row (of no consequence from then on) has its place.
    Works on the current stream, and waits for the selection once a step: the
    tables of pages are on the host."""

    def __init__(self, table: PageTable, pools: PagePools, prompts: Sequence[int], beams: int, end_token: int, max_tokens: int):
        import torch
        if beams < 1 or max_tokens < 1:
            raise ValueError("beams and max_tokens must be >= 1")
        if pools.num_pages < table.num_pages or pools.page_size != table.page_size:
            raise ValueError("the pools must have the table's pages")
        if pools.row_bytes % 16:
            raise ValueError("a token's row in the pools must be a multiple of 16 bytes (see pages_copy)")
        self.table, self.pools, self.beams, self.end_token = table, pools, int(beams), int(end_token)
        self.batch, self.steps, self._over = len(prompts), 0, False
        self.seqs: List[int] = []
        device = pools.pools[0].device
        shape = (self.batch, self.beams)
        self.scores = torch.zeros((self.batch, 1), dtype=torch.float32, device=device)
        self.finished = torch.zeros(shape, dtype=torch.bool, device=device)
        self._history = torch.full((*shape, int(max_tokens)), self.end_token, dtype=torch.int32, device=device)
        # (Last: what fails has taken no pages.)
        try:
            for p in prompts:
                self.seqs += table.fork(p, self.beams)
        except BaseException:
            table.free(self.seqs)
            raise
        self.done = self.batch == 0

    def step(self, logits):
        """Chooses each request's next beams; returns their tokens, int32 [batch,
        beams]. Where too few pages are free (a CasError), or anything else fails once
        the beams are chosen, the search ends as it is: results() and close() are left."""
        import torch
        if self._over or self.done or self.steps == self._history.shape[2]:
            raise RuntimeError("the search is over")
        first = self.steps == 0
        if logits.shape[:2] != (self.batch, 1 if first else self.beams):
            raise ValueError(f"logits must be [{self.batch}, {1 if first else self.beams}, vocab]")
        scores, parents, tokens = beam_select(logits, self.scores, self.beams, finished=None if first else self.finished,
                                              pad_token=self.end_token)
        t = self.steps
        self._over = True   # (until histories, pages and copies belong together again)
        if not first:
            states = [self._history[:, :, :t], self.finished]
            beam_reorder(states, parents, outs=states)
        self._history[:, :, t] = tokens
        self.finished |= tokens == self.end_token
        self.scores, self.steps = scores, t + 1
        # A beam at -inf (there were fewer candidates than beams) goes no further, either.
        host = torch.stack((parents, (self.finished | (scores == float("-inf"))).int())).cpu()
        if not first:
            base = torch.arange(self.batch, dtype=torch.int32)[:, None] * self.beams
            self.table.reorder(self.seqs, (host[0] + base).flatten().tolist())
        ended = host[1].flatten().tolist()
        for seq, e in zip(self.seqs, ended):
            if e:
                self.table.truncate(seq, 0)
        self.done = all(ended) or self.steps == self._history.shape[2]
        if not self.done:
            pages_copy(self.pools, self.table.extend(self.seqs, [1] * len(self.seqs)))
        self._over = False
        return tokens

    def problem(self, num_kv_heads: int, group_size: int, head_dim: int, softmax_scale: float) -> DecodeProblem:
        """The tables of the next token: one row per beam, request by request."""
        if self._over:
            raise RuntimeError("the search is over")
        # (The pools may have more pages than the table gives out; the paged calls go by the pools.)
        return DecodeProblem.from_tables([1] * len(self.seqs), *self.table.lists(self.seqs), self.pools.num_pages,
                                         self.table.page_size, num_kv_heads, group_size, head_dim, softmax_scale)

    def results(self):
        """(tokens int32 [batch, beams, steps], scores fp32 [batch, beams]), best first; behind a beam's end its end_token."""
        if self.steps == 0:
            raise RuntimeError("no step was made")
        return self._history[:, :, :self.steps].clone(), self.scores

    def close(self) -> None:
        """Frees the beams' pages (the prompts stay)."""
        seqs, self.seqs, self._over = self.seqs, [], True
        if seqs:
            self.table.free(seqs)
