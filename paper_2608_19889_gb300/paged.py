"""Sequences of a paged model whose cache blocks are managed on the device.

`PagedSeqs` keeps what the block operators work on (block table, lengths, counts, workspace, error word) for the cache of
a model created with AXON_KV_PAGED, and steps the model with it: blocks are taken before tokens are appended, shared by
forks, and given back when a sequence ends or, under a sliding window, when they have slid out of it. `check`, `lengths`
and `blocks_in_use` wait for the GPU, `extend` for the copy of its lengths; nothing else does.
"""
from __future__ import annotations

import torch

import paper_2608_19889_gb300 as ax


class PagedSeqs:
    """`rows` sequences of a model created with `cfg` (AXON_KV_PAGED); row b is sequence b of the model's calls."""

    def __init__(self, model, cfg, rows: int):
        if cfg.kv_layout != ax.AXON_KV_PAGED:
            raise ValueError("a model with a paged cache is wanted")
        if not 1 <= rows <= cfg.max_batch:
            raise ValueError(f"1 .. {cfg.max_batch} rows are wanted, got {rows}")
        self.model, self.rows = model, rows
        self.window, self.sinks = cfg.sliding_window, cfg.sink_tokens
        dev = dict(dtype=torch.int32, device="cuda")
        self.table = torch.full((rows, cfg.max_context // 16), -1, **dev)
        self.lens = torch.zeros(rows, **dev)
        self.cache = ax.axon_kv_cache_get(model)
        self.refs = torch.zeros(self.cache.num_blocks, **dev)
        self.err = torch.zeros(1, **dev)
        self.live = torch.zeros(1, **dev)
        self.seqs = ax.make_kv_seqs(self.table, self.lens, self.refs)
        self.work = ax.make_kv_workspace(self.cache, self.seqs)
        self.all = torch.arange(rows, **dev)
        self.one = torch.ones(rows, **dev)
        self.unused = torch.empty(rows, **dev)  # greedy tokens that nobody asked for

    def _first(self, n):
        if not 1 <= n <= self.rows:
            raise ValueError(f"1 .. {self.rows} rows are wanted, got {n}")
        if self.window:
            ax.axon_kv_release(self.cache, self.seqs, self.all[:n], window=self.window, sinks=self.sinks, err=self.err)

    def extend(self, ids, lengths, logits=None, next_tokens=None):
        """Append chunk b of `ids` (int32 [sum(lengths)], packed) to sequence b: axon_prefill_varlen after blocks that slid
        out of the window are given back and the chunk's taken. lengths: one positive host integer for each of the first
        rows; the others stay as they are. Under a window a long prompt that is fed in pieces holds no more than a piece, the
        window and the sinks reach."""
        n = len(lengths)
        if n and (min(lengths) < 1 or ids.numel() != sum(lengths)):
            raise ValueError(f"positive lengths that sum to the {ids.numel()} ids are wanted, got {lengths}")
        self._first(n)
        new = torch.tensor(lengths, dtype=torch.int32, device="cuda")
        cu = torch.nn.functional.pad(new.cumsum(0, dtype=torch.int32), (1, 0))
        ax.axon_kv_reserve(self.cache, self.seqs, self.all[:n], new, self.work, err=self.err)
        ax.axon_prefill_varlen(self.model, ids, cu, self.lens, max(lengths), block_table=self.table, logits=logits,
                               next_tokens=next_tokens)

    def step(self, tokens, logits=None, next_tokens=None):
        """One decode step of the first rows, one for each token; the others stay as they are (a row that ended takes no
        blocks if the live ones are kept in front: fork the last of them over it). Blocks that slid out of the window are
        given back, one is taken where the token begins it."""
        n = tokens.numel()
        self._first(n)
        ax.axon_kv_reserve(self.cache, self.seqs, self.all[:n], self.one[:n], self.work, err=self.err)
        ax.axon_decode_step(self.model, tokens, self.lens, block_table=self.table, logits=logits,
                            next_tokens=self.unused if next_tokens is None else next_tokens)

    def fork(self, src, dst):
        """Rows dst take over what rows src hold (int32 device tensors)."""
        ax.axon_kv_fork(self.cache, self.seqs, src, dst, self.work, err=self.err)

    def release(self, rows):
        """Rows (int32 device tensor) end: everything they hold is given back, their length is 0."""
        ax.axon_kv_release(self.cache, self.seqs, rows, err=self.err)

    def compact(self):
        """Move the blocks in use to the front of the pool."""
        ax.axon_kv_compact(self.cache, self.seqs, self.work, live=self.live, err=self.err)

    def blocks_in_use(self) -> int:
        return int((self.refs != 0).sum())

    def lengths(self) -> list:
        return self.lens.tolist()

    def check(self):
        """Wait, and raise what the device reported since the last check."""
        for rc, bits in (ax.axon_check_error(self.err), ax.axon_check_device(self.model)):
            if rc:
                raise ax.AxonError(f"paged sequences (error bits {bits})", rc)
