"""One tensor-parallel rank's attention block, from the layer's input to its share of the output projection, as a
serving loop runs it: every step on the library's kernels.

    x -> projections of Q and K (with Phase A), of V      qkn_proj_partial
      -> the requests' low-rank adapters, Phase A again   qkn_adapters_add
      -> the ranks' statistics are exchanged              the caller's `exchange`
      -> norm, rotary positions, K and V into the cache   qkn_rope_cache
      -> attention over the cache                         qkn_attn
      -> this rank's term of the output projection        qkn_proj_partial

A step's tensors are allocated once and its arguments checked once; the step then runs any number of times, by itself
or captured in a HIP graph, on whatever x, positions, slots, lengths, page tables and adapter numbers hold then.

``python -m paper_2608_09160_amd.block`` serves a few sequences: prompts first, then single tokens from a replayed
graph, and prints the time of a step.
"""
from __future__ import annotations

from dataclasses import dataclass
from typing import Callable, Optional

import torch

from ._lib import PreparedProj, ProjSeg
from ._serve import (AdapterSeg, KVCache, PreparedAdapters, PreparedAttn, PreparedRopeCache, RopeSeg, _on, qkn_rope_table)


@dataclass
class Weights:
    """One rank's slices (bf16; gammas fp32). Adapters: a [adapters, rank, hidden] and b [adapters, width, rank] for each
    of Q, K and V, or None."""

    wq: torch.Tensor                 # [heads * head_dim, hidden]
    wk: torch.Tensor                 # [kv heads * head_dim, hidden]
    wv: torch.Tensor
    wo: torch.Tensor                 # [hidden, heads * head_dim]
    gq: torch.Tensor                 # [heads * head_dim]
    gk: torch.Tensor
    adapters: Optional[tuple] = None  # ((aq, bq), (ak, bk), (av, bv))
    adapter_scale: Optional[torch.Tensor] = None  # fp32 [adapters]


@dataclass
class Batch:
    """What a step runs on, all of it read on the device when the step runs: int32, slots int64. max_q and max_kv bound
    the new and the cached tokens of a sequence for as long as the step is used. Tokens behind the last sequence's (a
    batch that has lost some: q_start 0, .., k, k, k, slots and ids -1) are padding, and zeros in the attention."""

    x: torch.Tensor            # bf16 [T, hidden]
    pos: torch.Tensor          # [T]
    slots: torch.Tensor        # [T], page * page size + row
    q_start: torch.Tensor      # [sequences + 1]
    kv_len: torch.Tensor       # [sequences], the new tokens included
    block_table: torch.Tensor  # [sequences, pages]
    max_q: int
    max_kv: int
    ids: Optional[torch.Tensor] = None  # [T], the token's adapter


class Step:
    """The block for batches of a given shape. exchange(stat_q, stat_k, rank): makes the other ranks' rows of the fp32
    [tp, T] statistics valid, this rank's row being so already (an all-gather in place); called between the kernels, on
    the same stream. Not needed at tp = 1. `out` is this rank's term of the block's output, to be added over the ranks."""

    def __init__(self, w: Weights, cache: KVCache, table: torch.Tensor, batch: Batch, tp: int = 1, rank: int = 0,
                 eps: float = 1e-6, window: int = 0, exchange: Optional[Callable] = None):
        if not 0 <= rank < tp:
            raise ValueError("rank must be one of tp")
        if tp > 1 and exchange is None:
            raise ValueError("exchange: needed with several ranks")
        if w.adapters is not None and batch.ids is None:
            raise ValueError("batch.ids: needed with adapters")
        x, T, D = batch.x, batch.x.shape[0], cache.k.shape[3]
        self.batch, self.tp, self.rank, self.exchange = batch, tp, rank, exchange
        # nothing is written here: the step may run on another stream than the current one
        self.stat_q, self.stat_k = (torch.empty(tp, T, dtype=torch.float32, device=x.device) for _ in range(2))
        qk = [ProjSeg(w.wq, partials=self.stat_q[rank]), ProjSeg(w.wk, partials=self.stat_k[rank])]
        v = [ProjSeg(w.wv)]
        self.projections = [PreparedProj(x, qk), PreparedProj(x, v)]
        self.q, self.k, self.v = qk[0].y, qk[1].y, v[0].y
        self.adapters = None
        if w.adapters is not None:
            self.adapters = PreparedAdapters(
                x, [AdapterSeg(a, b, y=y, partials=p) for (a, b), y, p in
                    zip(w.adapters, (self.q, self.k, self.v), (self.stat_q[rank], self.stat_k[rank], None))],
                batch.ids, w.adapter_scale)
        # in place: Q's rows are not needed unrotated, K's only in the cache
        self.rope = PreparedRopeCache(
            table, batch.pos, D, RopeSeg(self.q, w.gq, self.stat_q, tp * self.q.shape[1], self.q),
            RopeSeg(self.k, w.gk, self.stat_k, tp * self.k.shape[1]), self.v, cache, batch.slots, eps=eps)
        self.attn = PreparedAttn(self.q, cache, batch.block_table, batch.q_start, batch.kv_len, batch.max_q,
                                 batch.max_kv, window=window)
        o = ProjSeg(w.wo)
        self.output = PreparedProj(self.attn.out, [o])
        self.out = o.y

    def __call__(self, stream=None) -> torch.Tensor:
        for projection in self.projections:
            projection(stream)
        if self.adapters is not None:
            self.adapters(stream)
        if self.tp > 1:
            with _on(stream):
                self.exchange(self.stat_q, self.stat_k, self.rank)
        self.rope(stream)
        self.attn(stream)
        self.output(stream)
        return self.out


class Pages:
    """Sequences' pages, handed out in order: the host side of the cache, as small as it can be."""

    def __init__(self, sequences: int, max_tokens: int, page_size: int, device):
        self.page_size = page_size
        per = (max_tokens + page_size - 1) // page_size
        self.count = sequences * per
        # neighbouring pages of a sequence are far apart in the pool
        self.table = torch.arange(self.count, dtype=torch.int32).view(per, sequences).t().contiguous().to(device)

    def slots(self, sequence: torch.Tensor, pos: torch.Tensor) -> torch.Tensor:
        page = self.table[sequence.long(), (pos // self.page_size).long()].long()
        return page * self.page_size + pos % self.page_size


def main(prompts=(700, 64, 2048, 1), tokens: int = 16, hidden: int = 4096, heads: int = 16, kv_heads: int = 4,
         head_dim: int = 128, page_size: int = 16, adapters: int = 4, adapter_rank: int = 16) -> torch.Tensor:
    """Serves the prompts, then `tokens` tokens of each; returns the last step's output."""
    dev = torch.device("cuda")
    g = torch.Generator().manual_seed(0)

    def mat(*shape):
        return (torch.randn(*shape, generator=g) * shape[-1] ** -0.5).to(torch.bfloat16).to(dev)

    n_q, n_kv, B = heads * head_dim, kv_heads * head_dim, len(prompts)
    w = Weights(mat(n_q, hidden), mat(n_kv, hidden), mat(n_kv, hidden), mat(hidden, n_q), torch.ones(n_q, device=dev),
                torch.ones(n_kv, device=dev),
                tuple((mat(adapters, adapter_rank, hidden), mat(adapters, d, adapter_rank)) for d in (n_q, n_kv, n_kv)),
                torch.ones(adapters, device=dev))
    longest = max(prompts) + tokens
    pages = Pages(B, longest, page_size, dev)
    cache = KVCache(*(torch.empty(pages.count, kv_heads, page_size, head_dim, dtype=torch.bfloat16, device=dev)
                      for _ in range(2)))
    table = qkn_rope_table(longest, head_dim, device=dev)

    # the prompts, all in one call
    n = torch.tensor(prompts, dtype=torch.int32)
    T = int(n.sum())
    seq = torch.repeat_interleave(torch.arange(B), n.long()).to(dev)
    pos = torch.cat([torch.arange(m, dtype=torch.int32) for m in prompts]).to(dev)
    q_start = torch.cat([torch.zeros(1, dtype=torch.int32), n.cumsum(0).int()]).to(dev)
    x = torch.randn(T, hidden, generator=g).to(torch.bfloat16).to(dev)
    out = Step(w, cache, table, Batch(x, pos, pages.slots(seq, pos), q_start, n.to(dev), pages.table, max(prompts),
                                      max(prompts), (seq % adapters).int()))()
    last = out[q_start[1:].long() - 1]

    # then a token of each sequence at a time: one graph, replayed
    seq = torch.arange(B, device=dev)
    b = Batch(last.clone(), n.to(dev), pages.slots(seq, n.to(dev)), torch.arange(B + 1, dtype=torch.int32, device=dev),
              (n + 1).to(dev), pages.table, 1, longest, (seq % adapters).int())
    step = Step(w, cache, table, b)
    step()  # the first call outside the capture
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    spent = 0.0
    for _ in range(tokens):
        start.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        spent += start.elapsed_time(end)
        # the model's other layers would stand here; the next position of every sequence
        b.x.copy_(step.out)
        b.pos += 1
        b.kv_len += 1
        b.slots.copy_(pages.slots(seq, torch.clamp(b.pos, max=longest - 1)))
    print(f"{B} sequences, prompts {list(prompts)}: {1e3 * spent / tokens:.1f} us a step of {B} tokens")
    return step.out


if __name__ == "__main__":
    main()
