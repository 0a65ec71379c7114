"""Inputs and a plain float64 evaluation (keys and values formed, one query at a time) for the tests of the batch
entry points.  Values are drawn on the CPU and rounded to the storage type, so both sides see the same bits."""
from __future__ import annotations

from dataclasses import dataclass, field
from typing import List, Optional

import torch

BLOCK = 16


@dataclass
class BatchCase:
    lens: List[int]
    counts: List[int]
    causal: bool = False
    window: int = 0
    sinks: int = 0
    heads: tuple = (4, 2, 64)      # Hq, Hkv, d
    rank: int = 8
    dtype: torch.dtype = torch.bfloat16
    paged: bool = True
    rope: float = 0.0
    key_side: bool = True
    value_side: bool = True
    own_l: bool = False
    n_adapters: int = 3
    scale: float = 0.0
    seed: int = 0
    poison: bool = True            # rows that nothing sees: NaN, their blocks' table entries out of range
    head_major: bool = False
    extra_rank_stride: int = 0

    def label(self):
        return (f"{str(self.dtype)[6:]}-{self.heads}-r{self.rank}-n{self.lens}-c{self.counts}-{'causal' if self.causal else 'last'}"
                f"-w{self.window}-s{self.sinks}-{'paged' if self.paged else 'contig'}"
                + ("-rope" if self.rope else "") + ("" if self.key_side else "-vonly") + ("-ownL" if self.own_l else ""))


@dataclass
class Inputs:
    case: BatchCase
    q: torch.Tensor
    k: torch.Tensor          # [T][n_max][Hkv][d], the rows by sequence and token
    v: torch.Tensor
    l: torch.Tensor          # [A or 1][T][n_max][r]
    b_k: Optional[torch.Tensor]
    b_v: Optional[torch.Tensor]
    start: torch.Tensor
    adapter: torch.Tensor
    seen: torch.Tensor = field(default=None)   # [T][n_max]


def positions(c: BatchCase, t: int):
    n, m = c.lens[t], c.counts[t]
    return [n - m + k if c.causal else n - 1 for k in range(m)]


def visible(c: BatchCase, pos: int, n: int):
    j = torch.arange(n)
    keep = j <= pos
    if c.window > 0:
        keep &= (j > pos - c.window) | (j < c.sinks)
    return keep


def make(c: BatchCase) -> Inputs:
    g = torch.Generator().manual_seed(1000 + c.seed)
    hq, hkv, d = c.heads
    T, n_max, total = len(c.lens), max(max(c.lens), 1), sum(c.counts)

    def randn(*shape, std=1.0):
        return (torch.randn(*shape, generator=g) * std).to(c.dtype)

    x = Inputs(c, randn(total, hq, d), randn(T, n_max, hkv, d), randn(T, n_max, hkv, d),
               randn(c.n_adapters if c.own_l else 1, T, n_max, c.rank),
               randn(c.n_adapters, c.rank, hkv * d, std=0.15) if c.key_side else None,
               randn(c.n_adapters, c.rank, hkv * d, std=0.15) if c.value_side else None,
               torch.tensor([sum(c.counts[:t]) for t in range(T + 1)], dtype=torch.int32),
               torch.randint(0, c.n_adapters, (total,), generator=g, dtype=torch.int32))
    x.seen = torch.zeros(T, n_max, dtype=torch.bool)
    for t in range(T):
        for p in positions(c, t):
            if p >= 0:
                x.seen[t, :c.lens[t]] |= visible(c, p, c.lens[t])
    return x


def probabilities(x: Inputs):
    """Yields (query, sequence, adapter, visible tokens, [Hq][tokens] softmax in float64) for every query that sees something."""
    c = x.case
    hq, hkv, d = c.heads
    scale = c.scale or d ** -0.5
    for t, n in enumerate(c.lens):
        for k, p in enumerate(positions(c, t)):
            i = int(x.start[t]) + k
            a = min(max(int(x.adapter[int(x.start[t]) if c.causal else i]), 0), c.n_adapters - 1)
            if p < 0 or n <= 0:
                continue
            j = torch.nonzero(visible(c, p, n))[:, 0]
            key = x.k[t, j].double()
            low = x.l[a if c.own_l else 0, t, j].double()
            if x.b_k is not None:
                add = (low @ x.b_k[a].double()).view(-1, hkv, d)
                if c.rope:
                    ang = j[:, None, None].double() * c.rope ** (-torch.arange(0, d, 2).double() / d)
                    lo, hi = add[..., :d // 2], add[..., d // 2:]
                    add = torch.cat((lo * ang.cos() - hi * ang.sin(), hi * ang.cos() + lo * ang.sin()), -1)
                key = key + add
            s = torch.einsum("hgd,nhd->hgn", x.q[i].double().view(hkv, hq // hkv, d), key) * scale
            yield i, t, a, j, low, torch.softmax(s, -1)


def attention(x: Inputs) -> torch.Tensor:
    c = x.case
    hq, hkv, d = c.heads
    out = torch.zeros(x.q.shape, dtype=torch.float64)
    for i, t, a, j, low, pr in probabilities(x):
        val = x.v[t, j].double()
        if x.b_v is not None:
            val = val + (low @ x.b_v[a].double()).view(-1, hkv, d)
        out[i] = torch.einsum("hgn,nhd->hgd", pr, val).reshape(hq, d)
    return out


def key_weights(x: Inputs) -> torch.Tensor:
    w = torch.zeros(len(x.case.lens), max(max(x.case.lens), 1), dtype=torch.float64)
    for _, t, _, j, _, pr in probabilities(x):
        w[t, j] += pr.sum((0, 1))
    return w


class Device:
    """The inputs on the GPU in the documented layouts, with the descriptors of the binding."""

    def __init__(self, x: Inputs, lra, max_seq_len: Optional[int] = None):
        c = x.case
        hq, hkv, d = c.heads
        dev, nan = "cuda", float("nan")
        T, n_max = x.seen.shape
        A, R = x.l.shape[0], c.rank + c.extra_rank_stride
        g = torch.Generator().manual_seed(c.seed)
        self.token_rows = {}
        k, v, l = x.k, x.v, x.l
        if c.poison:
            k, v, l = k.clone(), v.clone(), l.clone()
            k[~x.seen], v[~x.seen], l[:, ~x.seen] = nan, nan, nan
        if c.paged:
            per = [-(-n // BLOCK) for n in c.lens]
            nb = sum(per) + 2
            order = torch.randperm(nb, generator=g).tolist()
            table = torch.full((T, max(max(per), -(-(max_seq_len or n_max) // BLOCK))), 1 << 24, dtype=torch.int32)
            kp = torch.full((nb, hkv, BLOCK, d), nan, dtype=c.dtype)
            vp, lp = torch.full_like(kp, nan), torch.full((A, nb, BLOCK, R), nan, dtype=c.dtype)
            for t in range(T):
                for b in range(per[t]):
                    blk, j0 = order.pop(), b * BLOCK
                    j1 = min(j0 + BLOCK, c.lens[t])
                    if bool(x.seen[t, j0:j1].any()) or not c.poison:
                        table[t, b] = blk
                    kp[blk, :, :j1 - j0] = k[t, j0:j1].transpose(0, 1)
                    vp[blk, :, :j1 - j0] = v[t, j0:j1].transpose(0, 1)
                    lp[:, blk, :j1 - j0, :c.rank] = l[:, t, j0:j1]
            self.table = table.to(dev)
            self.k, self.v, lp = kp.to(dev), vp.to(dev), lp.to(dev)
            self.l = lp[..., :c.rank]
        else:
            assert T == 1
            self.table = None
            if c.head_major:
                self.k, self.v = (y[0].transpose(0, 1).contiguous().to(dev).transpose(0, 1) for y in (k, v))
            else:
                self.k, self.v = k[0].to(dev), v[0].to(dev)
            full = torch.full((A, n_max, R), nan, dtype=c.dtype)
            full[..., :c.rank] = l[:, 0]
            self.l = full.to(dev)[..., :c.rank]
        self.lens = torch.tensor(c.lens, dtype=torch.int32, device=dev)
        self.q, self.start, self.adapter = x.q.to(dev), x.start.to(dev), x.adapter.to(dev)
        self.b_k = None if x.b_k is None else x.b_k.to(dev)
        self.b_v = None if x.b_v is None else x.b_v.to(dev)
        self.shape = lra.make_shape(self.q, hkv, c.rank, c.scale, c.rope)
        self.cache = lra.make_cache(self.k, self.v, self.l if c.own_l else self.l[0], self.lens, max_seq_len or n_max, self.table,
                                    l_per_adapter=c.own_l)
        self.batch = lra.make_batch(self.start, self.adapter, max(max(c.counts), 1), causal=c.causal, window=c.window, sinks=c.sinks)
        self.lra, self.case = lra, c

    def attend(self, stream=None):
        lra = self.lra
        out = torch.full_like(self.q, float("nan"))
        ws = torch.full((max(lra.lra_batch_workspace_bytes(self.shape, self.cache, self.batch), 256),), 255, dtype=torch.uint8, device="cuda")
        lra.lra_attn_batch(self.shape, self.cache, self.b_k, self.b_v, self.case.n_adapters, self.batch, self.q, out, ws, stream=stream)
        torch.cuda.synchronize()
        return out
