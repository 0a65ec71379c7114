"""Inputs and plain float64 evaluations for the tests of the 8-bit calls.  Values are drawn on the CPU; the attention of a batch is
that of batch_reference on the values that the codes stand for, with a bound for every output beside it."""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from tests import batch_reference as ref

BLOCK = 16
TOP = {"e4m3": 448.0, "int8": 127.0}
TORCH = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


def power(e: torch.Tensor) -> torch.Tensor:
    """2^e in float64, by its bits."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def values_of(codes: torch.Tensor, scale: torch.Tensor) -> torch.Tensor:
    """codes in float8 or int8, scale bytes that broadcast against them: float64."""
    return codes.float().double() * power(scale.long() - 127)


def least_exponent(top: torch.Tensor, code: str) -> torch.Tensor:
    """The least e >= -126 with top <= TOP 2^e (float64 in, exact)."""
    m, e = torch.frexp(top / TOP[code])          # top / TOP = m 2^e, 1/2 <= m < 1
    e = torch.where(m == 0.5, e - 1, e).long()
    e = torch.where(top > TOP[code] * power(e), e + 1, e)
    return torch.where(top == 0, -126, e).clamp(min=-126)


def half_step(x: torch.Tensor, code: str) -> torch.Tensor:
    """Half the distance of neighbouring codes at the scaled value x (to the larger side, at a power of two)."""
    if code == "int8":
        return torch.full_like(x, 0.5)
    return power(torch.frexp(x.abs().clamp(min=2.0 ** -6)).exponent.long() - 4) / 2


@dataclass
class Case8(ref.BatchCase):
    code: str = "e4m3"
    table: bool = True           # a block table (without one: one sequence, its blocks in order)
    layout: str = "dense"        # "dense", or "pool": K and V interleaved in one allocation, wider strides for scales and L

    def label(self):
        return (super().label() + f"-{self.code}" + ("" if self.table else "-inorder") + ("" if self.layout == "dense" else f"-{self.layout}"))


def quantized(x: torch.Tensor, code: str, g: torch.Generator):
    """Codes and scale bytes of x [T][n][Hkv][d] in blocks of 16 tokens: nearest codes, scales sometimes larger than needed."""
    T, n, hkv, d = x.shape
    nb = -(-n // BLOCK)
    pad = torch.zeros(T, nb * BLOCK, hkv, d, dtype=torch.float64)
    pad[:, :n] = x.double()
    z = pad.view(T, nb, BLOCK, hkv, d).transpose(2, 3)                       # [T][nb][Hkv][16][d]
    e = least_exponent(z.abs().amax((3, 4)), code) + torch.randint(0, 2, (T, nb, hkv), generator=g)
    y = z / power(e)[..., None, None]
    c = torch.round(y).to(torch.int8) if code == "int8" else y.float().to(torch.float8_e4m3fn)
    return c, (e + 127).to(torch.uint8)


def make8(c: Case8) -> ref.Inputs:
    """Inputs whose k and v are the values of codes; those in x.codes = (k codes, k scales, v codes, v scales)."""
    x = ref.make(c)
    g = torch.Generator().manual_seed(77 + c.seed)
    n = x.k.shape[1]
    # (a few wide channels among the keys, and blocks of different size)
    k = x.k.double() * (1 + 3 * (torch.rand(x.k.shape[-1], generator=g) < 0.05))
    v = x.v.double() * 2.0 ** torch.randint(-3, 3, (x.v.shape[0], n, 1, 1), generator=g)
    (kc, ks), (vc, vs) = quantized(k, c.code, g), quantized(v, c.code, g)
    x.codes = (kc, ks, vc, vs)
    flat = lambda cc, ss: values_of(cc, ss[..., None, None]).transpose(2, 3).reshape(x.k.shape[0], -1, *x.k.shape[2:])[:, :n]  # noqa: E731
    x.k, x.v = flat(kc, ks), flat(vc, vs)
    return x


def attention_with_bound(x: ref.Inputs):
    """The outputs in float64, and for each how far a kernel may be off that keeps sums in fp32 and, for bf16, rounds the
    probabilities, Qt = Q B_K^T and the output to bf16 (half a step: 2^-8 of the value)."""
    c = x.case
    hq, hkv, d = c.heads
    g = hq // hkv
    scale = c.scale or d ** -0.5
    half, u = (2.0 ** -8 if c.dtype == torch.bfloat16 else 2.0 ** -24), 2.0 ** -24
    out = torch.zeros(x.q.shape, dtype=torch.float64)
    bound = torch.zeros_like(out)
    for i, t, a, j, low, pr in ref.probabilities(x):
        v, big_v = x.v[t, j].double(), x.v[t, j].double().abs()
        if x.b_v is not None:
            v = v + (low @ x.b_v[a].double()).view(-1, hkv, d)
            big_v = big_v + (low.abs() @ x.b_v[a].double().abs()).view(-1, hkv, d)
        o = torch.einsum("hgn,nhd->hgd", pr, v)
        mass = torch.einsum("hgn,nhd->hgd", pr, big_v)
        q = x.q[i].double().view(hkv, g, d)
        # scores: sums of d + r products in fp32, and with a key side Qt rounded to bf16
        size = torch.einsum("hgd,nhd->hgn", q.abs(), x.k[t, j].double().abs())
        slip = size * (d + 8) * u
        if x.b_k is not None:
            qt = torch.einsum("hgd,rhd->hgr", q.abs(), x.b_k[a].double().abs().view(-1, hkv, d))
            slip = slip + torch.einsum("hgr,nr->hgn", qt, low.abs()) * ((d + c.rank) * u)
            if c.dtype == torch.bfloat16:
                real = torch.einsum("hgd,rhd->hgr", q, x.b_k[a].double().view(-1, hkv, d)).abs()
                slip = slip + torch.einsum("hgr,nr->hgn", real, low.abs()) * half
        move = scale * slip.amax(-1, keepdim=True)                # of a score; weights move by twice that at most, relatively
        rel = 2 * move + 4 * move * move + len(j) * u + 2.0 ** -20  # (sums of n weights, exp to some steps, products with B_V)
        if c.dtype == torch.bfloat16:
            rel = rel + half                                        # the probabilities' rounding (the row sum takes them unrounded or alike)
            rel = rel + 2.0 ** -16                                  # O_lr in two bf16 terms
        out[i] = o.reshape(hq, d)
        bound[i] = (mass * rel + half * o.abs() * (1 + rel) + 1e-30).reshape(hq, d)
    return out, bound


class Device8:
    """The inputs on the GPU in the documented layout: random blocks, slots past the end and blocks that nothing sees holding
    anything (codes that are no number, table entries out of range)."""

    def __init__(self, x: ref.Inputs, lra, max_seq_len=None, spare=2):
        c = x.case
        hq, hkv, d = c.heads
        dev = "cuda"
        T, n_max = x.seen.shape
        g = torch.Generator().manual_seed(c.seed)
        kc, ks, vc, vs = x.codes
        per = [-(-n // BLOCK) for n in c.lens]
        cap = -(-(max_seq_len or n_max) // BLOCK)
        nb = (sum(per) if c.table else cap) + spare
        bad = 0x7f if c.code == "e4m3" else 0x81
        kp = torch.full((nb, hkv, BLOCK, d), bad, dtype=torch.uint8)
        vp = torch.full((nb, hkv, d, BLOCK), bad, dtype=torch.uint8)
        sk, sv = (torch.full((nb, hkv), 255, dtype=torch.uint8) for _ in range(2))
        lp = torch.full((nb, BLOCK, c.rank), float("nan"), dtype=c.dtype)
        order = torch.randperm(nb, generator=g).tolist() if c.table else list(range(nb))[::-1]
        table = torch.full((T, max(cap, 1)), 1 << 24, dtype=torch.int32)
        bytes_of = lambda z: z.contiguous().view(torch.uint8)  # noqa: E731
        for t in range(T):
            for b in range(per[t]):
                j0, j1 = b * BLOCK, min((b + 1) * BLOCK, c.lens[t])
                blk = order.pop()
                if not (bool(x.seen[t, j0:j1].any()) or not c.poison):
                    continue
                table[t, b] = blk
                m = j1 - j0
                kp[blk, :, :m] = bytes_of(kc[t, b][:, :m])
                vp[blk, :, :, :m] = bytes_of(vc[t, b][:, :m].transpose(1, 2))
                sk[blk], sv[blk] = ks[t, b], vs[t, b]
                lp[blk, :m] = x.l[0, t, j0:j1]
        if c.layout == "pool":
            both = torch.full((nb, 2, hkv, BLOCK * d + 32), 0x55, dtype=torch.uint8)
            both[:, 0, :, :BLOCK * d], both[:, 1, :, :BLOCK * d] = kp.view(nb, hkv, -1), vp.view(nb, hkv, -1)
            both = both.to(dev)
            self.k = both[:, 0, :, :BLOCK * d].unflatten(2, (BLOCK, d)).view(TORCH[c.code])
            self.v = both[:, 1, :, :BLOCK * d].unflatten(2, (d, BLOCK)).view(TORCH[c.code])
            scales = torch.cat((sk, sv), 1).to(dev)
            self.k_scale, self.v_scale = scales[:, :hkv], scales[:, hkv:]
            wide = torch.full((nb, BLOCK, -(-c.rank // 8) * 8 + 8), float("nan"), dtype=c.dtype)
            wide[..., :c.rank] = lp
            self.l = wide.to(dev)[..., :c.rank]
        else:
            self.k, self.v = kp.to(dev).view(TORCH[c.code]), vp.to(dev).view(TORCH[c.code])
            self.k_scale, self.v_scale, self.l = sk.to(dev), sv.to(dev), lp.to(dev)
        self.table = table.to(dev) if c.table else None
        self.lens = torch.tensor(c.lens, dtype=torch.int32, device=dev)
        self.q, self.start, self.adapter = x.q.to(dev), x.start.to(dev), x.adapter.to(dev)
        self.b_k = None if x.b_k is None else x.b_k.to(dev)
        self.b_v = None if x.b_v is None else x.b_v.to(dev)
        self.shape = lra.make_shape(self.q, hkv, c.rank, c.scale)
        self.cache = lra.make_cache8(self.k, self.v, self.k_scale, self.v_scale, self.l, self.lens, max_seq_len or max(n_max, 1), self.table)
        self.batch = lra.make_batch(self.start, self.adapter, max(max(c.counts), 1), causal=c.causal, window=c.window, sinks=c.sinks)
        self.lra, self.case = lra, c

    def workspace(self):
        n = self.lra.lra_batch8_workspace_bytes(self.shape, self.cache, self.batch)
        return torch.full((max(n, 256),), 255, dtype=torch.uint8, device="cuda")

    def call(self, out, workspace, stream=None):
        self.lra.lra_attn_batch8(self.shape, self.cache, self.b_k, self.b_v, self.case.n_adapters, self.batch, self.q, out, workspace,
                                 stream=stream)

    def attend(self):
        out = torch.full_like(self.q, float("nan"))
        self.call(out, self.workspace())
        torch.cuda.synchronize()
        return out


def rotated(x: torch.Tensor, positions: torch.Tensor, theta: float) -> torch.Tensor:
    """x [n][Hkv][d] in float64, turned by its positions."""
    if theta <= 0:
        return x
    d = x.shape[-1]
    angle = positions.double()[:, None, None] * theta ** (-torch.arange(0, d, 2).double() / d)
    a, b = x[..., :d // 2], x[..., d // 2:]
    return torch.cat((a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()), -1)


def close_enough(got: torch.Tensor, want: torch.Tensor, bound: torch.Tensor, what: str = "") -> None:
    off = (got.double().cpu() - want).abs()
    worst = (off / bound.clamp(min=1e-300)).max().item() if off.numel() else 0.0  # (a bound of zero: exactly)
    assert math.isfinite(worst) and worst <= 1.0, f"{what}: {worst:.3f} times the bound"
