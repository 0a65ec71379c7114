"""Seeded random calls of the 8-bit entry points against the plain evaluations in 64 bits: shapes, ranks, lengths, windows, layouts and bounds
that no other test names."""
import random

import pytest
import torch

import paper_2602_01053_amd as lra
from tests.attn8_reference import Case8, Device8, attention_with_bound, close_enough, make8

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def random_case(seed):
    """A batch whose evaluation in 64 bits takes a second at most: queries times keys times heads are bounded."""
    rng = random.Random(seed)
    while True:
        hkv = rng.choice([1, 2, 3, 4, 5, 8])
        hq = hkv * rng.choice([1, 2, 3, 4, 7, 8, 16])
        d = rng.choice([64, 128])
        dtype = rng.choice([BF16, BF16, BF16, F32])
        rank = rng.choice([8, 16, 24, 32, 40, 48, 56, 64, 1, 5, 33] if dtype == BF16 else [1, 4, 8, 13, 16, 64])
        seqs = rng.choice([1, 1, 2, 3, 5, 9, 20])
        longest = int(2 ** rng.uniform(0, 12.5))
        lens = [rng.choice([0, 1, longest, rng.randint(0, longest), rng.randint(0, longest)]) for _ in range(seqs)]
        most = int(2 ** rng.uniform(0, rng.choice([2, 4, 7])))
        counts = [rng.choice([0, 1, most, rng.randint(0, most)]) for _ in range(seqs)]
        if sum(counts) == 0:
            counts[0] = most
        window = rng.choice([0, 0, rng.randint(1, longest + 1)])
        c = Case8(lens, counts, causal=rng.random() < 0.5, window=window, sinks=rng.choice([0, 1, 4, 70]), heads=(hq, hkv, d), rank=rank, dtype=dtype,
                  key_side=rng.random() < 0.7, value_side=rng.random() < 0.8, n_adapters=rng.randint(1, 4), scale=rng.choice([0.0, 0.0, 0.05]),
                  code=rng.choice(["e4m3", "int8"]), table=seqs > 1 or rng.random() < 0.5, layout=rng.choice(["dense", "pool"]), seed=seed)
        if hq * d * sum(n * k for n, k in zip(lens, counts)) < 3e7 and sum(lens) * hkv * d < 4e6:
            return c, rng


@pytest.mark.parametrize("seed", range(70))
def test_attention(seed):
    c, rng = random_case(seed)
    x = make8(c)
    want, bound = attention_with_bound(x)
    room = rng.choice([None, None, max(c.lens) + rng.randint(1, 500), 20000])
    dev = Device8(x, lra, max_seq_len=room)
    got = dev.attend()
    close_enough(got, want, bound, f"seed {seed} room {room} {c.label()}")
    assert torch.equal(got, dev.attend())


@pytest.mark.parametrize("seed", range(50))
def test_products(seed):
    rng = random.Random(1000 + seed)
    m, n, k = int(2 ** rng.uniform(0, 11)), int(2 ** rng.uniform(0, 12.5)), 16 * int(2 ** rng.uniform(0, 8))
    while m * n * k > 1 << 33:
        m = max(1, m // 2)
    dtype = rng.choice([BF16, F32])
    g = torch.Generator().manual_seed(seed)
    x, w = (torch.randint(-128, 128, (r, k), generator=g, dtype=torch.int8) for r in (m, n))
    sx, sw = torch.rand(m, generator=g) + 0.01, torch.rand(n, generator=g) * 0.01 + 1e-4
    pad = [16 * rng.randint(0, 3) for _ in range(2)]
    dx, dw = (torch.full((z.size(0), k + p), 77, dtype=torch.int8, device="cuda")[:, :k] for z, p in ((x, pad[0]), (w, pad[1])))
    dx.copy_(x), dw.copy_(w)
    buf = torch.full((m + 1, n + rng.choice([0, 1, 2, 4, 8])), -3.0, dtype=dtype, device="cuda")
    y = buf[:m, :n]
    lra.lra_matmul_i8(dx, sx.cuda(), dw, sw.cuda(), y)
    torch.cuda.synchronize()
    want = (x.double() @ w.double().t()) * sx.double()[:, None] * sw.double()
    # the sum's rounding to fp32, two products, and the output's own
    steps = 3 * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0)
    assert bool(((y.cpu().double() - want).abs() <= want.abs() * steps * (1 + 2.0 ** -8)).all()), (m, n, k)
    assert bool((buf[m:] == -3).all()) and bool((buf[:m, n:] == -3).all()), (m, n, k)
