"""The cache of 8-bit codes: rows appended (lra_cache8_append) and read back (lra_cache8_gather) against float64."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.attn8_reference import BLOCK, TOP, TORCH, half_step, least_exponent, power, rotated, values_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
THETA = 500000.0


class Pool:
    """A cache of codes on the GPU, its sequences' blocks in random order, every byte of it 0x55 to begin with."""

    def __init__(self, tokens, heads, d, rank, code, dtype, table=True, seed=0, spare=3):
        g = torch.Generator().manual_seed(seed)
        per = [-(-n // BLOCK) for n in tokens]
        nb = sum(per) + spare
        order = torch.randperm(nb, generator=g).tolist() if table else list(range(nb))
        self.blocks = [[order.pop(0) for _ in range(m)] for m in per]
        self.table = None
        if table:
            rows = torch.full((len(tokens), max(max(per), 1)), -1, dtype=torch.int32)
            for t, ids in enumerate(self.blocks):
                rows[t, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
            self.table = rows.cuda()
        byte = lambda *s: torch.full(s, 0x55, dtype=torch.uint8, device="cuda")  # noqa: E731
        self.k, self.v = byte(nb, heads, BLOCK, d).view(TORCH[code]), byte(nb, heads, d, BLOCK).view(TORCH[code])
        self.k_scale, self.v_scale = byte(nb, heads), byte(nb, heads)
        self.l = torch.full((nb, BLOCK, rank), 3.0, dtype=dtype, device="cuda")
        self.lens = torch.zeros(len(tokens), dtype=torch.int32, device="cuda")
        self.max_seq_len = max(max(tokens), 1)
        self.heads, self.d, self.rank, self.code, self.dtype = heads, d, rank, code, dtype
        self.shape = lra.make_shape(torch.empty(1, heads, d, dtype=dtype), heads, rank)

    @property
    def cache(self):
        return lra.make_cache8(self.k, self.v, self.k_scale, self.v_scale, self.l, self.lens, self.max_seq_len, self.table)

    def append(self, lens, counts, k, v, l, theta=THETA, positions=None, most=None):
        self.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        start = torch.tensor([sum(counts[:t]) for t in range(len(counts) + 1)], dtype=torch.int32, device="cuda")
        lra.lra_cache8_append(self.shape, self.cache, start, most or max(max(counts), 1), k, v, l, theta, positions)
        torch.cuda.synchronize()

    def bytes(self):
        return [z.cpu().clone() for z in (self.k.view(torch.uint8), self.v.view(torch.uint8), self.k_scale, self.v_scale, self.l)]


def rows_of(seed, n, heads, d, rank, dtype, wide=True):
    """Keys, values and low-rank rows as the columns of one product's output."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, 2 * heads * d + rank + (-rank) % 8, generator=g) * 2.0 ** torch.randint(-4, 4, (n, 1), generator=g)
    if wide:
        x[:, :d:7] *= 5
    x = x.to(dtype)
    y = x.cuda()
    cut = lambda z: (z[:, :heads * d].view(n, heads, d), z[:, heads * d:2 * heads * d].view(n, heads, d), z[:, 2 * heads * d:2 * heads * d + rank])  # noqa: E731
    return cut(x), cut(y)


def check_block(code, codes, scale, values, fresh, held, had, what):
    """One block and head: codes [16][d] and the scale byte against the new values (float64) of the slots `fresh`; `held` = the
    codes' values that slots [0, fresh.start) had before, at scale byte `had`."""
    lo, hi = fresh
    top = values.abs().max()
    want = int(least_exponent(top, code))
    e = int(scale) - 127
    lower = max(want, had - 127) if lo > 0 else want
    # fp32: a largest value within 2^-20 of the border may come out on either side
    near = abs(float(top) / (TOP[code] * 2.0 ** want) - 1) < 2.0 ** -20 or abs(float(top) / (TOP[code] * 2.0 ** (want - 1)) - 1) < 2.0 ** -20
    assert e == lower or (near and abs(e - lower) <= 1), (what, e, lower)
    unit = float(power(torch.tensor(e)))
    got = codes.float().double()
    y = values / unit
    off = (got[lo:hi] - y).abs()
    # rotated in fp32: two products and a sum of values up to 448 (or 127) scaled, three roundings, the angle's as well
    slack = 4 * 2.0 ** -24 * 2 * TOP[code]
    assert bool((off <= half_step(torch.maximum(y.abs(), got[lo:hi].abs()), code) + slack).all()), what
    if lo > 0:
        old = held / unit
        if e == had - 127:
            assert torch.equal(got[:lo], old), what
        else:
            assert bool(((got[:lo] - old).abs() <= half_step(torch.maximum(old.abs(), got[:lo].abs()), code)).all()), what


def check_append(pool, before, lens, counts, k, v, l, theta=THETA, positions=None):
    """Every byte of the pool after an append of rows k, v, l (CPU) against what it held before."""
    after = pool.bytes()
    touched = [torch.zeros(z.shape, dtype=torch.bool) for z in after]
    at = 0
    for t, (n, c) in enumerate(zip(lens, counts)):
        first = n - c
        if n <= pool.max_seq_len:
            pos = torch.arange(first, n) if positions is None else positions[at:at + c]
            kk = rotated(k[at:at + c].double(), pos, theta)
            for b in range(max(first, 0) // BLOCK, -(-n // BLOCK) if c > 0 else 0):
                blk, j0 = pool.blocks[t][b], b * BLOCK
                lo, hi = max(first - j0, 0), min(BLOCK, n - j0)
                rows = slice(j0 + lo - first, j0 + hi - first)
                touched[0][blk, :, :hi] = touched[1][blk, :, :, :hi] = True
                touched[2][blk] = touched[3][blk] = True
                for h in range(pool.heads):
                    for side, new in ((0, kk), (1, v[at:at + c].double())):
                        codes, was = (z[side][blk, h].view(TORCH[pool.code]) for z in (after, before))
                        if side == 1:
                            codes, was = codes.t(), was.t()
                        had = int(before[2 + side][blk, h])
                        held = values_of(was[:lo].contiguous(), torch.tensor(had)) if lo > 0 else None
                        check_block(pool.code, codes, after[2 + side][blk, h], new[rows, h], (lo, hi), held, had, (t, b, h, side))
                if l is not None:
                    touched[4][blk, lo:hi] = True
                    assert torch.equal(after[4][blk, lo:hi], l[at:at + c][rows])
        at += c
    for new, old, mask in zip(after, before, touched):
        assert torch.equal(new[~mask], old[~mask])      # nothing else was written


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,heads,d,rank", [(BF16, 2, 128, 16), (BF16, 3, 64, 8), (F32, 1, 128, 12), (F32, 4, 64, 5)])
def test_append_step_by_step(code, dtype, heads, d, rank):
    """Prompts, single tokens and chunks that end inside blocks, some sequences without new tokens; then the same call again."""
    room = [150, 40, 17, 90]
    pool = Pool(room, heads, d, rank, code, dtype, seed=1)
    lens = [0, 0, 0, 0]
    for step, counts in enumerate(([100, 16, 1, 0], [1, 1, 1, 0], [17, 0, 15, 33], [1, 5, 0, 1], [31, 18, 0, 47])):
        lens = [n + c for n, c in zip(lens, counts)]
        cpu, gpu = rows_of(10 * step, sum(counts), heads, d, rank, dtype)
        before = pool.bytes()
        pool.append(lens, counts, *gpu)
        check_append(pool, before, lens, counts, *cpu)
        again = pool.bytes()
        pool.append(lens, counts, *gpu)
        assert all(torch.equal(a, b) for a, b in zip(again, pool.bytes()))


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_append_options(code):
    """No rotation, positions of their own, no L rows, no block table, dense inputs, one kv head beside a pair."""
    heads, d, rank = 3, 128, 16
    for seed, (theta, positions, with_l, table) in enumerate(((0.0, None, True, True), (THETA, True, False, True), (10000.0, None, True, False))):
        pool = Pool([70], heads, d, rank, code, BF16, table=table, seed=seed)
        cpu, gpu = rows_of(seed, 61, heads, d, rank, BF16)
        pos = torch.randint(0, 1 << 20, (61,), dtype=torch.int32) if positions else None
        cpu = [z.contiguous() for z in cpu]
        gpu = [z.contiguous() for z in gpu]
        before = pool.bytes()
        pool.append([70], [61], gpu[0], gpu[1], gpu[2] if with_l else None, theta, None if pos is None else pos.cuda())
        # (the nine tokens before are what the pool was filled with: codes 0x55 at scale byte 0x55)
        check_append(pool, before, [70], [61], cpu[0], cpu[1], cpu[2] if with_l else None, theta, pos)


def test_append_far_positions():
    """Positions of a million tokens: the angles keep their accuracy."""
    heads, d = 1, 128
    pool = Pool([16], heads, d, 8, "int8", F32)
    cpu, gpu = rows_of(5, 16, heads, d, 8, F32, wide=False)
    pos = torch.arange(1_000_000, 1_000_016, dtype=torch.int32)
    before = pool.bytes()
    pool.append([16], [16], *gpu, THETA, pos.cuda())
    check_append(pool, before, [16], [16], *cpu, THETA, pos)


def test_append_passes_over_what_has_no_place():
    """Rows before a sequence's first token, a sequence beyond max_seq_len, a table entry out of range, a length of zero."""
    heads, d, rank = 2, 64, 8
    pool = Pool([40, 40, 40, 40], heads, d, rank, "e4m3", BF16)
    cpu, gpu = rows_of(3, 30 + 20 + 20 + 4, heads, d, rank, BF16)
    pool.table[2, 1] = 1 << 20
    before = pool.bytes()
    counts, lens = [30, 20, 20, 4], [11, 41, 35, 0]
    pool.append(lens, counts, *gpu)
    after = pool.bytes()
    # sequence 0: its last eleven rows; 1: nothing; 2: the blocks that have a place; 3: nothing
    k, v, l = cpu
    skipped = pool.blocks[2][1]
    assert all(torch.equal(a[skipped], b[skipped]) for a, b in zip(after, before))
    pool.blocks[2][1] = pool.blocks[2][0]  # (for the check: the block passed over is compared above)
    for t in (1, 3):
        for blk in pool.blocks[t]:
            assert all(torch.equal(a[blk], b[blk]) for a, b in zip(after, before))
    blk = pool.blocks[0][0]
    for h in range(heads):
        new = rotated(k[19:30].double(), torch.arange(11), THETA)[:, h]
        check_block("e4m3", after[0][blk, h].view(TORCH["e4m3"]), after[2][blk, h], new, (0, 11), None, 0, "short")
        check_block("e4m3", after[1][blk, h].view(TORCH["e4m3"]).t(), after[3][blk, h], v[19:30, h].double(), (0, 11), None, 0, "short")
    assert torch.equal(after[4][blk, :11], l[19:30]) and bool((after[0][blk, :, 11:] == 0x55).all())


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_append_zeros_and_borders(code):
    """Blocks of zeros have the smallest scale; largest values at the border and one step beyond it; tiny and huge values."""
    heads, d = 1, 64
    top = TOP[code]
    pool = Pool([16] * 6, heads, d, 8, code, F32)
    x = torch.zeros(6, 16, heads, d)
    x[1, 3, 0, 5] = top
    x[2, 3, 0, 5] = torch.nextafter(torch.tensor(top), torch.tensor(1e9))
    x[3, 0, 0, 0] = 1e-42
    x[4, :, 0, :] = 3e38
    x[5, 15, 0, 63] = -top / 8
    y = x.view(96, heads, d).cuda()
    pool.append([16] * 6, [16] * 6, y, y, None, 0.0)
    after = pool.bytes()
    want = [1, 127, 128, 1, int(least_exponent(torch.tensor(3e38).double(), code)) + 127, 124]
    for t in range(6):
        blk = pool.blocks[t][0]
        assert int(after[2][blk, 0]) == want[t] and int(after[3][blk, 0]) == want[t], t
        held = values_of(after[0][blk, 0].view(TORCH[code]), after[2][blk, 0])
        unit = 2.0 ** (want[t] - 127)
        assert bool(((held - x[t, :, 0].double()).abs() <= half_step(held / unit, code) * unit).all())


def test_append_not_a_number_stays_in_its_block_and_head():
    heads, d = 2, 128
    pool = Pool([40], heads, d, 8, "e4m3", BF16)
    cpu, gpu = rows_of(3, 40, heads, d, 8, BF16)
    clean = Pool([40], heads, d, 8, "e4m3", BF16)
    clean.append([40], [40], *gpu)
    gpu[0][20, 1, 3] = float("nan")
    gpu[1][20, 0, 3] = float("inf")
    pool.append([40], [40], *gpu)
    a, b = pool.bytes(), clean.bytes()
    blk = pool.blocks[0][1]
    assert int(a[2][blk, 1]) == 255 and int(a[3][blk, 0]) == 255
    for i in range(4):
        differs = (a[i] != b[i]).view(a[i].shape[0], heads, -1).any(2)
        assert differs.nonzero().tolist() == [[blk, 1 if i % 2 == 0 else 0]]


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,heads,d,rank", [(BF16, 2, 128, 16), (F32, 3, 64, 5)])
@pytest.mark.parametrize("kept", [False, True])
def test_gather(code, dtype, heads, d, rank, kept):
    room = [150, 1, 33, 90]
    pool = Pool(room, heads, d, rank, code, dtype, seed=4)
    _, gpu = rows_of(2, sum(room), heads, d, rank, dtype)
    pool.append(room, room, *gpu)
    rows = [100, 1, 33, 0]
    per = -(-max(rows) // BLOCK)
    dst = [torch.full((4 * per, heads, BLOCK, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)] + [torch.full((4 * per, BLOCK, rank), 7.0, dtype=dtype, device="cuda")]
    table = torch.arange(4 * per, dtype=torch.int32, device="cuda").view(4, per).flip(0).contiguous()
    lens = torch.tensor(rows, dtype=torch.int32, device="cuda")
    pick = None
    if kept:
        g = torch.Generator().manual_seed(0)
        pick = torch.full((4, max(rows) + 3), -5, dtype=torch.int32)
        for t, m in enumerate(rows):
            pick[t, :m] = torch.randperm(room[t], generator=g)[:m]
        pick[0, 5], pick[0, 6] = room[0], -1            # no such rows: left as they are
        pick = pick.cuda()
    lra.lra_cache8_gather(pool.shape, pool.cache, lra.make_cache(*dst, lens, max(rows), table), pick)
    torch.cuda.synchronize()
    want = [z.clone() for z in dst]
    for z in want:
        z.fill_(7.0)
    for t, m in enumerate(rows):
        for i in range(m):
            j = int(pick[t, i]) if kept else room[t] - m + i
            if not 0 <= j < room[t]:
                continue
            src, to = pool.blocks[t][j // BLOCK], int(table[t, i // BLOCK])
            want[0][to, :, i % BLOCK] = values_of(pool.k[src, :, j % BLOCK].cpu(), pool.k_scale[src].cpu()[:, None]).to(dtype).cuda()
            want[1][to, :, i % BLOCK] = values_of(pool.v[src, :, :, j % BLOCK].cpu(), pool.v_scale[src].cpu()[:, None]).to(dtype).cuda()
            want[2][to, i % BLOCK] = pool.l[src, j % BLOCK]
    assert all(torch.equal(a, b) for a, b in zip(dst, want))


def test_gather_to_contiguous_rows_and_more_than_there_are():
    pool = Pool([50], 2, 64, 8, "int8", BF16)
    _, gpu = rows_of(2, 50, 2, 64, 8, BF16)
    pool.append([50], [50], *gpu)
    k, v = (torch.full((2, 60, 64), 7.0, dtype=BF16, device="cuda").transpose(0, 1) for _ in range(2))
    l = torch.full((60, 16), 7.0, dtype=BF16, device="cuda")[:, :8]
    lens = torch.tensor([60], dtype=torch.int32, device="cuda")
    lra.lra_cache8_gather(pool.shape, pool.cache, lra.make_cache(k, v, l, lens, 60))
    torch.cuda.synchronize()
    ids = torch.tensor(pool.blocks[0])
    flat = lambda c, s: values_of(c.cpu(), s.cpu()[..., None, None])[ids]  # noqa: E731
    want_k = flat(pool.k, pool.k_scale).transpose(1, 2).reshape(-1, 2, 64)[:50]
    want_v = flat(pool.v, pool.v_scale).permute(0, 3, 1, 2).reshape(-1, 2, 64)[:50]
    assert bool((k[:10] == 7).all()) and bool((v[:10] == 7).all()) and bool((l[:10] == 7).all())
    assert torch.equal(k[10:].cpu().double(), want_k) and torch.equal(v[10:].cpu().double(), want_v)
    assert torch.equal(l[10:].cpu(), pool.l.cpu()[ids].view(-1, 8)[:50])


def test_append_in_a_graph():
    """A captured decode step: the lengths advance between the replays."""
    heads, d, rank = 2, 128, 8
    pool, twin = (Pool([64, 64], heads, d, rank, "e4m3", BF16, seed=9) for _ in range(2))
    _, (k, v, l) = rows_of(1, 2, heads, d, rank, BF16)
    start = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    pool.lens.copy_(torch.tensor([1, 31], dtype=torch.int32))
    cache = pool.cache
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lra.lra_cache8_append(pool.shape, cache, start, 1, k, v, l, THETA)
    for step in range(20):
        k.mul_(-1.07)
        v.add_(0.25)
        pool.lens.copy_(torch.tensor([1 + step, 31 + step], dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        twin.append([1 + step, 31 + step], [1, 1], k, v, l)
        assert all(torch.equal(a, b) for a, b in zip(pool.bytes(), twin.bytes())), step


def test_gather_in_a_graph():
    """Other kept rows, lengths and cache contents between the replays."""
    pool = Pool([120, 60], 2, 128, 16, "e4m3", BF16, seed=5)
    _, gpu = rows_of(3, 180, 2, 128, 16, BF16)
    pool.append([120, 60], [120, 60], *gpu)
    dst, twin = ([torch.zeros(8, 2, BLOCK, 128, dtype=BF16, device="cuda") for _ in range(2)] + [torch.zeros(8, BLOCK, 16, dtype=BF16, device="cuda")] for _ in range(2))
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4).contiguous()
    lens = torch.tensor([64, 10], dtype=torch.int32, device="cuda")
    kept = torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 1).contiguous()
    caches = [lra.make_cache(*z, lens, 64, table) for z in (dst, twin)]
    lra.lra_cache8_gather(pool.shape, pool.cache, caches[0], kept)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    cache = pool.cache
    with torch.cuda.graph(graph):
        lra.lra_cache8_gather(pool.shape, cache, caches[0], kept)
    for step, m in enumerate(([64, 10], [1, 60], [0, 0], [33, 17])):
        lens.copy_(torch.tensor(m, dtype=torch.int32))
        kept.copy_((kept * 7 + step) % 60)
        pool.k_scale.add_(1)
        for z in dst + twin:
            z.fill_(step)
        graph.replay()
        lra.lra_cache8_gather(pool.shape, pool.cache, caches[1], kept)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(dst, twin)), step


def test_appends_and_gathers_on_two_streams():
    pools = [Pool([90, 40], 2, 64, 8, "int8", BF16, seed=s) for s in (1, 2, 1, 2)]
    rows = [rows_of(s, 130, 2, 64, 8, BF16)[1] for s in (1, 2)]
    for pool, (k, v, l) in zip(pools[2:], rows):
        pool.append([90, 40], [90, 40], k, v, l)
    start = torch.tensor([0, 90, 130], dtype=torch.int32, device="cuda")
    streams = [torch.cuda.Stream() for _ in range(2)]
    for pool in pools[:2]:
        pool.lens.copy_(torch.tensor([90, 40], dtype=torch.int32))
    torch.cuda.synchronize()
    for _ in range(3):
        for pool, (k, v, l), stream in zip(pools, rows, streams):
            lra.lra_cache8_append(pool.shape, pool.cache, start, 90, k, v, l, THETA, stream=stream)
    torch.cuda.synchronize()
    for pool, twin in zip(pools[:2], pools[2:]):
        assert all(torch.equal(a, b) for a, b in zip(pool.bytes(), twin.bytes()))


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_values_over_all_scales(code, dtype):
    """Every code at every scale byte: exact from byte 3 (e4m3) or 0 (integers) to 246, the nearest number elsewhere."""
    d, n = 64, 255
    codes = [c for c in range(256) if code == "int8" or c & 127 != 127]
    every = torch.tensor((codes * 5)[:BLOCK * d], dtype=torch.uint8)
    k = every.view(1, 1, BLOCK, d).expand(n, 1, BLOCK, d).contiguous().cuda().view(TORCH[code])
    v = every.view(1, 1, d, BLOCK).expand(n, 1, d, BLOCK).contiguous().cuda().view(TORCH[code])
    scale = torch.arange(n, dtype=torch.uint8)[:, None]
    dev = scale.cuda()
    l, lens = torch.zeros(n, BLOCK, 8, dtype=dtype, device="cuda"), torch.tensor([n * BLOCK], dtype=torch.int32, device="cuda")
    out = [torch.full((n * BLOCK, 1, d), 7.0, dtype=dtype, device="cuda") for _ in range(2)] + [torch.zeros(n * BLOCK, 8, dtype=dtype, device="cuda")]
    shape = lra.make_shape(out[0], 1, 8)
    lra.lra_cache8_gather(shape, lra.make_cache8(k, v, dev, dev, l, lens, n * BLOCK), lra.make_cache(*out, lens, n * BLOCK))
    torch.cuda.synchronize()
    rows = every.view(TORCH[code]).view(1, BLOCK, d), every.view(TORCH[code]).view(1, d, BLOCK).transpose(1, 2)
    for got, c in zip(out, rows):
        want = values_of(c, scale[..., None])
        got = got.view(n, BLOCK, d).cpu()
        # (a double's way to bf16 is by fp32, which holds these values exactly, or as infinite)
        assert torch.equal(got, want.float().to(dtype))
        exact = slice(3 if code == "e4m3" and dtype == BF16 else 0, 247)
        assert torch.equal(got[exact].double(), want[exact])
