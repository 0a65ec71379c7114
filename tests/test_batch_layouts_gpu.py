"""The batch calls on caches whose rows lie far apart, and on buffers with room behind the sequences."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, attention, key_weights, make
from tests.test_batch_gpu import TOL
from tests.test_key_weights_gpu import TOL as WEIGHTS_TOL
from tests.test_key_weights_gpu import run as weigh

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
APART = 1 << 26  # elements between blocks: 128 MiB of bf16
BLOCKS = 42      # 5.6 GB: beyond 32-bit byte offsets


@pytest.fixture(scope="module")
def far_memory():
    memory = [torch.empty(BLOCKS * APART, dtype=BF16, device="cuda") for _ in range(2)]
    yield memory
    memory.clear()
    torch.cuda.empty_cache()


def far_pool(memory, dense):
    nb, hkv, bs, d = dense.shape
    assert APART * 2 * 17 > 1 << 31 and 17 < nb <= BLOCKS
    pool = memory.as_strided((nb, hkv, bs, d), (APART, bs * d, d, 1))
    pool.copy_(dense)
    return pool


def move_far(dev, far_memory):
    """The device's cache with its K_base and V_base blocks 128 MiB apart."""
    dev.k, dev.v = (far_pool(m, y) for m, y in zip(far_memory, (dev.k, dev.v)))
    dev.cache = lra.make_cache(dev.k, dev.v, dev.l[0], dev.lens, dev.cache.max_seq_len, dev.table)


FAR_CASES = [  # counts, causal, window, sinks: sequences of 1, 333 and 250 tokens
    ([1, 3, 2], False, 0, 0), ([1, 3, 2], False, 50, 20), ([1, 90, 0], True, 0, 0), ([1, 140, 33], True, 65, 20), ([0, 8, 1], True, 48, 0),
]


@pytest.mark.parametrize("variant", [0, 2])
@pytest.mark.parametrize("mask", range(len(FAR_CASES)))
@pytest.mark.parametrize("d,rank,side", [(128, 16, "bk"), (128, 64, "bk"), (128, 32, "none"), (128, 16, "rotary"), (128, 64, "rotary"), (128, 32, "rotary"),
                                         (64, 16, "none"), (64, 64, "bk"), (64, 32, "rotary"), (64, 8, "bk"), (64, 64, "rotary")])
def test_attention_on_a_pool_beyond_two_gigabytes(d, rank, side, mask, variant, far_memory):
    """The same blocks once dense and once 128 MiB apart: the same bits, by kernels that address them otherwise.  Blocks that nobody
    sees have ids out of range."""
    counts, causal, window, sinks = FAR_CASES[mask]
    c = BatchCase([1, 333, 250], counts, causal, window, sinks, (8, 2, d), rank, BF16, rope=10000.0 if side == "rotary" else 0.0,
                  key_side=side != "none", seed=41 + mask)
    x = make(c)
    old = lra.lra_set_kernel_variant(variant)
    try:
        dev = Device(x, lra)
        dense = dev.attend()
        move_far(dev, far_memory)
        far = dev.attend()
    finally:
        lra.lra_set_kernel_variant(old)
    ref = attention(x)
    assert float((far.double().cpu() - ref).norm() / ref.norm()) <= TOL[BF16]
    assert torch.equal(dense, far)


@pytest.mark.parametrize("mask", range(len(FAR_CASES)))
@pytest.mark.parametrize("d,rank,side", [(128, 16, "bk"), (128, 64, "bk"), (128, 32, "none"), (64, 24, "bk")])
def test_weights_and_gather_on_a_pool_beyond_two_gigabytes(d, rank, side, mask, far_memory):
    counts, causal, window, sinks = FAR_CASES[mask]
    c = BatchCase([1, 333, 250], counts, causal, window, sinks, (8, 2, d), rank, BF16, key_side=side != "none", seed=51 + mask)
    x = make(c)
    dev = Device(x, lra)
    start = torch.rand(3, 333, generator=torch.Generator().manual_seed(2)).cuda()
    dense = weigh(dev, 0.5, start.clone())
    near = dev.cache, dev.k, dev.v
    move_far(dev, far_memory)
    assert torch.equal(dense, weigh(dev, 0.5, start.clone()))
    inside = torch.arange(333) < torch.tensor(c.lens)[:, None]
    ref = key_weights(x) + 0.5 * start.cpu().double()
    assert float(((dense.cpu().double() - ref)[inside]).norm() / ref[inside].norm()) <= WEIGHTS_TOL

    # out of the far pool to a dense one: only tokens that were seen have blocks
    kept, new = torch.zeros(3, 64, dtype=torch.int32), []
    for t in range(3):
        seen = torch.nonzero(x.seen[t])[:, 0][-64:]
        kept[t, :len(seen)] = seen.int()
        new.append(len(seen))
    new_d = torch.tensor(new, dtype=torch.int32, device="cuda")
    table = torch.randperm(12).view(3, 4).to(torch.int32).cuda()
    out = {}
    for name, cache in (("near", near[0]), ("far", dev.cache)):
        k2, v2 = (torch.zeros(12, 2, 16, d, dtype=BF16, device="cuda") for _ in range(2))
        l2 = torch.zeros(12, 16, rank, dtype=BF16, device="cuda")
        lra.lra_cache_gather(dev.shape, cache, kept.cuda(), lra.make_cache(k2, v2, l2, new_d, 64, table))
        out[name] = (k2, v2, l2)
    torch.cuda.synchronize()
    for a, b in zip(*out.values()):
        assert torch.equal(a, b)
    i = torch.arange(64)
    for t in range(3):
        m = new[t]
        assert torch.equal(out["far"][0].cpu()[table.cpu()[t].long()[i[:m] // 16], :, i[:m] % 16], x.k[t, kept[t, :m].long()])
    # and into one
    back_k, back_v = (far_pool(m, torch.zeros(20, 2, 16, d, dtype=BF16, device="cuda")) for m in far_memory)
    l3 = torch.zeros(20, 16, rank, dtype=BF16, device="cuda")
    wide = torch.arange(19, 7, -1, dtype=torch.int32, device="cuda").view(3, 4)
    lra.lra_cache_gather(dev.shape, near[0], kept.cuda(), lra.make_cache(back_k, back_v, l3, new_d, 64, wide))
    torch.cuda.synchronize()
    for t in range(3):
        m = new[t]
        for got, rows in ((back_k, x.k), (back_v, x.v)):
            assert torch.equal(got[wide[t].long()[i[:m] // 16].cuda(), :, i[:m].cuda() % 16].cpu(), rows[t, kept[t, :m].long()])


@pytest.mark.parametrize("n", [120, 200])  # the matrix cores address 2^31 bytes of a kv head's rows, the vector-ALU kernels the rest
@pytest.mark.parametrize("counts,causal,window", [([3], False, 0), ([3], False, 50), ([70], True, 0), ([70], True, 33)])
def test_contiguous_rows_far_apart(counts, causal, window, n, far_memory):
    c = BatchCase([n], counts, causal, window, 4 if window else 0, (4, 2, 64), 16, BF16, paged=False, seed=61)
    x = make(c)
    dev = Device(x, lra)
    k, v = (m.as_strided((n, 2, 64), (1 << 23, 64, 1)) for m in far_memory)  # 16 MiB between tokens
    k.copy_(dev.k)
    v.copy_(dev.v)
    dev.cache = lra.make_cache(k, v, dev.l[0], dev.lens, n)
    ref = attention(x)
    assert float((dev.attend().double().cpu() - ref).norm() / ref.norm()) <= TOL[BF16]
    ref = key_weights(x)
    assert float((weigh(dev, 0.0, torch.empty(1, n, device="cuda")).double().cpu() - ref).norm() / ref.norm()) <= WEIGHTS_TOL


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 64), (BF16, 12)])
@pytest.mark.parametrize("variant", [0, 2])
@pytest.mark.parametrize("n", [1, 63, 130])
@pytest.mark.parametrize("counts,causal,window,rope", [([2], False, 0, 0.0), ([2], False, 40, 0.0), ([100], True, 0, 0.0), ([2], False, 0, 10000.0),
                                                       ([100], True, 33, 10000.0)])
def test_contiguous_buffers_with_room_behind_the_sequence(counts, causal, window, rope, n, variant, dtype, rank):
    """A buffer kept for a growing sequence: the rows behind it hold NaN, and the bound is the buffer's."""
    c = BatchCase([n], counts, causal, window, 3 if window else 0, (4, 2, 128), rank, dtype, paged=False, rope=rope, seed=71, n_adapters=2)
    x = make(c)
    dev = Device(x, lra)
    room = 1000
    k, v = (torch.full((room, 2, 128), float("nan"), dtype=dtype, device="cuda") for _ in range(2))
    l = torch.full((room, rank), float("nan"), dtype=dtype, device="cuda")
    k[:n], v[:n], l[:n] = dev.k, dev.v, dev.l[0]
    dev.cache = lra.make_cache(k, v, l, dev.lens, room)
    ref = attention(x)
    old = lra.lra_set_kernel_variant(variant)
    try:
        got = dev.attend().double().cpu()
        assert torch.isfinite(got).all() and float((got - ref).norm()) <= TOL[dtype] * float(ref.norm())
        if not rope:
            w = weigh(dev, 0.0, torch.full((1, room), 7.0, device="cuda")).cpu()
            ref = key_weights(x)
            assert (w[:, n:] == 7).all() and float((w[:, :n].double() - ref).norm()) <= WEIGHTS_TOL * float(ref.norm())
    finally:
        lra.lra_set_kernel_variant(old)


@pytest.mark.parametrize("rank,d,rope", [(16, 128, 0.0), (64, 64, 0.0), (32, 128, 10000.0)])
@pytest.mark.parametrize("counts,causal", [([4, 1, 0, 3], False), ([40, 1, 0, 150], True)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 0), (1999, 70), (300, 1100), (64, 1024), (1500, 1025)])
def test_tile_walking_over_groups_of_pages(window, sinks, counts, causal, rank, d, rope):
    """Block ids come 64 at a time, 1024 tokens: sinks that end in, at and behind such a group, windows that begin in a later one, shares
    that begin anywhere."""
    c = BatchCase([5000, 37, 900, 2311], counts, causal, window, sinks, (8, 2, d), rank, BF16, rope=rope, seed=81)
    x = make(c)
    ref = attention(x)
    old = lra.lra_set_kernel_variant(2)
    try:
        got = Device(x, lra).attend().double().cpu()
    finally:
        lra.lra_set_kernel_variant(old)
    assert torch.isfinite(got).all() and float((got - ref).norm() / ref.norm()) <= TOL[BF16]
    if not rope:
        ref = key_weights(x)
        got = weigh(Device(x, lra), 0.0, torch.zeros(4, 5000, device="cuda")).double().cpu()
        assert float((got - ref).norm() / ref.norm()) <= WEIGHTS_TOL
