"""lra_evict_select and lra_cache_gather: whole numbers and moved rows, so everything has to be equal."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, attention, make

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def expected(w, n, budget, sinks, recent):
    """By the definition: sorted on (weight, first index), NaN last."""
    if n <= budget:
        return list(range(n))
    mid = list(range(sinks, n - recent))
    key = lambda j: (-float("inf") if w[j] != w[j] else w[j])  # noqa: E731
    nan_last = lambda j: w[j] != w[j]  # noqa: E731
    mid.sort(key=lambda j: (nan_last(j), -key(j), j))
    return sorted(list(range(sinks)) + mid[:budget - sinks - recent] + list(range(n - recent, n)))


def cache_of(lens, max_seq_len):
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    z = torch.zeros(16, 1, 64, device="cuda")
    c = lra.make_cache(z, z, z[:, 0, :8], lens, max_seq_len)
    c.n_seqs = len(lens)  # (only the lengths are read)
    return c, lens


def select(lens, w, budget, sinks, recent, max_seq_len=None, alias=False, kept=None):
    c, lens_d = cache_of(lens, max_seq_len or max(max(lens), 1))
    kept = torch.full((len(lens), min(budget, c.max_seq_len) + 3), -7, dtype=torch.int32, device="cuda") if kept is None else kept
    new = lens_d if alias else torch.full((len(lens),), -7, dtype=torch.int32, device="cuda")
    lra.lra_evict_select(c, w.cuda(), budget, sinks, recent, kept, new)
    torch.cuda.synchronize()
    return kept.cpu(), new.cpu()


def check(lens, w, budget, sinks, recent, **kw):
    kept, new = select(lens, w, budget, sinks, recent, **kw)
    for t, n in enumerate(lens):
        ref = expected(w[t].tolist(), n, budget, sinks, recent)
        assert int(new[t]) == len(ref)
        assert kept[t, :len(ref)].tolist() == ref
        assert (kept[t, len(ref):] == -7).all(), "entries behind the kept ones are left alone"


def weights(T, n, kind, seed=0):
    g = torch.Generator().manual_seed(seed)
    if kind == "tail":
        return torch.rand(T, n, generator=g).clamp_(min=1e-6) ** -1.2
    if kind == "normal":
        return torch.randn(T, n, generator=g)
    if kind == "equal":
        return torch.full((T, n), 0.25)
    if kind == "few":
        return torch.randint(-2, 3, (T, n), generator=g).float() * 1e-3
    if kind == "zeros":
        return torch.where(torch.rand(T, n, generator=g) < 0.5, 0.0, -0.0)
    w = torch.randn(T, n, generator=g)  # "special"
    w[torch.rand(T, n, generator=g) < 0.1] = float("nan")
    w[torch.rand(T, n, generator=g) < 0.1] = float("inf")
    w[torch.rand(T, n, generator=g) < 0.1] = -float("inf")
    w[torch.rand(T, n, generator=g) < 0.1] = 1e-42
    return w


@pytest.mark.parametrize("kind", ["tail", "normal", "equal", "few", "zeros", "special"])
@pytest.mark.parametrize("lens,budget,sinks,recent", [
    ([1], 1, 0, 0), ([2], 1, 0, 0), ([2], 1, 1, 0), ([2], 1, 0, 1), ([5, 0, 3, 9], 4, 1, 2), ([70, 65, 64, 63], 64, 4, 10),
    ([100, 1000, 37], 37, 0, 37), ([1000], 999, 3, 5), ([1000, 999], 17, 16, 1), ([1025, 5000], 1000, 4, 100), ([4107], 11, 4, 7),
    ([4109, 4100], 300, 4, 7), ([16400, 7000], 4096, 4, 11), ([20000], 19999, 0, 0)])
def test_select(kind, lens, budget, sinks, recent):
    check(lens, weights(len(lens), max(lens), kind, seed=budget), budget, sinks, recent)


@pytest.mark.parametrize("kind", ["tail", "few", "special"])
@pytest.mark.parametrize("n", [65536, 65540, 65541, 200001])
def test_select_of_long_sequences(kind, n):
    check([n, n // 3], weights(2, n, kind, seed=n), 8192, 4, 0)


def test_select_with_a_bound_strides_and_lengths_in_place():
    w = weights(3, 6000, "normal")
    check([500, 3000, 40], w[:, :5000], 256, 4, 30, max_seq_len=4999)       # rows 6000 apart
    kept, new = select([500, 3000, 40], w, 256, 4, 30, alias=True)
    assert new.tolist() == [256, 256, 40]
    kept2, _ = select([500, 3000, 40], w, 256, 4, 30)
    assert torch.equal(kept, kept2)
    kept, new = select([500, 9000], w[:2], 256, 4, 30, max_seq_len=700)     # taken for 700
    assert kept[1, :256].tolist() == expected(w[1].tolist(), 700, 256, 4, 30)


LAYOUTS = ["paged", "paged_to_contig", "contig", "head_major", "contig_to_paged"]


@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dtype,rank,heads", [(BF16, 16, (8, 8, 128)), (BF16, 5, (4, 2, 64)), (F32, 8, (6, 3, 64)), (F32, 7, (2, 1, 128)),
                                              (BF16, 64, (7, 7, 64))])
@pytest.mark.parametrize("adapters", [1, 3])
def test_gather(layout, dtype, rank, heads, adapters):
    one = "contig" in layout or layout == "head_major"
    lens = [333] if one else [333, 90, 1, 200]
    budget = 101
    if adapters > 1 and rank % 8:
        pytest.skip("own low-rank caches lie a multiple of eight elements apart")
    c = BatchCase(lens, [1] * len(lens), heads=heads, rank=rank, dtype=dtype, paged=layout.startswith("paged"),
                  head_major=layout == "head_major", own_l=adapters > 1, poison=False, extra_rank_stride=8 if rank % 8 == 0 else 0)
    x = make(c)
    d = Device(x, lra)
    T, hkv, hd = len(lens), heads[1], heads[2]
    w = weights(T, max(lens), "normal").cuda()
    kept = torch.full((T, budget), -7, dtype=torch.int32, device="cuda")
    new = torch.zeros(T, dtype=torch.int32, device="cuda")
    lra.lra_evict_select(d.cache, w, budget, 2, 9, kept, new)
    to_pages = layout in ("paged", "contig_to_paged")
    A = adapters
    if to_pages:
        per = -(-budget // 16)
        table = torch.randperm(T * per + 1)[:T * per].view(T, per).to(torch.int32).cuda()
        k2, v2 = (torch.full((T * per + 1, hkv, 16, hd), 9.0, dtype=dtype, device="cuda") for _ in range(2))
        l2 = torch.full((A, T * per + 1, 16, rank), 9.0, dtype=dtype, device="cuda")
    else:
        table = None
        k2, v2 = (torch.full((budget + 2, hkv, hd), 9.0, dtype=dtype, device="cuda") for _ in range(2))
        l2 = torch.full((A, budget + 2, rank), 9.0, dtype=dtype, device="cuda")
    if layout == "paged_to_contig":  # one sequence of the batch at a time
        lens = lens[:1]
        T = 1
        d.cache.n_seqs = 1
        kept, new, w = kept[:1], new[:1], w[:1]
    dst = lra.make_cache(k2, v2, l2 if A > 1 else l2[0], new, budget, table, l_per_adapter=A > 1)
    w2 = torch.full((T, budget + 1), 9.0, device="cuda")
    lra.lra_cache_gather(d.shape, d.cache, kept, dst, n_adapters=A, weights=w, dst_weights=w2)
    torch.cuda.synchronize()
    touched_k, touched_l = torch.zeros(k2.shape[:3] if to_pages else k2.shape[:2], dtype=torch.bool), torch.zeros(l2.shape[:-1], dtype=torch.bool)
    for t, n in enumerate(lens):
        m = min(n, budget)
        assert int(new[t]) == m
        idx = kept[t, :m].cpu().long()
        assert torch.equal(w2[t, :m].cpu(), w[t].cpu()[idx]) and (w2[t, m:] == 9).all()
        i = torch.arange(m)
        if to_pages:
            blk, slot = table[t].cpu().long()[i // 16], i % 16
            assert torch.equal(k2.cpu()[blk, :, slot], x.k[t, idx]) and torch.equal(v2.cpu()[blk, :, slot], x.v[t, idx])
            assert torch.equal(l2.cpu()[:, blk, slot], x.l[:, t, idx])
            touched_k[blk, :, slot] = True
            touched_l[:, blk, slot] = True
        else:
            assert torch.equal(k2.cpu()[i], x.k[t, idx]) and torch.equal(v2.cpu()[i], x.v[t, idx])
            assert torch.equal(l2.cpu()[:, i], x.l[:, t, idx])
            touched_k[i] = True
            touched_l[:, i] = True
    assert (k2.cpu()[~touched_k] == 9).all() and (v2.cpu()[~touched_k] == 9).all() and (l2.cpu()[~touched_l] == 9).all()


def test_within_one_pool_of_pages():
    """dst's pages are free pages of src's own pool."""
    c = BatchCase([300, 150], [1, 1], heads=(4, 2, 64), rank=8, poison=False)
    x = make(c)
    d = Device(x, lra)
    nb = d.k.shape[0]
    per = -(-100 // 16)
    k, v = (torch.cat((y, torch.zeros(2 * per, *y.shape[1:], dtype=y.dtype, device="cuda"))) for y in (d.k, d.v))
    l = torch.cat((d.l[0], torch.zeros(2 * per, *d.l.shape[2:], dtype=d.l.dtype, device="cuda")))
    table2 = (nb + torch.arange(2 * per, device="cuda")).view(2, per).to(torch.int32)
    new = torch.empty(2, dtype=torch.int32, device="cuda")
    kept = torch.empty(2, 100, dtype=torch.int32, device="cuda")
    src, dst = lra.make_cache(k, v, l, d.lens, 300, d.table), lra.make_cache(k, v, l, new, 100, table2)
    lra.lra_evict_select(src, weights(2, 300, "normal").cuda(), 100, 4, 20, kept, new)
    lra.lra_cache_gather(d.shape, src, kept, dst)
    torch.cuda.synchronize()
    assert torch.equal(k[:nb].nan_to_num(7), d.k.nan_to_num(7))
    for t in range(2):
        i = torch.arange(100)
        assert torch.equal(k.cpu()[table2[t].cpu().long()[i // 16], :, i % 16], x.k[t, kept[t].cpu().long()])


def test_weights_eviction_and_attention_together():
    """As a serving loop uses them: decode steps add up weights, the caches are cut, and the next step attends over what is
    left; against the float64 evaluation on the tokens that stayed."""
    c = BatchCase([400, 90, 260], [4, 4, 4], False, 0, 0, (8, 2, 128), 16, BF16, seed=8, poison=False)
    x = make(c)
    d = Device(x, lra)
    w = torch.zeros(3, 400, device="cuda")
    ws = torch.empty(lra.lra_key_weights_workspace_bytes(d.shape, d.cache, d.batch), dtype=torch.uint8, device="cuda")
    for decay in (0.0, 0.9):
        lra.lra_key_weights(d.shape, d.cache, d.b_k, c.n_adapters, d.batch, d.q, decay, w, ws)
    budget = 128
    kept, new = torch.full((3, budget), -7, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    lra.lra_evict_select(d.cache, w, budget, 4, 32, kept, new)
    per = budget // 16
    table = torch.arange(3 * per, dtype=torch.int32, device="cuda").view(3, per)
    k2, v2 = (torch.empty(3 * per, 2, 16, 128, dtype=BF16, device="cuda") for _ in range(2))
    l2 = torch.empty(3 * per, 16, 16, dtype=BF16, device="cuda")
    dst = lra.make_cache(k2, v2, l2, new, budget, table)
    w2 = torch.empty(3, budget, device="cuda")
    lra.lra_cache_gather(d.shape, d.cache, kept, dst, weights=w, dst_weights=w2)
    out = torch.empty_like(d.q)
    ws2 = torch.empty(lra.lra_batch_workspace_bytes(d.shape, dst, d.batch), dtype=torch.uint8, device="cuda")
    lra.lra_attn_batch(d.shape, dst, d.b_k, d.b_v, c.n_adapters, d.batch, d.q, out, ws2)
    torch.cuda.synchronize()
    y = make(c)
    lens = new.tolist()
    for t in range(3):
        idx = kept[t, :lens[t]].cpu().long()
        assert idx.tolist() == expected(w[t].tolist(), c.lens[t], budget, 4, 32)
        for a, b in ((y.k, x.k), (y.v, x.v)):
            a[t, :lens[t]] = b[t, idx]
        y.l[:, t, :lens[t]] = x.l[:, t, idx]
    y.case = BatchCase(**{**c.__dict__, "lens": lens})
    ref = attention(y)
    assert float((out.double().cpu() - ref).norm() / ref.norm()) <= 5e-3
