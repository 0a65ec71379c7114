"""The batch calls as programs use them: two at once, replayed with other lengths, many sequences, bounds that are not met."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, attention, key_weights, make
from tests.test_batch_gpu import TOL, check
from tests.test_evict_gpu import expected
from tests.test_key_weights_gpu import TOL as WEIGHTS_TOL
from tests.test_key_weights_gpu import run as weigh

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 64)])
@pytest.mark.parametrize("causal", [False, True])
def test_two_calls_at_once(causal, dtype, rank):
    """On two streams, each with a workspace of its own."""
    cases = [BatchCase([3000, 900], [3, 2] if not causal else [150, 9], causal, 0, 0, (8, 2, 128), rank, dtype, seed=s) for s in (1, 2)]
    devs = [Device(make(c), lra) for c in cases]
    alone = [d.attend() for d in devs]
    alone_w = [weigh(d, 0.0, torch.zeros(2, 3000, device="cuda")) for d in devs]
    streams = [torch.cuda.Stream() for _ in devs]
    outs, ws = [torch.full_like(d.q, float("nan")) for d in devs], []
    w = [torch.zeros(2, 3000, device="cuda") for _ in devs]
    for d in devs:
        ws.append([torch.empty(size(d.shape, d.cache, d.batch), dtype=torch.uint8, device="cuda")
                   for size in (lra.lra_batch_workspace_bytes, lra.lra_key_weights_workspace_bytes)])
    torch.cuda.synchronize()
    for _ in range(5):
        for d, s, out, (a, b), x in zip(devs, streams, outs, ws, w):
            lra.lra_attn_batch(d.shape, d.cache, d.b_k, d.b_v, d.case.n_adapters, d.batch, d.q, out, a, stream=s)
            lra.lra_key_weights(d.shape, d.cache, d.b_k, d.case.n_adapters, d.batch, d.q, 0.0, x, b, stream=s)
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(outs[i], alone[i]) and torch.equal(w[i], alone_w[i])


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16)])
@pytest.mark.parametrize("causal,window", [(False, 0), (True, 100)])
def test_a_graph_serves_other_lengths_and_queries(causal, window, dtype, rank):
    """Weights, selection, gather and attention in one graph, replayed while sequences grow and queries move from one to another."""
    lens, budget = [700, 90, 400], 128
    c = BatchCase(lens, [5, 1, 2] if causal else [2, 1, 1], causal, window, 4 if window else 0, (8, 2, 64), rank, dtype, seed=3, poison=False)
    d = Device(make(c), lra)
    table = torch.arange(24, dtype=torch.int32, device="cuda").view(3, 8)
    dst = [torch.zeros(24, 2, 16, 64, dtype=dtype, device="cuda") for _ in range(2)] + [torch.zeros(24, 16, rank, dtype=dtype, device="cuda")]
    kept, new = torch.zeros(3, budget, dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    w, w2 = torch.zeros(3, 700, device="cuda"), torch.zeros(3, budget, device="cuda")
    cut = lra.make_cache(*dst, new, budget, table)
    batch = lra.make_batch(d.start, d.adapter, 8 if causal else 4, causal=causal, window=window, sinks=c.sinks)
    out, small = torch.empty_like(d.q), torch.empty_like(d.q)
    sizes = (lra.lra_key_weights_workspace_bytes(d.shape, d.cache, batch), lra.lra_batch_workspace_bytes(d.shape, d.cache, batch),
             lra.lra_batch_workspace_bytes(d.shape, cut, batch))
    ws = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]

    def step():
        lra.lra_key_weights(d.shape, d.cache, d.b_k, c.n_adapters, batch, d.q, 0.9, w, ws[0])
        lra.lra_attn_batch(d.shape, d.cache, d.b_k, d.b_v, c.n_adapters, batch, d.q, out, ws[1])
        lra.lra_evict_select(d.cache, w, budget, 2, 16, kept, new)
        lra.lra_cache_gather(d.shape, d.cache, kept, cut, weights=w, dst_weights=w2)
        lra.lra_attn_batch(d.shape, cut, d.b_k, d.b_v, c.n_adapters, batch, d.q, small, ws[2])

    results = (w, out, kept, new, *dst, w2, small)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    total = sum(c.counts)
    for now, starts in ((lens, [0, c.counts[0], c.counts[0] + 1, total]), ([17, 90, 129], [0, 0, 3, total]), ([300, 0, 400], [0, 2, 2, total]),
                        ([650, 64, 1], [0, 3, 4, total])):
        d.lens.copy_(i32(now))
        d.start.copy_(i32(starts))
        d.q.mul_(0.9)
        got = []
        for run in (graph.replay, step):
            w.fill_(0.5)
            for y in results[1:]:
                y.zero_()
            for y in ws:
                y.fill_(255)
            run()
            torch.cuda.synchronize()
            got.append([y.clone() for y in results])
        for a, b in zip(*got):
            assert torch.equal(a, b)
        for t in range(3):
            assert got[0][2][t, :int(got[0][3][t])].tolist() == expected(w[t].tolist(), now[t], budget, 2, 16)


@pytest.mark.parametrize("dtype,rank", [(BF16, 16), (BF16, 12)])
def test_more_sequences_than_a_grid_dimension_has_rows(dtype, rank):
    """70000 sequences of one token: O = V + L B_V of it, in 64 bits to half a step of the output and of P = 1 (none)."""
    n, hkv, d = 70000, 1, 64
    g = torch.Generator(device="cuda").manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    k, v, l = randn(n, hkv, 16, d), randn(n, hkv, 16, d), randn(n, 16, rank)
    b_k, b_v = randn(2, rank, d) * 0.1, randn(2, rank, d) * 0.1
    table = torch.randperm(n, generator=g, device="cuda").to(torch.int32).view(n, 1)
    lens = torch.ones(n, dtype=torch.int32, device="cuda")
    has = torch.rand(n, generator=g, device="cuda") < 0.7   # the others have no query
    start = torch.cat((torch.zeros(1, device="cuda", dtype=torch.int64), has.long().cumsum(0))).to(torch.int32)
    total = int(start[-1])
    q, adapter = randn(total, 2, d), torch.randint(0, 2, (total,), generator=g, device="cuda").to(torch.int32)
    shape, cache = lra.make_shape(q, hkv, rank), lra.make_cache(k, v, l, lens, 1, table)
    owner = table[has, 0].long()
    expect = v[owner, :, 0].double() + torch.einsum("nr,nrd->nd", l[owner, 0].cpu().double(), b_v.cpu().double()[adapter.long().cpu()]).cuda()[:, None]
    for causal in (False, True):
        batch = lra.make_batch(start, adapter, 1, causal=causal)
        out = torch.full_like(q, float("nan"))
        ws = torch.empty(max(lra.lra_batch_workspace_bytes(shape, cache, batch), 256), dtype=torch.uint8, device="cuda")
        lra.lra_attn_batch(shape, cache, b_k, b_v, 2, batch, q, out, ws)
        torch.cuda.synchronize()
        err = (out.double() - expect).abs()
        # half a step of the output, and sums of `rank` products in fp32 (O_lr goes in with 16 bits at least)
        assert (err <= 2 ** -8 * expect.abs() + 2 ** -14).all()
        with pytest.raises(lra.LraError):
            lra.lra_key_weights_workspace_bytes(shape, cache, batch)


@pytest.mark.parametrize("counts", [[2, 1, 2], [4, 0, 4], [5, 1, 0]])
@pytest.mark.parametrize("heads", [(16, 1, 128), (7, 1, 64), (32, 4, 64)])
def test_bounds_of_the_few_rows_kernels(heads, counts):
    """Groups and queries at, below and above 32 rows of a sequence."""
    check(BatchCase([700, 20, 310], counts, False, 0, 0, heads, 16, BF16, seed=27))
    check(BatchCase([700, 20, 310], counts, True, 90, 4, heads, 16, BF16, seed=28))


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 12)])
@pytest.mark.parametrize("causal", [False, True])
def test_a_bound_above_the_queries(causal, dtype, rank):
    """max_queries_per_seq is a bound: one that no sequence meets chooses other kernels, not other results."""
    c = BatchCase([500, 60, 0, 220], [3, 1, 0, 2], causal, 0, 0, (8, 2, 64), rank, dtype, seed=29)
    x = make(c)
    ref, ref_w = attention(x), key_weights(x)
    for most in (3, 6):
        d = Device(x, lra)
        d.batch = lra.make_batch(d.start, d.adapter, most, causal=causal)
        got = d.attend().double().cpu()
        assert float((got - ref).norm() / ref.norm()) <= TOL[dtype]
        w = weigh(d, 0.0, torch.zeros(4, 500, device="cuda")).double().cpu()
        assert float((w - ref_w).norm() / ref_w.norm()) <= WEIGHTS_TOL


@pytest.mark.parametrize("decay", [-1.0, 2.0, 1e-30])
def test_any_finite_decay(decay):
    c = BatchCase([130, 40], [2, 1], seed=30)
    x = make(c)
    old = torch.rand(2, 130)
    inside = torch.arange(130) < torch.tensor(c.lens)[:, None]
    ref = torch.where(inside, key_weights(x) + decay * old.double(), old.double())
    got = weigh(Device(x, lra), decay, old.clone().cuda()).double().cpu()
    assert float((got - ref).norm() / ref.norm()) <= WEIGHTS_TOL


def test_a_token_kept_twice():
    """kept is the caller's: any tokens of the sequence, in any order."""
    c = BatchCase([50, 31], [1, 1], heads=(4, 2, 64), poison=False)
    x = make(c)
    d = Device(x, lra)
    kept = i32([[49, 0, 0, 7, 49], [30, 30, 30, 30, 30]])
    k2, v2 = (torch.zeros(2, 2, 16, 64, dtype=BF16, device="cuda") for _ in range(2))
    l2 = torch.zeros(2, 16, 8, dtype=BF16, device="cuda")
    dst = lra.make_cache(k2, v2, l2, i32([5, 3]), 5, i32([[1], [0]]))
    lra.lra_cache_gather(d.shape, d.cache, kept, dst)
    torch.cuda.synchronize()
    for t, (blk, m) in enumerate(((1, 5), (0, 3))):
        idx = kept[t, :m].long().cpu()
        assert torch.equal(k2[blk, :, :m].cpu(), x.k[t, idx].transpose(0, 1)) and torch.equal(l2[blk, :m].cpu(), x.l[0, t, idx])
        assert (k2[blk, :, m:] == 0).all()
