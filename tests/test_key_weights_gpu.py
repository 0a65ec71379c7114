"""lra_key_weights against a float64 evaluation of the softmax."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, key_weights, make
from tests.test_batch_gpu import MASKS

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# Relative L2 error, derived before the first run.  A weight is exp of a score of size up to some 10 held in fp32 (an ulp of 2^-21 there:
# 5e-7 of the weight), against a sum of n weights in fp32; bf16 products are exact in fp32.  With Q B_K^T held as two bf16 terms its error
# is 2^-17 of terms of a size up to 3 (the inputs' 0.15 sqrt(128) per rank and sqrt(16..64) ranks over sqrt(d)): 2e-5 in the worst score,
# a third of that in the mean.
TOL = 2e-5


def run(d, decay, weights, stream=None):
    ws = torch.full((max(lra.lra_key_weights_workspace_bytes(d.shape, d.cache, d.batch), 256),), 255, dtype=torch.uint8, device="cuda")
    lra.lra_key_weights(d.shape, d.cache, d.b_k, d.case.n_adapters, d.batch, d.q, decay, weights, ws, stream=stream)
    torch.cuda.synchronize()
    return weights


def check(c: BatchCase, decay=0.0, stride_extra=0, **kw):
    print(c.label(), flush=True)
    x = make(c)
    d = Device(x, lra, **kw)
    T, n_max = x.seen.shape
    width = kw.get("max_seq_len", n_max) + stride_extra
    g = torch.Generator().manual_seed(9)
    old = torch.rand(T, width, generator=g)
    w = torch.full((T, width), float("nan")) if decay == 0 else old.clone()
    past = torch.arange(width) >= torch.tensor(c.lens)[:, None]
    w[past] = 7.0
    got = run(d, decay, w.cuda()).cpu()
    assert (got[past] == 7).all(), "entries behind the sequences are left alone"
    ref = torch.zeros(T, width, dtype=torch.float64)
    ref[:, :n_max] = key_weights(x)
    if decay:
        ref += decay * old.double()
    ref[past] = 7.0
    err = float((got.double() - ref)[~past].norm() / max(float(ref[~past].norm()), 1e-30)) if (~past).any() else 0.0
    assert err <= TOL, err
    if decay == 0:  # every query that sees something gives Hq in all
        hq = c.heads[0]
        per_seq = torch.tensor([sum(1 for k in range(m) if (n - m + k if c.causal else n - 1) >= 0) for n, m in zip(c.lens, c.counts)])
        assert torch.allclose(torch.where(past, 0.0, got.double()).sum(1), per_seq.double() * hq, rtol=2e-5, atol=1e-6)


@pytest.mark.parametrize("dtype,rank,heads", [(F32, 8, (4, 4, 64)), (F32, 5, (6, 2, 128)), (BF16, 16, (8, 2, 128)), (BF16, 12, (4, 2, 64)),
                                              (BF16, 8, (4, 2, 64)), (BF16, 64, (6, 3, 128)), (BF16, 24, (14, 2, 64))])
@pytest.mark.parametrize("mask", range(len(MASKS)))
def test_masks(mask, dtype, rank, heads):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, heads, rank, dtype, paged=True, seed=mask), decay=(0.0, 0.9, 1.0)[mask % 3])


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 64)])
@pytest.mark.parametrize("mask", [0, 2, 4, 5, 8, 10, 11])
@pytest.mark.parametrize("head_major", [False, True])
def test_contiguous(mask, dtype, rank, head_major):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, (8, 2, 64), rank, dtype, paged=False, head_major=head_major,
                    extra_rank_stride=8, seed=mask), stride_extra=3)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("mask", [4, 8, 10])
@pytest.mark.parametrize("kind", ["value_only", "own_l"])
def test_without_a_key_side_and_with_own_low_rank_caches(kind, mask, paged, dtype):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, (8, 2, 128), 16, dtype, paged=paged, key_side=kind != "value_only",
                    own_l=kind == "own_l", seed=mask))


@pytest.mark.parametrize("heads", [(1, 1, 64), (16, 1, 128), (3, 3, 64), (28, 4, 128), (32, 8, 128)])
def test_head_layouts(heads):
    check(BatchCase([333, 70, 1500], [4, 2, 7], False, 250, 4, heads, 16, seed=3))
    check(BatchCase([333, 70, 1500], [40, 2, 150], True, 0, 0, heads, 16, seed=4), max_seq_len=4000)


def test_long_contexts():
    check(BatchCase([9000, 20000], [3, 1], False, 0, 0, (8, 2, 128), 16, seed=1))
    check(BatchCase([9000, 20000], [40, 1], True, 5000, 4, (4, 1, 64), 32, seed=2))


@pytest.mark.parametrize("heads,rank", [((8, 4, 64), 16), ((6, 3, 128), 64), ((10, 5, 128), 32)])
@pytest.mark.parametrize("longest", [3000, 12000, 40000])  # (one, some and all of the heads to a workgroup)
def test_several_heads_of_a_workgroup(longest, heads, rank):
    check(BatchCase([1333, 2900], [70, 33], True, 0, 0, heads, rank, seed=7), max_seq_len=longest, decay=0.5)
    check(BatchCase([1333, 2900], [33, 170], True, 700, 3, heads, rank, seed=8), max_seq_len=longest)


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16)])
def test_scores_of_minus_infinity(dtype, rank):
    c = BatchCase([600], [3], False, 0, 0, (4, 2, 64), rank, dtype, key_side=False, seed=5)
    x = make(c)
    x.q.abs_().clamp_(min=0.5)
    x.k[0, :300] = -float("inf")
    x.k[0, 500:520] = -float("inf")
    got = run(Device(x, lra), 0.0, torch.empty(1, 600, device="cuda")).double().cpu()
    ref = key_weights(x)
    assert (got[0, :300] == 0).all() and float((got - ref).norm() / ref.norm()) <= TOL


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16)])
def test_equal_bits_and_replays(dtype, rank):
    c = BatchCase([700, 90, 1, 400], [60, 1, 1, 33], True, 0, 0, (8, 2, 64), rank, dtype)
    d = Device(make(c), lra)
    first = run(d, 0.0, torch.zeros(4, 700, device="cuda"))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(first, run(d, 0.0, torch.zeros(4, 700, device="cuda"), stream=side))
    w = torch.zeros(4, 700, device="cuda")
    ws = torch.empty(lra.lra_key_weights_workspace_bytes(d.shape, d.cache, d.batch), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lra.lra_key_weights(d.shape, d.cache, d.b_k, c.n_adapters, d.batch, d.q, 0.5, w, ws)
    w.zero_()
    expect = torch.zeros_like(w)
    for i in range(3):
        g.replay()
        torch.cuda.synchronize()
        run(d, 0.5, expect)
        assert torch.equal(w, expect)
        d.q.mul_(0.5)
    # nothing past the workspace's size
    big = torch.full((ws.numel() + 4096,), 171, dtype=torch.uint8, device="cuda")
    lra.lra_key_weights(d.shape, d.cache, d.b_k, c.n_adapters, d.batch, d.q, 0.5, w, big[:ws.numel()])
    torch.cuda.synchronize()
    assert (big[ws.numel():] == 171).all()
