"""lra_attn_batch against a float64 evaluation: windows and sinks, ragged chunks, pages, empty rows."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, attention, make

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
# Relative L2 error, derived before the first run.  fp32: sums of a few thousand terms in 32 bits and expf, some 1e-6, taken tenfold and
# a little more.  bf16: the output's rounding alone gives 2^-8 / sqrt(3) / 1.44 = 1.6e-3 (half a step, uniform), P and Q B_K^T rounded to
# bf16 once each as much again at most, 2.8e-3 together; the library's gate is 5e-3.
TOL = {F32: 2e-5, BF16: 5e-3}


def check(c: BatchCase, **kw):
    x = make(c)
    print(c.label(), flush=True)
    got = Device(x, lra, **kw).attend().double().cpu()
    ref = attention(x)
    assert torch.isfinite(got).all(), "rows that nothing sees leaked into the result"
    dead = ref.flatten(1).norm(dim=1) == 0
    assert (got[dead] == 0).all()
    if (~dead).any():
        rel = float((got - ref).norm() / ref.norm())
        each = float(((got - ref)[~dead].flatten(1).norm(dim=1) / ref[~dead].flatten(1).norm(dim=1)).max())
        assert max(rel, each) <= TOL[c.dtype], (rel, each)


MASKS = [  # lens, counts, causal, window, sinks
    ([1], [1], False, 0, 0),
    ([1], [1], True, 5, 3),
    ([17], [3], False, 1, 0),                      # every query sees one token
    ([130], [2], False, 64, 0),
    ([130], [2], False, 64, 4),
    ([130], [2], False, 63, 67),                   # sinks and window meet exactly
    ([130], [2], False, 64, 1000),                 # sinks reach into the window
    ([130], [2], False, 5000, 4),                  # window longer than the sequence
    ([257], [257], True, 0, 0),                    # a whole prompt
    ([300], [70], True, 33, 0),
    ([300], [70], True, 33, 5),
    ([300], [299], True, 1, 1),
    ([700, 1, 0, 33, 512], [2, 1, 0, 5, 0], False, 100, 4),
    ([700, 1, 0, 33, 512], [90, 1, 0, 33, 1], True, 100, 4),
    ([700, 40, 0, 33, 512], [90, 44, 2, 33, 7], True, 0, 0),   # chunks longer than their sequences: zeros in front
    ([200] * 9, [1, 0, 16, 3, 64, 1, 0, 5, 129], True, 48, 16),
]


@pytest.mark.parametrize("dtype,rank,heads", [(F32, 8, (4, 4, 64)), (F32, 5, (6, 2, 128)), (BF16, 16, (8, 2, 128)), (BF16, 12, (4, 2, 64)),
                                              (BF16, 8, (4, 2, 64)), (BF16, 64, (6, 3, 128)), (BF16, 32, (14, 2, 64))])
@pytest.mark.parametrize("mask", range(len(MASKS)))
def test_masks(mask, dtype, rank, heads):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, heads, rank, dtype, paged=True, seed=mask))


@pytest.mark.parametrize("variant", [1, 2])
@pytest.mark.parametrize("rank,heads", [(16, (8, 2, 128)), (64, (6, 3, 128)), (32, (14, 2, 64))])
@pytest.mark.parametrize("mask", range(len(MASKS)))
def test_masks_on_the_kernels_that_other_sizes_take(mask, rank, heads, variant):
    """1: the vector-ALU kernels, 2: the tile-walking kernel also where a sequence has few rows."""
    lens, counts, causal, window, sinks = MASKS[mask]
    old = lra.lra_set_kernel_variant(variant)
    try:
        check(BatchCase(lens, counts, causal, window, sinks, heads, rank, BF16, paged=mask % 2 == 0 or len(lens) > 1, seed=mask))
    finally:
        lra.lra_set_kernel_variant(old)


@pytest.mark.parametrize("heads,rank", [((8, 2, 128), 16), ((8, 2, 64), 32), ((4, 4, 128), 64), ((28, 4, 128), 8)])
@pytest.mark.parametrize("causal", [False, True])
def test_few_rows_on_long_contexts(causal, heads, rank):
    """Every wave of a share with several tiles, shares without keys, sequences without queries, a window that starts inside a block."""
    most = 32 // (heads[0] // heads[1])
    counts = [min(4, most), 1, 0, min(3, most)]
    check(BatchCase([5000, 37, 900, 2311], counts, causal, 0, 0, heads, rank, BF16, seed=6))
    check(BatchCase([5000, 37, 900, 2311], counts, causal, 1999, 70, heads, rank, BF16, seed=7))


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 12), (BF16, 64)])
@pytest.mark.parametrize("mask", [0, 2, 4, 5, 8, 10, 11])
@pytest.mark.parametrize("head_major", [False, True])
def test_contiguous(mask, dtype, rank, head_major):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, (8, 2, 64), rank, dtype, paged=False, head_major=head_major,
                    extra_rank_stride=8 if rank % 8 == 0 else 0, seed=mask))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("mask", [1, 4, 8, 10])
@pytest.mark.parametrize("kind", ["rope", "value_only", "own_l", "own_l_rope", "no_adapters"])
def test_key_side_and_low_rank_caches(kind, mask, paged, dtype):
    lens, counts, causal, window, sinks = MASKS[mask]
    check(BatchCase(lens, counts, causal, window, sinks, (8, 2, 128), 16, dtype, paged=paged, rope=10000.0 if "rope" in kind else 0.0,
                    key_side=kind not in ("value_only", "no_adapters"), value_side=kind != "no_adapters", own_l="own_l" in kind, seed=mask))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [(1, 1, 64), (16, 1, 128), (3, 3, 64), (28, 4, 128), (32, 8, 128)])
def test_head_layouts(heads, dtype):
    check(BatchCase([333, 70, 1500], [4, 2, 7], False, 250, 4, heads, 16, dtype, seed=3))
    check(BatchCase([333, 70, 1500], [40, 2, 150], True, 250, 4, heads, 16, dtype, seed=4))


def test_a_bound_above_the_lengths_and_one_below():
    """max_seq_len only bounds: above every length it changes nothing; a longer sequence ends there."""
    c = BatchCase([130, 40], [2, 1], False, 64, 4, paged=True)
    check(c, max_seq_len=5000)
    x = make(c)
    d = Device(x, lra, max_seq_len=130)
    whole = d.attend()
    d.lens[0] = 100000  # taken for 130, its own length (the table has that many blocks)
    assert torch.equal(whole, d.attend())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_bad_adapter_ids_stay_inside_the_table(dtype):
    c = BatchCase([130], [3], False, 64, 4, dtype=dtype)
    x = make(c)
    x.adapter[:] = torch.tensor([-5, 7, 1])
    got = Device(x, lra).attend().double().cpu()
    ref = attention(x)
    assert float((got - ref).norm() / ref.norm()) <= TOL[dtype]


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 12)])
@pytest.mark.parametrize("causal", [False, True])
def test_scores_of_minus_infinity(dtype, rank, causal):
    """A key whose every score is minus infinity has weight zero wherever it stands: the row's first tile, a whole share, its last."""
    c = BatchCase([600], [3], causal, 0, 0, (4, 2, 64), rank, dtype, key_side=False, seed=5)
    x = make(c)
    x.q.abs_().clamp_(min=0.5)
    x.k[0, :300] = -float("inf")
    x.k[0, 500:520] = -float("inf")
    got = Device(x, lra).attend().double().cpu()
    y = make(c)
    y.q, y.k = x.q, x.k.clone()
    ref = attention(y)
    assert torch.isfinite(ref).all()
    assert float((got - ref).norm() / ref.norm()) <= TOL[dtype]


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16)])
def test_equal_calls_give_equal_bits_on_any_stream_and_in_a_graph(dtype, rank):
    c = BatchCase([700, 90, 1, 400], [60, 1, 1, 33], True, 100, 4, (8, 2, 64), rank, dtype)
    d = Device(make(c), lra)
    first = d.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(first, d.attend(stream=side))
    out = torch.empty_like(first)
    ws = torch.empty(lra.lra_batch_workspace_bytes(d.shape, d.cache, d.batch), dtype=torch.uint8, device="cuda")
    call = lambda: lra.lra_attn_batch(d.shape, d.cache, d.b_k, d.b_v, c.n_adapters, d.batch, d.q, out, ws)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    q0 = d.q.clone()
    for i in range(3):
        d.q.copy_(q0 * (1 + i))  # (powers of the scale aside: other values, same tensors)
        out.fill_(float("nan"))
        ws.fill_(255)
        g.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        assert torch.equal(replayed, d.attend())


@pytest.mark.parametrize("dtype,rank,rope", [(F32, 8, 0.0), (BF16, 16, 0.0), (BF16, 8, 10000.0)])
def test_nothing_outside_the_outputs_is_written(dtype, rank, rope):
    c = BatchCase([300, 20], [70, 3], True, 33, 5, (8, 2, 64), rank, dtype, rope=rope)
    d = Device(make(c), lra)
    need = lra.lra_batch_workspace_bytes(d.shape, d.cache, d.batch)
    ws = torch.full((need + 4096,), 171, dtype=torch.uint8, device="cuda")
    arena = torch.full((d.q.shape[0] + 4, *d.q.shape[1:]), 7.0, dtype=dtype, device="cuda")
    out = arena[2:-2]
    lra.lra_attn_batch(d.shape, d.cache, d.b_k, d.b_v, c.n_adapters, d.batch, d.q, out, ws[:need])
    torch.cuda.synchronize()
    assert (ws[need:] == 171).all() and (arena[:2] == 7).all() and (arena[-2:] == 7).all()
    assert torch.equal(out, d.attend())


@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16)])
def test_key_shares_change_only_rounding(dtype, rank):
    c = BatchCase([2000, 77], [3, 1], False, 0, 0, (8, 2, 64), rank, dtype)
    d = Device(make(c), lra)
    ref = d.attend().double()
    for keys in (64, 320, 4096):
        old = lra.lra_set_decode_split_keys(keys)
        try:
            got = d.attend().double()
        finally:
            lra.lra_set_decode_split_keys(old)
        assert float((got - ref).norm() / ref.norm()) <= TOL[dtype]
