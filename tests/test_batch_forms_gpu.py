"""Forms of the batch calls that sizes, layouts and missing operands choose."""
import pytest
import torch

import paper_2602_01053_amd as lra
from tests.batch_reference import BatchCase, Device, attention, key_weights, make
from tests.test_batch_gpu import TOL, check
from tests.test_key_weights_gpu import TOL as WEIGHTS_TOL
from tests.test_key_weights_gpu import run as weigh

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("counts,causal,window", [([4, 1, 4], False, 0), ([4, 1, 4], False, 200), ([70, 1, 5], True, 0)])
def test_a_rotary_key_side_without_adapters_is_none(counts, causal, window, dtype):
    """Value-only adapters under key_rope_theta > 0: nothing is rotated, and the call is the one without, bit for bit."""
    same = dict(lens=[900, 33, 500], counts=counts, causal=causal, window=window, sinks=4 if window else 0, heads=(8, 2, 128), rank=16,
                dtype=dtype, key_side=False, seed=21)
    out = [Device(make(BatchCase(rope=theta, **same)), lra).attend() for theta in (0.0, 10000.0)]
    assert torch.equal(*out)
    check(BatchCase(rope=10000.0, **same))


@pytest.mark.parametrize("heads,rank", [((8, 2, 128), 64), ((7, 1, 128), 40), ((4, 4, 128), 32), ((8, 2, 64), 64), ((4, 2, 64), 24)])
@pytest.mark.parametrize("counts,causal,window", [([3, 1, 4], False, 0), ([3, 0, 2], False, 300), ([150, 1, 40], True, 0), ([33, 70, 5], True, 129)])
@pytest.mark.parametrize("paged", [False, True])
def test_rotated_key_sides_of_all_ranks(paged, counts, causal, window, heads, rank):
    """Several key shares of a row, each beginning in the middle of a sequence: its first angles are formed there."""
    lens = [1900, 75, 800]
    n = 3 if paged else 1
    check(BatchCase(lens[:n], counts[:n], causal, window, 5 if window else 0, heads, rank, BF16, paged=paged, rope=10000.0, seed=22))


@pytest.mark.parametrize("counts,causal", [([3], False), ([60], True)])
def test_rotated_key_sides_up_to_the_magnitudes_told(counts, causal):
    """Completed keys are held as fp16: magnitudes of 2^15, within the 65504 of the header, with queries that keep the scores at a few units.
    The keys' rounding (2^-11) adds 1e-3 to the error at most: scores of size 4 with 0.4 2^-11 in each."""
    c = BatchCase([300], counts, causal, 0, 0, (8, 2, 128), 16, BF16, rope=10000.0, seed=23, poison=False)
    x = make(c)
    x.k.clamp_(-4, 4).mul_(2 ** 13)
    x.q.mul_(2 ** -11)
    got = Device(x, lra).attend().double().cpu()
    ref = attention(x)
    assert torch.isfinite(got).all()
    assert float((got - ref).norm() / ref.norm()) <= TOL[BF16]


@pytest.mark.parametrize("counts,causal,variant", [([3, 1], False, 0), ([3, 1], False, 2), ([3, 2], True, 0), ([90, 7], True, 2)])
@pytest.mark.parametrize("heads,rank", [((8, 2, 64), 16), ((8, 2, 128), 64)])
def test_share_counts_change_only_rounding(heads, rank, counts, causal, variant):
    """Shares of a row go by the bound of the lengths: the same sequences under larger and larger ones, on the few-rows kernel and the
    tile-walking one, with shares of several tiles, of one and of none."""
    c = BatchCase([2000, 77], counts, causal, 0, 0, heads, rank, BF16, seed=24)
    x = make(c)
    ref, ref_w = attention(x), key_weights(x)
    old = lra.lra_set_kernel_variant(variant)
    sizes, sizes_w = [], []
    try:
        for bound in (2000, 3500, 12000, 60000):
            d = Device(x, lra, max_seq_len=bound)
            sizes.append(lra.lra_batch_workspace_bytes(d.shape, d.cache, d.batch))
            sizes_w.append(lra.lra_key_weights_workspace_bytes(d.shape, d.cache, d.batch))
            got = d.attend().double().cpu()
            assert float((got - ref).norm() / ref.norm()) <= TOL[BF16], bound
            w = weigh(d, 0.0, torch.zeros(2, bound, device="cuda")).double().cpu()[:, :2000]
            assert float((w - ref_w).norm() / ref_w.norm()) <= WEIGHTS_TOL, bound
    finally:
        lra.lra_set_kernel_variant(old)
    assert len(set(sizes)) >= 2 and sizes == sorted(sizes), sizes            # (at most 64 shares)
    assert len(set(sizes_w)) >= 2, sizes_w    # (at most 32; the sums of groups of heads, which go by the bound too, get fewer)


def test_shares_of_the_vector_kernels_change_only_rounding():
    """decode_split_keys reaches the vector-ALU kernels, so a bf16 call has to ask for them."""
    c = BatchCase([2000, 77], [3, 1], False, 0, 0, (8, 2, 64), 16, BF16, seed=25)
    x = make(c)
    ref = attention(x)
    sizes = set()
    old = lra.lra_set_kernel_variant(1)
    try:
        for keys in (64, 320, 4096):
            before = lra.lra_set_decode_split_keys(keys)
            try:
                d = Device(x, lra)
                sizes.add(lra.lra_batch_workspace_bytes(d.shape, d.cache, d.batch))
                got = d.attend().double().cpu()
            finally:
                lra.lra_set_decode_split_keys(before)
            assert float((got - ref).norm() / ref.norm()) <= TOL[BF16], keys
    finally:
        lra.lra_set_kernel_variant(old)
    assert len(sizes) == 3


@pytest.mark.parametrize("value", [-float("inf"), "lowest", -1e30, -1e12])
@pytest.mark.parametrize("counts,causal", [([3], False), ([90], True)])
@pytest.mark.parametrize("variant", [0, 1, 2])
@pytest.mark.parametrize("dtype,d,rank", [(F32, 64, 8), (BF16, 64, 16), (BF16, 128, 64), (BF16, 128, 12)])
def test_keys_of_no_weight(dtype, d, rank, variant, counts, causal, value):
    """Keys that nothing is to attend to, by one member of the type's lowest value or a very negative one: first tiles of a row, whole
    shares and a stretch in the middle hold no others."""
    c = BatchCase([900], counts, causal, 0, 0, (4, 2, d), rank, dtype, key_side=False, seed=26)
    x = make(c)
    x.q.abs_().clamp_(min=0.5)
    for lo, hi in ((0, 400), (600, 637)):
        x.k[0, lo:hi, :, 5] = torch.finfo(dtype).min if value == "lowest" else value
    old = lra.lra_set_kernel_variant(variant)
    try:
        dev = Device(x, lra)
        got = dev.attend().double().cpu()
        w = weigh(dev, 0.0, torch.empty(1, 900, device="cuda")).double().cpu()
    finally:
        lra.lra_set_kernel_variant(old)
    ref, ref_w = attention(x), key_weights(x)
    assert float((got - ref).norm() / ref.norm()) <= TOL[dtype]
    assert (w[0, :400] == 0).all() and float((w - ref_w).norm() / ref_w.norm()) <= WEIGHTS_TOL


@pytest.mark.parametrize("value", [-float("inf"), -1e30, "lowest"])
@pytest.mark.parametrize("counts,causal", [([3], False), ([90], True)])
@pytest.mark.parametrize("variant", [0, 1])
@pytest.mark.parametrize("dtype,rank", [(F32, 8), (BF16, 16), (BF16, 12)])
def test_rows_without_a_softmax_add_nothing(dtype, rank, variant, counts, causal, value):
    c = BatchCase([300], counts, causal, 0, 0, (4, 2, 64), rank, dtype, key_side=False, seed=27)
    x = make(c)
    x.q.abs_().clamp_(min=0.5)
    x.k[0, :, 0, 5] = torch.finfo(dtype).min if value == "lowest" else value   # one of two kv heads
    old = lra.lra_set_kernel_variant(variant)
    try:
        w = weigh(Device(x, lra), 0.0, torch.empty(1, 300, device="cuda")).double().cpu()
    finally:
        lra.lra_set_kernel_variant(old)
    x.k, x.q, x.case = x.k[:, :, 1:], x.q[:, 2:], BatchCase(**{**c.__dict__, "heads": (2, 1, 64)})  # the other head alone
    ref = key_weights(x)
    assert float((w - ref).norm() / ref.norm()) <= WEIGHTS_TOL
