"""Which kernel the batch calls take and what they need, asked of the planner compiled for the CPU (tests/batch_plan_query.cpp)."""
from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2602_01053_amd.binding import LraBatch, LraCache, LraShape, LraTuning

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FIELDS = ("few_rows", "tiles", "tile_places", "tile_per_query", "states", "n_splits", "split_keys", "launchable", "pages")
FAKE = 0x1000  # never dereferenced


@pytest.fixture(scope="module")
def planner(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no host C++ compiler")
    lib = str(tmp_path_factory.mktemp("plan") / "batch_plan_query.so")
    csrc = os.path.join(ROOT, "paper_2602_01053_amd", "csrc")
    subprocess.run([gxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    os.path.join(csrc, "lra_plan.cpp"), os.path.join(csrc, "lra_batch_plan.cpp"),
                    os.path.join(ROOT, "tests", "batch_plan_query.cpp"), "-o", lib], check=True)
    return ctypes.CDLL(lib)


def structs(hq, hkv, d, r, n, queries, *, seqs=1, causal=False, window=0, sinks=0, theta=0.0, fp32=False, variant=0, own=False):
    """The planner's arguments for a call: contiguous for one sequence, else pages; `queries` of each sequence."""
    cache = LraCache(FAKE, FAKE, FAKE, hkv * d, d, 0, 0, 0, 0, 1, 0, 0, None, FAKE, n)
    if seqs > 1:
        per = -(-n // 16)
        cache = LraCache(FAKE, FAKE, FAKE, d, 16 * d, 16 * d * hkv, 16, per, per * seqs, seqs, 0, 0, FAKE, FAKE, n)
    if own:
        cache.l_adapter_stride = n * seqs * 64
    return (LraShape(hq, hkv, d, r, int(fp32), 0.0, theta), cache,
            LraBatch(FAKE, FAKE, seqs * queries, queries, int(causal), window, sinks), LraTuning(kernel_variant=variant))


def plan(planner, *call, key_adapter=True, **kw):
    out = (ctypes.c_int32 * len(FIELDS))()
    planner.batch_plan_query(*(ctypes.byref(x) for x in structs(*call, **kw)), int(key_adapter), out)
    return dict(zip(FIELDS, out))


def need(planner, *call, **kw):
    return planner.batch_workspace_query(*(ctypes.byref(x) for x in structs(*call, **kw)))


CALLS = [dict(queries=4), dict(queries=4, window=4096, sinks=4), dict(queries=3, seqs=16, window=500), dict(queries=200, causal=True),
         dict(queries=7, seqs=5, causal=True), dict(queries=40, seqs=3), dict(queries=2, fp32=True), dict(queries=4, own=True)]


@pytest.mark.parametrize("call", CALLS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("layer", [(32, 8, 128), (28, 4, 128), (4, 4, 64)])
def test_a_rotary_key_side_without_adapters_is_planned_as_none(planner, layer, call):
    """Nothing is rotated where there is no B_K: the call takes the kernel and the shares of one without a rotary key side."""
    call = dict(call)
    queries = call.pop("queries")
    for n in (700, 33000):
        rotary = plan(planner, *layer, 16, n, queries, theta=500000.0, key_adapter=False, **call)
        plain = plan(planner, *layer, 16, n, queries, key_adapter=False, **call)
        assert rotary == plain
        # the workspace is told before it is known whether the call has a B_K
        size = need(planner, *layer, 16, n, queries, theta=500000.0, **call)
        assert size == max(rotary["pages"], plan(planner, *layer, 16, n, queries, theta=500000.0, **call)["pages"])


def test_a_rotated_key_side_at_high_ranks_has_one_workgroup_per_compute_unit(planner):
    """Key shares of batch_tiles_kernel where one workgroup fits a compute unit (d = 128, ranks above 32): full turns of 256, not of 512."""
    def workgroups(layer, r, n, queries, **kw):
        pl = plan(planner, *layer, r, n, queries, theta=500000.0, **kw)
        assert pl["tiles"] and not pl["few_rows"]
        seqs = kw.get("seqs", 1)
        tiles = pl["tile_places"] if pl["tile_per_query"] else max(-(-queries * seqs * layer[0] // layer[1] // 128), seqs)
        return tiles * layer[1] * pl["n_splits"]

    llama, qwen = (32, 8, 128), (28, 4, 128)
    assert workgroups(llama, 64, 16000, 4) == 256 and workgroups(llama, 32, 16000, 4) == 512
    assert workgroups(llama, 64, 16000, 128, causal=True) == 256
    assert workgroups(qwen, 40, 30000, 300, causal=True) == 476            # two turns: one of 204 would leave fifty units without work
    assert workgroups(llama, 64, 9000, 3, seqs=8) == 960                   # lengths that may differ: about four turns, not one of 192
    assert workgroups(llama, 64, 9000, 3, seqs=8, window=4000) == 768      # ... and hardly matter behind a window: three full ones
    assert workgroups(llama, 64, 5000, 20, seqs=4, causal=True) == 32 * 8  # one turn, more would have shares of a few tiles
    for n in (1, 64, 129, 1000, 100000):
        for queries in (1, 5, 60, 900):
            for causal in (False, True):
                pl = plan(planner, *llama, 64, n, queries, theta=500000.0, causal=causal)
                assert 1 <= pl["n_splits"] <= 64 and (pl["n_splits"] == 1 or pl["n_splits"] <= (n + queries + 127) // 64)


def weights_plan(planner, *call, **kw):
    out = (ctypes.c_int32 * 4)()
    planner.weights_plan_query(*(ctypes.byref(x) for x in structs(*call, **kw)), out)
    return dict(zip(("mfma", "n_splits", "tile_places", "sum_groups"), out))


def test_weights_statistics_fill_the_places_that_there_are(planner):
    """Three workgroups per compute unit, two at d = 128 and ranks above 32 (tests/test_batch_resources_cpu.py)."""
    assert weights_plan(planner, 32, 8, 128, 32, 18432, 100, causal=True)["n_splits"] == 768 // (4 * 8)
    assert weights_plan(planner, 32, 8, 128, 64, 18432, 100, causal=True)["n_splits"] == 512 // (4 * 8)
    assert weights_plan(planner, 8, 8, 64, 64, 18432, 400, causal=True)["n_splits"] == 768 // (4 * 8)
    assert weights_plan(planner, 32, 8, 128, 64, 8192, 4)["n_splits"] == 32


def test_the_largest_batch_of_weights_fits_the_grids(planner):
    """2^30 query rows: a grid dimension holds fewer than 2^32 threads, four to a row in the pass over the statistics."""
    fits = lambda q: (q * 16 + 63) // 64 * 256 < 1 << 32  # noqa: E731
    for queries in ((1 << 26) - 4, (1 << 26) - 3, 1 << 26):
        assert fits(queries) == (queries == (1 << 26) - 4)
        assert weights_plan(planner, 16, 1, 64, 8, 1000, queries, causal=True)["mfma"] == fits(queries)
