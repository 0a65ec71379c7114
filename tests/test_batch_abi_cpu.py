"""What the batch entry points refuse, before anything is launched (no GPU here)."""
import ctypes

import pytest
import torch

import paper_2602_01053_amd as lra
from paper_2602_01053_amd.binding import LraAdapters, LraBatch, LraCache, LraShape

NULL, SHAPE, DTYPE, UNSUP, WS = 1, 2, 3, 4, 5
FAKE = 0x1000  # never dereferenced


@pytest.fixture(scope="module")
def lib():
    return lra.load_library()


def good():
    return (LraShape(32, 8, 128, 16, 0, 0.0), LraCache(FAKE, FAKE, FAKE, 1024, 128, 0, 0, 0, 0, 1, 0, 0, None, FAKE, 8192),
            LraAdapters(FAKE, FAKE, 4), LraBatch(FAKE, FAKE, 4, 4, 0, 0, 0))


def attend(lib, sh, c, ad, b, q=FAKE, out=FAKE, ws=FAKE, ws_bytes=0):
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return lib.lra_attn_batch(ref(sh), ref(c), ref(ad), ref(b), q, out, ws, ws_bytes, None, None)


def test_attention_refuses_before_launch(lib):
    sh, c, ad, b = good()
    assert attend(lib, None, c, ad, b) == NULL and attend(lib, sh, None, ad, b) == NULL
    assert attend(lib, sh, c, None, b) == NULL and attend(lib, sh, c, ad, None) == NULL
    assert attend(lib, sh, c, ad, b, q=None) == NULL and attend(lib, sh, c, ad, b, out=None) == NULL
    assert attend(lib, sh, c, ad, b, q=FAKE + 8) == SHAPE and attend(lib, sh, c, ad, b, out=FAKE + 2) == SHAPE
    assert attend(lib, sh, c, ad, b) == WS                               # too small
    assert attend(lib, sh, c, ad, b, ws=None, ws_bytes=1 << 40) == WS
    assert attend(lib, sh, c, ad, b, ws=FAKE + 16, ws_bytes=1 << 40) == WS
    for field, bad in (("n_queries", 0), ("n_queries", -3), ("max_queries_per_seq", 0), ("max_queries_per_seq", 5), ("window", -1),
                       ("sinks", -1)):
        sh, c, ad, b = good()
        setattr(b, field, bad)
        assert attend(lib, sh, c, ad, b) == SHAPE, field
    for field in ("seq_query_start", "query_adapter"):
        sh, c, ad, b = good()
        setattr(b, field, None)
        assert attend(lib, sh, c, ad, b) == NULL, field
    for field, bad, want in (("dtype", 7, DTYPE), ("rank", 65, UNSUP), ("head_dim", 96, UNSUP), ("n_q_heads", 30, SHAPE),
                             ("key_rope_theta", -1.0, SHAPE), ("scale", float("nan"), SHAPE)):
        sh, c, ad, b = good()
        setattr(sh, field, bad)
        assert attend(lib, sh, c, ad, b) == want, field
    sh, c, ad, b = good()
    ad.n_adapters = 0
    assert attend(lib, sh, c, ad, b) == SHAPE
    sh, c, ad, b = good()
    b.n_queries, b.max_queries_per_seq = 1 << 28, 1 << 28
    assert attend(lib, sh, c, ad, b) == UNSUP


def test_workspace_size_says_what_is_refused(lib):
    refused = ctypes.c_size_t(-1).value
    size = lambda sh, c, b: lib.lra_batch_workspace_bytes(ctypes.byref(sh), ctypes.byref(c), ctypes.byref(b), None)  # noqa: E731
    sh, c, _, b = good()
    assert 0 < size(sh, c, b) < refused
    b.window = -1
    assert size(sh, c, b) == refused
    sh, c, _, b = good()
    sh.rank = 65
    assert size(sh, c, b) == refused
    for window, sinks in ((1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1)):  # sums stay in range
        sh, c, _, b = good()
        b.window, b.sinks, b.causal = window, sinks, 1
        assert 0 < size(sh, c, b) < refused


def test_binding_refuses_what_the_library_cannot_see():
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    with pytest.raises(lra.LraError):
        lra.make_batch(i32(0, 2).long(), i32(0, 1), 2)
    with pytest.raises(lra.LraError):
        lra.make_batch(i32(0, 2), torch.zeros(4, dtype=torch.int32)[::2], 2)
    batch = lra.make_batch(i32(0, 2), i32(0, 1), 2, window=8, sinks=1)
    assert (batch.n_queries, batch.window, batch.sinks, batch.causal) == (2, 8, 1, 0)
    q = torch.zeros(2, 4, 64)
    sh = lra.make_shape(q, 2, 8)
    _, c, _, _ = good()
    for bad_q, bad_out in ((q[:1], q), (q, q.bfloat16()), (q.transpose(0, 1).contiguous().transpose(0, 1), q)):
        with pytest.raises(lra.LraError):
            lra.lra_attn_batch(sh, c, None, None, 1, batch, bad_q, bad_out, None)


def weigh(lib, sh, c, ad, b, q=FAKE, decay=1.0, w=FAKE, stride=8192, ws=FAKE, ws_bytes=0):
    ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return lib.lra_key_weights(ref(sh), ref(c), ref(ad), ref(b), q, decay, w, stride, ws, ws_bytes, None, None)


def test_key_weights_refuse_before_launch(lib):
    sh, c, ad, b = good()
    assert weigh(lib, None, c, ad, b) == NULL and weigh(lib, sh, c, None, b) == NULL and weigh(lib, sh, c, ad, None) == NULL
    assert weigh(lib, sh, c, ad, b, q=None) == NULL and weigh(lib, sh, c, ad, b, w=None) == NULL
    assert weigh(lib, sh, c, ad, b) == WS
    assert weigh(lib, sh, c, ad, b, stride=8191) == SHAPE and weigh(lib, sh, c, ad, b, w=FAKE + 2) == SHAPE
    for decay in (float("nan"), float("inf")):
        assert weigh(lib, sh, c, ad, b, decay=decay) == SHAPE
    sh.key_rope_theta = 10000.0
    assert weigh(lib, sh, c, ad, b) == UNSUP
    ad.b_k = None                                  # nothing is rotated then
    assert weigh(lib, sh, c, ad, b) == WS
    sh, c, ad, b = good()
    b.n_queries = b.max_queries_per_seq = (1 << 25) + 1  # more than 2^30 rows
    assert weigh(lib, sh, c, ad, b, ws_bytes=1 << 50) == UNSUP
    assert lib.lra_key_weights_workspace_bytes(ctypes.byref(sh), ctypes.byref(c), ctypes.byref(b), None) == ctypes.c_size_t(-1).value


def test_eviction_refuses_before_launch(lib):
    def select(c, w=FAKE, stride=8192, budget=100, sinks=4, recent=10, kept=FAKE, ks=100, new=FAKE):
        return lib.lra_evict_select(None if c is None else ctypes.byref(c), w, stride, budget, sinks, recent, kept, ks, new, None)
    _, c, _, _ = good()
    assert select(None) == NULL and select(c, w=None) == NULL and select(c, kept=None) == NULL and select(c, new=None) == NULL
    for bad in (dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=95), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1), dict(stride=8191),
                dict(ks=99), dict(w=FAKE + 1), dict(kept=FAKE + 2), dict(new=FAKE + 3)):
        assert select(c, **bad) == SHAPE, bad
    c.max_seq_len = (1 << 30) + 1
    assert select(c, stride=1 << 31) == UNSUP
    c.max_seq_len = 0
    assert select(c) == SHAPE


def test_gather_refuses_before_launch(lib):
    def gather(sh, src, dst, n=1, kept=FAKE, ks=4096, w=None, wst=0, w2=None, w2st=0):
        ref = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
        return lib.lra_cache_gather(ref(sh), ref(src), n, kept, ks, ref(dst), w, wst, w2, w2st, None)

    def two():
        sh, src, _, _ = good()
        return sh, src, LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 1024, 128, 0, 0, 0, 0, 1, 0, 0, None, FAKE, 4096)
    sh, src, dst = two()
    assert gather(None, src, dst) == NULL and gather(sh, None, dst) == NULL and gather(sh, src, None) == NULL
    assert gather(sh, src, dst, kept=None) == NULL and gather(sh, src, dst, w=FAKE) == NULL and gather(sh, src, dst, w2=FAKE) == NULL
    assert gather(sh, src, dst, ks=4095) == SHAPE and gather(sh, src, dst, n=0) == SHAPE and gather(sh, src, dst, n=2) == SHAPE
    assert gather(sh, src, dst, w=FAKE, wst=8191, w2=FAKE, w2st=4096) == SHAPE
    assert gather(sh, src, dst, w=FAKE, wst=8192, w2=FAKE, w2st=4095) == SHAPE
    assert gather(sh, src, src, ks=8192) == SHAPE                       # in place
    for field in ("k_base", "v_base", "l"):
        sh, src, dst = two()
        setattr(dst, field, FAKE)
        assert gather(sh, src, dst) == SHAPE, field
    sh, src, dst = two()
    sh.key_rope_theta = 10000.0
    assert gather(sh, src, dst) == UNSUP
    page = lambda table: LraCache(FAKE, FAKE, FAKE, 128, 2048, 16384, 16, 512, 600, 3, 0, 0, table, FAKE, 8192)  # noqa: E731
    sh, src, dst = two()
    assert gather(sh, page(FAKE), dst) == SHAPE                         # three sequences and one
    assert gather(sh, page(FAKE), page(FAKE), ks=8192) == SHAPE         # one table over one pool


def test_gather_refuses_weights_in_place(lib):
    sh, src, _, _ = good()
    dst = LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 1024, 128, 0, 0, 0, 0, 1, 0, 0, None, FAKE, 4096)
    assert lib.lra_cache_gather(ctypes.byref(sh), ctypes.byref(src), 1, FAKE, 4096, ctypes.byref(dst), FAKE, 8192, FAKE, 8192, None) == SHAPE


def test_longest_sequences(lib):
    """Beyond 2^27 tokens a grid would hold 2^32 threads."""
    ref = ctypes.byref
    sh, c, ad, b = good()
    for n, status in ((1 << 27, WS), ((1 << 27) + 1, UNSUP)):
        c.max_seq_len = n
        assert weigh(lib, sh, c, ad, b, stride=n) == status
    dst = LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 1024, 128, 0, 0, 0, 0, 1, 0, 0, None, FAKE, (1 << 27) + 1)
    assert lib.lra_cache_gather(ref(sh), ref(c), 1, FAKE, 1 << 30, ref(dst), None, 0, None, 0, None) == UNSUP
