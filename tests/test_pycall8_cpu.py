"""The 8-bit calls through the CPython module and by ctypes: every argument arrives where the header says, and both refuse the same
tensors before the GPU is asked for (there is none here).  The C functions are replaced by callbacks that note what they get."""
import ctypes

import pytest
import torch

import paper_2602_01053_amd as lra
from paper_2602_01053_amd import binding as B

vp, i32, i64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64
P = ctypes.POINTER
STREAM = type("S", (), {"cuda_stream": 77})()


@pytest.fixture(params=["module", "ctypes"])
def noted(request, monkeypatch):
    lib = lra.load_library()
    calls = []

    def note(name, types, show):
        return ctypes.CFUNCTYPE(ctypes.c_int, *types)(lambda *a: calls.append((name, show(*a))) or 0)

    f = {
        "quantize": note("quantize", [vp, i32, i64, i32, i32, vp, i64, vp, vp], lambda *a: a),
        "matmul": note("matmul", [P(B.LraI8Operands), vp, i32, i64, vp, ctypes.c_size_t, vp],
                       lambda o, *a: tuple(getattr(o[0], n) for n, _ in B.LraI8Operands._fields_) + a),
        "append": note("append", [P(B.LraShape), P(B.LraCache8), P(B.LraNewRows), vp],
                       lambda s, c, r, st: (s[0].rank, c[0].n_seqs) + tuple(getattr(r[0], n) for n, _ in B.LraNewRows._fields_) + (st,)),
        "gather": note("gather", [P(B.LraShape), P(B.LraCache8), vp, i64, P(B.LraCache), vp], lambda s, c, k, ks, d, st: (k, ks, d[0].max_seq_len, st)),
        "attend": note("attend", [P(B.LraShape), P(B.LraCache8), P(B.LraAdapters), P(B.LraBatch), vp, vp, vp, ctypes.c_size_t, vp, vp],
                       lambda s, c, ad, b, *a: (ad[0].b_k, ad[0].b_v, ad[0].n_adapters, b[0].n_queries) + a),
    }
    if request.param == "ctypes":
        fake = type("Lib", (), {"lra_quantize_rows": f["quantize"], "lra_matmul_i8": f["matmul"], "lra_cache8_append": f["append"],
                                "lra_cache8_gather": f["gather"], "lra_attn_batch8": f["attend"]})
        fake = type("Lib", (), {k: staticmethod(v) for k, v in vars(fake).items() if k.startswith("lra_")})
        monkeypatch.setattr(B, "_calls8", B._CtypesCalls8(fake))
        yield calls
        return
    mod = B._entry_points8()
    if isinstance(mod, B._CtypesCalls8):
        pytest.skip("no headers to build the module with")
    mod.bind8(*[ctypes.cast(f[n], vp).value for n in ("quantize", "matmul", "append", "gather", "attend")], B.LraCache8, B.LraBatch,
              torch.bfloat16, torch.float32, torch.int8, torch.int32)
    yield calls
    B._lib = None
    lra.load_library()
    assert lib is not None


def cache():
    z = lambda *s, t: torch.zeros(*s, dtype=t)  # noqa: E731
    return lra.make_cache8(z(6, 2, 16, 64, t=torch.int8), z(6, 2, 64, 16, t=torch.int8), z(6, 2, t=torch.uint8), z(6, 2, t=torch.uint8),
                           z(6, 16, 8, t=torch.bfloat16), z(2, t=torch.int32), 40, z(2, 3, t=torch.int32))


def test_arguments_arrive(noted):
    p = lambda t: t.data_ptr()  # noqa: E731
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    x, codes, s = torch.zeros(3, 48)[:, :32], torch.zeros(3, 64, dtype=torch.int8)[:, :32], torch.zeros(3)
    lra.lra_quantize_rows(x, codes, s, stream=STREAM)
    lra.lra_quantize_rows(x[:1].bfloat16(), codes[:1], s[:1], stream=STREAM)
    w, sw, y, ws = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(7), torch.zeros(3, 9)[:, :7], torch.zeros(512, dtype=torch.uint8)
    lra.lra_matmul_i8(codes, s, w, sw, y, ws, stream=STREAM)
    c = cache()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    shape, out = lra.make_shape(q, 2, 8), torch.zeros_like(q)
    new = torch.zeros(5, 2 * 128 + 8, dtype=torch.bfloat16)
    k, v, l = new[:, :128].view(5, 2, 64), new[:, 128:256].view(5, 2, 64), new[:, 256:]
    start, pos = i(0, 2, 5), i(0, 1, 2, 3, 4)
    lra.lra_cache8_append(shape, c, start, 3, k, v, l, 10000, pos, stream=STREAM)
    lra.lra_cache8_append(shape, c, i(0, 0, 1), 1, k[:1], v[:1], None, stream=STREAM)
    dst = lra.make_cache(torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 16, 8).bfloat16(), i(20, 9), 32,
                         torch.zeros(2, 2, dtype=torch.int32))
    kept = torch.zeros(2, 50, dtype=torch.int32)[:, :33]
    lra.lra_cache8_gather(shape, c, dst, kept, stream=STREAM)
    lra.lra_cache8_gather(shape, c, dst, stream=STREAM)
    b = lra.make_batch(i(0, 1, 2), i(0, 0), 1)
    bk = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    lra.lra_attn_batch8(shape, c, None, bk, 3, b, q, out, ws, stream=STREAM)
    tun = ctypes.addressof(B._tuning)
    assert [n for n, _ in noted] == ["quantize", "quantize", "matmul", "append", "append", "gather", "gather", "attend"]
    a = [v for _, v in noted]
    assert a[0] == (p(x), 1, 48, 3, 32, p(codes), 64, p(s), 77)
    assert a[1][1:5] == (0, 32, 1, 32) and a[1][6] == 32               # one row: its own length apart
    assert a[2] == (p(codes), p(w), p(s), p(sw), 64, 32, 3, 7, 32, p(y), 1, 9, p(ws), 512, 77)
    assert a[3][:5] == (8, 2, p(k), p(v), p(l)) and a[3][5:8] == (264, 264, 264) and a[3][8:] == (p(start), p(pos), 5, 3, 10000.0, 77)
    assert a[4][2:5] == (p(k), p(v), None) and a[4][5:8] == (128, 128, 0) and a[4][9:] == (None, 1, 1, 0.0, 77)
    assert a[5] == (p(kept), 50, 32, 77) and a[6] == (None, 0, 32, 77)
    assert a[7] == (None, p(bk), 3, 2, p(q), p(out), p(ws), 512, tun, 77)


def test_what_is_refused(noted):
    c = cache()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    sh = lra.make_shape(q, 2, 8)
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    b = lra.make_batch(i(0, 1, 2), i(0, 0), 1)
    for bad_q, bad_out in ((q[:1], q), (q, q.float()), (q.transpose(0, 1).contiguous().transpose(0, 1), q), (q.view(2, 256), q)):
        with pytest.raises(lra.LraError):
            lra.lra_attn_batch8(sh, c, None, None, 1, b, bad_q, bad_out, None)
    with pytest.raises(lra.LraError):
        lra.lra_attn_batch8(lra.make_shape(q, 4, 8), c, None, None, 1, b, q, q, None)
    k, l, start = torch.zeros(5, 2, 64, dtype=torch.bfloat16), torch.zeros(5, 8, dtype=torch.bfloat16), i(0, 2, 5)
    for kw in (dict(k=k.float()), dict(v=k[:4]), dict(l=l[:, :4]), dict(seq_start=i(0, 5)), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)),
               dict(positions=i(1, 2)), dict(positions=torch.zeros(5)), dict(seq_start=torch.zeros(6, dtype=torch.int32)[::2])):
        args = dict(dict(seq_start=start, k=k, v=k, l=l, positions=None), **kw)
        with pytest.raises(lra.LraError):
            lra.lra_cache8_append(sh, c, args["seq_start"], 3, args["k"], args["v"], args["l"], 0.0, args["positions"])
    dst = lra.make_cache(torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 16, 8).bfloat16(), i(20, 9), 32,
                         torch.zeros(2, 2, dtype=torch.int32))
    for kept in (torch.zeros(2, 31, dtype=torch.int32), torch.zeros(1, 40, dtype=torch.int32), torch.zeros(2, 40), torch.zeros(2, 80, dtype=torch.int32)[:, ::2]):
        with pytest.raises(lra.LraError):
            lra.lra_cache8_gather(sh, c, dst, kept)
    x, codes, s = torch.zeros(3, 32), torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3)
    for bad in ((x[:2], codes, s), (x, codes, s[:2]), (x, codes.float(), s), (x, codes, s.double()), (x.double(), codes, s), (x, codes, torch.zeros(6)[::2])):
        with pytest.raises(lra.LraError):
            lra.lra_quantize_rows(*bad)
    w, sw = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(7)
    for bad in ((codes, s, w[:, :16], sw, torch.zeros(3, 7)), (codes, s, w, sw, torch.zeros(7, 3)), (codes, s, w, sw, torch.zeros(3, 7).double()),
                (codes, s, w, s, torch.zeros(3, 7)), (codes, s, w, sw, torch.zeros(3, 14)[:, ::2])):
        with pytest.raises(lra.LraError):
            lra.lra_matmul_i8(*bad)
    for bad in (dict(q=None), dict(shape=None), dict(batch=c)):
        args = dict(dict(shape=sh, cache=c, b_k=None, b_v=None, n_adapters=1, batch=b, q=q, out=q, workspace=None), **bad)
        with pytest.raises((TypeError, AttributeError, ctypes.ArgumentError)):
            lra.lra_attn_batch8(**args)
    assert not noted


def test_rows_are_read_back_into_what_has_room_for_them(noted):
    """A cache of fewer kv heads, of another head dimension or type, or of too small a rank would be written behind its rows."""
    c, q = cache(), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    sh = lra.make_shape(q, 2, 8)
    lens, table = torch.zeros(2, dtype=torch.int32), torch.zeros(2, 2, dtype=torch.int32)

    def dst(heads=2, d=64, rank=8, kv=torch.bfloat16, v=None, low=torch.bfloat16):
        return lra.make_cache(torch.zeros(4, heads, 16, d, dtype=kv), torch.zeros(4, heads, 16, d, dtype=v or kv), torch.zeros(4, 16, rank, dtype=low), lens, 32, table)

    for bad in (dict(heads=1), dict(heads=3), dict(d=32), dict(d=128), dict(rank=4), dict(kv=torch.float32), dict(low=torch.float32), dict(v=torch.float16),
                dict(kv=torch.float16, low=torch.float16), dict(kv=torch.float32, low=torch.float32)):
        with pytest.raises(lra.LraError):
            lra.lra_cache8_gather(sh, c, dst(**bad), stream=STREAM)
    one = torch.zeros(1, dtype=torch.int32)
    flat = lra.make_cache(torch.zeros(32, 1, 64).bfloat16(), torch.zeros(32, 1, 64).bfloat16(), torch.zeros(32, 8).bfloat16(), one, 32)
    with pytest.raises(lra.LraError):
        lra.lra_cache8_gather(sh, c, flat, stream=STREAM)
    assert not noted
    lra.lra_cache8_gather(sh, c, dst(), stream=STREAM)
    lra.lra_cache8_gather(sh, c, dst(rank=16), stream=STREAM)          # the first ranks of wider rows
    flat = lra.make_cache(torch.zeros(32, 2, 64).bfloat16(), torch.zeros(32, 2, 64).bfloat16(), torch.zeros(32, 8).bfloat16(), one, 32)
    lra.lra_cache8_gather(sh, c, flat, stream=STREAM)
    by_hand = B.LraCache(1 << 12, 1 << 12, 1 << 12, 64, 1024, 2048, 16, 2, 4, 2, 8, 0, 1 << 12, 1 << 12, 32)
    lra.lra_cache8_gather(sh, c, by_hand, stream=STREAM)
    assert [n for n, _ in noted] == ["gather"] * 4


def test_a_batch_has_the_sequences_of_its_cache(noted):
    """Two sequences in the cache: a start vector of one would be read behind its end, one of three mean other queries."""
    c, q = cache(), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    sh = lra.make_shape(q, 2, 8)
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    for start in (i(0, 2), i(0, 1, 2, 2), i(0)):
        with pytest.raises(lra.LraError):
            lra.lra_attn_batch8(sh, c, None, None, 1, lra.make_batch(start, i(0, 0), 1), q, torch.empty_like(q), None, stream=STREAM)
    assert not noted
    lra.lra_attn_batch8(sh, c, None, None, 1, lra.make_batch(i(0, 1, 2), i(0, 0), 1), q, torch.empty_like(q), None, stream=STREAM)
    lra.lra_attn_batch8(sh, c, None, None, 1, B.LraBatch(1 << 12, 1 << 12, 2, 1, 0, 0, 0), q, torch.empty_like(q), None, stream=STREAM)
    assert [n for n, _ in noted] == ["attend"] * 2


def test_adapters_are_as_large_as_they_are_said_to_be(noted):
    """B_K and B_V of fewer adapters, of another type or with gaps would be read behind their end."""
    c, q = cache(), torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    sh = lra.make_shape(q, 2, 8)
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    batch = lra.make_batch(i(0, 1, 2), i(0, 0), 1)
    call = lambda b_k, b_v, n=3: lra.lra_attn_batch8(sh, c, b_k, b_v, n, batch, q, torch.empty_like(q), None, stream=STREAM)  # noqa: E731
    good = torch.zeros(3, 8, 128, dtype=torch.bfloat16)
    for bad in (good[:2], good[:, :7].contiguous(), good.float(), good.half(), good[:, :, ::2], torch.zeros(3, 16, 128, dtype=torch.bfloat16)[:, :8],
                good.transpose(1, 2), good.view(1, 1, 3, 8, 128)):
        for args in ((bad, good), (good, bad), (None, bad), (bad, None)):
            with pytest.raises(lra.LraError):
                call(*args)
    with pytest.raises(lra.LraError):
        call(good, good, 4)
    assert not noted
    call(good, good)
    call(good.view(3, 8, 2, 64), good[:2], 2)
    call(None, torch.zeros(5, 8, 128, dtype=torch.bfloat16)[1:4])
    assert [n for n, _ in noted] == ["attend"] * 3
