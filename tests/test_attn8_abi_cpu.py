"""What the 8-bit entry points refuse, before anything is launched (no GPU here), and what the binding refuses itself."""
import ctypes

import pytest
import torch

import paper_2602_01053_amd as lra
from paper_2602_01053_amd.binding import LraAdapters, LraBatch, LraCache, LraCache8, LraI8Operands, LraNewRows, LraShape

NULL, SHAPE, DTYPE, UNSUP, WS = 1, 2, 3, 4, 5
FAKE = 0x1000  # never dereferenced
REFUSED = ctypes.c_size_t(-1).value


@pytest.fixture(scope="module")
def lib():
    return lra.load_library()


def ref(x):
    return None if x is None else ctypes.byref(x)


def good():
    return (LraShape(32, 8, 128, 16, 0, 0.0),
            LraCache8(FAKE, FAKE, FAKE, FAKE, FAKE, 8 * 2048, 2048, 0, 0, 0, 512, 2000, 3, FAKE, FAKE, 8192),
            LraAdapters(FAKE, FAKE, 4), LraBatch(FAKE, FAKE, 4, 4, 0, 0, 0))


def rows():
    return LraNewRows(FAKE, FAKE, FAKE, 1024, 1024, 16, FAKE, None, 10, 4, 500000.0)


def attend(lib, sh, c, ad, b, q=FAKE, out=FAKE, ws=FAKE, ws_bytes=0):
    return lib.lra_attn_batch8(ref(sh), ref(c), ref(ad), ref(b), q, out, ws, ws_bytes, None, None)


BAD_CACHE = [("k", None, NULL), ("v", None, NULL), ("k_scale", None, NULL), ("v_scale", None, NULL), ("l", None, NULL), ("seq_lens", None, NULL),
             ("k", FAKE + 8, SHAPE), ("v", FAKE + 1, SHAPE), ("l", FAKE + 4, SHAPE), ("code", 2, DTYPE), ("code", -1, DTYPE), ("n_seqs", 0, SHAPE),
             ("n_seqs", (1 << 20) + 1, UNSUP), ("max_seq_len", 0, SHAPE), ("max_seq_len", 8193, SHAPE), ("max_seq_len", (1 << 30) + 1, UNSUP),
             ("num_blocks", 0, SHAPE), ("max_blocks_per_seq", 0, SHAPE), ("kv_head_stride", 2032, SHAPE), ("kv_head_stride", 2056, SHAPE),
             ("kv_block_stride", 1024, SHAPE), ("kv_block_stride", 16384 + 8, SHAPE), ("kv_block_stride", 1 << 41, UNSUP),
             ("scale_block_stride", 7, SHAPE), ("scale_block_stride", -1, SHAPE), ("l_row_stride", 8, SHAPE), ("l_row_stride", 20, SHAPE),
             ("l_row_stride", -16, SHAPE), ("block_table", None, SHAPE)]
BAD_SHAPE = [("dtype", 7, DTYPE), ("rank", 65, UNSUP), ("rank", 0, SHAPE), ("head_dim", 96, UNSUP), ("n_q_heads", 30, SHAPE), ("n_kv_heads", 0, SHAPE),
             ("scale", float("nan"), SHAPE), ("scale", -1.0, SHAPE), ("key_rope_theta", -1.0, SHAPE)]


@pytest.mark.parametrize("field,bad,want", BAD_CACHE + BAD_SHAPE)
def test_every_call_refuses_a_bad_cache_or_shape(lib, field, bad, want):
    sh, c, ad, b = good()
    setattr(sh if hasattr(sh, field) and field not in ("k", "v", "l") else c, field, bad)
    dst = LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 128, 2048, 16384, 16, 512, 600, 3, 0, 0, FAKE, FAKE, 8192)
    assert attend(lib, sh, c, ad, b) == want
    assert lib.lra_batch8_workspace_bytes(ref(sh), ref(c), ref(b), None) == REFUSED
    assert lib.lra_cache8_append(ref(sh), ref(c), ref(rows()), None) == want
    assert lib.lra_cache8_gather(ref(sh), ref(c), None, 0, ref(dst), None) in (want, SHAPE)


def test_attention_refuses_before_launch(lib):
    sh, c, ad, b = good()
    assert attend(lib, None, c, ad, b) == NULL and attend(lib, sh, None, ad, b) == NULL
    assert attend(lib, sh, c, None, b) == NULL and attend(lib, sh, c, ad, None) == NULL
    assert attend(lib, sh, c, ad, b, q=None) == NULL and attend(lib, sh, c, ad, b, out=None) == NULL
    assert attend(lib, sh, c, ad, b, q=FAKE + 8) == SHAPE and attend(lib, sh, c, ad, b, out=FAKE + 2) == SHAPE
    assert attend(lib, sh, c, ad, b) == WS
    assert attend(lib, sh, c, ad, b, ws=None, ws_bytes=1 << 40) == WS and attend(lib, sh, c, ad, b, ws=FAKE + 16, ws_bytes=1 << 40) == WS
    for field, bad in (("n_queries", 0), ("max_queries_per_seq", 0), ("max_queries_per_seq", 5), ("window", -1), ("sinks", -1)):
        sh, c, ad, b = good()
        setattr(b, field, bad)
        assert attend(lib, sh, c, ad, b) == SHAPE, field
    for field in ("seq_query_start", "query_adapter"):
        sh, c, ad, b = good()
        setattr(b, field, None)
        assert attend(lib, sh, c, ad, b) == NULL, field
    sh, c, ad, b = good()
    ad.n_adapters = 0
    assert attend(lib, sh, c, ad, b) == SHAPE
    sh, c, ad, b = good()
    b.n_queries = b.max_queries_per_seq = 1 << 28
    assert attend(lib, sh, c, ad, b) == UNSUP
    sh, c, ad, b = good()
    sh.key_rope_theta = 10000.0
    assert attend(lib, sh, c, ad, b) == UNSUP
    ad.b_k = None                                  # nothing is rotated then
    assert attend(lib, sh, c, ad, b) == WS


def test_one_sequence_without_a_table(lib):
    sh, c, ad, b = good()
    c.block_table, c.n_seqs, c.max_blocks_per_seq = None, 1, 0
    assert attend(lib, sh, c, ad, b) == WS
    c.num_blocks = 511                             # fewer than max_seq_len needs
    assert attend(lib, sh, c, ad, b) == SHAPE


@pytest.mark.parametrize("window,sinks", [(1, 0), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31 - 1, 0), (0, 2 ** 31 - 1)])
def test_workspace_size_of_extreme_windows(lib, window, sinks):
    for causal in (0, 1):
        sh, c, _, b = good()
        b.window, b.sinks, b.causal = window, sinks, causal
        assert 0 < lib.lra_batch8_workspace_bytes(ref(sh), ref(c), ref(b), None) < REFUSED


def test_append_refuses_before_launch(lib):
    def call(**kw):
        sh, c, _, _ = good()
        n = rows()
        for k, v in kw.items():
            setattr(n, k, v)
        return lib.lra_cache8_append(ref(sh), ref(c), ref(n), None)
    sh, c, _, _ = good()
    assert lib.lra_cache8_append(None, ref(c), ref(rows()), None) == NULL and lib.lra_cache8_append(ref(sh), None, ref(rows()), None) == NULL
    assert lib.lra_cache8_append(ref(sh), ref(c), None, None) == NULL
    for field in ("k", "v", "seq_start"):
        assert call(**{field: None}) == NULL, field
    for kw in (dict(n_new=0), dict(max_new_per_seq=0), dict(max_new_per_seq=11), dict(rope_theta=-1.0), dict(rope_theta=float("inf")),
               dict(rope_theta=float("nan")), dict(k_token_stride=1023), dict(v_token_stride=1000), dict(l_token_stride=15), dict(k_token_stride=1028),
               dict(k=FAKE + 2), dict(v=FAKE + 8), dict(l=FAKE + 1)):
        assert call(**kw) == SHAPE, kw
    assert call(k_token_stride=1 << 32) == UNSUP


def test_gather_refuses_before_launch(lib):
    def call(sh, c, dst, kept=None, ks=0):
        return lib.lra_cache8_gather(ref(sh), ref(c), kept, ks, ref(dst), None)
    page = lambda: LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 128, 2048, 16384, 16, 512, 600, 3, 0, 0, FAKE, FAKE, 8192)  # noqa: E731
    sh, c, _, _ = good()
    assert call(None, c, page()) == NULL and call(sh, None, page()) == NULL and call(sh, c, None) == NULL
    assert call(sh, c, page(), kept=FAKE, ks=8191) == SHAPE and call(sh, c, page(), kept=FAKE + 2, ks=8192) == SHAPE
    one = LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 1024, 128, 0, 0, 0, 0, 1, 0, 0, None, FAKE, 8192)
    assert call(sh, c, one) == SHAPE                                    # three sequences and one
    for field in ("k_base", "v_base", "l"):                             # into its own memory
        dst = page()
        setattr(dst, field, FAKE)
        assert call(sh, c, dst) == SHAPE, field


def test_quantize_refuses_before_launch(lib):
    def call(x=FAKE, dtype=0, xs=256, r=4, cols=256, c=FAKE, cs=256, s=FAKE):
        return lib.lra_quantize_rows(x, dtype, xs, r, cols, c, cs, s, None)
    assert call(x=None) == NULL and call(c=None) == NULL and call(s=None) == NULL and call(dtype=2) == DTYPE
    for kw in (dict(r=0), dict(cols=0), dict(xs=255), dict(cs=240), dict(x=FAKE + 2), dict(c=FAKE + 8), dict(s=FAKE + 2), dict(xs=260), dict(cs=264)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(cols=8, xs=16, cs=16), dict(cols=(1 << 17) + 16, xs=1 << 18, cs=1 << 18), dict(r=1 << 24), dict(xs=1 << 41)):
        assert call(**kw) == UNSUP, kw


def test_matmul_refuses_before_launch(lib):
    def call(y=FAKE, dtype=0, ys=64, ws=None, n_ws=0, **kw):
        ops = LraI8Operands(FAKE, FAKE, FAKE, FAKE, 256, 256, 4, 64, 256)
        for k, v in kw.items():
            setattr(ops, k, v)
        return lib.lra_matmul_i8(ref(ops), y, dtype, ys, ws, n_ws, None)
    assert lib.lra_matmul_i8(None, FAKE, 0, 64, None, 0, None) == NULL and call(y=None) == NULL and call(dtype=5) == DTYPE
    for field in ("x", "w", "x_scale", "w_scale"):
        assert call(**{field: None}) == NULL, field
    for kw in (dict(m=0), dict(n=0), dict(k=0), dict(ys=63), dict(x_stride=255), dict(w_stride=240), dict(x_stride=264), dict(x=FAKE + 8), dict(w=FAKE + 4),
               dict(y=FAKE + 2), dict(x_scale=FAKE + 1), dict(w_scale=FAKE + 2)):
        assert call(**kw) == SHAPE, kw
    for kw in (dict(k=40), dict(k=1 << 17, x_stride=1 << 17, w_stride=1 << 17), dict(m=(1 << 20) + 1), dict(n=(1 << 20) + 1, ys=1 << 21), dict(x_stride=1 << 32)):
        assert call(**kw) == UNSUP, kw
    size = lib.lra_matmul_i8_workspace_bytes
    assert size(4, 64, 40, 0) == REFUSED and size(0, 64, 256, 0) == REFUSED and size(4, 64, 256, 3) == REFUSED and size(4, 64, 256, 1) < REFUSED


def cache_tensors(code=torch.int8, dtype=torch.bfloat16):
    z = lambda *s, t: torch.zeros(*s, dtype=t)  # noqa: E731
    return dict(k=z(6, 2, 16, 64, t=code), v=z(6, 2, 64, 16, t=code), k_scale=z(6, 2, t=torch.uint8), v_scale=z(6, 2, t=torch.uint8), l=z(6, 16, 8, t=dtype),
                seq_lens=z(2, t=torch.int32), max_seq_len=40, block_table=z(2, 3, t=torch.int32))


def test_binding_describes_and_refuses_caches():
    c = lra.make_cache8(**cache_tensors())
    assert (c.kv_block_stride, c.kv_head_stride, c.scale_block_stride, c.l_row_stride, c.code, c.num_blocks, c.n_seqs) == (2048, 1024, 2, 8, 1, 6, 2)
    both = torch.zeros(6, 2, 2, 1024 + 32, dtype=torch.uint8)
    t = cache_tensors(torch.float8_e4m3fn)
    t["k"] = both[:, 0, :, :1024].unflatten(2, (16, 64)).view(torch.float8_e4m3fn)
    t["v"] = both[:, 1, :, :1024].unflatten(2, (64, 16)).view(torch.float8_e4m3fn)
    c = lra.make_cache8(**t)
    assert (c.kv_block_stride, c.kv_head_stride, c.code) == (4 * 1056, 1056, 0)
    for field, bad in (("k", torch.zeros(6, 2, 16, 64)), ("v", torch.zeros(6, 2, 16, 64, dtype=torch.int8)), ("v", torch.zeros(6, 2, 64, 16).to(torch.float8_e4m3fn)),
                       ("k", torch.zeros(6, 2, 64, 16, dtype=torch.int8).transpose(2, 3)), ("k", torch.zeros(6, 4, 16, 64, dtype=torch.int8)[:, ::2]),
                       ("k_scale", torch.zeros(6, 2)), ("v_scale", torch.zeros(6, 3, dtype=torch.uint8)), ("v_scale", torch.zeros(6, 4, dtype=torch.uint8)[:, :2]),
                       ("l", torch.zeros(6, 8, 16)), ("l", torch.zeros(6, 17, 8)[:, :16]), ("seq_lens", torch.zeros(3, dtype=torch.int32)),
                       ("seq_lens", torch.zeros(2, dtype=torch.int64)), ("block_table", torch.zeros(2, 3, dtype=torch.int64)),
                       ("block_table", torch.zeros(2, 6, dtype=torch.int32)[:, ::2]), ("block_table", None)):
        with pytest.raises(lra.LraError):
            lra.make_cache8(**dict(cache_tensors(), **{field: bad}))


def test_binding_refuses_mismatched_calls():
    c = lra.make_cache8(**cache_tensors())
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    sh = lra.make_shape(q, 2, 8)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    b = lra.make_batch(i32(0, 1, 2), i32(0, 0), 1)
    for bad in (lra.make_shape(q, 4, 8), lra.make_shape(q, 2, 16), lra.make_shape(q.float(), 2, 8)):
        with pytest.raises(lra.LraError):
            lra.lra_attn_batch8(bad, c, None, None, 1, b, q if bad.dtype == 0 else q.float(), torch.empty_like(q if bad.dtype == 0 else q.float()), None)
    k = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    l = torch.zeros(5, 8, dtype=torch.bfloat16)
    start = i32(0, 2, 5)
    for kw in (dict(k=k.float()), dict(v=k[:4]), dict(l=l[:, :4]), dict(seq_start=i32(0, 5)), dict(k=k.transpose(1, 2).contiguous().transpose(1, 2)),
               dict(positions=i32(1, 2)), dict(positions=torch.zeros(5))):
        args = dict(dict(seq_start=start, k=k, v=k, l=l, positions=None), **kw)
        with pytest.raises(lra.LraError):
            lra.lra_cache8_append(sh, c, args["seq_start"], 3, args["k"], args["v"], args["l"], 0.0, args["positions"])
    x, codes, s = torch.zeros(3, 32), torch.zeros(3, 32, dtype=torch.int8), torch.zeros(3)
    for bad in ((x[:2], codes, s), (x, codes, s[:2]), (x, codes.float(), s), (x, codes, s.double())):
        with pytest.raises(lra.LraError):
            lra.lra_quantize_rows(*bad)
    w, sw = torch.zeros(7, 32, dtype=torch.int8), torch.zeros(7)
    for bad in ((codes, s, w[:, :16], sw, torch.zeros(3, 7)), (codes, s, w, sw, torch.zeros(7, 3)), (codes, s, w, sw, torch.zeros(3, 7).double()),
                (codes, s, w, s, torch.zeros(3, 7))):
        with pytest.raises(lra.LraError):
            lra.lra_matmul_i8(*bad)


def test_header_is_c_and_the_structs_are_the_bindings(tmp_path):
    """lra_attn8.h in a C program: sizes and the last fields' places of its structs."""
    import os
    import shutil
    import subprocess

    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no host C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    source, exe = tmp_path / "sizes.c", tmp_path / "sizes"
    source.write_text('''#include <stddef.h>
#include <stdio.h>
#include "lra_attn8.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %zu\\n", sizeof(lra_cache8), offsetof(lra_cache8, max_seq_len), sizeof(lra_new_rows), offsetof(lra_new_rows, rope_theta),
         sizeof(lra_i8_operands), offsetof(lra_i8_operands, k));
  return 0;
}
''')
    build = subprocess.run([gcc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I", os.path.join(root, "include"), str(source), "-o", str(exe)],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    got = [int(v) for v in subprocess.run([str(exe)], capture_output=True, text=True, check=True, env=dict(os.environ, LD_PRELOAD="")).stdout.split()]
    assert got == [ctypes.sizeof(LraCache8), LraCache8.max_seq_len.offset, ctypes.sizeof(LraNewRows), LraNewRows.rope_theta.offset,
                   ctypes.sizeof(LraI8Operands), LraI8Operands.k.offset]


def test_gather_of_kept_rows_with_the_rotary_key_side(lib):
    """A row's adapter part is rotated by its index: rows that move are refused, as lra_cache_gather refuses them."""
    sh, c, _, _ = good()
    sh.key_rope_theta = 10000.0
    page = LraCache(2 * FAKE, 2 * FAKE, 2 * FAKE, 128, 2048, 16384, 16, 512, 600, 3, 0, 0, FAKE, FAKE, 8192)
    assert lib.lra_cache8_gather(ref(sh), ref(c), FAKE, 8192, ref(page), None) == UNSUP
    assert lib.lra_cache8_gather(ref(sh), ref(c), FAKE, 8191, ref(page), None) == SHAPE
    other = LraCache(3 * FAKE, 3 * FAKE, 3 * FAKE, 128, 2048, 16384, 16, 512, 600, 3, 0, 0, FAKE, FAKE, 8192)
    assert lib.lra_cache_gather(ref(sh), ref(page), 1, FAKE, 8192, ref(other), None, 0, None, 0, None) == UNSUP


def test_sizes_at_the_documented_limits(lib):
    size = lib.lra_matmul_i8_workspace_bytes
    assert size(1 << 20, 1 << 20, (1 << 17) - 16, 0) < REFUSED
    for m, n, k in (((1 << 20) + 1, 16, 16), (16, (1 << 20) + 1, 16), (16, 16, 1 << 17)):
        assert size(m, n, k, 0) == REFUSED
    far = (1 << 31) + 16
    for field in ("x_stride", "w_stride"):
        ops = LraI8Operands(FAKE, FAKE, FAKE, FAKE, 256, 256, 4, 64, 256)
        setattr(ops, field, far)
        assert lib.lra_matmul_i8(ref(ops), FAKE, 0, 64, None, 0, None) == UNSUP, field
    ops = LraI8Operands(FAKE, FAKE, FAKE, FAKE, 256, 256, 4, 64, 256)
    assert lib.lra_matmul_i8(ref(ops), FAKE, 0, far, None, 0, None) == UNSUP
    assert lib.lra_quantize_rows(FAKE, 0, 256, 4, 256, FAKE, (1 << 40) + 16, FAKE, None) == UNSUP
    sh, c, ad, b = good()
    c.scale_block_stride = far
    assert lib.lra_batch8_workspace_bytes(ref(sh), ref(c), ref(b), None) == REFUSED
    for field in ("k_token_stride", "v_token_stride", "l_token_stride"):
        sh, c, _, _ = good()
        new = rows()
        setattr(new, field, far)
        assert lib.lra_cache8_append(ref(sh), ref(c), ref(new), None) == UNSUP, field


def test_binding_takes_a_cache_of_one_block():
    """Strides of a dimension of one mean nothing: scales and L rows of one block cut from wider tensors."""
    one = dict(k=torch.zeros(1, 2, 16, 64, dtype=torch.int8), v=torch.zeros(1, 2, 64, 16, dtype=torch.int8), k_scale=torch.zeros(1, 2, dtype=torch.uint8),
               v_scale=torch.zeros(1, 6, dtype=torch.uint8)[:, 2:4], l=torch.zeros(1, 40, 8, dtype=torch.bfloat16)[:, 16:32], seq_lens=torch.zeros(1, dtype=torch.int32),
               max_seq_len=16)
    c = lra.make_cache8(**one)
    assert (c.num_blocks, c.scale_block_stride, c.l_row_stride) == (1, 2, 8)
    two = {n: torch.cat((t, t)) if n in ("k", "v", "k_scale") else t for n, t in one.items()}
    two.update(v_scale=torch.zeros(2, 6, dtype=torch.uint8)[:, 2:4], l=torch.zeros(2, 16, 8, dtype=torch.bfloat16))
    with pytest.raises(lra.LraError):
        lra.make_cache8(**two)
    two.update(v_scale=torch.zeros(2, 2, dtype=torch.uint8), l=torch.zeros(2, 40, 8, dtype=torch.bfloat16)[:, 16:32])
    with pytest.raises(lra.LraError):
        lra.make_cache8(**two)
