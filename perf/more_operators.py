"""The layer path in 8 bits: projections of new tokens, a cache of 8-bit codes, and attention over it.

Operators of a serving loop, each through the public entry points:
  project  hidden states quantized token by token, and their product with 8-bit weights
  append   keys and values of new tokens, rotated and quantized into a cache that holds 8-bit codes with one scale per
           16-token block and head; then the rows of the blocks that were touched, as values (what the codes stand for)
  gather   rows of such a cache as values, in a cache of 16 or 32 bits
  attend   a batch of sequences, each with its own queries, over such a cache and the low-rank rows beside it

Codes are e4m3 or signed integers, scales powers of two held as biased exponents.  Sizes are those of the layers below;
lengths follow from the case alone (`length_seed`), values from the seed.
"""
from __future__ import annotations

import math
import random

import torch

own = False

ROPE_THETA = 500000.0
BLOCK = 16

# Attention layers: query heads, kv heads, head dimension, model dimension.
LAYERS = {
    "llama3_8b": (32, 8, 128, 4096),
    "qwen25_7b": (28, 4, 128, 3584),
    "tiny": (4, 4, 64, 256),
}


def _case(name, op, layer, n, *, rank=16, seqs=1, shortest=0, queries=1, causal=False, window=0, sinks=0, key_side=True,
          code="e4m3", dtype="bf16", rope=True, kept=0, features="kvl", length_seed=0):
    """n: cached tokens of the longest sequence, the new ones included (project: the tokens); queries: the most a sequence has
    (agents that decode one token each, or with `causal` the new tokens of one agent; append: the most new tokens).
    kept: rows that a gather takes; features: the projections that share a product (q, kvl or qkvl)."""
    c = {"op": op, "layer": layer, "n": n, "rank": rank, "seqs": seqs, "shortest": shortest or n, "queries": queries,
         "causal": causal, "window": window, "sinks": sinks, "key_side": key_side, "code": code, "dtype": dtype, "rope": rope,
         "kept": kept, "features": features, "length_seed": length_seed}
    return dict(c, name=name) if name else c


def listed():
    return [
        # The smallest attention call: two agents of a small fp32 model behind a short window, all latency.
        _case("attend8_fp32_tiny", "attend", "tiny", 700, rank=8, queries=2, window=256, sinks=4, code="int8", dtype="fp32"),
        # A decode step of four agents on one trajectory of 32k tokens.
        _case("attend8_a4_n32768", "attend", "llama3_8b", 32768, queries=4),
        # Serving: sixteen trajectories of 4k to 64k tokens, four agents each.
        _case("attend8_batch_int8", "attend", "qwen25_7b", 65536, rank=32, seqs=16, shortest=4096, queries=4, code="int8",
              length_seed=11),
        # Continuous batching: some sequences decode one token, others take a chunk of their prompt.
        _case("attend8_mixed_chunks", "attend", "llama3_8b", 8000, seqs=12, shortest=500, queries=256, causal=True, length_seed=3),
        # Two long prompts advance by a chunk of up to 2048 tokens.
        _case("attend8_chunk_2048", "attend", "llama3_8b", 18432, seqs=2, shortest=8000, queries=2048, causal=True, length_seed=7),
        # A decode step's tokens enter the caches of 64 sequences, each into a block that is partly full.
        _case("append8_tokens_64", "append", "llama3_8b", 9000, seqs=64, shortest=1000, queries=1, length_seed=5),
        # Tools' answers of a few hundred tokens.
        _case("append8_answers_int8", "append", "qwen25_7b", 5333, rank=32, seqs=12, shortest=700, queries=333, code="int8", length_seed=9),
        # Four prompts of up to 4096 tokens.
        _case("append8_prompts", "append", "llama3_8b", 4096, seqs=4, shortest=1500, queries=4096, length_seed=2),
        # What an eviction keeps of one long context, as 16-bit rows.
        _case("gather8_kept_4096", "gather", "llama3_8b", 16384, kept=4096),
        # Keys, values and low-rank rows of four new tokens: all weights are read for them.
        _case("project8_m4", "project", "llama3_8b", 4),
        # The same of a tool's answer.
        _case("project8_m333", "project", "qwen25_7b", 333, rank=32),
        # Queries too, for a long prompt.
        _case("project8_m8192_qkvl", "project", "llama3_8b", 8192, features="qkvl"),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def _draw_once(rng):
    op = rng.choice(("attend", "attend", "attend", "append", "append", "gather", "project", "project"))
    layer = rng.choice(("llama3_8b", "llama3_8b", "qwen25_7b", "tiny"))
    rank = rng.choice((8, 16, 16, 24, 32, 64))
    fp32 = layer == "tiny" and rng.random() < 0.5
    if fp32:
        rank = rng.choice((8, 12, 16))
    same = dict(rank=rank, dtype="fp32" if fp32 else "bf16", length_seed=rng.randrange(1 << 20), code=rng.choice(("e4m3", "int8")))
    if op == "project":
        return _case(None, op, layer, _log(rng, 1, 8192), features=rng.choice(("q", "kvl", "qkvl")), **same)
    seqs = rng.choice((1, _log(rng, 2, 64 if op == "append" else 16)))
    longest = _log(rng, 40, 65536 if seqs > 1 else 32768)
    shortest = max(1, int(longest * rng.uniform(0.05, 1.0))) if seqs > 1 else longest
    same.update(seqs=seqs, shortest=shortest)
    if op == "gather":
        return _case(None, op, layer, longest, kept=max(1, int(longest * rng.uniform(0.1, 1.0))) if rng.random() < 0.5 else 0, **same)
    if op == "append":
        return _case(None, op, layer, longest, queries=_log(rng, 1, min(4096, longest)), rope=rng.random() < 0.8, **same)
    causal = rng.random() < 0.5
    queries = min(shortest, _log(rng, 1, 1500) if causal else _log(rng, 1, 8))
    window = _log(rng, 16, 16384) if rng.random() < 0.4 else 0
    return _case(None, op, layer, longest, queries=queries, causal=causal, window=window,
                 sinks=rng.choice((0, 1, 4, 16, 64)) if window else 0, key_side=rng.random() < 0.6, **same)


def draw(rng):
    """Cases whose padded batch costs the plain form no more than the listed ones."""
    while True:
        c = _draw_once(rng)
        hq, hkv, d, _ = LAYERS[c["layer"]]
        if c["op"] == "project":
            return c
        lengths, counts = _sizes(c)
        if c["op"] == "attend":
            ok = c["seqs"] * hq * max(counts) * _span(c) <= 1 << 30 and c["seqs"] * _span(c) * hkv * d <= 1 << 29
        else:
            ok = c["seqs"] * max(counts) * hkv * d <= 1 << 25
        if ok and sum(lengths) <= 600000:
            return c


def _sizes(case):
    """Lengths and query (new token, kept row) counts of the sequences."""
    rng = random.Random(case["length_seed"])
    n, seqs = case["n"], case["seqs"]
    lengths = [n] + [rng.randint(case["shortest"], n) for _ in range(seqs - 1)]
    if case["op"] == "gather":
        return lengths, [min(m, case["kept"] or m) for m in lengths]
    most = case["queries"]
    ragged = case["causal"] or case["op"] == "append"
    return lengths, [most] + [min(lengths[t], _log(rng, 1, most)) if ragged else most for t in range(1, seqs)]


def _seen(case, n, c):
    """Sinks before the window, and the first key of the window of a sequence's first query."""
    first = n - c if case["causal"] else n - 1
    lo = max(0, first - case["window"] + 1) if case["window"] else 0
    return min(case["sinks"], lo) if case["window"] else 0, lo


def _span(case):
    """The most keys that any sequence's queries see together."""
    lengths, counts = _sizes(case)
    return max(s + n - lo for n, c in zip(lengths, counts) for s, lo in (_seen(case, n, c),))


def _features(case):
    hq, hkv, d, _ = LAYERS[case["layer"]]
    return {"q": hq * d, "kvl": 2 * hkv * d + case["rank"], "qkvl": hq * d + 2 * hkv * d + case["rank"]}[case["features"]]


def _touched(case):
    """First token of the first block that a sequence's new tokens touch."""
    return [(n - c) // BLOCK * BLOCK for n, c in zip(*_sizes(case))]


class _State:
    """Tensors and descriptors that a serving program holds for one layer."""


def _inputs(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    hq, hkv, d, dm = LAYERS[case["layer"]]
    r = case["rank"]

    def randn(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, generator=gen, device=dev, dtype=dtype).mul_(std)

    s = _State()
    if case["op"] == "project":
        # hidden states have a few channels that are some times larger than the others
        s.x = randn(case["n"], dm) * (1.0 + 6.0 * (torch.rand(dm, generator=gen, device=dev) < 0.02)).to(dt)
        n = _features(case)
        s.w = (randn(n, dm, dtype=torch.float32) * 32).round_().clamp_(-127, 127).to(torch.int8)
        s.w_scale = torch.rand(n, generator=gen, device=dev).add_(0.5).mul_(dm ** -0.5 / 32)
        return s
    lengths, counts = _sizes(case)
    seqs = case["seqs"]
    s.seq_lens = torch.tensor(lengths, dtype=torch.int32, device=dev)
    per_seq = torch.tensor([-(-n // BLOCK) for n in lengths], device=dev)
    blocks = sum(-(-n // BLOCK) for n in lengths)
    order = torch.randperm(blocks, generator=gen, device=dev).to(torch.int32)
    at = torch.arange(-(-max(lengths) // BLOCK), device=dev)
    index = (torch.cumsum(per_seq, 0) - per_seq)[:, None] + at
    s.block_table = torch.where(at < per_seq[:, None], order[index.clamp(max=blocks - 1)], -1).to(torch.int32).contiguous()

    def codes(*shape, channel):
        """Codes of about the spread that a block's largest value leaves the others; some channels of the keys are larger."""
        y = randn(*shape, dtype=torch.bfloat16) * channel
        if case["code"] == "e4m3":
            return y.mul_(64).clamp_(-448, 448).to(torch.float8_e4m3fn)
        return y.mul_(20).round_().clamp_(-127, 127).to(torch.int8)

    wide = (1.0 + 2.0 * (torch.rand(d, generator=gen, device=dev) < 0.06)).to(torch.bfloat16)
    s.k = codes(blocks, hkv, BLOCK, d, channel=wide)
    s.v = codes(blocks, hkv, d, BLOCK, channel=1.0)
    unit = 127 - (6 if case["code"] == "e4m3" else 4)
    s.k_scale, s.v_scale = (torch.randint(unit - 1, unit + 1, (blocks, hkv), generator=gen, device=dev).to(torch.uint8) for _ in range(2))
    s.l = randn(blocks, BLOCK, r)
    total = sum(counts)
    s.start = torch.tensor([sum(counts[:t]) for t in range(seqs + 1)], dtype=torch.int32, device=dev)
    if case["op"] == "append":
        # one product's output: keys, values and low-rank rows side by side
        s.new = randn(total, 2 * hkv * d + r)
        s.new[:, :hkv * d].view(total, hkv, d).mul_(wide.to(dt))
    elif case["op"] == "gather":
        s.kept = None
        if case["kept"]:
            s.kept = torch.zeros(seqs, max(counts), dtype=torch.int32, device=dev)
            for t, (n, c) in enumerate(zip(lengths, counts)):  # (an eviction keeps single tokens, sinks and the recent ones)
                s.kept[t, :c] = torch.randperm(n, generator=gen, device=dev)[:c].sort().values.int()
    else:
        s.n_adapters = 5
        s.b_k = randn(s.n_adapters, r, hkv * d, std=0.02) if case["key_side"] else None
        s.b_v = randn(s.n_adapters, r, hkv * d, std=0.02)
        s.q = randn(total, hq, d)
        per = torch.tensor(counts, device=dev)
        s.query_adapter = (torch.arange(seqs, device=dev).repeat_interleave(per) % s.n_adapters if case["causal"]
                           else torch.arange(total, device=dev) % s.n_adapters).to(torch.int32)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s.case = case
    hq, hkv, d, dm = LAYERS[case["layer"]]
    if case["op"] == "project":
        m, n, dev = case["n"], _features(case), s.x.device
        s.codes = torch.empty(m, dm, dtype=torch.int8, device=dev)
        s.scales = torch.empty(m, device=dev)
        s.y = torch.empty(m, n, dtype=s.x.dtype, device=dev)
        if own:
            import paper_2602_01053_amd as lra
            s.lra = lra
            s.workspace = torch.empty(max(lra.lra_matmul_i8_workspace_bytes(m, n, dm, s.y.dtype), 256), dtype=torch.uint8, device=dev)
        return s
    dev = s.k.device
    lengths, counts = _sizes(case)
    s.most, s.n_max = max(counts), max(lengths)
    if case["op"] == "attend":
        s.keys = _span(case)
        s.out = torch.empty_like(s.q)
    else:
        rows = counts if case["op"] == "gather" else [n - b for n, b in zip(lengths, _touched(case))]
        dt, per = s.l.dtype, -(-max(rows) // BLOCK)
        s.dst_lens = torch.tensor(rows, dtype=torch.int32, device=dev)
        s.dst_table = torch.arange(case["seqs"] * per, dtype=torch.int32, device=dev).view(case["seqs"], per).flip(0).contiguous()
        s.dst = [torch.zeros(shape, dtype=dt, device=dev) for shape in ((case["seqs"] * per, hkv, BLOCK, d),) * 2 + ((case["seqs"] * per, BLOCK, case["rank"]),)]
        s.rows = max(rows)
    if own:
        import paper_2602_01053_amd as lra
        s.lra = lra
        like = torch.empty(1, hq, d, dtype=s.l.dtype, device=dev)
        s.shape = lra.make_shape(like, hkv, case["rank"])
        s.cache = lra.make_cache8(s.k, s.v, s.k_scale, s.v_scale, s.l, s.seq_lens, s.n_max, s.block_table)
        if case["op"] == "attend":
            s.batch = lra.make_batch(s.start, s.query_adapter, s.most, causal=case["causal"], window=case["window"], sinks=case["sinks"])
            s.workspace = torch.empty(max(lra.lra_batch8_workspace_bytes(s.shape, s.cache, s.batch), 256), dtype=torch.uint8, device=dev)
        else:
            s.dst_cache = lra.make_cache(*s.dst, s.dst_lens, s.rows, s.dst_table)
    return s


def run(s):
    case = s.case
    hq, hkv, d, _ = LAYERS[case["layer"]]
    if case["op"] == "project":
        if own:
            s.lra.lra_quantize_rows(s.x, s.codes, s.scales)
            s.lra.lra_matmul_i8(s.codes, s.scales, s.w, s.w_scale, s.y, s.workspace)
        else:
            _plain_project(s)
        return {"y": s.y, "scales": s.scales}
    if case["op"] == "attend":
        if not own:
            return _plain_attend(s)
        s.lra.lra_attn_batch8(s.shape, s.cache, s.b_k, s.b_v, s.n_adapters, s.batch, s.q, s.out, s.workspace)
        return s.out
    if case["op"] == "append":
        total = s.new.shape[0]
        k, v = (s.new[:, i * hkv * d:(i + 1) * hkv * d].view(total, hkv, d) for i in (0, 1))
        low = s.new[:, 2 * hkv * d:]
        if own:
            s.lra.lra_cache8_append(s.shape, s.cache, s.start, s.most, k, v, low, ROPE_THETA if case["rope"] else 0.0)
        else:
            _plain_append(s, k, v, low)
    if own:
        s.lra.lra_cache8_gather(s.shape, s.cache, s.dst_cache, s.kept if case["op"] == "gather" else None)
    else:
        _plain_gather(s, s.kept if case["op"] == "gather" else None)
    return {"k": s.dst[0], "v": s.dst[1], "l": s.dst[2]}


# ---------------------------------------------------------------------------------------------------------------
# The plain forms: padded batches, 32 bits, rounded once.
# ---------------------------------------------------------------------------------------------------------------
def _plain_project(s):
    x = s.x.float()
    most = x.abs().amax(1)
    s.scales.copy_(most / 127)
    codes = torch.round(x * torch.where(most > 0, 127 / most, 0)[:, None])
    y = torch.matmul(codes, s.w.float().t())
    s.y.copy_(y * s.scales[:, None] * s.w_scale)


def _power(exponent):
    """2^(exponent - 127), by its bits (a power function may be a step off)."""
    return (exponent.int() << 23).view(torch.float32)


def _values(codes, exponent):
    """codes: float8 or int8, exponent: uint8 that broadcasts against them."""
    return codes.float() * _power(exponent)


def _plain_append(s, k, v, low):
    case, dev = s.case, s.k.device
    d = k.shape[-1]
    n, start = s.seq_lens.long(), s.start.long()
    first = n - (start[1:] - start[:-1])                                                               # [T]
    b0 = first // BLOCK
    blocks = torch.arange((s.most + 2 * BLOCK - 2) // BLOCK, device=dev)
    at = b0[:, None] + blocks                                                                          # [T][B]
    token = at[..., None] * BLOCK + torch.arange(BLOCK, device=dev)                                    # [T][B][16]
    new = (token >= first[:, None, None]) & (token < n[:, None, None])
    old = (token < first[:, None, None]) & (at * BLOCK < n[:, None])[..., None]
    here = new.any(-1)
    row = (start[:-1, None, None] + token - first[:, None, None]).clamp(0, k.shape[0] - 1)
    block = s.block_table[torch.arange(len(n), device=dev)[:, None], at.clamp(max=s.block_table.shape[1] - 1)].long()[here]
    token, new, old, row = token[here], new[here], old[here], row[here]                                # [N][16]
    x = k[row].float()                                                                                 # [N][16][Hkv][d]
    if case["rope"]:
        rate = ROPE_THETA ** (-torch.arange(0, d, 2, device=dev, dtype=torch.float64) / d)
        angle = token[..., None, None].double() * rate
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        a, b = x[..., :d // 2], x[..., d // 2:]
        x = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    x, y = x.transpose(1, 2), v[row].float().permute(0, 2, 3, 1)                                       # [N][Hkv][16][d], [N][Hkv][d][16]
    for cache, scale, z, slot in ((s.k, s.k_scale, x, (slice(None), None, slice(None), None)),
                                  (s.v, s.v_scale, y, (slice(None), None, None, slice(None)))):
        is_new, is_old = new[slot], old[slot]
        most = (z.abs() * is_new).amax((2, 3))
        bits = most.view(torch.int32)
        # the least power of two that brings the largest value to at most 448 (1.75 x 2^8) or 127 (1.984375 x 2^6)
        need = ((bits + 0x1fffff >> 23) - 8 if case["code"] == "e4m3" else (bits + 0x01ffff >> 23) - 6).clamp(min=1)
        had = scale[block].int()
        e = torch.where(is_old.any(3).any(2), torch.maximum(need, had), need)
        codes = cache[block]
        kept = codes.float() * _power((127 + had - e).clamp(min=1))[..., None, None]
        z = torch.where(is_new, z * _power(254 - e)[..., None, None], torch.where(is_old, kept, 0))
        z = z.to(torch.float8_e4m3fn) if case["code"] == "e4m3" else torch.round(z).to(torch.int8)
        # (slots behind the end keep what they held; as bytes, which may be no number)
        cache[block] = torch.where(is_new | is_old, z.view(torch.uint8), codes.view(torch.uint8)).view(codes.dtype)
        scale[block] = e.to(torch.uint8)
    i, j = torch.nonzero(new, as_tuple=True)
    s.l[block[i], j] = low[row[i, j]]


def _plain_gather(s, kept):
    n, rows = s.seq_lens.long()[:, None], s.dst_lens.long()[:, None]
    i = torch.arange(s.rows, device=n.device)
    t, at = torch.nonzero(i < rows, as_tuple=True)
    src = (i + n - rows)[t, at] if kept is None else kept[t, at].long()
    b, c = s.block_table[t, src // BLOCK].long(), src % BLOCK
    e, f = s.dst_table[t, at // BLOCK].long(), at % BLOCK
    dt = s.l.dtype
    s.dst[0][e, :, f] = _values(s.k[b, :, c], s.k_scale[b][..., None]).to(dt)
    s.dst[1][e, :, f] = _values(s.v[b, :, :, c], s.v_scale[b][..., None]).to(dt)
    s.dst[2][e, f] = s.l[b, c]


def _plain_attend(s):
    case, dev = s.case, s.q.device
    hq, hkv, d, _ = LAYERS[case["layer"]]
    r, g, seqs, most = case["rank"], hq // hkv, case["seqs"], s.most
    n = s.seq_lens.long()
    start = s.start.long()
    count = start[1:] - start[:-1]
    k_of = torch.arange(most, device=dev)
    query = torch.minimum(start[:-1, None] + k_of, start[1:, None] - 1)                                # [T][C]
    pos = (n - count)[:, None] + k_of if case["causal"] else (n - 1)[:, None].expand(seqs, most)
    first = pos[:, :1]
    lo = (first - case["window"] + 1).clamp(min=0) if case["window"] else torch.zeros_like(first)
    sinks = torch.minimum(torch.full_like(lo, case["sinks"]), lo) if case["window"] else lo
    u = torch.arange(s.keys, device=dev)
    token = torch.where(u < sinks, u, u - sinks + lo)                                                  # [T][U]
    live = token < n[:, None]
    token = torch.minimum(token, n[:, None] - 1)
    a, m = (1, most) if case["causal"] else (most, 1)
    adapter = s.query_adapter[query[:, ::m]].long()                                                    # [T][A]
    q = s.q[query].float().view(seqs, a, m, hkv, g, d).permute(0, 1, 3, 2, 4, 5).reshape(seqs, a, hkv, m * g, d)
    block, slot = s.block_table[torch.arange(seqs, device=dev)[:, None], token // BLOCK].long(), token % BLOCK
    keys = _values(s.k[block, :, slot], s.k_scale[block][..., None]).permute(0, 2, 3, 1).unsqueeze(1)  # [T][1][Hkv][d][U]
    low = s.l[block, slot].float()                                                                     # [T][U][r]
    scores = torch.matmul(q, keys)
    del keys
    if s.b_k is not None:
        b = s.b_k[adapter].float().view(seqs, a, r, hkv, d).permute(0, 1, 3, 2, 4)                     # [T][A][Hkv][r][d]
        scores += torch.matmul(torch.matmul(q, b.transpose(-1, -2)), low.transpose(-1, -2)[:, None, None])
    scores *= 1.0 / math.sqrt(d)
    seen = live[:, None] & (token[:, None] <= pos[..., None])
    if case["window"]:
        seen &= (token[:, None] > pos[..., None] - case["window"]) | (token[:, None] < case["sinks"])
    seen = seen.view(seqs, a, 1, m, 1, s.keys).expand(-1, -1, hkv, -1, g, -1).reshape(seqs, a, hkv, m * g, s.keys)
    scores.masked_fill_(~seen, -math.inf)
    scores -= scores.amax(-1, keepdim=True).clamp(min=-1e30)
    p = scores.exp_()
    total = p.sum(-1, keepdim=True)
    values = _values(s.v[block, :, :, slot], s.v_scale[block][..., None]).permute(0, 2, 1, 3).unsqueeze(1)  # [T][1][Hkv][U][d]
    b = s.b_v[adapter].float().view(seqs, a, r, hkv, d).permute(0, 1, 3, 2, 4)
    o = torch.matmul(p, values) + torch.matmul(torch.matmul(p, low[:, None, None]), b)
    o /= total
    o = o.view(seqs, a, hkv, m, g, d).permute(0, 1, 3, 2, 4, 5).reshape(seqs, most, hq, d)
    ours = torch.arange(most, device=o.device) < count[:, None]
    return o[ours].to(s.q.dtype)


# ---------------------------------------------------------------------------------------------------------------
# The definition in 64 bits, sequence by sequence and head by head.
# ---------------------------------------------------------------------------------------------------------------
def _two(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


def _exact_codes(z, least, e4m3):
    """Values of z [...][block's values] as the cache holds them, for the scale 2^least at least; and that scale's exponent."""
    top = z.abs().amax(-1, keepdim=True)
    most = 448.0 if e4m3 else 127.0
    e = torch.ceil(torch.log2(top / most)).clamp(min=-126)
    e = torch.where(top > most * _two(e), e + 1, torch.where((top <= most * _two(e - 1)) & (e > -126), e - 1, e))
    e = torch.maximum(e, least)
    y = z / _two(e)
    step = _two((torch.frexp(y.abs().clamp(min=2.0 ** -6)).exponent - 4)) if e4m3 else 1.0
    return torch.round(y / step) * step * _two(e), e


def exact(case, seed):
    s = _inputs(case, seed)
    hq, hkv, d, dm = LAYERS[case["layer"]]
    if case["op"] == "project":
        x = s.x.double()
        unit = x.abs().amax(1, keepdim=True) / 127
        codes = torch.round(x / unit.clamp(min=1e-300))
        w = s.w.double() * s.w_scale.double()[:, None]
        return {"y": (codes * unit) @ w.T, "scales": unit[:, 0]}
    g, r = hq // hkv, case["rank"]
    lengths, counts = _sizes(case)

    def row_of(t, j):
        blk = s.block_table[t, j // BLOCK].long()
        k = s.k[blk, :, j % BLOCK].double() * _two(s.k_scale[blk].long()[..., None] - 127)
        v = s.v[blk, :, :, j % BLOCK].double() * _two(s.v_scale[blk].long()[..., None] - 127)
        return k, v, s.l[blk, j % BLOCK].double()

    if case["op"] != "attend":
        rows = counts if case["op"] == "gather" else [n - b for n, b in zip(lengths, _touched(case))]
        per = -(-max(rows) // BLOCK)
        table = torch.arange(case["seqs"] * per, device=s.k.device).view(case["seqs"], per).flip(0)
        out = [torch.zeros(case["seqs"] * per, *shape, dtype=torch.float64, device=s.k.device) for shape in ((hkv, BLOCK, d), (hkv, BLOCK, d), (BLOCK, r))]
        at = 0
        for t, (n, c, m) in enumerate(zip(lengths, counts, rows)):
            j = torch.arange(n - m, n, device=s.k.device)
            if case["op"] == "gather" and s.kept is not None:
                j = s.kept[t, :c].long()
            k, v, low = row_of(t, j)
            if case["op"] == "append":
                y = s.new[at:at + c].double()
                x = y[:, :hkv * d].view(c, hkv, d)
                if case["rope"]:
                    turn = torch.arange(n - c, n, device=s.k.device)[:, None, None].double() / ROPE_THETA ** (torch.arange(d // 2, device=s.k.device).double() * 2 / d)
                    z = torch.polar(torch.ones_like(turn), turn) * torch.complex(x[..., :d // 2], x[..., d // 2:])
                    x = torch.cat((z.real, z.imag), -1)
                pad = -m % BLOCK
                least = torch.full((-(-m // BLOCK), hkv, 1), -126.0, dtype=torch.float64, device=s.k.device)
                first = s.block_table[t, (n - m) // BLOCK].long()
                for side, (vals, fresh, scale) in enumerate(((k, x, s.k_scale), (v, y[:, hkv * d:2 * hkv * d].view(c, hkv, d), s.v_scale))):
                    lo = least.clone()
                    if m > c:
                        lo[0, :, 0] = scale[first].double() - 127
                    z = torch.cat((vals[:m - c], fresh, torch.zeros(pad, hkv, d, dtype=torch.float64, device=s.k.device)))
                    z = z.view(-1, BLOCK, hkv, d).transpose(1, 2).reshape(-1, hkv, BLOCK * d)
                    z, _ = _exact_codes(z, lo, case["code"] == "e4m3")
                    z = z.view(-1, hkv, BLOCK, d).transpose(1, 2).reshape(-1, hkv, d)[:m]
                    if side == 0:
                        k = z
                    else:
                        v = z
                low = torch.cat((low[:m - c], y[:, 2 * hkv * d:]))
                at += c
            i = torch.arange(m, device=s.k.device)
            e, f = table[t, i // BLOCK], i % BLOCK
            out[0][e, :, f], out[1][e, :, f], out[2][e, f] = k, v, low
        return {"k": out[0], "v": out[1], "l": out[2]}
    out = torch.zeros(s.q.shape, dtype=torch.float64, device=s.q.device)
    at = 0
    for t, (n, c) in enumerate(zip(lengths, counts)):
        groups = [(at, c)] if case["causal"] else [(at + i, 1) for i in range(c)]
        for first, m in groups:
            a = int(s.query_adapter[first])
            p_of = n - m + torch.arange(m, device=s.q.device)
            j = torch.arange(n, device=s.q.device)
            mask = j[None, :] <= p_of[:, None]
            if case["window"] > 0:
                mask &= (p_of[:, None] - j[None, :] < case["window"]) | (j[None, :] < case["sinks"])
            some = torch.nonzero(mask.any(0))[:, 0]
            mask = mask[:, some]
            k, v, low = row_of(t, some)
            for h in range(hkv):
                cols = slice(h * d, (h + 1) * d)
                key = k[:, h] if s.b_k is None else k[:, h] + low @ s.b_k[a, :, cols].double()
                val = v[:, h] + low @ s.b_v[a, :, cols].double()
                for x in range(h * g, (h + 1) * g):
                    z = s.q[first:first + m, x].double() @ key.T / math.sqrt(d)
                    out[first:first + m, x] = torch.softmax(z.masked_fill(~mask, -math.inf), 1) @ val
        at += c
    return out


def work(case):
    """Bytes: every row that is needed once, as it is held (codes one byte, a scale per 16 rows and head), and what is
    written.  Operations: attention as per pair of a query row and a key it sees 2d for the score, 2d + 2r for the values (2r
    more with a key-side adapter) and the rank-r projections of each row; a product's 2 per weight and token."""
    hq, hkv, d, dm = LAYERS[case["layer"]]
    es = 2 if case["dtype"] == "bf16" else 4
    r, causal, win, sinks = case["rank"], case["causal"], case["window"], case["sinks"]
    if case["op"] == "project":
        m, n = case["n"], _features(case)
        return {"bytes": m * dm * es + n * (dm + 4) + m * (n * es + 4), "flops": 2 * m * n * dm}
    lengths, counts = _sizes(case)
    held = 2 * hkv * (d + 1 / BLOCK) + r * es
    row = (2 * hkv * d + r) * es
    if case["op"] == "gather":
        return {"bytes": sum(counts) * (held + row + (4 if case["kept"] else 0)), "flops": 0}
    if case["op"] == "append":
        rows = sum(n - b for n, b in zip(lengths, _touched(case)))
        return {"bytes": sum(counts) * (row + held) + rows * row + (rows - sum(counts)) * held, "flops": 0}
    pairs = keys = 0
    for n, c in zip(lengths, counts):
        s0, lo = _seen(case, n, c)
        keys += s0 + n - lo
        for p in (range(n - c, n) if causal else [n - 1] * c):
            first = max(0, p - win + 1) if win else 0
            pairs += p + 1 - first + (min(sinks, first) if win else 0)
    rows = sum(counts) * hq
    pairs *= hq
    used = min(5, case["seqs"] if causal else sum(counts))
    nbytes = keys * held + es * (2 * rows * d + (2 if case["key_side"] else 1) * used * r * hkv * d)
    flops = pairs * (4 * d + 2 * r) + 2 * rows * d * r + (pairs * 2 * r + 2 * rows * d * r if case["key_side"] else 0)
    return {"bytes": nbytes, "flops": flops}
