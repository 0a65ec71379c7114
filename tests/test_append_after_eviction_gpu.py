"""A trajectory that goes on behind an eviction: prompt, weights, cut, one more token, attention."""
import pytest
import torch

import paper_2602_01053_amd as lra

pytestmark = pytest.mark.gpu

BF16, DEV, THETA = torch.bfloat16, "cuda", 10000.0


def turned(x, pos, theta):
    """Rotate-half pairs of x [tokens][heads][d] turned by the tokens' positions, in float64."""
    d = x.shape[-1]
    ang = pos.double()[:, None, None] * theta ** (-torch.arange(0, d, 2, device=x.device).double() / d)
    a, b = x.double()[..., :d // 2], x.double()[..., d // 2:]
    return torch.cat((a * ang.cos() - b * ang.sin(), b * ang.cos() + a * ang.sin()), -1)


@pytest.mark.parametrize("theta", [0.0, THETA])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 4, 64)])
def test_append_after_eviction(theta, hq, hkv, d):
    """Kept keys have the angles of their first positions, and the appended ones get those of theirs although their indices in the
    cache are smaller: appended unrotated, turned by the caller."""
    r, d_model, n, budget, n_new, n_adapters = 16, 256, 400, 96, 3, 2
    g = torch.Generator().manual_seed(31)
    w = (torch.randn(2 * hkv * d + r, d_model, generator=g) / 16).to(BF16)
    x = torch.randn(n + n_new, d_model, generator=g).to(BF16)
    b_v = (torch.randn(n_adapters, r, hkv * d, generator=g) * 0.15).to(BF16)
    q = torch.randn(4, hq, d, generator=g).to(BF16)
    wd, xd, b_vd, qd = w.to(DEV), x.to(DEV), b_v.to(DEV), q.to(DEV)
    shape = lra.make_shape(qd, hkv, r)
    start, adapter = (torch.tensor(v, dtype=torch.int32, device=DEV) for v in ([0, 4], [0, 1, 1, 0]))

    def cache(tokens):
        blocks = -(-tokens // 16)
        return [torch.full((blocks, hkv, 16, d), float("nan"), dtype=BF16, device=DEV) for _ in range(2)] + [
            torch.full((blocks, 16, r), float("nan"), dtype=BF16, device=DEV),
            torch.randperm(blocks, generator=g).to(torch.int32).view(1, blocks).to(DEV)]

    k, v, l, table = cache(n)
    lens = torch.tensor([n], dtype=torch.int32, device=DEV)
    src = lra.make_cache(k, v, l, lens, n, table)
    lra.lra_cache_append(shape, src, wd, theta, xd[:n].contiguous(), 0)
    batch = lra.make_batch(start, adapter, 4)
    weights = torch.empty(1, n, device=DEV)
    ws = torch.empty(lra.lra_key_weights_workspace_bytes(shape, src, batch), dtype=torch.uint8, device=DEV)
    lra.lra_key_weights(shape, src, None, n_adapters, batch, qd, 0.0, weights, ws)
    k2, v2, l2, table2 = cache(budget + n_new)
    new = torch.empty(1, dtype=torch.int32, device=DEV)
    kept = torch.empty(1, budget, dtype=torch.int32, device=DEV)
    lra.lra_evict_select(src, weights, budget, 4, 16, kept, new)
    lra.lra_cache_gather(shape, src, kept, lra.make_cache(k2, v2, l2, new, budget, table2))
    # three tokens more
    new += n_new
    dst = lra.make_cache(k2, v2, l2, new, budget + n_new, table2)
    lra.lra_cache_append(shape, dst, wd, 0.0, xd[n:].contiguous(), 0)
    at = torch.arange(budget, budget + n_new, device=DEV)
    blk = table2[0, at // 16].long()
    pos = torch.arange(n, n + n_new, device=DEV)
    if theta:
        k2[blk, :, at % 16] = turned(k2[blk, :, at % 16], pos, theta).to(BF16)
    out = torch.full_like(qd, float("nan"))
    ws = torch.empty(lra.lra_batch_workspace_bytes(shape, dst, batch), dtype=torch.uint8, device=DEV)
    lra.lra_attn_batch(shape, dst, None, b_vd, n_adapters, batch, qd, out, ws)
    torch.cuda.synchronize()

    # The rows against the projection in float64, each at the position of its token.  A key is rounded once by the append (half a step,
    # 2^-8 of the value), and a new one again after the turn, which adds the errors of both members of a pair; sums of 256 products in
    # fp32 and angles taken to 1e-6 of a turn add some 1e-5 of sizes up to 5.
    token = torch.cat((kept[0].long(), pos)).cpu()
    where = torch.arange(budget + n_new)
    rows = lambda y: y.cpu()[table2.cpu()[0, where // 16].long(), :, where % 16]  # noqa: E731
    raw = (x.double() @ w.double().T)[token]
    key = raw[:, :hkv * d].view(-1, hkv, d)
    ref = turned(key, token, theta) if theta else key
    pair = key.abs() + torch.cat((key[..., d // 2:], key[..., :d // 2]), -1).abs()
    limit = 2 ** -8 * (ref.abs() + (pair if theta else 0)) + 1e-4
    got = rows(k2).double()
    assert ((got - ref).abs() <= limit).all()
    assert torch.equal(rows(k2)[:budget], k.cpu()[table.cpu()[0, token[:budget] // 16].long(), :, token[:budget] % 16])

    # the call on the rows that stand there
    val = rows(v2).double()
    low = l2.cpu()[table2.cpu()[0, where // 16].long(), where % 16].double()
    expect = torch.empty(4, hq, d, dtype=torch.float64)
    for i in range(4):
        a = int(adapter[i])
        p = torch.softmax(torch.einsum("hgd,nhd->hgn", q[i].double().view(hkv, -1, d), got) / d ** 0.5, -1)
        expect[i] = torch.einsum("hgn,nhd->hgd", p, val + (low @ b_v[a].double()).view(-1, hkv, d)).reshape(hq, d)
    assert float((out.double().cpu() - expect).norm() / expect.norm()) <= 5e-3  # as tests/test_batch_gpu.py
