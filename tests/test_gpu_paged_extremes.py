"""The paged cache's operators at the ends of what they take: the largest batch, a million positions, row tensors of more than 2^31 entries."""
import math

import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


@pytest.mark.parametrize("new,hd", [(1, 64), (3, 128), (40, 64), (70, 64), (130, 64), (5, 256)])
def test_the_largest_batch(ctx, new, hd):
    """65535 sequences; each one's last row sees one position alone, and its output is that position's value."""
    B, n_pages, page = 65535, 4096, 3
    g = torch.Generator(device="cuda").manual_seed(1)
    k, v = (torch.randn((n_pages, page, 1, hd), generator=g, device="cuda").half() for _ in range(2))
    lens = torch.randint(0, 7, (B,), generator=g, device="cuda").int()
    table = torch.randint(0, n_pages, (B, 2), generator=g, device="cuda").int()
    q = torch.randn((B * new, 1, hd), generator=g, device="cuda").half()
    out, lse = torch.full_like(q, 7.0), torch.empty((B * new, 1), device="cuda")
    ctx.poll_error()
    ctx.paged_attention(mrp.NewRows(lens, new), mrp.PagedCache(k, v, table), mrp.AttnCfg(1, 0.25, window=1), q, out, lse=lse)
    assert ctx.poll_error() == 0
    pos = lens.long()[:, None] - new + torch.arange(new, device="cuda")
    at = pos.clamp_min(0)
    where = table.long().gather(1, (at // page)), at % page
    want = torch.where((pos >= 0)[..., None], v[where[0], where[1], 0], 0.0).view(B * new, 1, hd)
    assert torch.equal(out, want)
    score = (q.view(B, new, hd).double() * k[where[0], where[1], 0].double()).sum(-1) * 0.25
    want = torch.where(pos >= 0, score, -math.inf).view(B * new, 1)
    assert torch.equal(torch.isneginf(lse), torch.isneginf(want))
    off = torch.where(pos.view(-1, 1) >= 0, (lse.double() - want).abs(), 0.0)
    assert float(off.max()) <= (hd + 10) * ref.U32 * 0.25 * float((q.float().abs().amax() * k.float().abs().amax()) * hd)


@pytest.mark.parametrize("new,H,hd,cache", [(1, 2, 64, torch.float8_e4m3fn), (1, 4, 128, torch.bfloat16), (16, 4, 64, torch.bfloat16), (25, 4, 64, torch.float8_e4m3fn),
                                            (300, 1, 64, torch.bfloat16), (3, 2, 256, torch.bfloat16)])
def test_a_million_positions(ctx, new, H, hd, cache):
    n, page = 1_000_003, 48
    g = torch.Generator(device="cuda").manual_seed(1)
    n_pages = -(-n // page)
    k, v = (torch.randn((n_pages, page, 1, hd), generator=g, device="cuda").to(cache) for _ in range(2))
    table = torch.randperm(n_pages, generator=g, device="cuda").int()[None].contiguous()
    q = torch.randn((new, H, hd), generator=g, device="cuda").bfloat16()
    out, lse = torch.empty_like(q), torch.empty((new, H), device="cuda")
    ctx.paged_attention(mrp.NewRows(torch.tensor([n], dtype=torch.int32, device="cuda"), new), mrp.PagedCache(k, v, table),
                        mrp.AttnCfg(H, 0.3, causal=False), q, out, lse=lse)
    order = table[0].long()
    kk, vv = (t.view(torch.uint8 if cache == torch.float8_e4m3fn else torch.int16)[order].view(-1, hd)[:n].view(cache) for t in (k, v))
    # 64 bits, a hundred thousand positions at a time
    qq, top, total, acc, mag = q.double().view(-1, hd), None, 0.0, 0.0, 0.0
    s = torch.cat([qq @ kk[i:i + 100000].double().T for i in range(0, n, 100000)], 1) * 0.3
    top = s.amax(1, keepdim=True)
    w = (s - top).exp()
    for i in range(0, n, 100000):
        acc = acc + w[:, i:i + 100000] @ vv[i:i + 100000].double()
        mag = mag + w[:, i:i + 100000] @ vv[i:i + 100000].double().abs()
    total = w.sum(1, keepdim=True)
    want, mag = (acc / total).view(out.shape), (mag / total).view(out.shape)
    qk = (qq.abs().sum(1) * float(kk.float().abs().amax()) * 0.3).view(new, H, 1)
    wlse = (top + total.log()).view(new, H)
    tol, ltol = ref.attention_tolerance(torch.bfloat16, want, wlse, mag, qk, hd, 20000, few=new * H <= 32 or hd == 256)    # (no chain is longer than a piece)
    ref.assert_close(out, want, tol, "out")
    ref.assert_close(lse, wlse, ltol, "lse")


def test_rows_beyond_two_to_the_31_entries(ctx):
    """Queries and outputs of 2^32 entries (8.6 GB each): the last rows against the same rows in a call of their own."""
    H, hd, n = 16, 64, (1 << 22) + 37
    q = torch.empty((n, H, hd), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    for at in range(0, n, 1 << 20):
        q[at:at + (1 << 20)] = torch.randn(q[at:at + (1 << 20)].shape, generator=g, device="cuda", dtype=torch.bfloat16)
    out = torch.empty_like(q)
    last = q[-37:].clone()
    rope = ctx.rope_table(100, hd, 1e4)
    pos = (torch.arange(n, device="cuda") % 100).int()
    qk = mrp.QkNormRope(H, 0, hd, rope, torch.ones(hd, device="cuda"), None)
    ctx.qk_norm_rope(qk, pos, q, None, out, None)
    want = torch.empty_like(last)
    ctx.qk_norm_rope(qk, pos[-37:].clone(), last, None, want, None)
    assert torch.equal(out[-37:], want)
    # sequences of 105 rows, and one of the last 37
    k, v = (torch.randn((7, 16, 2, hd), generator=g, device="cuda").bfloat16() for _ in range(2))
    cu = torch.tensor([0] + [min(n - 37, 105 * (i + 1)) for i in range(40000)] + [n], device="cuda").int()
    B = cu.shape[0] - 1
    lens = torch.full((B,), 112, dtype=torch.int32, device="cuda")
    table = torch.arange(7, dtype=torch.int32, device="cuda").repeat(B, 1)
    out.fill_(7.0)
    ctx.poll_error()
    ctx.paged_attention(mrp.NewRows(lens, 105, cu_rows=cu), mrp.PagedCache(k, v, table), mrp.AttnCfg(H, 0.125), q, out)
    assert ctx.poll_error() == 0
    one = torch.empty_like(last)
    ctx.paged_attention(mrp.NewRows(lens[:1].clone(), 105, cu_rows=torch.tensor([0, 37], dtype=torch.int32, device="cuda")),
                        mrp.PagedCache(k, v, table[:1].contiguous()), mrp.AttnCfg(H, 0.125), last, one)
    tol = 2 * ref.half_step(torch.bfloat16) * one.double().abs() + 2.0 ** -12
    assert ((out[-37:].double() - one.double()).abs() <= tol).all()
    assert torch.isfinite(out[::1001].float()).all()
