"""The paged cache's operators captured into graphs in the forms for many rows, and the gradient: replayed with other lengths and inputs, eager
work in between, every replay against the eager result."""
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


def _captured(step):
    step()
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step()
    return graph


@pytest.mark.parametrize("new,H,Hkv,hd", [([8, 8, 8], 4, 2, 128), ([16, 16], 8, 2, 64), ([24, 24], 8, 2, 128), ([100, 90], 4, 1, 128), ([16, 9], 8, 1, 256)])
def test_blocks_and_prompts(ctx, new, H, Hkv, hd):
    page, most = 16, 6000
    g = torch.Generator(device="cuda").manual_seed(3)
    batch = ref.Batch(new, [most] * len(new), page)
    pages = [torch.randn((batch.n_pages, page, Hkv, hd), generator=g, device="cuda").bfloat16() for _ in range(2)]
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    qk, cfg = mrp.QkNormRope(H, Hkv, hd, ctx.rope_table(most, hd, 1e6)), mrp.AttnCfg(H, hd ** -0.5)
    x = torch.randn((batch.n_rows, H + 2 * Hkv, hd), generator=g, device="cuda").bfloat16()
    q_out, out = (torch.empty((batch.n_rows, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.empty((batch.n_rows, H), device="cuda")

    def step():
        ctx.cache_append(rows, qk, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], paged, q_out)
        ctx.paged_attention(rows, paged, cfg, q_out, out, lse=lse)

    graph = _captured(step)
    for lens in ([most] * 3, [17, 300, 5], [4000, 0, 128], [most - 1, 90, 700]):
        batch.len_d.copy_(torch.tensor(lens[:len(new)], dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), pages[0].clone(), pages[1].clone()
        out.zero_()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, *pages)))
    assert ctx.poll_error() == 0


def test_gradient(ctx):
    n, H, Hkv, hd = 3000, 6, 2, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    qkv, dy, dk_out, dqkv, dg = r(n, H + 2 * Hkv, hd), r(n, H, hd), r(n, Hkv, hd), r(n, H + 2 * Hkv, hd), torch.empty((2, hd), device="cuda")
    gains = [(1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16() for _ in range(2)]
    qk = mrp.QkNormRope(H, Hkv, hd, ctx.rope_table(n, hd, 1e6), *gains)
    pos = torch.arange(n, device="cuda").int()

    def step():
        ctx.qk_norm_rope_grad(qk, pos, qkv[:, :H], qkv[:, H:H + Hkv], dy, dk_out, dqkv[:, :H], dqkv[:, H:H + Hkv], dg[0], dg[1])

    graph = _captured(step)
    for _ in range(4):
        for t in (qkv, dy, dk_out):
            t.copy_(torch.randn(t.shape, generator=g, device="cuda"))
        pos.copy_(torch.randint(0, n, (n,), generator=g, device="cuda"))
        dqkv.fill_(7.0), dg.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = dqkv.clone(), dg.clone()
        dqkv.fill_(7.0), dg.fill_(7.0)
        step()
        torch.cuda.synchronize()
        assert torch.equal(got[0], dqkv) and torch.equal(got[1], dg) and (dqkv[:, H + Hkv:] == 7.0).all()
