"""Pages that no row sees any more are not looked at: a program with a sliding window gives them back and clears their entries."""
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


# (pages that end inside a step of 32 or a tile of 64 positions, and such that do not)
@pytest.mark.parametrize("page", [1, 16, 48, 24, 32, 64])
@pytest.mark.parametrize("new,lens,H,Hkv,hd", [([1, 1, 1], [40, 300, 1500], 8, 2, 64), ([4, 8], [200, 999], 8, 2, 128), ([1, 5], [90, 700], 8, 1, 256),
                                               ([9, 16], [150, 800], 8, 2, 128), ([30, 24], [150, 5000], 8, 2, 64), ([70, 100], [300, 120], 4, 1, 128)])
@pytest.mark.parametrize("causal,window,sinks", [(True, 50, 4), (True, 64, 0), (False, 33, 70), (True, 1, 1)])
def test_pages_behind_the_window(ctx, page, new, lens, H, Hkv, hd, causal, window, sinks):
    batch = ref.Batch(new, lens, page)
    for b, (n, total) in enumerate(zip(new, lens)):
        low = max(0, total - n + 1 - window)
        for i in range(-(-total // page)):
            if (i + 1) * page <= low and i * page >= sinks:
                batch.table[b, i] = (-1, batch.n_pages, -2 ** 31)[i % 3]
    g = torch.Generator(device="cuda").manual_seed(0)
    pages = [torch.randn((batch.n_pages, page, Hkv, hd), generator=g, device="cuda").bfloat16() for _ in range(2)]
    q = torch.randn((batch.n_rows, H, hd), generator=g, device="cuda").bfloat16()
    out = torch.empty_like(q)
    rows = batch.rows(mrp)
    ctx.poll_error()
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), mrp.AttnCfg(H, hd ** -0.5, causal, window, sinks), q, out)
    assert ctx.poll_error() == 0
    batch.table.clamp_(0, batch.n_pages - 1)          # (the oracle looks pages up before it knows what a row sees)
    want, lse, mag, qk = ref.attention(batch, q, pages[0], pages[1], hd ** -0.5, causal, window, sinks)
    tol, _ = ref.attention_tolerance(torch.bfloat16, want, lse, mag, qk, hd, max(lens), few=batch.max_new * (H // Hkv) <= 32)
    ref.assert_close(out, want, tol, "out")


@pytest.mark.parametrize("new,H", [(1, 4), (16, 4), (24, 8), (70, 8)])
def test_a_missing_page_in_the_window_is_reported(ctx, new, H):
    batch = ref.Batch([new], [400], 16)
    batch.table[0, :15] = -1
    pages = [torch.randn((batch.n_pages, 16, 2, 64), device="cuda").bfloat16() for _ in range(2)]
    q = torch.randn((new, H, 64), device="cuda").bfloat16()
    rows, cfg = batch.rows(mrp), mrp.AttnCfg(H, 0.125, True, 401 - new - 240, 0)     # the first row sees positions from 240 on: page 15
    ctx.poll_error()
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), cfg, q, torch.empty_like(q))
    assert ctx.poll_error() == 0
    batch.table_d[0, 15] = -1
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), cfg, q, torch.empty_like(q))
    assert ctx.poll_error() == 128
    batch.table_d[0, 15] = int(batch.table[0, 15])
    batch.table_d[0, 24] = -1                          # the last position's
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), cfg, q, torch.empty_like(q))
    assert ctx.poll_error() == 128
