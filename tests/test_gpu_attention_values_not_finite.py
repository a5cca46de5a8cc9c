"""Values that are not finite, in every form of mrp_paged_attention: they reach the entries of the rows that see them, and nothing else."""
import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp
from test_gpu_attention_not_finite import FORMS, INF, NAN, T, _attend, _put

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


@pytest.mark.parametrize("form,value", [(f, v) for f in FORMS for v in (NAN, INF, -INF) if v != v or f[6] != "e4m3"])     # (8 bits have no infinity)
@pytest.mark.parametrize("back", [1, 3, 40, 70])
def test_values(ctx, form, value, back):
    """Position kv_len - back of every sequence, entry 5 of the last key head: the rows before it are as if it were any value."""
    new, lens, H, Hkv, hd, dtype, cache = form
    batch = ref.Batch(new, lens, 16)
    g = torch.Generator(device="cuda").manual_seed(4)
    pages = [torch.randn((batch.n_pages, 16, Hkv, hd), generator=g, device="cuda").to(T[cache]) for _ in range(2)]
    clean = pages[1].to(T[dtype])
    q = torch.randn((batch.n_rows, H, hd), generator=g, device="cuda").to(T[dtype])
    sees = torch.zeros(batch.n_rows, dtype=torch.bool, device="cuda")
    for b, (n, total) in enumerate(zip(new, lens)):
        at = total - back
        if at < 0:
            continue
        _put(pages[1][:, :, -1], batch.places(b, [at]), 5, value)
        p = torch.arange(total - n, total)
        sees[batch.cu[b]:batch.cu[b + 1]] = (p >= at).cuda()
    out, lse = _attend(ctx, batch, q, pages)
    want, wlse, mag, qk = ref.attention(batch, q, pages[0].to(T[dtype]), clean, 0.125, True, 0, 0)
    tol, ltol = ref.attention_tolerance(T[dtype], want, wlse, mag, qk, hd, max(lens), few=batch.max_new * (H // Hkv) <= 32)
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[:, H - H // Hkv:, 5] = sees[:, None]
    assert not torch.isfinite(out[hit]).any()
    ref.assert_close(torch.where(hit, 0.0, out.double()), torch.where(hit, 0.0, want), tol, "out")
    ref.assert_close(lse, wlse, ltol, "lse")


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("window,sinks", [(20, 0), (50, 3), (33, 40)])
def test_values_and_keys_that_no_row_sees(ctx, form, window, sinks):
    """Behind the window, between the first tokens and it, behind the end, in other pages: NaN."""
    new, lens, H, Hkv, hd, dtype, cache = form
    batch = ref.Batch(new, lens, 16)
    g = torch.Generator(device="cuda").manual_seed(5)
    pages = [torch.randn((batch.n_pages, 16, Hkv, hd), generator=g, device="cuda").to(T[cache]) for _ in range(2)]
    clean = [p.to(T[dtype]) for p in pages]
    unused = torch.ones(pages[0].shape[:2], dtype=torch.bool, device="cuda")
    for b, (n, total) in enumerate(zip(new, lens)):
        j = torch.arange(total)
        j = j[(j >= max(0, total - n + 1 - window)) | (j < sinks)]
        unused[batch.places(b, j)] = False
    where = tuple(unused.nonzero().T)
    for p in pages:
        raw = torch.uint8 if cache == "e4m3" else torch.int16
        p.view(raw)[where] = torch.full((), NAN, device="cuda").to(T[cache]).view(raw)
    q = torch.randn((batch.n_rows, H, hd), generator=g, device="cuda").to(T[dtype])
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    rows = batch.rows(mrp)
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), mrp.AttnCfg(H, 0.125, True, window, sinks), q, out, lse=lse)
    want, wlse, mag, qk = ref.attention(batch, q, *clean, 0.125, True, window, sinks)
    tol, ltol = ref.attention_tolerance(T[dtype], want, wlse, mag, qk, hd, max(lens), few=batch.max_new * (H // Hkv) <= 32)
    ref.assert_close(out, want, tol, "out")
    ref.assert_close(lse, wlse, ltol, "lse")
