"""fp16 weights far below the largest one: many of them add up, in the product as in the sum."""
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


# new rows (of one head): the form for up to 32 rows, and the three for more; heads of 64, 128 and 256
@pytest.mark.parametrize("new,hd", [(1, 64), (1, 128), (20, 128), (3, 256), (40, 64), (40, 128), (100, 128), (200, 64)])
@pytest.mark.parametrize("cache", [torch.float16, torch.float8_e4m3fn])
@pytest.mark.parametrize("keys,tail", [(4096, 17.75), (4096, 11.5), (1000, 15.0), (4090, 20.0)])
def test_a_long_tail_behind_large_weights(ctx, new, hd, cache, keys, tail):
    """Positions 0, 32, 64 and 96 (one for every wave that takes the positions in turn) weigh 1 and have the value 0; the others weigh
    exp(-tail) each (2^-25.6, 2^-16.6, 2^-21.6, 2^-28.9), with values of 1, 1.5 and -0.25 by turns.  All products are exact.  So many
    sequences read the same pages that none is cut into pieces."""
    page, B = 64, 1536
    n_pages = -(-keys // page)
    k, v = (torch.zeros((n_pages * page, hd), device="cuda") for _ in range(2))
    values = torch.tensor([1.0, 1.5, -0.25], device="cuda").repeat(hd)[:hd]
    k[:, 0], v[:] = -0.5, values
    for t in (k, v):
        t[[0, 32, 64, 96]] = 0.0
    pages = [t.to(cache).view(n_pages, page, 1, hd) for t in (k, v)]
    q = torch.zeros((B * new, 1, hd), dtype=torch.float16, device="cuda")
    q[:, 0, 0] = 2 * tail
    table = torch.arange(n_pages, dtype=torch.int32, device="cuda").repeat(B, 1)
    rows = mrp.NewRows(torch.full((B,), keys, dtype=torch.int32, device="cuda"), new)
    out, lse = torch.empty_like(q), torch.empty((B * new, 1), device="cuda")
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], table), mrp.AttnCfg(1, 1.0, causal=False), q, out, lse=lse)
    w = math.exp(-tail)
    total = 4 + (keys - 4) * w
    want = values.double() * ((keys - 4) * w / total)
    # a weight is off by half of fp16's smallest step, 2^-25, at most, where the largest is 2^10 (up to 32 rows, heads of 256) or 2^7; by
    # its exponential's and the chain's steps; in one term (more rows) by half a step of its own
    few = new <= 32 or hd == 256
    floor = 2.0 ** -25 * 2.0 ** -(10 if few else 7) * (keys - 4) / total
    own = ref.U32 * (keys + 64 + 8 + 4 * tail) + (0 if few else 2.0 ** -11)
    tol = ref.half_step(torch.float16) * want.abs() + floor * values.double().abs() + own * want.abs() + 2.0 ** -25
    err = (out[:, 0].double() - want).abs()
    assert (err <= tol).all(), f"{float((err / tol).max()):.2f} x the bound"
    assert (lse.double() - math.log(total)).abs().max() <= ref.U32 * (keys + 64 + 8 + 4 * tail)
