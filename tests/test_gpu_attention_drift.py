"""Rows of one tile share their keys, not their maxima: a row whose maximum stays is not touched when another's grows."""
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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_equal_scores_next_to_growing_ones(ctx, dtype):
    """Head 0 has the same score, 520.40625, at all 32768 positions; head 1's grows with every 32 of them.  Values are 0 in the first
    half and 1 in the second, so that head 0's output is 1/2 and its log-sum 520.40625 + ln 32768: all products are exact.
    In units of log 2 the score is 750.7875061, half a step of fp32 from its rounding: a factor of 2^(that half step) for every
    time that head 1's maximum grows would add up to 3e-3."""
    n, B, page, hd = 32768, 512, 64, 64
    step = torch.arange(n, device="cuda") // 32
    k, v = (torch.zeros((n, hd), device="cuda") for _ in range(2))
    k[:, 0], k[:, 1], k[:, 2] = 22.75, step % 256, step // 256
    v[n // 2:] = 1.0
    pages = [t.to(dtype).view(n // page, page, 1, hd) for t in (k, v)]
    q = torch.zeros((B, 2, hd), dtype=dtype, device="cuda")
    q[:, 0, 0], q[:, 1, 1], q[:, 1, 2] = 22.875, 0.5, 128.0
    table = torch.arange(n // page, dtype=torch.int32, device="cuda").repeat(B, 1)      # (all sequences read the same pages)
    rows = mrp.NewRows(torch.full((B,), n, dtype=torch.int32, device="cuda"), 1)
    out, lse = torch.empty_like(q), torch.empty((B, 2), device="cuda")
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], table), mrp.AttnCfg(2, 1.0), q, out, lse=lse)
    want = 520.40625 + math.log(n)
    # log 2's constants, the score in units of it and back, and the sum: six half steps of the score; a lane adds 256 times 8 weights
    assert (lse[:, 0].double() - want).abs().max() <= ref.U32 * (6 * want + 400)
    # 1/2 is exact; both halves of the sum are off by the chain of its additions at most
    assert (out[:, 0].double() - 0.5).abs().max() <= 0.5 * ref.half_step(dtype) + 400 * ref.U32
