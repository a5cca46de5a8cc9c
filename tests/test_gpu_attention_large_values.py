"""Values near the end of bf16's range: sums that a lagging maximum must not carry past fp32's."""
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


@pytest.mark.parametrize("new", [1, 20, 40, 100, 200])
@pytest.mark.parametrize("score", [1.0, 5.0, 5.5, 6.0])
def test_a_large_value_of_a_later_larger_weight(ctx, new, score):
    """64 keys of score 0, then one of `score` with the value 2^121, then 63 of score -30: the average is far below 2^121."""
    hd, page = 64, 64
    k, v = (torch.zeros((2 * page, hd), device="cuda") for _ in range(2))
    k[64, 0], k[65:, 0], v[64] = score, -30.0, 2.0 ** 121
    pages = [t.bfloat16().view(2, page, 1, hd) for t in (k, v)]
    q = torch.zeros((new, 1, hd), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 1.0
    table = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    rows = mrp.NewRows(torch.tensor([128], dtype=torch.int32, device="cuda"), new)
    out = torch.empty_like(q)
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], table), mrp.AttnCfg(1, 1.0, causal=False), q, out)
    w = math.exp(score)
    want = 2.0 ** 121 * w / (64 + w + 63 * math.exp(-30.0))
    assert (out[:max(0, new - 128)] == 0).all()        # (of 200 rows, 72 are padding)
    # the result is rounded once, and its weight; the rest is a few steps of fp32
    assert ((out[max(0, new - 128):].double() - want).abs() <= want * (2 * ref.half_step(torch.bfloat16) + 2.0 ** -16 + 64 * ref.U32)).all()
