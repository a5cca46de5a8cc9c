"""mrp_paged_attention in the forms that go by the rows of a key head and the head size: 65 to 128 rows, whole and cut into pieces, and heads
of 256 over caches of 8 bits, against 64 bits."""
import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp
from test_gpu_paged_attention import _run

pytestmark = pytest.mark.gpu
TYPES = [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")]


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


# (65, 96 and 128 rows of a key head; sequences with fewer rows, none, and padding among them)
ROWS = [(5, 1, [13, 13, 0, 1], [13, 200, 7, 90]), (4, 1, [24, 3, 24], [500, 3, 20]), (8, 2, [32, 31, 17], [32, 129, 300])]


@pytest.mark.parametrize("H,Hkv,new,lens", ROWS)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("page", [16, 64, 7])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 40, 5), (False, 70, 66)])
def test_65_to_128_rows(ctx, H, Hkv, new, lens, hd, dtype, cache, page, causal, window, sinks):
    _run(ctx, ref.Batch(new, lens, page, behind=2), H, Hkv, hd, dtype, cache, causal, window, sinks)


@pytest.mark.parametrize("H,Hkv,new,lens", [(5, 1, [13, 13, 5], [5000, 200, 5]), (8, 2, [32, 20, 1, 25], [3100, 4000, 256, 700]), (4, 1, [24], [9001])])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 1000, 70)])
def test_65_to_128_rows_in_pieces(ctx, H, Hkv, new, lens, hd, dtype, cache, causal, window, sinks):
    """Few row tiles behind long caches: cut into pieces of one size, some sequences shorter than one, and joined."""
    batch = ref.Batch(new, lens, 48)
    rows = batch.rows(mrp)
    pages = torch.empty((batch.n_pages, 48, Hkv, hd), dtype=torch.bfloat16, device="cuda")
    q = torch.empty((batch.n_rows, H, hd), dtype=torch.bfloat16, device="cuda")
    assert ctx.paged_attention_scratch_bytes(rows, mrp.PagedCache(pages, pages, batch.table_d), mrp.AttnCfg(H, 1.0), q) > 0
    _run(ctx, batch, H, Hkv, hd, dtype, cache, causal, window, sinks)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("new,lens", [([24, 13], [100, 130]), ([32], [4000])])
def test_missing_pages(ctx, dtype, cache, hd, new, lens):
    batch = ref.Batch(new, lens, 16)
    gone = [int(batch.table[0, 1]), int(batch.table[-1, 0])]

    def lose(bt, pages, clean):
        for value, page_no in zip((-1, batch.n_pages), gone):
            bt.table_d[bt.table_d == page_no] = value
    _run(ctx, batch, 4, 1, hd, dtype, cache, spoil=lose, gone=gone)


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("new,lens", [([2, 1], [2, 300]), ([4, 3, 0], [90, 400, 5]), ([8, 5], [8, 333]), ([13, 20], [900, 20]), ([16], [5000])])    # 16 to 160 rows
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 50, 5)])
def test_heads_of_256(ctx, dtype, cache, new, lens, page, causal, window, sinks):
    _run(ctx, ref.Batch(new, lens, page, behind=1), 8, 1, 256, dtype, cache, causal, window, sinks)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "e4m3")])
@pytest.mark.parametrize("hd", [64, 128, 256])
def test_prompts_and_tokens_in_one_batch(ctx, dtype, cache, hd):
    """Single tokens, a block and a prompt side by side take the form of the longest; each is right."""
    _run(ctx, ref.Batch([1, 150, 1, 16, 0, 1], [700, 150, 1, 300, 40, 3000], 32), 4, 1, hd, dtype, cache)
