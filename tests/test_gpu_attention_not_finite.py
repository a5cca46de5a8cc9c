"""Rows of mrp_paged_attention whose scores are not numbers: what the definition gives, softmax(scores) v in 64 bits, and zeros only
for rows that see nothing."""
import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


# new rows, kv_len, H, Hkv, hd, dtype, cache: each form of the kernels, whole and in pieces that are joined
FORMS = [
    ([1], [1], 4, 2, 64, "bf16", "bf16"),
    ([1, 1, 1], [1, 40, 700], 16, 2, 128, "bf16", "bf16"),
    ([1, 1], [33, 20000], 8, 1, 64, "f16", "f16"),
    ([4, 8], [30, 600], 8, 2, 128, "f16", "e4m3"),            # 32 rows of a key head
    ([1, 4], [5, 300], 8, 1, 256, "bf16", "bf16"),
    ([8, 8], [9, 300], 8, 1, 256, "bf16", "e4m3"),            # 64 rows, heads of 256
    ([10, 16], [12, 500], 8, 2, 128, "bf16", "bf16"),         # 64 rows
    ([16], [9000], 8, 2, 64, "f16", "e4m3"),
    ([24, 20], [24, 300], 8, 2, 128, "f16", "f16"),           # 96 rows
    ([32], [5000], 4, 1, 64, "bf16", "e4m3"),
    ([70, 3], [70, 90], 8, 2, 64, "bf16", "bf16"),            # 280 rows
    ([100], [9000], 4, 1, 128, "bf16", "bf16"),
]


def _inputs(form, seed=0):
    new, lens, H, Hkv, hd, dtype, cache = form
    batch = ref.Batch(new, lens, 16)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages = [torch.randn((batch.n_pages, 16, Hkv, hd), generator=g, device="cuda").to(T[cache]) for _ in range(2)]
    q = torch.randn((batch.n_rows, H, hd), generator=g, device="cuda").to(T[dtype])
    return batch, q, pages


def _put(pages, where, column, value):
    """pages[where][:, column] = value, of any type of cache (there is no indexed store of 8-bit floats)."""
    bits = torch.full((), value, device="cuda").to(pages.dtype)
    raw = torch.uint8 if pages.dtype == torch.float8_e4m3fn else torch.int16
    some = pages.view(raw)[where]
    some[..., column] = bits.view(raw)
    pages.view(raw)[where] = some


def _attend(ctx, batch, q, pages, causal=True, scale=0.125):
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    rows = batch.rows(mrp)
    ctx.paged_attention(rows, mrp.PagedCache(pages[0], pages[1], batch.table_d), mrp.AttnCfg(q.shape[1], scale, causal), q, out, lse=lse)
    return out, lse


def _check(batch, q, pages, got, causal=True, scale=0.125, finite_keys=None):
    out, lse = got
    G = q.shape[1] // pages[0].shape[2]
    want, wlse, mag, qk = ref.attention(batch, q, pages[0].to(q.dtype), pages[1].to(q.dtype), scale, causal, 0, 0)
    if finite_keys is not None:        # (the bound goes by the scores' magnitudes, infinite ones apart)
        qk = ref.attention(batch, q, finite_keys, pages[1], scale, causal, 0, 0)[3]
    tol, ltol = ref.attention_tolerance(q.dtype, want, wlse, mag, qk, q.shape[2], max(batch.kv_len), few=batch.max_new * G <= 32)
    assert torch.equal(torch.isnan(out), torch.isnan(want)), "out: other entries are NaN"
    ref.assert_close(out, want, tol.nan_to_num(0.0), "out")
    assert torch.equal(torch.isneginf(lse), torch.isneginf(wlse)), "lse: other entries are -inf"
    ref.assert_close(lse, wlse, ltol.nan_to_num(0.0), "lse")


@pytest.mark.parametrize("value", [NAN, INF, -INF])
@pytest.mark.parametrize("form", FORMS)
def test_queries(ctx, form, value):
    """One entry of a query that is not finite: its row of that head is NaN, the others are as ever."""
    batch, q, pages = _inputs(form)
    for row in {0, batch.n_rows // 2, batch.n_rows - 1}:
        q[row, row % q.shape[1], 3] = value
    _check(batch, q, pages, _attend(ctx, batch, q, pages))


@pytest.mark.parametrize("form", FORMS)
def test_all_keys(ctx, form):
    """Every key of a head that a sequence has."""
    batch, q, pages = _inputs(form, 1)
    _put(pages[0][:, :, -1], slice(None), 5, NAN)
    _check(batch, q, pages, _attend(ctx, batch, q, pages))


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("first,count", [(0, 1), (0, 32), (0, 300), (128, 32), (-1, 1)])
def test_some_keys(ctx, form, first, count):
    """A stretch of keys, as long as a wave's step or a piece of the positions, or one: NaN in out and in lse for the rows that see it."""
    batch, q, pages = _inputs(form, 2)
    for b in range(batch.B):
        at = torch.arange(batch.kv_len[b])
        at = at[at >= batch.kv_len[b] - 1] if first < 0 else at[(at >= first) & (at < first + count)]
        if len(at):
            _put(pages[0], batch.places(b, at), 2, NAN)
    _check(batch, q, pages, _attend(ctx, batch, q, pages))


@pytest.mark.parametrize("scale", [0.125, 3.0])
@pytest.mark.parametrize("form", [f for f in FORMS if f[6] != "e4m3"])
@pytest.mark.parametrize("count", [1, 32, 200, 10 ** 6])
def test_scores_of_minus_infinity(ctx, form, count, scale):
    """The first `count` keys give -inf: they weigh nothing where there are others, and leave NaN (lse: -inf) where there are none."""
    batch, q, pages = _inputs(form, 3)
    q[:, :, 0] = q[:, :, 0].abs() + 0.5
    finite = pages[0].clone()
    for b in range(batch.B):
        where = batch.places(b, torch.arange(min(count, batch.kv_len[b])))
        _put(pages[0], where, 0, -INF)
        _put(finite, where, 0, 0.0)
    _check(batch, q, pages, _attend(ctx, batch, q, pages, scale=scale), scale=scale, finite_keys=finite)


@pytest.mark.parametrize("new,lens,H", [([1, 3, 2], [0, 1, 0], 4), ([9, 20], [4, 0], 4), ([40, 30], [10, 0], 4), ([80], [0], 4)])
def test_rows_that_see_nothing(ctx, new, lens, H):
    """Padding stays zero and -inf whatever its query holds; so does a sequence whose pages are not there."""
    ctx.poll_error()
    batch = ref.Batch(new, lens, 16)
    pages = [torch.randn((batch.n_pages, 16, 2, 64), device="cuda").bfloat16() for _ in range(2)]
    q = torch.full((batch.n_rows, H, 64), NAN, device="cuda").bfloat16()
    out, lse = _attend(ctx, batch, q, pages)
    for b, (n, total) in enumerate(zip(new, lens)):
        empty = max(0, n - total)
        o, s = out[batch.cu[b]:batch.cu[b + 1]], lse[batch.cu[b]:batch.cu[b + 1]]
        assert (o[:empty] == 0).all() and torch.isneginf(s[:empty]).all()
        assert torch.isnan(o[empty:]).all() and torch.isnan(s[empty:]).all()
    batch = ref.Batch(new, [50] * len(new), 16, max_pages=4)
    batch.table[:] = -1
    out, lse = _attend(ctx, batch, q, pages, causal=False)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert ctx.poll_error() == 128
