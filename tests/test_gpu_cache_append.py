"""mrp_cache_append against 64 bits: what is written, that nothing else is, and what it refuses or skips."""
import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp

pytestmark = pytest.mark.gpu
EPS = 1e-6
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


def _bits(t):
    return t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t.view(torch.int16)


FORMS = [   # new rows, kv_len, page, uniform, H, Hkv, hd, rot, x, y, cache, with q
    ([1] * 5, [1, 2, 16, 17, 300], 16, True, 16, 8, 128, 128, "bf16", "bf16", "bf16", True),
    ([4, 4, 4], [4, 33, 70], 64, True, 32, 8, 128, 128, "f32", "bf16", "e4m3", True),
    ([5, 0, 1, 130, 0], [5, 7, 1, 131, 0], 48, False, 14, 2, 64, 32, "f16", "f16", "f16", True),
    ([3, 40], [50, 41], 1, False, 3, 1, 256, 256, "f32", "f16", "e4m3", True),
    ([3, 40], [50, 41], 7, False, 4, 4, 64, 0, "bf16", "bf16", "bf16", False),
    ([6, 2, 9], [4, 0, 9], 16, False, 4, 2, 128, 128, "bf16", "bf16", "bf16", True),     # padding: positions -2 .. , none
    ([1] * 300, [1 + 3 * b for b in range(300)], 32, False, 4, 2, 64, 64, "bf16", "bf16", "bf16", True),
]


@pytest.mark.parametrize("new,lens,page,uniform,H,Hkv,hd,rot,x,y,cache,with_q", FORMS)
def test_append(ctx, new, lens, page, uniform, H, Hkv, hd, rot, x, y, cache, with_q):
    batch = ref.Batch(new, lens, page, behind=0 if uniform else 3, uniform=uniform)
    g = torch.Generator(device="cuda").manual_seed(5)
    N = batch.n_rows
    qkv = torch.randn((N, H + 2 * Hkv, hd), generator=g, device="cuda").mul(2).to(T[x])
    q, k, v = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
    gq, gk = ((1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).bfloat16() for _ in range(2))
    rope = ctx.rope_table(1000, rot, 1e6) if rot else None
    pages = [torch.randn((batch.n_pages, page, Hkv, hd), generator=g, device="cuda").to(T[cache]) for _ in range(2)]
    before = [p.clone() for p in pages]
    scales = [0.01 + 0.02 * torch.rand(Hkv, generator=g, device="cuda") for _ in range(2)] if cache == "e4m3" else [None, None]
    q_out = torch.full((N, H, hd), 7.0, dtype=T[y], device="cuda") if with_q else None
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d, k_scale=scales[0], v_scale=scales[1])
    ctx.cache_append(rows, mrp.QkNormRope(H, Hkv, hd, rope, gq, gk, eps=EPS), q if with_q else None, k, v, paged, q_out)
    written = torch.zeros((batch.n_pages, page), dtype=torch.bool, device="cuda")
    for b in range(batch.B):
        n, at = new[b], batch.cu[b]
        pos = torch.arange(lens[b] - n, lens[b])
        real = pos >= 0
        if with_q and n:
            assert (q_out[at:at + n][(~real).cuda()] == 0).all()
        if not real.any():
            continue
        r = torch.arange(at, at + n)[real].cuda()
        table = None if rope is None else rope[pos[real].cuda()]
        if with_q:
            want, bound = ref.norm_rope(q[r], gq, table, EPS)
            ref.assert_close(q_out[r], want, ref.half_step(T[y]) * want.abs() + bound * (1 + 2 ** -7) + 2.0 ** -25, "q")
        where = batch.places(b, pos[real])
        written[where] = True
        kk, kbound = ref.norm_rope(k[r], gk, table, EPS)
        vv = v[r].double()
        for what, got, want, bound, sc in (("k", pages[0][where], kk, kbound, scales[0]), ("v", pages[1][where], vv, torch.zeros_like(vv), scales[1])):
            if cache == "e4m3":
                want, bound = want / sc.double()[:, None], bound / sc.double()[:, None] + ref.U32 * want.abs() / sc.double()[:, None]
                want = want.clamp(-448, 448)
                ref.assert_close(got.float(), want, ref.e4m3_tolerance(want) + bound * 1.1, what)
            else:
                ref.assert_close(got, want, ref.half_step(T[cache]) * want.abs() + bound * (1 + 2 ** -7) + 2.0 ** -25, what)
    for p, was in zip(pages, before):
        assert torch.equal(_bits(p)[~written], _bits(was)[~written])      # nothing else is written
    if with_q:
        assert (q_out[batch.cu[-1]:] == 7.0).all()                        # rows behind the last sequence
    assert ctx.poll_error() == 0


def test_e4m3_edges(ctx):
    """Ties to even, subnormals, saturation, infinities and NaN, as the values they stand for."""
    x = torch.tensor([0.0, -0.0, 1.0, 1.0625, 1.1875, 448.0, 449.0, 464.0, 1e6, -1e6, 2.0 ** -9, 2.0 ** -10, 3 * 2.0 ** -10, float("inf"), float("-inf"), float("nan")], device="cuda")
    want = torch.tensor([0.0, 0.0, 1.0, 1.0, 1.25, 448.0, 448.0, 448.0, 448.0, -448.0, 2.0 ** -9, 0.0, 2.0 ** -8, 448.0, -448.0, float("nan")], device="cuda")
    v = x.repeat(4).view(1, 1, 64)
    pages = [torch.zeros((1, 2, 1, 64), device="cuda").to(torch.float8_e4m3fn) for _ in range(2)]
    one = torch.ones(1, dtype=torch.int32, device="cuda")
    paged = mrp.PagedCache(pages[0], pages[1], torch.zeros((1, 1), dtype=torch.int32, device="cuda"))
    ctx.cache_append(mrp.NewRows(one, 1), mrp.QkNormRope(1, 1, 64), None, torch.zeros_like(v), v, paged, None)
    got = pages[1][0, 0, 0].float()
    assert torch.equal(got.nan_to_num(nan=99.0), want.repeat(4).nan_to_num(nan=99.0))


def test_bad_indices_are_skipped_and_reported(ctx):
    """A page that is not there, a length beyond the table, rows beyond max_new: the rest is written all the same."""
    batch = ref.Batch([2, 2, 5], [20, 40, 9], 16, max_pages=3)
    k = torch.randn((batch.n_rows, 2, 64), device="cuda").bfloat16()
    pages = [torch.full((batch.n_pages, 16, 2, 64), 3.0, device="cuda").bfloat16() for _ in range(2)]
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    qk = mrp.QkNormRope(2, 2, 64)
    ctx.poll_error()
    for value in (-1, batch.n_pages, 2 ** 31 - 1, -2 ** 31):
        batch.table_d[0, 1] = value
        ctx.cache_append(rows, qk, None, k, k, paged, None)
        assert ctx.poll_error() == 128 and "page" in ctx.last_error()
    pg, pl = batch.places(1, [38, 39])
    assert torch.equal(pages[1][pg, pl], k[2:4])
    batch.table_d[0, 1] = int(batch.table[0, 1])
    batch.len_d[1] = 49                                    # 3 pages of 16 hold 48: the new rows end at 48
    ctx.cache_append(rows, qk, None, k, k, paged, None)
    assert ctx.poll_error() == 64
    batch.len_d[1] = 40
    batch.cu_d[1] = 10 ** 9                                # sequence 0 ends beyond the rows, sequence 1 begins there
    ctx.cache_append(rows, qk, None, k, k, paged, None)
    assert ctx.poll_error() & 32
    batch.cu_d[1] = 2
    few = mrp.NewRows(batch.len_d, 3, cu_rows=batch.cu_d)   # sequence 2 has five rows
    for p in pages:
        p.fill_(3.0)
    ctx.cache_append(few, qk, None, k, k, paged, None)
    assert ctx.poll_error() == 32
    pg, pl = batch.places(2, [6, 7, 8])
    assert torch.equal(pages[1][pg, pl], k[4:7])           # its first three, as its last positions


def test_places_beyond_four_gigabytes(ctx):
    n_pages, page, Hkv, hd = 5000, 256, 16, 128            # 5.2 GB of keys, as many of values
    pages = [torch.zeros((n_pages, page, Hkv, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    table = torch.tensor([[n_pages - 1], [4100], [0]], dtype=torch.int32, device="cuda")
    paged = mrp.PagedCache(pages[0], pages[1], table)
    k = torch.randn((3, Hkv, hd), device="cuda").bfloat16()
    v = torch.randn((3, Hkv, hd), device="cuda").bfloat16()
    lens = torch.tensor([256, 17, 1], dtype=torch.int32, device="cuda")
    ctx.cache_append(mrp.NewRows(lens, 1), mrp.QkNormRope(Hkv, Hkv, hd), None, k, v, paged, None)
    for i, (pg, pl) in enumerate(((n_pages - 1, 255), (4100, 16), (0, 0))):
        assert torch.equal(pages[0][pg, pl], k[i]) and torch.equal(pages[1][pg, pl], v[i])
    q, out = torch.randn((3, Hkv, hd), device="cuda").bfloat16(), torch.empty((3, Hkv, hd), dtype=torch.bfloat16, device="cuda")
    # the last row alone in a window of one: its output is its value
    ctx.paged_attention(mrp.NewRows(lens, 1), paged, mrp.AttnCfg(Hkv, 0.1, window=1), q, out)
    assert torch.equal(out, v)
