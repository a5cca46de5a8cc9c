"""mrp_paged_attention against 64 bits: lengths from nothing to long, masks that leave rows empty, pages that end inside a step,
values that are not finite in masked places, shared and missing pages, strides, graphs and streams, and a run of the cache's
operators together."""
import pytest
import torch

import mrp_inputs as mi
import paged_reference as ref
import paper_2605_18817_amd as mrp

pytestmark = pytest.mark.gpu
T = {"bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


def _pages(batch, Hkv, hd, cache, g):
    out = [torch.randn((batch.n_pages, batch.page, Hkv, hd), generator=g, device="cuda") for _ in range(2)]
    if cache == "e4m3":
        return [(p * 30).to(T[cache]) for p in out], [0.02 + 0.02 * torch.rand(Hkv, generator=g, device="cuda") for _ in range(2)]
    return [p.to(T[cache]) for p in out], [None, None]


def _run(ctx, batch, H, Hkv, hd, dtype, cache, causal=True, window=0, sinks=0, seed=0, spoil=None, gone=(), lse=True, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    pages, scales = _pages(batch, Hkv, hd, cache, g)
    q = (torch.randn((batch.n_rows, H, hd), generator=g, device="cuda") * gain).to(T[dtype])
    rows = batch.rows(mrp)
    clean = [p.clone() for p in pages]
    if spoil:
        spoil(batch, pages, clean)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d, k_scale=scales[0], v_scale=scales[1])
    out = torch.full((batch.n_rows, H, hd), 7.0, dtype=T[dtype], device="cuda")
    sums = torch.full((batch.n_rows, H), 7.0, device="cuda") if lse else None
    scale = hd ** -0.5
    ctx.poll_error()
    ctx.paged_attention(rows, paged, mrp.AttnCfg(H, scale, causal, window, sinks), q, out, lse=sums)
    flags = ctx.poll_error()
    assert flags == (128 if gone else 0)
    want, wlse, mag, qk = ref.attention(batch, q, clean[0], clean[1], scale, causal, window, sinks, scales[0], scales[1], gone)
    n = batch.cu[-1]
    tol, ltol = ref.attention_tolerance(T[dtype], want, wlse, mag, qk, hd, max(batch.kv_len), few=batch.max_new * (H // Hkv) <= 32)
    ref.assert_close(out[:n], want[:n], tol[:n], "out")
    if lse:
        ref.assert_close(sums[:n], wlse[:n], ltol[:n], "lse")
        assert (sums[n:] == 7.0).all()
    assert (out[n:] == 7.0).all()        # rows behind the last sequence
    return out, sums


LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500]


@pytest.mark.parametrize("H,Hkv,hd", [(16, 8, 128), (32, 8, 128), (12, 12, 64), (14, 2, 64), (8, 1, 256), (24, 1, 128), (40, 8, 128)])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "e4m3"), ("f16", "e4m3")])
@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 5)])
def test_single_tokens(ctx, H, Hkv, hd, dtype, cache, window, sinks):
    _run(ctx, ref.Batch([1] * len(LENGTHS), LENGTHS, 32, uniform=True), H, Hkv, hd, dtype, cache, True, window, sinks)


@pytest.mark.parametrize("page", [1, 3, 16, 48, 64, 1000])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 40, 3), (False, 33, 0), (True, 1, 70), (True, 64, 64)])
@pytest.mark.parametrize("H,hd,dtype,cache", [(8, 128, "bf16", "bf16"), (16, 128, "f16", "e4m3"), (16, 64, "bf16", "bf16")])     # 32 and 64 rows of a key head
def test_blocks_pages_and_windows(ctx, page, causal, window, sinks, H, hd, dtype, cache):
    lens = [4, 16, 17, 40, 100, 257, 1]
    new = [4, 16, 1, 7, 16, 16, 1]
    _run(ctx, ref.Batch(new, lens, page, behind=2), H, 4, hd, dtype, cache, causal, window, sinks)


@pytest.mark.parametrize("H,Hkv,hd,dtype,cache", [(8, 2, 128, "bf16", "bf16"), (4, 1, 64, "f16", "f16"), (4, 4, 256, "bf16", "bf16"),
                                                  (6, 2, 128, "f16", "e4m3"), (5, 1, 64, "bf16", "e4m3")])
@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (True, 50, 5), (False, 0, 0)])
def test_prompts(ctx, H, Hkv, hd, dtype, cache, causal, window, sinks):
    _run(ctx, ref.Batch([130, 0, 65, 1, 200], [130, 9, 200, 40, 333], 16, behind=1), H, Hkv, hd, dtype, cache, causal, window, sinks)


@pytest.mark.parametrize("causal,window,sinks", [(True, 0, 0), (False, 0, 0), (True, 5, 2)])
def test_rows_that_see_nothing(ctx, causal, window, sinks):
    """Sequences of no positions, of fewer than they have new rows, and without rows."""
    out, lse = _run(ctx, ref.Batch([1, 6, 0, 9, 3], [0, 2, 5, 9, 0], 16), 4, 2, 64, "bf16", "bf16", causal, window, sinks)
    assert (out[:5] == 0).all() and torch.isneginf(lse[:5]).all() and torch.isfinite(lse[5:7]).all() and torch.isneginf(lse[-3:]).all()


def _spoil_unseen(batch, pages, clean):
    """NaN wherever no row may look: spare pages, places behind the last position."""
    used = torch.zeros(pages[0].shape[:2], dtype=torch.bool, device="cuda")
    for b in range(batch.B):
        if batch.kv_len[b] > 0:
            used[batch.places(b, torch.arange(batch.kv_len[b]))] = True
    for p in pages:
        p[~used] = float("nan")


@pytest.mark.parametrize("page", [16, 64, 5])
@pytest.mark.parametrize("new,lens", [([1, 1, 1], [5, 33, 100]), ([16, 3, 9], [16, 40, 70]), ([100, 70], [100, 99])])
def test_not_finite_behind_the_end(ctx, page, new, lens):
    _run(ctx, ref.Batch(new, lens, page), 4, 2, 128, "bf16", "bf16", spoil=_spoil_unseen)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("new,total,at,window,sinks", [(8, 40, 39, 0, 0), (8, 40, 35, 0, 0), (8, 100, 60, 36, 2), (120, 150, 149, 0, 0), (120, 150, 70, 0, 0)])
def test_not_finite_where_some_rows_look(ctx, value, new, total, at, window, sinks):
    """Rows that do not see position `at` are as if it were any value; the others take what is there."""
    H, Hkv, hd = 4, 2, 128
    batch = ref.Batch([new], [total], 16)
    g = torch.Generator(device="cuda").manual_seed(3)
    pages, _ = _pages(batch, Hkv, hd, "bf16", g)
    q = torch.randn((new, H, hd), generator=g, device="cuda").bfloat16()
    rows = batch.rows(mrp)
    where = batch.places(0, [at])
    clean = [p.clone() for p in pages]
    pages[1][where[0], where[1], :, 5] = value
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    out = torch.empty((new, H, hd), dtype=torch.bfloat16, device="cuda")
    ctx.paged_attention(rows, paged, mrp.AttnCfg(H, 0.1, True, window, sinks), q, out)
    want, lse, mag, qk = ref.attention(batch, q, clean[0], clean[1], 0.1, True, window, sinks)
    tol, _ = ref.attention_tolerance(torch.bfloat16, want, lse, mag, qk, hd, total, few=new * 2 <= 32)
    p = torch.arange(total - new, total)
    sees = (p >= at) & ((p - window < at) if window else torch.ones_like(p, dtype=torch.bool))
    assert sees.any() and not sees.all()
    keep = torch.ones(hd, dtype=torch.bool)
    keep[5] = False
    ref.assert_close(out[(~sees).cuda()], want[(~sees).cuda()], tol[(~sees).cuda()], "rows that do not see it")
    ref.assert_close(out[sees.cuda()][:, :, keep.cuda()], want[sees.cuda()][:, :, keep.cuda()], tol[sees.cuda()][:, :, keep.cuda()], "other entries")
    assert not torch.isfinite(out[sees.cuda()][:, :, 5]).any()
    # a key that is not finite
    pages[1].copy_(clean[1])
    pages[0][where[0], where[1], :, 5] = value
    ctx.paged_attention(rows, paged, mrp.AttnCfg(H, 0.1, True, window, sinks), q, out)
    ref.assert_close(out[(~sees).cuda()], want[(~sees).cuda()], tol[(~sees).cuda()], "rows that do not see the key")


@pytest.mark.parametrize("page", [32, 24])
def test_missing_pages_are_not_seen(ctx, page):
    batch = ref.Batch([1, 16, 90], [100, 100, 130], page)
    gone = [int(batch.table[0, 1]), int(batch.table[1, 0]), int(batch.table[2, 2])]

    def lose(bt, pages, clean):
        for value, page_no in zip((-1, batch.n_pages, 2 ** 31 - 1), gone):
            bt.table_d[bt.table_d == page_no] = value
    _run(ctx, batch, 4, 2, 64, "bf16", "bf16", spoil=lose, gone=gone)


def test_lengths_beyond_the_table_are_clamped(ctx):
    batch = ref.Batch([1, 1], [64, 30], 16)
    g = torch.Generator(device="cuda").manual_seed(3)
    pages, _ = _pages(batch, 2, 64, "bf16", g)
    q = torch.randn((2, 4, 64), generator=g, device="cuda").bfloat16()
    rows, outs = batch.rows(mrp), []
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    ctx.poll_error()
    for length, flag in ((64, 0), (65, 64), (2 ** 31 - 1, 64)):
        batch.len_d[0] = length
        out = torch.empty_like(q)
        ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.125), q, out)
        assert ctx.poll_error() == flag
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
    batch.len_d[0] = -5
    ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.125), q, out)
    assert ctx.poll_error() == 64 and (out[0] == 0).all() and torch.equal(out[1], outs[0][1])


def test_large_scores(ctx):
    """Scores of hundreds: the running maximum keeps the exponentials in range."""
    _run(ctx, ref.Batch([1, 16, 70], [700, 300, 400], 16), 4, 2, 128, "f16", "f16", gain=60.0)


@pytest.mark.parametrize("new,lens", [([1], [20000]), ([1, 1, 1], [9000, 17, 3001]), ([16], [12345]), ([40], [7000])])
def test_long_caches(ctx, new, lens):
    _run(ctx, ref.Batch(new, lens, 64), 8, 2, 128, "bf16", "bf16", causal=len(new) > 1)


@pytest.mark.parametrize("window,sinks", [(0, 0), (3000, 70), (2 ** 31 - 1, 5)])
def test_long_prompts_in_pieces(ctx, window, sinks):
    """Few workgroups over a long cache: the positions are cut into pieces and joined; a window wider than any sequence is none."""
    _run(ctx, ref.Batch([100, 9], [9100, 700], 32), 4, 1, 64, "f16", "f16", True, window, sinks)


@pytest.mark.parametrize("uniform", [True, False])
def test_many_sequences(ctx, uniform):
    lens = [1 + (37 * b) % 150 for b in range(700)]
    new = [1] * 700 if uniform else [(b * 7) % 3 for b in range(700)]
    _run(ctx, ref.Batch(new, lens, 16, uniform=uniform), 4, 2, 64, "bf16", "bf16")


def test_strided_queries_and_shared_pages(ctx):
    """q as a part of a fused projection; two sequences that read the same pages give the same rows."""
    batch = ref.Batch([1, 1], [50, 50], 16)
    batch.table[1] = batch.table[0]
    g = torch.Generator(device="cuda").manual_seed(3)
    pages, _ = _pages(batch, 2, 128, "bf16", g)
    fused = torch.randn((2, 8, 128), generator=g, device="cuda").bfloat16()
    fused[1] = fused[0]
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    out, dense = (torch.empty((2, 4, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.1), fused[:, :4], out)
    ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.1), fused[:, :4].contiguous(), dense)
    assert torch.equal(out, dense) and torch.equal(out[0], out[1])


def _layer(g, H, Hkv, hd, n):
    return torch.randn((n, H + 2 * Hkv, hd), generator=g, device="cuda").bfloat16()


def test_decoding_together(ctx):
    """A prompt in two parts, then tokens, through append and attention; every step against attention over all keys so far."""
    H, Hkv, hd, page = 8, 2, 128, 16
    g = torch.Generator(device="cuda").manual_seed(9)
    total = [75, 41]
    qkv = [_layer(g, H, Hkv, hd, t) for t in total]
    gq, gk = ((1 + 0.2 * torch.randn(hd, generator=g, device="cuda")).bfloat16() for _ in range(2))
    qk = mrp.QkNormRope(H, Hkv, hd, ctx.rope_table(100, hd, 1e6), gq, gk)
    done = [0, 0]
    full = ref.Batch(total, total, page)
    pages = [torch.full((full.n_pages, page, Hkv, hd), float("nan"), device="cuda").bfloat16() for _ in range(2)]
    for step in ([40, 30], [30, 0], [1, 1], [1, 1], [3, 9]):
        lens = [a + b for a, b in zip(done, step)]
        batch = ref.Batch(step, lens, page)
        batch.table, batch.n_pages = full.table, full.n_pages
        x = torch.cat([qkv[b][done[b]:lens[b]] for b in range(2)])
        rows = batch.rows(mrp)
        paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
        q_out, out = (torch.empty((batch.n_rows, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        ctx.cache_append(rows, qk, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], paged, q_out)
        ctx.paged_attention(rows, paged, mrp.AttnCfg(H, hd ** -0.5), q_out, out)
        want, lse, mag, qkm = ref.attention(batch, q_out, pages[0], pages[1], hd ** -0.5, True, 0, 0)
        tol, _ = ref.attention_tolerance(torch.bfloat16, want, lse, mag, qkm, hd, max(lens), few=batch.max_new * 4 <= 32)
        ref.assert_close(out, want, tol, f"step {step}")
        done = lens
    for b in range(2):
        where = full.places(b, torch.arange(total[b]))
        table = ref.rope_table(100, hd)[:total[b]].float()
        want, bound = ref.norm_rope(qkv[b][:, H:H + Hkv], gk, table, 1e-6)
        ref.assert_close(pages[0][where], want, 2.0 ** -8 * want.abs() + bound * 1.01 + 2.0 ** -25, "keys")
        assert torch.equal(pages[1][where], qkv[b][:, H + Hkv:])
    assert ctx.poll_error() == 0


def test_graph_of_append_and_attention(ctx):
    """Captured once, replayed with other lengths and rows; eager work in between; every replay against the eager result."""
    H, Hkv, hd, page = 8, 2, 128, 16
    g = torch.Generator(device="cuda").manual_seed(9)
    batch = ref.Batch([1, 1, 1], [500, 300, 64], page)
    pages = [torch.randn((batch.n_pages, page, Hkv, hd), generator=g, device="cuda").bfloat16() for _ in range(2)]
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    qk = mrp.QkNormRope(H, Hkv, hd, ctx.rope_table(600, hd, 1e6))
    cfg = mrp.AttnCfg(H, hd ** -0.5)
    x = _layer(g, H, Hkv, hd, 3)
    q_out, out = (torch.empty((3, H, hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.empty((3, H), device="cuda")
    scratch = torch.empty(max(16, ctx.paged_attention_scratch_bytes(rows, paged, cfg, q_out)), dtype=torch.uint8, device="cuda")

    def step(scratch):
        ctx.cache_append(rows, qk, x[:, :H], x[:, H:H + Hkv], x[:, H + Hkv:], paged, q_out)
        ctx.paged_attention(rows, paged, cfg, q_out, out, lse=lse, scratch=scratch)

    step(scratch)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        step(scratch)
    for rep, lens in enumerate(([500, 300, 64], [17, 1, 3], [250, 0, 64], [499, 299, 33])):
        batch.len_d.copy_(torch.tensor(lens, dtype=torch.int32))
        x.copy_(_layer(g, H, Hkv, hd, 3))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone(), pages[0].clone(), pages[1].clone()
        assert torch.isfinite(torch.randn(1000, device="cuda").sum())
        out.zero_()
        step(None)
        torch.cuda.synchronize()
        for a, b in zip(got, (out, lse, pages[0], pages[1])):
            assert torch.equal(a, b), f"replay {rep}"
    assert ctx.poll_error() == 0


def test_two_graphs_on_two_streams(ctx):
    """Each with a scratch of its own, replayed side by side."""
    H, Hkv, hd, page = 8, 2, 128, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    batch = ref.Batch([1, 1], [9000, 8000], page)
    pages = [torch.randn((batch.n_pages, page, Hkv, hd), generator=g, device="cuda").bfloat16() for _ in range(2)]
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    cfg = mrp.AttnCfg(H, hd ** -0.5)
    q = [torch.randn((2, H, hd), generator=g, device="cuda").bfloat16() for _ in range(2)]
    want, out = [torch.empty_like(t) for t in q], [torch.empty_like(t) for t in q]
    for t, w in zip(q, want):
        ctx.paged_attention(rows, paged, cfg, t, w)
    torch.cuda.synchronize()
    graphs, streams = [], [torch.cuda.Stream() for _ in q]
    for t, o, st in zip(q, out, streams):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=st):
            for _ in range(4):
                ctx.paged_attention(rows, paged, cfg, t, o)
    torch.cuda.synchronize()
    for _ in range(5):
        for o in out:
            o.zero_()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(out, want))


def test_another_stream(ctx):
    batch = ref.Batch([1], [300], 16)
    g = torch.Generator(device="cuda").manual_seed(1)
    pages, _ = _pages(batch, 2, 64, "bf16", g)
    q = torch.randn((1, 4, 64), generator=g, device="cuda").bfloat16()
    rows, cfg = batch.rows(mrp), mrp.AttnCfg(4, 0.125)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    want, out = torch.empty_like(q), torch.empty_like(q)
    ctx.paged_attention(rows, paged, cfg, q, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ctx.paged_attention(rows, paged, cfg, q, out)
    side.synchronize()
    assert torch.equal(out, want)


def test_append_fills_the_prefix_caches_of_the_transformer_body():
    """A contiguous prefix cache is one page a sequence: the chain reads what mrp_cache_append wrote there."""
    from harness import dev_bits
    from test_gpu_tbody import TfProblem
    cfg = mi.config(0, B=3, L=4, K=1)
    td = mi.TBodyDims(D=1, n_heads=4, n_kv_heads=2, head_dim=128, d_ff=256, P_max=50)
    prob = TfProblem(cfg, td)
    try:
        g = torch.Generator(device="cuda").manual_seed(4)
        plen = [50, 7, 23]
        x = torch.randn((sum(plen), td.n_heads + 2 * td.n_kv_heads, 128), generator=g, device="cuda").bfloat16()
        qk = mrp.QkNormRope(td.n_heads, td.n_kv_heads, 128, prob.ctx.rope_table(64, 128, td.rope_theta))
        filled, by_hand = ([torch.zeros((cfg.B, td.P_max, td.n_kv_heads, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)] for _ in range(2))
        table = torch.arange(cfg.B, dtype=torch.int32, device="cuda")[:, None].contiguous()
        cu = torch.tensor([0, 50, 57, 80], dtype=torch.int32, device="cuda")
        lens = torch.tensor(plen, dtype=torch.int32, device="cuda")
        k, v = x[:, td.n_heads:td.n_heads + td.n_kv_heads], x[:, td.n_heads + td.n_kv_heads:]
        prob.ctx.cache_append(mrp.NewRows(lens, 50, cu_rows=cu), qk, None, k, v, mrp.PagedCache(filled[0], filled[1], table), None)
        # the same values put there by torch
        k_out = torch.empty((sum(plen), td.n_kv_heads, 128), dtype=torch.bfloat16, device="cuda")
        pos = torch.cat([torch.arange(n) for n in plen]).int().cuda()
        kq = mrp.QkNormRope(td.n_kv_heads, 0, 128, qk.tensors[0])
        prob.ctx.qk_norm_rope(kq, pos, k, None, k_out, None)
        seq = torch.repeat_interleave(torch.arange(3), torch.tensor(plen)).cuda()
        by_hand[0][seq, pos.long()], by_hand[1][seq, pos.long()] = k_out, v
        outs = []
        for kc, vc in (filled, by_hand):
            lay = prob.layers_d[0]
            layers = [mrp.TLayer(lay.Wqkv_packed, lay.Wo_packed, lay.Wgu_packed, lay.Wdown_packed, lay.g1, lay.g2, kc, vc)]
            z, hr = torch.from_numpy(mi.logits0(cfg)).cuda(), torch.zeros((cfg.M, cfg.d), device="cuda")
            io = mrp.StepIO(cfg.B, cfg.L, 1)
            prob.ctx.chain_step_tf(cfg.B, 1, dev_bits(mi.hidden(cfg)), hr, prob.E_d, prob.Wp_d, prob.heads_d, layers, lens, z, mrp.RevealCfg(), io)
            outs.append((z, hr, io.tok))
        assert all(torch.equal(a, b) for a, b in zip(*outs))
        want, bound = ref.norm_rope(k, None, ref.rope_table(64, 128, td.rope_theta)[pos.long()].float(), 1e-6)
        ref.assert_close(filled[0][seq, pos.long()], want, 2.0 ** -8 * want.abs() + bound * 1.01 + 2.0 ** -25, "keys")
    finally:
        prob.close()


def test_binding_refuses_what_does_not_fit(ctx):
    batch = ref.Batch([1], [30], 16)
    pages, _ = _pages(batch, 2, 64, "bf16", torch.Generator(device="cuda").manual_seed(1))
    rows = batch.rows(mrp)
    paged = mrp.PagedCache(pages[0], pages[1], batch.table_d)
    q, out = (torch.zeros((1, 4, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cfg = mrp.AttnCfg(4, 0.125)
    ctx.paged_attention(rows, paged, cfg, q, out)
    bad = [lambda: ctx.paged_attention(rows, paged, cfg, q.half(), out),                       # another type than the cache
           lambda: ctx.paged_attention(rows, paged, cfg, q[:, :, :32], out),
           lambda: ctx.paged_attention(rows, paged, cfg, q.transpose(1, 2), out),
           lambda: ctx.paged_attention(rows, paged, mrp.AttnCfg(3, 0.125), q[:, :3], out[:, :3].contiguous()),
           lambda: ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.0), q, out),
           lambda: ctx.paged_attention(rows, paged, mrp.AttnCfg(4, 0.1, window=-1), q, out),
           lambda: ctx.paged_attention(rows, paged, cfg, q, out, lse=torch.zeros((1, 3), device="cuda")),
           lambda: ctx.paged_attention(rows, paged, cfg, q.cpu(), out),
           lambda: ctx.paged_attention(mrp.NewRows(torch.tensor([3, 4], dtype=torch.int32, device="cuda"), 1), paged, cfg, q, out),
           lambda: mrp.NewRows(torch.tensor([3], device="cuda"), 1),                           # int64 lengths
           lambda: mrp.PagedCache(pages[0], pages[1].half(), batch.table_d),
           lambda: mrp.PagedCache(pages[0].float(), pages[1].float(), batch.table_d),
           lambda: ctx.cache_append(rows, mrp.QkNormRope(4, 1, 64), None, q[:, :1], q[:, :1], paged, None),
           lambda: ctx.cache_append(rows, mrp.QkNormRope(4, 2, 64), q, q[:, :2], q[:, :2], paged, None),
           lambda: ctx.qk_norm_rope(mrp.QkNormRope(4, 0, 64), None, q, None, out.float(), None),   # bf16 -> fp32: no such form
           lambda: ctx.qk_norm_rope(mrp.QkNormRope(4, 0, 64, ctx.rope_table(8, 64, 1e4)), None, q, None, out, None)]
    for n, call in enumerate(bad):
        with pytest.raises(mrp.MrpError):
            call()
            print("not refused:", n)
    torch.cuda.synchronize()
