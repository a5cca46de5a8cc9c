"""The operators of a paged key-value cache, as cases that can be timed.

Three operators work on the queries, keys and values of one decoder layer:

* ``norm_rope``: every head of q and k is normalised (root mean square over the head, then a gain that all heads
  share) and rotated by its row's position; a training step takes its gradients too;
* ``append``: the same on the way into a cache whose positions lie in pages, with the values beside the keys;
* ``attend``: softmax attention of the new rows over the cache: single tokens, blocks whose rows see each other,
  prompts with a causal mask, a sliding window behind which the first tokens stay visible.

With ``own`` false, ``run`` computes them from elementary torch operations in 32 bits; with ``own`` true, it calls
the framework.  Head counts are those of the transformer head body's configurations (16 and 32 query heads over 8
key heads of 128) and generic ones; blocks have 4 to 16 positions, caches up to 32768.

A case says: rows (norm_rope) or B sequences with ``new`` rows each, ragged or alike, behind ``lo`` to ``hi`` cached
positions (the lengths follow from ``lens``, spread over their logarithm).
"""
from __future__ import annotations

import functools
import math
import random

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "e4m3": torch.float8_e4m3fn}
SIZE = {"f32": 4, "bf16": 2, "f16": 2, "e4m3": 1}
EPS = 1e-6
THETA = 1.0e6
E4M3_MAX = 448.0


def listed():
    return [
        # the rows of four sequences of one block each: a launch is all that it costs
        dict(name="norm_rope_block", op="norm_rope", grad=False, rows=64, H=16, Hkv=8, hd=128, rot=128, dtype="bf16"),
        # forward pass of a training batch of four sequences of 4096 tokens
        dict(name="norm_rope_forward", op="norm_rope", grad=False, rows=16384, H=32, Hkv=8, hd=128, rot=128, dtype="bf16"),
        # ... and its backward pass
        dict(name="norm_rope_backward", op="norm_rope", grad=True, rows=16384, H=32, Hkv=8, hd=128, rot=128, dtype="bf16"),
        # a small model trained in 32 bits: odd row count, short heads, half of each head rotated
        dict(name="norm_rope_backward_f32", op="norm_rope", grad=True, rows=2047, H=14, Hkv=2, hd=64, rot=32, dtype="f32"),
        # one new token for each of 64 sequences, pages of 16
        dict(name="append_token", op="append", B=64, new=1, ragged=False, lo=100, hi=4096, lens=1, H=32, Hkv=8, hd=128, rot=128,
             page=16, src="bf16", dtype="bf16", cache="bf16"),
        # a decoded block of 48 sequences into a cache of 8 bits, from the fp32 sums of the projection
        dict(name="append_block_e4m3", op="append", B=48, new=16, ragged=False, lo=64, hi=2048, lens=2, H=16, Hkv=8, hd=128, rot=128,
             page=64, src="f32", dtype="bf16", cache="e4m3"),
        # sixteen prompts of different lengths, pages that are no power of two
        dict(name="append_prompts", op="append", B=16, new=1000, ragged=True, lo=1, hi=500, lens=3, H=32, Hkv=8, hd=128, rot=128,
             page=48, src="f16", dtype="f16", cache="f16"),
        # the next token of one sequence: latency
        dict(name="attend_token", op="attend", B=1, new=1, ragged=False, lo=2046, hi=2046, lens=1, H=32, Hkv=8, hd=128, page=64,
             dtype="bf16", cache="bf16", causal=True, window=0, sinks=0, lse=False),
        # a served batch of 64 sequences, some a hundred times as long as others
        dict(name="attend_tokens_ragged", op="attend", B=64, new=1, ragged=False, lo=300, hi=32767, lens=5, H=32, Hkv=8, hd=128, page=64,
             dtype="bf16", cache="bf16", causal=True, window=0, sinks=0, lse=False),
        # a block of 16 positions whose rows all see each other, behind a cache of 8 bits; the sums are kept for a later join
        dict(name="attend_block_e4m3", op="attend", B=32, new=16, ragged=False, lo=1000, hi=8000, lens=6, H=32, Hkv=8, hd=128, page=64,
             dtype="bf16", cache="e4m3", causal=False, window=0, sinks=0, lse=True),
        # long conversations under a sliding window with four first tokens, pages of 16
        dict(name="attend_window", op="attend", B=32, new=1, ragged=False, lo=500, hi=32767, lens=7, H=32, Hkv=8, hd=128, page=16,
             dtype="f16", cache="f16", causal=True, window=1024, sinks=4, lse=False),
        # two prompts in parts: up to 4096 new rows behind what is cached already
        dict(name="attend_prompt", op="attend", B=2, new=4096, ragged=True, lo=2000, hi=4096, lens=8, H=32, Hkv=8, hd=128, page=64,
             dtype="bf16", cache="bf16", causal=True, window=0, sinks=0, lse=False),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(16, 8, 128), (32, 8, 128), (32, 8, 128), (40, 8, 128), (64, 8, 128), (14, 2, 64), (12, 12, 64), (8, 1, 256)]


def draw(rng):
    """One more case of the same ranges; none costs more than the largest of its operator."""
    op = rng.choice(["norm_rope", "append", "attend", "attend"])
    H, Hkv, hd = rng.choice(HEADS)
    lens = rng.randrange(1 << 20)
    rot = rng.choice([hd, hd, hd // 2])
    if op == "norm_rope":
        dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
        top = 16384 * 32 * 128 // (H * hd) // (2 if dtype == "f32" else 1)
        return dict(op=op, grad=rng.random() < 0.5, rows=_log(rng, 1, min(16384, top)), H=H, Hkv=Hkv, hd=hd, rot=rot, dtype=dtype)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    cache = rng.choice([dtype, dtype, "e4m3"])
    page = rng.choice([16, 16, 64, 64, 128, 256, 48, 1])
    if op == "append":
        new = rng.choice([1, 1, 4, 16, _log(rng, 30, 1000)])
        return dict(op=op, B=_log(rng, 1, min(256, 16000 // new)), new=new, ragged=new > 16, lo=1, hi=_log(rng, 16, 2048), lens=lens, H=H, Hkv=Hkv,
                    hd=hd, rot=rot, page=page, src=rng.choice([dtype, dtype, "f32"]), dtype=dtype, cache=cache)
    form = rng.choice(["token", "token", "block", "prompt"])
    window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 1, 4096), rng.choice([0, 1, 4, 65]))])
    if form == "prompt":
        new = _log(rng, 17, 4096)
        return dict(op=op, B=rng.choice([1, 2]), new=new, ragged=True, lo=1, hi=_log(rng, 16, 4096), lens=lens, H=min(H, 32), Hkv=Hkv, hd=min(hd, 128), page=page,
                    dtype=dtype, cache=cache, causal=True, window=window, sinks=sinks, lse=rng.random() < 0.3)
    hi = _log(rng, 100, 32767)
    new = 1 if form == "token" else rng.choice([4, 8, 16])
    most = min(64, max(1, 2 ** 28 // (hi * Hkv * hd) * 4))
    return dict(op=op, B=_log(rng, 1, most), new=new, ragged=False, lo=max(1, hi // 100), hi=hi, lens=lens, H=H, Hkv=Hkv, hd=hd, page=page, dtype=dtype, cache=cache,
                causal=form == "token", window=window, sinks=sinks, lse=rng.random() < 0.3)


def _lengths(case):
    """(new rows, cached positions before them) of every sequence."""
    rng = random.Random(case["lens"])
    new = [rng.randint((case["new"] + 1) // 2, case["new"]) if case["ragged"] else case["new"] for _ in range(case["B"])]
    new[0] = case["new"]
    return new, [_log(rng, case["lo"], case["hi"]) for _ in range(case["B"])]


def _visible(case, n, before):
    """(pairs of a row and a position that it sees, positions that any row sees) of one sequence."""
    total, W, S, pairs = before + n, case["window"], case["sinks"], 0
    first = total
    for p in range(before, total):
        top = p + 1 if case["causal"] else total
        low = max(0, p + 1 - W) if W else 0
        pairs += top - low + min(S, low)
        first = min(first, low)
    return pairs, total - first + min(S, first)


def _randn(g, shape, dtype, scale=1.0):
    if dtype == torch.float8_e4m3fn:
        return (torch.randn(shape, generator=g, device="cuda", dtype=torch.float16) * 30.0).to(dtype)
    if dtype == torch.float32 or scale != 1.0:
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _rope(n_pos, rot):
    """cos and sin of every position and pair, from angles in 64 bits."""
    freq = THETA ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    ang = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([ang.cos(), ang.sin()], dim=-1).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    H, Hkv, hd = case["H"], case["Hkv"], case["hd"]
    dtype = TYPES[case["dtype"]]
    s = dict(case=dict(case), seed=seed)
    if case["op"] == "norm_rope":
        N = case["rows"]
        # the fused projection's output: query heads, key heads, value heads of a row side by side
        qkv = _randn(g, (N, H + 2 * Hkv, hd), dtype, 1.5 if dtype == torch.float32 else 1.0)
        s["q"], s["k"] = qkv[:, :H], qkv[:, H:H + Hkv]
        s["rope"] = _rope(4096, case["rot"])
        s["pos"] = (torch.arange(N, device="cuda") % 4096).int()
        s["q_gain"], s["k_gain"] = ((1.0 + _randn(g, (hd,), torch.float32, 0.2)).bfloat16() for _ in range(2))
        if case["grad"]:
            s["dq_out"], s["dk_out"] = _randn(g, (N, H, hd), dtype), _randn(g, (N, Hkv, hd), dtype)
            s["dqkv"] = torch.zeros((N, H + 2 * Hkv, hd), dtype=dtype, device="cuda")
        else:
            s["q_out"], s["k_out"] = (torch.empty((N, h, hd), dtype=dtype, device="cuda") for h in (H, Hkv))
    else:
        new, before = _lengths(case)
        total = [n + b for n, b in zip(new, before)]
        page, B, N = case["page"], case["B"], sum(new)
        counts = [-(-t // page) for t in total]
        n_pages = sum(counts) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").int()
        ends = torch.tensor(counts, device="cuda").cumsum(0)
        width = max(counts)
        at = (ends - torch.tensor(counts, device="cuda"))[:, None] + torch.arange(width, device="cuda")
        s["page_table"] = order[torch.minimum(at, ends[:, None] - 1)].contiguous()
        s["cu_rows"] = torch.tensor([0] + new, device="cuda").cumsum(0).int()
        s["kv_len"] = torch.tensor(total, device="cuda").int()
        s["max_new"], s["max_len"] = max(new), max(total)
        cache = TYPES[case["cache"]]
        s["k_pages"], s["v_pages"] = (_randn(g, (n_pages, page, Hkv, hd), cache) for _ in range(2))
        s["k_scale"] = s["v_scale"] = None
        if case["cache"] == "e4m3":
            s["k_scale"], s["v_scale"] = (0.02 + 0.02 * torch.rand(Hkv, generator=g, device="cuda") for _ in range(2))
        if case["op"] == "append":
            src = TYPES[case["src"]]
            qkv = _randn(g, (N, H + 2 * Hkv, hd), src)
            s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
            s["rope"] = _rope(4096, case["rot"])
            s["q_gain"], s["k_gain"] = ((1.0 + _randn(g, (hd,), torch.float32, 0.2)).bfloat16() for _ in range(2))
            s["q_out"] = torch.empty((N, H, hd), dtype=dtype, device="cuda")
        else:
            s["q"] = _randn(g, (N, H, hd), dtype)
            s["scale"] = hd ** -0.5
            s["out"] = torch.empty((N, H, hd), dtype=dtype, device="cuda")
            s["lse"] = torch.empty((N, H), dtype=torch.float32, device="cuda") if case["lse"] else None
    if own:
        s["plan"] = _plan(s)
    return s


# ---- the framework's operators

@functools.lru_cache(maxsize=None)
def _context():
    import paper_2605_18817_amd as mrp
    return mrp.MrpContext(2048, 4096, 1024, 16)


def _plan(s):
    """What a program builds once for a layer and its cache: the descriptions that the calls take."""
    import paper_2605_18817_amd as mrp
    c, p = s["case"], {}
    _context()
    if "rope" in s:
        p["qk"] = mrp.QkNormRope(c["H"], c["Hkv"], c["hd"], s["rope"], s["q_gain"], s["k_gain"], eps=EPS)
    if "k_pages" in s:
        p["rows"] = mrp.NewRows(s["kv_len"], s["max_new"], cu_rows=s["cu_rows"])
        p["cache"] = mrp.PagedCache(s["k_pages"], s["v_pages"], s["page_table"], k_scale=s["k_scale"], v_scale=s["v_scale"])
    if c["op"] == "attend":
        p["attn"] = mrp.AttnCfg(c["H"], scale=s["scale"], causal=c["causal"], window=c["window"], n_sink=c["sinks"])
    return p


def _run_own(s):
    ctx, p, c = _context(), s["plan"], s["case"]
    if c["op"] == "norm_rope":
        if not c["grad"]:
            ctx.qk_norm_rope(p["qk"], s["pos"], s["q"], s["k"], s["q_out"], s["k_out"])
            return [s["q_out"], s["k_out"]]
        dq, dk = s["dqkv"][:, :c["H"]], s["dqkv"][:, c["H"]:c["H"] + c["Hkv"]]
        dgains = torch.empty((2, c["hd"]), dtype=torch.float32, device="cuda")
        ctx.qk_norm_rope_grad(p["qk"], s["pos"], s["q"], s["k"], s["dq_out"], s["dk_out"], dq, dk, dgains[0], dgains[1])
        return [dq, dk, dgains[0], dgains[1]]
    if c["op"] == "append":
        ctx.cache_append(p["rows"], p["qk"], s["q"], s["k"], s["v"], p["cache"], s["q_out"])
        return [s["q_out"], s["k_pages"], s["v_pages"]]
    ctx.paged_attention(p["rows"], p["cache"], p["attn"], s["q"], s["out"], lse=s["lse"])
    return [s["out"]] + ([s["lse"]] if c["lse"] else [])


# ---- their plain forms

def _normed(x, gain):
    return x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * gain


def _rotated(x, cos, sin):
    r = cos.shape[-1]
    a, b = x[..., :r], x[..., r:2 * r]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * r:]], dim=-1)


def _plain_norm_rope(x, gain, cs, dtype):
    return _rotated(_normed(x.float(), gain.float()), cs[..., 0], cs[..., 1]).to(dtype)


def _plain_norm_rope_grad(x, gain, cs, dy):
    x32, g = x.float(), gain.float()
    dn = _rotated(dy.float(), cs[..., 0], -cs[..., 1])
    inv = torch.rsqrt((x32 * x32).mean(dim=-1, keepdim=True) + EPS)
    t = dn * g
    dx = inv * t - x32 * inv * inv * inv * (x32 * t).mean(dim=-1, keepdim=True)
    return dx.to(x.dtype), (dn * x32 * inv).sum(dim=(0, 1))


def _row_places(s):
    """(sequence, place among its new rows, position) of every row."""
    cu, N = s["cu_rows"].long(), s["q"].shape[0]
    row = torch.arange(N, device="cuda")
    seq = torch.searchsorted(cu[1:].contiguous(), row, right=True)
    return seq, row - cu[seq], s["kv_len"].long()[seq] - cu[seq + 1] + row


def _stored(x, scale, dtype):
    if dtype != torch.float8_e4m3fn:
        return x.to(dtype)
    return (x / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(dtype).view(torch.uint8)


def _plain_append(s):
    c = s["case"]
    seq, _, pos = _row_places(s)
    slot = s["page_table"].long()[seq, pos // c["page"]] * c["page"] + pos % c["page"]
    cs = s["rope"][pos][:, None]
    q_out = _plain_norm_rope(s["q"], s["q_gain"], cs, TYPES[c["dtype"]])
    k = _plain_norm_rope(s["k"], s["k_gain"], cs, torch.float32)
    for pages, x, scale in ((s["k_pages"], k, s["k_scale"]), (s["v_pages"], s["v"].float(), s["v_scale"])):
        flat = pages.view(torch.uint8) if pages.dtype == torch.float8_e4m3fn else pages
        flat.view(-1, c["Hkv"], c["hd"])[slot] = _stored(x, scale, pages.dtype)
    return [q_out, s["k_pages"], s["v_pages"]]


def _plain_attend(s):
    c = s["case"]
    B, H, Hkv, hd, page, n, top = c["B"], c["H"], c["Hkv"], c["hd"], c["page"], s["max_new"], s["max_len"]
    j = torch.arange(top, device="cuda")
    slot = s["page_table"].long()[:, j // page] * page + j % page
    k, v = (p.view(-1, Hkv, hd)[slot].float().permute(0, 2, 1, 3) for p in (s["k_pages"], s["v_pages"]))
    if s["k_scale"] is not None:
        k, v = k * s["k_scale"][:, None, None], v * s["v_scale"][:, None, None]
    seq, place, _ = _row_places(s)
    cu, kv_len = s["cu_rows"].long(), s["kv_len"].long()
    row = torch.minimum(cu[:-1, None] + torch.arange(n, device="cuda"), cu[1:, None] - 1)
    q = s["q"][row].float().view(B, n, Hkv, H // Hkv, hd).permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, hd)
    score = (torch.matmul(q, k.transpose(2, 3)) * s["scale"]).view(B, Hkv, n, H // Hkv, top)
    p = (kv_len - (cu[1:] - cu[:-1]))[:, None] + torch.arange(n, device="cuda")
    seen = j < (p[:, :, None] + 1 if c["causal"] else kv_len[:, None, None])
    if c["window"]:
        seen = seen & ((j > p[:, :, None] - c["window"]) | (j < c["sinks"]))
    score = score.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    most = score.amax(dim=-1, keepdim=True)
    w = (score - most).exp_()
    total = w.sum(dim=-1, keepdim=True)
    out = torch.matmul(w.view(B, Hkv, -1, top), v.contiguous()).view(B, Hkv, n, -1, hd) / total
    lse = (most + total.log()).permute(0, 2, 1, 3, 4).reshape(B, n, H)[seq, place]
    out = out.permute(0, 2, 1, 3, 4).reshape(B, n, H, hd)[seq, place].to(s["q"].dtype)
    return [out] + ([lse] if c["lse"] else [])


def run(state):
    if own:
        return _run_own(state)
    c = state["case"]
    if c["op"] == "append":
        return _plain_append(state)
    if c["op"] == "attend":
        return _plain_attend(state)
    cs = state["rope"][state["pos"].long()][:, None]
    if not c["grad"]:
        return [_plain_norm_rope(state[n], state[n + "_gain"], cs, state[n].dtype) for n in ("q", "k")]
    (dq, gq), (dk, gk) = (_plain_norm_rope_grad(state[n], state[n + "_gain"], cs, state["d%s_out" % n]) for n in ("q", "k"))
    return [dq, dk, gq, gk]


# ---- 64 bits, from the definitions

def _exact_turn(x, gain, table):
    """One head vector after the other as complex numbers: normalised, scaled, turned."""
    x = x.double()
    y = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * gain.double()
    r = table.shape[-2]
    z = torch.complex(y[..., :r].contiguous(), y[..., r:2 * r].contiguous()) * torch.view_as_complex(table.double().contiguous())
    y[..., :r], y[..., r:2 * r] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    H, Hkv, hd = case["H"], case["Hkv"], case["hd"]
    if case["op"] == "norm_rope":
        table = s["rope"][s["pos"].long()].unsqueeze(1)
        if not case["grad"]:
            return [_exact_turn(s[n], s[n + "_gain"], table) for n in ("q", "k")]
        dx, dg = [], []
        for n in ("q", "k"):
            # the gradient of the definition itself, 2048 rows at a time
            gain, parts = s[n + "_gain"].double().requires_grad_(True), []
            for at in range(0, case["rows"], 2048):
                x = s[n][at:at + 2048].double().requires_grad_(True)
                y = x / (x.pow(2).sum(-1, keepdim=True) / hd + EPS).sqrt() * gain
                r = case["rot"] // 2
                t = table[at:at + 2048].double()
                u, w = y[..., :r], y[..., r:2 * r]
                dy = s["d%s_out" % n][at:at + 2048].double()
                loss = ((u * t[..., 0] - w * t[..., 1]) * dy[..., :r] + (w * t[..., 0] + u * t[..., 1]) * dy[..., r:2 * r]).sum() + (y[..., 2 * r:] * dy[..., 2 * r:]).sum()
                loss.backward()
                parts.append(x.grad)
            dx.append(torch.cat(parts))
            dg.append(gain.grad)
        return dx + dg
    new, before = _lengths(case)
    page, table = case["page"], s["page_table"].tolist()
    if case["op"] == "append":
        q = torch.empty((sum(new), H, hd), dtype=torch.float64, device="cuda")
        k_pages, v_pages = s["k_pages"].double(), s["v_pages"].double()
        at = 0
        for b, (n, m) in enumerate(zip(new, before)):
            rows = slice(at, at + n)
            turn = s["rope"][m:m + n].unsqueeze(1)
            q[rows] = _exact_turn(s["q"][rows], s["q_gain"], turn)
            where = torch.tensor([table[b][p // page] for p in range(m, m + n)], device="cuda"), torch.arange(m, m + n, device="cuda") % page
            for pages, x, scale in ((k_pages, _exact_turn(s["k"][rows], s["k_gain"], turn), s["k_scale"]), (v_pages, s["v"][rows].double(), s["v_scale"])):
                pages[where] = x if scale is None else (x / scale.double()[:, None]).clamp(-E4M3_MAX, E4M3_MAX)
            at += n
        return [q, k_pages, v_pages]
    out = torch.empty((sum(new), H, hd), dtype=torch.float64, device="cuda")
    lse = torch.empty((sum(new), H), dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, m) in enumerate(zip(new, before)):
        pages = s["page_table"][b, :-(-(m + n) // page)].long()
        place = torch.arange(m + n, device="cuda")
        own_place = torch.arange(m, m + n, device="cuda")[:, None]
        hidden = place > own_place if case["causal"] else place >= m + n
        if case["window"]:
            hidden = hidden | ((place <= own_place - case["window"]) & (place >= case["sinks"]))
        for h in range(Hkv):
            k, v = (p[pages, :, h].reshape(-1, hd)[:m + n].double() for p in (s["k_pages"], s["v_pages"]))
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            for x in range(h * (H // Hkv), (h + 1) * (H // Hkv)):
                score = (s["q"][at:at + n, x].double() @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
                lse[at:at + n, x] = score.logsumexp(-1)
                out[at:at + n, x] = score.softmax(-1) @ v
        at += n
    return [out] + ([lse] if case["lse"] else [])


def work(case):
    H, Hkv, hd = case["H"], case["Hkv"], case["hd"]
    if case["op"] == "norm_rope":
        N, size = case["rows"], SIZE[case["dtype"]]
        heads = N * (H + Hkv) * hd
        table = min(N, 4096) * case["rot"] * 4 + 4 * N
        return {"bytes": heads * size * (3 if case["grad"] else 2) + table + 12 * hd, "flops": heads * (24 if case["grad"] else 10)}
    new, before = _lengths(case)
    N = sum(new)
    if case["op"] == "append":
        places = {p for n, m in zip(new, before) for p in range(m, m + n)}
        moved = N * hd * ((H + 2 * Hkv) * SIZE[case["src"]] + H * SIZE[case["dtype"]] + 2 * Hkv * SIZE[case["cache"]])
        return {"bytes": moved + len(places) * case["rot"] * 4 + 8 * case["B"] + 4 * sum(-(-n // case["page"]) for n in new), "flops": N * (H + Hkv) * hd * 10}
    pairs, keys = (sum(x) for x in zip(*(_visible(case, n, m) for n, m in zip(new, before))))
    moved = keys * Hkv * hd * 2 * SIZE[case["cache"]] + 2 * N * H * hd * SIZE[case["dtype"]] + (4 * N * H if case["lse"] else 0)
    return {"bytes": moved + 8 * case["B"] + 4 * keys // case["page"], "flops": 4 * pairs * H * hd}
