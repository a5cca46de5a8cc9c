"""Plain 64-bit forms of the norm with rotation, of the cache in pages and of the attention over it, and what the
operators' roundings may add up to (used by the GPU tests; everything stays on the tensors' device)."""
import math

import torch

U32 = 2.0 ** -24                       # half a step of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def assert_close(got, want, tol, what=""):
    got = got.double()
    assert torch.equal(torch.isfinite(got), torch.isfinite(want)), f"{what}: other entries are finite"
    err = torch.where(torch.isfinite(want), (got - want).abs(), torch.zeros_like(want))
    over = err > tol
    assert not over.any(), f"{what}: {int(over.sum())} of {want.numel()} off, worst {float((err / tol.clamp_min(1e-300)).max()):.2f} x the bound"


def rope_table(n_pos, rot, theta=1e6):
    freq = float(theta) ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot)
    ang = torch.arange(n_pos, dtype=torch.float64, device="cuda")[:, None] * freq
    return torch.stack([ang.cos(), ang.sin()], dim=-1)


def turned(n, table, back=False):
    """R n (or R^T n) of heads n [rows, heads, hd] for table rows [rows, rot / 2, 2]; and the sum of the magnitudes."""
    r = table.shape[1]
    c, s = table[:, None, :, 0], table[:, None, :, 1] * (-1.0 if back else 1.0)
    a, b, rest = n[..., :r], n[..., r:2 * r], n[..., 2 * r:]
    y = torch.cat([a * c - b * s, b * c + a * s, rest], dim=-1)
    mag = torch.cat([(a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs(), rest.abs()], dim=-1)
    return y, mag


def norm_rope(x, gain, table, eps):
    """(y, bound on fp32 rounding before the last one) of heads x [rows, heads, hd], 64 bits."""
    x = x.double()
    hd = x.shape[-1]
    n = x if gain is None else x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * gain.double()
    if table is None:
        y, mag = n, n.abs()
    else:
        y, mag = turned(n, table.double())
    # the mean of hd squares is off by at most hd / 2 + 2 half steps of its value and its root by half of that; then a square
    # root, a division, two products, and the rotation's two products and sum
    return y, (hd / 4 + 12) * U32 * mag


def norm_rope_grad(x, gain, table, dy, eps):
    """dx, dgain and the bounds on their fp32 roundings, from the formulas."""
    x, dy = x.double(), dy.double()
    hd = x.shape[-1]
    dn, mag = (dy, dy.abs()) if table is None else turned(dy, table.double(), back=True)
    if gain is None:
        return dn, None, 4 * U32 * mag, None
    g = gain.double()
    inv = (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    t, tm = dn * g, mag * g.abs()
    dx = inv * t - x * inv ** 3 * (x * t).mean(-1, keepdim=True)
    terms = dn * x * inv
    # as above; the second mean adds hd / 2 half steps of its magnitudes
    bound = (hd + 24) * U32 * (inv * tm + x.abs() * inv ** 3 * (x.abs() * tm).mean(-1, keepdim=True))
    # a chain of additions as long as there are terms is the worst that any order can do
    count = x.shape[0] * x.shape[1]
    gain_bound = (min(count, 2048) + hd / 4 + 16) * U32 * (mag * x.abs() * inv).sum((0, 1))
    return dx, terms.sum((0, 1)), bound, gain_bound


def e4m3_tolerance(x):
    """Half a step of e4m3 at x: 2^-4 of the value, or half of the subnormals' step 2^-9."""
    return (x.abs() * 2.0 ** -4).clamp_min(2.0 ** -10)


class Batch:
    """A ragged batch over a cache in pages: lengths, page table (pages in a shuffled order, some spare), and where each row lies."""

    def __init__(self, new, kv_len, page, spare=2, behind=0, uniform=False, seed=0, max_pages=None):
        g = torch.Generator().manual_seed(seed)
        self.new, self.kv_len, self.page, self.B = list(new), list(kv_len), page, len(new)
        counts = [max(0, -(-t // page)) for t in kv_len]
        self.n_pages = sum(counts) + spare
        order = torch.randperm(self.n_pages, generator=g).tolist()
        width = max_pages or max(1, max(counts))
        self.table = torch.full((self.B, width), order[-1], dtype=torch.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = torch.tensor(order[at:at + c], dtype=torch.int32)
            at += c
        self.cu = [0]
        for n in new:
            self.cu.append(self.cu[-1] + n)
        self.n_rows = self.cu[-1] + behind
        self.max_new = max(1, max(new))
        self.uniform = uniform

    def rows(self, mrp):
        self.table_d = self.table.cuda()
        self.cu_d = torch.tensor(self.cu, dtype=torch.int32).cuda()
        self.len_d = torch.tensor(self.kv_len, dtype=torch.int32).cuda()
        return mrp.NewRows(self.len_d, self.max_new, cu_rows=None if self.uniform else self.cu_d)

    def places(self, b, positions):
        """(page, place) index tensors of positions of sequence b."""
        p = torch.as_tensor(positions)
        return self.table[b].long()[p // self.page].cuda(), (p % self.page).cuda()


def attention(batch, q, k_pages, v_pages, scale, causal, window, sinks, k_scale=None, v_scale=None, gone=()):
    """(out, lse, sum of w |v| / sum of w, largest sum of |q k| scale) in 64 bits, row by row; rows that see nothing: 0, -inf."""
    N, H, hd = q.shape
    Hkv = k_pages.shape[2]
    G = H // Hkv
    out = torch.zeros((N, H, hd), dtype=torch.float64, device=q.device)
    lse = torch.full((N, H), -math.inf, dtype=torch.float64, device=q.device)
    mag, qk = torch.zeros_like(out), torch.zeros((N, H, 1), dtype=torch.float64, device=q.device)
    for b in range(batch.B):
        n, total = batch.new[b], batch.kv_len[b]
        if n == 0 or total <= 0:
            continue
        pg, pl = batch.places(b, torch.arange(total))
        for i in range(n):
            p, row = total - n + i, batch.cu[b] + i
            if p < 0:
                continue
            j = torch.arange(total)
            seen = (j <= p) if causal else torch.ones(total, dtype=torch.bool)
            if window:
                seen &= (j > p - window) | (j < sinks)
            for page in gone:
                seen &= (batch.table[b].long()[j // batch.page] != page)
            if not seen.any():
                continue
            at = seen.nonzero()[:, 0].cuda()
            k, v = k_pages[pg[at], pl[at]].double(), v_pages[pg[at], pl[at]].double()      # [keys, Hkv, hd]
            if k_scale is not None:
                k, v = k * k_scale.double()[:, None], v * v_scale.double()[:, None]
            qq = q[row].double().view(Hkv, G, hd)
            s = torch.matmul(qq, k.permute(1, 2, 0).contiguous()) * scale                 # [Hkv, G, keys]
            w = torch.softmax(s, -1)
            vv = v.permute(1, 0, 2).contiguous()
            out[row] = torch.matmul(w, vv).view(H, hd)
            mag[row] = torch.matmul(w, vv.abs()).view(H, hd)
            lse[row] = torch.logsumexp(s, -1).view(H)
            qk[row] = (torch.matmul(qq.abs(), k.abs().permute(1, 2, 0).contiguous()) * scale).amax(-1).view(H, 1)
    return out, lse, mag, qk


def attention_tolerance(dtype, out, lse, mag, qk, hd, keys, few):
    """Bounds of out and lse.  A score is a sum of hd products in fp32: off by hd half steps of its magnitudes, then a product and
    an exponent's argument (4 of the score's) and the exponential (4): relative error d of a weight, twice that with
    the sum's.  Sums of `keys` terms add their half steps.  The weights enter the product as two terms of the type (few rows)
    or one, fp16 ones below its normals by half a step of 2^-24 absolutely; the result is rounded once."""
    u = half_step(dtype)
    d = (hd + 6) * U32 * qk + 8 * U32
    chain = (keys + 64) * U32
    w = u * u if few else u
    tol = u * out.abs() + (2 * d + 2 * chain + w) * mag * (1 + u)
    if dtype == torch.float16:
        tol = tol + 2.0 ** -25 * keys * mag.amax(-1, keepdim=True).clamp_min(1.0) + 2.0 ** -25
    return tol + 1e-30, (d + chain).squeeze(-1) + 4 * U32 * lse.abs().nan_to_num(0.0, 0.0, 0.0) + 1e-30
