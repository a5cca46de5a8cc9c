"""mrp_qk_norm_rope and its gradient against 64 bits: head layouts, types, partial and no rotation, with and without gains,
strided parts of a fused projection, positions far out; the gradient also against differences."""
import pytest
import torch

import paged_reference as ref
import paper_2605_18817_amd as mrp

pytestmark = pytest.mark.gpu
EPS = 1e-6
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def ctx():
    c = mrp.MrpContext(256, 4096, 64, 16)
    yield c
    c.close()


def _inputs(rows, H, Hkv, hd, x, gain_t, gains, seed=0, n_pos=5000):
    g = torch.Generator(device="cuda").manual_seed(seed)
    qkv = (torch.randn((rows, H + 2 * Hkv, hd), generator=g, device="cuda") * 2).to(x)
    gq = gk = None
    if gains:
        gq, gk = ((1 + 0.3 * torch.randn(hd, generator=g, device="cuda")).to(gain_t) for _ in range(2))
    pos = torch.randint(0, n_pos, (rows,), generator=g, device="cuda").int()
    if rows:
        pos[-1] = n_pos - 1
    return g, qkv[:, :H], qkv[:, H:H + Hkv], gq, gk, pos


def _table(rope, pos):
    return None if rope is None else rope[pos.long()]


FORMS = [   # rows, H, Hkv, hd, rot, x, y, gain, gains
    (1, 16, 8, 128, 128, "bf16", "bf16", "bf16", True),
    (7, 32, 8, 128, 128, "bf16", "bf16", "bf16", True),
    (33, 5, 1, 64, 64, "f16", "f16", "f16", True),
    (130, 14, 2, 64, 32, "f32", "f32", "f32", True),
    (65, 3, 3, 256, 256, "bf16", "bf16", "f32", True),
    (19, 8, 1, 256, 16, "f32", "bf16", "bf16", True),
    (40, 2, 2, 128, 48, "f32", "f16", "bf16", True),
    (50, 4, 2, 128, 0, "bf16", "bf16", "bf16", True),
    (50, 4, 2, 128, 128, "f16", "f16", "bf16", False),
    (257, 1, 0, 64, 64, "f32", "f32", "bf16", True),
]


@pytest.mark.parametrize("rows,H,Hkv,hd,rot,x,y,gt,gains", FORMS)
def test_forward(ctx, rows, H, Hkv, hd, rot, x, y, gt, gains):
    _, q, k, gq, gk, pos = _inputs(rows, H, Hkv, hd, T[x], T[gt], gains)
    rope = ctx.rope_table(5000, rot, 1e6) if rot else None
    qk = mrp.QkNormRope(H, Hkv, hd, rope, gq, gk, eps=EPS)
    q_out, k_out = (torch.full((rows, h, hd), 7.0, dtype=T[y], device="cuda") for h in (H, Hkv))
    ctx.qk_norm_rope(qk, pos, q, k if Hkv else None, q_out, k_out if Hkv else None)
    for a, gain, got in ((q, gq, q_out), (k, gk, k_out)):
        want, bound = ref.norm_rope(a, gain, _table(rope, pos), EPS)
        ref.assert_close(got, want, ref.half_step(T[y]) * want.abs() + bound * (1 + 2 ** -7) + 2.0 ** -25, "forward")
    assert ctx.poll_error() == 0


@pytest.mark.parametrize("rows,H,Hkv,hd,rot,x,y,gt,gains", FORMS)
def test_gradient(ctx, rows, H, Hkv, hd, rot, x, y, gt, gains):
    g, q, k, gq, gk, pos = _inputs(rows, H, Hkv, hd, T[x], T[gt], gains, seed=1)
    rope = ctx.rope_table(5000, rot, 1e6) if rot else None
    qk = mrp.QkNormRope(H, Hkv, hd, rope, gq, gk, eps=EPS)
    dy = [torch.randn((rows, h, hd), generator=g, device="cuda").to(T[y]) for h in (H, Hkv)]
    dqkv = torch.full((rows, H + 2 * Hkv, hd), 7.0, dtype=T[x], device="cuda")
    dg = torch.full((2, hd), 7.0, device="cuda")
    ctx.qk_norm_rope_grad(qk, pos, q, k if Hkv else None, dy[0], dy[1] if Hkv else None, dqkv[:, :H], dqkv[:, H:H + Hkv] if Hkv else None,
                          dg[0] if gains else None, dg[1] if gains and Hkv else None)
    for a, gain, d, got, got_g in ((q, gq, dy[0], dqkv[:, :H], dg[0]), (k, gk, dy[1], dqkv[:, H:H + Hkv], dg[1])):
        if a.shape[1] == 0:
            continue
        dx, dgain, bound, gbound = ref.norm_rope_grad(a, gain, _table(rope, pos), d, EPS)
        ref.assert_close(got, dx, ref.half_step(T[x]) * dx.abs() + bound * (1 + 2 ** -7) + 2.0 ** -25, "dx")
        if gains:
            ref.assert_close(got_g, dgain, gbound, "dgain")
    assert (dqkv[:, H + Hkv:] == 7.0).all()        # the values' part is not touched


def test_gradient_against_differences(ctx):
    rows, H, Hkv, hd, rot = 3, 2, 1, 64, 32
    g, q, k, gq, gk, pos = _inputs(rows, H, Hkv, hd, torch.float32, torch.float32, True, seed=2)
    rope = ctx.rope_table(5000, rot, 1e6)
    qk = mrp.QkNormRope(H, Hkv, hd, rope, gq, gk, eps=EPS)
    dy = [torch.randn((rows, h, hd), generator=g, device="cuda") for h in (H, Hkv)]
    dq, dk, dg = torch.empty_like(q), torch.empty_like(k), torch.empty((2, hd), device="cuda")
    ctx.qk_norm_rope_grad(qk, pos, q, k, dy[0], dy[1], dq, dk, dg[0], dg[1])
    table = rope[pos.long()]
    for x, gain, d, dx, dgain in ((q, gq, dy[0], dq, dg[0]), (k, gk, dy[1], dk, dg[1])):
        u, v = torch.randn(x.shape, generator=g, device="cuda").double(), torch.randn(hd, generator=g, device="cuda").double()
        e = 1e-5
        loss = lambda t: float((ref.norm_rope(x.double() + t * u, gain.double() + t * v, table, EPS)[0] * d.double()).sum())  # noqa: E731
        slope = (loss(e) - loss(-e)) / (2 * e)
        mine = float((dx.double() * u).sum() + (dgain.double() * v).sum())
        size = float((dx.double() * u).abs().sum() + (dgain.double() * v).abs().sum())
        # central differences of 64-bit values: e^2 and 2^-52 / e of the size, the gradient (hd + 40) half steps of it and more
        assert abs(slope - mine) <= 1e-4 * size


def test_gradient_sums_repeat_bit_for_bit(ctx):
    rows, H, Hkv, hd = 3000, 6, 2, 128
    g, q, k, gq, gk, pos = _inputs(rows, H, Hkv, hd, torch.bfloat16, torch.bfloat16, True, seed=3)
    qk = mrp.QkNormRope(H, Hkv, hd, ctx.rope_table(5000, 128, 1e6), gq, gk, eps=EPS)
    dy = [torch.randn((rows, h, hd), generator=g, device="cuda").bfloat16() for h in (H, Hkv)]
    got = []
    for _ in range(3):
        dq, dk, dg = torch.empty((rows, H, hd), dtype=torch.bfloat16, device="cuda"), torch.empty((rows, Hkv, hd), dtype=torch.bfloat16, device="cuda"), torch.empty((2, hd), device="cuda")
        ctx.qk_norm_rope_grad(qk, pos, q, k, dy[0], dy[1], dq, dk, dg[0], dg[1])
        got.append((dq, dk, dg))
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
    _, dgain, _, gbound = ref.norm_rope_grad(q, gq, ref.rope_table(5000, 128)[pos.long()].float(), dy[0], EPS)
    ref.assert_close(got[0][2][0], dgain, gbound, "dgain")


def test_rope_table(ctx):
    got = ctx.rope_table(70000, 64, 1e4).double()
    # the angle of position 70000 in 64 bits is off by far less than a half step of fp32 (about 1e-11)
    assert (got - ref.rope_table(70000, 64, 1e4)).abs().max() <= ref.U32 + 1e-9


def test_positions_out_of_range_are_clamped_and_reported(ctx):
    q = torch.randn((4, 2, 64), device="cuda")
    pos = torch.tensor([-3, 0, 9, 10 ** 6], dtype=torch.int32, device="cuda")
    qk = mrp.QkNormRope(2, 0, 64, ctx.rope_table(10, 64, 1e4), None, None)
    out, want = torch.empty_like(q), torch.empty_like(q)
    ctx.poll_error()
    ctx.qk_norm_rope(qk, pos, q, None, out, None)
    assert ctx.poll_error() == 16 and "position" in ctx.last_error()
    ctx.qk_norm_rope(qk, pos.clamp(0, 9), q, None, want, None)
    assert torch.equal(out, want) and ctx.poll_error() == 0


def test_empty_and_zero_rows(ctx):
    gain = torch.ones(64, device="cuda")
    qk = mrp.QkNormRope(2, 1, 64, ctx.rope_table(10, 64, 1e4), gain, gain)
    e = lambda h: torch.empty((0, h, 64), device="cuda")  # noqa: E731
    pos = torch.empty(0, dtype=torch.int32, device="cuda")
    dg = torch.full((2, 64), 5.0, device="cuda")
    ctx.qk_norm_rope(qk, pos, e(2), e(1), e(2), e(1))
    ctx.qk_norm_rope_grad(qk, pos, e(2), e(1), e(2), e(1), e(2), e(1), dg[0], dg[1])
    assert (dg == 0).all()
    # a head of zeros: eps keeps it finite, also with its gradient
    z, one = torch.zeros((3, 2, 64), device="cuda"), torch.ones((3, 2, 64), device="cuda")
    qk1 = mrp.QkNormRope(2, 0, 64, None, gain, None)
    out, dx = torch.empty_like(z), torch.empty_like(z)
    ctx.qk_norm_rope(qk1, None, z, None, out, None)
    ctx.qk_norm_rope_grad(qk1, None, z, None, one, None, dx, None)
    assert (out == 0).all() and ((dx - 1000.0).abs() <= 1e-2).all()      # 1 / sqrt(1e-6)
