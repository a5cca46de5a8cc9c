"""The host side's checks of the paged cache's entry points, without a GPU: a block of zeros stands in for a context, as far as
refusals write their message there.  Whatever is refused is refused before anything asks for a device."""
import ctypes as C

import pytest

import paper_2605_18817_amd as mrp
from paper_2605_18817_amd import binding as bd

NULL, SHAPE, ALIGN, WORKSPACE = -1, -2, -3, -4
A = 1 << 20          # an aligned address that nothing reads


@pytest.fixture()
def lib():
    return mrp.load_library()


@pytest.fixture()
def ctx():
    return C.cast(C.create_string_buffer(1 << 14), C.c_void_p)


def _qk(**over):
    f = dict(n_heads=8, n_kv_heads=2, head_dim=128, rotary_dim=64, x_dtype=1, y_dtype=1, gain_dtype=1, eps=1e-6, q_gain=A, k_gain=A, rope=A, n_pos=100)
    f.update(over)
    return bd._Qk(**f)


def _rows(**over):
    f = dict(B=3, max_new=4, cu_rows=A, kv_len=A)
    f.update(over)
    return bd._NewRows(**f)


def _cache(**over):
    f = dict(k_pages=A, v_pages=A, dtype=1, n_kv_heads=2, head_dim=128, n_pages=10, page_size=16, page_table=A, max_pages=5, k_scale=None, v_scale=None)
    f.update(over)
    return bd._PagedCache(**f)


def _attn(**over):
    f = dict(n_heads=8, dtype=1, scale=0.1, causal=1, window=0, n_sink=0)
    f.update(over)
    return bd._Attn(**f)


def test_null_contexts(lib):
    assert lib.mrp_rope_table(None, None, 8, 64, 1e4, A) == NULL
    assert lib.mrp_qk_norm_rope(None, None, 1, _qk(), A, A, 1024, A, 256, A, A) == NULL
    assert lib.mrp_qk_norm_rope_grad(None, None, 1, _qk(), A, A, 1024, A, 256, A, A, A, 1024, A, 256, A, A, A, 1 << 30) == NULL
    assert lib.mrp_cache_append(None, None, 1, _rows(), _qk(), A, 1024, A, 256, A, 256, _cache(), A) == NULL
    assert lib.mrp_paged_attention(None, None, 1, _rows(), _cache(), _attn(), A, 1024, A, None, None, 0) == NULL


@pytest.mark.parametrize("over,code", [
    (dict(head_dim=96), SHAPE), (dict(head_dim=32), SHAPE), (dict(n_heads=0), SHAPE), (dict(n_heads=1025), SHAPE), (dict(n_kv_heads=-1), SHAPE),
    (dict(rotary_dim=8), SHAPE), (dict(rotary_dim=144), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rope=None), NULL), (dict(n_pos=0), SHAPE),
    (dict(x_dtype=1, y_dtype=2), SHAPE), (dict(x_dtype=1, y_dtype=0), SHAPE), (dict(x_dtype=3, y_dtype=3), SHAPE), (dict(gain_dtype=3), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(q_gain=A + 8), ALIGN), (dict(rope=A + 8), ALIGN)])
def test_norm_and_rotation(lib, ctx, over, code):
    qk = _qk(**over)
    assert lib.mrp_qk_norm_rope(ctx, None, 5, qk, A, A, 1024, A, 256, A, A) == code
    assert lib.mrp_qk_norm_rope_grad(ctx, None, 5, qk, A, A, 1024, A, 256, A, A, A, 1024, A, 256, A, A, A, 1 << 30) == code
    assert lib.mrp_cache_append(ctx, None, 5, _rows(), qk, A, 1024, A, 256, A, 256, _cache(), A) == code


def test_row_tensors(lib, ctx):
    call = lambda n=5, pos=A, q=A, qs=1024, k=A, ks=256, qo=A, ko=A: lib.mrp_qk_norm_rope(ctx, None, n, _qk(), pos, q, qs, k, ks, qo, ko)  # noqa: E731
    assert call(n=-1) == SHAPE and call(n=1 << 25) == SHAPE
    assert call(n=0, pos=None, q=None, k=None, qo=None, ko=None) == 0
    assert call(pos=None) == NULL and call(q=None) == NULL and call(k=None) == NULL and call(qo=None) == NULL and call(ko=None) == NULL
    assert call(qs=1023) == SHAPE and call(ks=128) == SHAPE and call(qs=1028) == ALIGN and call(q=A + 2) == ALIGN and call(ko=A + 4) == ALIGN
    grad = lambda g=A, s=A, size=1 << 30, qk=None: lib.mrp_qk_norm_rope_grad(ctx, None, 5, qk or _qk(), A, A, 1024, A, 256, A, A, A, 1024, A, 256, g, g, s, size)  # noqa: E731
    need = lib.mrp_qk_norm_rope_grad_scratch_bytes(5, _qk())
    assert need > 0 and grad(s=None) == NULL and grad(s=A + 8) == ALIGN and grad(size=need - 1) == WORKSPACE
    assert grad(qk=_qk(q_gain=None)) == SHAPE          # a gradient of a gain that there is not
    assert lib.mrp_qk_norm_rope_grad_scratch_bytes(0, _qk()) == 0 and lib.mrp_qk_norm_rope_grad_scratch_bytes(5, None) == 0


@pytest.mark.parametrize("over,code", [(dict(B=-1), SHAPE), (dict(B=65536), SHAPE), (dict(max_new=0), SHAPE), (dict(kv_len=None), NULL),
                                       (dict(cu_rows=None, max_new=5), SHAPE)])     # three of five, but twelve rows
def test_new_rows(lib, ctx, over, code):
    assert lib.mrp_cache_append(ctx, None, 12, _rows(**over), _qk(), A, 1024, A, 256, A, 256, _cache(), A) == code
    assert lib.mrp_paged_attention(ctx, None, 12, _rows(**over), _cache(), _attn(), A, 1024, A, None, A, 1 << 40) == code


@pytest.mark.parametrize("over,code", [
    (dict(k_pages=None), NULL), (dict(page_table=None), NULL), (dict(dtype=0), SHAPE), (dict(dtype=4), SHAPE), (dict(head_dim=80), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(max_pages=0), SHAPE),
    (dict(n_pages=1 << 28, page_size=16), SHAPE), (dict(max_pages=1 << 28), SHAPE), (dict(v_pages=A + 8), ALIGN), (dict(k_scale=A), SHAPE)])
def test_caches(lib, ctx, over, code):
    assert lib.mrp_cache_append(ctx, None, 12, _rows(), _qk(), A, 1024, A, 256, A, 256, _cache(**over), A) == code
    assert lib.mrp_paged_attention(ctx, None, 12, _rows(), _cache(**over), _attn(), A, 1024, A, None, A, 1 << 40) == code


def test_append(lib, ctx):
    call = lambda cache=None, qk=None, q=A, k=A, v=A, qo=A, n=12, rows=None: lib.mrp_cache_append(  # noqa: E731
        ctx, None, n, rows or _rows(), qk or _qk(), q, 1024, k, 256, v, 256, cache or _cache(), qo)
    assert call(k=None) == NULL and call(v=None) == NULL and call(qo=None) == NULL and call(v=A + 2) == ALIGN
    assert call(cache=_cache(n_kv_heads=4)) == SHAPE and call(cache=_cache(head_dim=64)) == SHAPE
    assert call(qk=_qk(n_heads=7)) == SHAPE
    assert call(n=0) == 0 and call(rows=_rows(B=0)) == 0
    assert lib.mrp_cache_append(ctx, None, 12, None, _qk(), A, 1024, A, 256, A, 256, _cache(), A) == NULL


@pytest.mark.parametrize("over,code", [
    (dict(n_heads=7), SHAPE), (dict(n_heads=0), SHAPE), (dict(dtype=0), SHAPE), (dict(dtype=2), SHAPE), (dict(dtype=3), SHAPE), (dict(scale=0.0), SHAPE),
    (dict(scale=-1.0), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(scale=float("inf")), SHAPE), (dict(causal=2), SHAPE), (dict(window=-1), SHAPE),
    (dict(n_sink=-1), SHAPE)])
def test_attention_forms(lib, ctx, over, code):
    assert lib.mrp_paged_attention(ctx, None, 12, _rows(), _cache(), _attn(**over), A, 1024, A, None, A, 1 << 40) == code


def test_attention(lib, ctx):
    call = lambda q=A, qs=1024, out=A, s=A, size=1 << 40, n=12, rows=None, cache=None: lib.mrp_paged_attention(  # noqa: E731
        ctx, None, n, rows or _rows(), cache or _cache(), _attn(), q, qs, out, None, s, size)
    assert call(q=None) == NULL and call(out=None) == NULL and call(qs=1000) == SHAPE and call(qs=1028) == ALIGN
    assert call(q=A + 8) == ALIGN and call(out=A + 8) == ALIGN and call(s=A + 8) == ALIGN
    assert call(n=0, q=None, out=None) == 0 and call(rows=_rows(B=0)) == 0
    need = lib.mrp_paged_attention_scratch_bytes(ctx, 12, _rows(), _cache(), _attn())
    if need:
        assert call(s=None) == NULL and call(size=need - 1) == WORKSPACE


def test_tables(lib, ctx):
    assert lib.mrp_rope_table(ctx, None, 0, 64, 1e4, A) == SHAPE and lib.mrp_rope_table(ctx, None, 8, 24, 1e4, A) == SHAPE
    assert lib.mrp_rope_table(ctx, None, 8, 64, 1.0, A) == SHAPE and lib.mrp_rope_table(ctx, None, 8, 64, 1e4, None) == NULL
    assert lib.mrp_rope_table(ctx, None, 8, 64, 1e4, A + 4) == ALIGN
