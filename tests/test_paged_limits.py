"""Sizes at the ends of the integers that the paged cache's entry points count with, without a GPU: refused before anything asks for a
device (a block of zeros stands in for a context)."""
import ctypes as C

import pytest
import torch

import paper_2605_18817_amd as mrp
from paper_2605_18817_amd import binding as bd

SHAPE = -2
A = 1 << 20          # an aligned address that nothing reads


@pytest.mark.parametrize("max_pages,page_size", [(2 ** 31 - 1, 1), (2 ** 31 - 4095, 1), (1, 2 ** 31 - 64), (2 ** 27 - 1, 16), (2 ** 26 - 1, 32)])
def test_positions_next_to_the_end_of_an_int(max_pages, page_size):
    """A length that fills such a table (or one that is clamped to it) would take the first position of a following step or tile past
    2^31, and the look-up of its page in front of the table."""
    lib, ctx = mrp.load_library(), C.cast(C.create_string_buffer(1 << 14), C.c_void_p)
    qk = bd._Qk(8, 2, 128, 64, 1, 1, 1, 1e-6, A, A, A, 100)
    rows = bd._NewRows(3, 4, A, A)
    cache = bd._PagedCache(A, A, 1, 2, 128, 1, page_size, A, max_pages, None, None)
    attn = bd._Attn(8, 1, 0.1, 1, 0, 0)
    for call in (lambda: lib.mrp_cache_append(ctx, None, 12, rows, qk, A, 1024, A, 256, A, 256, cache, A),
                 lambda: lib.mrp_paged_attention(ctx, None, 12, rows, cache, attn, A, 1024, A, None, A, 1 << 60)):
        assert call() == SHAPE and b"a sequence out of range" in lib.mrp_last_error(ctx)      # (and not for want of a device)


def test_the_largest_table_is_taken():
    lib, ctx = mrp.load_library(), C.cast(C.create_string_buffer(1 << 14), C.c_void_p)
    cache = bd._PagedCache(A, A, 1, 2, 128, 1, 4096, A, 2 ** 19 - 1, None, None)          # 2^31 - 4096 positions
    qk = bd._Qk(8, 2, 128, 64, 1, 1, 1, 1e-6, A, A, A, 100)
    assert lib.mrp_cache_append(ctx, None, 0, bd._NewRows(3, 4, A, A), qk, A, 1024, A, 256, A, 256, cache, A) == 0


def test_sizes_that_an_int_does_not_hold():
    """ctypes keeps the low 32 bits of a size: what does not fit is refused, not taken for another."""
    with pytest.raises(mrp.MrpError, match="max_new"):
        mrp.NewRows(torch.zeros(3, dtype=torch.int32), 2 ** 32 + 1)
    ctx = object.__new__(mrp.MrpContext)                   # (nothing of a context is looked at before)
    with pytest.raises(mrp.MrpError, match="n_pos"):
        ctx.rope_table(2 ** 32 + 8, 64, 1e4)
    with pytest.raises(mrp.MrpError, match="rotary_dim"):
        ctx.rope_table(8, 2 ** 32 + 64, 1e4)


def test_batches_of_no_sequence():
    """B = 0 is a batch like any other; the table of such a batch has no address."""
    lib, ctx = mrp.load_library(), C.cast(C.create_string_buffer(1 << 14), C.c_void_p)
    qk = bd._Qk(8, 2, 128, 64, 1, 1, 1, 1e-6, A, A, A, 100)
    cache = bd._PagedCache(A, A, 1, 2, 128, 1, 16, None, 5, None, None)
    for n in (0, 12):                                      # (rows of no sequence are left as they are)
        for cu in (None, A):
            rows = bd._NewRows(0, 4, cu, None)
            assert lib.mrp_cache_append(ctx, None, n, rows, qk, A, 1024, A, 256, A, 256, cache, A) == 0
            assert lib.mrp_paged_attention(ctx, None, n, rows, cache, bd._Attn(8, 1, 0.1, 1, 0, 0), A, 1024, A, None, None, 0) == 0
