"""Host-side checks of the key/value cache's entry points (no kernel is launched, no GPU needed)."""
import ctypes as C
import os

import pytest

from paper_2602_21477_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2602_21477_amd import build
        build.build()
    return B.lib()


def config(n_pages=10, heads=2, dim=64, page=64, storage=B.PK_I8):
    return B.pk_kv_config(n_pages, heads, dim, page, storage)


def test_arena_bytes(lib):
    rows = 10 * 2 * 64 * 64
    # keys and values, their scales, bounds; regions are padded to 256 bytes
    assert 2 * rows + 2 * 10 * 2 * 64 * 4 <= B.pk_kv_arena_bytes(config()) <= 2 * rows + 2 * 10 * 2 * 64 * 4 + 10 * 2 * (2 * 64 + 4) + 6 * 256
    assert 4 * rows <= B.pk_kv_arena_bytes(config(storage=B.PK_BF16)) < B.pk_kv_arena_bytes(config()) * 2
    assert B.pk_kv_arena_bytes(config(n_pages=1 << 24, heads=8, dim=128)) > 1 << 40
    for bad in (dict(n_pages=0), dict(n_pages=1 << 31), dict(heads=0), dict(heads=1025), dict(dim=0), dict(dim=63), dict(dim=264), dict(page=48), dict(page=8),
                dict(page=256), dict(storage=B.PK_F32), dict(storage=5), dict(storage=-1)):
        assert B.pk_kv_arena_bytes(config(**bad)) == 0, bad
    assert lib.pk_kv_arena_bytes(None) == 0


def test_checks_before_anything_runs(lib):
    null, out = C.c_void_p(None), C.c_void_p()
    assert lib.pk_kv_create(None, null, 0, C.byref(out)) == B.PK_ERR_INVALID_ARG
    assert lib.pk_kv_create(C.byref(config()), null, 1 << 30, C.byref(out)) == B.PK_ERR_INVALID_ARG
    assert lib.pk_kv_create(C.byref(config()), C.c_void_p(256 + 8), 1 << 30, C.byref(out)) == B.PK_ERR_INVALID_ARG
    assert lib.pk_kv_create(C.byref(config()), C.c_void_p(256), 100, C.byref(out)) == B.PK_ERR_NOMEM
    assert lib.pk_kv_create(C.byref(config()), C.c_void_p(256), 100, None) == B.PK_ERR_INVALID_ARG
    batch, rows = B.pk_kv_batch(), B.pk_rows()
    fake = C.cast((C.c_uint64 * 64)(), C.c_void_p)
    for handle in (null, fake):
        assert lib.pk_kv_free(handle) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_append(handle, batch, rows, rows, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_read(handle, batch, null, null, 0, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_bounds(handle, null, 0, null, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_attend(handle, batch, rows, 2, 1.0, 0, null, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_select(handle, batch, rows, 2, 4, 1, 2, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_attend_blocks(handle, batch, rows, 2, 1.0, null, 4, null, null, null) == B.PK_ERR_BAD_HANDLE
