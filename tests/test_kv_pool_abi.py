"""Host-side checks of the entry points over a cache's pages (no kernel is launched, no GPU needed)."""
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


def test_pool_bytes(lib):
    a = B.pk_kv_pool_bytes(B.pk_kv_config(1000, 2, 64, 64, B.PK_I8))
    assert 4 * 4 * 1000 <= a <= 4 * 4 * 1000 + 2 * 4 * 32 + 3 * 4 * 65535 + 9 * 256
    assert B.pk_kv_pool_bytes(B.pk_kv_config(0x7fffffff, 1, 8, 16, B.PK_I8)) > 16 * 0x7fffffff
    assert B.pk_kv_pool_bytes(B.pk_kv_config(0, 2, 64, 64, B.PK_I8)) == 0
    assert lib.pk_kv_pool_bytes(None) == 0


def test_checks_before_anything_runs(lib):
    null, out, some = C.c_void_p(None), C.c_void_p(), C.c_void_p(256)
    fake = C.cast((C.c_uint64 * 64)(), C.c_void_p)
    batch, tables = B.pk_kv_batch(), B.pk_kv_tables()
    assert lib.pk_kv_pool_create(fake, some, 1 << 30, None) == B.PK_ERR_INVALID_ARG
    for handle in (null, fake):
        assert lib.pk_kv_pool_create(handle, some, 1 << 30, C.byref(out)) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_free(handle) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_clear(handle, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_adopt(handle, tables, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_grant(handle, batch, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_fork(handle, tables, null, null, null, 0, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_release(handle, tables, null, null, 0, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_compact(handle, handle, tables, tables, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_pool_counts(handle, null, null) == B.PK_ERR_BAD_HANDLE
        assert lib.pk_kv_copy(handle, handle, null, null, 0, null) == B.PK_ERR_BAD_HANDLE
