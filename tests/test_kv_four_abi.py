"""Host-side checks of a cache in 4 bits (no kernel is launched, no GPU needed)."""
import os

import pytest

from paper_2602_21477_amd import binding as B


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2602_21477_amd import build
        build.build()
    return B.lib()


def test_arena_bytes(lib):
    for heads, dim, held, page in ((2, 64, 64, 64), (3, 80, 128, 16), (1, 256, 256, 128)):
        rows = 10 * heads * page
        # codes of keys and values, a scale each, a byte for 32 channels of a key, bounds; regions are padded to 256 bytes
        need = rows * (held + 2 * 4 + held // 32) + 10 * heads * (2 * held + 4)
        assert need <= B.pk_kv_arena_bytes(B.pk_kv_config(10, heads, dim, page, B.PK_F4)) <= need + 7 * 256
    assert B.pk_kv_arena_bytes(B.pk_kv_config(1000, 8, 128, 64, B.PK_F4)) < 0.58 * B.pk_kv_arena_bytes(B.pk_kv_config(1000, 8, 128, 64, B.PK_I8))
    for bad in (dict(head_dim=60), dict(page_tokens=8), dict(storage=7), dict(storage=5)):
        assert B.pk_kv_arena_bytes(B.pk_kv_config(**{"n_pages": 10, "n_heads": 2, "head_dim": 64, "page_tokens": 64, "storage": B.PK_F4, **bad})) == 0, bad
