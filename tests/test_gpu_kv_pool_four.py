"""The pool over a cache of 4 bits, whose pages have a region of their own (the powers of two of their keys): what branches, compaction and copies of pages leave in them, bit for bit,
rows and bounds alike."""
import pytest
import torch

from paper_2602_21477_amd import binding as B
import test_gpu_kv_pool as pool
from test_gpu_kv_pool import ints

pytestmark = pytest.mark.gpu
pool.STORAGES.setdefault("f4", B.PK_F4)

SHAPES = [("f4", 3, 80, 16), ("f4", 1, 256, 64), ("f4", 2, 64, 128), ("f4", 1, 8, 32)]


class Setup(pool.Setup):
    """Keys whose groups of 32 channels are of sizes that differ, so that their powers of two do."""

    def rows(self, n):
        x = super().rows(n)
        groups = 2.0 ** torch.randint(-9, 1, (n, self.H, -(-self.D // 32), 1), device="cuda", generator=self.gen).float()
        return x * groups.expand(-1, -1, -1, 32).reshape(n, self.H, -1)[..., :self.D]


@pytest.fixture(autouse=True)
def such_rows(monkeypatch):
    monkeypatch.setattr(pool, "Setup", Setup)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_branches_write_into_pages_of_their_own(gpu_device, storage, H, D, P):
    pool.test_branches_write_into_pages_of_their_own(gpu_device, storage, H, D, P)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_the_last_of_a_pages_owners_keeps_it(gpu_device, storage, H, D, P):
    pool.test_the_last_of_a_pages_owners_keeps_it(gpu_device, storage, H, D, P)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_compaction_keeps_what_sequences_hold(gpu_device, storage, H, D, P):
    pool.test_compaction_keeps_what_sequences_hold(gpu_device, storage, H, D, P)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_pages_are_copied_whole(gpu_device, storage, H, D, P):
    pool.test_pages_are_copied_whole(gpu_device, storage, H, D, P)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_selection_from_copied_and_moved_pages(gpu_device, storage, H, D, P):
    """Bounds are copied and moved with their pages: a branch, and what is left after compaction, choose the blocks that the parent chooses."""
    s = Setup(storage, H, D, P, [9 * P + 3, 5 * P], rows=3, spare=6, seed=6)
    s.pool.release(s.tables, ints([1]))
    s.pool.fork(s.tables, ints(s.lens), ints([0]), ints([2]))
    s.lens[2] = s.lens[0]
    q = torch.randn(1, 2 * H, D, device="cuda", generator=s.gen).half()

    def chosen(cache, tables, row, length):
        b = B.KVBatch(tables[row:row + 1], ints([0, 1]), ints([length]), 1, 1, length)
        blocks = cache.select(q, b, 5)
        return blocks, *cache.attend_blocks(q, blocks, b, 0.1, want_lse=True)
    # the branch takes a copy of its last page and writes one token, as its parent does
    k, v = s.rows(1), s.rows(1)
    for row in (2, 0):
        b = pool.batch_of(s.tables, [row], [s.lens[row]], [s.lens[row] + 1])
        assert s.pool.grant(b).item() == 0
        s.cache.append(k, v, b)
    assert s.tables[0, 9] != s.tables[2, 9] and torch.equal(s.tables[0, :9], s.tables[2, :9])
    want = chosen(s.cache, s.tables, 0, s.lens[0] + 1)
    into = B.KVPool(B.KVCache(40, H, D, storage=B.PK_F4, page_tokens=P))
    into.cache.arena.fill_(0xff)
    tables, missing = s.pool.compact(into, s.tables)
    assert missing.item() == 0
    for got in (chosen(s.cache, s.tables, 2, s.lens[0] + 1), chosen(into.cache, tables, 0, s.lens[0] + 1), chosen(into.cache, tables, 2, s.lens[0] + 1)):
        for a, b in zip(got, want):
            assert torch.equal(a, b)
