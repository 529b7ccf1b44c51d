"""The pool of a cache's pages against a model of it on the host: whole numbers and copied bytes, so everything has to be equal."""
import pytest
import torch

from paper_2602_21477_amd import binding as B

pytestmark = pytest.mark.gpu


class Model:
    """Tables and owners as the entry points' contract says, one entry after the other."""

    def __init__(self, n_pages, rows, cols, P):
        self.n, self.P, self.refs, self.t = n_pages, P, [0] * n_pages, [[-1] * cols for _ in range(rows)]
        self.copied = []

    def there(self, e):
        return 0 <= e < self.n

    def grant(self, seqs, begins, lens):
        """Rows `seqs` of the tables get tokens begin .. len - 1."""
        touched = [(s, j, b > j * self.P) for s, b, l in zip(seqs, begins, lens) if l > b for j in range(b // self.P, min((l - 1) // self.P, len(self.t[s]) - 1) + 1)]
        users, last, free = {}, {}, [p for p in range(self.n) if self.refs[p] == 0]
        for s, j, _ in touched:
            e = self.t[s][j]
            if self.there(e) and self.refs[e] > 1:
                users[e], last[e] = users.get(e, 0) + 1, s
        refs, missing = list(self.refs), 0
        for s, j, older in touched:
            e = self.t[s][j]
            if self.there(e) and (refs[e] <= 1 or (users[e] == refs[e] and last[e] == s)):
                continue
            if not self.there(e) and older:
                self.t[s][j], missing = -1, missing + 1
                continue
            if self.there(e):
                self.refs[e] -= 1
            if not free:
                self.t[s][j], missing = -1, missing + 1
                continue
            new = free.pop(0)
            self.refs[new], self.t[s][j] = 1, new
            if self.there(e) and older:
                self.copied.append((new, e))
        return missing

    def fork(self, lens, pairs):
        for f, d in pairs:
            keep = -(-lens[f] // self.P)
            self.t[d] = [e if j < keep and self.there(e) else -1 for j, e in enumerate(self.t[f])]
            for e in self.t[d]:
                if e >= 0:
                    self.refs[e] += 1

    def release(self, rows, keep):
        for r, k in zip(rows, keep):
            for j in range(-(-k // self.P), len(self.t[r])):
                e, self.t[r][j] = self.t[r][j], -1
                if self.there(e) and self.refs[e]:
                    self.refs[e] -= 1

    def compact(self, room):
        live = [p for p in range(self.n) if self.refs[p]]
        name = {p: i for i, p in enumerate(live) if i < room}
        refs = [self.refs[p] for p in live[:room]] + [0] * max(0, room - len(live))
        return [[name.get(e, -1) for e in row] for row in self.t], refs, max(0, len(live) - room), live[:room]


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def batch_of(tables, rows, begins, lens, generous=False):
    """The rows have to be neighbours.  generous: the host only knows that one sequence may have all new tokens."""
    news = [l - b for b, l in zip(begins, lens)]
    return B.KVBatch(tables[rows[0]:rows[-1] + 1], ints([0] + news).cumsum(0).int(), ints(lens), sum(news), sum(news) if generous else max(news), max(max(lens), 1))


def same(pool, model, tables):
    assert pool.counts().tolist() == model.refs
    assert tables.tolist() == model.t


@pytest.mark.parametrize("P,n_pages,rows,cols", [(16, 77, 6, 12), (64, 33, 5, 9), (16, 40000, 40, 64), (128, 1000, 70, 20), (32, 5000, 9, 300)])
@pytest.mark.parametrize("seed", [0, 1, 2, 3])
def test_a_run_of_calls_is_the_model(gpu_device, P, n_pages, rows, cols, seed):
    """Steps that fit a thread for each entry, and others: by the numbers, and as the host knows no better."""
    gen = torch.Generator().manual_seed(seed)

    def pick(n):
        return int(torch.randint(0, max(n, 1), (1,), generator=gen))

    cache = B.KVCache(n_pages, 1, 8, storage=B.PK_I8, page_tokens=P)
    pool, model = B.KVPool(cache), Model(n_pages, rows, cols, P)
    wide = torch.full((rows, cols + 3), 12345678, dtype=torch.int32, device="cuda")
    tables = wide[:, 1:1 + cols]
    tables.fill_(-1)
    lens = [0] * rows
    same(pool, model, tables)
    for step in range(30):
        what = pick(4)
        if what <= 1:  # grant: neighbouring rows, some of them without new tokens
            a = pick(rows)
            some = list(range(a, min(rows, a + 1 + pick(rows))))
            begins = [lens[r] for r in some]
            after = [min(cols * P, b + [0, 1, pick(3 * P), pick(cols * P // 2)][pick(4)]) for b in begins]
            if sum(after) > sum(begins):
                missing = pool.grant(batch_of(tables, some, begins, after, generous=pick(2) == 0))
                assert missing.item() == model.grant(some, begins, after)
                for r, l in zip(some, after):
                    lens[r] = l
        elif what == 2:  # fork: into rows that are empty
            order = torch.randperm(rows, generator=gen).tolist()
            half = rows // 2
            targets = order[:1 + pick(half)]
            sources = [order[half + pick(rows - half)] for _ in targets]
            model.release(targets, [0] * len(targets))
            pool.release(tables, ints(targets))
            model.fork(lens, list(zip(sources, targets)))
            pool.fork(tables, ints(lens), ints(sources), ints(targets))
            for f, d in zip(sources, targets):
                lens[d] = lens[f]
        else:  # release: some rows in part; a row that is not there, and one twice
            some = torch.randperm(rows, generator=gen).tolist()[:1 + pick(rows)]
            keep = [pick(lens[r] + 1) for r in some]
            model.release(some, keep)
            pool.release(tables, ints(some + [rows + 5, -1, some[0]]), ints(keep + [0, 0, keep[0]]))
            for r, k in zip(some, keep):
                lens[r] = min(lens[r], k)
        same(pool, model, tables)
    for room in (sum(1 for x in model.refs if x) + 2, max(1, sum(1 for x in model.refs if x) // 2), n_pages):
        into = B.KVPool(B.KVCache(room, 1, 8, storage=B.PK_I8, page_tokens=P))
        into.adopt(ints([[0, room - 1]]))  # (lost)
        out, missing = pool.compact(into, tables)
        t, refs, short, _ = model.compact(room)
        assert out.tolist() == t and into.counts().tolist() == refs and missing.item() == short
        more = into.grant(batch_of(ints([[-1] * 3]), [0], [0], [2 * P + 1]))  # what is free there is known
        assert more.item() == max(0, 3 - refs.count(0))
    same(pool, model, tables)
    assert torch.all(wide[:, 0] == 12345678) and torch.all(wide[:, 1 + cols:] == 12345678)


SHAPES = [("f16", 3, 64, 16), ("bf16", 2, 128, 64), ("i8", 5, 80, 32), ("f8", 1, 256, 128)]
STORAGES = {"f16": B.PK_F16, "bf16": B.PK_BF16, "i8": B.PK_I8, "f8": B.PK_F8}


class Setup:
    """A cache whose rows' pages come from its pool; what its sequences hold is known on the host."""

    def __init__(self, storage, H, D, P, lens, rows, spare, seed=0):
        self.gen = torch.Generator("cuda").manual_seed(seed)
        self.H, self.D, self.P, self.lens = H, D, P, list(lens) + [0] * (rows - len(lens))
        cols = -(-max(lens) // P) + 3
        self.cache = B.KVCache(sum(-(-l // P) for l in lens) + spare, H, D, storage=STORAGES[storage], page_tokens=P)
        self.cache.arena.fill_(0xff)
        self.pool = B.KVPool(self.cache)
        self.tables = torch.full((rows, cols), -1, dtype=torch.int32, device="cuda")
        self.held = [None] * rows
        self.put(list(range(len(lens))), [0] * len(lens), lens)

    def rows(self, n):
        return torch.randn(n, self.H, self.D, device="cuda", generator=self.gen)

    def put(self, some, begins, lens):
        """Grants and appends; notes what the rows then hold."""
        b = batch_of(self.tables, some, begins, lens)
        missing = self.pool.grant(b)
        self.cache.append(self.rows(b.n_tokens), self.rows(b.n_tokens), b)
        for r, l in zip(some, lens):
            self.lens[r] = l
        for r in some:
            self.held[r] = self.read(r)
        return missing

    def read(self, r, cache=None, tables=None):
        l = self.lens[r]
        b = batch_of(self.tables if tables is None else tables, [r], [0], [l])
        k, v = (cache or self.cache).read(b, torch.float32)
        hi, lo = (cache or self.cache).bounds(b.tables[0, :-(-l // self.P)].contiguous())
        return torch.stack([k, v]), torch.stack([hi, lo])

    def check(self, some, cache=None, tables=None):
        for r in some:
            for a, b in zip(self.read(r, cache, tables), self.held[r]):
                assert torch.equal(a, b), r


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_branches_write_into_pages_of_their_own(gpu_device, storage, H, D, P):
    s = Setup(storage, H, D, P, [2 * P + 5, 3 * P, 1], rows=9, spare=12)
    parents = [x for x in s.held[:3]]
    s.pool.fork(s.tables, ints(s.lens), ints([0, 1, 2, 0, 1, 2]), ints([3, 4, 5, 6, 7, 8]))
    s.lens[3:] = s.lens[:3] * 2
    before = s.tables.clone()
    assert torch.equal(before[3:6], before[:3]) and torch.equal(before[6:], before[:3])
    assert s.put([3, 4, 5, 6, 7, 8], s.lens[3:], [l + m for l, m in zip(s.lens[3:], [1, 1, 1, 2, P, P + 1])]).item() == 0
    s.held[:3] = parents
    s.check(range(9))  # nobody's tokens changed under them
    for i in range(3, 9):
        l = s.lens[i % 3]
        full = l // P
        for a, b in zip(s.held[i][0], parents[i % 3][0]):
            assert torch.equal(a[:l], b)
        assert torch.equal(s.tables[i, :full], before[i, :full])  # full pages are still shared
        if l % P:
            assert s.tables[i, full] != before[i, full]
    s.pool.release(s.tables, ints([3, 4, 5, 6, 7, 8]))
    s.check(range(3))
    assert s.pool.counts().tolist() == [1 if p in before[:3].flatten().tolist() else 0 for p in range(s.cache.cfg.n_pages)]


@pytest.mark.parametrize("storage,H,D,P", SHAPES[:2])
def test_the_last_of_a_pages_owners_keeps_it(gpu_device, storage, H, D, P):
    s = Setup(storage, H, D, P, [P + 3], rows=3, spare=3)
    s.pool.fork(s.tables, ints(s.lens), ints([0, 0]), ints([1, 2]))
    s.lens[1:] = [P + 3] * 2
    page, old = s.tables[0, 1].item(), s.held[0]
    assert s.put([0, 1, 2], [P + 3] * 3, [P + 4] * 3).item() == 0
    assert s.tables[2, 1].item() == page and s.tables[0, 1].item() != page and s.tables[1, 1].item() != page
    for r in range(3):
        for a, b in zip(s.held[r][0], old[0]):
            assert torch.equal(a[:P + 3], b)
    s.check(range(3))
    assert sorted(s.pool.counts().tolist(), reverse=True)[:4] == [3, 1, 1, 1]


def test_too_few_pages(gpu_device):
    """The first in order get what there is; a shared page without a copy is not written into."""
    s = Setup("bf16", 1, 64, 16, [20], rows=3, spare=1)
    s.pool.fork(s.tables, ints(s.lens), ints([0, 0]), ints([1, 2]))
    s.lens[1:] = [20, 20]
    kept = s.held[0]
    b = batch_of(s.tables, [1, 2], [20, 20], [21, 40])
    assert s.pool.grant(b).item() == 2  # a copy for the first; none for the other, nor its third page
    assert s.tables[:, :3].tolist() == [[0, 1, -1], [0, 2, -1], [0, -1, -1]]
    assert s.pool.counts().tolist() == [3, 1, 1]
    s.cache.append(s.rows(21), s.rows(21), b)
    for a, c in zip(s.read(0), kept):
        assert torch.equal(a, c)
    # a page that has gone and would have to hold older tokens stays away
    s.tables[1, 1] = 77
    assert s.pool.grant(batch_of(s.tables, [1], [21], [22])).item() == 1
    assert s.tables[1, :3].tolist() == [0, -1, -1]


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_compaction_keeps_what_sequences_hold(gpu_device, storage, H, D, P):
    s = Setup(storage, H, D, P, [5 * P + 1, P, 3 * P + 7, 2, 4 * P], rows=6, spare=9, seed=3)
    s.pool.release(s.tables, ints([1, 3]))
    s.pool.fork(s.tables, ints(s.lens), ints([2]), ints([5]))
    s.lens[5] = s.lens[2]
    s.held[5] = s.held[2]
    live = sum(1 for x in s.pool.counts().tolist() if x)
    into = B.KVPool(B.KVCache(live, H, D, storage=STORAGES[storage], page_tokens=P))
    into.cache.arena.fill_(0xff)
    tables, missing = s.pool.compact(into, s.tables)
    assert missing.item() == 0 and sorted(set(tables.flatten().tolist())) == list(range(-1, live))
    s.check([0, 2, 4, 5], into.cache, tables)
    s.check([0, 2, 4, 5])
    q = torch.randn(1, 2 * H, D, device="cuda", generator=s.gen).to(torch.bfloat16 if storage == "bf16" else torch.float16)
    a, c = (cache.attend(q, B.KVBatch(t[2:3], ints([0, 1]), ints([s.lens[2]]), 1, 1, s.lens[2]), 0.1) for cache, t in ((s.cache, s.tables), (into.cache, tables)))
    assert torch.equal(a, c)
    out = s.tables.clone()  # in place
    B.pk_kv_pool_compact(s.pool.handle, into.handle, out, out)
    assert torch.equal(out, tables)


@pytest.mark.parametrize("storage,H,D,P", SHAPES)
def test_pages_are_copied_whole(gpu_device, storage, H, D, P):
    s = Setup(storage, H, D, P, [3 * P, 2 * P], rows=2, spare=4, seed=4)
    other = B.KVCache(50, H, D, storage=STORAGES[storage], page_tokens=P)
    other.arena.fill_(0xff)
    source, target = s.tables[0, :3].tolist(), [40, 0, 17]
    other.copy_pages(ints([99, -1] + target + [3]), s.cache, ints([source[0], source[1]] + source + [s.cache.cfg.n_pages]))
    s.check([0], other, ints([target + [-1] * (s.tables.shape[1] - 3)]))
    s.cache.copy_pages(s.tables[1, :2].contiguous(), s.cache, s.tables[0, 1:3].contiguous())  # within the cache
    s.lens[1] = 2 * P
    k, _ = s.read(1)
    assert torch.equal(k[0], s.held[0][0][0][P:])
    s.cache.copy_pages(ints([]), other, ints([]))


def test_a_step_of_branches_in_a_graph(gpu_device):
    """Fork, grant, append, read and release, replayed with other lengths and parents; eager work and grants between the replays."""
    P = 16
    s = Setup("i8", 2, 64, P, [40, 70, 33], rows=9, spare=40, seed=5)
    lens, sources, targets = ints(s.lens[:3] + [0] * 6), ints([0, 1, 2, 0, 1, 2]), ints([3, 4, 5, 6, 7, 8])
    after, offsets = ints([0] * 6), ints(range(7))
    k, v = s.rows(6), s.rows(6)
    b = B.KVBatch(s.tables[3:], offsets, after, 6, 1, 5 * P)
    look = B.KVBatch(s.tables[3:], ints([0, 99, 198, 297, 396, 495, 594]), after, 594, 99, 5 * P)
    state = {}

    def step():
        s.pool.fork(s.tables, lens, sources, targets)
        state["missing"] = s.pool.grant(b)
        s.cache.append(k, v, b)
        state["tables"] = s.tables.clone()
        state["kv"] = s.cache.read(look, torch.float32)
        s.pool.release(s.tables, targets)
        state["counts"] = s.pool.counts()

    def fill(seed):
        gen = torch.Generator().manual_seed(seed)
        sources.copy_(torch.randint(0, 3, (6,), generator=gen, dtype=torch.int32))
        lens[:3] = torch.randint(1, 33, (3,), generator=gen, dtype=torch.int32).cuda()
        after.copy_(lens[sources.long()] + 1)
        k.copy_(s.rows(6))

    fill(0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    captured = dict(state)
    for i in range(1, 5):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        got = {x: (y[0].clone(), y[1].clone()) if x == "kv" else y.clone() for x, y in captured.items()}
        step()
        for x in ("missing", "tables", "counts"):
            assert torch.equal(got[x], state[x]), (i, x)
        for row in range(6):
            n = int(after[row])
            for a, c in zip(got["kv"], state["kv"]):
                assert torch.equal(a[row * 99 + 99 - n:row * 99 + 99], c[row * 99 + 99 - n:row * 99 + 99]), (i, row)


@pytest.mark.parametrize("generous", [False, True])
def test_pools_of_many_pages(gpu_device, generous):
    """300 000 pages, more than a step of either kernel looks at: the lowest free ones, wherever they lie, and ranks among all."""
    n, P = 300_000, 16
    cache = B.KVCache(n, 1, 8, storage=B.PK_I8, page_tokens=P)
    pool = B.KVPool(cache)
    full = torch.arange(290_000, dtype=torch.int32, device="cuda").view(290, 1000)
    pool.adopt(full)
    empty = torch.full((3, 40_000), -1, dtype=torch.int32, device="cuda")
    b = B.KVBatch(empty, ints([0, 1, 1, 18]), ints([1, 0, 17]), 18, 18 if generous else 17, 40_000 * P if generous else 17)
    assert pool.grant(b).item() == 0
    assert empty[:, :2].tolist() == [[290_000, -1], [-1, -1], [290_001, 290_002]] and bool((empty[:, 2:] == -1).all())
    rows = torch.arange(1, 290, 2, dtype=torch.int32, device="cuda")
    pool.release(full, rows)
    more = torch.full((1, 40_000), -1, dtype=torch.int32, device="cuda")
    pages = 11_000  # of the first released rows: eleven and a bit, in 23 000 pages with holes between
    b = B.KVBatch(more, ints([0, pages * P]), ints([pages * P]), pages * P, pages * P, pages * P)
    assert pool.grant(b).item() == 0
    free = torch.arange(290_000, device="cuda").view(290, 1000)[1::2].flatten()[:pages]
    assert torch.equal(more[0, :pages].long(), free)
    counts = pool.counts()
    assert int(counts.sum()) == 145_000 + pages + 3 and int(counts.max()) == 1
    rank = (counts > 0).long().cumsum(0) - 1
    into = B.KVPool(B.KVCache(150_000, 1, 8, storage=B.PK_I8, page_tokens=P))
    whole = torch.cat([full.flatten(), more[0, :pages], empty[0, :1], empty[2, :2]])[None].contiguous()
    out, missing = pool.compact(into, whole)
    want = torch.where(whole >= 0, rank[whole.clamp(min=0).long()], torch.full_like(rank[:1], -1)).int()
    want[want >= 150_000] = -1
    assert torch.equal(out, want) and missing.item() == 145_000 + pages + 3 - 150_000
    assert bool((into.counts() == 1).all())
    cache.close()
    into.cache.close()


def test_refusals(gpu_device):
    cache = B.KVCache(4, 1, 64, page_tokens=16)
    pool, tables = B.KVPool(cache), torch.full((2, 4), -1, dtype=torch.int32, device="cuda")
    for call in (lambda: pool.fork(tables, ints([1]), ints([0]), ints([1])), lambda: pool.fork(tables, ints([1, 1]), ints([0]), ints([1, 0])), lambda: pool.release(tables, ints([0]), ints([1, 2])),
                 lambda: pool.adopt(tables.cpu()), lambda: pool.adopt(tables.long()), lambda: pool.adopt(tables.t()), lambda: cache.copy_pages(ints([0]), cache, ints([0, 1]))):
        with pytest.raises(ValueError):
            call()
    other = B.KVPool(B.KVCache(4, 2, 64, page_tokens=16))
    for call in (lambda: pool.compact(other, tables), lambda: cache.copy_pages(ints([0]), other.cache, ints([0]))):
        with pytest.raises(B.PancakeError) as e:
            call()
        assert e.value.status == B.PK_ERR_DIM_MISMATCH
    with pytest.raises(B.PancakeError) as e:
        pool.compact(pool, tables)
    assert e.value.status == B.PK_ERR_INVALID_ARG
    with pytest.raises(B.PancakeError) as e:
        pool.compact(B.KVPool(cache), tables)  # two pools of one cache
    assert e.value.status == B.PK_ERR_INVALID_ARG
    cache.close()
    with pytest.raises(ValueError):
        pool.counts()
    pool.close()
    other.close()
