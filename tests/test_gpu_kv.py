"""The key/value cache against plain forms in 64 bits, at the sizes, masks, strides and contents where it can go wrong.

What the cache holds is compared with the storages' definitions bit for bit, so the other tests take the stored values from
`read`.  Tolerances of attention, from the number formats (u: half a unit in the last place, 2^-8 for bfloat16, 2^-11 for half):
  out  u_out |o|                    its own rounding
       + u_w A, A = sum w|v|/sum w  the weights' rounding for the second product (in the storage's type; 8-bit codes: half, twice,
                                    as the values' scales are part of them)
       + e A                        e: relative error of a weight: twice the scores' error, (D + 8) 2^-24 sum|q k| scale at most
                                    each, and 2^-20 for the exponential, the sums and the scale
  lse  half of e, and 2^-20 of its size
"""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B

pytestmark = pytest.mark.gpu

STORAGES = {"f16": B.PK_F16, "bf16": B.PK_BF16, "i8": B.PK_I8, "f8": B.PK_F8}
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
U = {torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}


class Setup:
    """A cache whose sequences have `lens` tokens, the last `news` of them the batch's.  missing: table entries that are -1.
    The pages are taken in a random order out of more than are needed, and hold garbage (NaN for 16 bits) at first."""

    def __init__(self, storage, dtype, H, G, D, P, news, lens, seed=0, missing=(), spread=1.0, garbage=0xff, tail=0):
        self.gen = torch.Generator().manual_seed(seed)
        self.H, self.G, self.D, self.P, self.news, self.lens = H, G, D, P, news, lens
        self.storage, self.kind = storage, TYPES[dtype]
        pages = [-(-l // P) for l in lens]
        total = sum(pages) + 3
        self.cache = B.KVCache(total, H, D, storage=STORAGES[storage], page_tokens=P)
        self.cache.arena.fill_(garbage)
        order = torch.randperm(total, generator=self.gen)
        self.tables = torch.full((len(lens), max(max(pages), 1) + tail), -1, dtype=torch.int32)
        at = 0
        for i, m in enumerate(pages):
            self.tables[i, :m] = order[at:at + m].int()
            at += m
        for i, j in missing:
            self.tables[i, j] = -1
        self.k, self.v = ([self.normal(l, H, D, spread=spread) for l in lens] for _ in range(2))
        self.q = self.normal(sum(news), H * G, D, spread=spread)
        self.write(news=lens, rows=(self.k, self.v))
        self.batch = self.make_batch(news, lens)

    def normal(self, *shape, spread=1.0):
        x = torch.randn(*shape, generator=self.gen) * torch.exp(spread * torch.randn(*shape[:-1], 1, generator=self.gen))
        return x.to(self.kind)

    def make_batch(self, news, lens):
        offsets = torch.tensor([0] + list(news)).cumsum(0).int()
        return B.KVBatch(self.tables.cuda(), offsets.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), int(sum(news)), max(max(news), 0), max(max(lens), 1))

    def write(self, news, rows, lens=None):
        if sum(news):
            self.cache.append(torch.cat(rows[0]).cuda(), torch.cat(rows[1]).cuda(), self.make_batch(news, lens or self.lens))

    def stored(self):
        """Keys and values as they are held, [token, head, channel] of each sequence; zeros in missing pages."""
        got = self.cache.read(self.make_batch(self.lens, self.lens), torch.float32) if sum(self.lens) else (torch.zeros(0, self.H, self.D).cuda(),) * 2
        return tuple(list(torch.split(x.cpu().double(), self.lens)) for x in got)

    def there(self, i):
        """Which of a sequence's tokens lie in pages that it has."""
        return (self.tables[i] >= 0).repeat_interleave(self.P)[:self.lens[i]]

    def tokens(self):
        """(row of the batch, sequence, position)"""
        row = 0
        for i, (m, l) in enumerate(zip(self.news, self.lens)):
            for j in range(m):
                yield row, i, l - m + j
                row += 1

    def check(self, out, lse, scale, seen):
        """seen(row, sequence, position, head): which keys of its sequence a query sees."""
        ks, vs = self.stored()
        u_out, u_w = U[self.kind], 2 * U[torch.float16] if self.storage in ("i8", "f8") else U[self.kind]
        out, q = out.cpu().double(), self.q.double()
        for row, i, pos in self.tokens():
            for h in range(self.H):
                mask = seen(row, i, pos, h)
                k, v = ks[i][mask, h], vs[i][mask, h]
                for g in range(h * self.G, (h + 1) * self.G):
                    where = f"row {row} sequence {i} position {pos} head {g}"
                    if k.shape[0] == 0:
                        assert torch.all(out[row, g] == 0), where
                        assert lse is None or lse[row, g] == -math.inf, where
                        continue
                    x = (k @ q[row, g]) * scale
                    w = torch.softmax(x, 0)
                    size = float(((k.abs() @ q[row, g].abs()) * abs(scale)).max())
                    e = 2 * (self.D + 8) * 2.0 ** -24 * size + 2.0 ** -20
                    ref, a = w @ v, w @ v.abs()
                    bound = u_out * ref.abs() + (u_w + e) * (1 + u_out) * a + (2.0 ** -24 if self.kind == torch.float16 else 1e-38)
                    off = (out[row, g] - ref).abs()
                    assert torch.all(off <= bound), f"{where}: {float((off / bound).max())} of the bound"
                    if lse is not None:
                        full = float(torch.logsumexp(x, 0))
                        assert abs(float(lse[row, g]) - full) <= e / 2 + 2.0 ** -20 * abs(full), where


def definition(x, storage, kind):
    """Stored values of rows by the storage's definition, in the 32 bits that it is stated in."""
    x = x.float()
    if storage in ("f16", "bf16"):
        return x.to(TYPES[storage]).float()
    largest = 127.0 if storage == "i8" else 448.0
    most = x.abs().amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, largest) / most, torch.zeros_like(most))
    y = (x * up).clamp(-largest, largest)
    y = y.round() if storage == "i8" else y.to(torch.float8_e4m3fn).float()
    return y * (most * torch.tensor(1.0 / largest, dtype=torch.float32))


def bounds_of(rows):
    """hi, lo by the definition, from the stored values [token, head, channel] (float32)."""
    hi, lo = rows.amax(0), rows.amin(0)
    most = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, 127.0) / most, torch.zeros_like(most))
    scale = most * torch.tensor(1.0 / 127.0, dtype=torch.float32)
    return (hi * up - 2.0 ** -10).ceil().clamp(-127, 127), (lo * up + 2.0 ** -10).floor().clamp(-127, 127), scale


@pytest.mark.parametrize("storage,dtype", [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("i8", "f32"), ("f8", "f16"), ("f8", "f32"), ("bf16", "f32"), ("f16", "bf16")])
@pytest.mark.parametrize("H,D,P,lens", [(2, 64, 16, [1, 16, 17, 45]), (3, 80, 64, [0, 63, 64, 130]), (1, 128, 32, [33, 1]), (2, 256, 128, [257]), (1, 8, 64, [70])])
def test_what_is_written_is_what_the_definition_says(gpu_device, storage, dtype, H, D, P, lens):
    s = Setup(storage, dtype, H, 1, D, P, lens, lens, seed=1)
    if lens[-1] > 3:
        s.k[-1][3] = 0  # a row of zeros
        s.k[-1][2] = (s.k[-1][2].float() * 1e-6).to(s.kind)
        s.write(lens, (s.k, s.v))
    for want in (torch.float32, torch.float16, torch.bfloat16):
        for got, rows in zip(s.cache.read(s.batch, want), (s.k, s.v)):
            assert torch.equal(got.cpu(), definition(torch.cat(rows), storage, s.kind).to(want))
    pages = s.tables[s.tables >= 0]
    hi, lo = s.cache.bounds(pages.cuda())
    at = 0
    for i, l in enumerate(lens):
        held = definition(s.k[i], storage, s.kind)
        for j in range(-(-l // P)):
            h, w, scale = bounds_of(held[j * P:(j + 1) * P])
            assert torch.equal(hi[at].cpu(), h * scale) and torch.equal(lo[at].cpu(), w * scale), (i, j)
            at += 1


@pytest.mark.parametrize("storage,dtype,D,P", [("i8", "bf16", 64, 16), ("f8", "f16", 128, 64), ("bf16", "bf16", 96, 32), ("f16", "f16", 256, 128)])
def test_pages_do_not_depend_on_how_their_tokens_came(gpu_device, storage, dtype, D, P):
    """Chunks that begin and end inside pages, and single tokens, leave what one call leaves."""
    lens = [3 * P + 5, P, 7]
    whole = Setup(storage, dtype, 2, 1, D, P, lens, lens, seed=2)
    parts = Setup(storage, dtype, 2, 1, D, P, lens, lens, seed=2)
    parts.cache.arena.fill_(0xff)
    have = [0, 0, 0]
    for step in (1, 5, P, 1, 2 * P, 3):
        news = [min(step, l - n) for n, l in zip(have, lens)]
        parts.write(news, [[x[i][n:n + m] for i, (n, m) in enumerate(zip(have, news))] for x in (parts.k, parts.v)], lens=[n + m for n, m in zip(have, news)])
        have = [n + m for n, m in zip(have, news)]
    assert have == lens
    for a, b in zip(whole.cache.read(whole.batch, torch.float32), parts.cache.read(parts.batch, torch.float32)):
        assert torch.equal(a, b)
    pages = whole.tables[whole.tables >= 0].cuda()
    for a, b in zip(whole.cache.bounds(pages), parts.cache.bounds(pages)):
        assert torch.equal(a, b)


SHAPES = [
    # H, G, D, P, news, lens
    (1, 1, 64, 16, [1], [1]),
    (2, 4, 128, 64, [1, 1, 1], [1, 64, 65]),
    (3, 5, 64, 16, [7, 0, 1], [40, 0, 129]),
    (1, 8, 96, 32, [3, 17], [3, 130]),
    (2, 3, 256, 128, [2], [300]),
    (1, 16, 128, 64, [1, 1], [700, 1300]),
    (1, 20, 80, 16, [2], [100]),
    (2, 2, 128, 64, [90, 5], [90, 333]),
    (1, 4, 64, 32, [200], [517]),
    (1, 7, 128, 64, [131], [1031]),
]


@pytest.mark.parametrize("storage,dtype", [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("window", [0, 50])
def test_attention(gpu_device, storage, dtype, shape, window):
    H, G, D, P, news, lens = shape
    s = Setup(storage, dtype, H, G, D, P, news, lens, seed=3, tail=2)
    scale = D ** -0.5
    out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, window=window, want_lse=True)
    key = [torch.arange(l) for l in lens]
    s.check(out, lse.cpu(), scale, lambda row, i, pos, h: (key[i] <= pos) & (key[i] > pos - (window or 1 << 30)))
    assert torch.equal(s.cache.attend(s.q.cuda(), s.batch, scale, window=window), out)


PARTS = [
    # what the kernels cut: a long context of few queries (joined by the last workgroup, and by a launch of their own where there are
    # many), a chunk over a long context, wide heads, whole chunks from position 0
    (2, 4, 128, 64, [1], [2100]),
    (8, 1, 64, 16, [1] * 16, [1100 + 13 * i for i in range(16)]),
    (1, 4, 64, 32, [70], [2100]),
    (1, 4, 128, 64, [70, 3], [1601, 900]),
    (1, 2, 256, 64, [40, 1], [150, 700]),
    (1, 3, 256, 16, [30], [90]),
    (2, 1, 128, 128, [300], [300]),
]


@pytest.mark.parametrize("storage,dtype", [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("shape", PARTS, ids=lambda s: f"{s[:4]} {len(s[4])} of {max(s[4])} at {max(s[5])}")
def test_attention_in_parts(gpu_device, storage, dtype, shape):
    H, G, D, P, news, lens = shape
    s = Setup(storage, dtype, H, G, D, P, news, lens, seed=16)
    scale = D ** -0.5
    key = [torch.arange(l) for l in lens]
    out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
    s.check(out, lse.cpu(), scale, lambda row, i, pos, h: key[i] <= pos)
    for _ in range(3):
        assert torch.equal(s.cache.attend(s.q.cuda(), s.batch, scale), out)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16")])
@pytest.mark.parametrize("P", [16, 64])
@pytest.mark.parametrize("news", [[32], [33], [64], [65], [32, 33, 64, 65, 1], [129, 0, 128]], ids=str)
def test_either_side_of_few_rows(gpu_device, storage, dtype, P, news):
    """Sequences of 64, 66, 128 and 130 rows of queries: the kernel for few takes 64 of 16 bits at most, 128 of 8."""
    s = Setup(storage, dtype, 1, 2, 128, P, news, [n + 150 for n in news], seed=21)
    scale = 128 ** -0.5
    key = [torch.arange(l) for l in s.lens]
    out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
    s.check(out, lse.cpu(), scale, lambda row, i, pos, h: key[i] <= pos)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16")])
@pytest.mark.parametrize("scale", [-0.07, 0.0, 3.0])
def test_scales_of_any_sign(gpu_device, storage, dtype, scale):
    for news in ([2, 1], [90, 1]):
        s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=17, spread=0.3)
        key = [torch.arange(l) for l in s.lens]
        out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
        s.check(out, lse.cpu(), scale, lambda row, i, pos, h: key[i] <= pos)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("f8", "f16"), ("i8", "bf16")])
def test_attention_without_some_pages(gpu_device, storage, dtype):
    """Pages that the table has not: their keys are not seen, and a query without keys has zeros."""
    s = Setup(storage, dtype, 2, 3, 64, 16, [5, 1, 20, 33], [70, 17, 20, 90], seed=4, missing=[(0, 0), (0, 2), (1, 0), (1, 1), (2, 0), (3, 5), (3, 4), (3, 3)])
    key = [torch.arange(l) for l in s.lens]
    out, lse = s.cache.attend(s.q.cuda(), s.batch, 0.125, want_lse=True)
    s.check(out, lse.cpu(), 0.125, lambda row, i, pos, h: (key[i] <= pos) & s.there(i))
    assert torch.all(out[5] == 0)  # the second sequence has no page at all
    out = s.cache.attend(s.q.cuda(), s.batch, 0.125, window=7)
    s.check(out, None, 0.125, lambda row, i, pos, h: (key[i] <= pos) & (key[i] > pos - 7) & s.there(i))


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f8", "f16")])
def test_rows_of_any_size(gpu_device, storage, dtype):
    """Tokens whose keys and values differ in size by many powers of two, and scores of some hundred."""
    s = Setup(storage, dtype, 2, 2, 64, 64, [3, 1], [200, 75], seed=5, spread=2.5)
    scale = 0.5
    key = [torch.arange(l) for l in s.lens]
    out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
    s.check(out, lse.cpu(), scale, lambda row, i, pos, h: key[i] <= pos)


def test_tiny_and_large_values_of_8_bits(gpu_device):
    """Values near the ends of what bfloat16 holds come back with their size: their scale is not put through half precision."""
    for size in (1e-30, 1e30):
        s = Setup("i8", "bf16", 1, 4, 64, 16, [1], [100], seed=6)
        s.v = [(x.float() * size).to(s.kind) for x in s.v]
        s.write(s.lens, (s.k, s.v))
        key = torch.arange(100)
        s.check(s.cache.attend(s.q.cuda(), s.batch, 0.125), None, 0.125, lambda row, i, pos, h: key <= pos)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16")])
def test_strides_and_alignment(gpu_device, storage, dtype):
    """Rows that are parts of wider ones and begin at any element; tables that are parts of wider ones."""
    s = Setup(storage, dtype, 2, 2, 80, 32, [9, 4], [50, 71], seed=7)
    n, key = sum(s.lens), [torch.arange(l) for l in s.lens]
    wide = torch.zeros(n, 2 * (2 * 80 + 3) + 1, dtype=s.kind, device="cuda")
    k, v = (torch.as_strided(wide, (n, 2, 80), (wide.stride(0), 163, 1), at) for at in (1, 82))
    k.copy_(torch.cat(s.k))
    v.copy_(torch.cat(s.v))
    s.cache.arena.fill_(0xff)
    tables = torch.full((2, 11), 77, dtype=torch.int32, device="cuda")
    tables[:, 2:2 + s.tables.shape[1]] = s.tables.cuda()
    t = tables[:, 2:2 + s.tables.shape[1]]
    offsets = torch.tensor([0, 50, 121], dtype=torch.int32, device="cuda")
    s.cache.append(k, v, B.KVBatch(t, offsets, s.batch.lens, n, 71, 71))
    q = torch.zeros(13, 7, 81, dtype=s.kind, device="cuda")[:, 2:6, 1:]
    q.copy_(s.q)
    out = s.cache.attend(q, B.KVBatch(t, s.batch.offsets, s.batch.lens, 13, 9, 71), 0.1)
    s.check(out, None, 0.1, lambda row, i, pos, h: key[i] <= pos)


def choose(s, n, sink, local):
    """Blocks by the definition, in whole numbers and the 32 bits that it is stated in."""
    pages = s.tables.clamp(min=0).flatten().cuda()
    hi, lo = (x.cpu().view(*s.tables.shape, s.H, s.D) for x in s.cache.bounds(pages))
    most = torch.maximum(hi.abs(), lo.abs()).amax(-1, keepdim=True)
    unit = torch.where(most > 0, most / 127, torch.ones_like(most)).double()
    chi, clo = (hi / unit).round(), (lo / unit).round()
    scale = most[..., 0] / 127  # of codes times scale: what the scale was
    x = s.q.float()
    top = x.abs().amax(-1, keepdim=True)
    up = torch.where(top > 0, torch.full_like(top, 127.0) / top, torch.zeros_like(top))
    code, qs = (x * up).round().clamp(-127, 127).double(), (top * torch.tensor(1 / 127.0, dtype=torch.float32))[..., 0]
    chosen = torch.full((sum(s.news), s.H, n), -1, dtype=torch.int32)
    margin = math.inf
    for row, i, pos in s.tokens():
        mine = pos // s.P
        for h in range(s.H):
            c = code[row, h * s.G:(h + 1) * s.G]
            u = c.clamp(min=0) @ chi[i, :mine + 1, h].T + c.clamp(max=0) @ clo[i, :mine + 1, h].T  # [head, block]
            score = (u.float() * qs[row, h * s.G:(h + 1) * s.G, None]).amax(0) * scale[i, :mine + 1, h]
            block = torch.arange(mine + 1)
            score[(block < sink) | (block > mine - local)] = math.inf
            ok = s.tables[i, :mine + 1] >= 0
            order = sorted(block[ok].tolist(), key=lambda b: (-float(score[b]), b))
            take = sorted(order[:n])
            chosen[row, h, :len(take)] = torch.tensor(take, dtype=torch.int32)
            if len(order) > n and math.isfinite(score[order[n - 1]]):
                gap = float(score[order[n - 1]] - score[order[n]])
                if gap > 0:
                    margin = min(margin, gap / abs(float(score[order[n - 1]])))
    return chosen, margin


@pytest.mark.parametrize("storage,dtype", [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("H,G,D,P,news,lens,n,sink,local", [
    (2, 4, 128, 64, [1, 1], [1, 1500], 8, 1, 2),
    (1, 1, 64, 16, [5, 0, 3], [700, 0, 3], 6, 1, 2),
    (2, 5, 80, 32, [40], [900], 5, 0, 1),
    (1, 16, 256, 16, [2], [4500], 64, 3, 4),
    (1, 20, 64, 16, [1], [300], 3, 1, 2),
])
def test_selection_and_attention_to_it(gpu_device, storage, dtype, H, G, D, P, news, lens, n, sink, local):
    missing = [(0, 3)] if lens[0] > 5 * P else []
    s = Setup(storage, dtype, H, G, D, P, news, lens, seed=8, missing=missing)
    blocks = s.cache.select(s.q.cuda(), s.batch, n, sink=sink, local=local)
    want, margin = choose(s, n, sink, local)
    assert margin > 2.0 ** -20  # no near tie that the scale's own rounding (it is read back) could turn
    assert torch.equal(blocks.cpu(), want)
    scale = D ** -0.5
    mixed = blocks[..., torch.randperm(n, generator=s.gen).cuda()].contiguous()  # in any order
    out, lse = s.cache.attend_blocks(s.q.cuda(), mixed, s.batch, scale, want_lse=True)
    b = blocks.cpu()

    def seen(row, i, pos, h):
        key = torch.arange(lens[i])
        return (key <= pos) & torch.isin(key // P, b[row, h][b[row, h] >= 0]) & s.there(i)
    s.check(out, lse.cpu(), scale, seen)


@pytest.mark.parametrize("H,G,news,lens,n", [(8, 2, [1] * 20, [3000 + 7 * i for i in range(20)], 12), (2, 1, [33], [5000], 40), (1, 3, [9, 2], [8000, 70], 3)])
def test_selection_of_many_blocks(gpu_device, H, G, news, lens, n):
    """Workgroups of four waves and of sixteen, one token each and several, lists of many blocks."""
    s = Setup("bf16", "bf16", H, G, 64, 16, news, lens, seed=18, spread=0.2)
    got = s.cache.select(s.q.cuda(), s.batch, n)
    want, margin = choose(s, n, 1, 2)
    same = (got.cpu() == want).all(-1)
    # (the scales are read back with a rounding: a choice may differ where two scores are nearer than that)
    assert bool(same.all()) or margin < 2.0 ** -20
    assert float(same.float().mean()) > 0.99
    assert torch.equal(s.cache.select(s.q.cuda(), s.batch, n), got)


def test_equal_blocks_and_empty_lists(gpu_device):
    """Blocks of equal scores: the lower ones.  Lists without a block, and with numbers that there are no blocks for."""
    s = Setup("bf16", "bf16", 1, 2, 64, 16, [1], [16 * 40], seed=9)
    s.k = [s.k[0][:16].repeat(40, 1, 1)]
    s.write(s.lens, (s.k, s.v))
    got = s.cache.select(s.q.cuda(), s.batch, 9, sink=1, local=2).cpu()[0, 0]
    assert got.tolist() == [0, 1, 2, 3, 4, 5, 6, 38, 39]
    zeros = torch.zeros_like(s.q).cuda()
    assert s.cache.select(zeros, s.batch, 9, sink=0, local=1).cpu()[0, 0].tolist() == [0, 1, 2, 3, 4, 5, 6, 7, 39]
    empty = torch.full((1, 1, 5), -1, dtype=torch.int32, device="cuda")
    out, lse = s.cache.attend_blocks(s.q.cuda(), empty, s.batch, 0.1, want_lse=True)
    assert torch.all(out == 0) and torch.all(lse == -math.inf)
    odd = torch.tensor([[[40, 2 ** 30, -7, 39, 41]]], dtype=torch.int32, device="cuda")
    key = torch.arange(640)
    s.check(s.cache.attend_blocks(s.q.cuda(), odd, s.batch, 0.1), None, 0.1, lambda row, i, pos, h: key >= 39 * 16)


def test_every_block_listed_is_attention_to_all(gpu_device):
    s = Setup("i8", "bf16", 2, 4, 128, 64, [3, 40], [500, 650], seed=10)
    blocks = s.cache.select(s.q.cuda(), s.batch, 11)
    key = [torch.arange(l) for l in s.lens]
    s.check(s.cache.attend_blocks(s.q.cuda(), blocks, s.batch, 0.09), None, 0.09, lambda row, i, pos, h: key[i] <= pos)


def test_tables_shared_and_beyond_the_batch(gpu_device):
    """Two sequences over the same pages; host bounds that are larger than what the arrays hold."""
    s = Setup("i8", "f16", 2, 2, 64, 32, [4], [100], seed=11)
    q = torch.cat([s.q, s.q.flip(0)]).cuda()
    t = s.tables.repeat(2, 1).cuda()
    two = B.KVBatch(t, torch.tensor([0, 4, 8], dtype=torch.int32, device="cuda"), torch.tensor([100, 100], dtype=torch.int32, device="cuda"), 8, 8, 5000)
    out = s.cache.attend(q, two, 0.1)
    key = torch.arange(100)
    s.check(out[:4], None, 0.1, lambda row, i, pos, h: key <= pos)
    s.q = s.q.flip(0)
    s.check(out[4:], None, 0.1, lambda row, i, pos, h: key <= pos)


def test_calls_in_a_graph_follow_the_arrays(gpu_device):
    """A step captured once serves later ones: lengths and rows change between the replays, and every one is checked."""
    P, lens = 16, [40, 100]
    s = Setup("i8", "bf16", 2, 4, 64, P, [1, 1], [l + 8 for l in lens], seed=12)
    now = torch.tensor(lens, dtype=torch.int32, device="cuda")
    batch = B.KVBatch(s.batch.tables, s.batch.offsets, now, 2, 1, 200)
    k, v = (torch.empty(2, 2, 64, dtype=s.kind, device="cuda") for _ in range(2))
    q = torch.empty(2, 8, 64, dtype=s.kind, device="cuda")

    def step():
        s.cache.append(k, v, batch)
        blocks = s.cache.select(q, batch, 5)
        return s.cache.attend(q, batch, 0.1), blocks, s.cache.attend_blocks(q, blocks, batch, 0.1)

    def fill(j):
        now.copy_(torch.tensor([l + j + 1 for l in lens], dtype=torch.int32))
        k.copy_(torch.stack([s.k[i][l + j] for i, l in enumerate(lens)]))
        v.copy_(torch.stack([s.v[i][l + j] for i, l in enumerate(lens)]))
        q.copy_(s.normal(2, 8, 64))
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for j in range(6):
        fill(j)
        s.cache.arena[:0].zero_()
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in got]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b), j


def test_on_another_stream(gpu_device):
    s = Setup("bf16", "bf16", 2, 2, 64, 64, [30], [300], seed=13)
    q = s.q.cuda()
    want = s.cache.attend(q, s.batch, 0.1)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = s.cache.attend(q, s.batch, 0.1)
        torch.cuda.current_stream().synchronize()
    assert torch.equal(got, want)


def test_a_long_cache_has_offsets_beyond_32_bits(gpu_device):
    """Keys alone take 6 GB; the last pages are the ones in use."""
    H, D, P = 8, 128, 64
    pages = 6 * 2 ** 30 // (H * D * P)
    cache = B.KVCache(pages, H, D, storage=B.PK_I8, page_tokens=P)
    s = Setup("i8", "f16", H, 2, D, P, [3], [200], seed=14)
    s.cache, s.tables = cache, torch.tensor([[pages - 1, pages - 3, pages // 2, pages - 2]], dtype=torch.int32)
    s.write(s.lens, (s.k, s.v))
    for got, rows in zip(s.cache.read(s.make_batch(s.lens, s.lens), torch.float32), (s.k, s.v)):
        assert torch.equal(got.cpu(), definition(torch.cat(rows), "i8", s.kind))
    s.batch = s.make_batch(s.news, s.lens)
    key = torch.arange(200)
    s.check(cache.attend(s.q.cuda(), s.batch, 0.1), None, 0.1, lambda row, i, pos, h: key <= pos)
    blocks = cache.select(s.q.cuda(), s.batch, 4)
    s.check(cache.attend_blocks(s.q.cuda(), blocks, s.batch, 0.1), None, 0.1, lambda row, i, pos, h: key <= pos)
    cache.close()


def test_refusals(gpu_device):
    s = Setup("bf16", "bf16", 2, 2, 64, 16, [2], [20], seed=15)
    q, k = s.q.cuda(), torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(B.PancakeError) as e:
        s.cache.attend(q.half(), s.batch, 0.1)
    assert e.value.status == B.PK_ERR_UNSUPPORTED
    with pytest.raises(B.PancakeError) as e:
        s.cache.attend(q.float(), s.batch, 0.1)
    assert e.value.status == B.PK_ERR_UNSUPPORTED
    with pytest.raises(B.PancakeError) as e:
        s.cache.attend(q[:, :3], s.batch, 0.1)  # three query heads on two
    assert e.value.status == B.PK_ERR_INVALID_ARG
    for bad in (dict(window=-1), dict(scale=math.nan), dict(scale=math.inf)):
        with pytest.raises(B.PancakeError) as e:
            s.cache.attend(q, s.batch, **{"scale": 0.1, **bad})
        assert e.value.status == B.PK_ERR_INVALID_ARG
    for n, sink, local in ((0, 0, 1), (4, -1, 1), (4, 1, 0), (4, 2, 3)):
        with pytest.raises(B.PancakeError) as e:
            s.cache.select(q, s.batch, n, sink=sink, local=local)
        assert e.value.status == B.PK_ERR_INVALID_ARG
    with pytest.raises(B.PancakeError) as e:
        s.cache.append(k, k.float(), s.batch)
    assert e.value.status == B.PK_ERR_INVALID_ARG
    with pytest.raises(ValueError):
        s.cache.append(k[:1], k[:1], s.batch)
    with pytest.raises(ValueError):
        s.cache.append(k[..., ::2], k[..., ::2], s.batch)
    with pytest.raises(ValueError):
        s.cache.append(k.cpu(), k.cpu(), s.batch)
    with pytest.raises(ValueError):
        s.cache.attend(q.double(), s.batch, 0.1)
    nothing = B.KVBatch(s.batch.tables, torch.zeros(2, dtype=torch.int32, device="cuda"), s.batch.lens, 0, 0, 20)
    assert s.cache.attend(q[:0], nothing, 0.1).shape == (0, 4, 64)
    s.cache.append(k[:0], k[:0], nothing)


def test_batches_beyond_a_launch_are_refused(gpu_device):
    """Numbers that no launch could take are refused by the host, before anything runs."""
    cache = B.KVCache(1, 1, 8, storage=B.PK_F16, page_tokens=16)
    one = torch.zeros(8, dtype=torch.int32, device="cuda")
    rows = torch.zeros((1, 1, 8), dtype=torch.float16, device="cuda")
    most = 2 ** 31 - 1
    batch = B.pk_kv_batch(one.data_ptr(), one.data_ptr(), one.data_ptr(), 2 ** 26, 1, 2 ** 26, most, most, 2 ** 30)
    for call in (lambda: B.pk_kv_append(cache.handle, batch, rows, rows), lambda: B.pk_kv_read(cache.handle, batch, rows, rows.clone()),
                 lambda: B.pk_kv_attend(cache.handle, batch, rows, 1.0, 0, rows.clone())):
        with pytest.raises(B.PancakeError) as e:
            call()
        assert e.value.status == B.PK_ERR_UNSUPPORTED
