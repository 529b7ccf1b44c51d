"""What the key/value cache's header promises beside the values: host numbers that only bound the device arrays, rows of outputs that
belong to no token, scores and lengths at the ends of what 32 bits hold, batches as ragged as they come, exact choices."""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B
from test_gpu_kv import STORAGES, U, Setup, bounds_of, definition

pytestmark = pytest.mark.gpu

CODES = [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16"), ("f8", "f16")]


def causal(s, window=0):
    key = [torch.arange(l) for l in s.lens]
    return lambda row, i, pos, h: (key[i] <= pos) & (key[i] > pos - (window or 1 << 30))


def padded(x, rows, value=math.nan):
    """The rows of x, and more behind them that belong to no token."""
    return torch.cat([x, torch.full((rows - x.shape[0], *x.shape[1:]), value, dtype=x.dtype)]).cuda()


def attend(cache, batch, q, scale, window=0):
    """(out, lse) over outputs that hold NaN."""
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
    B.pk_kv_attend(cache.handle, batch.c, q, scale, window, out, lse)
    return out, lse


# ------------------------------------------------------------------------------- host numbers are bounds

@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("P,D", [(64, 128), (16, 64)])
@pytest.mark.parametrize("news", [[0], [1], [10], [16], [33], [5, 256], [0, 3], [17, 64], [1, 0, 200]], ids=str)
def test_fewer_tokens_than_the_host_says(gpu_device, storage, dtype, P, D, news):
    """n_tokens = n_seqs * max_new on the host, sequences of fewer on the device: each of a batch's rows is written, and no other."""
    s = Setup(storage, dtype, 2, 4, D, P, news, [n + 70 for n in news], seed=31)
    n = 256 * len(news)
    batch = B.KVBatch(s.batch.tables, s.batch.offsets, s.batch.lens, n, 256, max(s.lens) + 300)
    for window in (0, 40):
        out, lse = attend(s.cache, batch, padded(s.q, n), D ** -0.5, window)
        s.check(out, lse.cpu(), D ** -0.5, causal(s, window))
        assert torch.all(out[sum(news):].isnan()) and torch.all(lse[sum(news):].isnan())


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16")])
def test_chunks_in_a_graph_follow_the_arrays(gpu_device, storage, dtype):
    """Chunks captured once, replayed with other offsets and lengths, against 64 bits each time."""
    s = Setup(storage, dtype, 2, 4, 64, 32, [128, 128], [400, 300], seed=32)
    offsets, lens = s.batch.offsets.clone(), s.batch.lens.clone()
    batch = B.KVBatch(s.batch.tables, offsets, lens, 256, 128, 400)
    q = s.q.cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")
    B.pk_kv_attend(s.cache.handle, batch.c, q, 0.125, 0, out, lse)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.pk_kv_attend(s.cache.handle, batch.c, q, 0.125, 0, out, lse)
    full = s.q
    for news, ends in (([128, 128], [400, 300]), ([5, 3], [333, 90]), ([0, 128], [50, 299]), ([128, 1], [128, 300]), ([40, 16], [397, 16])):
        s.news, s.lens, s.q = news, ends, full[:sum(news)]
        offsets.copy_(torch.tensor([0, news[0], sum(news)], dtype=torch.int32))
        lens.copy_(torch.tensor(ends, dtype=torch.int32))
        out.fill_(math.nan)
        lse.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        s.check(out, lse.cpu(), 0.125, causal(s))
        assert torch.all(out[sum(news):].isnan()) and torch.all(lse[sum(news):].isnan())


# ------------------------------------------------------------------------------- rows of no token

@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16")])
@pytest.mark.parametrize("H,G,news,length,n,max_new", [
    (2, 4, [3, 1], 300, 4, 3),           # one part
    (2, 4, [1, 1, 1], 4200, 64, 1),      # parts, joined by the last workgroup
    (8, 2, [1] * 40, 4200, 64, 1),       # parts, joined by a launch
    (1, 20, [6, 2], 500, 5, 4),          # the host's max_new is less than what a sequence has: its last rows are left out
], ids=str)
def test_rows_of_no_token_are_left(gpu_device, storage, dtype, H, G, news, length, n, max_new):
    s = Setup(storage, dtype, H, G, 64, 64, news, [length + i for i in range(len(news))], seed=33)
    total = sum(news) + 5
    batch = B.KVBatch(s.batch.tables, s.batch.offsets, s.batch.lens, total, max_new, max(s.lens))
    mine = torch.zeros(total, dtype=torch.bool)
    at = 0
    for m in news:
        mine[at:at + min(m, max_new)] = True
        at += m
    q = padded(s.q, total)

    def check(what, fill, filled, call):
        got = [torch.full(shape, fill, dtype=kind, device="cuda") for shape, kind in filled]
        call(*got)
        for x in got:
            x = x.cpu()
            left = x[~mine].isnan() if fill != fill else x[~mine] == fill
            held = x[mine].isnan() if fill != fill else x[mine] == fill
            assert bool(left.all()), what
            assert not bool(held.any()), what
        return got
    outputs = [((total, H * G, 64), s.kind), ((total, H * G), torch.float32)]
    blocks, = check("select", -77, [((total, H, n), torch.int32)], lambda b: B.pk_kv_select(s.cache.handle, batch.c, q, n, 1, 2, b))
    check("attend", math.nan, outputs, lambda out, lse: B.pk_kv_attend(s.cache.handle, batch.c, q, 0.1, 0, out, lse))
    for listed in (blocks.clamp(min=-1), torch.zeros_like(blocks)):  # (zeros: the rows of no token list a block that there is; so do others, n times)
        check("attend_blocks", math.nan, outputs, lambda out, lse: B.pk_kv_attend_blocks(s.cache.handle, batch.c, q, 0.1, listed, out, lse))
    rows = [((total, H, 64), torch.float32)] * 2
    check("read", math.nan, rows, lambda k, v: B.pk_kv_read(s.cache.handle, batch.c, k, v))


# ------------------------------------------------------------------------------- ends of 32 bits

# Keys whose channels are all `kc` but the last, and queries of `qc`: every product and every sum of them is a whole number below 2^24 (times the
# codes' scale, which is 1), so that scores are exact whatever their order, and differ by the last channel times the scale.
LARGE = {"f16": (1200, 64), "bf16": (1200, 64), "i8": (127, 500), "f8": (448, 256)}


@pytest.mark.parametrize("storage,dtype", CODES)
@pytest.mark.parametrize("news,length", [([1], 90), ([1], 2100), ([150], 700)], ids=str)
@pytest.mark.parametrize("scale", [0.37, 2.3, 3.7, 47.0, -3.7])
def test_scores_beyond_24_bits(gpu_device, storage, dtype, news, length, scale):
    """Finite scores of any size: exact differences between them, some of 10^6 to 10^9, give the weights that they stand for.

    e, the relative error of a weight: 2^-20 for the exponential and the sums, and the differences' rounding (of the scale, and of their product
    with it): 2^-22 of the largest that has any weight (e^-30 is none)."""
    kc, qc = LARGE[storage]
    s = Setup(storage, dtype, 1, 2, 128, 64, news, [length], seed=34)
    step = torch.arange(length) * 5 // length  # (the maximum grows late: sums so far are rescaled)
    s.k[0][:] = kc
    s.k[0][:, 0, 127] = (4 - step if scale < 0 else step).to(s.kind)
    s.q[:] = qc
    s.q[:, :, 127] = 1
    s.write(s.lens, (s.k, s.v))
    k, v = (x[0].double() for x in s.stored())
    assert torch.equal(k, s.k[0].double())
    out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
    out, lse = out.cpu().double(), lse.cpu()
    u_out, u_w = U[s.kind], 2 * U[torch.float16] if storage in ("i8", "f8") else U[s.kind]
    e = 2.0 ** -20 + 2.0 ** -22 * min(30.0, 4 * abs(scale))
    for row, _, pos in s.tokens():
        for g in range(2):
            x = (k[:pos + 1, 0] @ s.q[row, g].double()) * scale
            w = torch.softmax(x, 0)
            ref, a = w @ v[:pos + 1, 0], w @ v[:pos + 1, 0].abs()
            assert torch.all((out[row, g] - ref).abs() <= u_out * ref.abs() + (u_w + e) * (1 + u_out) * a + 2.0 ** -24), (row, g)
            full = float(torch.logsumexp(x, 0))
            assert abs(float(lse[row, g]) - full) <= e + 2.0 ** -20 * abs(full), (row, g)


@pytest.mark.parametrize("storage", ["i8", "f8"])
def test_a_long_sum_in_one_part_keeps_its_size(gpu_device, storage):
    """2^20 keys of equal weight whose values are equal: the sum of weights that are 2^15 exactly times codes that are whole numbers needs no
    rounding, so a result is the value itself: its own rounding, and 2^-20 for the scales and the division.  Heads differ in their values' scale."""
    H, G, D, P, n, m, seqs = 64, 4, 64, 128, 1 << 20, 64, 8
    cache = B.KVCache(1, H, D, storage=STORAGES[storage], page_tokens=P)
    gen = torch.Generator().manual_seed(35)
    one = torch.full((D,), 64.0)
    one[0] = 127.0 if storage == "i8" else 448.0
    v = (one * (torch.rand(H, 1, generator=gen) + 0.1) * 0.01).expand(P, H, D)
    # every page of every sequence is the one page that there is
    def batch(m, length, seqs):
        tables = torch.zeros((seqs, length // P), dtype=torch.int32, device="cuda")
        offsets = torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * m
        return B.KVBatch(tables, offsets, torch.full((seqs,), length, dtype=torch.int32, device="cuda"), seqs * m, m, length)
    one_page = batch(P, P, 1)
    cache.append(torch.zeros(P, H, D, device="cuda"), v.contiguous().cuda(), one_page)
    held = cache.read(one_page, torch.float32)[1][0].cpu().double()  # [head, channel]
    q = torch.zeros(seqs * m, H * G, D, dtype=torch.float16, device="cuda")
    out, lse = cache.attend(q, batch(m, n, seqs), 0.125, want_lse=True)
    off = (out.cpu().double().view(-1, H, G, D) - held[:, None]).abs() / held[:, None]
    assert float(off.max()) <= 2.0 ** -11 + 2.0 ** -20
    pos = n - m + torch.arange(m).repeat(seqs)
    assert torch.allclose(lse.cpu().double(), torch.log(pos + 1.0).double()[:, None].expand(-1, H * G), rtol=2.0 ** -20, atol=0)


def test_windows_as_long_as_32_bits_have(gpu_device):
    """The longest window is none, also where a sequence has more new tokens than it holds (positions before the first are left out)."""
    for news, lens in (([40, 3], [100, 90]), ([24, 200], [20, 150])):
        s = Setup("bf16", "bf16", 1, 4, 64, 16, news, [max(n, l) for n, l in zip(news, lens)], seed=36)
        batch = B.KVBatch(s.batch.tables, s.batch.offsets, torch.tensor(lens, dtype=torch.int32, device="cuda"), sum(news), max(news), max(lens))
        want, got = (attend(s.cache, batch, s.q.cuda(), 0.1, window) for window in (0, 2 ** 31 - 1))
        for a, b in zip(want, got):
            assert not bool(a.isnan().any()) and torch.equal(a, b)


# ------------------------------------------------------------------------------- choices

def chosen(s, n, sink, local):
    """The choice by its definition, from the rows that were written, in the 32 bits that it is stated in: nothing is read back."""
    want = torch.full((sum(s.news), s.H, n), -1, dtype=torch.int32)
    x = s.q.float()
    top = x.abs().amax(-1, keepdim=True)
    up = torch.where(top > 0, torch.full_like(top, 127.0) / top, torch.zeros_like(top))
    code, qs = (x * up).round().clamp(-127, 127).double(), (top * torch.tensor(1.0 / 127.0))[..., 0]
    bounds = []
    for i, l in enumerate(s.lens):
        held = definition(s.k[i], s.storage, s.kind)
        bounds.append([bounds_of(held[j:j + s.P]) for j in range(0, l, s.P)])
    for row, i, pos in s.tokens():
        mine = pos // s.P
        for h in range(s.H):
            hi, lo, scale = (torch.stack([b[j][h] for b in bounds[i][:mine + 1]]) for j in range(3))
            c = code[row, h * s.G:(h + 1) * s.G]
            u = c.clamp(min=0) @ hi.double().T + c.clamp(max=0) @ lo.double().T
            score = (u.float() * qs[row, h * s.G:(h + 1) * s.G, None]).amax(0) * scale[:, 0]
            score[:sink] = math.inf
            score[max(mine + 1 - local, 0):] = math.inf
            take = torch.sort(score, descending=True, stable=True).indices[:n].sort().values
            want[row, h, :len(take)] = take.int()
    return want


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16")])
@pytest.mark.parametrize("H,G,news,lens,n", [
    (8, 2, [1] * 20, [3000 + 7 * i for i in range(20)], 12),
    (2, 1, [33], [5000], 40),
    (1, 3, [9, 2], [8000, 70], 3),
    (2, 4, [37, 1, 0, 1, 1, 1, 6, 1], [1200, 900, 5, 1, 333, 17, 640, 1024], 7),  # few of the tokens' places for so many sequences are taken
    (1, 20, [1, 1, 1, 11], [900, 1, 30, 500], 6),
    (1, 2, [1] * 90 + [45] + [0, 2] * 30, [40 + i for i in range(90)] + [300] + [3, 170] * 30, 4),
], ids=str)
def test_every_choice_is_exact(gpu_device, storage, dtype, H, G, news, lens, n):
    s = Setup(storage, dtype, H, G, 64, 16, news, lens, seed=37, spread=0.2)
    assert torch.equal(s.cache.select(s.q.cuda(), s.batch, n).cpu(), chosen(s, n, 1, 2))


def test_a_chunk_among_many_sequences(gpu_device):
    """64 sequences of 8 heads, one with a chunk of 32769 tokens: the same choices as of each sequence by itself."""
    H, P, D, n = 8, 128, 8, 3
    lens = [32769 + 200] + [1 + 37 * i for i in range(63)]
    news = [32769] + [1] * 63
    pages = [-(-l // P) for l in lens]
    cache = B.KVCache(sum(pages), H, D, storage=B.PK_F16, page_tokens=P)
    gen = torch.Generator("cuda").manual_seed(38)
    tables = torch.zeros((64, max(pages)), dtype=torch.int32)
    at = 0
    for i, p in enumerate(pages):
        tables[i, :p] = torch.arange(at, at + p, dtype=torch.int32)
        at += p
    tables = tables.cuda()

    def batch(which, m):
        offsets = torch.tensor([0] + [m[i] for i in which]).cumsum(0).int().cuda()
        t = tables[which[0]:which[-1] + 1]
        return B.KVBatch(t, offsets, torch.tensor([lens[i] for i in which], dtype=torch.int32, device="cuda"), sum(m[i] for i in which), max(m[i] for i in which),
                         max(lens[i] for i in which))
    for i in range(64):
        rows = torch.randn(lens[i], H, D, generator=gen, device="cuda").half()
        cache.append(rows, rows, batch([i], lens))
    q = torch.randn(sum(news), H, D, generator=gen, device="cuda").half()
    got = cache.select(q, batch(list(range(64)), news), n)
    at = 0
    for i in range(64):
        assert torch.equal(got[at:at + news[i]], cache.select(q[at:at + news[i]], batch([i], news), n)), i
        at += news[i]
    cache.close()


def test_bounds_of_more_pages_than_a_launch_has_workgroups(gpu_device):
    """2^24 and a few, of three pages and of numbers that there are no pages for: each as it is by itself."""
    s = Setup("i8", "bf16", 1, 1, 8, 16, [40], [40], seed=39)
    few = torch.tensor(s.tables[0].tolist() + [-1, 10 ** 9], dtype=torch.int32, device="cuda")
    want = s.cache.bounds(few)
    n = 2 ** 24 + 5
    which = torch.randint(0, 5, (n,), generator=torch.Generator("cuda").manual_seed(39), device="cuda")
    for got, x in zip(s.cache.bounds(few[which]), want):
        assert torch.equal(got, x[which])


def test_many_tokens_and_heads(gpu_device):
    """600 000 tokens of 8 heads that attend to a block each: as each part of them by itself."""
    H, D, P, n = 8, 8, 16, 600_000
    cache = B.KVCache(64, H, D, storage=B.PK_F16, page_tokens=P)
    gen = torch.Generator("cuda").manual_seed(40)
    tables = torch.arange(64, dtype=torch.int32, device="cuda").repeat(n // 64 // P + 1)[None]
    one = B.KVBatch(tables, torch.tensor([0, 1024], dtype=torch.int32, device="cuda"), torch.tensor([1024], dtype=torch.int32, device="cuda"), 1024, 1024, 1024)
    rows = torch.randn(1024, H, D, generator=gen, device="cuda").half()
    cache.append(rows, rows, one)
    q = torch.randn(n, H, D, generator=gen, device="cuda").half()
    blocks = (torch.arange(n, device="cuda", dtype=torch.int32) // P)[:, None, None].expand(n, H, 1).contiguous()

    def batch(length, m):
        return B.KVBatch(tables, torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda"), m, m, length)
    out = cache.attend_blocks(q, blocks, batch(n, n), 0.3)
    for at in (0, 299_000, n - 1000):
        assert torch.equal(out[at:at + 1000], cache.attend_blocks(q[at:at + 1000], blocks[at:at + 1000], batch(at + 1000, 1000), 0.3))
    cache.close()


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16")])
def test_a_step_in_a_graph_follows_offsets(gpu_device, storage, dtype):
    """Append, selection and attention to it, captured once for up to 64 tokens of four sequences (no more than 40 of one), replayed with other
    offsets and lengths: the cache's rows, the choices and the results are what they are by their definitions, each time."""
    s = Setup(storage, dtype, 2, 2, 64, 16, [16] * 4, [400, 330, 90, 500], seed=41)
    H, D, n = s.H, s.D, 5
    offsets, lens = s.batch.offsets.clone(), s.batch.lens.clone()
    batch = B.KVBatch(s.batch.tables, offsets, lens, 64, 40, 500)
    whole, keys, values = s.q, s.k, s.v
    q, k, v = s.q.cuda(), *(torch.zeros(64, H, D, dtype=s.kind, device="cuda") for _ in range(2))
    blocks, out = torch.empty(64, H, n, dtype=torch.int32, device="cuda"), torch.empty_like(q)

    def step():
        B.pk_kv_append(s.cache.handle, batch.c, k, v)
        B.pk_kv_select(s.cache.handle, batch.c, q, n, 1, 2, blocks)
        B.pk_kv_attend_blocks(s.cache.handle, batch.c, q, 0.125, blocks, out)
    step()
    s.cache.arena.fill_(0xff)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    have = [0, 0, 0, 0]
    for news in ([16] * 4, [40, 0, 1, 23], [1, 40, 0, 3], [0, 1, 33, 30], [5] * 4, [1] * 4, [0, 0, 0, 40]):
        s.news, s.lens = news, [a + m for a, m in zip(have, news)]
        rows = sum(news)
        s.q, s.k, s.v = whole[:rows], [x[:l] for x, l in zip(keys, s.lens)], [x[:l] for x, l in zip(values, s.lens)]
        offsets.copy_(torch.tensor([0] + news).cumsum(0).int())
        lens.copy_(torch.tensor(s.lens, dtype=torch.int32))
        k[:rows] = torch.cat([x[a:] for x, a in zip(s.k, have)]).cuda()
        v[:rows] = torch.cat([x[a:] for x, a in zip(s.v, have)]).cuda()
        k[rows:], v[rows:] = math.nan, math.nan
        blocks.fill_(-77)
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        for got, x in zip(s.cache.read(s.make_batch(s.lens, s.lens), torch.float32), (s.k, s.v)):
            assert torch.equal(got.cpu(), definition(torch.cat(x), storage, s.kind))
        assert torch.equal(blocks[:rows].cpu(), chosen(s, n, 1, 2))
        assert torch.all(blocks[rows:] == -77) and torch.all(out[rows:].isnan())
        b = blocks.cpu()
        key = [torch.arange(l) for l in s.lens]
        s.check(out, None, 0.125, lambda row, i, pos, h: (key[i] <= pos) & torch.isin(key[i] // 16, b[row, h][b[row, h] >= 0]))
        have = s.lens
