"""The key/value cache in 4 bits against its definition and plain forms in 64 bits.

What the cache holds is compared bit for bit; attention takes the stored values from `read`, with the tolerances of test_gpu_kv: a weight,
the values' scale in it, is rounded once to the queries' type.  Of 4 bits many are zeros, so that a channel may be made by keys of hardly any
weight alone: a weight below 2^-126 of the largest is none (the smallest normal number of 32 bits: exponentials, and the factors that
sums so far are rescaled by, are cut off there), which is 2^-126 sum|v| of a result at most.  Half precision rounds weights (the largest is 2^15)
to steps of 2^-24 at least: 2^-40 of the largest times the largest scale, 2^-40 sum max|v| in all."""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B
import test_gpu_kv as base
from test_gpu_kv import PARTS, SHAPES, U, bounds_of, choose

pytestmark = pytest.mark.gpu
base.STORAGES.setdefault("f4", B.PK_F4)

TYPES = ["bf16", "f16"]
VALUES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


class Setup(base.Setup):
    def check(self, out, lse, scale, seen):
        ks, vs = self.stored()
        u, out, q = U[self.kind], out.cpu().double(), self.q.double()
        for row, i, pos in self.tokens():
            for h in range(self.H):
                mask = seen(row, i, pos, h)
                k, v = ks[i][mask, h], vs[i][mask, h]
                rows = slice(h * self.G, (h + 1) * self.G)
                where = f"row {row} sequence {i} position {pos} head {h}"
                if k.shape[0] == 0:
                    assert torch.all(out[row, rows] == 0), where
                    assert lse is None or torch.all(lse[row, rows] == -math.inf), where
                    continue
                x = (q[row, rows] @ k.T) * scale
                w = torch.softmax(x, 1)
                size = ((q[row, rows].abs() @ k.abs().T) * abs(scale)).amax(1, keepdim=True)
                e = 2 * (self.D + 8) * 2.0 ** -24 * size + 2.0 ** -20
                ref, a = w @ v, w @ v.abs()
                cut = 2.0 ** -126 * v.abs().sum(0) + (2.0 ** -40 * v.shape[0] * v.abs().max() + 2.0 ** -24 if self.kind == torch.float16 else 2.0 ** -126)
                bound = u * ref.abs() + (u + e) * (1 + u) * a + cut
                off = (out[row, rows] - ref).abs()
                assert torch.all(off <= bound), f"{where}: {float((off / bound).max())} of the bound"
                if lse is not None:
                    full = torch.logsumexp(x, 1)
                    assert torch.all((lse[row, rows].double() - full).abs() <= e[:, 0] / 2 + 2.0 ** -20 * full.abs()), where


def nearest(y):
    """e2m1: the nearest value, the one with an even code where two are as near; 6 beyond."""
    a = y.abs().clamp(max=6.0)
    off = (a[..., None] - VALUES).abs()
    least = off.amin(-1, keepdim=True)
    code = torch.where(off == least, torch.arange(8), 99)
    low = code.amin(-1)
    even = torch.where((code < 99) & (code % 2 == 0), code, 99).amin(-1)
    tie = (code < 99).sum(-1) > 1
    return torch.copysign(VALUES[torch.where(tie, even, low)], y)


def definition(x, key):
    x = x.float()
    most = x.abs().amax(-1, keepdim=True)
    up = torch.where(most > 0, torch.full_like(most, 6.0) / most, torch.zeros_like(most))  # (a number over a tensor would be two roundings)
    power = torch.ones_like(x)
    if key:
        for at in range(0, x.shape[-1], 32):
            part = x[..., at:at + 32].abs().amax(-1, keepdim=True)
            (fm, em), (fp, ep) = torch.frexp(most), torch.frexp(part)
            e = torch.where(part > 0, (em - ep - (fp > fm).int()).clamp(0, 15), torch.full_like(em, 15))
            power[..., at:at + 32] = torch.exp2(e.float())
    return nearest((x * power) * up) / power * (most * torch.tensor(1.0 / 6.0, dtype=torch.float32))


def causal(s, window=0):
    key = [torch.arange(l) for l in s.lens]
    return lambda row, i, pos, h: (key[i] <= pos) & (key[i] > pos - (window or 1 << 30))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("H,D,P,lens", [(2, 64, 16, [1, 16, 17, 45]), (3, 80, 64, [0, 63, 64, 130]), (1, 128, 32, [33, 1]), (2, 256, 128, [257]), (1, 8, 64, [70]), (2, 104, 16, [31, 15])])
def test_what_is_written_is_what_the_definition_says(gpu_device, dtype, H, D, P, lens):
    s = Setup("f4", dtype, H, 1, D, P, lens, lens, seed=1)
    for x in (s.k, s.v):
        for i, l in enumerate(lens):
            if l > 12:
                x[i][3] = 0  # a row of zeros
                x[i][2] = (x[i][2].float() * 1e-6).to(s.kind)
                x[i][4, :, :D // 2] = 0  # groups of zeros
                x[i][5, :, :D // 2] = (x[i][5, :, :D // 2].float() * 2.0 ** -9).to(s.kind)  # and small ones
                x[i][6, :, 1:] = (x[i][6, :, 1:].float() * 2.0 ** -20).to(s.kind)
                # numbers in the middle of two codes, of both signs
                x[i][7] = ((torch.arange(D) % 14 - 7) * 0.25).to(s.kind)
                x[i][7, :, 0] = 6.0
                x[i][8] = -x[i][7]
                x[i][9] = (torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -6.0]).repeat(D // 8) * 2.0 ** -3).to(s.kind)
                x[i][10, :] = 1.0
                x[i][11, :] = -0.0
    s.write(lens, (s.k, s.v))
    for want in (torch.float32, torch.float16, torch.bfloat16):
        for got, rows, key in zip(s.cache.read(s.batch, want), (s.k, s.v), (True, False)):
            assert torch.equal(got.cpu(), definition(torch.cat(rows), key).to(want))
    pages = s.tables[s.tables >= 0]
    hi, lo = s.cache.bounds(pages.cuda())
    at = 0
    for i, l in enumerate(lens):
        held = definition(s.k[i], True)
        for j in range(-(-l // P)):
            h, w, scale = bounds_of(held[j * P:(j + 1) * P])
            assert torch.equal(hi[at].cpu(), h * scale) and torch.equal(lo[at].cpu(), w * scale), (i, j)
            at += 1


@pytest.mark.parametrize("dtype,D,P", [("bf16", 64, 16), ("f16", 128, 64), ("f32", 96, 32), ("f16", 256, 128)])
def test_pages_do_not_depend_on_how_their_tokens_came(gpu_device, dtype, D, P):
    """Chunks that begin and end inside pages and inside bytes, single tokens, and rows written again."""
    lens = [3 * P + 5, P, 7]
    whole = Setup("f4", dtype, 2, 1, D, P, lens, lens, seed=2)
    parts = Setup("f4", dtype, 2, 1, D, P, lens, lens, seed=2)
    parts.cache.arena.fill_(0xff)
    have = [0, 0, 0]
    for step in (1, 5, P, 1, 2 * P, 3):
        news = [min(step, l - n) for n, l in zip(have, lens)]
        parts.write(news, [[x[i][n:n + m] for i, (n, m) in enumerate(zip(have, news))] for x in (parts.k, parts.v)], lens=[n + m for n, m in zip(have, news)])
        have = [n + m for n, m in zip(have, news)]
    parts.write([3, 1, 0], [[x[0][8:11], x[1][P - 2:P - 1], x[2][:0]] for x in (parts.k, parts.v)], lens=[11, P - 1, 7])  # tokens in the middle, again
    parts.write([P - 3, 1, 1], [[x[0][P:2 * P - 3], x[1][P - 1:], x[2][6:]] for x in (parts.k, parts.v)], lens=[2 * P - 3, P, 7])
    assert have == lens
    for a, b in zip(whole.cache.read(whole.batch, torch.float32), parts.cache.read(parts.batch, torch.float32)):
        assert torch.equal(a, b)
    parts.write([1, 1, 1], [[x[i][-1:] for i in range(3)] for x in (parts.k, parts.v)])
    last = torch.tensor([whole.tables[i, (l - 1) // P] for i, l in enumerate(lens)], dtype=torch.int32).cuda()
    for a, b in zip(whole.cache.bounds(last), parts.cache.bounds(last)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("window", [0, 50])
def test_attention(gpu_device, dtype, shape, window):
    H, G, D, P, news, lens = shape
    s = Setup("f4", dtype, H, G, D, P, news, lens, seed=3, tail=2)
    out, lse = s.cache.attend(s.q.cuda(), s.batch, D ** -0.5, window=window, want_lse=True)
    s.check(out, lse.cpu(), D ** -0.5, causal(s, window))
    assert torch.equal(s.cache.attend(s.q.cuda(), s.batch, D ** -0.5, window=window), out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("shape", PARTS, ids=lambda s: f"{s[:4]} {len(s[4])} of {max(s[4])} at {max(s[5])}")
def test_attention_in_parts(gpu_device, dtype, shape):
    H, G, D, P, news, lens = shape
    s = Setup("f4", dtype, H, G, D, P, news, lens, seed=16)
    out, lse = s.cache.attend(s.q.cuda(), s.batch, D ** -0.5, want_lse=True)
    s.check(out, lse.cpu(), D ** -0.5, causal(s))
    for _ in range(3):
        assert torch.equal(s.cache.attend(s.q.cuda(), s.batch, D ** -0.5), out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("P,D", [(16, 128), (64, 128), (16, 64), (64, 256), (32, 256), (128, 64)])
@pytest.mark.parametrize("news", [[32, 33, 64, 65, 1], [129, 0, 128], [300]], ids=str)
def test_either_side_of_few_rows(gpu_device, dtype, P, D, news):
    s = Setup("f4", dtype, 1, 2, D, P, news, [n + 150 for n in news], seed=21)
    out, lse = s.cache.attend(s.q.cuda(), s.batch, D ** -0.5, want_lse=True)
    s.check(out, lse.cpu(), D ** -0.5, causal(s))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [-0.07, 0.0, 3.0])
def test_scales_of_any_sign(gpu_device, dtype, scale):
    for news in ([2, 1], [90, 1]):
        s = Setup("f4", dtype, 1, 2, 64, 32, news, [130, 40], seed=17, spread=0.3)
        out, lse = s.cache.attend(s.q.cuda(), s.batch, scale, want_lse=True)
        s.check(out, lse.cpu(), scale, causal(s))


@pytest.mark.parametrize("dtype", TYPES)
def test_attention_without_some_pages(gpu_device, dtype):
    s = Setup("f4", dtype, 2, 3, 64, 16, [5, 1, 20, 33], [70, 17, 20, 90], seed=4, missing=[(0, 0), (0, 2), (1, 0), (1, 1), (2, 0), (3, 5), (3, 4), (3, 3)])
    key = [torch.arange(l) for l in s.lens]
    out, lse = s.cache.attend(s.q.cuda(), s.batch, 0.125, want_lse=True)
    s.check(out, lse.cpu(), 0.125, lambda row, i, pos, h: (key[i] <= pos) & s.there(i))
    for x in s.cache.read(s.make_batch(s.lens, s.lens), torch.float32):
        for rows, i in zip(torch.split(x.cpu(), s.lens), range(4)):
            assert torch.all(rows[~s.there(i)] == 0) and not bool(rows.isnan().any())


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_any_size(gpu_device, dtype):
    """Tokens, and groups of a key's channels, that differ in size by many powers of two; values near the ends of bfloat16."""
    s = Setup("f4", dtype, 2, 2, 128, 64, [3, 1], [200, 75], seed=5, spread=2.5)
    s.k = [(x.float() * torch.exp2(-4.0 * (torch.arange(128) // 32 % 3))).to(s.kind) for x in s.k]
    s.write(s.lens, (s.k, s.v))
    out, lse = s.cache.attend(s.q.cuda(), s.batch, 0.5, want_lse=True)
    s.check(out, lse.cpu(), 0.5, causal(s))
    if dtype == "bf16":
        for size in (1e-30, 1e30):
            s.v = [(x.float() * size).to(s.kind) for x in s.v]
            s.write(s.lens, (s.k, s.v))
            s.check(s.cache.attend(s.q.cuda(), s.batch, 0.125), None, 0.125, causal(s))
            s.v = [(x.float() / size).to(s.kind) for x in s.v]


@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(gpu_device, dtype):
    s = Setup("f4", dtype, 2, 2, 80, 32, [9, 4], [50, 71], seed=7)
    n = sum(s.lens)
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
    s.check(out, None, 0.1, causal(s))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("H,G,D,P,news,lens,n,sink,local", [
    (2, 4, 128, 64, [1, 1], [1, 1500], 8, 1, 2),
    (1, 1, 64, 16, [5, 0, 3], [700, 0, 3], 6, 1, 2),
    (2, 5, 80, 32, [40], [900], 5, 0, 1),
    (1, 16, 256, 16, [2], [4500], 64, 3, 4),
    (1, 20, 64, 16, [1], [300], 3, 1, 2),
    (5, 3, 128, 128, [1, 7], [2000, 700], 5, 1, 2),
])
def test_selection_and_attention_to_it(gpu_device, dtype, H, G, D, P, news, lens, n, sink, local):
    missing = [(0, 3)] if lens[0] > 5 * P else []
    s = Setup("f4", dtype, H, G, D, P, news, lens, seed=8, missing=missing)
    blocks = s.cache.select(s.q.cuda(), s.batch, n, sink=sink, local=local)
    want, margin = choose(s, n, sink, local)
    same = (blocks.cpu() == want).all(-1)
    assert bool(same.all()) or margin < 2.0 ** -20  # (the bounds' scale is read back with a rounding)
    mixed = blocks[..., torch.randperm(n, generator=s.gen).cuda()].contiguous()  # in any order
    out, lse = s.cache.attend_blocks(s.q.cuda(), mixed, s.batch, D ** -0.5, want_lse=True)
    b = blocks.cpu()

    def seen(row, i, pos, h):
        key = torch.arange(lens[i])
        return (key <= pos) & torch.isin(key // P, b[row, h][b[row, h] >= 0]) & s.there(i)
    s.check(out, lse.cpu(), D ** -0.5, seen)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("news", [[10], [33], [0, 3], [17, 64]], ids=str)
def test_fewer_tokens_than_the_host_says(gpu_device, dtype, news):
    s = Setup("f4", dtype, 2, 4, 128, 64, news, [n + 70 for n in news], seed=31)
    n = 256 * len(news)
    batch = B.KVBatch(s.batch.tables, s.batch.offsets, s.batch.lens, n, 256, max(s.lens) + 300)
    q = torch.cat([s.q, torch.full((n - sum(news), 8, 128), math.nan, dtype=s.kind)]).cuda()
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
    B.pk_kv_attend(s.cache.handle, batch.c, q, 0.1, 0, out, lse)
    s.check(out, lse.cpu(), 0.1, causal(s))
    assert torch.all(out[sum(news):].isnan()) and torch.all(lse[sum(news):].isnan())


@pytest.mark.parametrize("dtype", TYPES)
def test_a_long_sum_in_one_part_keeps_its_size(gpu_device, dtype):
    """2^18 keys of equal weight with equal values, 6 of them the largest: only roundings of the result remain (the weights, all alike, are rounded
    alike in numerator and, unrounded, in the denominator: half a step)."""
    D, P, n = 64, 128, 1 << 18
    cache = B.KVCache(1, 1, D, storage=B.PK_F4, page_tokens=P)
    v = torch.full((P, 1, D), 3.0) * 0.0123
    tables = torch.zeros((1, n // P), dtype=torch.int32, device="cuda")

    def batch(m, length):
        return B.KVBatch(tables, torch.tensor([0, m], dtype=torch.int32, device="cuda"), torch.tensor([length], dtype=torch.int32, device="cuda"), m, m, length)
    cache.append(torch.zeros(P, 1, D, device="cuda"), v.cuda(), batch(P, P))
    held = cache.read(batch(P, P), torch.float32)[1][0, 0, 0].item()
    q = torch.zeros(300, 1, D, dtype=base.TYPES[dtype], device="cuda")
    out, lse = cache.attend(q, batch(300, n), 0.125, want_lse=True)
    assert float((out.double() - held).abs().max()) <= held * (2 * base.U[base.TYPES[dtype]] + 2.0 ** -18)
    pos = n - 300 + torch.arange(300)
    assert torch.allclose(lse.cpu().double()[:, 0], torch.log(pos + 1.0).double(), rtol=2.0 ** -20, atol=0)


def test_calls_in_a_graph_follow_the_arrays(gpu_device):
    P, lens = 16, [40, 101]
    s = Setup("f4", "bf16", 2, 4, 64, P, [1, 1], [l + 8 for l in lens], seed=12)
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
        graph.replay()
        torch.cuda.synchronize()
        kept = [x.clone() for x in got]
        for a, b in zip(kept, step()):
            assert torch.equal(a, b), j


def test_refusals(gpu_device):
    s = Setup("f4", "bf16", 2, 2, 64, 16, [2], [20], seed=15)
    for bad in (s.q.cuda().float(), s.q.cuda()[:, :3]):
        with pytest.raises(B.PancakeError) as e:
            s.cache.attend(bad, s.batch, 0.1)
        assert e.value.status == (B.PK_ERR_UNSUPPORTED if bad.dtype == torch.float32 else B.PK_ERR_INVALID_ARG)
