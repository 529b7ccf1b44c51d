"""Attention with capped or biased scores and with masks of documents and a prefix, against plain forms in 64 bits.

Tolerances are those of test_gpu_kv, with e, the relative error of a weight, from these errors of a score (twice their sum, a score's and the largest
one's, and 2^-20 for the exponential, the sums and the scale):
  (D + 8) 2^-24 sum|q k| scale   the product
  2^-21 min(cap, 2 largest |x|)  the cap: where a score x is beyond cap / 2, tanh = 1 - 2 / (1 + e^2z), in which the quotient is
                                 off by 2^-23, the sum below it by 2^-24 and the power by 2^-21 of itself (at z < 3, later it is none of
                                 the result's): 2 (2^-23 + 2^-24) / (1 + e) + 2^-21 / 2 of the cap, less than 2^-21; else a polynomial, off by
                                 2^-26 and six roundings, 2^-21 of the score
  2^-22 slope distance           the bias: its factor, its product and the distance are rounded
  2^-23 |score|                  their sum is rounded, and so is the largest
lse, of int8 under bfloat16: also 2^-17 ln 2.  Weights are 2^(x + 127 - m) there, up to 2^127, and 127 - m, between 128 and 256 where m is a little below 0, is rounded
to 2^-17: the same factor for all weights of a sum, which cancels in a result and is left in the logarithm.  (Found by a row of equal scores.)
and, for weights that are cut off, 2^-126 sum|v|, in half precision (steps of 2^-24 below 2^15) 2^-40 sum max|v| and 2^-24."""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B
import test_gpu_kv as base
from test_gpu_kv import U

pytestmark = pytest.mark.gpu
base.STORAGES.setdefault("f4", B.PK_F4)

CODES = [("f16", "f16"), ("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f8", "bf16"), ("f8", "f16"), ("f4", "bf16"), ("f4", "f16")]


class Setup(base.Setup):
    def how(self, cap=0.0, slopes=None, docs=0, prefix=None):
        """docs: the documents' length; they begin behind the prefix.  A token of none (in the prefix) has a document of its own."""
        h = {"cap": cap}
        if slopes is not None:
            h["slopes"] = torch.tensor([slopes * 2.0 ** -(i % 5) for i in range(self.H * self.G)])
        if prefix is not None:
            h["prefix"] = torch.tensor([prefix[i % len(prefix)] for i in range(len(self.lens))], dtype=torch.int32)
        if docs:
            first = [int(h["prefix"][i]) if prefix is not None else 0 for i in range(len(self.lens))]
            h["starts"] = torch.tensor([first[i] + (pos - first[i]) // docs * docs if pos >= first[i] else pos for _, i, pos in self.tokens()], dtype=torch.int32)
        return h

    def run(self, scale, how, window=0):
        on = {x: y.cuda() if torch.is_tensor(y) else y for x, y in how.items()}
        return self.cache.attend(self.q.cuda(), self.batch, scale, window=window, want_lse=True, **on)

    def check(self, out, lse, scale, how, window=0):
        ks, vs = self.stored()
        u_out, u_w = U[self.kind], 2 * U[torch.float16] if self.storage in ("i8", "f8") else U[self.kind]
        out, lse, q, cap = out.cpu().double(), lse.cpu().double(), self.q.double(), how["cap"]
        slopes = how["slopes"].double() if "slopes" in how else torch.zeros(self.H * self.G, dtype=torch.float64)
        for row, i, pos in self.tokens():
            key = torch.arange(self.lens[i])
            mask = key <= pos
            if window:
                mask &= key > pos - window
            if "starts" in how:
                mask &= key >= how["starts"][row]
            if "prefix" in how:
                mask |= key < how["prefix"][i]
            mask &= self.there(i)
            for h in range(self.H):
                k, v, far = ks[i][mask, h], vs[i][mask, h], (pos - key[mask]).abs().double()
                rows = slice(h * self.G, (h + 1) * self.G)
                where = f"row {row} sequence {i} position {pos} head {h}"
                if k.shape[0] == 0:
                    assert torch.all(out[row, rows] == 0) and torch.all(lse[row, rows] == -math.inf), where
                    continue
                x = (q[row, rows] @ k.T) * scale
                size = ((q[row, rows].abs() @ k.abs().T) * abs(scale)).amax(1, keepdim=True)
                most = x.abs().amax(1, keepdim=True)
                if cap:
                    x = cap * torch.tanh(x / cap)
                bias = slopes[rows, None] * far
                x = x - bias
                w = torch.softmax(x, 1)
                # (a key that is far below the largest has no weight, and its error none either)
                near = x > x.amax(1, keepdim=True) - 60
                off_score = (self.D + 8) * 2.0 ** -24 * size + (2.0 ** -21 * (2 * most).clamp(max=cap) if cap else 0.0)
                off_score = off_score + ((2.0 ** -22 * bias.abs() + 2.0 ** -23 * x.abs()) * near).amax(1, keepdim=True)
                e = 2 * off_score + 2.0 ** -20
                ref, a = w @ v, w @ v.abs()
                cut = 2.0 ** -126 * v.abs().sum(0) + (2.0 ** -40 * v.shape[0] * v.abs().max() + 2.0 ** -24 if self.kind == torch.float16 else 2.0 ** -126)
                bound = u_out * ref.abs() + (u_w + e) * (1 + u_out) * a + cut
                off = (out[row, rows] - ref).abs()
                assert torch.all(off <= bound), f"{where}: {float((off / bound).max())} of the bound"
                full = torch.logsumexp(x, 1)
                common = 2.0 ** -17 * math.log(2) if self.storage == "i8" and self.kind == torch.bfloat16 else 0.0
                assert torch.all((lse[row, rows] - full).abs() <= e[:, 0] / 2 + 2.0 ** -20 * full.abs() + common), f"{where}: lse"


SHAPES = [
    # H, G, D, P, news, lens
    (1, 1, 64, 16, [1], [1]),
    (2, 4, 128, 64, [1, 1, 1], [1, 64, 65]),
    (3, 5, 64, 16, [7, 0, 1], [40, 0, 129]),
    (2, 3, 256, 128, [2], [300]),
    (1, 16, 128, 64, [1, 1], [700, 1300]),
    (2, 2, 80, 64, [90, 5], [90, 333]),
    (1, 7, 128, 64, [131], [1031]),
    (1, 4, 64, 32, [200], [517]),
    (1, 2, 256, 16, [70], [150]),
    (1, 4, 128, 64, [1], [2100]),                                        # in parts
    (8, 1, 64, 16, [1] * 16, [1100 + 13 * i for i in range(16)]),        # joined by a launch
    (1, 4, 128, 64, [70, 3], [1601, 900]),
]
HOWS = {"cap": dict(cap=5.0), "wide cap": dict(cap=300.0), "slopes": dict(slopes=0.25), "docs": dict(docs=37), "prefix": dict(prefix=[70, 3, 0]),
        "all": dict(cap=20.0, slopes=0.01, docs=150, prefix=[17, 130])}


@pytest.mark.parametrize("storage,dtype", CODES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[:4]} {len(s[4])} of {max(s[4])} at {max(s[5])}")
@pytest.mark.parametrize("how", HOWS)
def test_scored_attention(gpu_device, storage, dtype, shape, how):
    H, G, D, P, news, lens = shape
    s = Setup(storage, dtype, H, G, D, P, news, lens, seed=51, tail=2, spread=0.5)
    h, window = s.how(**HOWS[how]), 100 if how == "all" else 0
    out, lse = s.run(D ** -0.5, h, window)
    s.check(out, lse, D ** -0.5, h, window)
    for got, want in zip(s.run(D ** -0.5, h, window), (out, lse)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16"), ("f4", "bf16")])
@pytest.mark.parametrize("news,lens", [([1, 1, 3], [40, 700, 90]), ([100, 33], [100, 300])], ids=str)
@pytest.mark.parametrize("window", [1, 64, 65, 2 ** 31 - 1])
def test_windows(gpu_device, storage, dtype, news, lens, window):
    s = Setup(storage, dtype, 2, 2, 64, 16, news, lens, seed=52)
    for kind in (dict(cap=9.0), dict(prefix=[5, 0, 64]), dict(docs=20, prefix=[64])):
        h = s.how(**kind)
        out, lse = s.run(0.125, h, window)
        s.check(out, lse, 0.125, h, min(window, 2 ** 30))


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("news,lens", [([1, 2], [130, 40]), ([90, 1], [90, 300])], ids=str)
def test_masks_at_their_ends(gpu_device, storage, dtype, news, lens):
    """Prefixes longer than the sequence, negative, of one; documents that begin behind the token (nothing is seen), before the first position, at 2^31 - 1."""
    s = Setup(storage, dtype, 2, 3, 64, 32, news, lens, seed=53)
    n = sum(news)
    for prefix in (None, [1, 1], [10 ** 6, 0], [-5, 64], [-2 ** 31, 2 ** 31 - 1]):
        for starts in (None, [2 ** 31 - 1] * n, [-2 ** 31] * n, [lens[i] if row % 2 else max(pos - 3, 0) for row, i, pos in s.tokens()], [pos for _, _, pos in s.tokens()]):
            h = {"cap": 0.0, **({"prefix": torch.tensor(prefix, dtype=torch.int32)} if prefix else {}), **({"starts": torch.tensor(starts, dtype=torch.int32)} if starts else {})}
            if len(h) > 1:
                s.check(*s.run(0.1, h), 0.1, h)


@pytest.mark.parametrize("storage,dtype", CODES)
@pytest.mark.parametrize("scale", [-0.3, 0.0, 8.0, 1e4])
def test_scales_and_caps_of_any_size(gpu_device, storage, dtype, scale):
    """Scores far beyond their cap (all of them plus or minus it), caps far beyond any score, slopes of either sign."""
    for news in ([2, 1], [90, 1]):
        s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=54, spread=0.3)
        for kind in (dict(cap=1.0), dict(cap=30.0), dict(cap=3e4), dict(cap=1e30), dict(slopes=-0.5), dict(slopes=40.0), dict(cap=50.0, slopes=-3.0)):
            if scale == 1e4 and kind.get("cap", 1e30) > 1e4:
                continue  # (scores of 10^5: their own error is beyond any weight's)
            h = s.how(**kind)
            s.check(*s.run(scale, h), scale, h)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f4", "f16")])
def test_caps_and_scales_at_the_ends_of_32_bits(gpu_device, storage, dtype):
    for news in ([2, 1], [90, 1]):
        s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=62, spread=0.3)
        s.q[1] = 0  # (scores of 0)
        for scale, kind in ((0.125, dict(cap=3e38)), (0.125, dict(cap=1e-40)), (0.125, dict(cap=1e-30, slopes=0.1)), (1e-40, dict(cap=2.0)), (2.0 ** -60, dict(slopes=0.1)), (1e-40, dict(docs=9))):
            h = s.how(**kind)
            s.check(*s.run(scale, h), scale, h)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f4", "f16")])
def test_without_some_pages(gpu_device, storage, dtype):
    s = Setup(storage, dtype, 2, 3, 64, 16, [5, 1, 20, 33], [70, 17, 20, 90], seed=55, missing=[(0, 0), (0, 2), (1, 0), (1, 1), (2, 0), (3, 5), (3, 4), (3, 3)])
    for kind in (dict(cap=9.0), dict(prefix=[40, 17, 20, 1]), dict(docs=33, slopes=0.1)):
        h = s.how(**kind)
        s.check(*s.run(0.125, h), 0.125, h)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16"), ("f4", "bf16")])
@pytest.mark.parametrize("P,D", [(64, 128), (16, 64)])
@pytest.mark.parametrize("news", [[10], [33], [5, 256], [0, 3], [17, 64]], ids=str)
def test_fewer_tokens_than_the_host_says(gpu_device, storage, dtype, P, D, news):
    """Rows of no token, of queries and of starts alike, are neither read nor written."""
    s = Setup(storage, dtype, 2, 4, D, P, news, [n + 70 for n in news], seed=56)
    n = 256 * len(news)
    batch = B.KVBatch(s.batch.tables, s.batch.offsets, s.batch.lens, n, 256, max(s.lens) + 300)
    h = s.how(cap=9.0, slopes=0.1, docs=31, prefix=[20])
    q = torch.cat([s.q, torch.full((n - sum(news), 8, D), math.nan, dtype=s.kind)]).cuda()
    starts = torch.cat([h["starts"], torch.full((n - sum(news),), -77, dtype=torch.int32)]).cuda()
    out, lse = torch.full_like(q, math.nan), torch.full(q.shape[:2], math.nan, device="cuda")
    B.pk_kv_attend_scored(s.cache.handle, batch.c, q, 0.1, 0, 9.0, h["slopes"].cuda(), starts, h["prefix"].cuda(), out, lse)
    s.check(out[:sum(news)], lse[:sum(news)], 0.1, h)
    assert torch.all(out[sum(news):].isnan()) and torch.all(lse[sum(news):].isnan())


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "f16"), ("f4", "bf16")])
def test_what_no_query_sees_changes_no_bit(gpu_device, storage, dtype):
    """Rows behind a sequence's end, other sequences' scores beside the cap, other contents of pages that are free."""
    got = []
    for garbage, size in ((0xff, 1.0), (0x00, 1.0), (0x7b, 40.0)):
        s = Setup(storage, dtype, 2, 4, 64, 64, [1, 40, 1], [75, 100, 300], seed=61, garbage=garbage)
        s.q[0] *= size  # (another sequence's queries)
        out, lse = s.run(0.125, s.how(cap=1000.0, slopes=0.01))
        got.append((out[1:], lse[1:]))
    for out, lse in got[1:]:
        assert torch.equal(out, got[0][0]) and torch.equal(lse, got[0][1])


def test_calls_in_a_graph_follow_the_arrays(gpu_device):
    """Lengths, documents, prefixes and slopes change between replays."""
    s = Setup("i8", "bf16", 2, 4, 64, 16, [1, 40], [400, 300], seed=58)
    n = 41
    offsets, lens, q = s.batch.offsets.clone(), s.batch.lens.clone(), s.q.cuda()
    batch = B.KVBatch(s.batch.tables, offsets, lens, n, 40, 400)
    starts, prefix, slopes = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device="cuda")

    def step():
        B.pk_kv_attend_scored(s.cache.handle, batch.c, q, 0.125, 0, 12.0, slopes, starts, prefix, out, lse)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i, (news, ends, kind) in enumerate([([1, 40], [400, 300], dict(docs=50)), ([40, 1], [390, 20], dict(prefix=[100, 7], slopes=0.2)), ([0, 30], [0, 30], dict(docs=11, prefix=[5, 20]))]):
        s.news, s.lens = news, ends
        h = {"starts": torch.zeros(sum(news), dtype=torch.int32), "prefix": torch.zeros(2, dtype=torch.int32), "slopes": torch.zeros(8), **s.how(**kind), "cap": 12.0}
        offsets.copy_(torch.tensor([0, news[0], sum(news)], dtype=torch.int32))
        lens.copy_(torch.tensor(ends, dtype=torch.int32))
        starts[:sum(news)] = h["starts"].cuda()
        prefix.copy_(h["prefix"])
        slopes.copy_(h["slopes"])
        out.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        whole = s.q
        s.q = whole[:sum(news)]
        s.check(out[:sum(news)], lse[:sum(news)], 0.125, h)
        s.q = whole
        assert torch.all(out[sum(news):].isnan()), i


def test_on_another_stream_and_beside_another_cache(gpu_device):
    a, b = (Setup("bf16", "bf16", 2, 2, 64, 64, [30, 1], [300, 2500], seed=59 + i) for i in range(2))
    hows = [x.how(cap=8.0, docs=100) for x in (a, b)]
    want = [x.run(0.1, h) for x, h in zip((a, b), hows)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(5):
        for i, (x, h, stream) in enumerate(zip((a, b), hows, streams)):
            with torch.cuda.stream(stream):
                got[i] = x.run(0.1, h)
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])


def test_refusals(gpu_device):
    s = Setup("bf16", "bf16", 2, 2, 64, 16, [2], [20], seed=60)
    q, good = s.q.cuda(), torch.zeros(4, device="cuda")
    for cap in (-1.0, math.nan, math.inf):
        with pytest.raises(B.PancakeError) as e:
            s.cache.attend(q, s.batch, 0.1, cap=cap)
        assert e.value.status == B.PK_ERR_INVALID_ARG
    for bad in (dict(slopes=good[:3]), dict(slopes=good.double()), dict(slopes=good.cpu()), dict(starts=torch.zeros(3, dtype=torch.int32, device="cuda")),
                dict(starts=torch.zeros(2, device="cuda")), dict(prefix=torch.zeros(2, dtype=torch.int32, device="cuda"))):
        with pytest.raises(ValueError):
            s.cache.attend(q, s.batch, 0.1, **bad)
    with pytest.raises(B.PancakeError) as e:
        s.cache.attend(q, s.batch, 1e-30, slopes=good)
    assert e.value.status == B.PK_ERR_UNSUPPORTED
    for bad in (dict(window=-1), dict(scale=math.nan)):
        with pytest.raises(B.PancakeError) as e:
            s.cache.attend(q, s.batch, **{"scale": 0.1, "cap": 2.0, **bad})
        assert e.value.status == B.PK_ERR_INVALID_ARG
    nothing = B.KVBatch(s.batch.tables, torch.zeros(2, dtype=torch.int32, device="cuda"), s.batch.lens, 0, 0, 20)
    assert s.cache.attend(q[:0], nothing, 0.1, cap=2.0).shape == (0, 4, 64)
    assert B.lib().pk_kv_attend_scored(s.cache.handle, s.batch.c, B._rows(q, "q"), 4, 0.1, 0, None, q.data_ptr(), None, None) == B.PK_ERR_INVALID_ARG
