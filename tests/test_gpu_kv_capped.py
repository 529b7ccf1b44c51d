"""Attention with caps, slopes and scales at the ends of what they may be, and lse of rows that see few keys with scores far below their cap.

Tolerances are those of test_gpu_kv_scored, but for a score's error by its cap, which there is 2^-21 of the score or of the cap.  Caps up to 64 are -1 / (1 + 2^p) in units of twice the cap, whatever the score:
p is off by 4 roundings, 2^-22 of itself, which moves 1 / (1 + 2^p) by 2^-22 |z| sech^2 z / 2 <= 2^-22 0.23; 2^p by 2^-23 of itself, which moves it by 2^-25; the sum is rounded by 2^-24 of itself and the
reciprocal by 2^-23 of itself, but no more than 2^-24 as it is below 1: together below (0.23 + 0.125 + 0.25 + 0.25) 2^-22, twice the cap: 2^-21 0.86 of it.  A sum with 1/2, for lse, adds 2^-25 of twice the cap
where it is not exact: 2^-21 of the cap in all.
lse: also 2^-20 ln 2, of int8 under bfloat16 2^-17 ln 2.  Weights are 2^(x + top - m), top 15, 16 or 127: top - m, where m is a little below 0, is rounded to 2^-20 (16 to 32) or 2^-17 (128 to 256), the
same factor for all weights of a sum, which cancels in a result and is left in the logarithm."""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B
import test_gpu_kv as base
import test_gpu_kv_scored as scored
from test_gpu_kv import U

pytestmark = pytest.mark.gpu


class Setup(scored.Setup):
    def check_all(self, out, lse, scale, how):
        """All of test_gpu_kv_scored's, but for the cap's error."""
        ks, vs = self.stored()
        u_out, u_w = U[self.kind], 2 * U[torch.float16] if self.storage in ("i8", "f8") else U[self.kind]
        out, lse, q, cap = out.cpu().double(), lse.cpu().double(), self.q.double(), float(how["cap"])
        slopes = how["slopes"].double() if "slopes" in how else torch.zeros(self.H * self.G, dtype=torch.float64)
        for row, i, pos in self.tokens():
            key = torch.arange(self.lens[i])
            mask = key <= pos
            if "starts" in how:
                mask &= key >= how["starts"][row]
            if "prefix" in how:
                mask |= key < how["prefix"][i]
            for h in range(self.H):
                k, v, far = ks[i][mask, h], vs[i][mask, h], (pos - key[mask]).abs().double()
                rows = slice(h * self.G, (h + 1) * self.G)
                where = f"row {row} sequence {i} position {pos} head {h}"
                x = (q[row, rows] @ k.T) * scale
                size = ((q[row, rows].abs() @ k.abs().T) * abs(scale)).amax(1, keepdim=True)
                most = x.abs().amax(1, keepdim=True)
                if cap:
                    x = cap * torch.tanh(x / cap)
                bias = slopes[rows, None] * far
                x = x - bias
                w = torch.softmax(x, 1)
                near = x > x.amax(1, keepdim=True) - 60
                by_cap = 2.0 ** -21 * cap if cap <= 64 else 2.0 ** -21 * (2 * most).clamp(max=cap)
                off_score = (self.D + 8) * 2.0 ** -24 * size + by_cap + ((2.0 ** -22 * bias.abs() + 2.0 ** -23 * x.abs()) * near).amax(1, keepdim=True)
                e = 2 * off_score + 2.0 ** -20
                ref, a = w @ v, w @ v.abs()
                cut = 2.0 ** -126 * v.abs().sum(0) + (2.0 ** -40 * v.shape[0] * v.abs().max() + 2.0 ** -24 if self.kind == torch.float16 else 2.0 ** -126)
                bound = u_out * ref.abs() + (u_w + e) * (1 + u_out) * a + cut
                off = (out[row, rows] - ref).abs()
                assert torch.all(off <= bound), f"{where}: {float((off / bound).max())} of the bound"
                full = torch.logsumexp(x, 1)
                common = math.log(2) * (2.0 ** -17 if self.storage == "i8" and self.kind == torch.bfloat16 else 2.0 ** -20)
                assert torch.all((lse[row, rows] - full).abs() <= e[:, 0] / 2 + 2.0 ** -20 * full.abs() + common), f"{where}: lse"


@pytest.mark.parametrize("storage,dtype", scored.CODES)
@pytest.mark.parametrize("cap", [1.0, 30.0, 50.0, 64.0, 65.0, 1000.0])
@pytest.mark.parametrize("docs", [1, 3])
def test_few_keys_with_scores_far_below_the_cap(gpu_device, storage, dtype, cap, docs):
    for news in ([3, 2], [90, 1]):
        s = Setup(storage, dtype, 2, 3, 64, 32, news, [130, 40], seed=81, spread=1.0)
        s.q = (s.q.float() * 0.02).to(s.kind)
        h = s.how(cap=cap, docs=docs)
        s.check_all(*s.run(0.125, h), 0.125, h)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("cap", [65.0, 1e6, 1e30, 1e37, 3e38])
@pytest.mark.parametrize("power", [12, 7])
def test_wide_caps_of_small_scales(gpu_device, dtype, cap, power):
    """Large products that a small scale brings to scores of a few units: a cap beyond 64 leaves them, whatever its size over the scale's."""
    for storage in (dtype, "i8", "f8", "f4"):
        for news in ([2, 1], [90, 1]):
            s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=82, spread=0.3)
            large, scale = 2.0 ** power, 2.0 ** (-2 * power - 3)
            s.q = s.q * large
            s.k = [x * large for x in s.k]
            s.write(news=s.lens, rows=(s.k, s.v))
            h = s.how(cap=cap)
            s.check_all(*s.run(scale, h), scale, h)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f4", "f16")])
@pytest.mark.parametrize("cap", [0.0, 1e-38, 2.0, 1000.0])
@pytest.mark.parametrize("slope", [1e9, 1e25, 3e38])
def test_steep_slopes_leave_the_nearest_key(gpu_device, storage, dtype, cap, slope):
    """All weight is the nearest key's (with the other sign the farthest one's), and no product with a distance is anything but a number."""
    for news in ([2, 1], [90, 1]):
        for sign in (1.0, -1.0):
            s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=83, spread=0.3)
            n = sum(news)
            _, vs = s.stored()
            where = {"slopes": torch.full((2,), sign * slope), "cap": cap}
            # everything; and a prefix alone, each query's nearest key then far away
            for extra, nearest, farthest in (({}, lambda pos: pos, lambda pos: 0), ({"starts": torch.full((n,), 10 ** 6, dtype=torch.int32), "prefix": torch.tensor([9, 9], dtype=torch.int32)},
                                                                                     lambda pos: min(pos, 8), lambda pos: 0 if pos >= 4 else 8)):
                out, lse = s.run(0.125, {**where, **extra})
                for row, i, pos in s.tokens():
                    if "prefix" in extra and pos in (4,):
                        continue  # (both ends as far)
                    v = vs[i][nearest(pos) if sign > 0 else farthest(pos), 0]
                    off = (out[row].cpu().double() - v).abs()
                    # one weight, of 1: its rounding with a value's scale, and the result's
                    assert bool((off <= 2 * 2 * U[s.kind] * v.abs() + 2.0 ** -24).all()), (row, pos, sign, float(off.max()))
                    assert not bool(lse[row].isnan().any()), (row, pos)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("f8", "f16")])
@pytest.mark.parametrize("cap", [1e-40, 1e-25, 2.0 ** -61])
def test_caps_of_next_to_nothing(gpu_device, storage, dtype, cap):
    """Every key that is seen weighs the same, or by its distance alone."""
    for news in ([2, 1], [90, 1]):
        s = Setup(storage, dtype, 1, 2, 64, 32, news, [130, 40], seed=84, spread=0.3)
        for kind in (dict(cap=cap), dict(cap=cap, slopes=1.0), dict(cap=cap, slopes=-0.01)):
            h = s.how(**kind)
            s.check_all(*s.run(0.125, h), 0.125, h)
