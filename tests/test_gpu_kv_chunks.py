"""Attention of chunks on either side of what decides how their launch is cut, all rows of them, against 64 bits on the GPU.

Tolerances as in test_gpu_kv: an output's own rounding u_out, the weights' u_w (codes of 8 bits: half, twice), a score's error (D + 8) 2^-24 sum|q k| scale, twice, and 2^-20;
half a step of half precision's smallest numbers, 2^-25.  lse: half of the score's, 2^-20 of itself, and of int8 under bfloat16 2^-17 ln 2, as there 127 less the maximum is rounded to
2^-17 (test_gpu_kv_scored)."""
import math

import pytest
import torch

from paper_2602_21477_amd import binding as B
from test_gpu_kv import STORAGES, TYPES, U

pytestmark = pytest.mark.gpu


def filled(storage, dtype, H, G, D, P, news, lens, seed=0):
    """A cache with sequences of `lens` tokens, their queries, the batch of the last `news` of them, and what is stored."""
    gen = torch.Generator("cuda").manual_seed(seed)
    cols = [-(-n // P) for n in lens]
    cache = B.KVCache(sum(cols) + 2, H, D, storage={**STORAGES, "f4": B.PK_F4}[storage], page_tokens=P)
    cache.arena.fill_(0xff)
    order = torch.randperm(sum(cols) + 2, generator=gen, device="cuda").int()
    tables = torch.full((len(lens), max(cols)), -1, dtype=torch.int32, device="cuda")
    for i, at in enumerate(torch.tensor([0] + cols).cumsum(0)[:-1].tolist()):
        tables[i, :cols[i]] = order[at:at + cols[i]]

    def batch(news):
        return B.KVBatch(tables, torch.tensor([0] + news).cumsum(0).int().cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), sum(news), max(news), max(lens))
    k, v = (torch.randn(sum(lens), H, D, generator=gen, device="cuda").to(TYPES[dtype]) for _ in range(2))
    cache.append(k, v, batch(lens))
    q = torch.randn(sum(news), H * G, D, generator=gen, device="cuda").to(TYPES[dtype])
    return cache, q, batch(news), [x.double() for x in cache.read(batch(lens), torch.float32)]


def check(out, lse, q, stored, news, lens, scale, storage, window=0):
    kind, (G, D) = q.dtype, (q.shape[1] // stored[0].shape[1], q.shape[2])
    u_out, u_w = U[kind], 2 * U[torch.float16] if storage in ("i8", "f8") else U[kind]
    common = 2.0 ** -17 * math.log(2) if storage == "i8" and kind == torch.bfloat16 else 0.0
    row, token = 0, 0
    for m, n in zip(news, lens):
        for h in range(stored[0].shape[1]):
            k, v = (x[token:token + n, h] for x in stored)
            for r in range(row, row + m, 256):  # (a part of the rows at a time)
                some = slice(r, min(r + 256, row + m))
                pos = torch.arange(n - m, n, device="cuda")[r - row:r - row + 256]
                x = q[some, h * G:(h + 1) * G].double()
                size = (x.abs() @ k.abs().T).amax(-1, keepdim=True) * abs(scale)
                x = x @ k.T * scale
                key = torch.arange(n, device="cuda")
                seen = (key <= pos[:, None]) & ((key > pos[:, None] - window) if window else True)
                x = x.masked_fill(~seen[:, None], -torch.inf)
                w = torch.softmax(x, -1)
                ref, a, e = w @ v, w @ v.abs(), 2 * (D + 8) * 2.0 ** -24 * size + 2.0 ** -20
                bound = u_out * ref.abs() + (u_w + e) * (1 + u_out) * a + (2.0 ** -25 if kind == torch.float16 else 2.0 ** -126)
                off = (out[some, h * G:(h + 1) * G].double() - ref).abs()
                assert bool((off <= bound).all()), f"rows {some} head {h}: {float((off / bound).max())} of the bound"
                full = torch.logsumexp(x, -1)
                assert bool(((lse[some, h * G:(h + 1) * G].double() - full).abs() <= e[..., 0] / 2 + 2.0 ** -20 * full.abs() + common).all()), f"rows {some} head {h}: lse"
        row, token = row + m, token + n


def run(storage, dtype, H, G, D, P, news, lens, window=0, seed=0):
    cache, q, batch, stored = filled(storage, dtype, H, G, D, P, news, lens, seed)
    out, lse = cache.attend(q, batch, D ** -0.5, window=window, want_lse=True)
    check(out, lse, q, stored, news, lens, D ** -0.5, storage, window)
    again = cache.attend(q, batch, D ** -0.5, window=window, want_lse=True)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    cache.close()


@pytest.mark.parametrize("storage", ["bf16", "f16", "i8"])
@pytest.mark.parametrize("H,G,D,P,news,lens", [(8, 4, 64, 64, [100], [100]),                          # fewer workgroups than the chip has CUs
                                               (8, 4, 64, 128, [2048], [2111]),                       # as many
                                               (8, 8, 64, 64, [1111], [1300]), (2, 8, 40, 64, [999, 1500, 3, 2000], [1000, 1500, 900, 2077])],  # more
                         ids=str)
def test_chunks_of_64_channels(gpu_device, storage, H, G, D, P, news, lens):
    run(storage, "f16" if storage == "f16" else "bf16", H, G, D, P, news, lens, seed=1)


@pytest.mark.parametrize("storage,dtype", [("bf16", "bf16"), ("i8", "bf16"), ("f4", "f16")])
@pytest.mark.parametrize("H,G,D,P,news,lens", [(1, 8, 64, 64, [32], [70001]), (2, 8, 128, 16, [33], [33000]), (1, 8, 256, 64, [32], [66000]), (1, 16, 64, 32, [40, 20], [50000, 35000])], ids=str)
def test_chunks_of_few_heads_in_many_parts(gpu_device, storage, dtype, H, G, D, P, news, lens):
    """A part for every eight tiles of 64 keys, 64 and more of them."""
    run(storage, dtype, H, G, D, P, news, lens, seed=2)
