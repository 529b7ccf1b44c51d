"""Rows with an element that is no number, quiet or signalling: it is ignored where a row's largest magnitude and a page's bounds are looked for, so that everything else is stored as if
it were zero.  Bits have to be equal."""
import pytest
import torch

from paper_2602_21477_amd import binding as B

pytestmark = pytest.mark.gpu

STORAGES = {"f16": B.PK_F16, "bf16": B.PK_BF16, "i8": B.PK_I8, "f8": B.PK_F8, "f4": B.PK_F4}
# type, its bits, and its quiet and signalling numbers
TYPES = {"f16": (torch.float16, torch.int16, 0x7e00, 0x7c01), "bf16": (torch.bfloat16, torch.int16, 0x7fc0, 0x7f81), "f32": (torch.float32, torch.int32, 0x7fc00000, 0x7f800001)}


@pytest.mark.parametrize("storage", STORAGES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("D,P", [(64, 16), (128, 64), (256, 32), (40, 128)])
@pytest.mark.parametrize("signalling", [False, True])
@pytest.mark.parametrize("in_parts", [False, True])
def test_an_element_that_is_no_number_is_ignored(gpu_device, storage, dtype, D, P, signalling, in_parts):
    kind, bits, quiet, signal = TYPES[dtype]
    H, n = 2, 2 * P + 5
    gen = torch.Generator().manual_seed(71)
    k, v = (torch.randn(n, H, D, generator=gen) for _ in range(2))
    where = torch.zeros(n, H, D, dtype=torch.bool)
    for i in range(0, n, 3):  # each lane's place in turn, with the row's largest before it, and behind it
        at = (5 * i + 1) % D
        where[i, i % H, at] = True
        for x in (k, v):
            x[i, :, (at - 1) % D if i % 2 else (at + 1) % D] = 9.0
    got = []
    for planted in (False, True):
        cache = B.KVCache(4, H, D, storage=STORAGES[storage], page_tokens=P)
        cache.arena.fill_(0)
        tables = torch.tensor([[2, 0, 3]], dtype=torch.int32, device="cuda")
        rows = []
        for x in (k, v):
            x = torch.where(where, torch.zeros(()), x).to(kind)
            if planted:
                x.view(bits)[where] = signal if signalling else quiet
            rows.append(x.cuda())
        for begin, end in ([(0, 1), (1, P + 2), (P + 2, n)] if in_parts else [(0, n)]):
            batch = B.KVBatch(tables, torch.tensor([0, end - begin], dtype=torch.int32).cuda(), torch.tensor([end], dtype=torch.int32).cuda(), end - begin, end - begin, end)
            cache.append(rows[0][begin:end], rows[1][begin:end], batch)
        whole = B.KVBatch(tables, torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda(), n, n, n)
        got.append(([x.cpu() for x in cache.read(whole, torch.float32)], [x.cpu() for x in cache.bounds(tables[0])]))
    (want, want_bounds), (have, have_bounds) = got
    for a, b in zip(want, have):
        assert torch.equal(a[~where], b[~where])
    pages = torch.zeros(3, H, D, dtype=torch.bool)  # channels of pages that have such an element
    for i in range(n):
        pages[i // P] |= where[i]
    for a, b in zip(want_bounds, have_bounds):
        assert torch.equal(a[~pages], b[~pages])
