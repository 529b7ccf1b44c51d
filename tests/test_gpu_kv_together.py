"""The pool, 4 bits and scored attention as they are used together: agents read documents, branch, go on, are moved, and forget."""
import pytest
import torch

from paper_2602_21477_amd import binding as B
from paper_2602_21477_amd.context_example import Agents

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("storage", [B.PK_F4, B.PK_I8, B.PK_BF16])
def test_branches_of_the_example_are_what_longer_sequences_are(gpu_device, storage):
    """A token tried in a branch is scored as the same token appended by itself is, and leaves the agent's context and pages as they were."""
    agents = Agents(n_agents=3, passages=300, storage=storage, page=16, branches=2)
    questions = torch.nn.functional.normalize(torch.randn(3, agents.d, generator=agents.gen, device="cuda"), dim=-1)
    agents.read(agents.recall(questions, k=4), tokens_each=7)
    tables, counts = agents.tables.clone(), agents.pool.counts()
    tries = questions[:, None] + 0.1 * torch.randn(3, 2, agents.d, generator=agents.gen, device="cuda")
    got = agents.try_tokens(tries)
    assert torch.equal(agents.tables, tables) and torch.equal(agents.pool.counts(), counts)
    q, k, v = agents.layer(tries[:, 1])
    batch = agents.step([1, 1, 1])
    agents.cache.append(k, v, batch)
    _, lse = agents.cache.attend(q, batch, agents.scale, want_lse=True, cap=30.0)
    # (of the same stored rows, but cut into other parts: sums of 32 bits, and scores of 30 at most)
    assert float((lse.amax(-1) - got[:, 1]).abs().max()) <= 2.0 ** -16
    for i in range(3):
        agents.forget(i)
    assert int(agents.pool.counts().sum()) == 0 and bool((agents.tables == -1).all())
    agents.close()


@pytest.mark.parametrize("storage,dtype", [(B.PK_F4, torch.bfloat16), (B.PK_F4, torch.float16), (B.PK_F8, torch.float16)])
@pytest.mark.parametrize("P,D", [(16, 64), (64, 128)])
def test_a_life_of_sequences(gpu_device, storage, dtype, P, D):
    """Documents behind a shared prompt, forks of it, tokens in the branches, compaction into a cache of another size, and on: every output against
    64 bits over the rows that the sequences hold by then."""
    H, G, gen = 2, 2, torch.Generator("cuda").manual_seed(3)
    u = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -11
    cache = B.KVCache(80, H, D, storage=storage, page_tokens=P)
    cache.arena.fill_(0xff)
    pool, rows = B.KVPool(cache), 4
    tables = torch.full((rows, 12), -1, dtype=torch.int32, device="cuda")
    lens, held = [0] * rows, [None] * rows
    scale, cap, slopes = D ** -0.5, 12.0, torch.tensor([0.05, 0.01, 0.0, 0.2], device="cuda")

    def step(some, new, prefix, doc):
        cache = state["cache"]
        for r, m in zip(some, new):
            lens[r] += m
        n = sum(new)
        b = B.KVBatch(state["tables"][some[0]:some[-1] + 1], ints([0] + new).cumsum(0).int(), ints([lens[r] for r in some]), n, max(new), max(lens))
        assert state["pool"].grant(b).item() == 0
        q, k, v = (torch.randn(n, h, D, device="cuda", generator=gen).to(dtype) for h in (H * G, H, H))
        cache.append(k, v, b)
        where = [(r, lens[r] - m + j) for r, m in zip(some, new) for j in range(m)]
        starts = [max(prefix[r] + (p - prefix[r]) // doc * doc, 0) if p >= prefix[r] else p for r, p in where]
        out, lse = cache.attend(q, b, scale, cap=cap, slopes=slopes, starts=ints(starts), prefix=ints([prefix[r] for r in some]), want_lse=True)
        for r in some:
            whole = B.KVBatch(state["tables"][r:r + 1], ints([0, lens[r]]), ints([lens[r]]), lens[r], lens[r], lens[r])
            now = torch.stack(cache.read(whole, torch.float32)).double()
            if held[r] is not None:
                assert torch.equal(now[:, :held[r].shape[1]], held[r]), f"row {r}: what it held has changed"
            held[r] = now
        for i, ((r, p), start) in enumerate(zip(where, starts)):
            key = torch.arange(lens[r], device="cuda")
            seen = ((key >= start) & (key <= p)) | (key < prefix[r])
            for h in range(H * G):
                kk, vv = held[r][0][seen, h // G], held[r][1][seen, h // G]
                raw = (kk @ q[i, h].double()) * scale
                x = cap * torch.tanh(raw / cap) - slopes[h].double() * (p - key[seen]).abs()
                w = torch.softmax(x, 0)
                ref, a = w @ vv, w @ vv.abs()
                # the tolerances of test_gpu_kv_scored (the largest of each error)
                e = 2 * ((D + 8) * 2.0 ** -24 * float((kk.abs() @ q[i, h].double().abs()).max()) * scale + 2.0 ** -21 * cap + 2.0 ** -22 * 0.2 * lens[r] + 2.0 ** -23 * float(x.abs().max())) + 2.0 ** -20
                bound = u * ref.abs() + (2 * u + e) * (1 + u) * a + 2.0 ** -24 + 2.0 ** -40 * float(vv.abs().sum())
                assert torch.all((out[i, h].double() - ref).abs() <= bound), (r, p, h)
                assert abs(float(lse[i, h]) - float(torch.logsumexp(x, 0))) <= e / 2 + 2.0 ** -20 * abs(float(torch.logsumexp(x, 0))), (r, p, h)

    state = {"cache": cache, "pool": pool, "tables": tables}
    prompt = P + 5
    step([0], [prompt], [prompt] * 4, 9)  # a prompt that sees itself in both directions
    pool.fork(tables, ints(lens), ints([0, 0, 0]), ints([1, 2, 3]))
    for r in (1, 2, 3):
        lens[r], held[r] = lens[0], held[0]
    assert sorted(pool.counts().tolist())[-2:] == [4, 4]
    step([0, 1, 2, 3], [1, 40, 3, 9], [prompt] * 4, 11)  # everybody writes into the shared page: the last one keeps it
    step([2, 3], [70, 1], [prompt] * 4, 25)
    pool.release(tables, ints([1, 3]), ints([0, prompt]))
    lens[1], held[1], lens[3], held[3] = 0, None, prompt, held[3][:, :prompt]
    live = int((pool.counts() > 0).sum())
    into = B.KVPool(B.KVCache(live + 7, H, D, storage=storage, page_tokens=P))
    into.cache.arena.fill_(0xff)
    moved, missing = pool.compact(into, tables)
    assert missing.item() == 0
    cache.arena.fill_(0x55)  # (what was is not needed any more)
    state = {"cache": into.cache, "pool": into, "tables": moved}
    step([0], [1], [prompt] * 4, 30)
    step([2, 3], [1, 2], [prompt] * 4, 30)
    assert int((into.counts() > 0).sum()) == len(set(moved.flatten().tolist()) - {-1})
    cache.close()
    into.cache.close()
