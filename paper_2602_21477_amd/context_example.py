"""Agents that remember, read what they remembered, and answer: the memory's search and the context's cache together.

    python -m paper_2602_21477_amd.context_example

Every agent has a memory of its own (an index of passage vectors) and a sequence of its own in one layer's key/value cache, whose pages
come from one pool as sequences grow.  A turn is what an agent's serving loop does on the GPU:

  1. the agents' questions are searched, each in its agent's memory, in one call;
  2. the passages that were found become tokens, whose keys and values are appended to the agents' sequences (a chunk each, of
     another length for every agent): documents that see all that was before, and not one another;
  3. every agent tries several next tokens at once: its sequence branches, the branches share its pages, and the one whose attention is
     the least spread goes on;
  4. the agents answer token by token: the new token's key and value are appended, its query picks the blocks of the context whose
     bounds promise the most, and attends to those alone.

A model's layers are stood in for by fixed random projections of the passages' vectors; nothing else is left out.
"""
from __future__ import annotations

import torch

from . import binding as B


class Agents:
    def __init__(self, n_agents=4, passages=2000, d=128, heads=4, group=4, head_dim=64, max_tokens=4096, page=32, storage=B.PK_I8, branches=3, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.gen, self.n, self.d, self.heads, self.group, self.head_dim, self.page, self.branches = gen, n_agents, d, heads, group, head_dim, page, branches
        self.scale = head_dim ** -0.5
        # memories: passages, and centroids from a sample of them
        self.passages = torch.nn.functional.normalize(torch.randn(n_agents, passages, d, generator=gen, device="cuda"), dim=-1)
        self.memories = [B.Index(p[torch.randperm(passages, generator=gen, device="cuda")[:32]].contiguous(), p.contiguous()) for p in self.passages]
        # one layer's cache for all agents: a row of the tables for each, and for each of its branches (by agent: 0 .. branches - 1)
        cols = max_tokens // page
        self.cache = B.KVCache(n_agents * (cols + branches), heads, head_dim, storage=storage, page_tokens=page)
        self.pool = B.KVPool(self.cache)
        self.tables = torch.full((n_agents * (1 + branches), cols), -1, dtype=torch.int32, device="cuda")
        self.lens = [0] * n_agents
        self.max_tokens = max_tokens
        self.project = torch.randn(d, (group * heads + 2 * heads) * head_dim, generator=gen, device="cuda", dtype=torch.bfloat16) * 0.3

    def layer(self, x):
        """Queries, keys and values of tokens, as parts of one product's rows."""
        rows = (x.to(torch.bfloat16) @ self.project).view(x.shape[0], -1, self.head_dim)
        hq = self.heads * self.group
        return rows[:, :hq], rows[:, hq:hq + self.heads], rows[:, hq + self.heads:]

    def batch(self, rows, lens, new):
        """A step of rows of the tables (a range of them) that has pages for its new tokens."""
        if max(lens) > self.max_tokens:
            raise ValueError(f"a sequence of {max(lens)} tokens, and room for {self.max_tokens}")
        offsets = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32)
        batch = B.KVBatch(self.tables[rows], offsets.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), sum(new), max(new), max(lens))
        self.pool.grant(batch)
        return batch

    def step(self, new):
        """The batch of a step in which agent i gets new[i] tokens."""
        self.lens = [l + m for l, m in zip(self.lens, new)]
        return self.batch(slice(0, self.n), self.lens, new)

    def recall(self, questions, k=8, nprobe=8):
        """Ids of the passages nearest to every agent's question."""
        ids, _ = B.search_multi(self.memories, list(range(self.n + 1)), questions, k, nprobe)
        return ids

    def read(self, ids, tokens_each=24):
        """The found passages as tokens (agent i takes i more of each), appended and attended from: each passage is a document."""
        each = [tokens_each + i for i in range(self.n)]
        new = [ids.shape[1] * m for m in each]
        x = torch.cat([self.passages[i][ids[i]].repeat_interleave(m, 0) for i, m in enumerate(each)])
        x = x + 0.2 * torch.randn(x.shape, generator=self.gen, device="cuda")
        q, k, v = self.layer(x)
        before = torch.tensor(self.lens, dtype=torch.int32).cuda()
        starts = torch.cat([l + torch.arange(n) // m * m for l, n, m in zip(self.lens, new, each)]).to(torch.int32).cuda()
        batch = self.step(new)
        self.cache.append(k, v, batch)
        return self.cache.attend(q, batch, self.scale, starts=starts, prefix=before)

    def try_tokens(self, x):
        """Several next tokens of every agent, x [agent, branch, d], each in a branch of its sequence: how much its query's attention is
        concentrated (the largest logarithm of a sum of weights), [agent, branch].  The branches are given up again."""
        n, w = self.n, self.branches
        targets = torch.arange(n, n * (1 + w), dtype=torch.int32).cuda()
        sources = torch.arange(n, dtype=torch.int32).repeat_interleave(w).cuda()
        self.pool.fork(self.tables, torch.tensor(self.lens + [0] * (n * w), dtype=torch.int32).cuda(), sources, targets)
        q, k, v = self.layer(x.reshape(n * w, -1))
        batch = self.batch(slice(n, n * (1 + w)), [l + 1 for l in self.lens for _ in range(w)], [1] * (n * w))
        self.cache.append(k, v, batch)
        _, lse = self.cache.attend(q, batch, self.scale, want_lse=True, cap=30.0)
        self.pool.release(self.tables, targets)
        return lse.amax(-1).view(n, w)

    def answer(self, x, blocks=8):
        """One token of every agent: (output, blocks it attended to)."""
        q, k, v = self.layer(x)
        batch = self.step([1] * self.n)
        self.cache.append(k, v, batch)
        chosen = self.cache.select(q, batch, blocks)
        return self.cache.attend_blocks(q, chosen, batch, self.scale), chosen, (q, batch)

    def forget(self, agent):
        """An agent's context is given up."""
        self.pool.release(self.tables, torch.tensor([agent], dtype=torch.int32).cuda())
        self.lens[agent] = 0

    def close(self):
        self.pool.close()
        self.cache.close()
        for m in self.memories:
            m.close()


def main(turns=2, words=16):
    """A few turns; returns how much of the full attention's weight the chosen blocks held, on average, over all answers."""
    agents = Agents()
    kept = []
    for turn in range(turns):
        questions = torch.nn.functional.normalize(torch.randn(agents.n, agents.d, generator=agents.gen, device="cuda"), dim=-1)
        ids = agents.recall(questions)
        agents.read(ids)
        tries = questions[:, None] + 0.1 * torch.randn(agents.n, agents.branches, agents.d, generator=agents.gen, device="cuda")
        x = tries[torch.arange(agents.n), agents.try_tokens(tries).argmax(-1).cpu()]
        for _ in range(words):
            out, chosen, (q, batch) = agents.answer(x)
            _, part = agents.cache.attend_blocks(q, chosen, batch, agents.scale, want_lse=True)
            _, whole = agents.cache.attend(q, batch, agents.scale, want_lse=True)
            kept.append(torch.exp(part - whole).mean())
            x = x + 0.1 * torch.randn(x.shape, generator=agents.gen, device="cuda")
        print("turn %d: sequences of %s tokens, %d pages in use, the chosen blocks hold %.3f of the weight" %
              (turn, agents.lens, int((agents.pool.counts() > 0).sum()), torch.stack(kept).mean().item()), flush=True)
    share = torch.stack(kept).mean().item()
    agents.close()
    return share


if __name__ == "__main__":
    main()
