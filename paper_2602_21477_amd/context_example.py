"""Agents that remember, read what they remembered, and answer: the memory's search and the context's cache together.

    python -m paper_2602_21477_amd.context_example

Every agent has a memory of its own (an index of passage vectors) and a sequence of its own in one layer's key/value cache.
A turn is what an agent's serving loop does on the GPU:

  1. the agents' questions are searched, each in its agent's memory, in one call;
  2. the passages that were found become tokens, whose keys and values are appended to the agents' sequences (a chunk each, of
     another length for every agent) and which attend to all that is before them;
  3. the agents answer token by token: the new token's key and value are appended, its query picks the blocks of the context whose
     bounds promise the most, and attends to those alone.

A model's layers are stood in for by fixed random projections of the passages' vectors; nothing else is left out.
"""
from __future__ import annotations

import torch

from . import binding as B


class Agents:
    def __init__(self, n_agents=4, passages=2000, d=128, heads=4, group=4, head_dim=64, max_tokens=4096, page=32, storage=B.PK_I8, seed=0):
        gen = torch.Generator("cuda").manual_seed(seed)
        self.gen, self.n, self.d, self.heads, self.group, self.head_dim, self.page = gen, n_agents, d, heads, group, head_dim, page
        self.scale = head_dim ** -0.5
        # memories: passages, and centroids from a sample of them
        self.passages = torch.nn.functional.normalize(torch.randn(n_agents, passages, d, generator=gen, device="cuda"), dim=-1)
        self.memories = [B.Index(p[torch.randperm(passages, generator=gen, device="cuda")[:32]].contiguous(), p.contiguous()) for p in self.passages]
        # one layer's cache for all agents, its pages handed out as their sequences grow
        per_agent = max_tokens // page
        self.cache = B.KVCache(n_agents * per_agent, heads, head_dim, storage=storage, page_tokens=page)
        free = torch.randperm(n_agents * per_agent, generator=torch.Generator().manual_seed(seed), dtype=torch.int32)
        self.tables = free.view(n_agents, per_agent).cuda()  # (all of an agent's pages at once, for brevity: pages beyond its length are not touched)
        self.lens = [0] * n_agents
        self.max_tokens = max_tokens
        self.project = torch.randn(d, (group * heads + 2 * heads) * head_dim, generator=gen, device="cuda", dtype=torch.bfloat16) * 0.3

    def layer(self, x):
        """Queries, keys and values of tokens, as parts of one product's rows."""
        rows = (x.to(torch.bfloat16) @ self.project).view(x.shape[0], -1, self.head_dim)
        hq = self.heads * self.group
        return rows[:, :hq], rows[:, hq:hq + self.heads], rows[:, hq + self.heads:]

    def step(self, new):
        """The batch of a step in which agent i gets new[i] tokens."""
        self.lens = [l + m for l, m in zip(self.lens, new)]
        if max(self.lens) > self.max_tokens:
            raise ValueError(f"a sequence of {max(self.lens)} tokens, and room for {self.max_tokens}")
        offsets = torch.tensor([0] + list(new)).cumsum(0).to(torch.int32)
        return B.KVBatch(self.tables, offsets.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), sum(new), max(new), max(self.lens))

    def recall(self, questions, k=8, nprobe=8):
        """Ids of the passages nearest to every agent's question."""
        ids, _ = B.search_multi(self.memories, list(range(self.n + 1)), questions, k, nprobe)
        return ids

    def read(self, ids, tokens_each=24):
        """The found passages as tokens (agent i takes i more of each), appended and attended from."""
        new = [ids.shape[1] * (tokens_each + i) for i in range(self.n)]
        x = torch.cat([self.passages[i][ids[i]].repeat_interleave(tokens_each + i, 0) for i in range(self.n)])
        x = x + 0.2 * torch.randn(x.shape, generator=self.gen, device="cuda")
        q, k, v = self.layer(x)
        batch = self.step(new)
        self.cache.append(k, v, batch)
        return self.cache.attend(q, batch, self.scale)

    def answer(self, x, blocks=8):
        """One token of every agent: (output, blocks it attended to)."""
        q, k, v = self.layer(x)
        batch = self.step([1] * self.n)
        self.cache.append(k, v, batch)
        chosen = self.cache.select(q, batch, blocks)
        return self.cache.attend_blocks(q, chosen, batch, self.scale), chosen, (q, batch)

    def close(self):
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
        x = questions
        for _ in range(words):
            out, chosen, (q, batch) = agents.answer(x)
            _, part = agents.cache.attend_blocks(q, chosen, batch, agents.scale, want_lse=True)
            _, whole = agents.cache.attend(q, batch, agents.scale, want_lse=True)
            kept.append(torch.exp(part - whole).mean())
            x = x + 0.1 * torch.randn(x.shape, generator=agents.gen, device="cuda")
        print("turn %d: sequences of %s tokens, the chosen blocks hold %.3f of the weight" % (turn, agents.lens, torch.stack(kept).mean().item()), flush=True)
    share = torch.stack(kept).mean().item()
    agents.close()
    return share


if __name__ == "__main__":
    main()
