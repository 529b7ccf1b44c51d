"""The example that uses memories and the key/value cache together runs, and what it computes is attention."""
import pytest
import torch

from paper_2602_21477_amd import binding as B
from paper_2602_21477_amd.context_example import Agents, main

pytestmark = pytest.mark.gpu


def test_the_example_runs(gpu_device):
    share = main(turns=1, words=4)
    assert 0.0 < share <= 1.0 + 1e-3


@pytest.mark.parametrize("storage", [B.PK_I8, B.PK_F8, B.PK_BF16])
def test_a_turn_with_all_blocks_is_full_attention(gpu_device, storage):
    agents = Agents(n_agents=3, passages=300, storage=storage, page=16)
    questions = torch.nn.functional.normalize(torch.randn(3, agents.d, generator=agents.gen, device="cuda"), dim=-1)
    ids = agents.recall(questions, k=4)
    exact = torch.stack([(p @ q).topk(4).indices.sort().values for p, q in zip(agents.passages, questions)])
    assert (ids.sort(-1).values == exact).float().mean() > 0.2  # (eight of 32 lists are probed)
    agents.read(ids, tokens_each=7)
    out, chosen, (q, batch) = agents.answer(questions, blocks=-(-max(agents.lens) // 16) + 1)
    for i, l in enumerate(agents.lens):
        assert chosen[i, 0].tolist()[:-(-l // 16)] == list(range(-(-l // 16)))
    full = agents.cache.attend(q, batch, agents.scale)
    # both are rounded once to bfloat16, and their weights once (8-bit codes: twice as finely)
    assert torch.allclose(out.float(), full.float(), rtol=2.0 ** -6, atol=2.0 ** -6)
    agents.close()
