"""Greedy verification among the kernels that write its inputs: drafts, boundaries and lengths rewritten by kernels directly in front of it, in one graph
with several steps, replayed without waiting in between."""
import pytest
import torch

from paper_2609_07306_b200.verify import verify_drafts

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("batch,vocab", [(1, 40), (96, 1000)])
def test_greedy_steps_in_a_graph(batch, vocab):
    """Each step takes its drafts, its sequences' boundaries and its lengths from the step before; all are the same memory throughout."""
    drafts, steps, replays = 5, 12, 20
    rows = drafts + 1
    T = batch * rows
    g = torch.Generator(device="cuda").manual_seed(vocab)
    scores = torch.randn((T, vocab), generator=g, device="cuda")
    best = scores.argmax(1).int()
    right = torch.randint(0, rows, (steps, batch), generator=g, device="cuda", dtype=torch.int32)      # drafts that are right, by step
    begin, count = torch.arange(0, T, rows, device="cuda").int(), torch.randint(1, rows + 1, (steps, batch), generator=g, device="cuda", dtype=torch.int32)
    at = torch.arange(T, device="cuda").int()
    tokens, cu, lens, new = torch.zeros(T, dtype=torch.int32, device="cuda"), ints([0] * (batch + 1)), ints([0] * batch), ints([0] * batch)
    kept = torch.zeros((steps, batch), dtype=torch.int32, device="cuda")

    def step(s):
        cu[1:].copy_(count[s].cumsum(0))
        seq = torch.searchsorted(cu[1:], at, right=True).clamp_max(batch - 1)
        i = at - cu[seq]                                   # row of its sequence
        draft = torch.where(i <= right[s][seq], best.roll(1), (best.roll(1) + 1) % vocab)
        tokens.copy_(draft)
        lens.add_(kept[s - 1])                             # (something that the step before has written)
        _, accepted = verify_drafts(scores, tokens, cu, lens=lens, new_lens=lens)
        kept[s].copy_(accepted)

    for s in range(2):
        step(s)
    lens.zero_()
    kept.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for s in range(steps):
            step(s)
    for _ in range(replays):
        graph.replay()
    want = torch.minimum(right, count - 1)                 # accepted drafts: as many as are right, and there
    assert torch.equal(kept, want)
    grown = (want.sum(0) * 2 + steps) * replays - want[-1]  # a step's accepted drafts and one more, and the accepted ones of the step before
    assert torch.equal(lens, grown.int())
