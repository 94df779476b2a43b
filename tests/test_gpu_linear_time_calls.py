"""Calls of the recurrence and the distillation loss in an order, layout or setting of their own, on the GPU."""
import pytest
import torch

from gpu_util import say
from paper_2305_19370_amd.gpt import GPT, GPTShape

pytestmark = pytest.mark.gpu
KW = dict(L=2, B=2, S=150, D=256, H=4, F=512, V=500, Bq=64, Bkv=64)


def lists(T, V, K, g):
    return torch.randn(T, K, generator=g).cuda() * 2, torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int().cuda()


def test_other_lists_between_the_replays_of_a_graph():
    """Passes captured with one length of the lists and targets, eager ones with other lengths, temperatures and no targets between the
    replays: every replay and every eager pass gives what it gives alone, and memory that others take meanwhile stays theirs."""
    say("case captured distillation, other configurations between")
    m = GPT(GPTShape(dtype="bf16", recurrent=True, pos_table=False, **KW), seed=1)
    g = torch.Generator().manual_seed(3)
    T = m.shape.B * m.shape.S
    tok, tgt = (torch.randint(0, 500, (T,), generator=g, dtype=torch.int32).cuda() for _ in range(2))
    calls = [dict(lists=lists(T, 500, 16, g), targets=tgt, tau=2.0, soft=0.8, hard=0.2), dict(lists=lists(T, 500, 7, g), tau=1.0),
             dict(lists=lists(T, 500, 256, g), targets=tgt, tau=1.5, soft=0.5, hard=0.5)]

    def passes(lists, **kw):
        loss = m.distill_forward(tok, *lists, **kw)
        m.distill_backward(tok)
        return loss

    def result(loss):
        torch.cuda.synchronize()
        return [t.clone() for t in (loss, m.decay.g, m.nodecay.g)]

    refs = [result(passes(**c)) for c in calls]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = passes(**calls[0])
    for k in (1, 2, 1):
        assert all(torch.equal(a, b) for a, b in zip(result(passes(**calls[k])), refs[k])), k
        others = [torch.full((1 << n,), 7, dtype=torch.uint8, device="cuda") for n in range(12, 25)]
        for t in (loss, m.decay.g, m.nodecay.g):
            t.zero_()
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(result(loss), refs[0])), k
        assert all(bool((t == 7).all()) for t in others), k
