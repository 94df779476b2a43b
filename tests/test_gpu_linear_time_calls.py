"""Calls of the recurrence and the distillation loss in an order, layout or setting of their own, on the GPU."""
import pytest
import torch

from gpu_util import say
from paper_2305_19370_amd import bpt
from paper_2305_19370_amd.gpt import GPT, GPTShape
from test_linear_time_calls import BROADCAST

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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", BROADCAST)
def test_a_broadcast_gradient(name, dtype):
    """The gradient of a mean or a sum, expanded over steps or sequences: what its dense copy gives."""
    for B, S in ((3, 140), (2, 1), (1, 70)):
        say(f"case broadcast dy {name} {B} {S}")
        g = torch.Generator(device="cuda").manual_seed(S)
        rn = lambda *n: torch.randn(*n, generator=g, device="cuda")  # noqa: E731
        x, r, i = (rn(B, S, 72).to(dtype) for _ in range(3))
        lam, rec, part = rn(72), bpt.GatedRecurrence(), BROADCAST[name](B, S, 72, dtype)
        dy = torch.randn(part.untyped_storage().nbytes() // part.element_size(), generator=g, device="cuda").to(dtype).as_strided(part.shape, part.stride())
        _, _, saved = rec.forward(x, r, i, lam, save=True)
        got, ref = (rec.backward(x, r, i, lam, saved, d) for d in (dy, dy.contiguous().clone()))
        for k in ref:
            assert torch.equal(got[k], ref[k]), k


@pytest.mark.parametrize("S", [1, 140])
def test_inputs_off_16_bytes(S):
    """Views that start anywhere: what aligned copies give, forward and backward."""
    B, D = 3, 72
    g = torch.Generator(device="cuda").manual_seed(S)
    v = [torch.randn(B, S, D, generator=g, device="cuda").bfloat16() for _ in range(4)]
    lam, rec = torch.randn(D, generator=g, device="cuda"), bpt.GatedRecurrence()

    def run(x, r, i, dy):
        y, hT, saved = rec.forward(x, r, i, lam, save=True)
        return dict(rec.backward(x, r, i, lam, saved, dy), y=y, hT=hT)

    ref = run(*v)
    for k in range(4):
        for first in (1, 4):
            say(f"case input {k} off by {first} elements")
            odd = torch.empty(B * S * D + first, dtype=torch.bfloat16, device="cuda")[first:].view(B, S, D)
            got = run(*(odd.copy_(t) if n == k else t for n, t in enumerate(v)))
            assert all(torch.equal(got[n], ref[n]) for n in ref)
