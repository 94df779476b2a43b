"""WindowAttention on tensors as programs hold them: columns of one projection, head-major tensors, parts of a cache, an output
that is a view, an upstream gradient that is broadcast. Each gives the bits that contiguous tensors give."""
import pytest
import torch

from gpu_util import say
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
B, S, HQ, HKV, DH = 2, 210, 4, 2, 64


def rn(*shape, seed=0, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


def projection(dtype):
    x = rn(B, S, HQ + 2 * HKV, DH, dtype=dtype)
    return x[:, :, :HQ], x[:, :, HQ:HQ + HKV], x[:, :, HQ + HKV:]


def heads_first(dtype):
    return tuple(rn(B, h, S, DH, seed=h, dtype=dtype).transpose(1, 2) for h in (HQ, HKV, HKV))


def cache(dtype):
    k, v = rn(B, 5 * S, HKV, DH, seed=3, dtype=dtype), rn(B, 5 * S, HKV, DH, seed=4, dtype=dtype)
    return rn(B, S, HQ, DH, seed=5, dtype=dtype), k[:, 7:S + 7], v[:, :S]


def broadcast(dtype):
    return (rn(B, S, HQ, DH, seed=5, dtype=dtype), rn(B, S, 1, DH, seed=6, dtype=dtype).expand(B, S, HKV, DH),
            rn(1, S, HKV, DH, seed=7, dtype=dtype).expand(B, S, HKV, DH))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("make", [projection, heads_first, cache, broadcast])
def test_backward_of_views(make, dtype):
    say(f"case {make.__name__} {dtype}")
    q, k, v = make(dtype)
    do = rn(B, S, HQ, DH, seed=8, dtype=dtype)
    att = bpt.WindowAttention(window=40, sinks=3)
    dense = [t.contiguous() for t in (q, k, v)]
    o, lse = att.forward(*dense)
    want = att.backward(*dense, o, lse, do)
    o2, lse2 = att.forward(q, k, v)
    got = att.backward(q, k, v, o2, lse2, do)
    torch.cuda.synchronize()
    assert torch.equal(o2, o) and torch.equal(lse2, lse)
    for t, g, w in zip((q, k, v), got, want):
        assert g.shape == t.shape and g.dtype == t.dtype and torch.equal(g, w)
    if make in (projection, heads_first):            # no copies of the inputs
        assert all(g.stride() == t.stride() for g, t in zip(got, (q, k, v)))
    else:
        assert all(g.is_contiguous() for g in got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_output_and_upstream_gradient_of_other_strides(dtype):
    """O as columns of a wider tensor, dO dense, head-major or broadcast."""
    q, k, v = (t.contiguous() for t in projection(dtype))
    att = bpt.WindowAttention(window=40, sinks=3)
    o, lse = att.forward(q, k, v)
    wide = torch.full((B, S, HQ + 3, DH), float("nan"), dtype=dtype, device="cuda")
    wide[:, :, 2:2 + HQ] = o
    view = wide[:, :, 2:2 + HQ]
    ones = torch.ones(1, dtype=dtype, device="cuda").expand(B, S, HQ, DH)
    do = rn(B, S, HQ, DH, seed=8, dtype=dtype)
    cases = [(do, do), (do, do.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)), (ones.contiguous(), ones)]
    for dense, given in cases:
        want = att.backward(q, k, v, o, lse, dense)
        for out in (o, view):
            got = att.backward(q, k, v, out, lse, given)
            torch.cuda.synchronize()
            assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_one_token_with_strides_of_its_own():
    """A single token of a single sequence whose dimensions of one element show strides that are no multiple of 16 bytes."""
    k, v, q = rn(1, S, HKV, DH, seed=1), rn(1, S, HKV, DH, seed=2), rn(1, 1, HQ, DH, seed=3)
    att = bpt.WindowAttention(window=40, sinks=3)
    want, lse = att.forward(q, k, v)
    odd = q.as_strided(q.shape, (13, 7, DH, 1))
    got, lse2 = att.forward(odd, k.as_strided(k.shape, (3, HKV * DH, DH, 1)), v)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(lse, lse2)
