"""Rotary positions on the GPU against float64. Each result is one fp32 expression of two products rounded to the
type: |error| <= half a step of the result + (angle and cosine errors, a few 2^-24) of |a| + |b|."""
import math

import pytest
import torch

from gpu_util import say
from long_context_ref import HALF, U32, check, rope, rope_freqs
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}

CASES = [
    # rows, S, H, dh, rot, layout, kw
    (1, 1, 1, 8, 2, "half", {}),
    (1, 1, 40, 128, 128, "half", {}),
    (7, 3, 5, 64, 64, "interleaved", {}),
    (333, 111, 12, 64, 64, "half", dict(scaling="linear", factor=4.0)),
    (1000, 250, 3, 128, 32, "half", dict(theta=500000.0)),
    (129, 129, 2, 128, 48, "interleaved", dict(scaling="base", factor=8.0)),
    (65, 65, 2, 72, 10, "half", dict(pos0=1000003)),
    (65, 13, 2, 72, 10, "interleaved", dict(mscale=1.3)),
    (4500, 4500, 4, 128, 128, "half", dict(scaling="by_parts", factor=16.0, orig_len=2048, mscale=1.1, pos0=-7)),
    (5001, 5001, 1, 128, 64, "interleaved", dict(scaling="by_parts", factor=2.0, orig_len=512)),
    (50, 50, 1, 256, 128, "half", {}),
]


def bound(x, y, mscale, half):
    """x, y float64 before and after; pairs mix at most |a| + |b|. Errors of the angle: a float32 fraction of a turn (2 pi
    2^-25), of the sine and cosine 2 steps, of mscale, two products and a sum 4 half steps."""
    n = x.shape[-1]
    s = (x.abs().amax(dim=-1, keepdim=True) * 2).expand(*x.shape[:-1], n)
    return half * y.abs() + mscale * (2 * math.pi / 2 + 8) * U32 * s


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c[:6])))
def test_forward_and_backward(case, dtype):
    rows, S, H, dh, rot, layout, kw = case
    say(f"case rope {case} {dtype}")
    g = torch.Generator(device="cuda").manual_seed(rows)
    pad = 16
    X = torch.randn(rows, H * dh + pad, generator=g, device="cuda").to(DT[dtype])
    cfg = bpt.make_rope_config(rows, S, H, dh, rot=rot, ldx=H * dh + pad, layout=layout, dtype=dtype, **kw)
    bpt._check(bpt.rope_validate(cfg))
    freqs = rope_freqs(rot, **{k: v for k, v in kw.items() if k not in ("pos0", "mscale")})
    ms, half = kw.get("mscale", 1.0), HALF[DT[dtype]]
    given = torch.randint(-2 ** 20, 2 ** 22, (rows,), generator=g, device="cuda", dtype=torch.int32)
    for pos in (None, given):
        at = (kw.get("pos0", 0) + torch.arange(rows) % S) if pos is None else pos.cpu().long()
        x = X[:, :H * dh].view(rows, H, dh).cpu()
        Y = torch.full((rows, H, dh), math.nan, dtype=DT[dtype], device="cuda")
        bpt.rope_fwd(cfg, X, Y, pos)
        torch.cuda.synchronize()
        ref = rope(x, at, freqs, layout, ms)
        err = bound(x.double(), ref, ms, half)
        err[..., rot:] = 0.0                         # copied
        check(Y.cpu(), ref, err, "Y")
        # backward: the transposed rotation; into a strided dX whose padding stays
        dX = torch.full_like(X, 7.0)
        bpt.rope_bwd(cfg, Y, dX, pos)
        torch.cuda.synchronize()
        dref = rope(Y.cpu(), at, freqs, layout, ms, sign=-1.0)
        derr = bound(Y.cpu().double(), dref, ms, half)
        derr[..., rot:] = 0.0
        check(dX[:, :H * dh].view(rows, H, dh).cpu(), dref, derr, "dX")
        assert bool((dX[:, H * dh:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout,rot", [("half", 64), ("interleaved", 64), ("half", 22), ("interleaved", 6)])
def test_in_place_is_the_same(layout, rot, dtype):
    rows, H, dh, ld = 75, 4, 64, 400
    X = torch.randn(rows, ld, device="cuda").to(DT[dtype])
    cfg = bpt.make_rope_config(rows, rows, H, dh, rot=rot, ldx=ld, ldy=ld, layout=layout, dtype=dtype)
    Y = torch.full_like(X, 3.0)
    bpt.rope_fwd(cfg, X, Y)
    Z = X.clone()
    bpt.rope_fwd(cfg, Z, Z)
    torch.cuda.synchronize()
    assert torch.equal(Z[:, :H * dh], Y[:, :H * dh])
    assert torch.equal(Z[:, H * dh:], X[:, H * dh:]) and bool((Y[:, H * dh:] == 3.0).all())


def test_gradient_is_the_transpose():
    """<R x, y> = <x, R^T y> in fp32: rope_bwd is the adjoint of rope_fwd (each side off by fp32 roundings of
    4096 terms of size ~1)."""
    rows, H, dh = 16, 2, 128
    cfg = bpt.make_rope_config(rows, rows, H, dh, rot=96, dtype="f32", mscale=1.7, pos0=12345)
    x, y = torch.randn(rows, H, dh, device="cuda"), torch.randn(rows, H, dh, device="cuda")
    Rx, Ry = torch.empty_like(x), torch.empty_like(x)
    bpt.rope_fwd(cfg, x, Rx)
    bpt.rope_bwd(cfg, y, Ry)
    a, b = float((Rx.double() * y.double()).sum()), float((x.double() * Ry.double()).sum())
    assert abs(a - b) <= 2 * 4096 * 16 * U32, (a, b)


def test_replays_from_a_graph():
    X = torch.randn(500, 4, 64, device="cuda").bfloat16()
    pos = torch.randint(0, 9999, (500,), device="cuda", dtype=torch.int32)
    Y = torch.empty_like(X)
    cfg = bpt.make_rope_config(500, 500, 4, 64)
    bpt.rope_fwd(cfg, X, Y, pos)
    ref = Y.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        bpt.rope_fwd(cfg, X, Y, pos)
    for _ in range(3):
        Y.fill_(math.nan)
        torch.randn(1000, device="cuda").sum().item()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, ref)
