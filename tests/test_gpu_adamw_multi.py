"""AdamW over a list of tensors on the GPU: 32-bit moments against the formula in float64 and against
bpt_adamw_step, 8-bit moments against their definition (codes, exponents, expectation of the rounding)."""
import math

import pytest
import torch

from gpu_util import say
from long_context_ref import U32, e4m3_values, moments
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu

SIZES = [1, 3, 255, 256, 257, 1000, 4096, 70001]
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


def tensors(sizes, bits, grad=torch.float32, low=torch.bfloat16, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda n, s: torch.randn(n, generator=g, device="cuda") * s  # noqa: E731
    out = []
    for j, n in enumerate(sizes):
        t = dict(p=rn(n, 0.1), g=rn(n, 0.01 * 10 ** (j % 4 - 2)).to(grad), weight_decay=0.1 * (j % 3),
                 p_lowp=torch.empty(n, dtype=low, device="cuda") if low is not None else None)
        if bits == 32:
            t.update(m=rn(n, 0.01), v=rn(n, 0.01).square())
        else:
            t.update(m=torch.zeros(n, dtype=torch.uint8, device="cuda"), r=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                     exps=torch.zeros((n + 255) // 256, 2, dtype=torch.uint8, device="cuda"))
        out.append(t)
    return out


def formula(p, g, m, v, wd, step):
    p, g, m, v = (x.double().cpu() for x in (p, g, m, v))
    m = HP["beta1"] * m + (1 - HP["beta1"]) * g
    v = HP["beta2"] * v + (1 - HP["beta2"]) * g * g
    up = HP["lr"] * (m / (1 - HP["beta1"] ** step)) / (torch.sqrt(v / (1 - HP["beta2"] ** step)) + HP["eps"])
    return p * (1 - HP["lr"] * wd) - up, m, v, up


def near(got, ref, lim, what):
    d = (got.double().cpu() - ref).abs()
    assert bool((d <= lim).all()), (what, float((d / lim).max()))


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("low", [torch.bfloat16, torch.float32, None])
def test_32_bit_moments(grad, low):
    ts = tensors(SIZES, 32, grad, low)
    refs = [formula(t["p"], t["g"], t["m"], t["v"], t["weight_decay"], 7) for t in ts]
    mags = [(t["m"].abs().double().cpu(), t["g"].abs().double().cpu()) for t in ts]
    bpt.adamw_multi(bpt.AdamWTensors(ts, bits=32), 7, **HP)
    torch.cuda.synchronize()
    for t, (p, m, v, up), (m0, g0) in zip(ts, refs, mags):
        # constants and each operation: half a step; the update takes 12 of them, two of a whole step
        em = 5 * U32 * (m0 + g0)
        near(t["m"], m, em + 1e-40, "m")
        near(t["v"], v, 6 * U32 * v + 1e-40, "v")
        scale = HP["lr"] / (1 - HP["beta1"] ** 7) / (torch.sqrt(v / (1 - HP["beta2"] ** 7)) + HP["eps"])
        near(t["p"], p, 3 * U32 * p.abs() + 2 * U32 * up.abs() + 20 * U32 * up.abs() + scale * em, "p")
        if low is not None:
            assert torch.equal(t["p_lowp"], t["p"].to(low))


def test_agrees_with_the_single_tensor_step():
    """The same formula in another order of roundings: within 16 half steps of p and of the update."""
    n = 5000
    a = tensors([n], 32)[0]
    b = {k: v.clone() if torch.is_tensor(v) else v for k, v in a.items()}
    old = a["p"].clone()
    bpt.adamw_multi(bpt.AdamWTensors([dict(a, weight_decay=0.1)], bits=32), 3, **HP)
    bpt.adamw_step(b["p"], b["g"], b["m"], b["v"], 3, weight_decay=0.1, p_lowp=b["p_lowp"], **HP)
    torch.cuda.synchronize()
    lim = 16 * U32 * (old.abs() + (b["p"] - old).abs() * 4 + 1e-3 * 4)
    assert bool(((a["p"] - b["p"]).abs() <= lim).all())


def neighbours(x):
    """The largest e4m3 value <= |x| and the smallest >= |x|, float64 (|x| <= 256)."""
    tab = e4m3_values()[:127]
    i = torch.searchsorted(tab, x.contiguous(), right=True) - 1
    lo = tab[i]
    hi = torch.where(lo == x, lo, tab[(i + 1).clamp_max(126)])
    return lo, hi


@pytest.mark.parametrize("grad", [torch.float32, torch.bfloat16])
def test_8_bit_moments(grad):
    """Five steps from zero moments: each step's p from the formula on the moments that the bytes stood for, each new
    code one of the two around the formula's value, the exponent that of the block's largest value."""
    ts = tensors(SIZES, 8, grad, seed=3)
    plan = bpt.AdamWTensors(ts, bits=8)
    for step in range(1, 6):
        for j, t in enumerate(ts):
            t["g"].copy_((torch.randn(t["g"].numel(), generator=torch.Generator().manual_seed(100 * step + j)) * 10.0 ** (-j)).to(grad))
        before = [(t["p"].clone(), moments(t["m"], t["exps"], 0, True), moments(t["r"], t["exps"], 1, False)) for t in ts]
        bpt.adamw_multi(plan, step, seed=77, **HP)
        torch.cuda.synchronize()
        for t, (p0, m0, r0) in zip(ts, before):
            p, m, v, up = formula(p0, t["g"], m0, r0 * r0, t["weight_decay"], step)
            near(t["p"], p, 3 * U32 * p.abs() + 30 * U32 * up.abs() + HP["lr"] * 1e-5, "p")
            r = torch.sqrt(v)
            for codes, x, col in ((t["m"], m.abs(), 0), (t["r"], r, 1)):
                e = t["exps"].cpu()[:, col].double()
                blocks = torch.nn.functional.pad(x, (0, -x.numel() % 256)).view(-1, 256)
                top = blocks.amax(dim=1) * torch.exp2(134.0 - e)
                assert bool(((top >= 128 * (1 - 1e-6)) & (top < 256 * (1 + 1e-6))).all())
                y = (blocks * torch.exp2(134.0 - e)[:, None]).reshape(-1)[:x.numel()]
                got = (moments(codes, t["exps"], col, col == 0).abs() * torch.exp2(134.0 - e.repeat_interleave(256)[:x.numel()]))
                lo, _ = neighbours((y * (1 - 1e-5)).clamp_max(256))
                _, hi = neighbours((y * (1 + 1e-5)).clamp_max(256))
                assert bool(((got >= lo) & (got <= hi)).all())
                if col == 1:
                    assert bool(((got > 0) | (x == 0)).all())


def test_rounding_follows_its_expectation():
    """A constant moment between two codes: the mean over 65536 elements lies within 6 deviations of it. And no value moves
    without a gradient's help upwards: zero gradients from zero moments stay zero."""
    n = 65536
    t = tensors([n], 8)[0]
    t["g"].fill_(1.0)
    plan = bpt.AdamWTensors([t], bits=8)
    bpt.adamw_multi(plan, 1, seed=5, **HP)
    torch.cuda.synchronize()
    for codes, col, want in ((t["m"], 0, 0.1), (t["r"], 1, math.sqrt(0.05))):
        x = moments(codes, t["exps"], col, True)
        lo, hi = float(x.min()), float(x.max())
        assert lo <= want <= hi and hi - lo <= want / 8
        f = (want - lo) / (hi - lo)
        sd = (hi - lo) * math.sqrt(f * (1 - f) / n)
        assert abs(float(x.mean()) - want) <= 6 * sd + want * 2.0 ** -16, (float(x.mean()), want)
    z = tensors([1000], 8)[0]
    z["g"].zero_()
    bpt.adamw_multi(bpt.AdamWTensors([z], bits=8), 1, seed=5, **HP)
    torch.cuda.synchronize()
    assert not bool(z["m"].any()) and not bool(z["r"].any())


def test_steps_repeat_and_seeds_differ():
    a, b, c = (tensors([3000], 8, seed=1)[0] for _ in range(3))
    for t, seed in ((a, 1), (b, 1), (c, 2)):
        bpt.adamw_multi(bpt.AdamWTensors([t], bits=8), 1, seed=seed, **HP)
    torch.cuda.synchronize()
    assert torch.equal(a["m"], b["m"]) and torch.equal(a["r"], b["r"]) and torch.equal(a["exps"], b["exps"])
    assert not torch.equal(a["m"], c["m"])


@pytest.mark.parametrize("bits", [8, 32])
def test_many_tensors_in_any_place(bits):
    """More tensors than one launch takes, some empty: each as on its own (32-bit: the same bits), and the bytes behind
    every tensor stay."""
    sizes = [(7 * j) % 600 for j in range(130)]
    ts = tensors(sizes, bits, seed=9)
    say(f"case {len(ts)} tensors, {bits} bits")
    guard = []
    for t in ts:
        for k in ("p", "g", "m", "v", "r", "p_lowp"):
            if t.get(k) is not None:
                buf = torch.full((t[k].numel() + 64,), 3, dtype=t[k].dtype, device="cuda")
                buf[:t[k].numel()] = t[k]
                t[k] = buf[:t[k].numel()]
                guard.append(buf)
    want = [formula(t["p"], t["g"], t["m"], t["v"], t["weight_decay"], 1) if bits == 32 else None for t in ts]
    bpt.adamw_multi(bpt.AdamWTensors(ts, bits=bits), 1, seed=4, **HP)
    torch.cuda.synchronize()
    for t, w in zip(ts, want):
        if w is not None and t["p"].numel():
            near(t["p"], w[0], 3 * U32 * w[0].abs() + 40 * U32 * (w[3].abs() + HP["lr"] * 50), "p")
        if bits == 8 and t["p"].numel():
            assert bool((t["exps"][:, 0] >= 27).all()) and bool(t["r"].all())
    for buf in guard:
        assert bool((buf[-64:] == 3).all())


@pytest.mark.parametrize("bits", [8, 32])
def test_replays_from_a_graph(bits):
    ts = tensors([1000, 77], bits, seed=2)
    first = [{k: v.clone() for k, v in t.items() if torch.is_tensor(v)} for t in ts]
    plan = bpt.AdamWTensors(ts, bits=bits)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        bpt.adamw_multi(plan, 2, seed=1, **HP)

    def start():
        for t, f in zip(ts, first):
            for k, v in f.items():
                t[k].copy_(v)

    start()
    bpt.adamw_multi(plan, 2, seed=1, **HP)
    torch.cuda.synchronize()
    ref = [{k: v.clone() for k, v in t.items() if torch.is_tensor(v)} for t in ts]
    for _ in range(3):
        start()
        torch.randn(100, device="cuda").sum().item()
        g.replay()
        torch.cuda.synchronize()
        for t, r in zip(ts, ref):
            assert all(torch.equal(t[k], v) for k, v in r.items())
