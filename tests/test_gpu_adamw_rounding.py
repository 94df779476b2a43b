"""AdamW over a list of tensors on the GPU, bit for bit: with 32-bit moments every operation of the formula rounds once, in the
order it is written in, and the 8-bit moments' bytes follow their definition exactly, over many steps."""
import pytest
import torch

from gpu_util import say
from paper_2305_19370_amd import bpt
from perf import operators as plain

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


def f32(x):
    """A float64 result of two fp32 numbers' sum, product, quotient or of a root: to fp32 (53 bits are enough for the second
    rounding to change nothing)."""
    return x.float().double()


def const(x):
    return torch.tensor(x, dtype=torch.float64, device="cuda").float().double()


def formula(p, g, m, v, wd, step):
    """p, m and v after a step: fp32 operations, constants formed in 64 bits and rounded."""
    b1, b2, lr, eps = HP["beta1"], HP["beta2"], HP["lr"], HP["eps"]
    p, g, m, v = (x.double() for x in (p, g, m, v))
    m = f32(f32(const(b1) * m) + f32(const(1 - b1) * g))
    v = f32(f32(const(b2) * v) + f32(const(1 - b2) * f32(g * g)))
    den = f32(f32(torch.sqrt(f32(v * const(1 / (1 - b2 ** step))))) + const(eps))
    up = f32(f32(const(lr) * f32(m * const(1 / (1 - b1 ** step)))) / den)
    return f32(f32(p * const(1 - lr * wd)) - up).float(), m.float(), v.float()


def test_8_bit_moments_byte_for_byte():
    """61 tensors (more than a launch takes) of 4.5 million elements, 60 steps of new gradients: every byte of m, r and the
    exponents is that of the plain form, elementary torch operations on the same state. A root that is a step of fp32 off changes
    a code where the carry of the random bits hangs on it, about one in 7 million per step."""
    case = dict(plain.ADAMW, tensors="layers", L=5, D=264, F=1055, V=1001, bits=8)
    a, b = (plain.prepare(case, 3) for _ in range(2))
    plan = plain._plan(b)
    n = a["g"].numel()
    assert len(plan.tensors) > 48 and n > 4_000_000
    say(f"case {len(plan.tensors)} tensors, {n} elements")
    real = (a["p"] != 0).float()
    gen = torch.Generator(device="cuda").manual_seed(9)
    for step in range(1, 61):
        size = torch.exp(torch.randn(n // 256, 1, generator=gen, device="cuda")) * 10.0 ** (step % 3 - 3)
        if step % 7 == 0:
            size[::5] = 0.0                          # blocks whose moments only decay
        if step % 11 == 0:
            size[1::9] = 1e-21                       # squares below fp32's normal numbers
        g = (torch.randn(n // 256, 256, generator=gen, device="cuda") * size).view(-1) * real
        for s in (a, b):
            s["g"].copy_(g)
            s["step"] = step
        plain._run_adamw(a)
        bpt.adamw_multi(plan, step, plain.LR, plain.B1, plain.B2, plain.EPS, seed=plain.SEED)
        torch.cuda.synchronize()
        for k in ("m", "r", "exps"):
            assert torch.equal(a[k], b[k]), (step, k, int((a[k] != b[k]).sum()))


def test_tiny_second_moments_byte_for_byte():
    """Gradients whose squares are below fp32's normal numbers, from zero moments."""
    case = dict(plain.ADAMW, tensors="vectors", L=1, D=520, F=2083, V=0, bits=8)
    a, b = (plain.prepare(case, 5) for _ in range(2))
    plan = plain._plan(b)
    n = a["g"].numel()
    real = (a["p"] != 0).float()
    for s in (a, b):
        for k in ("m", "r", "exps"):
            s[k].zero_()
    for step in range(1, 21):
        g = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(step), device="cuda") * real * 3e-21
        for s in (a, b):
            s["g"].copy_(g)
            s["step"] = step
        plain._run_adamw(a)
        bpt.adamw_multi(plan, step, plain.LR, plain.B1, plain.B2, plain.EPS, seed=plain.SEED)
        torch.cuda.synchronize()
        for k in ("m", "r", "exps"):
            assert torch.equal(a[k], b[k]), (step, k, int((a[k] != b[k]).sum()))


def test_moments_of_every_size_byte_for_byte():
    """Blocks from 1e-22 to 1e17, within a block elements from 1e-8 of the largest up, and zeros: m from its least block scale on, r
    from squares below fp32's normal numbers to near its largest."""
    case = dict(plain.ADAMW, tensors="layers", L=1, D=264, F=1055, V=501, bits=8)
    a, b = (plain.prepare(case, 7) for _ in range(2))
    plan = plain._plan(b)
    n = a["g"].numel()
    real = (a["p"] != 0).float()
    for s in (a, b):
        for k in ("m", "r", "exps"):
            s[k].zero_()
    gen = torch.Generator(device="cuda").manual_seed(2)
    u = lambda *s: torch.rand(*s, generator=gen, device="cuda")  # noqa: E731
    for step in range(1, 13):
        size = 10.0 ** (39.0 * u(n // 256, 1) - 22.0) * 10.0 ** (-8.0 * u(n // 256, 256)) * (u(n // 256, 256) > 0.1)
        g = (torch.randn(n // 256, 256, generator=gen, device="cuda") * size).view(-1) * real
        for s in (a, b):
            s["g"].copy_(g)
            s["step"] = step
        plain._run_adamw(a)
        bpt.adamw_multi(plan, step, plain.LR, plain.B1, plain.B2, plain.EPS, seed=plain.SEED)
        torch.cuda.synchronize()
        for k in ("m", "r", "exps"):
            assert torch.equal(a[k], b[k]), (step, k, int((a[k] != b[k]).sum()))
        assert bool(torch.isfinite(b["p"]).all())


def make(sizes, bits, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda n, s: torch.randn(n, generator=g, device="cuda") * s  # noqa: E731
    out = []
    for j, n in enumerate(sizes):
        t = dict(p=rn(n, 0.1), g=rn(n, 0.01), weight_decay=0.1 * (j % 3), p_lowp=torch.empty(n, dtype=torch.bfloat16, device="cuda"))
        if bits == 32:
            t.update(m=rn(n, 0.01), v=rn(n, 0.01).square())
        else:
            t.update(m=torch.zeros(n, dtype=torch.uint8, device="cuda"), r=torch.zeros(n, dtype=torch.uint8, device="cuda"),
                     exps=torch.zeros((n + 255) // 256, 2, dtype=torch.uint8, device="cuda"))
        out.append(t)
    return out


@pytest.mark.parametrize("step", [1, 7, 5000])
def test_32_bit_step_rounds_as_written(step):
    """p, m and v of every element of 130 tensors (three launches, some tensors empty): the formula's operations, each rounded
    once, so that a tensor's place in the list changes nothing either."""
    sizes = [(7 * j) % 600 for j in range(129)] + [300001]
    ts = make(sizes, 32, step)
    want = [formula(t["p"], t["g"], t["m"], t["v"], t["weight_decay"], step) for t in ts]
    bpt.adamw_multi(bpt.AdamWTensors(ts, bits=32), step, **HP)
    torch.cuda.synchronize()
    for j, (t, w) in enumerate(zip(ts, want)):
        for k, x in zip(("p", "m", "v"), w):
            assert torch.equal(t[k], x), (j, k, int((t[k] != x).sum()), t[k].numel())
        assert torch.equal(t["p_lowp"], t["p"].bfloat16())


def test_8_bit_step_updates_p():
    """The parameters of 130 tensors after a step from zero 8-bit moments, against 64 bits. The update is off by half a step for each
    of: c1, m c1, lr, lr (m c1), r, the constant root of c2, their product, eps and the sum (each at most), and the quotient, and by what m
    (three roundings of (1 - b1) g) and r (half of four of (1 - b2) g^2) are off by: 10 + 3 + 2 half steps. p is off by half a step for
    the decay, its product and the difference."""
    sizes = [(7 * j) % 600 for j in range(129)] + [300001]
    ts = make(sizes, 8, 4)
    old = [t["p"].double() for t in ts]
    bpt.adamw_multi(bpt.AdamWTensors(ts, bits=8), 1, seed=4, **HP)
    torch.cuda.synchronize()
    for j, (t, p) in enumerate(zip(ts, old)):
        g = t["g"].double()
        up = HP["lr"] * g / (g.abs() + HP["eps"])    # m / (1 - b1) = g, v / (1 - b2) = g^2
        want = p * (1 - HP["lr"] * t["weight_decay"]) - up
        lim = 2.0 ** -24 * (3 * p.abs() + 15 * up.abs()) * 1.001
        assert bool(((t["p"].double() - want).abs() <= lim).all()), j


@pytest.mark.parametrize("bits", [8, 32])
def test_gradients_without_a_square(bits):
    """Finite gradients whose squares are not: their elements' update is zero, the others' what it is without them; a gradient
    that is not a number leaves only its own block's 8-bit moments (32 bits: its own element) without meaning."""
    n = 1000
    a, b = (make([n], bits, 6)[0] for _ in range(2))
    if bits == 32:
        for t in (a, b):
            t["m"].zero_(), t["v"].zero_()
    b["g"][[5, 700]] = 1e25
    p = b["p"].clone()
    for t in (a, b):
        bpt.adamw_multi(bpt.AdamWTensors([dict(t, weight_decay=0.0)], bits=bits), 1, seed=1, **HP)
    torch.cuda.synchronize()
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[[5, 700]] = False
    assert bool(torch.isfinite(b["p"]).all()) and torch.equal(b["p"][~rest], p[~rest])
    assert bool(((a["p"] - b["p"])[rest].abs() <= 2.0 ** -22 * a["p"][rest].abs() + 2.0 ** -20 * HP["lr"]).all())
    c = make([n], bits, 6)[0]
    c["g"][300] = float("nan")
    bpt.adamw_multi(bpt.AdamWTensors([c], bits=bits), 1, seed=1, **HP)
    torch.cuda.synchronize()
    assert torch.equal(torch.isnan(c["p"]).nonzero().view(-1).cpu(), torch.tensor([300]))
    if bits == 8:
        assert int(c["m"][300]) & 127 == 127 and int(c["r"][300]) == 127
