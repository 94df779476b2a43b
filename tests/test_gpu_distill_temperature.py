"""The distillation loss at temperatures far from 1 and with logits far from 0, where |z| / tau is large and what is asked is a difference of
two such numbers. The logits here are exact in float32 (two products of few bits, zeros otherwise), so that their own roundings, which
the temperature magnifies, stay out of the bounds."""
import math

import pytest
import torch

from gpu_util import say
from long_context_ref import HALF, U32, check
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
F64 = torch.float64


def inputs(T, V, K, tau, dtype, seed):
    """Logits of about 20 or -20 that differ by up to some 20 tau, multiples of 2^-18 (tau below 1e-5: most are 0 or far off); every
    fifth column far below; a teacher's values of the same kind."""
    g = torch.Generator().manual_seed(seed)
    ldw = (V + 63) // 64 * 64
    step = 2.0 ** -18 * 2.0 ** max(0, math.floor(math.log2(20 * tau / 255 * 2 ** 18))) if tau > 1e-6 else 2.0 ** -18
    W = torch.randn(64, ldw, generator=g)
    W[0] = 20.0
    W[0, ::5] = 10.0
    W[1] = torch.randint(0, 256, (ldw,), generator=g) * step
    h = torch.zeros(T, 64)
    h[:, 0], h[:, 1] = 1.0, 1.0
    h[1::4, 0] = -1.0
    values = 8.0 + torch.randint(0, 8, (T, K), generator=g) * (2.0 ** round(math.log2(tau)) if tau > 2.0 ** -20 else 2.0 ** -20)
    index = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int()
    targets = torch.randint(0, V, (T,), generator=g, dtype=torch.int32)
    return dict(h=h.to(dtype).cuda(), W=W.to(dtype).cuda(), values=values.cuda(), index=index.cuda(), targets=targets.cuda())


def reference(t, V, tau, soft, hard, half):
    """In float64, with bounds. u = U32. A weight exp((z - max) / tau): a difference (exact or u), the rounded factor, a product and the
    exponential: (4 span + 8) u, span = (max - z) / tau. Their sum: V / 64 + 80 additions and rescalings. p: the exponent (span and the
    logarithm of the sum, 3 roundings each and the constants': 6) and the exponential. Nothing is in proportion to |z| / tau."""
    h, W, values = (t[k].double().cpu() for k in ("h", "W", "values"))
    index, y = t["index"].long().cpu(), t["targets"].long().cpu()
    T, K = index.shape
    z = h @ W[:, :V]
    assert torch.equal(z, z.float().double())
    m = z.amax(dim=1, keepdim=True)

    def soft_of(tau):
        span = (m - z) / tau
        e = torch.exp(-span)
        l = e.sum(dim=1, keepdim=True)
        p, ll = e / l, torch.log(l)
        e_l = (p * (4 * span + 8)).sum(dim=1, keepdim=True) * U32 + (V / 64 + 80) * U32
        # exponentials below the smallest normal number may be 0
        return span, ll, p, e_l, (6 * span + 6 * ll + 16) * U32 + e_l, p + 2.0 ** -125

    span, ll, p, e_l, e_p, _ = soft_of(tau)
    span1, ll1, p1, e_l1, e_p1, _ = soft_of(1.0)
    mv = values.amax(dim=1, keepdim=True)
    e = torch.exp((values - mv) / tau)
    q = e / e.sum(dim=1, keepdim=True)
    eq = (4 * (mv - values) / tau + 2 * K + 8) * U32
    logq = torch.log(torch.where(q > 0, q, 1.0))
    term = logq + span.gather(1, index) + ll
    e_term = 8 * U32 * (logq.abs() + span.gather(1, index) + ll) + e_l + 4 * U32
    tiny = q < 2.0 ** -120                           # may be left out
    kl = torch.where(tiny, 0.0, q * term).sum(dim=1)
    e_kl = (q * (eq * (term.abs() + 1) + e_term)).sum(dim=1) + (K + 8) * U32 * (q * term.abs()).sum(dim=1) + torch.where(tiny, q * term.abs(), 0.0).sum(dim=1)
    at = y[:, None]
    ce = (span1.gather(1, at) + ll1)[:, 0]
    e_ce = (e_l1 + 4 * U32 * (span1.gather(1, at) + ll1 + 1))[:, 0]
    w = 1.0 / T
    sums = torch.stack([kl.sum(), ce.sum()]) * w
    adds = (T / 1024 + 16) * U32
    e_sums = torch.stack([(e_kl + adds * kl.abs()).sum(), (e_ce + adds * ce).sum()]) * w
    factor = torch.tensor([soft * tau * tau, hard], dtype=F64)
    out = {"tokens": torch.stack([kl, ce]), "tokens_err": torch.stack([e_kl, e_ce]), "loss": torch.cat([(factor * sums).sum()[None], sums]),
           "loss_err": torch.cat([(factor * (e_sums + 5 * U32 * sums.abs())).sum()[None], e_sums])}
    Q = torch.zeros(T, V, dtype=F64).scatter_(1, index, q)
    EQ = torch.zeros(T, V, dtype=F64).scatter_(1, index, q * eq)
    hot = torch.zeros(T, V, dtype=F64).scatter_(1, at, 1.0)
    gs, gh = w * soft * tau, w * hard
    G = gs * (p - Q) + gh * (p1 - hot)
    eG = gs * (p * e_p + EQ + 2.0 ** -120) + gh * (p1 * e_p1 + 2.0 ** -120) + 8 * U32 * (gs * (p + Q) + gh * (p1 + hot)) + half * G.abs()
    Wv = W[:, :V]
    out["dh"] = G @ Wv.t()
    out["dh_err"] = eG @ Wv.abs().t() + (V + 2) * U32 * (G.abs() @ Wv.abs().t()) + half * out["dh"].abs()
    out["dW"], out["dW_err"] = torch.zeros_like(W), torch.zeros_like(W)
    out["dW"][:, :V] = h.t() @ G
    out["dW_err"][:, :V] = h.abs().t() @ eG + (T + 2) * U32 * (h.abs().t() @ G.abs()) + half * out["dW"][:, :V].abs()
    return out


@pytest.mark.parametrize("keep", [0, -1])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [100.0, 1.0, 1e-2, 1e-3, 1e-4, 1e-5, 1e-6, 1e-12, 1e-18])
def test_temperatures(tau, dtype, keep):
    for T, V, K in ((1, 65, 3), (70, 700, 9)):
        say(f"case tau {tau} {dtype} keep {keep} T {T}")
        t = inputs(T, V, K, tau, dtype, T)
        name = "f32" if dtype == torch.float32 else "bf16"
        for soft, hard in ((1.0, 0.0), (0.7, 0.3)):
            cfg = bpt.make_distill_config(T, 64, V, K, tau=tau, soft=soft, hard=hard, dtype=name, grad_dtype=name, keep_bytes=keep)
            d = bpt.DistillLoss(cfg)
            loss, tokens, saved = d.forward(t["h"], t["W"], t["values"], t["index"], t["targets"] if hard else None)
            dh, dW = d.backward(t["h"], t["W"], saved)
            ref = reference(t, V, cfg.tau, cfg.soft, cfg.hard, HALF[dtype])
            if not hard:
                ref["tokens"][1], ref["tokens_err"][1] = 0.0, 0.0
                ref["loss"][2], ref["loss_err"][2] = 0.0, 0.0
            for k, v in dict(tokens=tokens, loss=loss, dh=dh, dW=dW).items():
                check(v.cpu(), ref[k], ref[k + "_err"], k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_logits_formed_again_are_those_that_were_summed(dtype):
    """A gradient from logits that the forward kept and one from logits formed again, of blocks of other sizes: the same bits, so that a
    temperature magnifies nothing between the two."""
    g = torch.Generator(device="cuda").manual_seed(1)
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    for T, D, V, K in ((1, 64, 65, 3), (50, 512, 300, 9), (300, 1024, 2000, 20)):
        h, W = torch.randn(T, D, generator=g, device="cuda").to(dt), torch.randn(D, (V + 63) // 64 * 64, generator=g, device="cuda").to(dt)
        values, index = torch.randn(T, K, generator=g, device="cuda"), torch.randint(0, V, (T, K), generator=g, device="cuda", dtype=torch.int32)
        for tau in (1.0, 0.01, 1e-6):
            say(f"case formed again {dtype} {T} {D} {V} tau {tau}")
            out = []
            for keep, rows in ((-1, 0), (-1, 64), (64 * W.shape[1] * 4 if T > 64 else -1, 64)):      # the last: kept for the first block
                d = bpt.DistillLoss(bpt.make_distill_config(T, D, V, K, tau=tau, dtype=dtype, keep_bytes=keep, block_rows=rows))
                loss, tokens, saved = d.forward(h, W, values, index)
                out.append((loss, tokens, d.backward(h, W, saved)[0]))
            for o in out[1:]:
                assert all(bool(torch.isfinite(a).all()) for a in o)
                assert all(torch.equal(a, b) for a, b in zip(o, out[0])), tau


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,first,last", [(65, 64, 65), (200, 64, 128), (200, 0, 64), (5000, 4480, 4544), (300, 130, 131), (64, 0, 64)])
def test_a_nan_among_the_logits_reaches_losses_and_gradients(V, first, last, dtype):
    """Whole groups of 64 columns of NaN, a last group of one column, one column: in no list and no target, but in every sum."""
    say(f"case NaN in columns {first}..{last} of {V} {dtype}")
    T, K = 40, 5
    t = inputs(T, V, K, 1.0, torch.float32 if dtype == "f32" else torch.bfloat16, 1)
    t["W"][:, first:last] = math.nan
    t["index"].clamp_(max=V - 1)
    keep = [v for v in range(V) if not first <= v < last] or [0]
    t["index"][:], t["targets"][:] = keep[0], keep[-1]
    weights = torch.ones(T, device="cuda")
    weights[::3] = 0.0
    for hard, tau in ((0.0, 1.0), (0.5, 2.0)):
        d = bpt.DistillLoss(bpt.make_distill_config(T, 64, V, K, tau=tau, hard=hard, dtype=dtype))
        loss, tokens, saved = d.forward(t["h"], t["W"], t["values"], t["index"], t["targets"] if hard else None, weights)
        dh, _ = d.backward(t["h"], t["W"], saved)
        on = weights != 0
        assert bool(loss[:2].isnan().all()) and bool(tokens[0, on].isnan().all()) and bool(dh[on].isnan().all())
        assert bool((tokens[:, ~on] == 0).all())
        if hard:
            assert bool(loss[2].isnan()) and bool(tokens[1, on].isnan().all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_values_and_logits(dtype):
    """A value of +inf has no probability in a softmax: its token's kl and gradient are NaN, those of other tokens as without it. A logit of
    -inf has probability 0: a gradient of 0 where no list asks for it, an infinite kl where one does."""
    T, V, K = 12, 200, 5
    t = inputs(T, V, K, 1.0, torch.float32 if dtype == "f32" else torch.bfloat16, 2)
    t["index"][:] = torch.arange(10, 10 + K, device="cuda", dtype=torch.int32)
    d = bpt.DistillLoss(bpt.make_distill_config(T, 64, V, K, tau=1.5, dtype=dtype))

    def run(**kw):
        a = {**t, **kw}
        loss, tokens, saved = d.forward(a["h"], a["W"], a["values"], a["index"])
        return (tokens[0].clone(), *d.backward(a["h"], a["W"], saved))

    ref = run()
    values = t["values"].clone()
    values[3, 2] = math.inf
    kl, dh, _ = run(values=values)
    rest = torch.arange(T, device="cuda") != 3
    assert bool(kl[3].isnan()) and bool(dh[3].isnan().all()) and torch.equal(kl[rest], ref[0][rest]) and torch.equal(dh[rest], ref[1][rest])
    h, W = t["h"].clone(), t["W"].clone()
    h[:], h[:, 2] = 0.0, 1.0                         # the logits are row 2 of W
    W[2] = 0.5
    W[2, 100] = -math.inf
    loss, tokens, saved = d.forward(h, W, t["values"], t["index"])
    want = math.log(V - 1)                           # the others have 1 / (V - 1) each
    q = torch.softmax(t["values"].double().cpu() / 1.5, dim=1)
    kl = (q * torch.log(q)).sum(dim=1) + want
    # K terms of some units, a sum of V / 64 + 80 parts, its logarithm
    check(tokens[0].cpu(), kl, (V / 64 + 120) * U32 * (1 + want) + 20 * K * U32 * (1 + kl.abs()), "kl")
    _, dW = d.backward(h, W, saved)
    assert bool((dW[:, 100] == 0).all()) and bool(torch.isfinite(dW).all())
    t["index"][5, 1] = 100
    _, tokens, _ = d.forward(h, W, t["values"], t["index"])
    assert float(tokens[0, 5]) == math.inf and bool(torch.isfinite(tokens[0, :5]).all())
