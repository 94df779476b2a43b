"""The layer with rotary positions and windowed attention, and a GPT training step with both and 8-bit AdamW moments,
against float64 autograd of the same formulas (torch, CPU)."""
import math

import pytest
import torch

from bpt_inputs import make_inputs, small_workload
from gpu_util import bf16_limits, say
from long_context_ref import rope, rope_freqs, visible
from paper_2305_19370_amd import bpt
from paper_2305_19370_amd.gpt import GPT, GPTShape

pytestmark = pytest.mark.gpu
NAMES = ("Wq", "Wk", "Wv", "Wo", "W1", "W2", "ln1_g", "ln1_b", "ln2_g", "ln2_b", "b1", "b2")


class Rounded(torch.autograd.Function):
    """x, rounded to bf16 where `value`; its gradient rounded where `grad`."""

    @staticmethod
    def forward(ctx, x, value, grad):
        ctx.grad = grad
        return x.bfloat16().double() if value else x.clone()

    @staticmethod
    def backward(ctx, g):
        return (g.bfloat16().double() if ctx.grad else g), None, None


def exactly(x, value=True, grad=False):
    return x


def rounded(x, value=True, grad=False):
    return Rounded.apply(x, value, grad)


def attend(q, k, v, causal, window, sinks, R):
    ok = visible(q.shape[0], k.shape[0], q.shape[0], k.shape[0], causal, window, sinks)
    s = R(torch.einsum("qhd,khd->hqk", q, k) / math.sqrt(q.shape[2]), False, True)
    return torch.einsum("hqk,khd->qhd", R(torch.softmax(torch.where(ok[None], s, -math.inf), dim=-1)), v)


def layer(X, p, H, causal=True, window=0, sinks=0, turn=None, R=exactly):
    """One layer of the framework's formula on X [B, S, D], float64; turn(x [S, H, dh]) or None. R rounds where the bf16
    kernels do: the operands of matrix products, on the way forward and of gradients on the way back."""
    B, S, D = X.shape
    ln = lambda x, g, b: torch.nn.functional.layer_norm(x, (D,), g, b, 1e-5)  # noqa: E731
    u = R(ln(X, p["ln1_g"], p["ln1_b"]))
    q, k, v = (R((u @ p[n]).view(B, S, H, D // H), True, True) for n in ("Wq", "Wk", "Wv"))
    o = []
    for b in range(B):
        qb, kb = (R(turn(q[b]), True, True), R(turn(k[b]), True, True)) if turn else (q[b], k[b])
        o.append(attend(qb, kb, v[b], causal, window, sinks, R).reshape(S, D))
    h = X + R(R(torch.stack(o), True, True) @ p["Wo"], False, True)
    z = R(R(ln(h, p["ln2_g"], p["ln2_b"])) @ p["W1"] + p["b1"], False, True)
    return h + R(torch.nn.functional.gelu(z)) @ p["W2"] + p["b2"]


def turner(S, dh, kw):
    f = rope_freqs(kw["rot"], kw.get("theta", 1e4), kw.get("scaling", "none"), kw.get("factor", 1.0), kw.get("orig_len", 0))
    pos = kw.get("pos0", 0) + torch.arange(S)
    half = kw["rot"] // 2
    ang = pos.double()[:, None] * f[None]
    c, s = (kw.get("mscale", 1.0) * t(ang)[:, None, :] for t in (torch.cos, torch.sin))

    def turn(x):
        i = torch.arange(2 * half)
        a, b = (i[:half], i[half:]) if kw.get("layout", "half") == "half" else (i[0::2], i[1::2])
        y = x.clone()
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        return y
    # the reference's own rotation agrees with the tests' complex-free one
    z = torch.randn(S, 1, dh, dtype=torch.float64)
    assert torch.allclose(turn(z), rope(z, pos, f, kw.get("layout", "half"), kw.get("mscale", 1.0)))
    return turn


def errors(got, ref):
    d, rms = (got.double().cpu() - ref).abs(), float(ref.square().mean().sqrt()) or 1.0
    return float(d.max()) / rms, float(d.mean()) / rms


CASES = [
    dict(B=2, S=300, H=4, opt=dict(window=50, sinks=3)),
    dict(B=1, S=333, H=4, opt=dict(rot=64)),
    dict(B=2, S=200, H=2, opt=dict(rot=32, layout="interleaved", pos0=1000, mscale=1.1)),
    dict(B=1, S=1300, H=2, opt=dict(rot=128, scaling="by_parts", factor=4.0, orig_len=256, window=100, sinks=40)),
    dict(B=1, S=150, H=4, causal=False, opt=dict(rot=64, layout="interleaved", window=20, sinks=2)),
    dict(B=3, S=700, H=4, opt=dict(rot=64, window=130, sinks=2)),            # more rows than the forward for few takes
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_layer_with_options(case, dtype):
    """Y, dX and every gradient. fp32: max|diff| <= 1e-4 rms, the layer's bound. bf16: the gate of the
    layer's parity tests (gpu_util.bf16_limits) over the rounding model of the layer with these options. (The layer without
    options is no yardstick: it averages over all keys, n = 150 of the last case, where a window leaves 20 to 41: errors of the
    attention's part fall as 1 / sqrt(n), here by up to sqrt(150 / 22) = 2.6.)"""
    c = CASES[case]
    causal, H, opt = c.get("causal", True), c["H"], c["opt"]
    w = small_workload(dtype, B=c["B"], S=c["S"], D=256, H=H, F=512, causal=causal, Bq=64, Bkv=64)
    say(f"case layer options {c} {dtype}")
    inp = make_inputs(w, seed=case, affine=True, biases=True)
    dev = {k: v.cuda() for k, v in inp.items()}
    cfg = bpt.make_config(w.B, w.S, w.D, H, w.F, 64, 64, causal, dtype, "f32")

    def run(options):
        lay = bpt.Layer(cfg, options=options)
        Y, saved = lay.forward(dev["X"], dev)
        dX, g = lay.backward(dev["X"], dev, saved, dev["dY"])
        torch.cuda.synchronize()
        return {"Y": Y, "dX": dX, **g}

    def reference(**kw):
        p = {k: inp[k].double().requires_grad_() for k in NAMES}
        X = inp["X"].double().requires_grad_()
        Y = layer(X, p, H, causal, **kw)
        Y.backward(inp["dY"].double())
        return {"Y": Y.detach(), "dX": X.grad, **{"d" + k: p[k].grad for k in NAMES}}

    got = run(bpt.make_layer_options(**opt))
    ref = reference(window=opt.get("window", 0), sinks=opt.get("sinks", 0),
                    turn=turner(w.S, w.D // H, opt) if opt.get("rot") else None)
    model = reference(window=opt.get("window", 0), sinks=opt.get("sinks", 0),
                      turn=turner(w.S, w.D // H, opt) if opt.get("rot") else None, R=rounded) if dtype == "bf16" else None
    bad = []
    for n, r in ref.items():
        e_max, e_mean = errors(got[n], r)
        if model:
            m_max, m_mean = errors(model[n], r)
            lim = bf16_limits({"e_max": m_max, "e_mean": m_mean})
        else:
            lim = 1e-4, 1e-4
        print(f"{n}: {e_max:.2e} <= {lim[0]:.2e}, {e_mean:.2e} <= {lim[1]:.2e}", flush=True)
        if not (e_max <= lim[0] and e_mean <= lim[1]):
            bad.append((n, e_max, e_mean, lim))
    assert not bad, bad


def test_empty_options_are_the_layer():
    w = small_workload("bf16", B=2, S=200, D=256, H=2, F=512, causal=True, Bq=64, Bkv=64)
    inp = make_inputs(w, seed=3, affine=True, biases=True)
    dev = {k: v.cuda() for k, v in inp.items()}
    cfg = bpt.make_config(w.B, w.S, w.D, w.H, w.F, 64, 64, True, "bf16")
    out = []
    for o in (None, bpt.make_layer_options()):
        lay = bpt.Layer(cfg, options=o)
        Y, saved = lay.forward(dev["X"], dev)
        dX, g = lay.backward(dev["X"], dev, saved, dev["dY"])
        out.append((Y, dX, *g.values()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*out))


GPT_KW = dict(L=2, B=2, S=300, D=256, H=4, F=512, V=500, Bq=64, Bkv=64, pos_table=False, rope="half", window=60, sinks=4,
              opt_bits=8)


def test_gpt_step_f32():
    """Loss and every gradient of a GPT with rotary positions and a window, fp32, within 1e-4 rms of float64 autograd; then one
    AdamW step with 8-bit moments: p within a step of its formula."""
    s = GPTShape(dtype="f32", **GPT_KW)
    m = GPT(s, seed=1)
    g = torch.Generator().manual_seed(2)
    tok, tgt = (torch.randint(0, s.V, (s.B * s.S,), generator=g, dtype=torch.int32) for _ in range(2))
    # gains and biases of their own
    for n in m.nodecay.index:
        m.master(n).add_(0.1 * torch.randn(m.master(n).shape, generator=g).cuda())
    P = {n: m.master(n).double().cpu().requires_grad_() for n in m.names()}
    x = P["Wte"][tok.long()].view(s.B, s.S, s.D)
    turn = turner(s.S, s.D // s.H, dict(rot=s.D // s.H))
    for l in range(s.L):
        x = layer(x, {k: P[f"{l}.{k}"] for k in NAMES}, s.H, True, s.window, s.sinks, turn)
    h = torch.nn.functional.layer_norm(x, (s.D,), P["lnf_g"], P["lnf_b"], 1e-5)
    loss = torch.nn.functional.cross_entropy((h @ P["Wout"][:, :s.V]).view(-1, s.V), tgt.long())
    loss.backward()
    got = m.forward(tok.cuda(), tgt.cuda())
    m.backward(tok.cuda(), tgt.cuda())
    torch.cuda.synchronize()
    assert abs(float(got) - float(loss.detach())) <= 1e-5 * float(loss.detach())
    for n in m.names():
        r = P[n].grad
        e_max, _ = errors(m.grad(n), r)
        assert e_max <= 1e-4, (n, e_max)
    before, grad = {n: m.master(n).double().cpu() for n in m.names()}, {n: m.grad(n).double().cpu() for n in m.names()}
    m.optimizer_step(1e-3, weight_decay=0.1)
    torch.cuda.synchronize()
    for n in m.names():
        # the first step from zero moments: m / (1 - b1) = g, sqrt(v / (1 - b2)) = |g|
        wd = 0.1 if n in m.decay.index else 0.0
        want = before[n] * (1 - 1e-3 * wd) - 1e-3 * grad[n] / (grad[n].abs() + 1e-8)
        assert float((m.master(n).double().cpu() - want).abs().max()) <= 1e-3 * 1e-5 + 2e-7 * float(before[n].abs().max()) + 1e-9, n


def test_gpt_bf16_trains_and_replays():
    """A bf16 step of the same model runs, is finite, repeats bit for bit, and its optimiser step replays from a graph."""
    s = GPTShape(dtype="bf16", **GPT_KW)
    g = torch.Generator().manual_seed(2)
    tok, tgt = (torch.randint(0, s.V, (s.B * s.S,), generator=g, dtype=torch.int32).cuda() for _ in range(2))
    runs = []
    for _ in range(2):
        m = GPT(s, seed=1)
        for step in range(3):
            loss = m.train_step(tok, tgt, 1e-3)
        torch.cuda.synchronize()
        assert math.isfinite(float(loss))
        runs.append([t.clone() for grp in (m.decay, m.nodecay) for t in (grp.p, grp.m, grp.r, grp.exps)])
    assert all(torch.equal(a, b) for a, b in zip(*runs))
    graph = torch.cuda.CUDAGraph()
    m.forward(tok, tgt)
    m.backward(tok, tgt)
    torch.cuda.synchronize()
    ref = m.loss.clone(), m.decay.g.clone(), m.nodecay.g.clone()
    with torch.cuda.graph(graph):
        m.forward(tok, tgt)
        m.backward(tok, tgt)
    for _ in range(3):
        m.decay.g.fill_(math.nan)
        m.nodecay.g.fill_(math.nan)
        m.decay.g.zero_()
        m.nodecay.g.zero_()
        torch.randn(1000, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(m.loss, ref[0]) and torch.equal(m.decay.g, ref[1]) and torch.equal(m.nodecay.g, ref[2])
