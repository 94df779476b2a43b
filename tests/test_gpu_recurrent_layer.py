"""The layer with a recurrence in place of attention, and GPT steps with it and the distillation loss, against float64 autograd of the
same formulas (torch, CPU)."""
import math

import pytest
import torch

from bpt_inputs import make_inputs, small_workload
from gpu_util import bf16_limits, say
from linear_time_ref import recur
from paper_2305_19370_amd import bpt
from paper_2305_19370_amd.gpt import GPT, GPTShape
from test_gpu_layer_options import NAMES, errors, exactly, layer as attention_layer, rounded

pytestmark = pytest.mark.gpu


def mix(x, r, i, lam, c, h):
    """The recurrence over [B, S, D], differentiable: (y, last state)."""
    l = -c * torch.nn.functional.softplus(lam) * torch.sigmoid(r)
    a, b = torch.exp(l), torch.sqrt(-torch.expm1(2 * l)) * torch.sigmoid(i) * x
    y = []
    for t in range(x.shape[1]):
        h = a[:, t] * h + b[:, t]
        y.append(h)
    return torch.stack(y, 1), h


def layer(X, p, h0=None, c=8.0, R=exactly):
    """One layer on X [B, S, D], float64; R rounds where the bf16 kernels do."""
    B, S, D = X.shape
    ln = lambda x, g, b: torch.nn.functional.layer_norm(x, (D,), g, b, 1e-5)  # noqa: E731
    u = R(ln(X, p["ln1_g"], p["ln1_b"]))
    x, r, i = (R(u @ p[n], True, True) for n in ("Wq", "Wk", "Wv"))
    o, hT = mix(x, r, i, p["lam"], c, torch.zeros(B, D, dtype=torch.float64) if h0 is None else h0)
    h = X + R(R(o, True, True) @ p["Wo"], False, True)
    z = R(R(ln(h, p["ln2_g"], p["ln2_b"])) @ p["W1"] + p["b1"], False, True)
    return h + R(torch.nn.functional.gelu(z)) @ p["W2"] + p["b2"], hT


def test_the_reference_is_the_recurrence():
    """This file's differentiable form and the step by step one agree."""
    g = torch.Generator().manual_seed(0)
    x, r, i, dy = (torch.randn(2, 30, 8, generator=g, dtype=torch.float64) for _ in range(4))
    lam, h0, dhT = (torch.randn(*n, generator=g, dtype=torch.float64) for n in ((8,), (2, 8), (2, 8)))
    v = [t.requires_grad_() for t in (x, r, i, lam, h0)]
    y, hT = mix(v[0], v[1], v[2], v[3], 8.0, v[4])
    ((y * dy).sum() + (hT * dhT).sum()).backward()
    ref = recur(x, r, i, lam, 8.0, h0, None, dy, dhT)
    for t, k in zip(v, ("dx", "dr", "di", "dlam", "dh0")):
        assert torch.allclose(t.grad, ref[k], rtol=1e-10, atol=1e-12), k
    assert torch.allclose(y, ref["y"]) and torch.allclose(hT, ref["hT"])


CASES = [dict(B=2, S=300, H=4, h0=True), dict(B=1, S=64, H=2, h0=False), dict(B=3, S=1, H=4, h0=True), dict(B=1, S=577, H=2, h0=True),
         dict(B=2, S=150, H=4, h0=False, Bq=32, group_blocks=1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_recurrent_layer(case, dtype):
    """Y, the last states, dX and every gradient. fp32: max|diff| <= 1e-4 rms, the layer's bound. bf16: the gate of the layer's
    parity tests over its rounding model."""
    c = dict(CASES[case])
    say(f"case recurrent layer {c} {dtype}")
    w = small_workload(dtype, B=c["B"], S=c["S"], D=256, H=c["H"], F=512, causal=True, Bq=min(c.get("Bq", 64), c["S"]), Bkv=1)
    inp = make_inputs(w, seed=case, affine=True, biases=True)
    g = torch.Generator().manual_seed(10 + case)
    inp["lam"] = torch.randn(256, generator=g) - 4.0
    h0, dhT = (torch.randn(w.B, 256, generator=g) for _ in range(2)) if c["h0"] else (None, None)
    dev = {k: v.cuda() for k, v in inp.items()}
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    cfg = bpt.make_config(w.B, w.S, w.D, w.H, w.F, w.Bq, 1, True, dtype, "f32", group_blocks=c.get("group_blocks", 0))
    lay = bpt.RecurrentLayer(cfg)
    Y, hT, saved = lay.forward(dev["X"], dev, on(h0))
    dX, grads = lay.backward(dev["X"], dev, saved, dev["dY"], on(h0), on(dhT))
    torch.cuda.synchronize()
    got = {"Y": Y, "hT": hT, "dX": dX, **grads}

    def reference(R):
        p = {k: inp[k].double().requires_grad_() for k in NAMES + ("lam",)}
        X = inp["X"].double().requires_grad_()
        h = None if h0 is None else h0.double().requires_grad_()
        y, last = layer(X, p, h, R=R)
        ((y * inp["dY"].double()).sum() + (0.0 if dhT is None else (last * dhT.double()).sum())).backward()
        out = {"Y": y.detach(), "hT": last.detach(), "dX": X.grad, **{"d" + k: t.grad for k, t in p.items()}}
        return dict(out, dh0=h.grad) if h is not None else out

    ref = reference(exactly)
    model = reference(rounded) if dtype == "bf16" else None
    bad = []
    for n, r in ref.items():
        e_max, e_mean = errors(got[n], r)
        lim = (1e-4, 1e-4)
        if model:
            m_max, m_mean = errors(model[n], r)
            lim = bf16_limits({"e_max": m_max, "e_mean": m_mean})
        print(f"{n}: {e_max:.2e} <= {lim[0]:.2e}, {e_mean:.2e} <= {lim[1]:.2e}", flush=True)
        if not (e_max <= lim[0] and e_mean <= lim[1]):
            bad.append((n, e_max, e_mean, lim))
    assert not bad, bad


def test_a_sequence_in_pieces_and_token_by_token():
    """The layer over pieces of a sequence, the states handed on in place: what the whole gives, within fp32's bound of the layer."""
    B, S, D = 2, 70, 256
    w = small_workload("f32", B=B, S=S, D=D, H=2, F=512, causal=True, Bq=64, Bkv=1)
    inp = make_inputs(w, seed=1, affine=True, biases=True)
    dev = {k: v.cuda() for k, v in inp.items()}
    dev["lam"] = torch.randn(D, device="cuda") - 4.0
    mk = lambda n: bpt.make_config(B, n, D, 2, 512, n, 1, True, "f32")  # noqa: E731
    whole, last, _ = bpt.RecurrentLayer(mk(S)).forward(dev["X"], dev)
    h, parts = torch.zeros(B, D, device="cuda"), []
    for lo, hi in [(0, 40)] + [(t, t + 1) for t in range(40, 50)] + [(50, S)]:
        cfg = mk(hi - lo)
        X = dev["X"][:, lo:hi].contiguous()
        Y = torch.empty_like(X)
        saved, ws = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (bpt.layer_recurrent_saved_bytes(cfg),
                                                                                bpt.layer_recurrent_workspace_bytes(cfg, False)))
        bpt.layer_fwd_recurrent(cfg, bpt.recur_mixer(cfg, dev["lam"], h0=h, hT=h), X, dev, Y, saved, ws)
        parts.append(Y)
    for got, ref in ((torch.cat(parts, 1), whole), (h, last)):
        assert errors(got, ref.double().cpu())[0] <= 2e-4


def gpt_reference(m, tok, head, mixer):
    """Loss of a GPT by float64 autograd from its masters; head(h, Wout) gives the loss."""
    s = m.shape
    P = {n: m.master(n).double().cpu().requires_grad_() for n in m.names()}
    x = P["Wte"][tok.long()].view(s.B, s.S, s.D)
    if s.pos_table:
        x = x + P["Wpe"]
    for l in range(s.L):
        x = mixer(x, {k: P[f"{l}.{k}"] for k in NAMES + (("lam",) if s.recurrent else ())})
    h = torch.nn.functional.layer_norm(x, (s.D,), P["lnf_g"], P["lnf_b"], 1e-5)
    loss = head(h.view(-1, s.D) @ P["Wout"][:, :s.V])
    loss.backward()
    return loss.detach(), P


KW = dict(L=2, B=2, S=150, D=256, H=4, F=512, V=500, Bq=64, Bkv=64)


def teacher_lists(T, V, K, g):
    values = torch.randn(T, K, generator=g) * 2
    index = torch.stack([torch.randperm(V, generator=g)[:K] for _ in range(T)]).int()
    index[::4, K // 2:] = -1
    weights = (torch.rand(T, generator=g) > 0.2).float() / T
    return values, index, weights


@pytest.mark.parametrize("recurrent", [True, False])
@pytest.mark.parametrize("kind", ["train", "distill"])
def test_gpt_step_f32(kind, recurrent):
    """Loss and every gradient, fp32, within 1e-4 rms of float64 autograd."""
    s = GPTShape(dtype="f32", recurrent=recurrent, pos_table=not recurrent, **KW)
    m = GPT(s, seed=1)
    g = torch.Generator().manual_seed(2)
    T, K, tau = s.B * s.S, 12, 2.0
    tok, tgt = (torch.randint(0, s.V, (T,), generator=g, dtype=torch.int32) for _ in range(2))
    for n in m.nodecay.index:
        m.master(n).add_(0.1 * torch.randn(m.master(n).shape, generator=g).cuda())
    values, index, weights = teacher_lists(T, s.V, K, g)

    def head(z):
        ce = torch.nn.functional.cross_entropy(z, tgt.long(), reduction="none")
        if kind == "train":
            return ce.mean()
        q = torch.softmax(values.double().masked_fill(index < 0, -math.inf) / tau, dim=1)
        logp = torch.log_softmax(z / tau, dim=1).gather(1, index.long().clamp(min=0))
        kl = (torch.special.xlogy(q, q) - q * logp).sum(dim=1)
        return (weights.double() * (0.7 * tau * tau * kl + 0.3 * ce)).sum()

    mixer = (lambda x, p: layer(x, p)[0]) if recurrent else (lambda x, p: attention_layer(x, p, s.H))
    want, P = gpt_reference(m, tok, head, mixer)
    if kind == "train":
        got = m.forward(tok.cuda(), tgt.cuda())
        m.backward(tok.cuda(), tgt.cuda())
    else:
        got = m.distill_forward(tok.cuda(), values.cuda(), index.cuda(), tgt.cuda(), weights.cuda(), tau, 0.7, 0.3)
        m.distill_backward(tok.cuda())
    torch.cuda.synchronize()
    assert abs(float(got[0]) - float(want)) <= 1e-5 * abs(float(want))
    for n in m.names():
        assert errors(m.grad(n), P[n].grad)[0] <= 1e-4, n


def test_a_recurrent_student_learns_from_a_model_with_attention():
    """The whole of it in bf16: the teacher's largest logits from its head, a student with recurrences and 8-bit moments, three steps
    that are finite and the same bit for bit when repeated, and a step's passes replayed from a graph."""
    teacher = GPT(GPTShape(dtype="bf16", **KW), seed=5)
    g = torch.Generator().manual_seed(3)
    T, K = teacher.shape.B * teacher.shape.S, 16
    tok, tgt = (torch.randint(0, 500, (T,), generator=g, dtype=torch.int32).cuda() for _ in range(2))
    teacher.forward(tok, tgt)
    values, index = (teacher.hf.float() @ teacher.weight("Wout")[:, :500].float()).topk(K, dim=1)
    values, index = values.contiguous(), index.int().contiguous()
    runs = []
    for _ in range(2):
        m = GPT(GPTShape(dtype="bf16", recurrent=True, pos_table=False, opt_bits=8, **KW), seed=1)
        for _ in range(3):
            loss = m.distill_step(tok, values, index, 1e-3, targets=tgt, tau=2.0, soft=0.8, hard=0.2)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(loss).all())
        runs.append([t.clone() for grp in (m.decay, m.nodecay) for t in (grp.p, grp.m, grp.r, grp.exps)] + [loss.clone()])
    assert all(torch.equal(a, b) for a, b in zip(*runs))

    def passes():
        out = m.distill_forward(tok, values, index, tgt, tau=2.0, soft=0.8, hard=0.2)
        m.distill_backward(tok)
        return out

    loss = passes()
    torch.cuda.synchronize()
    ref = loss.clone(), m.decay.g.clone(), m.nodecay.g.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        passes()
    for _ in range(3):
        for t in (loss, m.decay.g, m.nodecay.g):
            t.zero_()
        torch.randn(1000, device="cuda").sum().item()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, ref[0]) and torch.equal(m.decay.g, ref[1]) and torch.equal(m.nodecay.g, ref[2])


def test_dropout_of_a_recurrent_layer_repeats():
    w = small_workload("bf16", B=2, S=100, D=256, H=2, F=512, causal=True, Bq=64, Bkv=1)
    inp = make_inputs(w, seed=1)
    dev = {k: v.cuda() for k, v in inp.items() if v is not None}
    dev["lam"] = torch.randn(256, device="cuda") - 4.0
    cfg = bpt.make_config(w.B, w.S, w.D, w.H, w.F, 64, 1, True, "bf16", dropout=0.1, dropout_seed=3)
    out = []
    for _ in range(2):
        lay = bpt.RecurrentLayer(cfg)
        Y, hT, saved = lay.forward(dev["X"], dev)
        dX, g = lay.backward(dev["X"], dev, saved, dev["dY"])
        out.append((Y, hT, dX, *g.values()))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and bool(torch.isfinite(a.float()).all()) for a, b in zip(*out))
