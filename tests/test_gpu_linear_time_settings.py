"""The recurrence, the layer with it and GPT steps in settings other than their defaults: other decays, dropout, ReLU, no biases, a bf16
head with fp32 weight gradients. References in float64."""
import math

import pytest
import torch

from bpt_inputs import make_inputs, small_workload
from gpu_util import say
from linear_time_ref import distill, recur
from long_context_ref import HALF, check
from oracle.dropout import dropout_factor
from paper_2305_19370_amd import bpt
from paper_2305_19370_amd.gpt import GPT, GPTShape
from test_gpu_layer_options import NAMES, errors
from test_gpu_recur import inputs
from test_gpu_recurrent_layer import KW, gpt_reference, layer, mix, teacher_lists

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [1, 70, 300])
def test_other_decays(S, dtype):
    """One layout, several c one after the other (sizes and layouts are kept between calls, c is not): the bounds of the default's tests."""
    t = inputs(2, S, 72, dtype, S)
    half = HALF[t["x"].dtype]
    for c in (0.5, 20.0, 8.0, 1e-3, 0.5):
        say(f"case c {c} S {S} {dtype}")
        rec = bpt.GatedRecurrence(c)
        y, hT, saved = rec.forward(t["x"], t["r"], t["i"], t["lam"], t["h0"], save=True)
        out = dict(rec.backward(t["x"], t["r"], t["i"], t["lam"], saved, t["dy"], t["dhT"], t["h0"]), y=y, hT=hT)
        ref = recur(t["x"], t["r"], t["i"], t["lam"], bpt.recur_config_of(t["x"], t["r"], t["i"], y, c).c, t["h0"], None, t["dy"], t["dhT"])
        for k in ("y", "hT", "dx", "dr", "di", "dlam", "dh0"):
            last = half if k in ("y", "dx", "dr", "di") else 0.0
            check(out[k].cpu(), ref[k], ref[k + "_err"] * 1.01 + last * ref[k].abs(), k)


SETTINGS = [dict(c=0.5), dict(c=20.0), dict(dropout=0.1), dict(activation="relu"), dict(activation="relu", dropout=0.3, c=2.0), dict(bare=True)]


@pytest.mark.parametrize("kw", SETTINGS, ids=lambda kw: "-".join(f"{k}={v}" for k, v in kw.items()))
def test_layer(kw):
    """Y, the last states, dX and every gradient in fp32, max|diff| <= 1e-4 rms: the layer's bound. bare: no gains, shifts or biases."""
    say(f"case recurrent layer {kw}")
    B, S, D, F, c, rate = 2, 150, 256, 512, kw.get("c", 8.0), kw.get("dropout", 0.0)
    bare = kw.get("bare", False)
    w = small_workload("f32", B=B, S=S, D=D, H=2, F=F, causal=True, Bq=64, Bkv=1)
    inp = make_inputs(w, seed=4, affine=not bare, biases=not bare)
    g = torch.Generator().manual_seed(5)
    inp["lam"] = torch.randn(D, generator=g) - 4.0
    h0, dhT = torch.randn(B, D, generator=g), torch.randn(B, D, generator=g)
    dev = {k: v.cuda() if v is not None else None for k, v in inp.items()}
    cfg = bpt.make_config(B, S, D, 2, F, 64, 1, True, "f32", activation=kw.get("activation", "gelu"), dropout=rate, dropout_seed=0xABCDEF0123)
    lay = bpt.RecurrentLayer(cfg, c=c)
    Y, hT, saved = lay.forward(dev["X"], dev, h0.cuda())
    dX, grads = lay.backward(dev["X"], dev, saved, dev["dY"], h0.cuda(), dhT.cuda())
    got = {"Y": Y, "hT": hT, "dX": dX, **grads}

    names = [k for k in NAMES + ("lam",) if inp.get(k) is not None]
    p = {k: inp[k].double().requires_grad_() for k in names}
    X, h = inp["X"].double().requires_grad_(), h0.double().requires_grad_()
    ln = lambda x, n: torch.nn.functional.layer_norm(x, (D,), p.get(n + "_g"), p.get(n + "_b"), 1e-5)  # noqa: E731
    drop = [torch.from_numpy(dropout_factor(B * S, D, 0xABCDEF0123, k, rate)).view(B, S, D) for k in (0, 1)]
    u = ln(X, "ln1")
    o, last = mix(u @ p["Wq"], u @ p["Wk"], u @ p["Wv"], p["lam"], c, h)
    r = X + drop[0] * (o @ p["Wo"])
    z = ln(r, "ln2") @ p["W1"] + p.get("b1", 0.0)
    y = r + drop[1] * ((torch.relu(z) if kw.get("activation") else torch.nn.functional.gelu(z)) @ p["W2"] + p.get("b2", 0.0))
    ((y * inp["dY"].double()).sum() + (last * dhT.double()).sum()).backward()
    ref = {"Y": y.detach(), "hT": last.detach(), "dX": X.grad, "dh0": h.grad, **{"d" + k: t.grad for k, t in p.items()}}
    assert set(ref) == set(got)
    for n in ref:
        assert errors(got[n], ref[n])[0] <= 1e-4, n


@pytest.mark.parametrize("c", [1.0, 16.0])
def test_gpt_step_with_another_decay(c):
    s = GPTShape(dtype="f32", recurrent=True, recur_c=c, pos_table=False, **KW)
    m = GPT(s, seed=1)
    g = torch.Generator().manual_seed(2)
    tok, tgt = (torch.randint(0, s.V, (s.B * s.S,), generator=g, dtype=torch.int32) for _ in range(2))
    want, P = gpt_reference(m, tok, lambda z: torch.nn.functional.cross_entropy(z, tgt.long()), lambda x, p: layer(x, p, c=c)[0])
    got = m.forward(tok.cuda(), tgt.cuda())
    m.backward(tok.cuda(), tgt.cuda())
    torch.cuda.synchronize()
    assert abs(float(got[0]) - float(want)) <= 1e-5 * abs(float(want))
    for n in m.names():
        assert errors(m.grad(n), P[n].grad)[0] <= 1e-4, n


@pytest.mark.parametrize("recurrent,keep", [(True, 0), (False, 0), (True, -1)])
def test_distillation_of_a_bf16_gpt(recurrent, keep):
    """The head's part of a bf16 step, whose dW is fp32: losses, dh and dW against float64 from the head's input as the model has it. What lies
    below the head takes this dh: the gradients of the same passes from an upstream gradient of the cross entropy's in its place."""
    s = GPTShape(dtype="bf16", recurrent=recurrent, pos_table=not recurrent, distill_keep_bytes=keep, **KW)
    m = GPT(s, seed=1)
    g = torch.Generator().manual_seed(2)
    T, K, tau = s.B * s.S, 12, 2.0
    tok, tgt = (torch.randint(0, s.V, (T,), generator=g, dtype=torch.int32).cuda() for _ in range(2))
    values, index, weights = (t.cuda() for t in teacher_lists(T, s.V, K, g))
    m.weight("Wout").mul_(20.0)                      # logits of some units
    loss = m.distill_forward(tok, values, index, tgt, weights, tau, 0.7, 0.3)
    m.distill_backward(tok, -1.5)
    cfg, (_, tokens, _, _) = m.distill, m.distill_bufs
    ref = distill(m.hf, m.weight("Wout"), s.V, values, index, cfg.tau, cfg.soft, cfg.hard, tgt, weights, -1.5, HALF[torch.bfloat16], HALF[torch.float32])
    for k, v in dict(loss=loss, tokens=tokens, dh=m.dh, dW=m.grad("Wout")).items():
        check(v.cpu(), ref[k], ref[k + "_err"], k)
    # the passes below the head, from the same dh
    below = [n for n in m.names() if n != "Wout"]
    grads = {n: m.grad(n).clone() for n in below}
    dh = m.dh.clone()
    m.forward(tok, tgt)
    m.backward(tok, tgt)
    assert any(not torch.equal(m.grad(n), grads[n]) for n in below)
    m.dh.copy_(dh)
    m._body_backward(tok)
    for n in below:
        assert torch.equal(m.grad(n), grads[n]) and bool(torch.isfinite(grads[n]).all()) and math.isfinite(float(grads[n].abs().max())), n
