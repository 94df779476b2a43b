"""The layer's windowed paths beside its other settings: dropout, ReLU, no biases or gains, some gradients only, weight gradients
in slices of the tokens, and sums of key blocks and sinks that the workspace has little room for."""
import math

import pytest
import torch

from bpt_inputs import make_inputs, small_workload
from gpu_util import bf16_limits, say
from paper_2305_19370_amd import bpt
from test_gpu_layer_options import NAMES, errors, layer, rounded, turner

pytestmark = pytest.mark.gpu


def run(w, inp, dtype, opt, activation="gelu", dropout=0.0, want=None):
    dev = {k: v.cuda() for k, v in inp.items() if v is not None}
    cfg = bpt.make_config(w.B, w.S, w.D, w.H, w.F, 64, 64, True, dtype, "f32", activation=activation, dropout=dropout, dropout_seed=11)
    lay = bpt.Layer(cfg, options=opt)
    bpt.profile_enable(True)
    Y, saved = lay.forward(dev["X"], dev)
    dX, g = lay.backward(dev["X"], dev, saved, dev["dY"], want=want)
    torch.cuda.synchronize()
    bpt.profile_enable(False)
    return {"Y": Y, "dX": dX, **g}, bpt.profile_report()


def compare(got, ref, lim):
    bad = []
    for n in ref:
        e_max, e_mean = errors(got[n], ref[n].double().cpu())
        print(f"{n}: {e_max:.2e}, {e_mean:.2e} <= {lim(n)}", flush=True)
        if not (e_max <= lim(n)[0] and e_mean <= lim(n)[1]):
            bad.append((n, e_max, e_mean))
    assert not bad, bad


SETTINGS = [
    dict(), dict(dropout=0.1), dict(activation="relu"), dict(activation="relu", dropout=0.3), dict(affine=False, biases=False),
]


@pytest.mark.parametrize("shape", [(2, 300, 256, 4, 512), (1, 3000, 128, 2, 256), (1, 256, 512, 4, 64)])
@pytest.mark.parametrize("kw", SETTINGS, ids=lambda k: "-".join(f"{a}={b}" for a, b in k.items()) or "plain")
def test_a_window_of_everything_is_the_layer(kw, shape):
    """fp32: a window as long as the sequence leaves the layer's own results. Both are within 1e-4 rms of the formula, the layer's
    bound, so within 2e-4 of one another."""
    B, S, D, H, F = shape
    say(f"case whole window {shape} {kw}")
    kw = dict(kw)
    w = small_workload("f32", B=B, S=S, D=D, H=H, F=F, causal=True, Bq=64, Bkv=64)
    inp = make_inputs(w, seed=1, affine=kw.pop("affine", True), biases=kw.pop("biases", True))
    ref, _ = run(w, inp, "f32", None, **kw)
    got, rep = run(w, inp, "f32", bpt.make_layer_options(window=S), **kw)
    assert "win.fwd" in rep and "win.bwd" in rep and "attn.fwd" not in rep
    assert got.keys() == ref.keys()
    compare(got, ref, lambda n: (2e-4, 2e-4))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_some_gradients(dtype):
    """Any set of weight gradients has the bits that all together have, also where they are formed in slices of the tokens."""
    w = small_workload(dtype, B=1, S=3000, D=128, H=2, F=256, causal=True, Bq=64, Bkv=64)
    inp = make_inputs(w, seed=4, affine=True, biases=True)
    opt = bpt.make_layer_options(rot=32, window=100, sinks=2)
    every, rep = run(w, inp, dtype, opt, dropout=0.1)
    assert "reduce.ksplit" in rep                    # slices
    for want in ((), ("dWq",), ("dWk", "dWo"), ("dWv", "dln1_g", "dln1_b"), ("dW1", "dWq", "dWk", "dWv")):
        some, _ = run(w, inp, dtype, opt, dropout=0.1, want=want)
        assert some.keys() == {"Y", "dX", *want}
        assert all(torch.equal(some[n], every[n]) for n in some), want


ROOM = [
    # S, D, H, F, window, sinks: the key blocks' chunks (8) fit the FFN group's buffers as 4, or not at all; the sinks' chunks
    (2000, 128, 2, 512, 400, 4),
    (2000, 128, 2, 64, 400, 4),
    (2500, 128, 1, 64, 60, 300),
]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", ROOM, ids=str)
def test_little_room_for_sums(shape, dtype):
    """fp32: within 1e-4 rms of the formula in float64; bf16: the gate of the layer's parity tests over its rounding model. The mean
    error of n elements is itself a sample: half-normal errors have a deviation of sqrt(pi / 2 - 1) of their mean, the ratio of two such
    means (the kernels' and the model's) one of sqrt(2) sqrt(pi / 2 - 1) / sqrt(n), 9.4 % for the 128 elements of a gain's
    gradient. The gate is wider by four of them, which adds 4 % or less for the matrices."""
    S, D, H, F, window, sinks = shape
    say(f"case room {shape} {dtype}")
    w = small_workload(dtype, B=1, S=S, D=D, H=H, F=F, causal=True, Bq=64, Bkv=64)
    inp = make_inputs(w, seed=7, affine=True, biases=True)
    opt = dict(rot=64, window=window, sinks=sinks)
    got, rep = run(w, inp, dtype, bpt.make_layer_options(**opt))
    print({n: r["count"] for n, r in rep.items() if n.startswith("win")}, flush=True)

    def reference(**kw):
        p = {k: inp[k].double().requires_grad_() for k in NAMES}
        X = inp["X"].double().requires_grad_()
        Y = layer(X, p, H, True, window=window, sinks=sinks, turn=turner(S, D // H, opt), **kw)
        Y.backward(inp["dY"].double())
        return {"Y": Y.detach(), "dX": X.grad, **{"d" + k: p[k].grad for k in NAMES}}

    ref = reference()
    if dtype == "f32":
        compare(got, ref, lambda n: (1e-4, 1e-4))
    else:
        model = reference(R=rounded)
        lims = {n: bf16_limits(dict(zip(("e_max", "e_mean"), errors(model[n], ref[n])))) for n in ref}
        sample = {n: 4 * math.sqrt(2) * math.sqrt((math.pi / 2 - 1) / r.numel()) for n, r in ref.items()}
        compare(got, ref, lambda n: (lims[n][0], lims[n][1] * (1 + sample[n])))


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 1), (70, 0)])
@pytest.mark.parametrize("B,S", [(1, 1), (3, 5), (2, 63), (1, 64), (2, 65)])
def test_short_sequences(B, S, window, sinks):
    """From one token to one past a tile, fp32, with rotary positions: within 1e-4 rms of the formula."""
    say(f"case short {B} x {S} window {window} sinks {sinks}")
    w = small_workload("f32", B=B, S=S, D=128, H=2, F=256, causal=True, Bq=min(64, S), Bkv=min(64, S))
    inp = make_inputs(w, seed=S, affine=True, biases=True)
    opt = dict(rot=16, layout="interleaved", window=window, sinks=sinks, pos0=3)
    dev = {k: v.cuda() for k, v in inp.items()}
    lay = bpt.Layer(bpt.make_config(B, S, 128, 2, 256, min(64, S), min(64, S), True, "f32", "f32"), options=bpt.make_layer_options(**opt))
    Y, saved = lay.forward(dev["X"], dev)
    dX, g = lay.backward(dev["X"], dev, saved, dev["dY"])
    torch.cuda.synchronize()
    p = {k: inp[k].double().requires_grad_() for k in NAMES}
    X = inp["X"].double().requires_grad_()
    ref = layer(X, p, 2, True, window=window, sinks=sinks, turn=turner(S, 64, opt))
    ref.backward(inp["dY"].double())
    grads = {"Y": ref.detach(), "dX": X.grad, **{"d" + k: p[k].grad for k in NAMES}}
    got = {"Y": Y, "dX": dX, **g}
    for n, r in grads.items():                       # one key in sight: dS is 0 in the formula, rounding here
        d = (got[n].double().cpu() - r).abs().max()
        scale = max(float(r.square().mean().sqrt()), 1e-3 * float(grads["dWv"].square().mean().sqrt()))
        assert float(d) <= 1e-4 * scale, (n, float(d), scale)
