"""The gradients of Q, K and V that a layer's backward leaves behind, with rotary positions."""
import pytest
import torch

from bpt_inputs import make_inputs, small_workload
from gpu_util import say
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu


def run(opt, dtype="f32", seed=2):
    w = small_workload(dtype, B=2, S=150, D=256, H=4, F=512, causal=True, Bq=64, Bkv=64)
    inp = make_inputs(w, seed=seed, affine=True, biases=True)
    dev = {k: v.cuda() for k, v in inp.items()}
    lay = bpt.Layer(bpt.make_config(w.B, w.S, w.D, w.H, w.F, 64, 64, True, dtype, "f32"), options=opt)
    Y, saved = lay.forward(dev["X"], dev)
    dX, g = lay.backward(dev["X"], dev, saved, dev["dY"], qkv_grads=True)
    torch.cuda.synchronize()
    return inp, g


def test_of_the_projection_before_it_turns():
    """dWq = U^T dQ and so on for Q = U Wq, whatever turns Q afterwards (fp32)."""
    say("case qkv gradients with rotary positions")
    inp, g = run(bpt.make_layer_options(rot=64, layout="interleaved", mscale=1.2, pos0=77))
    x = inp["X"].double().view(-1, 256)
    u = torch.nn.functional.layer_norm(x, (256,), inp["ln1_g"].double(), inp["ln1_b"].double(), 1e-5)
    for n in ("q", "k", "v"):
        want = u.T @ g[f"d{n.upper()}"].double().cpu().reshape(-1, 256)
        got = g[f"dW{n}"].double().cpu()
        # the sums of 300 products: fp32 accumulation and the rounding of U and dQ, 300 * 2^-24 = 1.8e-5 of the sum of magnitudes
        lim = 2e-5 * (u.abs().T @ g[f"d{n.upper()}"].double().abs().cpu().reshape(-1, 256)) + 1e-6
        assert bool(((got - want).abs() <= lim).all()), n


def test_empty_options_leave_the_layers():
    a, b = run(None, "bf16")[1], run(bpt.make_layer_options(), "bf16")[1]
    assert a.keys() == b.keys() and {"dQ", "dK", "dV"} <= a.keys()
    assert all(torch.equal(a[n], b[n]) for n in a)
