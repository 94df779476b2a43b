"""Calls that the recurrence, the layer with it and the distillation loss take or refuse on the host: buffers that stay where a captured
graph has them, gradients that lie otherwise than dense ones, arguments that must not share memory."""
import os

import pytest
import torch

from paper_2305_19370_amd import bpt

needs_lib = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")


# ---------------------------------------------------------------- a GPT's buffers for the distillation loss
@needs_lib
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_distillation_buffers_of_a_gpt_stay(monkeypatch, dtype):
    """A graph may hold their addresses: they are made once, large enough for every list, with and without targets."""
    from paper_2305_19370_amd.gpt import GPT, GPTShape
    m = GPT(GPTShape(L=1, B=3, S=50, D=64, H=1, F=64, V=300, Bq=50, Bkv=50, dtype=dtype, xent_block_rows=64), device="cpu", init=False)
    calls = []

    def fwd(cfg, h, W, values, index, loss, tokens, saved, ws, targets, weights):
        calls.append((cfg, loss, tokens, saved, ws))

    monkeypatch.setattr(m, "_body_forward", lambda tokens: None)
    monkeypatch.setattr(bpt, "distill_fwd", fwd)
    tok = torch.zeros(150, dtype=torch.int32)
    for K, tau, hard in ((8, 2.0, 0.0), (8, 2.0, 0.2), (256, 1.0, 0.5), (1, 1.5, 0.0), (64, 1.0, 0.0), (8, 2.0, 0.0)):
        values, index = torch.zeros(150, K), torch.zeros(150, K, dtype=torch.int32)
        m.distill_forward(tok, values, index, tok if hard else None, tau=tau, hard=hard)
        cfg, *bufs = calls[-1]
        assert (cfg.K, cfg.tau, cfg.hard) == (K, tau, pytest.approx(hard))
        assert all(a is b for a, b in zip(bufs, calls[0][1:])), (K, tau, hard)
        assert bufs[2].numel() >= bpt.distill_saved_bytes(cfg)
        assert bufs[3].numel() >= max(bpt.distill_workspace_bytes(cfg, back) for back in (False, True))


@needs_lib
def test_distillation_of_a_gpt_keeps_what_its_shape_says(monkeypatch):
    from paper_2305_19370_amd.gpt import GPT, GPTShape
    sizes = []
    for keep in (0, -1, 64 * 320 * 4):
        m = GPT(GPTShape(L=1, B=3, S=50, D=64, H=1, F=64, V=300, Bq=50, Bkv=50, xent_block_rows=64, distill_keep_bytes=keep), device="cpu", init=False)
        monkeypatch.setattr(m, "_body_forward", lambda tokens: None)
        monkeypatch.setattr(bpt, "distill_fwd", lambda cfg, h, W, values, index, loss, tokens, saved, *rest: sizes.append((cfg.keep_bytes, saved.numel())))
        m.distill_forward(torch.zeros(150, dtype=torch.int32), torch.zeros(150, 4), torch.zeros(150, 4, dtype=torch.int32))
    assert [k for k, _ in sizes] == [0, -1, 64 * 320 * 4]
    assert sizes[0][1] - sizes[1][1] == 150 * 320 * 4 and sizes[2][1] - sizes[1][1] == 64 * 320 * 4


# ---------------------------------------------------------------- arguments that must not share memory
A = 1 << 20                                          # an aligned address that nothing may touch


@needs_lib
def test_recurrent_layer_refuses_shared_memory():
    lib, cfg = bpt.load(), bpt.make_config(2, 300, 256, 4, 512, 64, 64, True, "bf16")
    names = ("lam", "h0", "hT", "X", "Y", "saved", "ws") + bpt.PARAM_FIELDS
    good = {k: (n + 1) * A for n, k in enumerate(names)}

    def fwd(n=0, **kw):                              # n = 0: without a workspace, the last check before anything runs
        a = {**good, **kw}
        return lib.bpt_layer_fwd_recurrent(cfg, bpt.RecurMixer(8.0, a["lam"], a["h0"], a["hT"]), a["X"], bpt.Params(*[a[k] for k in bpt.PARAM_FIELDS]),
                                           a["Y"], a["saved"], a["ws"], n, None)

    assert fwd() == 3 and fwd(hT=good["h0"]) == 3 and fwd(hT=None) == 3 and fwd(h0=None) == 3
    for k in names:
        if k not in ("h0", "hT"):
            assert fwd(hT=good[k]) == 1, k
    for k in ("Y", "saved", "ws"):
        for q in ("lam", "h0", "hT"):
            assert fwd(**{k: good[q]}) == 1, (k, q)

    names = ("lam", "h0", "dhT", "X", "saved", "dY", "dX", "dlam", "dh0", "ws") + bpt.PARAM_FIELDS + bpt.GRAD_FIELDS
    good = {k: (n + 1) * A for n, k in enumerate(names)}

    def bwd(n=0, **kw):
        a = {**good, **kw}
        return lib.bpt_layer_bwd_recurrent(cfg, bpt.RecurMixer(8.0, a["lam"], a["h0"], None), a["X"], bpt.Params(*[a[k] for k in bpt.PARAM_FIELDS]),
                                           a["saved"], a["dY"], a["dhT"], a["dX"], bpt.Grads(*[a[k] for k in bpt.GRAD_FIELDS]), a["dlam"], a["dh0"],
                                           a["ws"], n, None)

    assert bwd() == 3 and bwd(dh0=good["dhT"]) == 3 and bwd(dlam=None, dh0=None, dhT=None, h0=None) == 3
    for k in names:
        if k != "dlam":
            assert bwd(dlam=good[k]) == 1, k
        if k not in ("dh0", "dhT"):
            assert bwd(dh0=good[k]) == 1, k
    for k in ("dX", "ws") + bpt.GRAD_FIELDS:
        for q in ("lam", "h0", "dhT"):
            assert bwd(**{k: good[q]}) == 1, (k, q)


@needs_lib
def test_operators_refuse_shared_memory():
    """Every pair of arguments of which one is written, but hT = h0 and dh0 = dhT."""
    lib, x = bpt.load(), torch.empty(2, 300, 72, dtype=torch.bfloat16)
    rec, dis = bpt.recur_config_of(x, x, x, x), bpt.make_distill_config(100, 64, 1000, 20, tau=2.0, soft=0.5, hard=0.5)
    for f, names, written, may in (
            (lambda *a: lib.bpt_recur_fwd(rec, *a, 1, None), "x r i lam lens h0 y hT saved ws", "y hT saved ws", ("h0", "hT")),
            (lambda *a: lib.bpt_recur_bwd(rec, *a, 1, None), "x r i lam lens h0 saved dy dhT dx dr di dlam dh0 ws", "dx dr di dlam dh0 ws", ("dhT", "dh0")),
            (lambda *a: lib.bpt_distill_fwd(dis, *a, 1, None), "h W values index targets weights loss tokens saved ws", "loss tokens saved ws", None),
            (lambda h, W, saved, *a: lib.bpt_distill_bwd(dis, h, W, saved, 1.0, *a, 1, None), "h W saved dh dW ws", "dh dW ws", None)):
        names = names.split()
        good = {k: (n + 1) * A for n, k in enumerate(names)}
        assert f(*good.values()) == 3, names         # the workspace of one byte, the last check
        for k in written.split():
            for q in names:
                if q != k:
                    want = 3 if may and {k, q} == set(may) else 1
                    assert f(*{**good, k: good[q]}.values()) == want, (names, k, q)


# ---------------------------------------------------------------- layouts that the class takes, on the CPU: the last refusal is that of the place
BROADCAST = {"mean over tokens": lambda B, S, D, dt: torch.ones(B, 1, D, dtype=dt).expand(B, S, D),
             "one gradient of all sequences": lambda B, S, D, dt: torch.ones(1, S, D, dtype=dt).expand(B, S, D),
             "one row": lambda B, S, D, dt: torch.ones(D, dtype=dt).expand(B, S, D),
             "one number": lambda B, S, D, dt: torch.ones((), dtype=dt).expand(B, S, D),
             "windows of one sequence": lambda B, S, D, dt: torch.ones(B + S, D, dtype=dt).as_strided((B, S, D), (D, D, 1))}


@needs_lib
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", BROADCAST)
def test_a_broadcast_gradient_is_taken(name, dtype):
    for B, S in ((2, 30), (2, 1), (1, 30), (1, 1)):
        x, lam = torch.zeros(B, S, 72, dtype=dtype), torch.zeros(72)
        with pytest.raises(ValueError, match="on the GPU"):
            bpt.GatedRecurrence().backward(x, x, x, lam, torch.empty(1 << 16, dtype=torch.uint8), BROADCAST[name](B, S, 72, dtype))


@needs_lib
@pytest.mark.parametrize("S", [1, 30])
def test_a_forward_takes_inputs_off_16_bytes(monkeypatch, S):
    """As the backward does: they are copied, and what the library gets is aligned. (Here it stands in for the library.)"""
    got = []
    monkeypatch.setattr(bpt, "_stream_on", lambda dev, same: 0)
    monkeypatch.setattr(bpt.load(), "bpt_recur_fwd", lambda cfg, *a: got.append(a) or 0)
    x, odd = torch.ones(2, S, 72), torch.ones(2 * S * 72 + 1)[1:].view(2, S, 72)
    for t in ((odd, x, x), (x, odd, x), (x, x, odd), (x, x, x)):
        y, _, _ = bpt.GatedRecurrence().forward(*t, torch.zeros(72))
        assert all(p % 16 == 0 for p in got[-1][:3]) and y.shape == x.shape
        assert [p == a.data_ptr() for p, a in zip(got[-1], t)] == [a is x for a in t]      # aligned ones are not copied


# ---------------------------------------------------------------- decays at the start
@needs_lib
@pytest.mark.parametrize("c", [1e-4, 1e-3, 0.01, 1.0, 8.0, 1e3])
def test_decays_of_a_new_gpt(c):
    """Between 0.9 and 0.999 where the gate is open, whatever their scale is."""
    from paper_2305_19370_amd.gpt import GPT, GPTShape
    m = GPT(GPTShape(L=1, B=1, S=8, D=256, H=4, F=64, V=10, Bq=8, Bkv=8, recurrent=True, recur_c=c), device="cpu")
    a = torch.exp(-c * torch.nn.functional.softplus(m.master("0.lam").double()))
    assert float(a.min()) >= 0.8999 and float(a.max()) <= 0.99901
