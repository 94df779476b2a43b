"""Refusals of the gated recurrence, the layer with it and the distillation loss: every one is made on the host, before anything is
launched (the pointers here are made up); and the float64 references these operators are compared with, against differences."""
import ctypes
import math
import os

import pytest
import torch

from linear_time_ref import distill, recur
from paper_2305_19370_amd import bpt

needs_lib = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")
A = 1 << 20                                          # an aligned address that nothing may touch
BF = torch.bfloat16


def err():
    return bpt.load().bpt_last_error().decode()


# ---------------------------------------------------------------- the references
def differences(f, tensors, grads, eps=1e-5):
    for name, t in tensors.items():
        for k in range(0, t.numel(), max(1, t.numel() // 9)):
            lo, hi = t.clone(), t.clone()
            lo.view(-1)[k] -= eps
            hi.view(-1)[k] += eps
            d = (f(**{**tensors, name: hi}) - f(**{**tensors, name: lo})) / (2 * eps)
            # the third derivative's part of the difference, and its cancellation
            assert abs(float(d - grads[name].reshape(-1)[k])) <= 1e-7 * (1 + abs(float(d))), (name, k)


def test_recurrence_reference_against_differences():
    g = torch.Generator().manual_seed(1)
    rn = lambda *n: torch.randn(*n, generator=g, dtype=torch.float64)  # noqa: E731
    B, S, D = 3, 9, 8
    t = dict(x=rn(B, S, D), r=rn(B, S, D), i=rn(B, S, D), lam=rn(D) - 3, h0=rn(B, D))
    dy, dhT, lens = rn(B, S, D), rn(B, D), torch.tensor([9, 4, 0])

    def f(x, r, i, lam, h0):
        o = recur(x, r, i, lam, 8.0, h0, lens)
        return (o["y"] * dy).sum() + (o["hT"] * dhT).sum()

    o = recur(**t, c=8.0, lens=lens, dy=dy, dhT=dhT)
    differences(f, t, dict(x=o["dx"], r=o["dr"], i=o["di"], lam=o["dlam"], h0=o["dh0"]))


def test_distillation_reference_against_differences():
    g = torch.Generator().manual_seed(2)
    T, D, V, K = 6, 4, 7, 3
    t = dict(h=torch.randn(T, D, generator=g, dtype=torch.float64), W=torch.randn(D, 8, generator=g, dtype=torch.float64))
    values, index = torch.randn(T, K, generator=g, dtype=torch.float64), torch.randint(-1, V, (T, K), generator=g)
    index[2], index[3] = -1, 5
    y, w = torch.tensor([0, 9, 3, 2, 6, -1]), torch.rand(T, generator=g, dtype=torch.float64)
    w[4] = 0.0
    f = lambda h, W: distill(h, W, V, values, index, 1.7, 0.6, 0.4, y, w)["loss"][0]  # noqa: E731
    o = distill(**t, V=V, values=values, index=index, tau=1.7, soft=0.6, hard=0.4, targets=y, weights=w)
    differences(f, t, dict(h=o["dh"], W=o["dW"]))
    assert bool((o["dW"][:, V:] == 0).all()) and bool((o["dh"][4] == 0).all())


# ---------------------------------------------------------------- the recurrence
def rcfg(**kw):
    x = torch.empty(2, 300, 72, dtype=BF)
    c = bpt.recur_config_of(x, x, x, x)
    for k, v in kw.items():
        if "." in k:
            setattr(getattr(c, k.split(".")[0]), k.split(".")[1], v)
        else:
            setattr(c, k, v)
    return c


@needs_lib
def test_recurrence_accepts():
    for c in (rcfg(), rcfg(S=1), rcfg(dtype=0), rcfg(D=8), rcfg(**{"x.sb": 0, "r.st": 0}), rcfg(**{"x.st": 1 << 20, "x.sb": 1 << 35})):
        assert bpt.recur_validate(c) == 0, err()
    assert bpt.recur_saved_bytes(rcfg()) == 2 * 4 * 72 * 4 and bpt.recur_saved_bytes(rcfg(S=64)) == 0
    assert bpt.recur_workspace_bytes(rcfg(S=1), False) == 0 and bpt.recur_workspace_bytes(rcfg(), True) > 0


BAD = [(dict(B=0), 1), (dict(S=0), 1), (dict(D=0), 1), (dict(D=-8), 1), (dict(c=0.0), 1), (dict(c=-1.0), 1), (dict(c=math.nan), 1),
       (dict(c=math.inf), 1), (dict(reserved=1), 1), (dict(dtype=2), 1), (dict(dtype=-1), 1), ({"x.sb": -8}, 1), ({"r.st": -8}, 1),
       ({"i.st": 73}, 1), ({"y.sb": 300 * 72 + 4}, 1), ({"y.sb": 72}, 1), ({"y.st": 64}, 1), ({"y.st": 0}, 1), (dict(D=70), 2), (dict(D=4), 2),
       (dict(S=1 << 29), 2), (dict(D=1 << 21), 2), ({"x.st": 1 << 21}, 2), ({"x.sb": 1 << 39}, 2),
       ({"B": 1 << 40, "y.sb": 300 * 72}, 2), (dict(B=1 << 23), 2), (dict(S=1 << 62), 2), (dict(D=1 << 62), 2)]


@needs_lib
@pytest.mark.parametrize("kw,code", BAD)
def test_recurrence_refuses(kw, code):
    c, lib = rcfg(**kw), bpt.load()
    assert bpt.recur_validate(c) == code and err()
    assert bpt.recur_saved_bytes(c) == 0 and bpt.recur_workspace_bytes(c, False) == 0 and bpt.recur_workspace_bytes(c, True) == 0
    assert lib.bpt_recur_fwd(c, A, A, A, A, None, None, 2 * A, None, None, 3 * A, 1 << 40, None) == code
    assert lib.bpt_recur_bwd(c, A, A, A, A, None, None, 2 * A, 3 * A, None, 4 * A, 5 * A, 6 * A, None, None, 7 * A, 1 << 40, None) == code
    assert lib.bpt_recur_validate(None) == 1


@needs_lib
def test_recurrence_refuses_pointers():
    c, lib = rcfg(), bpt.load()
    n = bpt.recur_workspace_bytes(c, False)
    good = dict(x=A, r=2 * A, i=3 * A, lam=4 * A, lens=5 * A, h0=6 * A, y=7 * A, hT=8 * A, saved=9 * A, ws=10 * A, n=n)
    call = lambda **kw: lib.bpt_recur_fwd(c, *{**good, **kw}.values(), None)  # noqa: E731
    for k in ("x", "r", "i", "lam", "y"):
        assert call(**{k: None}) == 1, k
    for k in ("x", "r", "i", "lam", "lens", "h0", "y", "hT", "saved", "ws"):
        assert call(**{k: good[k] + 8}) == 1, k
    for k in ("x", "r", "i", "lam", "lens", "h0"):
        assert call(y=good[k]) == 1, k
    for k in ("x", "r", "i", "lam", "lens", "y"):
        assert call(hT=good[k]) == 1, k
    assert call(saved=good["y"]) == 1 and call(saved=good["hT"]) == 1
    assert call(n=n - 1) == 3 and call(ws=None) == 3
    n = bpt.recur_workspace_bytes(c, True)
    good = dict(x=A, r=2 * A, i=3 * A, lam=4 * A, lens=5 * A, h0=6 * A, saved=9 * A, dy=7 * A, dhT=8 * A, dx=11 * A, dr=12 * A, di=13 * A,
                dlam=14 * A, dh0=15 * A, ws=10 * A, n=n)
    call = lambda **kw: lib.bpt_recur_bwd(c, *{**good, **kw}.values(), None)  # noqa: E731
    for k in ("x", "r", "i", "lam", "saved", "dy", "dx", "dr", "di", "ws"):
        assert call(**{k: None}) == 1, k
    for k in good:
        if k != "n":
            assert call(**{k: good[k] + 4}) == 1, k
    for k in ("dx", "dr", "di", "dlam", "dh0"):
        for q in ("x", "r", "i", "lam", "dy", "saved", "h0"):
            assert call(**{k: good[q]}) == 1, (k, q)
    assert call(dx=good["dhT"]) == 1 and call(dr=good["dx"]) == 1 and call(dh0=good["dlam"]) == 1
    assert call(n=n - 1) == 3
    for k in ("x", "r", "i"):                        # gradients need places of their own
        bad = rcfg(**{k + ".st": 0})
        assert lib.bpt_recur_bwd(bad, *good.values(), None) == 1


# ---------------------------------------------------------------- its binding, on the CPU: the last refusal is that of the place
def test_recurrence_binding_refuses():
    x, lam = torch.zeros(2, 30, 72, dtype=BF), torch.zeros(72)
    y, h = torch.empty_like(x), torch.zeros(2, 72)
    if not os.path.exists(bpt.LIB_PATH):
        pytest.skip("libbpt.so not built")
    cfg = bpt.recur_config_of(x, x, x, y)
    ok = dict(x=x, r=x, i=x, lam=lam, y=y, h0=h, hT=h)
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.recur_fwd(cfg, **ok)
    for k, bad in (("x", x.float()), ("r", x[:, :29]), ("i", x.transpose(0, 1)), ("y", x.float()), ("y", torch.empty(2, 30, 144, dtype=BF)[..., :72]),
                   ("lam", lam[:71]), ("lam", lam.to(BF)), ("h0", h.to(BF)), ("hT", h[:1]), ("h0", torch.zeros(72, 2).t())):
        with pytest.raises(ValueError, match=f"^{k} must"):
            bpt.recur_fwd(cfg, **{**ok, k: bad})
    g = dict(x=x, r=x, i=x, lam=lam, saved=None, dy=x, dx=y, dr=y, di=y, workspace=torch.empty(9999, dtype=torch.uint8), dlam=lam, dh0=h)
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.recur_bwd(cfg, **g)
    for k, bad in (("dy", x.float()), ("dx", x[:1]), ("dr", torch.empty(2, 30, 144, dtype=BF)[..., :72]), ("di", x.half()), ("dlam", lam[1:]),
                   ("dh0", h[:, :8]), ("dhT", h.double())):
        with pytest.raises(ValueError, match=f"^{k} must"):
            bpt.recur_bwd(cfg, **{**g, k: bad})
    for bad in ((x, x, x.float(), y), (x, x[:1], x, y), (x[0], x[0], x[0], y[0]), (x.half(), x.half(), x.half(), y.half())):
        with pytest.raises(ValueError):
            bpt.recur_config_of(*bad)
    with pytest.raises(ValueError, match="adjacent"):
        bpt.recur_config_of(x.transpose(1, 2), x.transpose(1, 2), x.transpose(1, 2), y.transpose(1, 2))
    rec = bpt.GatedRecurrence()
    with pytest.raises(ValueError, match="on the GPU"):
        rec.forward(x, x, x, lam)
    with pytest.raises(ValueError, match="share"):
        rec.forward(x, x.float(), x, lam)
    with pytest.raises(bpt.BptError):
        rec.forward(x[..., :70], x[..., :70], x[..., :70], lam[:70])
    with pytest.raises(ValueError, match="^dy must"):
        rec.backward(x, x, x, lam, torch.empty(1), x.float())
    long = torch.zeros(1, 200, 8)
    with pytest.raises(ValueError, match="^saved must"):
        bpt.recur_bwd(bpt.recur_config_of(long, long, long, long), long, long, long, torch.zeros(8), torch.empty(8), long, long, long, long,
                      torch.empty(9))


# ---------------------------------------------------------------- the layer with it
@needs_lib
def test_recurrent_layer_refuses():
    lib = bpt.load()
    cfg = bpt.make_config(2, 300, 256, 4, 512, 64, 64, True, "bf16")
    assert bpt.layer_recurrent_validate(cfg) == 0
    assert bpt.layer_recurrent_saved_bytes(cfg) == bpt.saved_bytes(cfg) + 2 * 4 * 256 * 4
    assert bpt.layer_recurrent_workspace_bytes(cfg, True) > bpt.workspace_bytes(cfg, True)
    for bad, c in ((bpt.make_config(2, 300, 256, 4, 512, 64, 64, False, "bf16"), 8.0), (cfg, 0.0), (cfg, math.nan),
                   (bpt.make_config(2, 300, 256, 3, 512, 64, 64, True, "bf16"), 8.0)):
        assert bpt.layer_recurrent_validate(bad, c) == 1
        m = bpt.RecurMixer(c, A, None, None)
        p = bpt.Params(*[A] * 12)
        assert lib.bpt_layer_fwd_recurrent(bad, m, A, p, 2 * A, 3 * A, 4 * A, 1 << 40, None) == 1
        assert lib.bpt_layer_bwd_recurrent(bad, m, A, p, 3 * A, 2 * A, None, 5 * A, None, None, None, 4 * A, 1 << 40, None) == 1
    p, n = bpt.Params(*[A] * 12), bpt.layer_recurrent_workspace_bytes(cfg, False)
    fwd = lambda m, n=n: lib.bpt_layer_fwd_recurrent(cfg, m, A, p, 2 * A, 3 * A, 4 * A, n, None)  # noqa: E731
    assert fwd(None) == 1 and fwd(bpt.RecurMixer(8.0, None, None, None)) == 1
    for k in range(3):
        at = [A, A, A]
        at[k] += 4
        assert fwd(bpt.RecurMixer(8.0, *at)) == 1
    assert fwd(bpt.RecurMixer(8.0, A, None, None), n - 1) == 3
    n = bpt.layer_recurrent_workspace_bytes(cfg, True)
    bwd = lambda m, dhT=None, dlam=None, dh0=None, n=n: lib.bpt_layer_bwd_recurrent(  # noqa: E731
        cfg, m, A, p, 3 * A, 2 * A, dhT, 5 * A, None, dlam, dh0, 4 * A, n, None)
    m = bpt.RecurMixer(8.0, A, 6 * A, None)
    assert bwd(m, dhT=A + 4) == 1 and bwd(m, dlam=A + 8) == 1 and bwd(m, dh0=A + 2) == 1 and bwd(m, dh0=6 * A) == 1
    assert bwd(m, dlam=9 * A, dh0=9 * A) == 1 and bwd(m, n=n - 1) == 3 and bwd(bpt.RecurMixer(8.0, None, None, None)) == 1


@needs_lib
def test_recurrent_gpt_refuses():
    from paper_2305_19370_amd.gpt import GPT, GPTShape
    kw = dict(L=1, B=1, S=8, D=64, H=1, F=64, V=10, Bq=8, Bkv=8, recurrent=True)
    for bad in (dict(rope="half"), dict(window=4)):
        with pytest.raises(ValueError, match="recurrent"):
            GPT(GPTShape(**kw, **bad), device="cpu", init=False)
    for bad in (dict(causal=False), dict(recur_c=0.0)):
        with pytest.raises(bpt.BptError):
            GPT(GPTShape(**kw, **bad), device="cpu", init=False)
    m = GPT(GPTShape(**kw), device="cpu")
    lam = m.master("0.lam")
    a = torch.exp(-8.0 * torch.nn.functional.softplus(lam))
    assert float(a.min()) >= 0.8999 and float(a.max()) <= 0.99901
    with pytest.raises(ValueError, match="follows"):
        m.distill_backward(torch.zeros(8, dtype=torch.int32))
    assert m.shape.n_params() == sum(m.master(n).numel() for n in m.names()) - 64 * (m.shape.ldw - 10)


@needs_lib
def test_recurrent_layer_binding_refuses_the_place():
    cfg = bpt.make_config(1, 64, 64, 1, 64, 64, 64, True, "bf16")
    X, raw, p = torch.zeros(1, 64, 64, dtype=BF), torch.zeros(1 << 21, dtype=torch.uint8), dict.fromkeys(bpt.PARAM_FIELDS)
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.layer_fwd_recurrent(cfg, bpt.RecurMixer(8.0, A, None, None), X, p, X.clone(), raw, raw)
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.layer_bwd_recurrent(cfg, bpt.RecurMixer(8.0, A, None, None), X, p, raw, X, X.clone(), {}, raw)


# ---------------------------------------------------------------- the distillation loss
def dcfg(**kw):
    c = bpt.make_distill_config(100, 64, 1000, 20, tau=2.0, soft=0.5, hard=0.5)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@needs_lib
def test_distillation_accepts():
    for c in (dcfg(), dcfg(K=256), dcfg(K=1, T=1), dcfg(hard=0.0), dcfg(soft=0.0), dcfg(dtype=0), dcfg(grad_dtype=1), dcfg(ldw=4096),
              dcfg(block_rows=7)):
        assert bpt.distill_validate(c) == 0, err()
        assert bpt.distill_saved_bytes(c) >= 100 * 12 or c.T == 1
        assert bpt.distill_workspace_bytes(c, False) > 0 and bpt.distill_workspace_bytes(c, True) > 0


DBAD = [(dict(T=0), 1), (dict(D=0), 1), (dict(V=0), 1), (dict(K=0), 1), (dict(K=-1), 1), (dict(ldw=960), 1), (dict(block_rows=-1), 1),
        (dict(tau=0.0), 1), (dict(tau=-1.0), 1), (dict(tau=math.nan), 1), (dict(tau=math.inf), 1), (dict(tau=1e-40), 1), (dict(tau=3e-39), 1), (dict(tau=1e19), 1), (dict(soft=-0.1), 1),
        (dict(hard=-0.1), 1), (dict(soft=math.nan), 1), (dict(hard=math.inf), 1), (dict(dtype=3), 1), (dict(grad_dtype=2), 1), (dict(reserved=1), 1),
        (dict(K=257), 2), (dict(D=65), 2), (dict(ldw=1001), 2), (dict(dtype=0, grad_dtype=1), 2), (dict(T=1 << 31), 2),
        (dict(D=1 << 40), 2), (dict(D=1 << 20, ldw=1 << 20), 2), (dict(V=(1 << 31) - 64, ldw=1 << 31), 2),
        (dict(T=1 << 23, block_rows=1 << 23), 2)]


@needs_lib
@pytest.mark.parametrize("kw,code", DBAD)
def test_distillation_refuses(kw, code):
    c, lib = dcfg(**kw), bpt.load()
    assert bpt.distill_validate(c) == code and err()
    assert bpt.distill_saved_bytes(c) == 0 and bpt.distill_workspace_bytes(c, False) == 0 and bpt.distill_workspace_bytes(c, True) == 0
    assert lib.bpt_distill_fwd(c, *[A] * 10, 1 << 50, None) == code
    assert lib.bpt_distill_bwd(c, A, A, A, 1.0, 2 * A, 3 * A, 4 * A, 1 << 50, None) == code
    with pytest.raises(bpt.BptError):
        bpt.DistillLoss(c)


@needs_lib
def test_distillation_keeps_whole_blocks():
    """Logits within keep_bytes, 4 GiB by itself; those that a block would exceed are not kept."""
    row = 4 * 1024
    size = lambda **kw: bpt.distill_saved_bytes(dcfg(**kw))  # noqa: E731
    none = size(keep_bytes=-1)
    up = lambda n: (n + 255) // 256 * 256  # noqa: E731
    assert size() - none == up(100 * row)
    for keep, tokens in ((1, 0), (100 * row - 1, 0), (100 * row, 100), (1 << 62, 100), (-1 << 63, 0)):
        assert size(keep_bytes=keep) - none == up(tokens * row), keep
    for keep, tokens in ((33 * row - 1, 0), (33 * row, 33), (70 * row, 66), (99 * row, 99), (100 * row, 100)):
        assert size(keep_bytes=keep, block_rows=33) - none == up(tokens * row), keep
    big = dict(T=1 << 20, block_rows=1 << 10)
    assert size(**big) - size(keep_bytes=-1, **big) == 4 << 30


@needs_lib
def test_distillation_refuses_pointers():
    c, lib = dcfg(), bpt.load()
    n = bpt.distill_workspace_bytes(c, False)
    good = dict(zip(("h", "W", "values", "index", "targets", "weights", "loss", "tokens", "saved", "ws"), (k * A for k in range(1, 11))), n=n)
    call = lambda c=c, **kw: lib.bpt_distill_fwd(c, *{**good, **kw}.values(), None)  # noqa: E731
    for k in good:
        if k == "n":
            continue
        if k != "weights":
            assert call(**{k: None}) == 1, k
        assert call(**{k: good[k] + 8}) == 1, k
    assert call(n=n - 1) == 3
    n = bpt.distill_workspace_bytes(c, True)
    call = lambda h=A, W=2 * A, saved=3 * A, dh=4 * A, dW=5 * A, ws=6 * A, n=n: lib.bpt_distill_bwd(  # noqa: E731
        c, h, W, saved, 1.0, dh, dW, ws, n, None)
    for k in ("h", "W", "saved", "dh", "ws"):
        assert call(**{k: None}) == 1 and call(**{k: 7 * A + 4}) == 1, k
    assert call(dW=7 * A + 2) == 1 and call(dh=A) == 1 and call(dW=2 * A) == 1 and call(dW=4 * A) == 1 and call(n=n - 1) == 3


@needs_lib
def test_distillation_binding_refuses():
    c = dcfg(grad_dtype=1)
    T, D, K, L = c.T, c.D, c.K, c.ldw
    z = lambda *n, dt=torch.float32: torch.zeros(*n, dtype=dt)  # noqa: E731
    raw = torch.empty(bpt.distill_workspace_bytes(c, False) + bpt.distill_workspace_bytes(c, True) + bpt.distill_saved_bytes(c), dtype=torch.uint8)
    ok = dict(h=z(T, D, dt=BF), W=z(D, L, dt=BF), values=z(T, K), index=z(T, K, dt=torch.int32), loss=z(3), tokens=z(2, T), saved=raw, workspace=raw,
              targets=z(T, dt=torch.int32), weights=z(T))
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.distill_fwd(c, **ok)
    for k, bad in (("h", z(T, D)), ("h", z(D, T, dt=BF).t()), ("W", z(D, 1000, dt=BF)), ("values", z(T, K, dt=BF)), ("values", z(T, K + 1)[:, :K]),
                   ("index", z(T, K, dt=torch.int64)), ("loss", z(1)), ("tokens", z(T, 2)), ("targets", z(T, dt=torch.int64)),
                   ("weights", z(T, dt=torch.float64))):
        with pytest.raises(ValueError, match=f"^{k} must"):
            bpt.distill_fwd(c, **{**ok, k: bad})
    with pytest.raises(ValueError, match="^saved must"):
        bpt.distill_fwd(c, **{**ok, "saved": raw[:100]})
    back = dict(h=ok["h"], W=ok["W"], saved=raw, dloss=1.0, dh=z(T, D, dt=BF), dW=z(D, L, dt=BF), workspace=raw)
    with pytest.raises(ValueError, match="on the GPU"):
        bpt.distill_bwd(c, **back)
    for k, bad in (("dh", z(T, D)), ("dW", z(D, L)), ("dW", z(L, D, dt=BF).t()), ("W", z(D, L))):
        with pytest.raises(ValueError, match=f"^{k} must"):
            bpt.distill_bwd(c, **{**back, k: bad})
