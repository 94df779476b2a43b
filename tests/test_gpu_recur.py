"""The gated recurrence on the GPU against float64, step by step. Bounds: linear_time_ref.recur's (float32 throughout) plus half a
step of the type for y, dx, dr and di."""
import math

import pytest
import torch

from gpu_util import say
from linear_time_ref import recur
from long_context_ref import HALF, check
from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def inputs(B, S, D, dtype, seed, joint=False, h0=True, wide=False):
    """Inputs on the GPU: gates around 0 (wide: also far open and closed), decays from fast to nearly none."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    rn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    dt = DT[dtype]
    if joint:
        p = rn(B, S, 3 * D).to(dt)
        x, r, i = p[..., :D], p[..., D:2 * D], p[..., 2 * D:]
    else:
        x, r, i = (rn(B, S, D).to(dt) for _ in range(3))
    if wide:
        r, i = r * 12, i * 12
    lam = rn(D) * 2 - 5
    return dict(x=x, r=r, i=i, lam=lam, h0=rn(B, D) if h0 else None, dy=rn(B, S, D).to(dt), dhT=rn(B, D) if h0 else None)


def run(t, lens=None):
    rec = bpt.GatedRecurrence()
    y, hT, saved = rec.forward(t["x"], t["r"], t["i"], t["lam"], t["h0"], lens, save=True)
    out = rec.backward(t["x"], t["r"], t["i"], t["lam"], saved, t["dy"], t["dhT"], t["h0"], lens)
    torch.cuda.synchronize()
    return dict(out, y=y, hT=hT)


def compare(t, out, lens=None):
    ref = recur(t["x"], t["r"], t["i"], t["lam"], 8.0, t["h0"], lens, t["dy"], t["dhT"])
    half = HALF[t["x"].dtype]
    for name in ("y", "hT", "dx", "dr", "di", "dlam", "dh0"):
        last = half if name in ("y", "dx", "dr", "di") else 0.0
        check(out[name].cpu(), ref[name], ref[name + "_err"] * 1.01 + last * ref[name].abs(), name)


CASES = [
    # B, S, D, joint, h0
    (1, 1, 8, False, True), (3, 1, 2048, True, True), (2, 2, 24, True, False), (1, 15, 64, False, True), (2, 33, 72, False, True),
    (1, 127, 128, True, False), (2, 128, 40, False, True), (1, 129, 64, False, True), (3, 255, 8, False, False), (1, 256, 200, True, True),
    (2, 257, 64, False, True), (1, 1000, 136, False, True), (5, 640, 16, True, False), (1, 4100, 8, False, True),
    (1, 8200, 16, False, False), (1, 35000, 8, True, True), (4, 5, 520, True, True), (9001, 2, 8, False, True), (3, 8, 264, False, False), (600, 130, 8, False, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(map(str, c)))
def test_forward_and_backward(case, dtype):
    B, S, D, joint, h0 = case
    say(f"case recur {case} {dtype}")
    t = inputs(B, S, D, dtype, S + D, joint, h0)
    compare(t, run(t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S", [1, 70, 600])
def test_gates_far_open_and_closed(S, dtype):
    t = inputs(2, S, 32, dtype, S, wide=True)
    t["lam"][:4] = torch.tensor([-80.0, -30.0, 3.0, 20.0], device="cuda")     # nearly no decay; all of it at once
    t["r"][:, :, 4:8], t["i"][:, :, 4:8] = -200.0, 200.0                      # a closed gate: m = 0
    compare(t, run(t))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,lens", [(1, (1, 0)), (40, (17, 0, 40)), (300, (0, 128, 129, 300)), (520, (512, 1, 0, 260))])
def test_lengths(S, lens, dtype):
    """What the inputs hold behind a sequence's length changes nothing; y and the gradients are 0 there."""
    t = inputs(len(lens), S, 72, dtype, S)
    ln = torch.tensor(lens, dtype=torch.int32, device="cuda")
    behind = torch.arange(S, device="cuda")[None, :] >= ln[:, None]
    first = run(t, ln)
    compare(t, first, ln)
    for k, bad in (("x", math.nan), ("r", math.inf), ("i", -math.inf), ("dy", math.nan)):
        t[k][behind] = bad
    again = run(t, ln)
    for k in first:
        assert torch.equal(first[k], again[k]), k
    for k in ("y", "dx", "dr", "di"):
        assert bool((again[k][behind] == 0.0).all()), k


def test_lengths_are_clamped():
    t = inputs(3, 50, 8, "f32", 1)
    a = run(t, torch.tensor([50, 0, 50], dtype=torch.int32, device="cuda"))
    b = run(t, torch.tensor([99, -3, 2 ** 31 - 1], dtype=torch.int32, device="cuda"))
    for k in a:
        assert torch.equal(a[k], b[k]), k


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_of_a_sequence(dtype):
    """A sequence in pieces, states and their gradients handed on: what the whole gives, within the bounds of both."""
    B, S, D = 2, 391, 40
    t = inputs(B, S, D, dtype, 7)
    rec, cuts = bpt.GatedRecurrence(), (0, 1, 200, 391)
    h, parts = t["h0"], []
    for lo, hi in zip(cuts, cuts[1:]):
        v = [t[k][:, lo:hi] for k in ("x", "r", "i")]
        y, hT, saved = rec.forward(*v, t["lam"], h, save=True)
        parts.append((v, h, y, saved))
        h = hT
    out = {"y": torch.cat([p[2] for p in parts], 1), "hT": h}
    dh, grads, dlam = t["dhT"], [], 0.0
    for (v, h0, _, saved), lo, hi in list(zip(parts, cuts, cuts[1:]))[::-1]:
        g = rec.backward(*v, t["lam"], saved, t["dy"][:, lo:hi], dh, h0)
        dh, dlam = g["dh0"], dlam + g["dlam"]
        grads.insert(0, g)
    out.update({k: torch.cat([g[k] for g in grads], 1) for k in ("dx", "dr", "di")}, dh0=dh, dlam=dlam)
    compare(t, out)


def test_state_in_place():
    """A serving loop: hT is h0, one token at a time, against the whole sequence."""
    B, S, D = 5, 20, 264
    t = inputs(B, S, D, "f32", 3)
    ref = recur(t["x"], t["r"], t["i"], t["lam"], 8.0, t["h0"])
    h = t["h0"].clone()
    for s in range(S):
        x, r, i = (t[k][:, s:s + 1] for k in ("x", "r", "i"))
        y = torch.empty(B, 1, D, device="cuda")
        bpt.recur_fwd(bpt.recur_config_of(x, r, i, y), x, r, i, t["lam"], y, h, h)
        check(y[:, 0].cpu(), ref["y"][:, s], ref["y_err"][:, s] * 1.01, "y")
    check(h.cpu(), ref["hT"], ref["hT_err"] * 1.01, "hT")


@pytest.mark.parametrize("S", [1, 20, 50, 64, 150, 3000])
def test_gradient_of_the_state_in_place(S):
    """dh0 is dhT: every wave and every chunk has read it before the first chunk's result is written."""
    t = inputs(2, S, 64, "f32", 4)
    rec = bpt.GatedRecurrence()
    _, _, saved = rec.forward(t["x"], t["r"], t["i"], t["lam"], t["h0"], save=True)
    ref = rec.backward(t["x"], t["r"], t["i"], t["lam"], saved, t["dy"], t["dhT"], t["h0"])
    d = t["dhT"].clone()
    v = (t["x"], t["r"], t["i"])
    cfg = bpt.recur_config_of(*v, t["dy"])
    g = [torch.empty_like(t["x"]) for _ in range(3)]
    ws = torch.empty(max(256, bpt.recur_workspace_bytes(cfg, True)), dtype=torch.uint8, device="cuda")
    bpt.recur_bwd(cfg, *v, t["lam"], saved, t["dy"], *g, ws, h0=t["h0"], dhT=d, dh0=d)
    assert torch.equal(d, ref["dh0"]) and torch.equal(g[0], ref["dx"])


def test_strides_and_what_lies_beside():
    """Tensors of unlike strides; what is not theirs stays as it was."""
    B, S, D = 2, 137, 72
    t = inputs(B, S, D, "bf16", 5)
    wide = {k: torch.full((S, B, D + 24), 3.0, dtype=torch.bfloat16, device="cuda") for k in ("x", "r", "y")}
    for k in ("x", "r"):
        wide[k][:, :, 8:8 + D] = t[k].transpose(0, 1)
    view = {k: w[:, :, 8:8 + D].transpose(0, 1) for k, w in wide.items()}
    cfg = bpt.recur_config_of(view["x"], view["r"], t["i"], view["y"])
    saved = torch.empty(max(256, bpt.recur_saved_bytes(cfg)), dtype=torch.uint8, device="cuda")
    ws = torch.empty(max(256, bpt.recur_workspace_bytes(cfg, True), bpt.recur_workspace_bytes(cfg, False)), dtype=torch.uint8, device="cuda")
    bpt.recur_fwd(cfg, view["x"], view["r"], t["i"], t["lam"], view["y"], t["h0"], None, saved, ws)
    dy = torch.full_like(wide["y"], 5.0)
    dyv = dy[:, :, 8:8 + D].transpose(0, 1)
    dyv.copy_(t["dy"])
    d = {k: torch.full_like(wide["x"], 7.0) for k in ("x", "r")}
    dv = {k: w[:, :, 8:8 + D].transpose(0, 1) for k, w in d.items()}
    di, dlam, dh0 = torch.empty_like(t["i"]), torch.empty(D, device="cuda"), torch.empty(B, D, device="cuda")
    bpt.recur_bwd(cfg, view["x"], view["r"], t["i"], t["lam"], saved, dyv, dv["x"], dv["r"], di, ws, dlam, t["h0"], t["dhT"], dh0)
    want = run(t)
    got = dict(y=view["y"], dx=dv["x"], dr=dv["r"], di=di, dlam=dlam, dh0=dh0)
    for k, v in got.items():
        assert torch.equal(v, want[k]), k
    for w, fill in ((wide["y"], 3.0), (d["x"], 7.0), (d["r"], 7.0)):
        assert bool((w[:, :, :8] == fill).all()) and bool((w[:, :, 8 + D:] == fill).all())


@pytest.mark.parametrize("S", [1, 3, 140])
def test_layouts_of_a_backward(S):
    """Inputs that lie otherwise than dense ones: the same gradients, laid out like them where that leaves no gaps."""
    B, D = 3, 72
    t = inputs(B, S, D, "bf16", 8)
    ref = run(t)
    full = lambda *n: torch.full(n, 3.0, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    turned = full(S, B, D).transpose(0, 1)
    wide = full(B, S, 2 * D)[..., 8:8 + D]
    odd = full(B * S * D + 1)[1:].view(B, S, D)      # off the 16 bytes
    for name, view in (("x", turned), ("r", wide), ("i", odd), ("dy", odd), ("dy", wide), ("dy", turned)):
        view.copy_(t[name])
        got = run({**t, name: view}) if name != "i" else None
        if got is None:                              # the forward takes no such pointer; the backward copies
            rec = bpt.GatedRecurrence()
            _, _, saved = rec.forward(t["x"], t["r"], t["i"], t["lam"], t["h0"], save=True)
            got = rec.backward(t["x"], t["r"], view, t["lam"], saved, t["dy"], t["dhT"], t["h0"])
        for k, v in got.items():
            assert torch.equal(v, ref[k]), (name, k)
        if name == "x":
            assert got["dx"].stride() == turned.stride()
    p = full(B, S, 3 * D)
    for order in ("xri", "irx"):
        v = {k: p[..., n * D:(n + 1) * D] for n, k in enumerate(order)}
        for k in order:
            v[k].copy_(t[k])
        got = run({**t, **v})
        for k, g in got.items():
            assert torch.equal(g, ref[k]), (order, k)
        assert all(got["d" + k].data_ptr() == got["d" + order[0]].data_ptr() + 2 * n * D for n, k in enumerate(order))


def test_offsets_past_32_bits():
    """Sequences more than 2^31 elements apart: what dense tensors give."""
    B, S, D = 2, 300, 72
    t = inputs(B, S, D, "bf16", 7)
    ref = run(t)
    gap = (1 << 31) + 64                             # between the starts of two sequences of one projection

    def far(*values):
        flat = torch.empty(gap + S * 3 * D, dtype=torch.bfloat16, device="cuda")
        views = [flat.as_strided((B, S, D), (gap, 3 * D, 1), k * D) for k in range(3)]
        for view, v in zip(views, values):
            view.copy_(v)
        return views

    (x, r, i), (y, dy, _), (dx, dr, di) = far(t["x"], t["r"], t["i"]), far(t["dy"], t["dy"]), far()
    cfg = bpt.recur_config_of(x, r, i, y)
    ws = torch.empty(max(bpt.recur_workspace_bytes(cfg, k) for k in (False, True)), dtype=torch.uint8, device="cuda")
    saved, hT = torch.empty(bpt.recur_saved_bytes(cfg), dtype=torch.uint8, device="cuda"), torch.empty(B, D, device="cuda")
    bpt.recur_fwd(cfg, x, r, i, t["lam"], y, t["h0"], hT, saved, ws)
    dlam, dh0 = torch.empty(D, device="cuda"), torch.empty(B, D, device="cuda")
    bpt.recur_bwd(cfg, x, r, i, t["lam"], saved, dy, dx, dr, di, ws, dlam, t["h0"], t["dhT"], dh0)
    for k, v in dict(y=y, hT=hT, dx=dx, dr=dr, di=di, dlam=dlam, dh0=dh0).items():
        assert torch.equal(v, ref[k]), k


def test_a_nan_stays_in_its_channel_and_after_its_step():
    t = inputs(2, 300, 64, "f32", 6)
    ref = run(t)
    t["x"] = t["x"].clone()
    t["x"][1, 130, 9] = math.nan
    out = run(t)
    bad = torch.zeros_like(t["x"], dtype=torch.bool)
    bad[1, 130:, 9] = True
    assert bool(out["y"][bad].isnan().all()) and torch.equal(out["y"][~bad], ref["y"][~bad])
    assert bool(out["dlam"][9].isnan()) and torch.equal(out["dlam"][:9], ref["dlam"][:9])


@pytest.mark.parametrize("B,S,D", [(2, 700, 64), (1, 20000, 64), (1, 1, 512)])
def test_the_same_every_time_and_from_a_graph(B, S, D):
    t = inputs(B, S, D, "bf16", 8)
    rec = bpt.GatedRecurrence()
    ref = run(t)
    v = (t["x"], t["r"], t["i"])
    y, hT = torch.empty_like(t["x"]), torch.empty(B, D, device="cuda")
    cfg = bpt.recur_config_of(*v, y)
    saved = rec._bytes(bpt.recur_saved_bytes(cfg), "cuda")
    ws = [rec._bytes(bpt.recur_workspace_bytes(cfg, k), "cuda") for k in (False, True)]
    g = [torch.empty_like(t["x"]) for _ in range(3)]
    dlam, dh0 = torch.empty(D, device="cuda"), torch.empty(B, D, device="cuda")

    def step():
        bpt.recur_fwd(cfg, *v, t["lam"], y, t["h0"], hT, saved, ws[0])
        bpt.recur_bwd(cfg, *v, t["lam"], saved, t["dy"], *g, ws[1], dlam, t["h0"], t["dhT"], dh0)

    graph = torch.cuda.CUDAGraph()
    step()
    with torch.cuda.graph(graph):
        step()
    outs = dict(y=y, hT=hT, dx=g[0], dr=g[1], di=g[2], dlam=dlam, dh0=dh0)
    for _ in range(4):
        for o in list(outs.values()) + ws + [saved]:
            o.fill_(77)
        graph.replay()
        torch.cuda.synchronize()
        for k, o in outs.items():
            assert torch.equal(o, ref[k]), k
        eager = run(t)
        for k in ref:
            assert torch.equal(eager[k], ref[k]), k


def test_two_streams_at_once():
    """Two calls with buffers of their own, on two streams: each gives what it gives alone."""
    ts = [inputs(1, 9000, 256, "bf16", 20 + k) for k in range(2)]
    refs = [run(t) for t in ts]
    streams = [torch.cuda.Stream() for _ in ts]
    torch.cuda.synchronize()
    outs = [None, None]
    for k, st in enumerate(streams):
        with torch.cuda.stream(st):
            rec = bpt.GatedRecurrence()
            t = ts[k]
            y, hT, saved = rec.forward(t["x"], t["r"], t["i"], t["lam"], t["h0"], save=True)
            outs[k] = dict(rec.backward(t["x"], t["r"], t["i"], t["lam"], saved, t["dy"], t["dhT"], t["h0"]), y=y, hT=hT)
    torch.cuda.synchronize()
    for o, ref in zip(outs, refs):
        for k in ref:
            assert torch.equal(o[k], ref[k]), k
