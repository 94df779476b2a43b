"""Rotary positions, attention with a sliding window and sinks, and AdamW over many tensors, as cases that can be timed and compared.

Kinds of case:

  rope    rotary positions of the heads of a projection: forward alone (serving) or forward and
          backward (training)
  attn    attention with a window and sinks: mode "train" (forward, then dQ, dK, dV), "fwd" (a prompt or
          a piece of one) or "token" (one or few new tokens per sequence against a cache)
  adamw   one optimiser step over a list of tensors, moments in 32 or in 8 bits

With `own` false a pass computes the plain form, elementary torch operations in float32; with
`own` true it makes the calls of paper_2305_19370_amd.bpt that a user's program makes.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}

ROPE = dict(kind="rope", mode="train", dtype="bf16", layout="half", theta=10000.0, scaling="none", factor=1.0, orig_len=0,
            mscale=1.0, pos0=0, positions=False)
ATTN = dict(kind="attn", mode="train", dtype="bf16", dh=128, causal=True, window=0, sinks=0, ragged=False, heads_first=False)
ADAMW = dict(kind="adamw", bits=8, grad="f32", lowp=True)


def listed():
    return [
        # one new token of each of 8 sequences, 32 query and 8 key heads: a serving loop, where latency counts
        dict(ROPE, name="rope_token_b8_h40", mode="fwd", B=8, S=1, H=40, dh=128, rot=128, pad=1024, positions=True),
        # the query and key heads of the GPT-XL benchmark's projection [16384, 3 x 2048], forward and backward
        dict(ROPE, name="rope_train_t16384_h32", B=1, S=16384, H=32, dh=128, rot=128, pad=2048),
        # float32, interleaved pairs on half of the head, context stretched by parts, odd lengths far into a long document
        dict(ROPE, name="rope_parts_f32_b4_s1003", B=4, S=1003, H=12, dh=128, rot=64, pad=0, dtype="f32", layout="interleaved",
             scaling="by_parts", factor=8.0, orig_len=4096, mscale=1.2, pos0=900001),
        # one new token against a short cache with a window: the smallest call
        dict(ATTN, name="attn_token_b1_l1500_w1024", mode="token", B=1, Sq=1, Skv=1500, Hq=16, Hkv=4, window=1024, sinks=4),
        # one new token of each of 24 sequences of unequal lengths against full caches, grouped heads
        dict(ATTN, name="attn_token_b24_l16384", mode="token", B=24, Sq=1, Skv=16384, Hq=32, Hkv=8, ragged=True),
        # the float32 parity workload's heads (bpt_inputs: fp32_s512_d256) with a window, forward and backward
        dict(ATTN, name="attn_f32_s512_h4_w128", B=1, Sq=512, Skv=512, Hq=4, Hkv=4, dh=64, dtype="f32", window=128, sinks=4),
        # a small model's training on a padded batch of odd length, heads of 64, one sequence empty
        dict(ATTN, name="attn_train_b4_s1000_h12_w256", B=4, Sq=1000, Skv=1000, Hq=12, Hkv=12, dh=64, window=256, sinks=4, ragged=True),
        # the 1B-shaped layer's 16 heads on four key heads, 8192 tokens, window and sinks
        dict(ATTN, name="attn_train_s8192_h16_w1024", B=1, Sq=8192, Skv=8192, Hq=16, Hkv=4, window=1024, sinks=4),
        # a prompt of 16384 tokens, head-major tensors, window of 4096 and many sinks: forward alone
        dict(ATTN, name="attn_fwd_s16384_h16_w4096", mode="fwd", B=1, Sq=16384, Skv=16384, Hq=16, Hkv=8, window=4096, sinks=64,
             heads_first=True),
        # the LayerNorm vectors and biases of the 24-layer GPT-XL benchmark: many small tensors
        dict(ADAMW, name="adamw8_vectors_l24", tensors="vectors", L=24, D=2048, F=8192, V=0, lowp=False),
        # the matrices and vectors of one 1B-shaped layer, 32-bit moments
        dict(ADAMW, name="adamw32_layer_d2048", tensors="layers", L=1, D=2048, F=8192, V=0, bits=32),
        # an embedding of an odd vocabulary and two layers, 8-bit moments, bf16 gradients
        dict(ADAMW, name="adamw8_l2_d1600_v50257", tensors="layers", L=2, D=1600, F=6400, V=50257, grad="bf16"),
    ]


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rope(rng):
    dh = rng.choice((64, 128))
    rot = dh if rng.random() < 0.6 else rng.choice((16, 32, 48, dh // 2, dh - 16))
    mode = rng.choice(("train", "train", "fwd"))
    B = _log(rng, 1, 64)
    S = 1 if mode == "fwd" and rng.random() < 0.4 else _log(rng, 2, max(2, 32768 // B))
    scaling = rng.choice(("none", "none", "linear", "base", "by_parts"))
    return dict(ROPE, mode=mode, dtype=rng.choice(("bf16", "bf16", "f32")), layout=rng.choice(("half", "interleaved")),
                theta=rng.choice((10000.0, 500000.0)), scaling=scaling, factor=1.0 if scaling == "none" else rng.choice((2.0, 8.0, 32.0)),
                orig_len=4096 if scaling == "by_parts" else 0, mscale=1.2 if scaling == "by_parts" else 1.0,
                pos0=rng.choice((0, 0, _log(rng, 1, 1000000))), positions=rng.random() < 0.4, B=B, S=S, H=_log(rng, 1, 48), dh=dh,
                rot=rot, pad=rng.choice((0, 64, 1000, 2048)))


def _draw_attn(rng):
    while True:
        mode = rng.choice(("train", "train", "train", "fwd", "token"))
        dtype = "f32" if rng.random() < 0.2 else "bf16"
        Hkv, G = rng.choice((1, 2, 3, 4, 8)), rng.choice((1, 1, 2, 4, 5, 8))
        if mode == "token":
            B, Skv, Sq = _log(rng, 1, 32), _log(rng, 1, 24000), rng.choice((1, 1, 1, 2, 5))
            Sq = min(Sq, Skv)
        else:
            B, Skv = _log(rng, 1, 8), _log(rng, 16, 2000 if dtype == "f32" else 10000)
            Sq = Skv if mode == "train" or rng.random() < 0.5 else _log(rng, 1, Skv)
        window = 0 if rng.random() < 0.25 else _log(rng, 1, 4096)
        c = dict(ATTN, mode=mode, dtype=dtype, dh=rng.choice((64, 128)), causal=rng.random() < 0.85, window=window,
                 sinks=rng.choice((0, 1, 4, 16, 64)) if window else 0, ragged=rng.random() < 0.4, heads_first=rng.random() < 0.3,
                 B=B, Sq=Sq, Skv=Skv, Hq=Hkv * G, Hkv=Hkv)
        scores = B * Hkv * G * Sq * Skv
        if scores <= 1.2e9 and (dtype == "bf16" or scores <= 1.2e8) and B * Skv * Hkv * c["dh"] <= 4.2e8:
            return c


def _draw_adamw(rng):
    kind = rng.choice(("vectors", "layers", "layers"))
    D = 8 * _log(rng, 8, 250)
    c = dict(ADAMW, tensors=kind, L=_log(rng, 1, 24 if kind == "vectors" or D < 512 else 2), D=D, F=4 * D - rng.choice((0, 0, 1, 7)),
             V=0 if kind == "vectors" else rng.choice((0, _log(rng, 500, 20000))), bits=rng.choice((8, 8, 32)),
             grad=rng.choice(("f32", "f32", "bf16")), lowp=rng.random() < 0.7)
    return c


def draw(rng):
    return rng.choice((_draw_rope, _draw_attn, _draw_attn, _draw_adamw))(rng)


# ---------------------------------------------------------------- shapes that follow from a case
def _lens(c):
    """(query lengths, key lengths) per sequence: unequal where ragged, the last of several sequences empty."""
    B, Sq, Skv = c["B"], c["Sq"], c["Skv"]
    if not c["ragged"]:
        return [Sq] * B, [Skv] * B
    kv = [Skv - (b * Skv) // B for b in range(B)]
    if B > 1:
        kv[-1] = 0
    return ([min(Sq, n) for n in kv] if c["mode"] != "token" else [Sq] * B), kv


def _visible(c):
    """Visible (query, key) pairs of one head, and keys that some query sees, over the batch."""
    pairs = keys = 0
    for nq, nk in zip(*_lens(c)):
        p = np.arange(nq, dtype=np.int64) + nk - nq
        p = p[p >= 0] if c["causal"] else p
        if nk == 0 or p.size == 0:
            continue
        W, sinks = c["window"], c["sinks"]
        hi = np.minimum(p, nk - 1) if c["causal"] else np.minimum(p + W - 1, nk - 1) if W else np.full_like(p, nk - 1)
        lo = np.maximum(p - W + 1, 0) if W else np.zeros_like(p)
        near = np.maximum(hi - lo + 1, 0)
        seen = np.minimum(np.minimum(p + 1, nk) if c["causal"] else nk, sinks) if W else np.zeros_like(p)
        both = np.maximum(np.minimum(hi + 1, seen) - lo, 0)
        pairs += int((near + seen - both).sum())
        keys += int(min(nk, hi.max() - lo.min() + 1 + min(sinks, lo.min())))
    return pairs, keys


def _shapes(c):
    D, F, L = c["D"], c["F"], c["L"]
    vecs = [(D,), (D,), (D,), (D,), (F,), (D,)]
    if c["tensors"] == "vectors":
        return vecs * L
    mats = [(D, D), (D, D), (D, D), (D, D), (D, F), (F, D)]
    return ([(c["V"], D)] if c["V"] else []) + (mats + vecs) * L


def work(case):
    c = case
    if c["kind"] == "rope":
        n, e = c["B"] * c["S"], 2 if c["dtype"] == "bf16" else 4
        passes = 2 if c["mode"] == "train" else 1
        return {"bytes": passes * (2 * n * c["H"] * c["dh"] * e + (4 * n if c["positions"] else 0)),
                "flops": passes * 3.0 * n * c["H"] * c["rot"]}
    if c["kind"] == "attn":
        pairs, keys = _visible(c)
        e = 2 if c["dtype"] == "bf16" else 4
        q, kv, row = c["B"] * c["Sq"] * c["Hq"] * c["dh"] * e, keys * c["Hkv"] * c["dh"] * e, c["B"] * c["Hq"] * c["Sq"] * 4
        if c["mode"] != "train":
            return {"bytes": 2 * q + 2 * kv + row, "flops": 4.0 * c["dh"] * c["Hq"] * pairs}
        return {"bytes": 4 * q + 4 * kv + row, "flops": 14.0 * c["dh"] * c["Hq"] * pairs}
    n = sum(math.prod(s) for s in _shapes(c))
    state = 4 if c["bits"] == 8 else 16
    return {"bytes": n * (8 + (2 if c["grad"] == "bf16" else 4) + state + (2 if c["lowp"] else 0)), "flops": 14.0 * n}


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return lambda *s, std=1.0, dt=torch.float32: torch.randn(s, generator=g, device="cuda").mul_(std).to(dt)


def _view(t, heads_first):
    """[B, S, H, dh] as the case stores it: token-major, or a view of a head-major tensor."""
    return t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) if heads_first else t


def prepare(case, seed):
    c, rn = dict(case), _gen(seed)
    s = {"case": c}
    if c["kind"] == "rope":
        T, w = c["B"] * c["S"], c["H"] * c["dh"]
        # the heads are the first columns of a wider projection (its values follow them)
        s["X"] = rn(T, w + c["pad"], dt=DT[c["dtype"]])[:, :w].view(T, c["H"], c["dh"])
        if c["mode"] == "train":
            s["dY"] = rn(T, c["H"], c["dh"], dt=DT[c["dtype"]])
        s["pos"] = None
        if c["positions"]:
            g = torch.Generator(device="cuda")
            g.manual_seed(seed + 1)
            s["pos"] = torch.randint(0, 200000, (T,), generator=g, device="cuda", dtype=torch.int32) + c["pos0"]
    elif c["kind"] == "attn":
        B, dh, dt = c["B"], c["dh"], DT[c["dtype"]]
        q, k, v = rn(B, c["Sq"], c["Hq"], dh, dt=dt), rn(B, c["Skv"], c["Hkv"], dh, dt=dt), rn(B, c["Skv"], c["Hkv"], dh, dt=dt)
        s["q"], s["k"], s["v"] = (_view(t, c["heads_first"]) for t in (q, k, v))
        if c["mode"] == "train":
            s["do"] = _view(rn(B, c["Sq"], c["Hq"], dh, dt=dt), c["heads_first"])
        nq, nk = _lens(c)
        s["q_lens"] = torch.tensor(nq, dtype=torch.int32, device="cuda") if c["ragged"] else None
        s["kv_lens"] = torch.tensor(nk, dtype=torch.int32, device="cuda") if c["ragged"] else None
    else:
        s.update(_adamw_state(c, rn))
    if own:
        s["plan"] = _plan(s)
    return s


def _places(c):
    """Offset, size and shape of every tensor in the flat buffers (each starts on a block of 256), and the
    buffers' length."""
    off, out = 0, []
    for shape in _shapes(c):
        n = math.prod(shape)
        out.append((off, n, shape))
        off += (n + 255) // 256 * 256
    return out, off


def _adamw_state(c, rn):
    """Flat buffers of parameters, gradients and moments in training, zero between the tensors. Sizes
    differ from block to block, as those of a vocabulary's rows do."""
    places, n = _places(c)
    nb = n // 256
    dev, block = "cuda", np.arange(nb)
    start = np.array([o // 256 for o, _, _ in places])
    which = np.searchsorted(start, block, side="right") - 1
    real = torch.zeros(n, device=dev)
    for o, size, _ in places:
        real[o:o + size] = 1.0
    real = real.view(nb, 256)
    size = torch.exp(rn(nb, 1)) * real
    s = {"p": (rn(nb, 256, std=0.02) * real).view(-1), "g": (rn(nb, 256, std=1e-3) * size).view(-1).to(DT[c["grad"]])}
    m, r = (rn(nb, 256, std=3e-4) * size).view(-1), ((rn(nb, 256, std=1e-3).abs() + 1e-5) * size).view(-1)
    # what an optimiser knows of each block: its tensor, its weight decay, its first element's index there
    s["decay"] = torch.tensor([0.1 if len(places[w][2]) > 1 else 0.0 for w in which], device=dev)[:, None]
    s["tensor"] = torch.tensor(which, device=dev)
    s["first"] = torch.tensor((block - start[which]) * 256, device=dev)
    if c["bits"] == 8:
        dither = _dither(s, 0)
        s["m"], me = _quant_m(m.view(nb, 256), dither & 0xFFFF)
        s["r"], re = _quant_r((r * r).view(nb, 256), dither >> 16)
        s["exps"] = torch.stack([me, re], dim=1).to(torch.uint8)
    else:
        s["m"], s["v"] = m, r * r
    s["low"] = s["p"].bfloat16() if c["lowp"] else None
    s["step"] = 100
    return s


LR, B1, B2, EPS, SEED = 2e-4, 0.9, 0.95, 1e-8, 12345


# ---------------------------------------------------------------- the calls of the framework
def _plan(s):
    """What a user's program builds once: configurations, and the list of tensors of an optimiser."""
    from paper_2305_19370_amd import bpt
    c = s["case"]
    if c["kind"] == "rope":
        return bpt.make_rope_config(c["B"] * c["S"], c["S"], c["H"], c["dh"], rot=c["rot"], ldx=s["X"].stride(0), layout=c["layout"],
                                    theta=c["theta"], scaling=c["scaling"], factor=c["factor"], orig_len=c["orig_len"],
                                    mscale=c["mscale"], pos0=c["pos0"], dtype=c["dtype"])
    if c["kind"] == "attn":
        return bpt.attn_config_of(s["q"], s["k"], s["v"], s["q"], causal=c["causal"], window=c["window"], sinks=c["sinks"])
    at = lambda name, o, n: s[name][o:o + n] if s.get(name) is not None else None  # noqa: E731
    second = "r" if c["bits"] == 8 else "v"
    return bpt.AdamWTensors([dict(p=at("p", o, n), g=at("g", o, n), m=at("m", o, n), p_lowp=at("low", o, n),
                                  exps=at("exps", o // 256, (n + 255) // 256), weight_decay=0.1 if len(shape) > 1 else 0.0,
                                  **{second: at(second, o, n)}) for o, n, shape in _places(c)[0]], bits=c["bits"])


def _run_own(s):
    from paper_2305_19370_amd import bpt
    c, plan = s["case"], s["plan"]
    if c["kind"] == "rope":
        x = s["X"]
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        bpt.rope_fwd(plan, x, y, s["pos"])
        if c["mode"] == "fwd":
            return {"Y": y}
        w = x.stride(0)
        dx = torch.empty((x.shape[0], w), dtype=x.dtype, device=x.device)[:, :c["H"] * c["dh"]].view(x.shape)
        bpt.rope_bwd(plan, s["dY"], dx, s["pos"])
        return {"Y": y, "dX": dx}
    if c["kind"] == "attn":
        q, k, v = s["q"], s["k"], s["v"]
        o = torch.empty_like(q)
        lse = torch.empty((c["B"], c["Hq"], c["Sq"]), dtype=torch.float32, device=q.device)
        ws = torch.empty(bpt.attn_workspace_bytes(plan, c["mode"] == "train"), dtype=torch.uint8, device=q.device)
        bpt.attn_fwd(plan, q, k, v, o, lse, ws, s["q_lens"], s["kv_lens"])
        if c["mode"] != "train":
            return {"O": o, "lse": lse}
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        bpt.attn_bwd(plan, q, k, v, o, lse, s["do"], dq, dk, dv, ws, s["q_lens"], s["kv_lens"])
        return {"O": o, "lse": lse, "dQ": dq, "dK": dk, "dV": dv}
    bpt.adamw_multi(plan, s["step"], LR, B1, B2, EPS, seed=SEED)
    return _adamw_out(s)


# ---------------------------------------------------------------- the plain forms
def _freqs(c, xp):
    """Angle per position of each pair, float64."""
    i = xp.arange(c["rot"] // 2, dtype=xp.float64)
    theta = c["theta"]
    if c["scaling"] == "base" and c["rot"] > 2:
        theta = theta * c["factor"] ** (c["rot"] / (c["rot"] - 2))
    f = theta ** (-2.0 * i / c["rot"])
    if c["scaling"] == "linear":
        f = f / c["factor"]
    if c["scaling"] == "by_parts":
        turns = c["orig_len"] * f / (2 * math.pi)
        g = ((turns - 1.0) / (32.0 - 1.0)).clip(0.0, 1.0)
        f = f * (g + (1.0 - g) / c["factor"])
    return f


def _rotate(c, x, cos, sin):
    """x [T, H, dh] in float32 or 64, cos and sin [T, 1, rot / 2]."""
    r = c["rot"]
    if c["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).reshape(*x.shape[:-1], r)
    return torch.cat([y, x[..., r:]], dim=-1)


def _run_rope(s):
    c, x = s["case"], s["X"]
    T = x.shape[0]
    pos = s["pos"].double() if s["pos"] is not None else c["pos0"] + torch.arange(T, device=x.device).remainder(c["S"]).double()
    ang = pos[:, None] * _freqs(c, torch).to(x.device)
    cos, sin = ((c["mscale"] * t).float()[:, None, :] for t in (ang.cos(), ang.sin()))
    out = {"Y": _rotate(c, x.float(), cos, sin).to(x.dtype)}
    if c["mode"] == "train":
        out["dX"] = _rotate(c, s["dY"].float(), cos, -sin).to(x.dtype)
    return out


def _grouped(t, Hkv):
    """[B, S, H, dh] as float32 [B, Hkv, G S, dh]."""
    B, S, H, dh = t.shape
    return t.permute(0, 2, 1, 3).float().reshape(B, Hkv, (H // Hkv) * S, dh)


def _ungrouped(t, H, dtype):
    B, Hkv, R, dh = t.shape
    return t.reshape(B, H, R * Hkv // H, dh).permute(0, 2, 1, 3).to(dtype)


def _mask(s):
    """[B, Sq, Skv]: which query sees which key."""
    c, dev = s["case"], s["q"].device
    nq = s["q_lens"].long() if s["q_lens"] is not None else torch.full((c["B"],), c["Sq"], device=dev)
    nk = s["kv_lens"].long() if s["kv_lens"] is not None else torch.full((c["B"],), c["Skv"], device=dev)
    i, k = torch.arange(c["Sq"], device=dev)[None, :, None], torch.arange(c["Skv"], device=dev)[None, None, :]
    p = (nk - nq)[:, None, None] + i
    ok = (k < nk[:, None, None]) & (i < nq[:, None, None])
    if c["causal"]:
        ok = ok & (k <= p)
    if c["window"]:
        ok = ok & (((p - k).abs() < c["window"]) | (k < c["sinks"]))
    return ok


def _run_attn(s):
    c = s["case"]
    q, k, v = s["q"], s["k"], s["v"]
    B, Hq, Hkv, G, dt = c["B"], c["Hq"], c["Hkv"], c["Hq"] // c["Hkv"], q.dtype
    scale = c["dh"] ** -0.5
    qf, kf, vf = _grouped(q, Hkv), _grouped(k, Hkv), _grouped(v, Hkv)
    hidden = ~_mask(s)[:, None].expand(B, G, c["Sq"], c["Skv"]).reshape(B, 1, G * c["Sq"], c["Skv"])
    x = torch.matmul(qf, kf.transpose(-1, -2)).mul_(scale).masked_fill_(hidden, -math.inf)
    m = x.amax(dim=-1, keepdim=True)
    lse = m + torch.log(torch.exp(x - m.clamp_min(-1e30)).sum(dim=-1, keepdim=True))
    p = torch.exp(x.sub_(lse.clamp_min(-1e30)))
    out = {"O": _ungrouped(torch.matmul(p, vf), Hq, dt), "lse": lse.reshape(B, Hq, c["Sq"])}
    if c["mode"] == "train":
        g = _grouped(s["do"], Hkv)
        out["dV"] = _ungrouped(torch.matmul(p.transpose(-1, -2), g), Hkv, dt)
        dp = torch.matmul(g, vf.transpose(-1, -2))
        ds = p.mul_(dp - (p * dp).sum(dim=-1, keepdim=True)).mul_(scale)
        out["dQ"] = _ungrouped(torch.matmul(ds, kf), Hq, dt)
        out["dK"] = _ungrouped(torch.matmul(ds.transpose(-1, -2), qf), Hkv, dt)
    return out


U32 = 0xFFFFFFFF


def _mix(x):
    """32 well-mixed bits of a 32-bit number (int64 tensors or ints that hold one)."""
    x = x ^ (x >> 16)
    x = (x * 0x9E3779B1) & U32
    x = x ^ (x >> 15)
    x = (x * 0x6A09E667) & U32
    return x ^ (x >> 16)


def _dither(s, step):
    """The random bits of every element, [blocks, 256]: a mix of its index in its tensor, the tensor's
    place in the list, the step and the seed."""
    key = _mix(_mix(_mix(SEED & U32) ^ (SEED >> 32) ^ step) ^ s["tensor"])
    i = s["first"][:, None] + torch.arange(256, device=key.device)[None, :]
    return _mix(i ^ key[:, None])


def _power(e):
    """2^(e - 127) of biased exponents."""
    return (e.int() << 23).view(torch.float32)


def _e4m3(y, dither):
    """Codes of y >= 0 (below 256), rounded up with the probability of its place between two codes: the 16
    bits of dither are added below the third mantissa bit. Steps below 2^-6 are all 2^-9."""
    small = y < 2.0 ** -6
    bits = (y + 2.0 ** -6 * small).view(torch.int32) + (dither.int() << 4)
    return (bits >> 20) - 120 * 8 - 8 * small.int()


def _quant_m(m, dither):
    """First moments as signed e4m3 codes, blocks scaled by a power of two: largest value in [128, 256)."""
    e = (m.abs().amax(dim=1).view(torch.int32) >> 23).clamp(27, 254)
    y = m.abs() * _power(261 - e)[:, None]
    return (_e4m3(y, dither) + 128 * (m < 0).int()).to(torch.uint8).view(-1), e


def _quant_r(v, dither):
    """Second moments' square roots as e4m3 codes; a root above zero keeps a code above zero."""
    e = ((v.amax(dim=1).view(torch.int32) >> 23) + 127) >> 1
    y = v.sqrt() * _power(261 - e)[:, None]
    return torch.maximum(_e4m3(y, dither), (v > 0).int()).to(torch.uint8).view(-1), e


def _values(codes, e):
    return codes.view(torch.float8_e4m3fn).float().view(-1, 256) * _power(e.int() - 7)[:, None]


def _run_adamw(s):
    """One step, the buffers updated in place."""
    bits, step = s["case"]["bits"], s["step"]
    g, p = s["g"].float().view(-1, 256), s["p"].view(-1, 256)
    c1, c2 = 1.0 / (1.0 - B1 ** step), 1.0 / (1.0 - B2 ** step)
    if bits == 8:
        m, v = _values(s["m"], s["exps"][:, 0]), _values(s["r"], s["exps"][:, 1]).square()
    else:
        m, v = s["m"].view(-1, 256), s["v"].view(-1, 256)
    m = B1 * m + (1.0 - B1) * g
    v = B2 * v + (1.0 - B2) * (g * g)
    p.copy_(p * (1.0 - LR * s["decay"]) - LR * (m * c1) / ((v * c2).sqrt() + EPS))
    if bits == 8:
        dither = _dither(s, step)
        mc, me = _quant_m(m, dither & 0xFFFF)
        rc, re = _quant_r(v, dither >> 16)
        s["m"].copy_(mc), s["r"].copy_(rc), s["exps"].copy_(torch.stack([me, re], dim=1))
    else:
        s["m"].copy_(m.view(-1)), s["v"].copy_(v.view(-1))
    if s["low"] is not None:
        s["low"].copy_(s["p"])
    return _adamw_out(s)


def _adamw_out(s):
    """The updated buffers; 8-bit moments as the e4m3 values that they hold beside the blocks' exponents."""
    out = {k: s[k] for k in ("p", "low", "v", "exps") if s.get(k) is not None}
    out["m"] = s["m"].view(torch.float8_e4m3fn) if s["case"]["bits"] == 8 else s["m"]
    return {**out, "r": s["r"].view(torch.float8_e4m3fn)} if s["case"]["bits"] == 8 else out


def run(state):
    if own:
        return _run_own(state)
    return {"rope": _run_rope, "attn": _run_attn, "adamw": _run_adamw}[state["case"]["kind"]](state)


# ---------------------------------------------------------------- the definitions in 64 bits
def _exact_rope(c, s):
    """Pairs as complex numbers, turned by exp(i p f)."""
    half = c["rot"] // 2
    theta = c["theta"] * (c["factor"] ** (c["rot"] / (c["rot"] - 2)) if c["scaling"] == "base" and half > 1 else 1.0)
    f = np.array([theta ** (-i / half) for i in range(half)])
    if c["scaling"] == "linear":
        f /= c["factor"]
    if c["scaling"] == "by_parts":
        keep = np.clip((c["orig_len"] / (2 * np.pi / f) - 1.0) / 31.0, 0.0, 1.0)
        f = keep * f + (1.0 - keep) * f / c["factor"]
    T = s["X"].shape[0]
    p = s["pos"].cpu().numpy().astype(np.float64) if s["pos"] is not None else c["pos0"] + np.arange(T) % c["S"] * 1.0
    turn = torch.tensor(c["mscale"] * np.exp(1j * np.outer(p, f)), device="cuda")[:, None, :]

    def turned(x, by):
        x = x.double().clone()
        a, b = ((x[..., :half], x[..., half:2 * half]) if c["layout"] == "half" else (x[..., 0:2 * half:2], x[..., 1:2 * half:2]))
        z = torch.complex(a.contiguous(), b.contiguous()) * by
        a.copy_(z.real), b.copy_(z.imag)
        return x

    out = {"Y": turned(s["X"], turn)}
    if c["mode"] == "train":
        out["dX"] = turned(s["dY"], turn.conj())
    return out


def _exact_attn(c, s):
    """Head by head, in blocks of queries."""
    B, Sq, Hq, Hkv, dh = c["B"], c["Sq"], c["Hq"], c["Hkv"], c["dh"]
    f64 = dict(dtype=torch.float64, device="cuda")
    out = {"O": torch.zeros(B, Sq, Hq, dh, **f64), "lse": torch.full((B, Hq, Sq), -math.inf, **f64)}
    if c["mode"] == "train":
        out.update(dQ=torch.zeros(B, Sq, Hq, dh, **f64), dK=torch.zeros(B, c["Skv"], Hkv, dh, **f64),
                   dV=torch.zeros(B, c["Skv"], Hkv, dh, **f64))
    scale = 1.0 / math.sqrt(dh)
    for b, (nq, nk) in enumerate(zip(*_lens(c))):
        for h in range(Hq if nk else 0):
            kv = h * Hkv // Hq
            k, v = s["k"][b, :nk, kv].double(), s["v"][b, :nk, kv].double()
            at = torch.arange(nk, device="cuda")
            for i in range(0, nq, 4096):
                rows = slice(i, min(nq, i + 4096))
                q = s["q"][b, rows, h].double()
                p = torch.arange(rows.start, rows.stop, device="cuda")[:, None] + (nk - nq)
                seen = (at <= p) if c["causal"] else torch.ones(len(q), nk, dtype=torch.bool, device="cuda")
                if c["window"]:
                    seen &= ((at - p).abs() < c["window"]) | (at < c["sinks"])
                x = torch.where(seen, (q @ k.T) * scale, -math.inf)
                lse = torch.logsumexp(x, dim=1)
                w = torch.where(seen, torch.exp(x - lse[:, None]), 0.0)
                o = w @ v
                out["O"][b, rows, h], out["lse"][b, h, rows] = o, lse
                if c["mode"] == "train":
                    do = s["do"][b, rows, h].double()
                    dx = w * (do @ v.T - (do * o).sum(dim=1, keepdim=True)) * scale
                    out["dQ"][b, rows, h] = dx @ k
                    out["dK"][b, :nk, kv] += dx.T @ q
                    out["dV"][b, :nk, kv] += w.T @ do
    return out


def _exact_adamw(c, s):
    step, g, p = s["step"], s["g"].double(), s["p"].double()
    decay = s["decay"].double().expand(-1, 256).reshape(-1)
    scale = lambda col: torch.exp2(s["exps"][:, col].double() - 134.0)[:, None].expand(-1, 256).reshape(-1)  # noqa: E731
    if c["bits"] == 8:
        m = s["m"].view(torch.float8_e4m3fn).double() * scale(0)
        v = (s["r"].view(torch.float8_e4m3fn).double() * scale(1)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = m + (1.0 - B1) * (g - m), v + (1.0 - B2) * (g * g - v)
    new = p - LR * decay * p - LR * (m / (1.0 - B1 ** step)) / (torch.sqrt(v / (1.0 - B2 ** step)) + EPS)
    out = {"p": new}
    if s["low"] is not None:
        out["low"] = new
    if c["bits"] == 32:
        return {**out, "m": m, "v": v}
    bits = _dither(s, step).reshape(-1)

    def code(x, top, bits16):
        """Value of the code next below or above x, as bits16 / 2^16 is below or above its distance."""
        y = (x.view(-1, 256) / top).view(-1) * 128.0
        unit = torch.exp2(torch.floor(torch.log2(y.clamp_min(2.0 ** -6))) - 3.0)
        return torch.floor(y / unit + bits16 / 65536.0) * unit

    def under(x):
        """The power of two at or below a block's largest value."""
        return torch.exp2(torch.floor(torch.log2(x.clamp_min(2.0 ** -100))))

    top = under(m.abs().view(-1, 256).amax(dim=1))[:, None]
    out["m"] = torch.sign(m) * code(m.abs(), top, bits & 0xFFFF)
    r = torch.sqrt(v)
    root = under(r.view(-1, 256).amax(dim=1).square() * (1 + 1e-12))
    top = torch.exp2(torch.floor(torch.log2(root) / 2.0))[:, None]
    got = code(r, top, bits >> 16)
    out["r"] = torch.where(r > 0, got.clamp_min(2.0 ** -9), got)
    return {**out, "exps": None}


def exact(case, seed):
    c, s = dict(case), prepare(case, seed)
    return {"rope": _exact_rope, "attn": _exact_attn, "adamw": _exact_adamw}[c["kind"]](c, s)
