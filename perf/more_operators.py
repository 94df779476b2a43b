"""A gated linear recurrence and the distillation loss of a language-model head, as cases that can be timed and compared.

Kinds of case:

  recur    the recurrence over [B, S, D]: mode "train" (forward, then the gradients), "fwd" (a prompt) or "token" (one new
           token of each sequence)
  distill  a student's head trained on its teacher's largest logits: mode "train" (loss, then dh and dW) or "fwd" (the loss
           alone)

With `own` false a pass computes the plain form, elementary torch operations in float32; with
`own` true it makes the calls of paper_2305_19370_amd.bpt that a user's program makes.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "f32": torch.float32}

RECUR = dict(kind="recur", mode="train", dtype="bf16", c=8.0, joint=False, ragged=False, h0=False)
DISTILL = dict(kind="distill", mode="train", dtype="bf16", tau=1.0, soft=1.0, hard=0.0, ragged=False, pad=0.0)


def listed():
    return [
        # one new token of each of 8 sequences at the 1B-shaped layer's width: a serving loop, where latency counts
        dict(RECUR, name="recur_token_b8_d2048", mode="token", B=8, S=1, D=2048, h0=True),
        # one new token of each of 1024 sequences at the 13B-shaped layer's width, gates and input from one projection
        dict(RECUR, name="recur_token_b1024_d5120", mode="token", B=1024, S=1, D=5120, h0=True, joint=True),
        # float32, odd lengths, a padded batch whose last sequence is empty, a state carried in: a piece of a longer document
        dict(RECUR, name="recur_f32_b3_s1003_d768", B=3, S=1003, D=768, dtype="f32", ragged=True, h0=True),
        # the GPT-XL benchmark's 16384 tokens of width 2048, gates and input from one projection
        dict(RECUR, name="recur_train_b4_s4096_d2048", B=4, S=4096, D=2048, joint=True),
        # the trajectory workload's 96000 tokens of width 1024: one long sequence
        dict(RECUR, name="recur_train_b1_s96000_d1024", B=1, S=96000, D=1024),
        # a prompt of 65536 tokens at the 13B-shaped layer's width, forward alone
        dict(RECUR, name="recur_fwd_s65536_d5120", mode="fwd", B=1, S=65536, D=5120),
        # the float32 parity workload's width with a small vocabulary: the smallest call
        dict(DISTILL, name="distill_f32_t512_d256_v1000", T=512, D=256, V=1000, K=8, dtype="f32", tau=2.0, hard=0.5),
        # a small model's padded batch, lists of unequal lengths, targets beside the teacher
        dict(DISTILL, name="distill_t4000_d768_v50257", T=4000, D=768, V=50257, K=32, tau=2.0, soft=0.7, hard=0.3, ragged=True,
             pad=0.2),
        # the loss of a validation batch of odd length
        dict(DISTILL, name="distill_fwd_t1003_d2048_v50257", mode="fwd", T=1003, D=2048, V=50257, K=100),
        # the 1B-shaped model's head on 8192 tokens
        dict(DISTILL, name="distill_t8192_d2048_v50257", T=8192, D=2048, V=50257, K=64),
        # the 7B-shaped model's head on 16384 tokens, two temperatures
        dict(DISTILL, name="distill_t16384_d4096_v50257", T=16384, D=4096, V=50257, K=128, tau=1.5, soft=0.9, hard=0.1),
    ]


# ---------------------------------------------------------------- drawn cases
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_recur(rng):
    while True:
        mode = rng.choice(("train", "train", "train", "fwd", "token"))
        B = _log(rng, 1, 1024 if mode == "token" else 64)
        c = dict(RECUR, mode=mode, B=B, S=1 if mode == "token" else _log(rng, 2, 100000), D=8 * _log(rng, 1, 640),
                 dtype=rng.choice(("bf16", "bf16", "f32")), joint=rng.random() < 0.4, ragged=rng.random() < 0.3,
                 h0=mode == "token" or rng.random() < 0.5)
        n = c["B"] * c["S"] * c["D"] * (2 if c["dtype"] == "f32" else 1)
        if n <= (1.2e8 if mode == "train" else 3.3e8):
            return c


def _draw_distill(rng):
    while True:
        dtype = rng.choice(("bf16", "bf16", "bf16", "f32"))
        hard = rng.choice((0.0, 0.3, 0.5))
        c = dict(DISTILL, mode=rng.choice(("train", "train", "fwd")), T=_log(rng, 1, 20000), D=64 * _log(rng, 1, 64),
                 V=_log(rng, 100, 60000), dtype=dtype, tau=rng.choice((1.0, 1.0, 0.7, 2.0, 4.0)), soft=1.0 - hard, hard=hard,
                 ragged=rng.random() < 0.5, pad=rng.choice((0.0, 0.0, 0.1, 0.5)))
        c["K"] = min(_log(rng, 1, 256), c["V"])
        n = c["T"] * c["D"] * c["V"] * (10 if dtype == "f32" else 1)
        if n <= 3.3e12 and c["T"] * c["V"] <= 8.3e8:
            return c


def draw(rng):
    return rng.choice((_draw_recur, _draw_distill))(rng)


# ---------------------------------------------------------------- what a case cannot do without
def _lens(c):
    """Steps of each sequence: unequal where ragged, the last of several sequences empty."""
    B, S = c["B"], c["S"]
    if not c["ragged"]:
        return [S] * B
    n = [S - (b * S) // B for b in range(B)]
    if B > 1:
        n[-1] = 0
    return n


def _ldw(c):
    return (c["V"] + 63) // 64 * 64


def work(case):
    c = case
    e = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "recur":
        n, full, row = sum(_lens(c)) * c["D"], c["B"] * c["S"] * c["D"], 4 * c["B"] * c["D"]
        # x and both gates in, y out; then x, the gates and dy in, dx and the gates' gradients out; states; lambda and its gradient
        by = (3 * n + full) * e + row * (2 if c["h0"] else 1) + 4 * c["D"]
        if c["mode"] == "train":
            by += (4 * n + 3 * full) * e + row * (2 if c["h0"] else 1) + 8 * c["D"]
        return {"bytes": by, "flops": (20.0 + (35.0 if c["mode"] == "train" else 0.0)) * n}
    T, D, V, K = c["T"], c["D"], c["V"], c["K"]
    by = (T * D + D * V) * e + T * K * 8 + 8 * T + (4 * T if c["hard"] else 0) + (4 * T if c["pad"] else 0)
    if c["mode"] == "train":
        by += (T * D + D * V) * e
    return {"bytes": by, "flops": (6.0 if c["mode"] == "train" else 2.0) * T * D * V}


# ---------------------------------------------------------------- inputs
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def prepare(case, seed):
    c, g = dict(case), _gen(seed)
    dt = DT[c["dtype"]]
    rn = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda").mul_(std)  # noqa: E731
    s = {"case": c}
    if c["kind"] == "recur":
        B, S, D = c["B"], c["S"], c["D"]
        if c["joint"]:                               # columns of one projection
            p = rn(B, S, 3 * D).to(dt)
            s["x"], s["r"], s["i"] = p[..., :D], p[..., D:2 * D], p[..., 2 * D:]
        else:
            s["x"], s["r"], s["i"] = (rn(B, S, D).to(dt) for _ in range(3))
        # decays between 0.9 and 0.999 where the gate is fully open
        sp = -torch.log(torch.rand(D, generator=g, device="cuda") * 0.099 + 0.9) / c["c"]
        s["lam"] = torch.log(torch.expm1(sp))
        s["h0"] = rn(B, D) if c["h0"] else None
        s["lens"] = torch.tensor(_lens(c), dtype=torch.int32, device="cuda") if c["ragged"] else None
        if c["mode"] == "train":
            s["dy"] = rn(B, S, D).to(dt)
            s["dhT"] = rn(B, D) if c["h0"] else None
    else:
        T, D, V, K = c["T"], c["D"], c["V"], c["K"]
        s["h"] = rn(T, D).to(dt)
        W = rn(D, _ldw(c), std=2.0 / math.sqrt(D))
        W[:, V:] = 0.0                               # padding columns
        s["W"] = W.to(dt)
        # the teacher: its K largest of logits that resemble the student's
        s["top"], s["index"] = torch.empty(T, K, device="cuda"), torch.empty(T, K, dtype=torch.int32, device="cuda")
        for t0 in range(0, T, 4096):
            ht = s["h"][t0:t0 + 4096].float() * 0.8 + rn(min(4096, T - t0), D, std=0.6)
            v, k = (ht.bfloat16() @ s["W"][:, :V].bfloat16().contiguous()).float().topk(K, dim=1)
            s["top"][t0:t0 + 4096], s["index"][t0:t0 + 4096] = v + 1e-3 * rn(*v.shape), k.int()
        if c["ragged"]:                              # as many as hold most of the teacher's mass; the rest marked -1
            n = torch.randint(0 if T > 1 else 1, K + 1, (T, 1), generator=g, device="cuda")
            s["index"].masked_fill_(torch.arange(K, device="cuda") >= n, -1)
        s["targets"] = torch.randint(0, V, (T,), generator=g, device="cuda", dtype=torch.int32) if c["hard"] else None
        s["weights"] = None
        if c["pad"]:                                 # padding tokens count nothing, the others all the same
            real = (torch.rand(T, generator=g, device="cuda") >= c["pad"]).float()
            real[0] = 1.0
            s["weights"] = real / real.sum()
    if own:
        s["plan"] = _plan(s)
    return s


# ---------------------------------------------------------------- the calls of the framework
def _plan(s):
    """What a user's program builds once."""
    from paper_2305_19370_amd import bpt
    c = s["case"]
    if c["kind"] == "recur":
        return bpt.GatedRecurrence(c=c["c"])
    return bpt.DistillLoss(bpt.make_distill_config(c["T"], c["D"], c["V"], c["K"], ldw=_ldw(c), tau=c["tau"], soft=c["soft"],
                                                   hard=c["hard"], dtype=c["dtype"], grad_dtype=c["dtype"]))


def _run_own(s):
    c, plan = s["case"], s["plan"]
    if c["kind"] == "recur":
        train = c["mode"] == "train"
        y, hT, saved = plan.forward(s["x"], s["r"], s["i"], s["lam"], h0=s["h0"], lens=s["lens"], save=train)
        if not train:
            return {"y": y, "hT": hT}
        g = plan.backward(s["x"], s["r"], s["i"], s["lam"], saved, s["dy"], dhT=s["dhT"], h0=s["h0"], lens=s["lens"])
        return {"y": y, "hT": hT, "dx": g["dx"], "dr": g["dr"], "di": g["di"], "dlam": g["dlam"],
                "dh0": g["dh0"] if c["h0"] else None}
    loss, tokens, saved = plan.forward(s["h"], s["W"], s["top"], s["index"], targets=s["targets"], weights=s["weights"])
    if c["mode"] == "fwd":
        return {"loss": loss, "tokens": tokens}
    dh, dW = plan.backward(s["h"], s["W"], saved)
    return {"loss": loss, "tokens": tokens, "dh": dh, "dW": dW}


# ---------------------------------------------------------------- the plain forms
def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along dimension 1 from h_{-1} = 0, by doubling: spans of 1, 2, 4 .. steps joined."""
    n = 1
    while n < a.shape[1]:
        b = torch.cat([b[:, :n], b[:, n:] + a[:, n:] * b[:, :-n]], dim=1)
        a = torch.cat([a[:, :n], a[:, n:] * a[:, :-n]], dim=1) if 2 * n < a.shape[1] else a
        n *= 2
    return b


def _recur_plain(s):
    c, dt, f = s["case"], s["x"].dtype, torch.float32
    x, gr, gi, lam = s["x"].float(), s["r"].float(), s["i"].float(), s["lam"]
    B, S, D = x.shape
    r, i = 1.0 / (1.0 + torch.exp(-gr)), 1.0 / (1.0 + torch.exp(-gi))
    sp = torch.log1p(torch.exp(-lam.abs())) + lam.clamp(min=0.0)
    la = -c["c"] * sp * r                            # log of the decay
    m = torch.sqrt(-torch.expm1(2.0 * la))
    a, b = torch.exp(la), m * (i * x)
    live = None
    if s["lens"] is not None:
        live = (torch.arange(S, device=x.device)[None, :] < s["lens"][:, None])[..., None]
        a, b = torch.where(live, a, 1.0), torch.where(live, b, 0.0)
    h0 = s["h0"] if s["h0"] is not None else torch.zeros(B, D, dtype=f, device=x.device)
    b[:, 0] += a[:, 0] * h0
    h = _scan(a, b)
    out = {"y": (h if live is None else torch.where(live, h, 0.0)).to(dt), "hT": h[:, -1].clone()}
    if c["mode"] != "train":
        return out
    dy = s["dy"].float()
    if live is not None:
        dy = torch.where(live, dy, 0.0)
    if s["dhT"] is not None:
        dy[:, -1] += s["dhT"]
    one = torch.ones(B, 1, D, dtype=f, device=x.device)
    d = _scan(torch.cat([one, a[:, 1:].flip(1)], dim=1), dy.flip(1)).flip(1)   # d_t = dy_t + a_{t+1} d_{t+1}
    prev = torch.cat([h0[:, None], h[:, :-1]], dim=1)
    dl = d * (a * prev - a * a / m * (i * x))        # of the logarithm of the decay
    du = d * m
    if live is not None:
        dl, du = torch.where(live, dl, 0.0), torch.where(live, du, 0.0)
    sl = 1.0 / (1.0 + torch.exp(-lam))
    out.update(dx=(du * i).to(dt), dr=(dl * la * (1.0 - r)).to(dt), di=(du * x * i * (1.0 - i)).to(dt),
               dlam=(dl * r).sum(dim=(0, 1)) * (-c["c"]) * sl, dh0=a[:, 0] * d[:, 0] if c["h0"] else None)
    return out


def _teacher(c, top, index, V, f):
    """The teacher's probabilities over its list, the list's places, and whether it has any."""
    keep = (index >= 0) & (index < V)
    v = torch.where(keep, top.to(f) / c["tau"], -math.inf)
    mx = v.amax(dim=1, keepdim=True)
    some = mx > -math.inf
    e = torch.exp(v - torch.where(some, mx, 0.0))
    q = e / torch.where(some, e.sum(dim=1, keepdim=True), 1.0)
    return q, torch.where(keep, index, 0).long(), some.to(f)


def _lse(z):
    mx = z.amax(dim=1, keepdim=True)
    return mx + torch.log(torch.exp(z - mx).sum(dim=1, keepdim=True))


def _distill_plain(s):
    c, h, W = s["case"], s["h"].float(), s["W"].float()
    T, V, tau = c["T"], c["V"], c["tau"]
    z = h @ W[:, :V]
    q, at, some = _teacher(c, s["top"], s["index"], V, torch.float32)
    w = (s["weights"] if s["weights"] is not None else torch.full((T,), 1.0 / T, device=h.device))[:, None]
    lt = _lse(z / tau)
    logq = torch.log(torch.where(q > 0.0, q, 1.0))
    kl = some * lt + (q * (logq - z.gather(1, at) / tau)).sum(dim=1, keepdim=True)
    ce = torch.zeros_like(kl)
    if c["hard"]:
        l1, y = _lse(z), s["targets"].long()[:, None]
        ce = l1 - z.gather(1, y)
    tokens = torch.cat([kl, ce], dim=1).t() * (w != 0.0).t()    # tokens of no weight are left out
    kl, ce = (w * kl).sum(), (w * ce).sum()
    out = {"loss": torch.stack([c["soft"] * tau * tau * kl + c["hard"] * ce, kl, ce]), "tokens": tokens}
    if c["mode"] == "fwd":
        return out
    G = torch.exp(z / tau - lt) * (w * some * (c["soft"] * tau))
    G.scatter_add_(1, at, -(w * (c["soft"] * tau)) * q)
    if c["hard"]:
        G += torch.exp(z - l1) * (w * c["hard"])
        G.scatter_add_(1, y, -c["hard"] * w)
    dW = torch.zeros_like(W)
    dW[:, :V] = h.t() @ G
    out.update(dh=(G @ W[:, :V].t()).to(s["h"].dtype), dW=dW.to(s["W"].dtype))
    return out


def run(state):
    if own:
        return _run_own(state)
    return _recur_plain(state) if state["case"]["kind"] == "recur" else _distill_plain(state)


# ---------------------------------------------------------------- from the definitions, in 64 bits
def _recur_exact(s):
    """The recurrence step by step."""
    c, f = s["case"], torch.float64
    x, gr, gi = (s[k].to(f) for k in ("x", "r", "i"))
    B, S, D = x.shape
    lam = s["lam"].to(f)
    nats = -c["c"] * torch.logaddexp(lam, torch.zeros_like(lam)) * torch.sigmoid(gr)
    a, i, m = nats.exp(), torch.sigmoid(gi), (-torch.expm1(2 * nats)).sqrt()
    step = torch.arange(S, device=x.device)[None, :, None]
    n = s["lens"].long()[:, None, None] if s["lens"] is not None else torch.full((B, 1, 1), S, device=x.device)
    past = step >= n
    a, drive = a.masked_fill(past, 1.0), (m * i * x).masked_fill(past, 0.0)
    first = s["h0"].to(f) if s["h0"] is not None else torch.zeros(B, D, dtype=f, device=x.device)
    H = torch.empty(S + 1, B, D, dtype=f, device=x.device)
    H[0] = first
    rows = H.unbind(0)
    for t, (at, bt) in enumerate(zip(a.unbind(1), drive.unbind(1))):
        torch.addcmul(bt, at, rows[t], out=rows[t + 1])
    after = H[1:].transpose(0, 1)
    out = {"y": after.masked_fill(past, 0.0), "hT": H[S].clone()}
    if c["mode"] != "train":
        return out
    dy = s["dy"].to(f).masked_fill(past, 0.0)
    if s["dhT"] is not None:
        dy[:, -1] += s["dhT"].to(f)
    G = torch.empty(S, B, D, dtype=f, device=x.device)
    rows, back, decay = G.unbind(0), dy.unbind(1), a.unbind(1)
    rows[S - 1].copy_(back[S - 1])
    for t in range(S - 2, -1, -1):
        torch.addcmul(back[t], decay[t + 1], rows[t + 1], out=rows[t])
    G = G.transpose(0, 1)
    out["dh0"] = a[:, 0] * G[:, 0] if c["h0"] else None
    dnats = (G * (a * H[:-1].transpose(0, 1) - (2 * nats).exp() / m * i * x)).masked_fill(past, 0.0)
    dgate = (G * m).masked_fill(past, 0.0)
    out["dx"], out["di"] = dgate * i, dgate * x * i * (1 - i)
    out["dr"] = dnats * nats * torch.sigmoid(-gr)
    out["dlam"] = -c["c"] * torch.sigmoid(lam) * (dnats * torch.sigmoid(gr)).sum(dim=(0, 1))
    return out


def _distill_exact(s):
    """The loss and its gradients, a thousand tokens at a time."""
    c, f = s["case"], torch.float64
    T, V, tau = c["T"], c["V"], c["tau"]
    h, W = s["h"].to(f), s["W"][:, :V].to(f)
    w = s["weights"].to(f) if s["weights"] is not None else torch.full((T,), 1.0 / T, dtype=f, device=h.device)
    tokens = torch.zeros(2, T, dtype=f, device=h.device)
    dh, dW = torch.empty_like(h), torch.zeros(s["W"].shape, dtype=f, device=h.device)
    for t0 in range(0, T, 1024):
        t = slice(t0, t0 + 1024)
        z = h[t] @ W
        idx = s["index"][t].long()
        has = (idx >= 0) & (idx < V)
        val = (s["top"][t].to(f) / tau).masked_fill(~has, -math.inf)
        any_ = has.any(dim=1)
        q = torch.zeros_like(val)
        q[any_] = torch.softmax(val[any_], dim=1)
        target = torch.zeros_like(z).scatter_add_(1, idx.clamp(min=0), q.masked_fill(~has, 0.0))
        logp = torch.log_softmax(z / tau, dim=1)
        # sum q log q of the entries, minus sum q log p
        tokens[0, t] = torch.special.xlogy(q, q).sum(dim=1) - (target * logp).sum(dim=1)
        G = c["soft"] * tau * (logp.exp() * any_[:, None] - target)
        if c["hard"]:
            y = s["targets"][t].long()
            log1 = torch.log_softmax(z, dim=1)
            tokens[1, t] = -log1[torch.arange(len(y), device=y.device), y]
            hot = log1.exp()
            hot[torch.arange(len(y), device=y.device), y] -= 1.0
            G += c["hard"] * hot
        if c["mode"] == "train":
            G *= w[t][:, None]
            dh[t] = G @ W.t()
            dW[:, :V] += h[t].t() @ G
    tokens *= w != 0.0
    kl, ce = (tokens * w).sum(dim=1)
    out = {"loss": torch.stack([c["soft"] * tau * tau * kl + c["hard"] * ce, kl, ce]), "tokens": tokens}
    if c["mode"] == "train":
        out.update(dh=dh, dW=dW)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    return _recur_exact(s) if case["kind"] == "recur" else _distill_exact(s)
