"""Plain float64 forms of attention with a window and sinks, of rotary positions and of AdamW with 8-bit
moments, written from their formulas, and bounds on what rounding can do to a kernel's results."""
import math

import torch

U32 = 2.0 ** -24                                    # half a step of fp32, relative
HALF = {torch.float64: 2.0 ** -53, torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def visible(Sq, Skv, nq, nk, causal, window, sinks, device="cpu"):
    """[Sq, Skv]: which query sees which key (nq, nk: the lengths that exist)."""
    i, k = torch.arange(Sq, device=device)[:, None], torch.arange(Skv, device=device)[None, :]
    p = nk - nq + i
    ok = (k < nk) & (i < nq)
    if causal:
        ok = ok & (k <= p)
    if window:
        ok = ok & (((p - k).abs() < window) | (k < sinks))
    return ok


def attention(q, k, v, do=None, causal=True, window=0, sinks=0, scale=None, q_lens=None, kv_lens=None):
    """O, lse and, given do, dQ, dK, dV in float64, and for each the bound on a kernel's error.

    A kernel forms scores of inputs as they are with fp32 accumulation, weights P (rounded to the inputs'
    type before they meet V and dO), dS = P (dP - Delta) (rounded so too) and rounds its results once. With h
    the type's half step, u that of fp32 and M >= sum |q k| scale:
      score: 2 dh u M; hence P (1 + eP), eP = u (2 dh M + 16) + h
      O: eP sum P|v| + h |O|, Delta: sum |dO| dO_err, dS: (eP + h) |P (dP - Delta)| + P Delta_err + u dh P sum |dO v|
    and sums of n terms add n u of the sum of magnitudes."""
    B, Sq, Hq, dh = q.shape
    Skv, Hkv = k.shape[1], k.shape[2]
    G, h = Hq // Hkv, HALF[q.dtype]
    dev = q.device
    scale = dh ** -0.5 if scale is None else scale
    z = lambda *s: torch.zeros(*s, dtype=torch.float64, device=dev)  # noqa: E731
    out = {"O": z(B, Sq, Hq, dh), "lse": torch.full((B, Hq, Sq), -math.inf, dtype=torch.float64, device=dev)}
    err = {"O": z(B, Sq, Hq, dh), "lse": z(B, Hq, Sq)}
    if do is not None:
        for n, s in (("dQ", q.shape), ("dK", k.shape), ("dV", v.shape)):
            out[n], err[n] = z(*s), z(*s)
    for b in range(B):
        nq = Sq if q_lens is None else int(q_lens[b])
        nk = Skv if kv_lens is None else int(kv_lens[b])
        ok = visible(Sq, Skv, nq, nk, causal, window, sinks, dev)
        rows, keys = ok.any(dim=1), ok.any(dim=0)
        if not bool(ok.any()):
            continue
        for hq in range(Hq):
            hk = hq // G
            # what nobody sees may hold anything
            Q, K, V = (torch.where(m[:, None], t.double(), 0.0) for t, m in
                       ((q[b, :, hq], rows), (k[b, :, hk], keys), (v[b, :, hk], keys)))
            M = float((Q.abs() @ K.abs().T).max()) * scale
            eP = U32 * (2 * dh * M + 16) + (h if q.dtype == torch.bfloat16 else 0.0)
            n = int(ok.sum(dim=1).max())
            S = torch.where(ok, Q @ K.T * scale, -math.inf)
            lse = torch.logsumexp(S, dim=1)
            P = torch.where(ok, torch.exp(S - torch.where(rows, lse, 0.0)[:, None]), 0.0)
            O = P @ V
            out["O"][b, :, hq], out["lse"][b, hq] = O, lse
            eO = (eP + n * U32) * (P @ V.abs()) + h * O.abs()
            err["O"][b, :, hq] = eO
            err["lse"][b, hq] = torch.where(rows, U32 * (2 * dh * M + n + 16) + U32 * 8 * torch.where(rows, lse, 0.0).abs(), 0.0)
            if do is None:
                continue
            dO = torch.where(rows[:, None], do[b, :, hq].double(), 0.0)
            dP = dO @ V.T
            D = (dO * O).sum(dim=1, keepdim=True)
            eD = (dO.abs() * eO).sum(dim=1, keepdim=True) + U32 * dh * (dO * O).abs().sum(dim=1, keepdim=True)
            dS = P * (dP - D)
            eS = (eP + h) * dS.abs() + P * eD + U32 * 2 * dh * P * (dO.abs() @ V.abs().T + D.abs())
            out["dQ"][b, :, hq] = dS @ K * scale
            err["dQ"][b, :, hq] = ((eS + n * U32 * dS.abs()) @ K.abs()) * scale + h * (dS @ K * scale).abs()
            out["dK"][b, :, hk] += dS.T @ Q * scale
            err["dK"][b, :, hk] += ((eS + Sq * G * U32 * dS.abs()).T @ Q.abs()) * scale
            out["dV"][b, :, hk] += P.T @ dO
            err["dV"][b, :, hk] += ((eP + Sq * G * U32) * P).T @ dO.abs()
    if do is not None:
        for n in ("dK", "dV"):
            err[n] += h * out[n].abs()
    return out, err


def check(got, ref, err, what):
    """Every element of got within its bound (plus fp32's smallest steps); the same places not finite."""
    got = got.double()
    fine = torch.isfinite(ref)
    assert torch.equal(fine, torch.isfinite(got)), f"{what}: not finite in other places"
    d = torch.where(fine, (got - torch.where(fine, ref, 0.0)).abs(), 0.0)
    lim = err * 1.01 + 1e-30                        # the bounds are first order in the half steps
    bad = d > lim
    worst = float((d / lim.clamp_min(1e-30)).max()) if d.numel() else 0.0
    print(f"{what}: at most {worst:.2f} of the bound", flush=True)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, up to {worst:.2f} of the bound"


# ---------------------------------------------------------------- rotary positions
def rope_freqs(rot, theta=10000.0, scaling="none", factor=1.0, orig_len=0, beta_fast=32.0, beta_slow=1.0):
    half = rot // 2
    if scaling == "base":
        theta = theta * factor ** (rot / (rot - 2))
    f = [theta ** (-2.0 * i / rot) for i in range(half)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "by_parts":
        g = [min(1.0, max(0.0, (orig_len * x / (2 * math.pi) - beta_slow) / (beta_fast - beta_slow))) for x in f]
        f = [x * (y + (1 - y) / factor) for x, y in zip(f, g)]
    return torch.tensor(f, dtype=torch.float64)


def rope(x, positions, freqs, layout, mscale=1.0, sign=1.0):
    """x [rows, H, dh] turned in float64."""
    x = x.double()
    half = freqs.numel()
    ang = sign * positions.double()[:, None] * freqs[None, :]
    c, s = (mscale * t[:, None, :] for t in (torch.cos(ang), torch.sin(ang)))
    y = x.clone()
    a = x[..., :half] if layout == "half" else x[..., 0:2 * half:2]
    b = x[..., half:2 * half] if layout == "half" else x[..., 1:2 * half:2]
    at = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    return y


# ---------------------------------------------------------------- 8-bit moments
def e4m3_values():
    """The value of each of the 128 codes without a sign, from the format's definition."""
    v = []
    for c in range(127):
        e, m = c >> 3, c & 7
        v.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return torch.tensor(v + [math.nan], dtype=torch.float64)


def moments(codes, exps, col, signed):
    """float64 moments that bytes [n] and exponents [blocks, 2] stand for."""
    c = codes.cpu().long()
    v = e4m3_values()[c & 127] * torch.where(c >= 128, -1.0, 1.0).double()
    assert signed or not bool((c >= 128).any())
    n = c.numel()
    e = exps.cpu().view(-1, 2)[:, col].double().repeat_interleave(256)[:n]
    return v * torch.exp2(e - 134.0)
