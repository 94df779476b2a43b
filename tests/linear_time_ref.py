"""The gated recurrence and the distillation loss in float64 on the CPU, step by step and from whole logits, and bounds on the
error of results that are computed in float32 and rounded once.

U32 is half a step of float32, the relative error of one rounding. The hardware's exponential, reciprocal and root are within a step
(2 U32), sums, products and divisions within U32."""
import math
from typing import Dict, Optional

import torch

from long_context_ref import U32

F64 = torch.float64


def sigma_error(g):
    """Relative error of a sigmoid: the argument's product with log2(e) is off by its rounding and the constant's (2 U32 |g| of
    the exponential), exponential and reciprocal 2 each, a sum and a product 1 each."""
    return (2 * g.abs() + 6) * U32


def recur(x, r, i, lam, c: float, h0=None, lens=None, dy=None, dhT=None) -> Dict[str, torch.Tensor]:
    """y, hT and, given dy, the gradients, each with its bound as "name_err" (without the last rounding of y, dx, dr, di)."""
    x, r, i, lam = (t.detach().cpu().to(F64) for t in (x, r, i, lam))
    B, S, D = x.shape
    n = torch.full((B,), S) if lens is None else lens.detach().cpu().long().clamp(0, S)
    live = (torch.arange(S)[None, :] < n[:, None])[..., None]
    x, r, i = (torch.where(live, t, torch.zeros((), dtype=F64)) for t in (x, r, i))
    sp = torch.logaddexp(lam, torch.zeros_like(lam))
    R, I = torch.sigmoid(r), torch.sigmoid(i)
    l = -c * sp * R
    a, s = torch.exp(l), -torch.expm1(2 * l)
    m, u = torch.sqrt(s), I * x
    # relative errors: l from softplus (8: exponential, logarithm and sum of the library), three products and R; a from l's absolute
    # error and its own exponential; m from 1 - a^2: where the series ends (2 l = -1/16) a^2 is off by 2 (a's error + U32), and
    # 1 - a^2 is 1/17 at least, halved by the root; where it holds, l's error and 8 roundings
    el = 12 * U32 + sigma_error(r)
    ea = l.abs() * el + 3 * U32
    em = torch.where(2 * l > -0.0625, 0.5 * el + 8 * U32, 17 * (ea + U32) + 4 * U32)
    # an s below the smallest normal number may be taken as 0: m, and -l / m, which is m / 2 there, are then at most 2^-63
    tiny = torch.where(s < 2.0 ** -125, 2.0 ** -62, 0.0)
    eu = sigma_error(i) + 2 * U32
    eb = em + eu
    a1, b = torch.where(live, a, 1.0), torch.where(live, m * u, 0.0)
    h = torch.zeros(B, D, dtype=F64) if h0 is None else h0.detach().cpu().to(F64).clone()
    eh = torch.zeros_like(h)
    # one step: its products and sums, and those of the joins of runs that carry it on (at most 16: 2 in a wave, 8 in a workgroup
    # and its tail), charge the terms they touch
    J = 16 * U32
    H, EH, y = [h], [eh], []
    for t in range(S):
        lv = live[:, t]
        nh = a1[:, t] * h + b[:, t]
        eh = torch.where(lv, a1[:, t] * eh + (ea[:, t] + J) * (a1[:, t] * h).abs() + (eb[:, t] + J) * b[:, t].abs() + (tiny * u.abs())[:, t] + U32 * nh.abs(), eh + J * h.abs())
        h = nh
        H.append(h)
        EH.append(eh)
        y.append(torch.where(lv, h, 0.0))
    out = {"y": torch.stack(y, 1), "y_err": torch.where(live, torch.stack(EH[1:], 1), 0.0), "hT": h, "hT_err": eh}
    if dy is None:
        return out
    dy = torch.where(live, dy.detach().cpu().to(F64), 0.0)
    e = torch.zeros(B, D, dtype=F64) if dhT is None else dhT.detach().cpu().to(F64).clone()
    ee = torch.zeros_like(e)
    d, ed = [None] * S, [None] * S
    for t in range(S - 1, -1, -1):
        lv = live[:, t]
        d[t] = dy[:, t] + e
        ed[t] = ee + U32 * d[t].abs()
        ne = a1[:, t] * d[t]
        # terms that enter a step with opposite signs are charged with their sizes
        ee = torch.where(lv, a1[:, t] * ed[t] + (ea[:, t] + J) * a1[:, t] * (dy[:, t].abs() + e.abs()), ee + J * e.abs())
        e = ne
    out["dh0"], out["dh0_err"] = e, ee
    d, ed, Hp, EHp = torch.stack(d, 1), torch.stack(ed, 1), torch.stack(H[:-1], 1), torch.stack(EH[:-1], 1)
    zero = torch.zeros((), dtype=F64)
    q = torch.where(s > 0, a * a * u * l / torch.where(s > 0, m, 1.0), zero)
    p = l * a * Hp
    w = torch.where(live, d * (p - q), zero)
    ew = torch.where(live, ed * (p - q).abs() + d.abs() * ((el + ea + 3 * U32) * p.abs() + (l * a).abs() * EHp + (2 * ea + eu + el + em + 6 * U32) * q.abs() + tiny * u.abs()), zero)
    fx, fi = torch.where(live, m * I, zero), torch.where(live, m * u * torch.sigmoid(-i), zero)
    out["dr"], out["dr_err"] = w * torch.sigmoid(-r), (ew + (sigma_error(r) + 2 * U32) * w.abs()) * torch.sigmoid(-r)
    out["dx"], out["dx_err"] = d * fx, ed * fx.abs() + (d * fx).abs() * (em + sigma_error(i) + 4 * U32) + (d * I).abs() * tiny
    out["di"], out["di_err"] = d * fi, ed * fi.abs() + (d * fi).abs() * (em + eu + sigma_error(i) + 4 * U32) + (d * u).abs() * tiny
    ratio = torch.sigmoid(lam) / sp
    # sums of w: at most 128 + 16 + rows / 16 additions of what they hold, charged with the sizes of the terms
    adds = 160 + B * ((S + 127) // 128) / 16
    out["dlam"], out["dlam_err"] = ratio * w.sum((0, 1)), ratio * (ew.sum((0, 1)) + (adds + 24) * U32 * w.abs().sum((0, 1)))
    return out


def distill(h, W, V: int, values, index, tau: float, soft: float, hard: float = 0.0, targets=None, weights=None,
            dloss: float = 1.0, half: float = U32, half_dw: Optional[float] = None) -> Dict[str, torch.Tensor]:
    """loss, tokens, dh and dW from the whole logits, each with its bound as "name_err". half: half a step of h's type, to which the
    logits' gradient and dh are rounded; half_dw: that of dW's."""
    h, W, values = (t.detach().cpu().to(F64) for t in (h, W, values))
    index = index.detach().cpu().long()
    T, D = h.shape
    K = index.shape[1]
    w = torch.full((T,), 1.0 / T, dtype=F64) if weights is None else weights.detach().cpu().to(F64)
    y = torch.full((T,), -1) if targets is None or not hard else targets.detach().cpu().long()
    valid = (index >= 0) & (index < V) & (values > -math.inf)
    some, has = valid.any(dim=1), (y >= 0) & (y < V)
    left = (w != 0) & (some | has)
    h = torch.where(left[:, None], h, 0.0)
    z = h @ W[:, :V]
    # sums of D exact products
    dz = (D + 2) * U32 * (h.abs() @ W[:, :V].abs())
    v = torch.where(valid, values / tau, -math.inf)
    mx = torch.where(some, v.amax(dim=1), 0.0)[:, None]
    e = torch.exp(v - mx)
    q = e / torch.where(some, e.sum(dim=1), 1.0)[:, None]
    # exponents: a difference, its factor and the product (and log2 e in the factor); a sum of K, a quotient, K of the doubles
    eq = torch.where(valid, (mx - v), 0.0).nan_to_num(posinf=0.0) * 4 * U32 + (2 * K + 8) * U32
    Q = torch.zeros(T, V, dtype=F64).scatter_add_(1, torch.where(valid, index, 0), torch.where(valid, q, 0.0))
    EQ = torch.zeros(T, V, dtype=F64).scatter_add_(1, torch.where(valid, index, 0), torch.where(valid, q * eq, 0.0))

    def soft_of(scale):
        s = z * scale
        lse = torch.logsumexp(s, dim=1, keepdim=True)
        p = torch.exp(s - lse)
        span = s.amax(dim=1, keepdim=True) - s
        # each weight: its logit, the exponent's roundings; a sum of at most 64 + V / 64 parts and their rescaling; the logarithm
        e_lse = (p * (dz * scale + (5 * span + 8) * U32)).sum(dim=1, keepdim=True) + (V / 64 + 80) * U32 + 8 * U32 * lse.abs()
        e_p = dz * scale + e_lse + (6 * (s.abs() + lse.abs()) + 8) * U32        # relative
        return s, lse, p, e_lse, e_p

    s, lt, pt, elt, ept = soft_of(1.0 / tau)
    logq = torch.log(torch.where(Q > 0, Q, 1.0))
    term = torch.where(Q > 0, logq - s + lt, 0.0)
    kl = (Q * term).sum(dim=1)
    ekl = (EQ * (term.abs() + 1) + Q * (dz / tau + elt + 8 * U32 * (logq.abs() + s.abs() + lt.abs()))).sum(dim=1) + (K + 8) * U32 * (Q * term.abs()).sum(dim=1)
    s1, l1, p1, el1, ep1 = soft_of(1.0)
    at = torch.where(has, y, 0)[:, None]
    ce = torch.where(has, (l1 - z.gather(1, at))[:, 0], 0.0)
    ece = torch.where(has, (el1 + dz.gather(1, at) + 4 * U32 * (l1.abs() + z.gather(1, at).abs()))[:, 0], 0.0)
    kl, ekl, ce, ece = (torch.where(left, t, 0.0) for t in (kl, ekl, ce, ece))
    out = {"tokens": torch.stack([kl, ce]), "tokens_err": torch.stack([ekl, ece])}
    sums = torch.stack([(w * kl).sum(), (w * ce).sum()])
    adds = (T / 1024 + 14) * U32
    esums = torch.stack([(w.abs() * (ekl + adds * kl.abs())).sum(), (w.abs() * (ece + adds * ce.abs())).sum()])
    total = soft * tau * tau * sums[0] + hard * sums[1]
    out["loss"] = torch.cat([total[None], sums])
    out["loss_err"] = torch.cat([(soft * tau * tau * (esums[0] + 5 * U32 * sums[0].abs()) + hard * (esums[1] + 3 * U32 * sums[1].abs()))[None], esums])
    gs, gh = (dloss * w * soft * tau * some)[:, None], (dloss * w * hard * has)[:, None]
    hot = torch.zeros(T, V, dtype=F64)
    hot[torch.arange(T)[has], y[has]] = 1.0
    G = gs * (pt - Q) + gh * (p1 - hot)
    eG = gs.abs() * (pt * ept + EQ) + gh.abs() * p1 * ep1 + 8 * U32 * (gs.abs() * (pt + Q) + gh.abs() * (p1 + hot)) + half * G.abs()
    G, eG = torch.where(left[:, None], G, 0.0), torch.where(left[:, None], eG, 0.0)
    Wv = W[:, :V]
    dh = G @ Wv.t()
    out["dh"], out["dh_err"] = dh, eG @ Wv.abs().t() + (V + 2) * U32 * (G.abs() @ Wv.abs().t()) + half * dh.abs()
    dW = torch.zeros_like(W)
    dW[:, :V] = h.t() @ G
    e = torch.zeros_like(W)
    e[:, :V] = h.abs().t() @ eG + (T + 2) * U32 * (h.abs().t() @ G.abs())
    out["dW"], out["dW_err"] = dW, e + (U32 if half_dw is None else half_dw) * dW.abs()
    return out
