"""Plain 64-bit forms of the log-probabilities and losses over vocabulary rows (torch on the CPU), with closed-form gradients,
and the tolerances of the 32-bit kernels, as arrays beside the results.

Rounding errors of the kernels, h = 2^-24 (half a step of float):
  exponentials   e = 2^t, t = z log2 e - m: t is rounded once (h |t|, i.e. h |t| ln 2 of e), the exponential itself is good to a
                 step (2 h).  In a sum over the row the terms' errors weigh like the terms: sum p |t| ln 2 <= H + |ln s| <= ln V.
  sums           a chain of one addition per vector of a lane (turns), 8 inside a vector, 12 across the workgroup and the slices.
  so             |d lse| <= h (ln V + 2 + turns + 20) =: r, and the same relative error for 1 / s.
  entropy        weights |t| on the same errors: <= r (1 + H + ln V).
  KL             terms e dd, dd = (z - zr) log2 e - c with two roundings: r (sum p |dd| + |c - lse + lse_ref| + 1), |dd| <= |D| + |D_x|.
  gradient       p (k0 + ...): the errors of p and the three products, <= (r + h (|t| + 12)) p (sum of the coefficients' magnitudes),
                 that of a at the token (4 h), then half a step of the type (float 2^-24, bf16 2^-8).
"""
import math

import numpy as np
import torch

H24 = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def rows(z, x, zr=None):
    """z [..., V] any float type, x [...]: dict of 64-bit results."""
    z = z.double()
    V = z.shape[-1]
    lse = torch.logsumexp(z, -1)
    lnp = z - lse[..., None]
    p = lnp.exp()
    lnp0 = torch.where(p > 0, lnp, 0.0)
    H = -(p * lnp0).sum(-1)
    known = (x >= 0) & (x < V)
    at = torch.where(known, x, 0).long()[..., None]
    lp = torch.where(known, lnp.gather(-1, at)[..., 0], math.nan)
    out = dict(p=p, lnp=lnp0, lse=lse, H=H, lp=lp, at=at, known=known)
    # vectors that a lane may add up one after the other (a row in one slice of 256 lanes at the most), float being the longer
    out["r"] = H24 * (math.log(V) + 22 + V / (4 * 256) + 1)
    if zr is not None:
        zr = zr.double()
        lnq = zr - torch.logsumexp(zr, -1)[..., None]
        D = torch.where(p > 0, lnp - lnq, 0.0)
        out["D"], out["kl"] = D, (p * D).sum(-1)
        Dx = (lnp - lnq).gather(-1, at)[..., 0].abs()
        out["spread"] = (p * D.abs()).sum(-1) + torch.where(torch.isfinite(Dx), Dx, (torch.logsumexp(z, -1) - torch.logsumexp(zr, -1)).abs()) + 1.0
    return out


def tol_lp(o):
    return H24 * o["lp"].abs() + o["r"]


def tol_H(o):
    V = o["p"].shape[-1]
    return H24 * o["H"] + o["r"] * (1.0 + o["H"] + math.log(V))


def tol_kl(o):
    return H24 * o["kl"].abs() + 2 * o["r"] * o["spread"]


def grad(o, a, c=None, k=None, dtype=torch.float32, a_err=0.0, k_err=0.0):
    """a (1[j=x] - p) - c p (ln p + H) + k p (D - KL), and its tolerance.  a_err: error of a itself (it may hang on a log-probability)."""
    p, V = o["p"], o["p"].shape[-1]
    a = a.double()
    g = -a[..., None] * p
    g.scatter_add_(-1, o["at"], a[..., None])
    a_err = torch.as_tensor(a_err, dtype=torch.float64).expand_as(a)
    t = -(o["lnp"] - o["lnp"].amax(-1, keepdim=True))
    rel = o["r"] + H24 * (t + 12)
    size = a.abs()[..., None] * p
    tol = rel * size + a_err[..., None] * p
    at_x = torch.zeros_like(p).scatter_add_(-1, o["at"], (4 * H24 * a.abs() + a_err)[..., None])
    if c is not None:
        c = c.double()
        part = (o["lnp"] + o["H"][..., None]) * p
        g = g - c[..., None] * part
        tol = tol + c.abs()[..., None] * p * (rel * (o["lnp"].abs() + o["H"][..., None]) + tol_H(o)[..., None] + 4 * H24 * math.log(V) + o["r"])
    if k is not None:
        k = k.double()
        g = g + k[..., None] * p * (o["D"] - o["kl"][..., None])
        tol = tol + k.abs()[..., None] * p * (rel * (o["D"].abs() + o["kl"].abs()[..., None]) + (2 * tol_kl(o) + 8 * H24 * o["spread"])[..., None])
    return g, HALF[dtype] * g.abs() + tol + at_x + 1e-37


def policy(z, x, adv, weight=None, old=None, ref=None, zref=None, lo=0.2, hi=0.2, kl_coef=0.0, ent=0.0, scale=1.0):
    o = rows(z, x, zref)
    w = torch.ones_like(o["lp"]) if weight is None else weight.double()
    on = w != 0
    A = adv.double()
    A = A[:, None].expand_as(w) if A.dim() < w.dim() else A
    lp = o["lp"]
    ratio = torch.exp(lp - old.double()) if old is not None else torch.where(torch.isnan(lp), lp, 1.0)
    free, held = ratio * A, ratio.clamp(1.0 - float(np.float32(lo)), 1.0 + float(np.float32(hi))) * A
    clipped = held < free
    term = torch.where(A == 0, 0.0, -torch.where(clipped, held, free))
    a = torch.where((A == 0) | clipped, 0.0, -free)
    a_err = torch.where((A == 0) | clipped, 0.0, free.abs() * (o["r"] + 2 * H24))
    term_err = a_err.clone()
    kl = torch.zeros_like(lp)
    tkl = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        kl = torch.expm1(d) - d
        tkl = torch.expm1(d).abs() * o["r"] + o["r"] ** 2 + H24 * kl
        a = a - kl_coef * torch.expm1(d)
        a_err = a_err + kl_coef * torch.exp(d) * (o["r"] + 2 * H24)
    if zref is not None:
        kl, tkl = o["kl"], tol_kl(o)
    if kl_coef:
        term, term_err = term + kl_coef * kl, term_err + abs(kl_coef) * tkl
    if ent:
        term, term_err = term - ent * o["H"], term_err + abs(ent) * tol_H(o)
    zero = lambda v: torch.where(on, v, 0.0)  # noqa: E731
    term = zero(term)
    W = zero(w * scale)
    g, tg = grad(o, zero(a * W), c=-W * ent if ent else None, k=W * kl_coef if zref is not None and kl_coef else None, dtype=z.dtype,
                 a_err=zero(a_err * W.abs()))
    g, tg = (torch.where(on[..., None], v, 0.0) for v in (g, tg))
    term_err = zero(term_err)
    return dict(loss=zero(w * term).sum(), loss_tol=zero(w.abs() * term_err).sum() + H24 * zero(w * term).sum().abs() + 1e-30,
                term=term, term_tol=term_err + H24 * term.abs(), lp=zero(lp), lp_tol=zero(tol_lp(o)), H=zero(o["H"]), H_tol=zero(tol_H(o)),
                kl=zero(kl), kl_tol=zero(tkl), g=g, g_tol=tg)


def preference(z, x, weight=None, ref=None, pair_weight=None, kind="logistic", beta=0.1, margin=0.0, smoothing=0.0, scale=1.0):
    o = rows(z, x)
    P = z.shape[0] // 2
    w = torch.ones_like(o["lp"]) if weight is None else weight.double()
    on = w != 0
    rf = torch.zeros_like(w) if ref is None else ref.double()
    per = torch.where(on, w * (o["lp"] - rf), 0.0)
    score = per.sum(1)
    score_tol = (torch.where(on, w, 0.0).abs() * o["r"]).sum(1) + H24 * score.abs()
    D = score[:P] - score[P:]
    D_err = score_tol[:P] + score_tol[P:]
    beta, margin, e = (float(np.float32(v)) for v in (beta, margin, smoothing))
    if kind == "squared":
        m = D - margin
        d = m - 0.5 / beta
        pair, slope, s_err, l_err = d * d, 2 * d, 2 * D_err, 2 * d.abs() * D_err
        m_err = D_err
    else:
        m = beta * D - margin
        m_err = beta * D_err
        if kind == "hinge":
            pair, slope = (1 - m).clamp_min(0.0), torch.where(m < 1, -beta, 0.0).double()
            s_err, l_err = torch.zeros_like(m), m_err
        else:
            sp = torch.nn.functional.softplus
            soft = lambda v: torch.where(v > 30, v + torch.exp(-v), sp(v, threshold=1000.0))  # noqa: E731
            pair = (1 - e) * soft(-m) + e * soft(m)
            slope = beta * (e * torch.sigmoid(m) - (1 - e) * torch.sigmoid(-m))
            s_err, l_err = beta * m_err, m_err
    pw = torch.full((P,), 1.0 / P, dtype=torch.float64) if pair_weight is None else pair_weight.double()
    use = pw != 0
    loss = torch.where(use, pw * pair, 0.0).sum()
    coef = torch.where(use, scale * pw * slope, 0.0)
    c_err = torch.where(use, scale * pw.abs() * (s_err + 4 * H24 * slope.abs()), 0.0)
    both = torch.cat([coef, -coef])[:, None]
    a = torch.where(on, both * torch.where(on, w, 0.0), 0.0)
    g, tg = grad(o, a, dtype=z.dtype, a_err=torch.cat([c_err, c_err])[:, None] * torch.where(on, w, 0.0).abs())
    g, tg = (torch.where((on & (both != 0))[..., None], v, 0.0) for v in (g, tg))
    zero = lambda v: torch.where(on, v, 0.0)  # noqa: E731
    return dict(loss=loss, loss_tol=(torch.where(use, pw, 0.0).abs() * l_err).sum() + 2 * H24 * loss.abs() + 1e-30,
                pair=pair, pair_tol=l_err + 2 * H24 * pair.abs() + 1e-30, margin=m, margin_tol=m_err + 2 * H24 * m.abs(),
                score=score, score_tol=score_tol + 1e-30, lp=zero(o["lp"]), lp_tol=zero(tol_lp(o)), g=g, g_tol=tg)


def near(got, want, tol, what=""):
    got, want, tol = got.detach().cpu().double(), want.detach().cpu().double(), torch.as_tensor(tol).cpu().double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    ok = same | ((got - want).abs() <= tol)
    if not bool(ok.all()):
        at = tuple(torch.nonzero(~ok)[0].tolist())
        raise AssertionError(f"{what} at {at}: {got[at].item()!r}, expected {want[at].item()!r}, off by "
                             f"{abs(got[at].item() - want[at].item()):.3g}, allowed {tol.expand_as(got)[at].item():.3g}; "
                             f"{int((~ok).sum())} of {ok.numel()}")
