"""Plain attention in 64 bits over keys and values as they are given, with the error that the formulas allow a kernel: for shared
prefixes and for quantised caches."""
import math

import torch

UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}      # largest relative error of one rounding


def attend(q, k, v, sees, far, softcap=0.0, slopes=None, scale=None, weights=None, tiny=None):
    """(out, lse, out_tolerance, lse_tolerance) of one request: q [n, heads, d] of its type, k and v [key heads, keys, d] in 64 bits, sees
    [n, keys], far [n, keys] = key's position - query's.

    Tolerances, for a unit `weights` of the weights' type (default: q's), and sums of D products in 32 bits: a score is off by at
    most e = D * 2^-23 * scale * sum|q||k| (each of D additions rounds or cuts one unit) plus a few 2^-22 of its own
    size for scale, cap, bias and the change to log2, so a weight by 2e relative to their sum, and by `weights` for its
    rounding (plus, in float16, `tiny` of the largest weight below the normal numbers); the result rounds once more."""
    n, heads, d = q.shape
    kv, keys, _ = k.shape
    group = heads // kv
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    u = UNIT[q.dtype]
    w_unit = u if weights is None else weights
    tiny = (2.0 ** -25 if w_unit == 2.0 ** -11 else 0.0) if tiny is None else tiny
    out = torch.zeros((n, heads, d), dtype=torch.float64, device=q.device)
    lse = torch.full((n, heads), -math.inf, dtype=torch.float64, device=q.device)
    out_tol, lse_tol = torch.zeros_like(out), torch.zeros_like(lse)
    if n == 0 or keys == 0:
        return out, lse, out_tol, lse_tol
    used = sees.any(0)
    for h in range(heads):
        kh, vh = k[h // group].clone(), v[h // group].clone()
        kh[~used] = 0
        vh[~used] = 0
        qh = q[:, h].double()
        x = qh @ kh.T * scale
        e = d * 2.0 ** -23 * scale * (qh.abs() @ kh.abs().T)
        if softcap:
            x = softcap * torch.tanh(x / softcap)
            e = e + softcap * 2.0 ** -20
        if slopes is not None:
            x = x + slopes[h].double() * far
        e = e + 2.0 ** -21 * x.abs()
        x = torch.where(sees, x, -math.inf)
        top = x.amax(1, keepdim=True)
        base = torch.where(torch.isneginf(top), 0.0, top)
        w = torch.where(sees, torch.exp(x - base), 0.0)
        total = w.sum(1, keepdim=True)
        w = torch.where(total != 0, w / total, 0.0)
        bad = ~torch.isfinite(vh).all(1)
        clean = torch.where(torch.isfinite(vh), vh, 0.0)
        o = w @ clean
        for key in bad.nonzero()[:, 0].tolist():                  # 0 * inf: only the queries that see such a value have it
            o = torch.where(sees[:, key:key + 1], o + w[:, key:key + 1] * torch.where(torch.isfinite(vh[key]), 0.0, vh[key]), o)
        eb = torch.where(sees, e, 0.0).amax(1, keepdim=True)
        a = w @ clean.abs()
        out[:, h] = o
        out_tol[:, h] = u * o.abs() + (w_unit + 2 * eb + 2.0 ** -18) * a + tiny * keys * clean.abs().amax()
        lse[:, h] = (base + total.log())[:, 0]
        lse_tol[:, h] = eb[:, 0] + 2.0 ** -18 + 2.0 ** -21 * torch.where(torch.isfinite(lse[:, h]), lse[:, h].abs(), 0.0)
    return out, lse, out_tol, lse_tol


def assert_near(got, want):
    """dict(out, lse) within the tolerances of (out, lse, out_tolerance, lse_tolerance); not a number where that is wanted."""
    out, lse, out_tol, lse_tol = want
    d = (got["out"].double() - out).abs()
    same = (got["out"].double() == out) | (torch.isnan(out) & torch.isnan(got["out"]))
    assert ((d <= out_tol) | same).all(), f"out is off by {(d / out_tol.clamp(min=1e-12)).nan_to_num(9e9).max().item():.3g} of the tolerance"
    dl = (got["lse"].double() - lse).abs()
    same = (got["lse"].double() == lse) | (torch.isnan(lse) & torch.isnan(got["lse"]))
    assert ((dl <= lse_tol) | same).all(), f"lse is off by {(dl / lse_tol.clamp(min=1e-12)).nan_to_num(9e9).max().item():.3g} of the tolerance"
