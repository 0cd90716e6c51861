"""Plain fp64 forms of the operators without an expert cache, with bounds on
what fp32 sums may be off by (not collected by pytest).

u = 2^-24 is half a step of fp32 relative to the value; a sum of n products in
any order and association is off by at most n u times the sum of the products'
magnitudes (first order)."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def pow2(e):
    """2^e, exactly."""
    return torch.ldexp(torch.ones((), dtype=torch.float64), torch.as_tensor(e, dtype=torch.int32))


def quantize(v):
    """fp64 [..][n] -> (e4m3 values, exponents, scale bytes) from the definition:
    E the smallest exponent >= -127 with amax <= 448 2^E, values to the nearest
    m 2^k with m of four bits and k >= -9, ties to even."""
    b = v.double().reshape(*v.shape[:-1], v.shape[-1] // 32, 32)
    bad = ~torch.isfinite(b).all(-1)
    amax = torch.where(bad, 1.0, b.abs().amax(-1))
    m, x = torch.frexp(amax)  # amax = m 2^x, 1/2 <= m < 1; 448 = 7/8 2^9
    E = torch.where(m <= 0.875, x - 9, x - 8)
    E = torch.where(amax == 0, -127, E).clamp(min=-127)
    t = b * pow2(-E).unsqueeze(-1)
    step = pow2(torch.frexp(t.abs().clamp(min=2.0 ** -6))[1] - 4)
    q = torch.where(bad.unsqueeze(-1), math.nan, torch.round(t / step) * step)
    return q.reshape(v.shape), E, torch.where(bad, 255, E + 127)


def dequantize(q8, byte):
    """fp64 values of e4m3 bytes and scale bytes (CPU tensors)."""
    q = q8.view(torch.float8_e4m3fn).double().reshape(*q8.shape[:-1], q8.shape[-1] // 32, 32)
    s = torch.where(byte == 255, math.nan, pow2(byte.int() - 127))
    return (q * s.unsqueeze(-1)).reshape(q8.shape)


def norm(residual, delta, weight, eps):
    """(r in the residual's type, h in fp64)."""
    r = residual.double()
    if delta is not None:
        # the addition is fp32: exact in fp64, rounded to fp32, then to the type
        r = (r + delta.double()).float().to(residual.dtype).double()
    h = r / torch.sqrt((r * r).mean(1, keepdim=True) + eps)
    return r.to(residual.dtype), h if weight is None else h * weight.double()


def norm_error(d):
    """Relative error of fp32 h before its rounding: a thread's chain of squares
    and the tree above it, halved by the root, and five more roundings."""
    return U * ((max(64, d / 256) + 24) / 2 + 6)


def route(h, w_router, bias, K):
    """(selected, gates, logits) of [T][d] rows."""
    z = h.double() @ w_router.double().t()
    if bias is not None:
        z = torch.where(bias == -math.inf, -math.inf, z + bias.double())
    z = z.float()
    T = z.shape[0]
    sel = torch.full((T, K), -1, dtype=torch.int32)
    gates = torch.zeros((T, K), dtype=torch.float64)
    for t in range(T):
        row = [math.inf if v != v else v for v in z[t].tolist()]
        nan = [v != v for v in z[t].tolist()]
        order = sorted(range(len(row)), key=lambda e: (not nan[e], -row[e], e))[:K]
        order = [e for e in order if nan[e] or row[e] > -math.inf]
        for k, e in enumerate(order):
            sel[t, k] = e
        if order:
            zs = z[t, order].double()
            gates[t, :len(order)] = torch.exp(zs - zs[0]) / torch.exp(zs - zs[0]).sum()
    return sel, gates, z


def experts(x, sel, gates, weights, d, F):
    """(y, bound on its fp32 error) of x [T][d]; weights(e) gives the fp64
    W_gate [F][d], W_up [F][d], W_down [d][F] of expert e."""
    T = x.shape[0]
    x = x.double()
    y = torch.zeros((T, d), dtype=torch.float64)
    err = torch.zeros((T, d), dtype=torch.float64)
    mag = torch.zeros((T, d), dtype=torch.float64)
    for e in sorted(set(sel.flatten().tolist()) - {-1}):
        t, k = (sel == e).nonzero(as_tuple=True)
        wg, wu, wd = weights(e)
        g, u = x[t] @ wg.t(), x[t] @ wu.t()
        dg, du = d * U * (x[t].abs() @ wg.abs().t()), d * U * (x[t].abs() @ wu.abs().t())
        s = torch.sigmoid(g)
        a = g * s * u
        # |silu'| <= 1.1; the exponential, the sum, the quotient, the product and the
        # intermediate's last bits: ten half steps
        da = 1.1 * dg * (u.abs() + du) + (g * s).abs() * du + 10 * U * a.abs()
        o, m = a @ wd.t(), a.abs() @ wd.abs().t()
        do = da @ wd.abs().t() + 3 * F * U * (m + da @ wd.abs().t())
        w = gates[t, k].unsqueeze(1)
        y.index_add_(0, t, w * o)
        mag.index_add_(0, t, w * o.abs())
        err.index_add_(0, t, w * do)
    # gates: two exponentials' errors, the sum of K and a quotient; then K products and additions
    K = sel.shape[1]
    return y, err + (2 * K + 16) * U * (mag + err)


def split_expert(w, d, F):
    w = w.double()
    return w[:F * d].view(F, d), w[F * d:2 * F * d].view(F, d), w[2 * F * d:].view(d, F)
