"""Plain 64-bit forms of the operators around the scan, with bounds on what an implementation that rounds as the header says may be off by.

Every function returns (values, bounds) by name.  A rounding to the storage type is off by at most h = eps / 2 of the value.  A sum of n products in fp32 is off
by at most (n + 2) 2^-24 of the sum of their magnitudes.  fp32 exponentials, error functions and divisions: within 2^-20 of the value over the arguments
here (|z| < 30: the argument's own rounding, |z| 2^-24, and a few units of the function)."""
import math

import torch

U = 2.0 ** -24                     # fp32
FUNC = 2.0 ** -20                  # an fp32 activation, weight or quotient, relative
TD = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
TINY = {"f32": 1e-30, "bf16": 1e-30, "f16": 2.0 ** -25}      # half a step of the smallest numbers


def half(dtype):
    return torch.finfo(TD[dtype]).eps / 2


def act(z, name):
    """Activation, its derivative and bounds of the slopes of both."""
    if name == "none":
        return z, torch.ones_like(z), 1.0, 0.0
    if name == "gelu":
        phi = 0.5 * (1 + torch.erf(z / math.sqrt(2)))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 1.13, 0.8
    g = torch.sigmoid(z)
    if name == "sigmoid":
        return g, g * (1 - g), 0.25, 0.1
    return z * g, g + z * g * (1 - g), 1.1, 0.5


def _store(v, bound, dtype):
    """The bound of a value that is rounded to the storage type at the end."""
    return bound + half(dtype) * (v.abs() + bound) + TINY[dtype]


def product(x, P, bias, residual, gout, name, dtype, gated):
    """x [B,K,H,W], P [rows,K], ... double.  out, and with gout gin, gP, gbias."""
    B, K, H, W = x.shape
    xf = x.reshape(B, K, H * W)
    b = torch.zeros(P.shape[0], dtype=torch.float64) if bias is None else bias
    pre = P @ xf + b[:, None]
    d_pre = (K + 3) * U * (P.abs() @ xf.abs() + b.abs()[:, None])
    M = P.shape[0] // 2 if gated else P.shape[0]
    a, da, s1, s2 = act(pre[:, :M], name)
    d_a = s1 * d_pre[:, :M] + FUNC * (a.abs() + pre[:, :M].abs()) * (name != "none")
    d_da = s2 * d_pre[:, :M] + FUNC * 2 * (name != "none")
    if gated:
        u, d_u = pre[:, M:], d_pre[:, M:]
        out = a * u
        d_out = d_a * u.abs() + a.abs() * d_u + d_a * d_u + 2 * U * out.abs()
    else:
        out, d_out = a, d_a
        if residual is not None:
            out = out + residual.reshape(B, M, H * W)
            d_out = d_out + U * (out.abs() + d_out)
    shape = (B, M, H, W)
    v, e = {"out": out.reshape(shape)}, {"out": _store(out, d_out, dtype).reshape(shape)}
    if gout is None:
        return v, e
    g = gout.reshape(B, M, H * W)
    if gated:
        d_g = torch.cat((g.abs() * (d_u * da.abs() + (u.abs() + d_u) * d_da), g.abs() * d_a), 1)
        g = torch.cat((g * u * da, g * a), 1)
    else:
        d_g = g.abs() * d_da
        g = g * da
    d_g = d_g + 3 * U * g.abs()
    rounded = d_g if name == "none" and not gated else _store(g, d_g, dtype)      # as the products read it
    gin = P.t() @ g
    v["gin"] = gin.reshape(x.shape)
    mag = P.abs().t() @ (g.abs() + rounded)
    e["gin"] = _store(gin, P.abs().t() @ rounded + (P.shape[0] + 2) * U * mag, dtype).reshape(x.shape)
    n = B * H * W
    gP = torch.einsum("bmn,bkn->mk", g, xf)
    mag = torch.einsum("bmn,bkn->mk", g.abs() + rounded, xf.abs())
    v["gP"], e["gP"] = gP, _store(gP, torch.einsum("bmn,bkn->mk", rounded, xf.abs()) + (n + 2) * U * mag, dtype)
    gb = g.sum((0, 2))
    v["gbias"], e["gbias"] = gb, _store(gb, d_g.sum((0, 2)) + (n + 2) * U * (g.abs() + d_g).sum((0, 2)), dtype)
    return v, e


def attend(q, k, v, mask, gout, heads, kv, scale, dtype):
    """q [B,heads*D,H,W], k, v [B,L,kv*D], mask [B,L] bool or None, double.  out and lse, and with gout gq, gk, gv."""
    B, C, H, W = q.shape
    D, N, L, per = C // heads, H * W, k.shape[1], heads // kv
    Q = q.reshape(B, heads, D, N)
    rep = lambda t: t.reshape(B, L, kv, D).repeat_interleave(per, 2).permute(0, 2, 1, 3)          # [B,heads,L,D]
    keep = torch.ones(B, 1, L, 1, dtype=torch.bool) if mask is None else mask.reshape(B, 1, L, 1)
    K, V = (torch.where(keep, rep(t), torch.zeros((), dtype=torch.float64)) for t in (k, v))      # (what masked tokens hold is never used)
    s = scale * (K @ Q)
    d_s = (D + 4) * U * scale * (K.abs() @ Q.abs())
    s = torch.where(keep, s, torch.full((), -math.inf, dtype=torch.float64))
    top = s.amax(2, keepdim=True)
    some = torch.isfinite(top)
    w = torch.where(keep, torch.exp(s - torch.where(some, top, 0.0)), 0.0)
    total = w.sum(2, keepdim=True)
    p = w / torch.where(total > 0, total, 1.0)
    off = d_s.amax(2, keepdim=True) * 2 + FUNC + (L + 8) * U + 8 * U * torch.where(keep, (s - torch.where(some, top, 0.0)).abs(), 0.0).amax(2, keepdim=True)
    h = half(dtype)
    out = V.transpose(2, 3) @ p                                                                   # [B,heads,D,N]
    mag = V.abs().transpose(2, 3) @ p
    # weights below the type's smallest are lost: relative to the largest weight, 1 at least 2^-8 of the reference
    flush = TINY[dtype] * 256 * V.abs().sum(2).unsqueeze(3)
    d_out = (off + h + (L + 2) * U) * mag + flush
    img = lambda t: t.reshape(B, C, H, W)
    val, err = {"out": img(out)}, {"out": img(_store(out, d_out, dtype))}
    lse = (torch.where(some, top, 0.0) + torch.log(torch.where(total > 0, total, 0.0))).squeeze(2)
    val["lse"], err["lse"] = lse.reshape(B, heads, H, W), (off.squeeze(2) + FUNC * (1 + lse.abs().clamp(max=1e30))).reshape(B, heads, H, W)
    if gout is None:
        return val, err
    g = gout.reshape(B, heads, D, N)
    d_p = off * 2 * p + err["lse"].reshape(B, heads, 1, N).clamp(max=1.0) * p
    dp = V @ g
    d_dp = (D + 2) * U * (V.abs() @ g.abs())
    delta = (g * out).sum(2, keepdim=True)
    d_delta = (g.abs() * err["out"].reshape(B, heads, D, N)).sum(2, keepdim=True) + (D + L + 2) * U * (g.abs() * (out.abs() + mag)).sum(2, keepdim=True) \
        + (p * d_dp + d_p * dp.abs()).sum(2, keepdim=True)
    ds = p * (dp - delta)
    d_ds = (p + d_p) * (d_dp + d_delta) + d_p * (dp - delta).abs() + 2 * U * ds.abs()
    r_p, r_ds = _store(p, d_p, dtype), _store(ds, d_ds, dtype)                                   # as the products read them
    gq = scale * (K.transpose(2, 3) @ ds)
    e_q = scale * (K.abs().transpose(2, 3) @ (r_ds + (L + 3) * U * (ds.abs() + r_ds)))
    sum_heads = lambda t: t.reshape(B, kv, per, L, D).sum(2).permute(0, 2, 1, 3).reshape(B, L, kv * D)
    n = per * N
    gk, gv = sum_heads(scale * (ds @ Q.transpose(2, 3))), sum_heads(p @ g.transpose(2, 3))
    e_k = sum_heads(scale * ((r_ds + (n + 3) * U * (ds.abs() + r_ds)) @ Q.abs().transpose(2, 3)))
    e_v = sum_heads((r_p + (n + 3) * U * (p + r_p)) @ g.abs().transpose(2, 3))
    for name, t, e in (("gq", img(gq), img(e_q)), ("gk", gk, e_k), ("gv", gv, e_v)):
        val[name], err[name] = t, _store(t, e, dtype)
    if mask is not None:                                                                          # tokens that take no part: exactly 0
        gone = ~mask.reshape(B, L, 1).expand(B, L, kv * D)
        for name in ("gk", "gv"):
            val[name] = torch.where(gone, 0.0, val[name])
            err[name] = torch.where(gone, 0.0, err[name])
    return val, err


def check(got, val, err, what):
    """Every element of every output within its bound; infinities where they belong."""
    for name in val:
        if name not in got or got[name] is None:
            continue
        a, r, b = got[name].detach().double().cpu(), val[name], err[name]
        fine = torch.isfinite(r)
        assert torch.equal(a[~fine], r[~fine]), (what, name, "infinities")
        assert torch.isfinite(a[fine]).all(), (what, name, "not finite")
        d = (a - r).abs()[fine]
        worst = (d - b[fine])
        assert (worst <= 0).all(), (what, name, "off by", float(d.max()), "at a bound of", float(b[fine][worst.argmax()]), "elements outside", int((worst > 0).sum()))
