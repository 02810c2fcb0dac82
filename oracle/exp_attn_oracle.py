"""Exponential attention in float64 on the CPU, straight from the definition, with bounds on what float32 arithmetic and bf16
roundings may change: test infrastructure, no code shared with the library.

Bounds, element by element.  A rounding to bf16 is off by at most U = 2^-8 of the value.  The library rounds the weights P that
multiply v (not those that the denominator sums), the gradients t of the products, the results, and D = dO.O is formed from the rounded O.
With ds the error of a score in float32 (products exact, d additions, a few operations of the score, at the size of the numbers that
enter) and n the number of keys, whose weights are added in float32:
    dL_i    <= sum_j P_ij ds_ij + n 2^-24
    |dO_i|  <= U |O_i| + sum_j P_ij (U + ds_ij + dL_i) |v_j|                          =: eO_i
    |dD_i|  <= sum_c |dO_ic| eO_ic
    |dP_ij| <= P_ij (ds_ij + dL_i)
    |dt_ij| <= |t_ij| (U + ds_ij + dL_i) + P_ij (dD_i + 2^-20 |dO_i|.|v_j|)
and each gradient's sums weigh those, plus U of the result."""
import math

import torch

U = 2.0 ** -8


def ranges(B, T, Tk, window=0, lo=None, hi=None):
    pos = torch.arange(T) + (Tk - T)
    first = torch.zeros(B, T, dtype=torch.long) if lo is None else lo.long()
    last = (pos + 1).expand(B, T) if hi is None else hi.long()
    if window:
        first = torch.maximum(first, pos - window + 1)
    return pos, first, last


def exp_attn(q, k, v, scale=1.0, cap=0.0, window=0, slopes=None, lo=None, hi=None, g=None, held=0.0):
    """q [B, H, T, d], k, v [B, Hk, Tk, d], g = dO (CPU tensors of any float type) -> dict of O, L, and with g dQ, dK, dV; e + name:
    the bound of that result's error.  L is -inf in rows that see nothing.  held: what a key's or value's elements are rounded to
    before they enter, relative (and 2^-24 absolute where it is not 0)."""
    q, k, v = q.double(), k.double(), v.double()
    B, H, T, d = q.shape
    Hk, Tk = k.shape[1], k.shape[2]
    pos, first, last = ranges(B, T, Tk, window, lo, hi)
    j = torch.arange(Tk)
    names = ["O", "L"] + (["dQ", "dK", "dV"] if g is not None else [])
    like = {"O": q, "L": q[..., 0], "dQ": q, "dK": k, "dV": v}
    out = {p + n: torch.zeros_like(like[n]) for n in names for p in ("", "e")}
    for b in range(B):
        see = (j >= first[b][:, None]) & (j < last[b][:, None])
        seen = see.any(0)
        some = see.any(1)
        for h in range(H):
            hk = h // (H // Hk)
            # what nobody sees, and rows that see nothing, may hold anything
            kk, vv = torch.where(seen[:, None], k[b, hk], 0.0), torch.where(seen[:, None], v[b, hk], 0.0)
            qq = torch.where(some[:, None], q[b, h], 0.0)
            x = qq @ kk.T * scale
            ds = scale * d * 2.0 ** -23 * (qq.abs() @ kk.abs().T) + 2.0 ** -22 * x.abs()
            s, w = x, torch.ones_like(x)
            if held:
                ds = ds + scale * (qq.abs() @ (held * kk.abs() + 2.0 ** -24).T)
            if cap:
                s = cap * torch.tanh(x / cap)
                w = 1.0 - torch.tanh(x / cap) ** 2
                ds = ds + 2.0 ** -20 * cap
            if slopes is not None:
                far = (pos[:, None] - j).abs().double()
                s = s - slopes[h].double() * far
                ds = ds + 2.0 ** -21 * slopes[h].abs().double() * far
            s = torch.where(see, s, -math.inf)
            L = torch.logsumexp(s, 1)
            P = torch.where(see, torch.exp(s - torch.where(some, L, 0.0)[:, None]), 0.0)
            ds = torch.where(see, ds + 2.0 ** -21 * (1.0 + torch.where(see, s, 0.0).abs()), 0.0)
            O = P @ vv
            dL = (P * ds).sum(1) + Tk * 2.0 ** -24
            eO = U * O.abs() + (P * (U + ds + dL[:, None])) @ vv.abs() + 1e-30
            if held:
                eO = eO + P @ (held * vv.abs() + 2.0 ** -24)
            out["O"][b, h], out["eO"][b, h] = O, eO
            out["L"][b, h] = torch.where(some, L, -math.inf)
            out["eL"][b, h] = dL + 2.0 ** -21 * torch.where(some, L, 0.0).abs()
            if g is None:
                continue
            gg = torch.where(some[:, None], g[b, h].double(), 0.0)
            e = gg @ vv.T - (gg * O).sum(1, keepdim=True)
            t = P * e * w * scale
            dD = (gg.abs() * eO).sum(1)
            et = t.abs() * (U + ds + dL[:, None]) + scale * P * w.abs() * (dD[:, None] + 2.0 ** -20 * (gg.abs() @ vv.abs().T))
            if cap:     # 1 - tanh^2 formed from a rounded 1 / (exp + 1)
                et = et + scale * P * e.abs() * 2.0 ** -20
            out["dQ"][b, h] = t @ kk
            out["edQ"][b, h] = U * out["dQ"][b, h].abs() + et @ kk.abs() + 1e-30
            out["dK"][b, hk] += t.T @ qq
            out["edK"][b, hk] += et.T @ qq.abs() + 1e-30
            out["dV"][b, hk] += P.T @ gg
            out["edV"][b, hk] += (P * (U + ds + dL[:, None])).T @ gg.abs() + 1e-30
    if g is not None:
        for n in ("dK", "dV"):
            out["e" + n] += U * out[n].abs()
    return out


def rotated(x, pos, cos, sin, adjacent=False):
    """float32 [..., T, d] at table rows pos [T], each operation rounded to float32; angle a = cos[t][a], sin[t][a]"""
    rot = 2 * cos.shape[1]
    c, s = cos[pos], sin[pos]
    y = x.clone()
    first, second = (slice(0, rot, 2), slice(1, rot, 2)) if adjacent else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., first], x[..., second]
    y[..., first] = a * c - b * s
    y[..., second] = b * c + a * s
    return y


def held4(x):
    """The values that 4 bits hold for float32 rows [..., d]: 32 channels share a unit and a minimum, both fp16"""
    g = x.reshape(*x.shape[:-1], -1, 32)
    nan = g.isnan().any(-1, keepdim=True)
    g = g.clamp(-65024.0, 65024.0)
    low, high = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
    unit, low = ((high - low) * torch.full_like(low, 1.0 / 15.0)).half().float(), low.half().float()
    code = torch.where(unit > 0, ((g - low) / torch.where(unit > 0, unit, 1.0)).round().clamp(0, 15), 0.0)
    return torch.where(nan, math.nan, code * unit + low).reshape(x.shape)
