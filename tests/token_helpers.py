"""Plain float64 forms of the operators around the feed-forward products, and the error bounds their kernels are held to.

Bounds are elementwise and come from the arithmetic: half a step for the rounding to a tensor's type, and for the float
arithmetic in front of it a number of roundings (2^-24 each) on the magnitudes that enter: a sum over a row or a column takes at
most SUM of them (32 terms a thread one after another, 5 in a warp, 16 among warps, or 64 rows and 16 row slots), a
normalised value a handful more."""
import math

import numpy as np
import torch

from ffn_helpers import HALF, act, dact

U = 2.0 ** -24
SUM = 96
NORMS = {"none": 0, "rms": 1, "layer": 2}


# ---- dropout ------------------------------------------------------------------------------------------------------
def philox(counter, key):
    """Philox 4x32-10 on Python integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(rows, cols, p, key, step, site=0, row0=0):
    """rows x cols truth values and the factor of what stays, from the documented counter (vectorised over groups)."""
    cut = int(math.floor(p * 65536 + 0.5))
    per = -(-cols // 8)
    n = (np.arange(row0, row0 + rows, dtype=np.uint64)[:, None] * np.uint64(per) + np.arange(per, dtype=np.uint64)[None]).reshape(-1)
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    key, step = key & (2 ** 64 - 1), step & (2 ** 64 - 1)
    c = [n & low, (n >> sh) | np.uint64(site << 8), np.full_like(n, step & 0xFFFFFFFF), np.full_like(n, step >> 32)]
    k = [key & 0xFFFFFFFF, key >> 32]
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> sh) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> sh) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    halves = np.stack([h for w in c for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 1).reshape(rows, per * 8)[:, :cols]
    return torch.from_numpy(halves >= np.uint64(cut)), (65536.0 / (65536 - cut) if cut < 65536 else 0.0)


# ---- join ---------------------------------------------------------------------------------------------------------
def moments(v, kind, eps):
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros(v.shape[0], 1, dtype=v.dtype)
    return mean, 1.0 / torch.sqrt(((v - mean) ** 2).mean(1, keepdim=True) + eps)


def normed(v, kind, eps):
    """Normalised rows, 1 / deviation, and the bound of the error of the former in float."""
    if kind == "none":
        return v, None, torch.zeros_like(v)
    mean, r = moments(v, kind, eps)
    n = (v - mean) * r
    err = 2 * SUM * U * (n.abs() + (r * v.abs().mean(1, keepdim=True) if kind == "layer" else 0.0)) + 4 * U * r * (v.abs() + mean.abs())
    return n, r, err


def affine(n, w, b):
    n = n * w if w is not None else n
    return n + b if b is not None else n


def rows_of_gate(gate, gate_rows, rows):
    if gate is None:
        return torch.ones(1, dtype=torch.float64)
    return gate.repeat_interleave(gate_rows, 0)[:rows] if gate_rows else gate


def join_forward(u, x, c):
    """s and its bound before the rounding; c: a dict of options and float64 vectors."""
    n, _, en = normed(u, c["post"], c["eps"])
    v = affine(n, c["w_post"], c["b_post"])
    w = 1.0 if c["w_post"] is None else c["w_post"].abs()
    ev = en * w + 3 * U * ((n * w).abs() + (0.0 if c["b_post"] is None else c["b_post"].abs()))
    k = c["beta"] * rows_of_gate(c["gate"], c["gate_rows"], u.shape[0]) * c["mask"]
    xa = 0.0 if x is None else c["alpha"] * x
    s = xa + torch.where(c["mask"] == 0, torch.zeros_like(v), k * v)
    return s, k.abs() * ev + 4 * U * ((k * v).abs() + (0.0 if x is None else xa.abs()))


def pre_forward(s, c):
    n, _, en = normed(s, c["pre"], c["eps"])
    w = 1.0 if c["w_pre"] is None else c["w_pre"].abs()
    y = affine(n, c["w_pre"], c["b_pre"])
    return y, en * w + 3 * U * ((n * w).abs() + (0.0 if c["b_pre"] is None else c["b_pre"].abs()))


def norm_back(n, r, kind, g, en, eg):
    """Gradient in front of a norm from that of its normalised rows, and its bound."""
    if kind == "none":
        return g, eg
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    layer = 1.0 if kind == "layer" else 0.0
    d = r * (g - layer * mean(g) - n * mean(g * n))
    big = r * (g.abs() + layer * mean(g.abs()) + n.abs() * mean((g * n).abs()))
    err = r * (eg + layer * mean(eg) + n.abs() * mean(eg * n.abs() + en * g.abs()) + en * mean((g * n).abs())) + 2 * SUM * U * big
    return d, err


def join_backward(u, s, dy, ds, c):
    """All gradients with their bounds before the rounding to their type."""
    rows, cols = (dy if dy is not None else ds).shape
    one = torch.ones(cols, dtype=torch.float64)
    z = torch.zeros(rows, cols, dtype=torch.float64)
    d, ed = (ds, z) if ds is not None else (z, z)
    out = {}
    if c["pre"] != "none":
        n, r, en = normed(s, c["pre"], c["eps"])
        w = one if c["w_pre"] is None else c["w_pre"]
        g = dy * w
        b, eb = norm_back(n, r, c["pre"], g, en, 2 * U * g.abs())
        d, ed = d + b, ed + eb + 2 * U * (d.abs() + b.abs())
        out["dw_pre"] = ((dy * n).sum(0), (dy.abs() * en + SUM * U * (dy * n).abs()).sum(0))
        out["db_pre"] = (dy.sum(0), SUM * U * dy.abs().sum(0))
    out["dx"] = (c["alpha"] * d, abs(c["alpha"]) * ed + 2 * U * (c["alpha"] * d).abs())
    gate = rows_of_gate(c["gate"], c["gate_rows"], rows)
    base, ebase = c["beta"] * c["mask"] * d, (c["beta"] * c["mask"]).abs() * ed + 3 * U * (c["beta"] * c["mask"] * d).abs()
    dv, edv = base * gate, ebase * gate.abs() + 2 * U * (base * gate).abs()
    if u is None:
        out["du"] = (dv, edv)
        return out
    n, r, en = normed(u, c["post"], c["eps"])
    w = one if c["w_post"] is None else c["w_post"]
    b = 0 * one if c["b_post"] is None else c["b_post"]
    v, ev = n * w + b, en * w.abs() + 3 * U * ((n * w).abs() + b.abs())
    dg, edg = base * v, ebase * v.abs() + base.abs() * ev + 2 * U * (base * v).abs()
    if c["gate"] is not None:
        if c["gate_rows"] == 0:
            out["dgate"] = (dg.sum(0), (edg + SUM * U * dg.abs()).sum(0))
        else:
            k = -(-rows // c["gate_rows"])
            at = torch.arange(rows) // c["gate_rows"]
            zero = torch.zeros(k, cols, dtype=torch.float64)
            out["dgate"] = (zero.index_add(0, at, dg), zero.index_add(0, at, edg + SUM * U * dg.abs()))
    out["dw_post"] = ((dv * n).sum(0), (edv * n.abs() + dv.abs() * en + SUM * U * (dv * n).abs()).sum(0))
    out["db_post"] = (dv.sum(0), (edv + SUM * U * dv.abs()).sum(0))
    out["du"] = norm_back(n, r, c["post"], dv * w, en, edv * w.abs() + 2 * U * (dv * w).abs())
    return out


# ---- recurrence ----------------------------------------------------------------------------------------------------
def gates(f):
    return torch.sigmoid(f), torch.sigmoid(-f)


def slack(dt):
    """Relative error of the smaller of a and 1 - a, and the error of an activation relative to max(1, |o|)."""
    return (2.0 ** -20, 2.0 ** -18) if dt == torch.bfloat16 else (2.0 ** -21, 2.0 ** -20)


def recurrence(f, v, o, h0, name, coupled, dt):
    """One sequence (steps x channels, float64): h, y, their bounds before the rounding of y; a step at a time."""
    eg, ea = slack(dt)
    a, other = gates(f)
    b = other * v if coupled else v
    small = torch.minimum(a, other)
    h, big, err = h0, h0.abs(), torch.zeros_like(h0)
    hs, es = [], []
    for t in range(f.shape[0]):
        err = a[t] * err + (4 * U * a[t] + eg * small[t]) * big + (4 * U + (eg if coupled else 0.0)) * b[t].abs()
        big = a[t] * big + b[t].abs()
        h = a[t] * h + b[t]
        hs.append(h)
        es.append(err)
    hs = torch.stack(hs) if hs else torch.zeros_like(f)
    es = torch.stack(es) if es else torch.zeros_like(f)
    if o is None:
        return hs, es, hs, es
    p = act(o, name)
    return hs, es, p * hs, p.abs() * es + ea * o.abs().clamp(min=1.0) * hs.abs() + 2 * U * (p * hs).abs()


def recurrence_backward(f, v, o, h0, dy, dh1, name, coupled, dt):
    """df, dv, do, dh0 with bounds, one sequence."""
    eg, ea = slack(dt)
    a, other = gates(f)
    small = torch.minimum(a, other)
    hs, eh, _, _ = recurrence(f, v, None, h0, name, coupled, dt)
    before = torch.cat([h0[None], hs[:-1]]) if len(hs) else hs
    ebefore = torch.cat([torch.zeros_like(h0)[None], eh[:-1]]) if len(hs) else eh
    if o is None:
        e, ee, do = dy, torch.zeros_like(dy), None
    else:
        p, q = act(o, name), dact(o, name)
        top = o.abs().clamp(min=1.0)
        e, ee = dy * p, ea * top * dy.abs() + 2 * U * (dy * p).abs()
        do = (dy * hs * q, dy.abs() * (eh * q.abs() + hs.abs() * ea * top) + 3 * U * (dy * hs * q).abs())
    q, big, err = dh1, dh1.abs(), torch.zeros_like(dh1)
    df, dv, edf, edv = [], [], [], []
    for t in range(f.shape[0] - 1, -1, -1):
        d, ed, bigd = e[t] + q, ee[t] + err + 2 * U * (e[t].abs() + big), e[t].abs() + big
        w = before[t] - v[t] if coupled else before[t]
        ew = ebefore[t] + 2 * U * (before[t].abs() + (v[t].abs() if coupled else 0.0))
        q = a[t] * d
        err = a[t] * ed + (eg * small[t] + 4 * U * a[t]) * bigd
        big = a[t] * bigd
        df.append(q * other[t] * w)
        edf.append(err * other[t] * w.abs() + q.abs() * other[t] * (eg * w.abs() + ew) + 4 * U * (q * other[t] * w).abs())
        dv.append(d * other[t] if coupled else d)
        edv.append((ed * other[t] + (eg + 2 * U) * (d * other[t]).abs()) if coupled else ed)
    back = lambda x: torch.stack(x[::-1]) if x else torch.zeros_like(f)  # noqa: E731
    return {"df": (back(df), back(edf)), "dv": (back(dv), back(edv)), "do": do, "dh0": (q, err)}


# ---- log probabilities ----------------------------------------------------------------------------------------------
def additions(vocab):
    return max(64, vocab // 512) + 64


def logprob(x, targets, scale):
    """Of float64 logits: logp (0 without a target), entropy, (m, log sum), log probabilities, and bounds for logp and entropy."""
    z = x * scale
    m = x.max(1, keepdim=True).values
    none = m == -math.inf
    t = torch.where(none, torch.full_like(z, -math.inf), (x - m) * scale)
    total = t.exp().sum(1, keepdim=True)
    lp = t - total.log()
    lp = torch.where(none, torch.full_like(z, -math.inf), lp)
    p = lp.exp()
    mean = (p * torch.where(p > 0, t, torch.zeros_like(t))).sum(1)
    entropy = torch.where(none[:, 0], torch.zeros_like(mean), total.log()[:, 0] - mean)
    given = (targets >= 0) & (targets < x.shape[1])
    at = targets.clamp(0, x.shape[1] - 1).long()[:, None]
    logp = torch.where(given, lp.gather(1, at)[:, 0], torch.zeros_like(mean))
    # terms: exponential 2^-21, argument 2 U |t|; sums: the additions
    rel = 2.0 ** -20 + additions(x.shape[1]) * U + 4 * U * mean.abs()
    gap = torch.where(torch.isfinite(logp), logp.abs(), torch.zeros_like(logp)) + total.log()[:, 0].abs().nan_to_num(0, 0, 0)
    return logp, entropy, torch.cat([m, total.log()], 1), lp, rel + 4 * U * gap, 2 * rel * (1 + mean.abs()) + 4 * U * entropy


def logprob_backward(x, targets, scale, dlogp, dentropy):
    logp, entropy, lse, lp, e1, e2 = logprob(x, targets, scale)
    p = lp.exp()
    given = ((targets >= 0) & (targets < x.shape[1]) & (lse[:, 0] != -math.inf))[:, None]
    hot = torch.zeros_like(p).scatter_(1, targets.clamp(0, x.shape[1] - 1).long()[:, None], 1.0)
    dl = torch.where(given, dlogp[:, None] if dlogp is not None else torch.zeros(1, dtype=x.dtype), torch.zeros(1, dtype=x.dtype))
    dh = dentropy[:, None] if dentropy is not None else torch.zeros(1, 1, dtype=x.dtype)
    safe = torch.where(p > 0, lp, torch.zeros_like(lp))
    d = scale * (dl * (hot - p) - dh * p * (safe + entropy[:, None]))
    weight = dl.abs() + dh.abs() * (safe.abs() + entropy[:, None])
    err = scale * (p * weight * (2.0 ** -20 + 2 * e1[:, None] + 8 * U * safe.abs()) + dh.abs() * p * (e2 + e1)[:, None] + 4 * U * (hot * dl).abs())
    return d, err
