"""fp64 definitions of the layer operators on NumPy arrays (test infrastructure only).

Each function follows the formula sequence by sequence and head by head; it shares no code
with the library. The attention also returns, per output element, the sum of the absolute
values of the terms it is a sum of: the scale that rounding errors are bounded by.
"""
import numpy as np


def rotate(x, cos, sin, rot, layout, sign=1.0):
    """x [T, H, D]; cos, sin [T, rot / 2]; sign -1 is the transposed rotation."""
    y = x.copy()
    half = rot // 2
    a, b = (np.arange(half), np.arange(half) + half) if layout == "half" else \
        (np.arange(half) * 2, np.arange(half) * 2 + 1)
    c, s = cos[:, None], sign * sin[:, None]
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def qk_norm_rope(x, w, cos, sin, rot, layout, eps):
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    return rotate(x, cos, sin, rot, layout)


def qk_norm_rope_backward(x, w, cos, sin, rot, layout, eps, grad):
    """(grad_x, grad_w, scale of grad_w)."""
    g = rotate(grad, cos, sin, rot, layout, -1.0)
    if w is None:
        return g, None, None
    r = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    n = x * r
    h = g * w
    return (r * (h - n * (h * n).mean(-1, keepdims=True)), (g * n).sum((0, 1)),
            np.abs(g * n).sum((0, 1)))


def _seen(n, plen, slen):
    """[n, plen + slen] of what each query sees."""
    j = np.arange(slen)[None]
    i = np.arange(n)[:, None]
    return np.concatenate([np.ones((n, plen), bool), j <= slen - n + i], 1)


def attention(seqs, scale, hq, hk, grad=False):
    """seqs: a list of dicts q [n, hq, D], k, v [P + S, hk, D] (prefix rows, then the suffix),
    plen, and do [n, hq, D] when grad. Adds out, lse, the scale of out, and for grad dq, dk,
    dv with scales, to each."""
    g = hq // hk
    for s in seqs:
        q, k, v = s["q"], s["k"], s["v"]
        n, L = q.shape[0], k.shape[0]
        see = _seen(n, s["plen"], L - s["plen"])
        s["out"], s["out_abs"] = np.zeros_like(q), np.zeros_like(q)
        s["lse"] = np.full((n, hq), -np.inf)
        s["z_abs"] = 0.0
        for name, like in (("dq", q), ("dk", k), ("dv", v)):
            s[name], s[name + "_abs"] = np.zeros_like(like), np.zeros_like(like)
        for h in range(hq):
            kk, vv, qq = k[:, h // g], v[:, h // g], q[:, h]
            with np.errstate(invalid="ignore"):
                z = np.where(see, qq @ kk.T * scale, -np.inf)
            fin = np.where(see, np.abs(qq) @ np.abs(kk).T * abs(scale), 0.0)
            s["z_abs"] = max(s["z_abs"], float(np.max(fin, initial=0.0)))
            top = z.max(1, initial=-np.inf)
            live = top > -np.inf
            p = np.where(see & live[:, None], np.exp(z - np.where(live, top, 0.0)[:, None]), 0.0)
            total = p.sum(1)
            safe = np.where(live, total, 1.0)
            s["lse"][:, h] = np.where(live, np.where(live, top, 0.0) + np.log(safe), -np.inf)
            p = p / safe[:, None]
            vz = np.where(np.isfinite(vv), vv, 0.0)
            s["out"][:, h] = p @ vz
            s["out_abs"][:, h] = p @ np.abs(vz)
            for j in np.nonzero(~np.isfinite(vv).all(1))[0]:     # values that are not finite
                rows = see[:, j]
                bad = ~np.isfinite(vv[j])
                s["out"][np.ix_(rows, [h], bad)] += (p[rows, j][:, None] * vv[j][bad])[:, None]
            if not grad:
                continue
            do = s["do"][:, h]
            dp = do @ vv.T
            delta = (do * s["out"][:, h]).sum(1, keepdims=True)
            dz = p * (dp - delta) * scale
            # what dz is a sum of, and what the rounded output adds to it
            dza = p * (np.abs(do) @ np.abs(vv).T + (np.abs(do) * np.abs(s["out"][:, h])).sum(1, keepdims=True)) \
                * abs(scale)
            s["dq"][:, h] = dz @ kk
            s["dq_abs"][:, h] = dza @ np.abs(kk)
            s["dk"][:, h // g] += dz.T @ qq
            s["dk_abs"][:, h // g] += dza.T @ np.abs(qq)
            s["dv"][:, h // g] += p.T @ do
            s["dv_abs"][:, h // g] += p.T @ np.abs(do)
    return seqs


def clip(grads, max_norm):
    """(scaled gradients, norm) of a list of float64 arrays."""
    norm = np.sqrt(sum(float((g * g).sum()) for g in grads))
    f = min(1.0, max_norm / (norm + 1e-6)) if np.isfinite(norm) else 1.0
    return [g * f for g in grads], norm
