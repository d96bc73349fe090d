"""The operators of sequence policies in 64 bits, written from their definitions.

Plain numpy loops over rows and time steps: the token loss and the preference loss with their
logits' gradients, the gated scan, and dropout + residual + root-mean-square norm with its mask.
Arrays are float64; every function returns a dict.
"""
from __future__ import annotations

import numpy as np


def log_softmax(x, temperature=1.0):
    x = x / temperature
    m = x.max(axis=1, keepdims=True)
    with np.errstate(divide="ignore"):
        return x - m - np.log(np.exp(x - m).sum(axis=1, keepdims=True))


def token_loss(logits, action, adv=None, logp_old=None, logp_ref=None, weight=None, clip_low=0.2,
               clip_high=0.2, c_kl=0.0, c_entropy=0.0, temperature=1.0):
    """Loss, statistics, per-row values and the gradient; `scale` bounds the gradient's terms."""
    n, V = logits.shape
    w = np.full(n, 1.0 / max(n, 1)) if weight is None else weight
    grad, scale = np.zeros((n, V)), np.zeros((n, V))
    lp, H, terms = np.zeros(n), np.zeros(n), np.zeros((n, 4))
    size = np.zeros(4)
    for i in range(n):
        if w[i] == 0:
            continue
        l = log_softmax(logits[i:i + 1], temperature)[0]
        p = np.exp(l)
        a = action[i]
        lf = np.where(p > 0, l, 0.0)
        lp[i], H[i] = l[a], -(p * lf).sum()
        c, ca = 0.0, 0.0
        if adv is not None:
            rho = 1.0 if logp_old is None else np.exp(lp[i] - logp_old[i])
            un, cl = rho * adv[i], min(max(rho, 1 - clip_low), 1 + clip_high) * adv[i]
            clipped = cl < un
            terms[i, 0], terms[i, 3] = -min(un, cl), float(clipped)
            c += 0.0 if clipped else -un
            ca += abs(rho * adv[i]) * (1 + abs(lp[i]))
            size[0] += abs(w[i] * rho * adv[i]) * (1 + abs(lp[i]))
        if logp_ref is not None:
            d = logp_ref[i] - lp[i]
            terms[i, 1] = np.exp(d) - d - 1
            c += c_kl * (1 - np.exp(d))
            ca += abs(c_kl) * (1 + np.exp(d)) * (1 + abs(lp[i]))
            size[1] += abs(w[i]) * (np.exp(d) + 1) * (1 + abs(lp[i]))
        terms[i, 2] = H[i]
        size[2] += abs(w[i]) * (1 + H[i])
        size[3] += abs(w[i])
        hot = np.zeros(V)
        hot[a] = 1
        grad[i] = w[i] * (c * (hot - p) + c_entropy * p * (lf + H[i])) / temperature
        scale[i] = abs(w[i]) * (ca * (hot + p) + abs(c_entropy) * p * (abs(lf) + H[i] + 1)) / temperature
    s = (w[:, None] * terms).sum(axis=0)
    s = np.where(np.isnan(s), np.nan, s)
    loss = s[0] + c_kl * s[1] - c_entropy * s[2] if logp_ref is not None else s[0] - c_entropy * s[2]
    size = np.concatenate([[size[0] + abs(c_kl) * size[1] + abs(c_entropy) * size[2]], size])
    return {"stats": np.concatenate([[loss], s]), "stats_scale": size, "logp": lp, "entropy": H,
            "grad": grad, "scale": scale}


def softplus(v):
    return np.maximum(v, 0) + np.log1p(np.exp(-np.abs(v)))


def preference_loss(logits, token, start, logp_ref=None, mask=None, weight=None, beta=0.1,
                    smoothing=0.0, temperature=1.0):
    n, V = logits.shape
    pairs = len(start) // 2
    w = np.full(pairs, 1.0 / max(pairs, 1)) if weight is None else weight
    ratio, size = np.zeros(2 * pairs), np.zeros(2 * pairs)
    grad, scale = np.zeros((n, V)), np.zeros((n, V))
    rows = {}
    for q in range(2 * pairs):
        for i in range(start[q], start[q + 1]):
            if mask is not None and not mask[i]:
                continue
            l = log_softmax(logits[i:i + 1], temperature)[0]
            ratio[q] += l[token[i]] - (0.0 if logp_ref is None else logp_ref[i])
            size[q] += 1 + abs(l[token[i]])
            rows[i] = (q, np.exp(l))
    h = beta * (ratio[0::2] - ratio[1::2])
    hs = abs(beta) * (size[0::2] + size[1::2])
    loss = (1 - smoothing) * softplus(-h) + smoothing * softplus(h)
    slope = 1 / (1 + np.exp(-h)) - (1 - smoothing)
    for i, (q, p) in rows.items():
        c = w[q // 2] * beta * slope[q // 2] * (1 if q % 2 == 0 else -1)
        hot = np.zeros(V)
        hot[token[i]] = 1
        grad[i] = c * (hot - p) / temperature
        # the slope moves by at most a quarter of the margin's error
        scale[i] = abs(w[q // 2] * beta) * (abs(slope[q // 2]) + hs[q // 2] / 4) * (hot + p) / temperature
    stats = np.array([(w * loss).sum(), (w * (h > 0)).sum(), (w * h).sum()])
    return {"stats": stats, "stats_scale": np.array([(abs(w) * (loss + hs)).sum(), abs(w).sum(),
                                                     (abs(w) * hs).sum()]),
            "ratio": ratio, "ratio_scale": size, "margin": h, "margin_scale": hs, "grad": grad,
            "scale": scale}


def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1 / (1 + e), e / (1 + e))


def gated_scan(x, gate, bias=None, h0=None, done=None):
    """h, h_last, and a bound on the error per unit of relative error in each step's own terms."""
    B, T, C = x.shape
    z = gate if bias is None else gate + bias
    a, b = sigmoid(z), sigmoid(-z)
    s = np.zeros((B, C)) if h0 is None else h0.copy()
    e = np.zeros((B, C))
    h, err = np.zeros((B, T, C)), np.zeros((B, T, C))
    for t in range(T):
        h[:, t] = a[:, t] * s + b[:, t] * x[:, t]
        e = a[:, t] * e + np.abs(s) + np.abs(x[:, t])
        err[:, t] = e
        s = h[:, t].copy()
        if done is not None:
            s[done[:, t] != 0] = 0
            e[done[:, t] != 0] = 0
    return {"h": h, "h_last": s, "err": err, "err_last": e}


def gated_scan_grad(x, gate, h, dh, bias=None, h0=None, done=None, dh_last=None):
    B, T, C = x.shape
    z = gate if bias is None else gate + bias
    a, b = sigmoid(z), sigmoid(-z)
    mu = np.zeros((B, C)) if dh_last is None else dh_last.copy()
    e = np.zeros((B, C))
    dx, dg, ex, eg = (np.zeros((B, T, C)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        if done is not None:
            mu[done[:, t] != 0] = 0
            e[done[:, t] != 0] = 0
        lam = dh[:, t] + mu
        s = (np.zeros((B, C)) if h0 is None else h0) if t == 0 else h[:, t - 1].copy()
        if t > 0 and done is not None:
            s[done[:, t - 1] != 0] = 0
        le = e + np.abs(mu) + np.abs(dh[:, t])
        dx[:, t], ex[:, t] = b[:, t] * lam, b[:, t] * le
        dg[:, t] = a[:, t] * b[:, t] * (s - x[:, t]) * lam
        eg[:, t] = a[:, t] * b[:, t] * (np.abs(s) + np.abs(x[:, t])) * le
        mu = a[:, t] * lam
        e = a[:, t] * le
    return {"dx": dx, "dgate": dg, "dbias": dg.sum(axis=(0, 1)), "dh0": mu, "err_dx": ex,
            "err_dgate": eg, "err_dbias": eg.sum(axis=(0, 1)), "err_dh0": e + np.abs(mu)}


def philox(c, k):
    """Philox4x32-10 on Python integers."""
    c, k = list(c), list(k)
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(n, width, p, seed, step, row_base=0):
    """(keep [n, width], scale): 16-bit fields of a draw per 8 columns against round(65536 p)."""
    thr = int(np.floor(np.float64(np.float32(p)) * 65536 + 0.5))
    if thr == 0:
        return np.ones((n, width), bool), 1.0
    keep = np.zeros((n, width), bool)
    for i in range(n):
        for g in range((width + 7) // 8):
            words = philox((g, row_base + i, step, 6), (seed & 0xFFFFFFFF, seed >> 32))
            for j in range(min(8, width - 8 * g)):
                keep[i, 8 * g + j] = (words[j // 2] >> (16 * (j % 2)) & 0xFFFF) >= thr
    return keep, 65536.0 / (65536 - thr)


def dropout_add_norm(x, gain, residual=None, keep=None, scale=1.0, eps=1e-6):
    u = x if keep is None else np.where(keep, x * scale, 0.0)
    z = u if residual is None else residual + u
    rstd = 1 / np.sqrt((z * z).mean(axis=1) + eps)
    return {"z": z, "rstd": rstd, "y": z * rstd[:, None] * gain,
            "z_scale": np.abs(u) + (0.0 if residual is None else np.abs(residual))}


def dropout_add_norm_grad(z, gain, rstd, dy, dz=None, keep=None, scale=1.0):
    r = rstd[:, None]
    zh, g = z * r, dy * gain
    d = r * (g - zh * (g * zh).mean(axis=1, keepdims=True))
    size = r * (np.abs(g) + np.abs(zh) * np.abs(g * zh).mean(axis=1, keepdims=True))
    if dz is not None:
        d, size = d + dz, size + np.abs(dz)
    dx = d if keep is None else np.where(keep, d * scale, 0.0)
    return {"dresidual": d, "dx": dx, "dgain": (dy * zh).sum(axis=0), "scale": size,
            "dgain_scale": np.abs(dy * zh).sum(axis=0)}
