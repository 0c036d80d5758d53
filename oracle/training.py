"""Plain float64 forms of the gradients and of the calls that train the gate and the predictor, token by token or row by row.

Arguments are float64 numpy arrays (index arrays: integers); nothing is rounded.  Beside a value, the scan gives a bound for the error
of a binary32 evaluation: ``steps`` half-units in the last place (2^-24) relative for every gate, product and sum, carried along the same recurrence.  With ``bf16``, a wider one, which also holds
for c = z + f (c - z) and h = w + r (tanh c - w): these round the differences and have 1 - f and 1 - r from f and r, 4 half-units of the values' own
magnitudes; and tanh may be off by 2.5e-5 of itself.
"""
from __future__ import annotations

import numpy as np

EPS = 2.0 ** -24


def _sigmoid(z):
    return np.where(z >= 0, 1.0 / (1.0 + np.exp(-np.abs(z))), np.exp(-np.abs(z)) / (1.0 + np.exp(-np.abs(z))))


def _scan_terms(u, x, b_f, b_r):
    B, L, W = u.shape
    H = x.shape[2] if x is not None else W // 4
    blocks = u.reshape(B, L, -1, H)
    zf, zr = blocks[:, :, 1] + b_f, blocks[:, :, 2] + b_r
    return blocks[:, :, 0], _sigmoid(zf), _sigmoid(-zf), _sigmoid(zr), _sigmoid(-zr), x if x is not None else blocks[:, :, 3]


def sru_scan(u, x, b_f, b_r, c0, lengths, steps=32, bf16=False):
    """-> dict(h, c_last, c [B,L+1,H] the states from c0 on, c_err their bounds, h_err)."""
    z, f, fr, r, rr, w = _scan_terms(u, x, b_f, b_r)
    B, L, H = z.shape
    c = np.empty((B, L + 1, H))
    err = np.zeros((B, L + 1, H))
    h, h_err = np.zeros((B, L, H)), np.zeros((B, L, H))
    c[:, 0] = c0
    e = steps * EPS
    blend, off = (4 * EPS, 2.5e-5) if bf16 else (0.0, 0.0)
    for b in range(B):
        for t in range(L):
            if t >= lengths[b]:
                c[b, t + 1], err[b, t + 1] = c[b, t], err[b, t]
                continue
            keep, new = f[b, t] * c[b, t], fr[b, t] * z[b, t]
            c[b, t + 1] = keep + new
            err[b, t + 1] = f[b, t] * err[b, t] + e * (np.abs(keep) + np.abs(new)) + blend * (np.abs(c[b, t]) + np.abs(z[b, t]))
            g = np.tanh(c[b, t + 1])
            h[b, t] = r[b, t] * g + rr[b, t] * w[b, t]
            h_err[b, t] = r[b, t] * (1 - g * g) * err[b, t + 1] + err[b, t + 1] ** 2 + e * (np.abs(r[b, t] * g) + np.abs(rr[b, t] * w[b, t])) \
                + blend * (np.abs(g) + np.abs(w[b, t])) + off * np.abs(r[b, t] * g)
    return dict(h=h, c_last=c[:, -1].copy(), c=c, c_err=err, h_err=h_err)


def sru_scan_backward(dh, dc_last, u, x, b_f, b_r, c0, lengths, steps=32, bf16=False):
    """-> dict(du, dx, db_f, db_r, dc0) and a dict of bounds under the same keys."""
    fw = sru_scan(u, x, b_f, b_r, c0, lengths, steps, bf16)
    off = 2.5e-5 if bf16 else 0.0
    c, c_err = fw["c"], fw["c_err"]
    z, f, fr, r, rr, w = _scan_terms(u, x, b_f, b_r)
    B, L, H = z.shape
    e = steps * EPS
    parts = [np.zeros((B, L, H)) for _ in range(4)]
    errs = [np.zeros((B, L, H)) for _ in range(4)]
    dc0, dc0_err = np.array(dc_last, dtype=np.float64), np.zeros((B, H))
    for b in range(B):
        dc, dc_e = dc0[b], dc0_err[b]
        for t in reversed(range(min(L, int(lengths[b])))):
            g, ce, d = np.tanh(c[b, t + 1]), c_err[b, t + 1], dh[b, t]
            slope = 1 - g * g
            through = d * r[b, t] * slope
            full = dc + through
            # the slope's own slope is -2 g slope, below 0.77
            full_e = dc_e + e * (np.abs(dc) + np.abs(through)) + np.abs(d * r[b, t]) * (0.77 * ce + ce ** 2)
            gap = c[b, t] - z[b, t]
            parts[0][b, t], errs[0][b, t] = full * fr[b, t], fr[b, t] * (full_e + e * np.abs(full))
            s = f[b, t] * fr[b, t]
            parts[1][b, t] = full * gap * s
            errs[1][b, t] = s * (full_e * (np.abs(gap) + c_err[b, t]) + np.abs(full) * (c_err[b, t] + e * (np.abs(c[b, t]) + np.abs(z[b, t]))))
            parts[2][b, t] = d * (g - w[b, t]) * r[b, t] * rr[b, t]
            errs[2][b, t] = np.abs(d) * r[b, t] * rr[b, t] * (slope * ce + ce ** 2 + e * (np.abs(g) + np.abs(w[b, t])) + off * np.abs(g))
            parts[3][b, t], errs[3][b, t] = d * rr[b, t], e * np.abs(d * rr[b, t])
            dc, dc_e = full * f[b, t], f[b, t] * (full_e + e * np.abs(full))
        dc0[b], dc0_err[b] = dc, dc_e

    def packed(p):
        q = p[:3] if x is not None else p
        return np.stack(q, 2).reshape(B, L, -1), p[3] if x is not None else None

    def total(p, q):
        # a sum of n terms in any order: each term's error, and half a unit of the running magnitude for each addition along its path
        return p.sum((0, 1)), q.sum((0, 1)) + EPS * (L + B + 64) * np.abs(p).sum((0, 1))

    (du, dx), (du_e, dx_e) = packed(parts), packed(errs)
    db_f, db_f_e = total(parts[1], errs[1])
    db_r, db_r_e = total(parts[2], errs[2])
    return (dict(du=du, dx=dx, db_f=db_f, db_r=db_r, dc0=dc0), dict(du=du_e, dx=dx_e, db_f=db_f_e, db_r=db_r_e, dc0=dc0_err))


def combine_backward(dout, y_perm, inv, weight, residual):
    """-> dict(dy_perm, dweight, dx); rows of dy_perm that inv does not name are NaN here."""
    k, T = inv.shape
    dy = np.full_like(y_perm, np.nan)
    dw, dx = np.zeros((k, T)), np.zeros_like(dout)
    for s in range(T):
        if residual or (inv[:, s] < 0).all():
            dx[s] = dout[s]
        for j in range(k):
            r = inv[j, s]
            if r >= 0:
                dy[r] = weight[j, s] * dout[s]
                dw[j, s] = dout[s] @ y_perm[r]
    return dict(dy_perm=dy, dweight=dw, dx=dx)


def dispatch_backward(dx_perm, inv, dx_add):
    k, T = inv.shape
    dx = np.zeros((T, dx_perm.shape[1])) if dx_add is None else dx_add.copy()
    for s in range(T):
        for j in range(k):
            if inv[j, s] >= 0:
                dx[s] += dx_perm[inv[j, s]]
    return dx


def route_weights(logits, idx, renormalize):
    """The weights [k,T] of moe_route_topk for given ids.  Renormalised they are the softmax of the chosen logits: a quotient of probabilities that
    have underflowed would be none."""
    chosen = np.stack([logits[np.arange(len(logits)), i] for i in idx])
    top = (chosen.max(0) if renormalize else logits.max(1))[None, :]
    w = np.exp(chosen - top)
    return w / (w.sum(0) if renormalize else np.exp(logits - top.T).sum(1))


def route_backward(logits, idx, dweight, renormalize):
    T, E = logits.shape
    k = len(idx)
    p = np.exp(logits - logits.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    w = route_weights(logits, idx, renormalize)
    d = np.zeros((T, E))
    for s in range(T):
        mean = (w[:, s] * dweight[:, s]).sum()
        if not renormalize:
            d[s] = -p[s] * mean
        for j in range(k):
            d[s, idx[j, s]] += w[j, s] * (dweight[j, s] - (mean if renormalize else 0.0))
    return d


def token_logprobs(logits, target, k):
    """-> dict(logprob, entropy, lse, top_idx, top_logprob); logits of -inf are masked."""
    N, V = logits.shape
    out = dict(logprob=np.zeros(N), entropy=np.zeros(N), lse=np.full(N, -np.inf), top_idx=np.zeros((N, k), np.int32),
               top_logprob=np.full((N, k), -np.inf))
    for n in range(N):
        x = logits[n]
        out["top_idx"][n] = np.argsort(-x, kind="stable")[:k]
        if x.max() == -np.inf:
            out["logprob"][n] = -np.inf if 0 <= target[n] < V else 0.0
            continue
        m = x.max()
        s = np.exp(x - m)
        lp = x - m - np.log(s.sum())
        p = s / s.sum()
        out["lse"][n] = m + np.log(s.sum())
        out["entropy"][n] = -(p[p > 0] * lp[p > 0]).sum()
        out["logprob"][n] = lp[target[n]] if 0 <= target[n] < V else 0.0
        out["top_logprob"][n] = lp[out["top_idx"][n]]
    return out


def token_logprobs_backward(logits, target, dlogprob, dentropy):
    N, V = logits.shape
    fw = token_logprobs(logits, target, 0)
    d = np.zeros((N, V))
    for n in range(N):
        if fw["lse"][n] == -np.inf:
            continue
        # under the maximum: beside 3e38, float64's lse too has lost the logarithm of the sum
        lp = logits[n] - logits[n].max()
        lp = lp - np.log(np.exp(lp).sum())
        p = np.exp(lp)
        on = p > 0
        d[n, on] = -dentropy[n] * p[on] * (lp[on] + fw["entropy"][n])
        if 0 <= target[n] < V:
            d[n] -= dlogprob[n] * p
            d[n, target[n]] += dlogprob[n]
    return d
