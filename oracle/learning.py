"""Plain float64 forms of the gated experts, of the head over a vocabulary and of clipping, with their gradients, and a bound for the error of
an evaluation that multiplies and adds in binary32 and rounds to the tensors' type where the library says so.

A Bounded carries values and the most they may be off by.  ``half`` is half a step of the type a value is rounded to (2^-24, 2^-8 in bfloat16).  A
product's sums of K terms, in any order: K + 4 steps of 2^-23 of the sum of magnitudes (a matrix instruction may cut bits where it aligns its terms, a step
instead of half of one).
"""
from __future__ import annotations

import math

import numpy as np

STEP = 2.0 ** -23
_erf = np.vectorize(math.erf, otypes=[float])


def _of(v):
    """numpy, or torch where the values are its (float64) tensors: for sizes that take too long here."""
    if isinstance(v, (np.ndarray, float, int)):
        return np
    import torch
    return torch


class Bounded:
    def __init__(self, value, off=0.0):
        self.value = np.asarray(value, dtype=np.float64) if _of(value) is np else value
        self.off = off + 0.0 * _of(self.value).abs(_of(self.value).nan_to_num(self.value)) if isinstance(off, float) else off

    @property
    def T(self):
        return Bounded(self.value.T, self.off.T)

    def __add__(self, o):
        v = self.value + o.value
        return Bounded(v, self.off + o.off + STEP * abs(v))

    def __mul__(self, o):
        v = self.value * o.value
        off = abs(self.value) * o.off + self.off * abs(o.value) + self.off * o.off
        return Bounded(v, off + STEP * (abs(v) + off))

    def __matmul__(self, o):
        a, b = abs(self.value), abs(o.value)
        off = a @ o.off + self.off @ b + self.off @ o.off
        return Bounded(self.value @ o.value, off + (self.value.shape[1] + 4) * STEP * (a @ b + off))

    def rounded(self, half):
        return Bounded(self.value, self.off + half * (abs(self.value) + self.off))


def sigmoid(z):
    xp = _of(z)
    e = xp.exp(-abs(z))
    return xp.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def activation(name, g):
    """act(g) and act'(g) of a Bounded g."""
    v, off, xp = g.value, g.off, _of(g.value)
    if name == "silu":
        s = sigmoid(v)
        rel = (abs(v) + 8) * STEP                                    # the exponent's product and the reciprocal
        # slopes at most 1.1 and 0.5
        return (Bounded(v * s, 1.1 * off + rel * abs(v * s)),
                Bounded(s * (1 + v * (1 - s)), 0.5 * off + 2 * rel * s * (1 + abs(v))))
    if name == "gelu":
        erf = _erf if xp is np else xp.erf
        phi, bell = 0.5 * (1 + erf(v * math.sqrt(0.5))), xp.exp(-0.5 * v * v)
        rel = (v * v + 8) * STEP
        phi_off = 1.5e-7 + 4 * STEP * phi + rel * bell               # the form of the tail, its evaluation, its exponential
        # slopes at most 1.13 and 0.8
        return (Bounded(v * phi, 1.13 * off + abs(v) * phi_off),
                Bounded(phi + v * bell / math.sqrt(2 * math.pi), 0.8 * off + phi_off + abs(v) * bell * rel))
    on = (v > 0) * (1.0 + 0.0 * xp.nan_to_num(v))
    return Bounded(v * on, off), Bounded(on, ((abs(v) <= off) & (off > 0)) * (1.0 + 0.0 * off))


def gated_ffn(x, w_gate, w_up, w_down, act, half, dy=None):
    """One expert's rows -> dict of Bounded y and, with dy, dx, dw_gate, dw_up, dw_down."""
    x, w_gate, w_up, w_down = (Bounded(t) for t in (x, w_gate, w_up, w_down))
    u = x @ w_up
    a, slope = activation(act, x @ w_gate)
    h = (a * u).rounded(half)
    out = dict(y=(h @ w_down).rounded(half))
    if dy is not None:
        dy = Bounded(dy)
        dh = dy @ w_down.T
        du, dg = (dh * a).rounded(half), (dh * u * slope).rounded(half)
        out["dx"] = (dg @ w_gate.T + du @ w_up.T).rounded(half)
        out["dw_gate"], out["dw_up"], out["dw_down"] = (x.T @ dg).rounded(half), (x.T @ du).rounded(half), (h.T @ dy).rounded(half)
    return out


def head_logprobs(h, w, b, target, half, dlogprob=None):
    """-> dict of Bounded logprob, lse and, with dlogprob, dh, dw_head, db_head.  Rows of h at padded positions are taken as zero in the gradient."""
    N, V = h.shape[0], w.shape[0]
    on = (target >= 0) & (target < V)
    z = Bounded(h) @ Bounded(w).T
    bias = np.zeros(V) if b is None else b
    masked = np.isneginf(bias)
    value = np.where(masked, -np.inf, z.value + np.where(masked, 0.0, bias))
    off = np.where(masked, 0.0, z.off + STEP * abs(np.where(masked, 0.0, value)))
    m = value.max(1, keepdims=True)
    none = np.isneginf(m)
    m0 = np.where(none, 0.0, m)
    e = np.exp(value - m0)
    s = e.sum(1, keepdims=True)
    with np.errstate(divide="ignore"):
        lse = m0 + np.log(s)
    p = np.where(none, 0.0, e / np.where(none, 1.0, s))
    # the logits' errors weighted by p, exponents (|z - m| + 8 steps), the sum: lanes, tiles and their join
    with np.errstate(invalid="ignore"):
        far = np.where(p > 0, (m0 - value) + 8, 0.0)
    rel = (p * (1.01 * off + far * STEP)).sum(1, keepdims=True) + (64 + V / 4096) * STEP + 1e-12
    lse_off = rel + 2 * STEP * abs(np.where(none, 0.0, lse))
    at = np.clip(target, 0, V - 1)[:, None]
    zt = np.take_along_axis(value, at, 1)
    gone = np.isneginf(zt)
    lp = np.where(gone, -np.inf, np.where(gone, 0.0, zt) - np.where(none, 0.0, lse))
    lp_off = np.where(gone, 0.0, np.take_along_axis(off, at, 1) + rel + 4 * STEP * (abs(np.where(gone, 0.0, zt - m0)) + abs(np.where(none, 0.0, lse - m0))))
    out = dict(logprob=Bounded(np.where(on, lp[:, 0], 0.0), np.where(on, lp_off[:, 0], 0.0)), lse=Bounded(lse[:, 0], lse_off[:, 0]))
    if dlogprob is not None:
        counts = on & np.isfinite(dlogprob) & (dlogprob != 0)
        top = abs(dlogprob[counts]).max() if counts.any() else 1.0
        g = np.where(on, dlogprob, 0.0)[:, None] / top
        with np.errstate(invalid="ignore"):
            gap = np.where(p > 0, abs(value - np.where(none, 0.0, lse)) + 8, 0.0)
        p_off = 1.01 * p * (off + lse_off + gap * STEP)
        hit = np.zeros((N, V))
        np.put_along_axis(hit, at, 1.0, 1)
        dz = Bounded(g, abs(g) * STEP) * Bounded(hit - p, p_off + STEP)
        dzr = dz.rounded(half)
        scale = Bounded(np.full((1, 1), top), 0.0)
        clean = np.where(on[:, None], h, 0.0)
        for name, v, last in (("dh", dzr @ Bounded(w), half), ("dw_head", dzr.T @ Bounded(clean), half),
                              ("db_head", Bounded(np.ones((1, N))) @ dz, 2.0 ** -24)):
            out[name] = (v * scale).rounded(last)
        out["db_head"] = Bounded(out["db_head"].value[0], out["db_head"].off[0])
    return out


def clip(gradients, max_norm):
    """-> (norm, factor)."""
    norm = float(np.sqrt(sum(float(np.square(g).sum()) for g in gradients)))
    return norm, (max_norm / norm if np.isfinite(norm) and norm > max_norm else 1.0)
