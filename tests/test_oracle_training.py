"""The float64 gradients of oracle/training.py against central differences of the float64 forwards, and its values against torch's."""
import numpy as np
import pytest
import torch

from oracle import training as ot

STEP = 1e-5
# central differences: the third derivative times STEP^2 / 6, and the rounding of values of order 1 .. 30 over STEP
DIFF_TOL = 2e-8


def _differences(f, a, where):
    out = []
    for i in where:
        old = a.flat[i]
        a.flat[i] = old + STEP
        up = f()
        a.flat[i] = old - STEP
        down = f()
        a.flat[i] = old
        out.append((up - down) / (2 * STEP))
    return np.array(out)


@pytest.mark.parametrize("highway", [True, False])
def test_scan_gradient_is_the_slope(highway):
    g = np.random.default_rng(3)
    B, L, H = 3, 7, 4
    u = g.standard_normal((B, L, (3 if highway else 4) * H))
    x = g.standard_normal((B, L, H)) if highway else None
    b_f, b_r, c0 = g.standard_normal(H), g.standard_normal(H), g.standard_normal((B, H))
    lengths = np.array([7, 0, 4])
    dh, dc = g.standard_normal((B, L, H)), g.standard_normal((B, H))
    got, bounds = ot.sru_scan_backward(dh, dc, u, x, b_f, b_r, c0, lengths)

    def loss():
        f = ot.sru_scan(u, x, b_f, b_r, c0, lengths)
        return (f["h"] * dh).sum() + (f["c_last"] * dc).sum()

    for key, a in (("du", u), ("dx", x), ("db_f", b_f), ("db_r", b_r), ("dc0", c0)):
        if a is None:
            assert got[key] is None
            continue
        want = _differences(loss, a, range(a.size))
        assert np.abs(got[key].ravel() - want).max() <= DIFF_TOL, key
        assert bounds[key].shape == got[key].shape and (bounds[key] >= 0).all()


def test_scan_is_the_printed_recurrence():
    """Against torch in float64, written out with its own functions; an empty sequence keeps its state."""
    g = torch.Generator().manual_seed(4)
    B, L, H = 2, 9, 5
    u, x = (torch.randn(B, L, n * H, generator=g, dtype=torch.float64) for n in (3, 1))
    b_f, b_r, c = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((H,), (H,), (B, H)))
    f = ot.sru_scan(u.numpy(), x.numpy(), b_f.numpy(), b_r.numpy(), c.numpy(), [L, 0])
    assert (f["c_last"][1] == c[1].numpy()).all() and (f["h"][1] == 0).all()
    c = c[0]
    for t in range(L):
        z, a, r = u[0, t].view(3, H)
        fg, rg = torch.sigmoid(a + b_f), torch.sigmoid(r + b_r)
        c = fg * c + (1 - fg) * z
        h = rg * torch.tanh(c) + (1 - rg) * x[0, t]
        assert np.abs(f["h"][0, t] - h.numpy()).max() < 1e-14
    assert np.abs(f["c_last"][0] - c.numpy()).max() < 1e-14


@pytest.mark.parametrize("k,residual", [(1, 0), (3, 1), (2, 0)])
def test_combine_and_dispatch_gradients_are_the_slopes(k, residual):
    g = np.random.default_rng(5)
    T, d = 5, 3
    inv = np.full((k, T), -1)
    kept = g.permutation(k * T)[: k * T - 3]
    inv.flat[kept] = g.permutation(len(kept))
    inv[:, 2] = -1
    x, y, w = g.standard_normal((T, d)), g.standard_normal((k * T, d)), g.random((k, T))
    dout = g.standard_normal((T, d))

    def loss():
        out = np.zeros((T, d))
        for s in range(T):
            if residual or (inv[:, s] < 0).all():
                out[s] = x[s]
            for j in range(k):
                if inv[j, s] >= 0:
                    out[s] += w[j, s] * y[inv[j, s]]
        return (out * dout).sum()

    got = ot.combine_backward(dout, y, inv, w, residual)
    named = np.isin(np.arange(k * T), inv)
    assert np.isnan(got["dy_perm"][~named]).all()
    want = _differences(loss, y, range(y.size)).reshape(y.shape)
    assert np.abs(got["dy_perm"] - want)[named].max() <= DIFF_TOL
    assert np.abs(got["dweight"].ravel() - _differences(loss, w, range(w.size))).max() <= DIFF_TOL
    assert np.abs(got["dx"].ravel() - _differences(loss, x, range(x.size))).max() <= DIFF_TOL
    # the rows' own way back: x_perm[inv] = x
    dxp = g.standard_normal((k * T, d))

    def copied():
        return sum((x[s] * dxp[inv[j, s]]).sum() for j in range(k) for s in range(T) if inv[j, s] >= 0)

    assert np.abs(ot.dispatch_backward(dxp, inv, None).ravel() - _differences(copied, x, range(x.size))).max() <= DIFF_TOL
    assert np.allclose(ot.dispatch_backward(dxp, inv, x), x + ot.dispatch_backward(dxp, inv, None), atol=1e-15)


@pytest.mark.parametrize("renorm", [False, True])
def test_gate_gradient_is_the_slope(renorm):
    g = np.random.default_rng(6)
    T, E, k = 4, 6, 3
    logits, dw = g.standard_normal((T, E)), g.standard_normal((k, T))
    idx = np.argsort(-logits, 1)[:, :k].T.copy()
    got = ot.route_backward(logits, idx, dw, renorm)
    want = _differences(lambda: (ot.route_weights(logits, idx, renorm) * dw).sum(), logits, range(logits.size))
    assert np.abs(got.ravel() - want).max() <= DIFF_TOL


def test_scores_and_their_gradient():
    g = np.random.default_rng(7)
    N, V = 5, 9
    x = g.standard_normal((N, V)) * 2
    x[1, [0, 4]] = -np.inf
    x[3] = -np.inf
    target = np.array([2, 5, -1, 1, 9])
    f = ot.token_logprobs(x, target, 4)
    t = torch.from_numpy(x)
    for n in (0, 1, 2, 4):
        lp = torch.log_softmax(t[n], 0)
        ent = torch.distributions.Categorical(logits=torch.where(t[n] > -np.inf, t[n], -1e30)).entropy()
        assert abs(f["entropy"][n] - ent.item()) < 1e-12
        assert f["logprob"][n] == pytest.approx(lp[target[n]].item(), abs=1e-12) if target[n] in range(V) else f["logprob"][n] == 0
        assert f["lse"][n] == pytest.approx(torch.logsumexp(t[n], 0).item(), abs=1e-12)
        order = sorted(range(V), key=lambda i: (-x[n, i], i))[:4]
        assert f["top_idx"][n].tolist() == order
    assert f["logprob"][3] == -np.inf and f["entropy"][3] == 0 and f["top_idx"][3].tolist() == [0, 1, 2, 3]
    dl, de = g.standard_normal(N), g.standard_normal(N)
    got = ot.token_logprobs_backward(x, target, dl, de)
    assert (got[3] == 0).all() and (got[1, [0, 4]] == 0).all()

    def loss():
        q = ot.token_logprobs(x, target, 0)
        on = [0, 1, 2, 4]
        return (q["logprob"][on] * dl[on]).sum() + (q["entropy"][on] * de[on]).sum()

    where = [i for i in range(N * V) if np.isfinite(x.flat[i])]
    assert np.abs(got.flat[where] - _differences(loss, x, where)).max() <= DIFF_TOL
