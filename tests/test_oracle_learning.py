"""oracle/learning.py against central differences of its own forward and against torch in float64."""
import numpy as np
import pytest
import torch

from oracle import learning as ol


def _differences(f, args, i, step=1e-5):
    x = args[i]
    g = np.zeros_like(x)
    for at in np.ndindex(x.shape):
        both = []
        for s in (step, -step):
            moved = [a.copy() if a is x else a for a in args]
            moved[i][at] += s
            both.append(f(*moved))
        g[at] = (both[0] - both[1]) / (2 * step)
    return g


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_gated(act):
    g = np.random.default_rng(3)
    x, wg, wu, wd = g.normal(size=(4, 3)), g.normal(size=(3, 5)), g.normal(size=(3, 5)), g.normal(size=(5, 3))
    dy = g.normal(size=(4, 3))
    got = ol.gated_ffn(x, wg, wu, wd, act, 0.0, dy)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[act]
    t = [torch.from_numpy(v) for v in (x, wg, wu, wd)]
    np.testing.assert_allclose(got["y"].value, ((f(t[0] @ t[1]) * (t[0] @ t[2])) @ t[3]).numpy(), rtol=1e-12)
    for i, k in enumerate(("dx", "dw_gate", "dw_up", "dw_down")):
        want = _differences(lambda *a: (ol.gated_ffn(*a, act, 0.0)["y"].value * dy).sum(), [x, wg, wu, wd], i)
        np.testing.assert_allclose(got[k].value, want, atol=1e-8)


def test_head():
    g = np.random.default_rng(4)
    h, w, b, dl = g.normal(size=(4, 3)), g.normal(size=(6, 3)), g.normal(size=6), g.normal(size=4)
    b[2] = -np.inf
    target = np.array([1, 5, -1, 0])
    got = ol.head_logprobs(h, w, b, target, 0.0, dl)
    lp = torch.log_softmax(torch.from_numpy(h) @ torch.from_numpy(w).T + torch.from_numpy(b), 1).numpy()
    np.testing.assert_allclose(got["logprob"].value, np.where(target >= 0, lp[np.arange(4), target], 0.0), rtol=1e-12)
    loss = lambda *a: (ol.head_logprobs(*a, target, 0.0)["logprob"].value * dl).sum()
    for i, k in enumerate(("dh", "dw_head", "db_head")):
        with np.errstate(invalid="ignore"):
            np.testing.assert_allclose(got[k].value, _differences(loss, [h, w, b], i), atol=1e-8)
    masked = ol.head_logprobs(h, w, np.full(6, -np.inf), target, 0.0, dl)
    assert np.isneginf(masked["lse"].value).all() and (masked["dh"].value[2] == 0).all()


def test_clip():
    a, b = np.full(3, 2.0), np.full((2, 2), 1.0)
    assert ol.clip([a, b], 2.0) == (4.0, 0.5) and ol.clip([a, b], 5.0) == (4.0, 1.0) and ol.clip([a * np.inf, b], 2.0)[1] == 1.0


def test_bounds_hold_for_binary32():
    """The bound of a product holds for numpy's binary32 product."""
    g = np.random.default_rng(5)
    a, b = g.normal(size=(7, 300)).astype(np.float32), g.normal(size=(300, 9)).astype(np.float32)
    v = ol.Bounded(a) @ ol.Bounded(b)
    assert (np.abs(a @ b - v.value) <= v.off).all() and v.off.max() < 1e-2
