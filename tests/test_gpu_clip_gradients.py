"""moe_clip_gradients against numpy in float64.  norm: sums in binary64, rounded once (2^-24 of itself).  A scaled element: the factor rounded
to binary32 (2^-24), its product (2^-24), the rounding to the tensor's type (half a step); what is not scaled is the gradient bit for bit."""
import numpy as np
import pytest
import torch

from oracle import learning as ol

pytestmark = pytest.mark.gpu


def make(shapes, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(s, generator=g, device="cuda") * std * (1 + i % 3)).to(t) for i, (s, t) in enumerate(shapes)]


def check(grads, norm, out, max_norm):
    want, factor = ol.clip([g.double().cpu().numpy() for g in grads], max_norm)
    assert abs(float(norm) - want) <= 2.0 ** -24 * 1.001 * want
    for g, o in zip(grads, out):
        assert g.shape == o.shape and g.dtype == o.dtype
        if factor == 1.0:
            assert torch.equal(g, o)
            continue
        v = g.double() * factor
        tiny = 2.0 ** -149 if g.dtype == torch.float32 else 2.0 ** -133
        assert ((o.double() - v).abs() <= v.abs() * (torch.finfo(g.dtype).eps / 2 + 2.1 * 2.0 ** -24) + tiny).all()


F, B = torch.float32, torch.bfloat16
LISTS = [
    [((1,), F)], [((1,), B)], [((3, 5), F), ((7,), B)], [((0,), F), ((4096,), F), ((0, 3), B)], [((4097,), F), ((8193,), B), ((5,), F)],
    [((256, 768), F)] * 5 + [((256,), F)] * 10 + [((128, 256), B)], [((17 * i + 1,), (F, B)[i % 2]) for i in range(300)], [((3000, 2001), B), ((2, 3, 4), F)],
]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("shapes", LISTS, ids=range(len(LISTS)))
def test_norm_and_scaling(shapes, in_place):
    import paper_2605_11537_amd as moe
    grads = make(shapes, len(shapes))
    total = ol.clip([g.double().cpu().numpy() for g in grads], 1.0)[0]
    for max_norm in (0.37 * total, 1.5 * total, float("inf"), 1e-30):
        given = [g.clone() for g in grads]
        norm, out = moe.moe_clip_gradients(given, max_norm, out=given if in_place else None)
        check(grads, norm, out, np.float32(max_norm).item())
        if not in_place:
            assert all(torch.equal(a, b) for a, b in zip(given, grads))
        else:
            assert all(a is b for a, b in zip(given, out))


@pytest.mark.parametrize("std", [1e30, 1e-30, 1e-40])
def test_far_values(std):
    """Squares past binary32's range."""
    import paper_2605_11537_amd as moe
    grads = make([((5000,), F), ((333,), F)], 3, std)
    norm, out = moe.moe_clip_gradients(grads, 0.1 * std * 70)
    want, factor = ol.clip([g.double().cpu().numpy() for g in grads], np.float32(0.1 * std * 70).item())
    assert abs(float(norm) - want) <= 2.0 ** -24 * 1.001 * want + 2.0 ** -149
    for g, o in zip(grads, out):
        assert ((o.double() - g.double() * factor).abs() <= g.double().abs() * factor * 2.0 ** -22 + 2.0 ** -149).all()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_a_norm_that_is_no_number_scales_nothing(bad):
    import paper_2605_11537_amd as moe
    grads = make([((5000,), F), ((333,), B)], 4)
    grads[1][7] = bad
    kept = [g.clone() for g in grads]
    norm, out = moe.moe_clip_gradients(grads, 0.5, out=grads)
    assert not torch.isfinite(norm).any() and torch.equal(out[0], kept[0]) and torch.equal(out[1].view(torch.int16), kept[1].view(torch.int16))


def test_views_on_any_element():
    """Pieces of one flat buffer, most of them off 16 bytes, clipped in place: what lies between them is left as it was."""
    import paper_2605_11537_amd as moe
    for t in (F, B):
        flat = make([((40000,), t)], 5)[0]
        kept = flat.clone()
        edges = [1, 8, 9, 5000, 5003, 17000, 39999]
        views = [flat[a:b] for a, b in zip(edges, edges[1:-1])]
        norm, _ = moe.moe_clip_gradients(views, 1.0, out=views)
        check([kept[a:b] for a, b in zip(edges, edges[1:-1])], norm, views, 1.0)
        assert torch.equal(flat[:1], kept[:1]) and torch.equal(flat[17000:], kept[17000:])


def test_refusals():
    import paper_2605_11537_amd as moe
    g = make([((64,), F), ((64,), F)], 6)
    for grads, out, error in (([g[0], g[0]], [g[0], g[0]], moe.MoeError), (g, [g[1], g[0]], moe.MoeError), ([g[0][:40], g[0][32:]], [g[0][:40], g[0][32:]], moe.MoeError),
                              (g, g[:1], ValueError), (g, [g[0], g[1].to(B)], ValueError), ([g[0].half()], None, ValueError), ([g[0].cpu()], None, ValueError),
                              ([g[0].view(8, 8).t()], [g[1].view(8, 8)], ValueError), ([g[0], 3], [g[0], g[1]], TypeError)):
        with pytest.raises(error):
            moe.moe_clip_gradients(grads, 1.0, out=out)
    for bad in (0.0, -1.0, float("nan")):
        with pytest.raises(moe.MoeError):
            moe.moe_clip_gradients(g, bad)
    # the same gradient read twice is no harm while nothing is written over it
    norm, out = moe.moe_clip_gradients([g[0], g[0]], 1e9)
    assert torch.equal(out[0], g[0]) and torch.equal(out[1], g[0])
    norm, out = moe.moe_clip_gradients([], 1.0, norm=torch.ones(1, device="cuda"))
    assert out == [] and float(norm) == 0.0
