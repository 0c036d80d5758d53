"""The training and scoring calls used together, as a program uses them: a predictor's training step, a layer's backward, the predictor's own
forward rebuilt from its parts; on other streams, in captured graphs that are replayed on new inputs, and with workspaces that two graphs share.

Gradients are held against float64 autograd of the same computation with torch's own functions.  Tolerance: a chain of at most eight binary32
sums of at most 1024 terms (256 in a product, a softmax, a sequence's biases), each off by at most its length times 2^-24 of its terms' magnitudes:
8 * 1024 * 2^-24 = 5e-4 of the largest gradient of a tensor."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TOL = 8 * 1024 * 2.0 ** -24


def _near(got, want, what):
    want = want.to(torch.float64).cpu()
    err = (got.double().cpu() - want).abs().max()
    assert err <= TOL * want.abs().max(), f"{what}: {err:.2e} against {want.abs().max():.2e}"


def _scan64(u, x, b_f, b_r, c, lengths):
    """torch's functions, token by token."""
    B, L, H = x.shape
    z, a, r = u.view(B, L, 3, H).unbind(2)
    f, r = torch.sigmoid(a + b_f), torch.sigmoid(r + b_r)
    rows = []
    for t in range(L):
        on = (t < lengths)[:, None]
        c = torch.where(on, f[:, t] * c + (1 - f[:, t]) * z[:, t], c)
        rows.append(torch.where(on, r[:, t] * torch.tanh(c) + (1 - r[:, t]) * x[:, t], torch.zeros_like(c)))
    return torch.stack(rows, 1), c


def _predictor(seed, B=3, L=70, H=96, E=40, layers=2):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s, std=1.0: torch.randn(*s, generator=g, dtype=torch.float64) * std
    p = dict(emb=n(B, L, H), head=n(H, E, std=0.3), c0=n(B, H, std=0.3))
    for i in range(layers):
        p.update({f"w{i}": n(H, 3 * H, std=0.15), f"bf{i}": n(H) + 1.0, f"br{i}": n(H)})
    lengths = torch.tensor([L, 11, L - 1][:B])
    target = torch.randint(0, E, (B, L), generator=g)
    target[torch.arange(L)[None, :] >= lengths[:, None]] = -1
    # float32 has these values exactly
    return {k: v.float().double() for k, v in p.items()}, lengths, target, layers


def _predictor_reference(p, lengths, target, layers):
    p = {k: v.clone().requires_grad_() for k, v in p.items()}
    x = p["emb"]
    for i in range(layers):
        x, _ = _scan64(x @ p[f"w{i}"], x, p[f"bf{i}"], p[f"br{i}"], p["c0"], lengths)
    logp = torch.log_softmax(x @ p["head"], -1)
    on = target >= 0
    entropy = -(logp.exp() * logp).sum(-1)
    loss = -(logp.gather(2, target.clamp(min=0)[:, :, None])[:, :, 0] * on).sum() / on.sum() - 0.05 * entropy.mean()
    loss.backward()
    return loss.item(), {k: v.grad for k, v in p.items()}


def _predictor_step(p, lengths, target, layers):
    """The same step on the framework's calls, products by torch.  p: float32 device tensors -> (loss terms, gradients)."""
    import paper_2605_11537_amd as moe
    B, L, H = p["emb"].shape
    xs, saved = [p["emb"]], []
    for i in range(layers):
        u = (xs[-1].view(-1, H) @ p[f"w{i}"]).view(B, L, 3 * H)
        h, _, states = moe.sru_scan(u, xs[-1], p[f"bf{i}"], p[f"br{i}"], p["c0"], lengths, want_states=True)
        xs.append(h)
        saved.append((u, states))
    flat = xs[-1].view(-1, H)
    logits = flat @ p["head"]
    s = moe.moe_token_logprobs(logits, target.view(-1), 2)
    n = (target >= 0).sum()
    dlogits = moe.moe_token_logprobs_backward(logits, target.view(-1), s["lse"], s["entropy"], (-1.0 / n).expand(B * L).contiguous(),
                                              torch.full((B * L,), -0.05 / (B * L), device="cuda"))
    grads = dict(head=flat.t() @ dlogits, c0=torch.zeros_like(p["c0"]))
    d = (dlogits @ p["head"].t()).view(B, L, H)
    for i in reversed(range(layers)):
        u, states = saved[i]
        g = moe.sru_scan_backward(d, u, states, xs[i], p[f"bf{i}"], p[f"br{i}"], None, lengths)
        du = g["du"].view(-1, 3 * H)
        grads.update({f"w{i}": xs[i].reshape(-1, H).t() @ du, f"bf{i}": g["db_f"], f"br{i}": g["db_r"]})
        grads["c0"] += g["dc0"]
        d = g["dx"] + (du @ p[f"w{i}"].t()).view(B, L, H)
    grads["emb"] = d
    return -s["logprob"].sum() / n - 0.05 * s["entropy"].mean(), grads


def test_a_training_step_of_the_predictor():
    p, lengths, target, layers = _predictor(1)
    loss, want = _predictor_reference(p, lengths, target, layers)
    dev = {k: v.float().cuda() for k, v in p.items()}
    got_loss, got = _predictor_step(dev, lengths.int().cuda(), target.int().cuda(), layers)
    assert abs(float(got_loss) - loss) <= TOL * abs(loss)
    for k in want:
        _near(got[k], want[k], k)


@pytest.mark.parametrize("k,renorm,residual,E", [(1, False, 0, 16), (2, True, 1, 20), (3, False, 1, 16)])
def test_the_gradient_of_a_layer(k, renorm, residual, E):
    """Router, plan, dispatch, experts (torch products over the kept rows), combine; back through every one of them."""
    import paper_2605_11537_amd as moe
    g = torch.Generator().manual_seed(k)
    T, d, F, budget, cap = 300, 64, 48, 4, max(8, 300 * k // E)
    n = lambda *s, std=1.0: (torch.randn(*s, generator=g) * std)
    p = dict(x=n(T, d), wr=n(d, E, std=0.3), br=n(E, std=0.3), w1=n(E, d, F, std=0.2), w2=n(E, F, d, std=0.2))
    dout = n(T, d, std=0.1).cuda()
    c = {key: v.cuda() for key, v in p.items()}
    idx, w, logits = moe.moe_route_topk(c["x"], c["wr"], c["br"], k, renorm, want_logits=True)
    plan = moe.replica_plan(idx.view(-1), E, budget, cap)
    disp = moe.moe_dispatch_topk(c["x"], idx, plan["replicas"], E, cap, E + budget)
    inv, offset = disp["inv"], disp["expert_offset"].tolist()
    K = offset[E]
    assert 0 < K < k * T                                             # some were dropped
    xp = disp["x_perm"]
    hidden, y = torch.zeros(k * T, F, device="cuda"), torch.zeros(k * T, d, device="cuda")
    for e in range(E):
        rows = slice(offset[e], offset[e + 1])
        hidden[rows] = torch.relu(xp[rows] @ c["w1"][e])
        y[rows] = hidden[rows] @ c["w2"][e]
    out = moe.moe_combine_topk(y, c["x"], inv, w, residual)
    b = moe.moe_combine_topk_backward(dout, y, inv, w, residual)
    dy, dw1, dw2, dxp = b["dy_perm"], torch.zeros_like(c["w1"]), torch.zeros_like(c["w2"]), torch.zeros(k * T, d, device="cuda")
    for e in range(E):
        rows = slice(offset[e], offset[e + 1])
        dh = (dy[rows] @ c["w2"][e].t()) * (hidden[rows] > 0)
        dw2[e], dw1[e] = hidden[rows].t() @ dy[rows], xp[rows].t() @ dh
        dxp[rows] = dh @ c["w1"][e].t()
    dx = moe.moe_dispatch_topk_backward(dxp, inv, dx_add=b["dx"], out=b["dx"])
    dlogits = moe.moe_route_topk_backward(logits, idx, b["dweight"], renorm)
    got = dict(x=dx + dlogits @ c["wr"].t(), wr=c["x"].t() @ dlogits, br=dlogits.sum(0), w1=dw1, w2=dw2)

    q = {key: v.double().requires_grad_() for key, v in p.items()}
    prob = torch.softmax(q["x"] @ q["wr"] + q["br"], 1)
    ids, kept = idx.long().cpu(), (inv >= 0).cpu()
    weight = prob.gather(1, ids.t()).t()
    if renorm:
        weight = weight / weight.sum(0)
    ref = torch.zeros(T, d, dtype=torch.float64)
    ref = ref + q["x"] * (1.0 if residual else (~kept.any(0)).double()[:, None])
    for j in range(k):
        h = torch.relu(torch.bmm(q["x"][:, None], q["w1"][ids[j]]))
        ref = ref + torch.bmm(h, q["w2"][ids[j]])[:, 0] * (weight[j] * kept[j])[:, None]
    _near(out, ref.detach(), "out")
    ref.backward(dout.double().cpu())
    for key in got:
        _near(got[key], q[key].grad, key)


def test_the_predictor_from_its_parts():
    """sru_predict's logits from torch products, sru_scan layer by layer and the head: the same columns, the same recurrence.  5e-3 of the
    largest logit is what its own test allows sru_predict in bfloat16; the parts round the states alike and keep the products in binary32."""
    import paper_2605_11537_amd as moe
    B, L, n_in, H, E = 2, 130, 128, 128, 64
    g = torch.Generator().manual_seed(8)
    bf = lambda *s, std: (torch.randn(*s, generator=g) * std).to(torch.bfloat16).cuda()
    emb, w0, w1, head = bf(B, L, n_in, std=1.0), bf(n_in, 3 * H, std=0.1), bf(H, 3 * H, std=0.1), bf(H, E, std=0.2)
    b = [torch.randn(H, generator=g).cuda() for _ in range(4)]
    weights = moe.SruWeights([w0, w1], [b[0], b[2]], [b[1], b[3]], head)
    pred, logits = moe.sru_predict(emb, weights, want_logits=True)
    x = emb.float()
    for w, b_f, b_r in ((w0, b[0], b[1]), (w1, b[2], b[3])):
        u = (x.view(B * L, -1) @ w.float()).view(B, L, -1)
        x = moe.sru_scan(u, x, b_f, b_r)[0].to(torch.bfloat16).float()
    mine = x.view(-1, H) @ head.float()
    assert (mine - logits).abs().max() <= 5e-3 * logits.abs().max()
    best = moe.moe_token_logprobs(logits, pred, 2)
    assert torch.equal(best["top_idx"][:, 0], pred) and torch.equal(best["top_logprob"][:, 0], best["logprob"])


def _chain(moe, s):
    """Every call once, on fixed buffers."""
    moe.sru_scan(s["u"], s["x"], s["b"], s["b"], s["c0"], s["len"], out=s["scan"], ws=s["ws"])
    moe.sru_scan_backward(s["dh"], s["u"], s["scan"][2], s["x"], s["b"], s["b"], s["dc"], s["len"], out=s["grads"], ws=s["ws"])
    moe.moe_token_logprobs(s["logits"], s["target"], 4, out=s["score"], ws=s["ws"])
    moe.moe_token_logprobs_backward(s["logits"], s["target"], s["score"]["lse"], s["score"]["entropy"], s["q"], s["q"], out=s["dlogits"])
    moe.moe_combine_topk_backward(s["dout"], s["y"], s["inv"], s["w"], 0, out=s["back"])
    moe.moe_dispatch_topk_backward(s["y"], s["inv"], s["back"]["dx"], out=s["dx"])
    moe.moe_route_topk_backward(s["gate"], s["idx"], s["back"]["dweight"], False, out=s["dgate"])


def _outputs(s):
    return [*s["scan"][:2], *(v for v in s["grads"].values()), *s["score"].values(), s["dlogits"], *s["back"].values(), s["dx"], s["dgate"]]


def _buffers(moe, ws=None, dtype=torch.bfloat16):
    """Sizes at which the scan is cut into segments and the logits into parts."""
    B, L, H, N, V, T, k, d, E = 2, 1500, 192, 2, 140000, 500, 2, 64, 32
    e = lambda *s, dt=torch.float32: torch.zeros(*s, dtype=dt, device="cuda")
    L_ = moe.lib()
    code = moe.MOE_BF16 if dtype == torch.bfloat16 else moe.MOE_F32
    need = max(L_.sru_scan_workspace_bytes(B, L, H, code), L_.sru_scan_backward_workspace_bytes(B, L, H, code),
               L_.moe_token_logprobs_workspace_bytes(N, V, 4, code))
    assert L_.sru_scan_workspace_bytes(B, L, H, code) > 0 and L_.moe_token_logprobs_workspace_bytes(N, V, 4, code) > 0
    s = dict(u=e(B, L, 3 * H, dt=dtype), x=e(B, L, H, dt=dtype), b=e(H), c0=e(B, H), len=e(B, dt=torch.int32), dh=e(B, L, H, dt=dtype), dc=e(B, H),
             logits=e(N, V, dt=dtype), target=e(N, dt=torch.int32), q=e(N), dout=e(T, d, dt=dtype), y=e(k * T, d, dt=dtype),
             inv=e(k, T, dt=torch.int32), w=e(k, T), gate=e(T, E), idx=e(k, T, dt=torch.int32),
             scan=(e(B, L, H, dt=dtype), e(B, H), e(L_.sru_scan_states_bytes(B, L, H) // 4)),
             grads=dict(du=e(B, L, 3 * H, dt=dtype), dx=e(B, L, H, dt=dtype), db_f=e(H), db_r=e(H), dc0=e(B, H)),
             score=dict(logprob=e(N), entropy=e(N), lse=e(N), top_idx=e(N, 4, dt=torch.int32), top_logprob=e(N, 4)), dlogits=e(N, V, dt=dtype),
             back=dict(dy_perm=e(k * T, d, dt=dtype), dweight=e(k, T), dx=e(T, d, dt=dtype)), dx=e(T, d, dt=dtype), dgate=e(T, E),
             ws=ws if ws is not None else e(need, dt=torch.uint8))
    return s


def _fill(s, seed):
    """New inputs into the same buffers."""
    g = torch.Generator().manual_seed(seed)
    for key in ("u", "x", "b", "c0", "dh", "dc", "logits", "q", "dout", "y", "w", "gate"):
        s[key].copy_(torch.randn(s[key].shape, generator=g))
    B, L, _ = s["x"].shape
    s["len"].copy_(torch.tensor([L, L - 1 - seed % 700]))
    s["target"].copy_(torch.randint(0, s["logits"].shape[1], s["target"].shape, generator=g))
    k, T = s["inv"].shape
    inv = torch.full((k * T,), -1)
    on = torch.randperm(k * T, generator=g)[: k * T - 37]
    inv[on] = torch.randperm(len(on), generator=g)
    s["inv"].copy_(inv.view(k, T))
    s["idx"].copy_(torch.rand(T, s["gate"].shape[1], generator=g).topk(k, 1).indices.t())
    s["back"]["dy_perm"].zero_()


def _eager(moe, s):
    _chain(moe, s)
    torch.cuda.synchronize()
    return [t.clone() for t in _outputs(s)]


def test_captured_and_replayed():
    """Replays on new inputs, with eager calls of the same chain between them, against the eager results."""
    import paper_2605_11537_amd as moe
    s, other = _buffers(moe), _buffers(moe)
    _fill(s, 1)
    _eager(moe, s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _chain(moe, s)
    for seed in range(2, 7):
        _fill(other, seed)
        want = _eager(moe, other)
        _fill(s, seed)
        for t in _outputs(s):
            if t is not s["back"]["dy_perm"]:
                t.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(_outputs(s), want)):
            assert torch.equal(a, b), (seed, i)


def test_two_graphs_share_a_workspace():
    """One after the other on a stream: nothing is kept in a workspace from call to call."""
    import paper_2605_11537_amd as moe
    a = _buffers(moe)
    b = _buffers(moe, ws=a["ws"])
    graphs = []
    for i, s in enumerate((a, b)):
        _fill(s, 20 + i)
        _eager(moe, s)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _chain(moe, s)
        graphs.append(g)
    want = []
    for s in (a, b):
        want.append(_eager(moe, s))
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        a["ws"].random_(0, 256)
        for i in order:
            graphs[i].replay()
        torch.cuda.synchronize()
        for i in set(order):
            assert all(torch.equal(x, y) for x, y in zip(_outputs((a, b)[i]), want[i])), order


def test_on_other_streams():
    """Two chains at once on streams of their own, workspaces of their own, against the same chains one after the other."""
    import paper_2605_11537_amd as moe
    sets = [_buffers(moe, dtype=t) for t in (torch.bfloat16, torch.float32)]
    want = []
    for i, s in enumerate(sets):
        _fill(s, 30 + i)
        want.append(_eager(moe, s))
    streams = [torch.cuda.Stream() for _ in sets]
    for s in sets:
        for t in _outputs(s):
            if t is not s["back"]["dy_perm"]:
                t.fill_(7)
    torch.cuda.synchronize()
    for _ in range(3):
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                _chain(moe, s)
    torch.cuda.synchronize()
    for s, w in zip(sets, want):
        assert all(torch.equal(a, b) for a, b in zip(_outputs(s), w))


def test_another_device_is_refused(monkeypatch):
    """Kernels go to the current device's stream: tensors of another one are refused before anything is enqueued."""
    import paper_2605_11537_amd as moe
    from paper_2605_11537_amd import binding
    monkeypatch.setattr(binding, "_device", lambda: 1)
    x, t = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: moe.moe_token_logprobs(x, t), lambda: moe.moe_dispatch_topk_backward(x, t),
                 lambda: moe.sru_scan(torch.zeros(1, 4, 24, device="cuda"), torch.zeros(1, 4, 8, device="cuda"))):
        with pytest.raises(ValueError, match="the current device is 1"):
            call()


def test_sizes_past_an_int_are_refused():
    """A size is never reduced to the int that the library counts in: 2^32 + 8 is not 8."""
    import paper_2605_11537_amd as moe
    far = 2 ** 32 + 8
    e = lambda *s, dt=torch.float32: torch.zeros(*[1] * len(s), dtype=dt, device="cuda").expand(*s)
    one = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, device="cuda")
    out = torch.zeros(1, 1, device="cuda").expand(1, far)
    for call in (lambda: moe.moe_token_logprobs(e(1, far), one),
                 lambda: moe.moe_token_logprobs_backward(e(1, far), one, q, q, q, out=out),
                 lambda: moe.moe_token_logprobs(e(far, 8), e(far, dt=torch.int32)),
                 lambda: moe.moe_route_topk_backward(e(1, far), one[None], q[None], out=out),
                 lambda: moe.moe_route_topk_backward(e(1, 8), e(far, 1, dt=torch.int32), e(far, 1), out=e(1, 8)),
                 lambda: moe.moe_combine_topk_backward(e(far, 8), e(far, 8), e(far, dt=torch.int32), e(far),
                                                       out=dict(dy_perm=e(far, 8), dweight=None, dx=None)),
                 lambda: moe.moe_dispatch_topk_backward(e(far, 8), e(far, dt=torch.int32), out=e(far, 8)),
                 lambda: moe.sru_scan(e(1, far, 24), e(1, far, 8)),
                 lambda: moe.sru_scan_backward(e(1, far, 8), e(1, far, 24), None, e(1, far, 8))):
        with pytest.raises(ValueError, match="does not fit an int"):
            call()


def test_workspaces_lie_beside_the_tensors():
    """A workspace of another place or type is refused as any other tensor is."""
    import paper_2605_11537_amd as moe
    s = _buffers(moe)
    for ws in (s["ws"].cpu(), s["ws"].view(torch.float32)):
        for call in (lambda: moe.sru_scan(s["u"], s["x"], ws=ws), lambda: moe.sru_scan_backward(s["dh"], s["u"], s["scan"][2], s["x"], ws=ws),
                     lambda: moe.moe_token_logprobs(s["logits"], s["target"], ws=ws)):
            with pytest.raises(ValueError, match="ws "):
                call()


def test_captured_with_tensors_of_its_own():
    """A graph whose calls allocate their outputs and workspaces themselves, replayed on new inputs between eager calls."""
    import paper_2605_11537_amd as moe

    def chain(s):
        h, c, states = moe.sru_scan(s["u"], s["x"], s["b"], s["b"], s["c0"], s["len"], want_states=True)
        grads = moe.sru_scan_backward(s["dh"], s["u"], states, s["x"], s["b"], s["b"], s["dc"], s["len"])
        score = moe.moe_token_logprobs(s["logits"], s["target"], 4)
        slope = moe.moe_token_logprobs_backward(s["logits"], s["target"], score["lse"], score["entropy"], s["q"], s["q"])
        back = moe.moe_combine_topk_backward(s["dout"], s["y"], s["inv"], s["w"])
        dx = moe.moe_dispatch_topk_backward(s["y"], s["inv"], back["dx"])
        gate = moe.moe_route_topk_backward(s["gate"], s["idx"], back["dweight"])
        return [h, c, *grads.values(), *score.values(), slope, *back.values(), dx, gate]

    s, other = _buffers(moe), _buffers(moe)
    _fill(s, 40)
    chain(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = chain(s)
    for seed in range(41, 45):
        _fill(other, seed)
        want = [t.clone() for t in chain(other)]
        _fill(s, seed)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for i, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (seed, i)
