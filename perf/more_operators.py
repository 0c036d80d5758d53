"""The products that training a routed layer and its predictor take beside `perf/operators.py`, and the step before the optimizer: the gated
experts with their gradient, the log probability of given ids under a head over a large vocabulary with its gradient and without logits in
memory, and clipping by the norm over all gradients.

A case is a dict of plain values:

  kind "gated"        moe_gated_ffn: y = (act(x W_gate) * (x W_up)) W_down over rows sorted by expert
  kind "gated_train"  the same with saved states, then moe_gated_ffn_backward
  kind "head"         moe_head_logprobs: log softmax(h W^T + b)[target] and the log of the sum
  kind "head_train"   the same, then moe_head_logprobs_backward
  kind "clip"         moe_clip_gradients

`own` chooses between the framework's calls and a plain form in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}
ACTIVATIONS = {"silu": 0, "gelu": 1, "relu": 2}


# ------------------------------------------------------------------------------------------------- the cases
def _gated(kind, dtype, T, k, d, F, E, zipf, hot, cf, act):
    return dict(kind=kind, dtype=dtype, T=T, k=k, d=d, F=F, E=E, zipf=zipf, hot=hot, cf=cf, act=act)


def _head(kind, dtype, N, d, V, bias, padded):
    return dict(kind=kind, dtype=dtype, N=N, d=d, V=V, bias=bias, padded=padded)


def _clip(dtype, layers, d, E, F, V, share):
    return dict(kind="clip", dtype=dtype, layers=layers, d=d, E=E, F=F, V=V, share=share)


def listed():
    return [
        # one token through one block that every token takes: a model that answers a single user
        dict(name="gated_dense_1", **_gated("gated", "bf16", 1, 1, 768, 2048, 1, 0.0, 0.0, 1.0, "silu")),
        # one token for each of 37 sequences, sorted over 128 experts: most experts idle, the others with a row or a few
        dict(name="gated_decode_37", **_gated("gated", "bf16", 37, 1, 768, 2048, 128, 1.0, 0.0, 4.0, "silu")),
        # the usual batch of a 128-expert layer, some tokens over capacity
        dict(name="gated_4096", **_gated("gated", "bf16", 4096, 1, 768, 2048, 128, 1.0, 0.0, 1.25, "gelu")),
        # a training step of a top-2 layer with 16 experts, one of them hot
        dict(name="gated_train_8192", **_gated("gated_train", "bf16", 8192, 2, 1024, 2816, 16, 0.8, 0.2, 2.0, "silu")),
        # a training step of a block that every token takes
        dict(name="gated_train_dense_8192", **_gated("gated_train", "bf16", 8192, 1, 1024, 4096, 1, 0.0, 0.0, 1.0, "gelu")),
        # binary32 training of a small model on an odd batch, with experts of a few rows and of none
        dict(name="gated_train_f32_1501", **_gated("gated_train", "f32", 1501, 1, 512, 1376, 32, 1.2, 0.0, 2.0, "silu")),
        # the next id of three sequences scored over a large vocabulary
        dict(name="head_3x131072", **_head("head", "bf16", 3, 768, 131072, False, 0.0)),
        # the predictor's imitation loss over the usual batch: its head has a bias, its classes are experts
        dict(name="head_train_experts_4096x128", **_head("head_train", "bf16", 4096, 256, 128, True, 0.05)),
        # a language model's loss on a batch of sequences, a part of it padding
        dict(name="head_train_8192x50257", **_head("head_train", "bf16", 8192, 768, 50257, False, 0.1)),
        # binary32 fine-tuning on a few sequences, odd in every size
        dict(name="head_train_f32_777x5003", **_head("head_train", "f32", 777, 320, 5003, True, 0.1)),
        # the gradients of a ten-layer predictor
        dict(name="clip_predictor", **_clip("f32", 10, 256, 0, 0, 128, 1.0)),
        # the gradients of a layer of 128 gated experts, its router and an embedding
        dict(name="clip_layer", **_clip("bf16", 1, 768, 128, 2048, 50257, 0.8)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["gated", "gated_train", "gated_train", "head", "head_train", "head_train", "clip"])
    dtype = "bf16" if rng.random() < 0.75 else "f32"
    size = SIZE[dtype] // 2
    if kind.startswith("gated"):
        d = rng.choice([128, 256, 512, 768, 1024, 2048, 8 * rng.randint(20, 180)])
        F = rng.choice([256, 512, 1024, 1376, 2048, 2816, 4096, 8 * rng.randint(30, 500)])
        E = rng.choice([1, 1, 8, 16, 32, 64, 128])
        while E > 1 and E * d * F > 200_000_000 // size:
            E //= 2
        k = 1 if E == 1 else rng.choice([1, 1, 2, 3])
        T = _log_int(rng, 1, min(16384, 40_000_000_000 // (size * size * d * F * k)))
        return _gated(kind, dtype, T, k, d, F, E, 0.0 if E == 1 else round(rng.uniform(0.5, 1.4), 2),
                      0.0 if E == 1 else rng.choice([0.0, 0.0, round(rng.uniform(0.1, 0.5), 2)]), rng.choice([1.0, 1.25, 2.0, 4.0]) if E > 1 else 1.0,
                      rng.choice(["silu", "silu", "gelu", "relu"]))
    if kind.startswith("head"):
        d = rng.choice([128, 256, 512, 768, 1024, 2048, 8 * rng.randint(12, 200)])
        V = rng.choice([8, 64, 100, 128, 256, 1000, _log_int(rng, 2000, 150000), _log_int(rng, 2000, 150000), _log_int(rng, 2000, 150000)])
        N = _log_int(rng, 1, min(32768, 280_000_000_000 // (size * size * d * V), 400_000_000 // (size * V)))
        return _head(kind, dtype, N, d, V, rng.random() < 0.4, rng.choice([0.0, 0.1, 0.5]) if N > 4 else 0.0)
    E = rng.choice([0, 0, 8, 32, 64])
    d = rng.choice([128, 256, 512, 768, 8 * rng.randint(12, 120) + rng.randint(0, 7)])
    F = rng.choice([512, 1024, 2048]) if E else 0
    layers = _log_int(rng, 1, 20 if E == 0 else max(1, min(4, 180_000_000 // (size * E * d * F))))
    return _clip(dtype, layers, d, E, F, rng.choice([100, 128, 1000, _log_int(rng, 2000, 60000)]), rng.choice([1.0, 0.5, 0.8]))


# ------------------------------------------------------------------------------------------------- inputs
def _kept(case):
    """Rows that each popularity rank keeps: a share `hot` on rank 0 and Zipf over the rest, as whole tokens; choice j of a token lies a step
    further in the ranks; what is over the capacity is dropped."""
    T, k, E, hot = case["T"], case["k"], case["E"], case["hot"]
    w = np.arange(1, E + 1, dtype=np.float64) ** -case["zipf"]
    if hot > 0.0:
        w = np.concatenate([[hot], (1.0 - hot) * w[:-1] / w[:-1].sum()])
    edges = np.round(np.cumsum(w / w.sum()) * T).astype(np.int64)
    edges[-1] = T
    n = np.diff(edges, prepend=0)
    n = sum(np.roll(n, j * max(1, E // 8)) for j in range(k))
    return np.minimum(n, max(4, math.ceil(case["cf"] * k * T / E))) if E > 1 else n


def _shapes(case):
    """(dtype, shape) of the gradients: SRU layers (their products, two biases each), gated experts with a router, an embedding or head."""
    dt, d, E, F = DTYPES[case["dtype"]], case["d"], case["E"], case["F"]
    shapes = []
    for _ in range(case["layers"]):
        if E:
            shapes += [(dt, (E, d, F)), (dt, (E, d, F)), (dt, (E, F, d)), (torch.float32, (d, E)), (torch.float32, (E,))]
        else:
            shapes += [(dt, (d, 3 * d)), (torch.float32, (d,)), (torch.float32, (d,))]
    return shapes + [(dt, (case["V"], d)), (torch.float32, (case["V"],))]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return torch.randn(*shape, generator=g, device="cuda").mul_(std).to(dtype)

    s = dict(case=case)
    if case["kind"].startswith("gated"):
        R, d, F, E = case["T"] * case["k"], case["d"], case["F"], case["E"]
        n = _kept(case)
        if E > 1:
            n = n[torch.randperm(E, generator=g, device="cuda").cpu().numpy()]
        s["first"] = [0] + np.cumsum(n).tolist()                # what the plain form cuts by; the calls read the table on the device
        s["offset"] = torch.tensor(s["first"], dtype=torch.int32, device="cuda") if E > 1 else None
        s["x"] = normal(R, d)
        s["w_gate"], s["w_up"], s["w_down"] = normal(E, d, F, std=d ** -0.5), normal(E, d, F, std=d ** -0.5), normal(E, F, d, std=F ** -0.5)
        # rows behind the last kept one are not written: a program's buffers, zero from the start
        s["y"] = torch.zeros(R, d, dtype=dt, device="cuda")
        if case["kind"] == "gated_train":
            s["dy"] = normal(R, d, std=0.01)
            s["out"] = dict(dx=torch.zeros_like(s["x"]), dw_gate=torch.empty_like(s["w_gate"]), dw_up=torch.empty_like(s["w_up"]),
                            dw_down=torch.empty_like(s["w_down"]))
    elif case["kind"].startswith("head"):
        N, d, V = case["N"], case["d"], case["V"]
        s["h"], s["w"] = normal(N, d), normal(V, d, std=2.0 * d ** -0.5)
        s["b"] = normal(V, std=0.5, dtype=torch.float32) if case["bias"] else None
        s["target"] = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        s["target"][torch.rand(N, generator=g, device="cuda") < case["padded"]] = -1
        s["dlogprob"] = torch.where(s["target"] >= 0, -1.0 / (s["target"] >= 0).sum().clamp(min=1), 0.0).float()    # the mean over what counts
    else:
        # a gradient's size differs from tensor to tensor
        s["gradients"] = [normal(*shape, std=0.01 * 2.0 ** (i % 5 - 2), dtype=t) for i, (t, shape) in enumerate(_shapes(case))]
        s["out"] = [torch.empty_like(t) for t in s["gradients"]]
        # share 1: within the limit, as in most steps of a run
        total = math.sqrt(sum(float(t.double().square().sum()) for t in s["gradients"]))
        s["max_norm"] = total * (case["share"] if case["share"] < 1.0 else 1.5)
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _act(name, g):
    """act(g) and its derivative."""
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    if name == "gelu":
        phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * phi, phi + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    return torch.where(g > 0, g, torch.zeros_like(g)), (g > 0).to(g.dtype)


def _gated_plain(s, train):
    case, first = s["case"], s["first"]
    y, x = s["y"], s["x"]
    for e in range(case["E"]):
        lo, hi = first[e], first[e + 1]
        if train and lo == hi:
            s["out"]["dw_gate"][e], s["out"]["dw_up"][e], s["out"]["dw_down"][e] = 0, 0, 0
        if lo == hi:
            continue
        xe, wg, wu, wd = x[lo:hi].float(), s["w_gate"][e].float(), s["w_up"][e].float(), s["w_down"][e].float()
        u = xe @ wu
        a, da = _act(case["act"], xe @ wg)
        h = a * u
        y[lo:hi] = (h @ wd).to(y.dtype)
        if train:
            dy = s["dy"][lo:hi].float()
            dh = dy @ wd.t()
            du, dg = dh * a, dh * u * da
            out = s["out"]
            out["dx"][lo:hi] = (dg @ wg.t() + du @ wu.t()).to(y.dtype)
            out["dw_gate"][e] = (xe.t() @ dg).to(y.dtype)
            out["dw_up"][e] = (xe.t() @ du).to(y.dtype)
            out["dw_down"][e] = (h.t() @ dy).to(y.dtype)
    return dict(y=y, **s["out"]) if train else dict(y=y)


def _head_plain(s, train):
    h, w, dt = s["h"].float(), s["w"].float(), s["h"].dtype
    z = h @ w.t()
    if s["b"] is not None:
        z += s["b"]
    m = z.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))
    on = (s["target"] >= 0) & (s["target"] < z.shape[1])
    at = s["target"].long().clamp(0, z.shape[1] - 1)[:, None]
    out = dict(logprob=torch.where(on, (z.gather(1, at) - lse)[:, 0], torch.zeros_like(lse[:, 0])), lse=lse[:, 0])
    if train:
        g = torch.where(on, s["dlogprob"], torch.zeros_like(s["dlogprob"]))[:, None]
        dz = -g * torch.exp(z - lse)
        dz.scatter_add_(1, at, g)
        out.update(dh=(dz @ w).to(dt), dw_head=(dz.t() @ h).to(dt))
        if s["b"] is not None:
            out["db_head"] = dz.double().sum(0).float()
    return out


def _clip_plain(s):
    norm = torch.sqrt(torch.stack([t.double().square().sum() for t in s["gradients"]]).sum())
    scale = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    for t, o in zip(s["gradients"], s["out"]):
        o.copy_(t.float() * scale)
    return dict(norm=norm.float().reshape(1), gradients=s["out"])


# ------------------------------------------------------------------------------------------------- the framework's calls
def _gated_own(s, train):
    import paper_2605_11537_amd as moe
    act = ACTIVATIONS[s["case"]["act"]]
    w = s["w_gate"], s["w_up"], s["w_down"]
    y, states = moe.moe_gated_ffn(s["x"], *w, s["offset"], act, want_states=train, out=s["y"])
    if not train:
        return dict(y=y)
    return dict(y=y, **moe.moe_gated_ffn_backward(s["dy"], s["x"], *w, states, s["offset"], act, out=s["out"]))


def _head_own(s, train):
    import paper_2605_11537_amd as moe
    out = moe.moe_head_logprobs(s["h"], s["w"], s["target"], s["b"])
    if train:
        grads = moe.moe_head_logprobs_backward(s["h"], s["w"], s["target"], out["lse"], s["dlogprob"], s["b"])
        out.update({k: v for k, v in grads.items() if v is not None})
    return out


def _clip_own(s):
    import paper_2605_11537_amd as moe
    norm, out = moe.moe_clip_gradients(s["gradients"], s["max_norm"], out=s["out"])
    return dict(norm=norm, gradients=out)


def run(state):
    kind = state["case"]["kind"]
    if kind == "clip":
        return _clip_own(state) if own else _clip_plain(state)
    train = kind.endswith("_train")
    if kind.startswith("gated"):
        return _gated_own(state, train) if own else _gated_plain(state, train)
    return _head_own(state, train) if own else _head_plain(state, train)


# ------------------------------------------------------------------------------------------------- work
def work(case):
    z = SIZE[case["dtype"]]
    if case["kind"] == "clip":
        n = sum((2 if t == torch.bfloat16 else 4) * math.prod(shape) for t, shape in _shapes(case))
        return dict(bytes=2 * n, flops=3 * n // z)
    if case["kind"].startswith("gated"):
        d, F, E = case["d"], case["F"], case["E"]
        n = _kept(case)
        K, hit = int(n.sum()), int((n > 0).sum())
        train = case["kind"] == "gated_train"
        # the tokens and y; the weights of the experts that have rows; for training dy, dx and a gradient for every weight
        return dict(bytes=(K * d * (4 if train else 2) + 3 * d * F * (hit + (E if train else 0))) * z, flops=6 * K * d * F * (3 if train else 1))
    N, d, V = case["N"], case["d"], case["V"]
    train = case["kind"] == "head_train"
    # without the logits in memory their product is made again for the gradient
    return dict(bytes=(N + V) * d * z * (2 if train else 1) + N * (16 if train else 12) + (4 * V * (2 if train else 1) if case["bias"] else 0),
                flops=2 * N * d * V * (4 if train else 1))


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"gat": _gated_exact, "hea": _head_exact, "cli": _clip_exact}[case["kind"][:3]](s, case)


def _gated_exact(s, case):
    """Expert by expert, the gradients by differentiating the product."""
    train = case["kind"] == "gated_train"
    act = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[case["act"]]
    y = torch.zeros_like(s["x"], dtype=torch.float64)
    got = {k: torch.zeros_like(v, dtype=torch.float64) for k, v in s["out"].items()} if train else {}
    for e, (lo, hi) in enumerate(zip(s["first"], s["first"][1:])):
        if lo == hi:
            continue
        leaves = [v.double().requires_grad_(train) for v in (s["x"][lo:hi], s["w_gate"][e], s["w_up"][e], s["w_down"][e])]
        x, wg, wu, wd = leaves
        ye = torch.mm(act(torch.mm(x, wg)) * torch.mm(x, wu), wd)
        y[lo:hi] = ye.detach()
        if train:
            grads = torch.autograd.grad(ye, leaves, s["dy"][lo:hi].double())
            got["dx"][lo:hi] = grads[0]
            got["dw_gate"][e], got["dw_up"][e], got["dw_down"][e] = grads[1:]
    return dict(y=y, **got)


def _head_exact(s, case):
    """By differentiating the log of the softmax, rows in blocks."""
    train = case["kind"] == "head_train"
    w = s["w"].double().requires_grad_(train)
    b = s["b"].double().requires_grad_(train) if s["b"] is not None else None
    N, V = case["N"], case["V"]
    lps, lses, dhs = [], [], []
    dw, db = torch.zeros_like(w), None if b is None else torch.zeros_like(b)
    step = max(1, 100_000_000 // V)
    for lo in range(0, N, step):
        h = s["h"][lo:lo + step].double().requires_grad_(train)
        z = torch.mm(h, w.t().contiguous())
        z = z if b is None else z + b
        on = s["target"][lo:lo + step] >= 0
        lp = torch.log_softmax(z, 1).gather(1, s["target"][lo:lo + step].long().clamp(min=0)[:, None])[:, 0]
        lp = torch.where(on, lp, 0.0)
        lps.append(lp.detach())
        lses.append(torch.logsumexp(z.detach(), 1))
        if train:
            grads = torch.autograd.grad(lp, [h, w] + ([] if b is None else [b]), s["dlogprob"][lo:lo + step].double())
            dhs.append(grads[0])
            dw += grads[1]
            if b is not None:
                db += grads[2]
    out = dict(logprob=torch.cat(lps), lse=torch.cat(lses))
    if train:
        out.update(dh=torch.cat(dhs), dw_head=dw.detach())
        if b is not None:
            out["db_head"] = db.detach()
    return out


def _clip_exact(s, case):
    norm = torch.linalg.vector_norm(torch.stack([torch.linalg.vector_norm(t.double()) for t in s["gradients"]]))
    factor = min(1.0, s["max_norm"] / float(norm))
    return dict(norm=norm.reshape(1), gradients=[t.double() * factor for t in s["gradients"]])
