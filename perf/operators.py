"""The operators that train the predictor and the gate, and serve the predictor token by token, on the sizes they meet: the gated
recurrence of an SRU layer with its gradient, the gradient of sorting tokens by expert and back, and log probabilities of given ids with
entropy, alternatives and gradient.

A case is a dict of plain values:

  kind "scan"        sru_scan: the recurrence over [B, L, H] with an initial and a final state
  kind "scan_train"  the same with saved states, then sru_scan_backward
  kind "back"        the routing's part of a layer's backward: moe_combine_topk_backward, moe_dispatch_topk_backward and
                     moe_route_topk_backward on the tables of one batch (the experts' own products run between the first two)
  kind "score"       moe_token_logprobs
  kind "score_train" the same, then moe_token_logprobs_backward

`own` chooses between the framework's calls and a plain form in elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------------------- the cases
def _scan(kind, dtype, B, L, H, k, ragged):
    return dict(kind=kind, dtype=dtype, B=B, L=L, H=H, k=k, ragged=ragged)


def _back(dtype, T, k, d, E, zipf, hot, cf, residual, renorm):
    return dict(kind="back", dtype=dtype, T=T, k=k, d=d, E=E, zipf=zipf, hot=hot, cf=cf, residual=residual, renorm=renorm)


def _score(kind, dtype, N, V, k, masked):
    return dict(kind=kind, dtype=dtype, N=N, V=V, k=k, masked=masked)


def listed():
    return [
        # one token for each of 64 sequences, states carried from call to call: the predictor while a model decodes
        dict(name="scan_decode_64", **_scan("scan", "bf16", 64, 1, 256, 3, False)),
        # two long documents, scored in one go: few channels, so the work has to be split along the sequence
        dict(name="scan_long_2x16384", **_scan("scan", "bf16", 2, 16384, 768, 3, False)),
        # a training step of a predictor's layer on 64 sequences of 512 tokens
        dict(name="scan_train_64x512", **_scan("scan_train", "bf16", 64, 512, 768, 3, False)),
        # binary32 training on a padded batch of odd lengths and an odd width, with a projected highway
        dict(name="scan_train_f32_5x777", **_scan("scan_train", "f32", 5, 777, 321, 4, True)),
        # fine-tuning on a few sequences' last tokens
        dict(name="back_37", **_back("bf16", 37, 1, 768, 128, 1.0, 0.0, 1.25, 0, False)),
        # the usual batch of a 128-expert layer under top-3 routing
        dict(name="back_top3_4096", **_back("bf16", 4096, 3, 768, 128, 1.0, 0.0, 1.25, 0, True)),
        # a binary32 layer of a small model on an odd batch, top-2
        dict(name="back_f32_3001", **_back("f32", 3001, 2, 512, 64, 1.0, 0.0, 1.0, 1, True)),
        # a large batch with half of its tokens on one expert, inside a residual stack
        dict(name="back_skew_65536", **_back("bf16", 65536, 1, 768, 256, 1.0, 0.5, 4.0, 1, False)),
        # the predictor's logits of the usual batch: the router's ids under them, and the three next experts to prefetch
        dict(name="score_experts_4096x128", **_score("score", "f32", 4096, 128, 3, False)),
        # next-token candidates of three sequences over a large vocabulary, part of it masked
        dict(name="score_decode_3x131072", **_score("score", "bf16", 3, 131072, 8, True)),
        # the predictor's imitation loss over 64 sequences of 512 tokens
        dict(name="score_train_experts_32768x256", **_score("score_train", "f32", 32768, 256, 1, False)),
        # a language model's loss on a batch of sequences; the odd vocabulary leaves rows on odd addresses
        dict(name="score_train_8192x50257", **_score("score_train", "bf16", 8192, 50257, 4, False)),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["scan", "scan_train", "back", "back", "score", "score_train"])
    dtype = "bf16" if rng.random() < 0.7 else "f32"
    if kind.startswith("scan"):
        H = rng.choice([128, 256, 320, 512, 768, 1024, rng.randint(65, 1100)])
        top = 25_000_000 // (1 if dtype == "bf16" else 2)
        L = _log_int(rng, 1, 16384)
        B = _log_int(rng, 1, max(1, min(256, top // (L * H))))
        return _scan(kind, dtype, B, L, H, rng.choice([3, 4]), L > 1 and rng.random() < 0.4)
    if kind == "back":
        k = rng.choice([1, 1, 2, 3, 4, 8])
        d = rng.choice([128, 256, 384, 512, 768, 1024, 2048, 8 * rng.randint(20, 200)])
        T = _log_int(rng, 16, 65536 * 768 // (d * (k + 1) * SIZE[dtype] // 4 + 256))
        E = rng.choice([8, 16, 60, 64, 100, 128, 256])
        return _back(dtype, T, k, d, E, round(rng.uniform(0.6, 1.4), 2), rng.choice([0.0, 0.0, round(rng.uniform(0.1, 0.6), 2)]),
                     rng.choice([1.0, 1.25, 2.0, 4.0]), rng.randint(0, 1), rng.random() < 0.5)
    V = rng.choice([8, 64, 100, 128, 256, 1000, _log_int(rng, 2000, 200000), _log_int(rng, 2000, 200000)])
    N = _log_int(rng, 1, min(65536, 400_000_000 // (V * SIZE[dtype] // 2)))
    return _score(kind, dtype, N, V, rng.randint(0, 8), rng.random() < 0.3)


# ------------------------------------------------------------------------------------------------- inputs
def _counts(case):
    """Tokens of each popularity rank: a share `hot` on rank 0 and Zipf over the rest, rounded to whole tokens."""
    T, E, hot = case["T"], case["E"], case["hot"]
    w = np.arange(1, E + 1, dtype=np.float64) ** -case["zipf"]
    if hot > 0.0:
        w = np.concatenate([[hot], (1.0 - hot) * w[:-1] / w[:-1].sum()])
    edges = np.round(np.cumsum(w / w.sum()) * T).astype(np.int64)
    edges[-1] = T
    return np.diff(edges, prepend=0)


def _capacity(case):
    return max(4, math.ceil(case["cf"] * case["k"] * case["T"] / case["E"]))


def _step(case):
    return max(1, case["E"] // 8)                       # choice j of a token lies j steps further in the ranks


def _kept(case):
    n = _counts(case)
    total = sum(np.roll(n, j * _step(case)) for j in range(case["k"]))
    return np.minimum(total, _capacity(case))


def _lengths(case, g):
    L = case["L"]
    n = torch.randint(max(1, L // 3), L + 1, (case["B"],), generator=g, device="cuda", dtype=torch.int32)
    n[0] = L
    return n


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = dict(case=case)
    if case["kind"].startswith("scan"):
        B, L, H, k = case["B"], case["L"], case["H"], case["k"]
        s["u"] = normal(B, L, k * H)
        s["x"] = normal(B, L, H) if k == 3 else None
        # forget gates from short memories to memories of some fifty tokens
        s["b_f"] = torch.rand(H, generator=g, device="cuda") * 4.0
        s["b_r"] = normal(H, std=0.5, dtype=torch.float32)
        s["c0"] = normal(B, H, std=0.5, dtype=torch.float32)
        s["lengths"] = _lengths(case, g) if case["ragged"] else None
        if case["kind"] == "scan_train":
            s["dh"] = normal(B, L, H, std=0.1)
            s["dc_last"] = normal(B, H, std=0.1, dtype=torch.float32)
    elif case["kind"] == "back":
        T, k, d, E = case["T"], case["k"], case["d"], case["E"]
        rank = torch.repeat_interleave(torch.arange(E, device="cuda"), torch.from_numpy(_counts(case)).cuda())
        rank = rank[torch.randperm(T, generator=g, device="cuda")]
        id_of_rank = torch.randperm(E, generator=g, device="cuda")
        idx = torch.stack([id_of_rank[(rank + j * _step(case)) % E] for j in range(k)])
        flat = idx.reshape(-1)                          # all first choices before all second choices
        order = torch.sort(flat, stable=True).indices
        counts = torch.zeros(E, dtype=torch.int64, device="cuda").index_add_(0, flat, torch.ones_like(flat))
        first = torch.cumsum(counts, 0) - counts
        place = torch.empty_like(flat)
        place[order] = torch.arange(k * T, device="cuda") - first[flat[order]]
        kept = torch.clamp(counts, max=_capacity(case))
        offset = torch.cumsum(kept, 0) - kept
        inv = torch.where(place < kept[flat], offset[flat] + place, -1).to(torch.int32).view(k, T)
        s["expert_idx"], s["inv"] = idx.to(torch.int32), inv
        s["logits"] = normal(T, E, std=0.5, dtype=torch.float32)
        top = 4.0 - 0.5 * torch.arange(k, device="cuda")[:, None] + 0.2 * torch.rand(k, T, generator=g, device="cuda")
        s["logits"].scatter_(1, idx.t().contiguous(), top.t().contiguous())
        p = torch.softmax(s["logits"], 1).gather(1, idx.t()).t()
        s["weight"] = (p / p.sum(0) if case["renorm"] else p).contiguous()
        s["dout"] = normal(T, d, std=0.1)
        s["y_perm"] = normal(k * T, d, std=0.5)
        s["dx_perm"] = normal(k * T, d, std=0.1)
        # rows behind the last kept assignment are not written: a program's buffer, zero from the start
        s["out"] = dict(dy_perm=torch.zeros(k * T, d, dtype=dt, device="cuda"),
                        dweight=torch.empty(k, T, dtype=torch.float32, device="cuda"), dx=torch.empty(T, d, dtype=dt, device="cuda"))
    else:
        N, V = case["N"], case["V"]
        s["logits"] = normal(N, V, std=2.0)
        if case["masked"]:
            off = torch.rand(V, generator=g, device="cuda") < 0.25
            off[0] = False
            s["logits"][:, off] = -math.inf
        s["target"] = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
        if case["masked"]:
            s["target"][off[s["target"].long()]] = 0
        if N > 1:
            s["target"][torch.rand(N, generator=g, device="cuda") < 0.05] = -1       # padded positions
        if case["kind"] == "score_train":
            s["dlogprob"] = torch.full((N,), -1.0 / N, device="cuda")
            s["dentropy"] = torch.full((N,), -0.01 / N, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------- plain forms
def _carry(f, b, c0):
    """c_t = f_t c_{t-1} + b_t over axis 1 by doubling: after a step of width w, an entry spans 2 w positions."""
    a, c = f.clone(), b.clone()
    c[:, 0] += a[:, 0] * c0
    w = 1
    while w < f.shape[1]:
        c[:, w:] = c[:, w:] + a[:, w:] * c[:, :-w]
        a[:, w:] = a[:, w:] * a[:, :-w]
        w *= 2
    return c


def _scan_plain(s, train):
    case = s["case"]
    B, L, H, k, dt = case["B"], case["L"], case["H"], case["k"], DTYPES[case["dtype"]]
    u = s["u"].float().view(B, L, k, H)
    z, w = u[:, :, 0], (s["x"].float() if k == 3 else u[:, :, 3])
    f = 1.0 / (1.0 + torch.exp(-(u[:, :, 1] + s["b_f"])))
    r = 1.0 / (1.0 + torch.exp(-(u[:, :, 2] + s["b_r"])))
    on = None
    if s["lengths"] is not None:
        on = (torch.arange(L, device="cuda")[None, :] < s["lengths"][:, None])[:, :, None]
        f = torch.where(on, f, torch.ones_like(f))      # a state stands still behind its sequence's end
    c = _carry(f, (1.0 - f) * z, s["c0"])
    t = torch.tanh(c)
    h = r * t + (1.0 - r) * w
    h = h if on is None else torch.where(on, h, torch.zeros_like(h))
    out = dict(h=h.to(dt), c_last=c[:, -1].clone())
    if not train:
        return out
    dh = s["dh"].float()
    if on is not None:
        dh = torch.where(on, dh, torch.zeros_like(dh))
    # dc_t = dh_t r_t (1 - tanh^2 c_t) + f_{t+1} dc_{t+1}: the same recurrence from the end
    e = dh * r * (1.0 - t * t)
    e[:, -1] += s["dc_last"]
    nxt = torch.cat([f[:, 1:], torch.zeros_like(f[:, :1])], 1)
    dc = _carry(nxt.flip(1), e.flip(1), torch.zeros_like(s["c0"])).flip(1)
    before = torch.cat([s["c0"][:, None], c[:, :-1]], 1)
    du_f = dc * (before - z) * f * (1.0 - f)
    du_r = dh * (t - w) * r * (1.0 - r)
    parts = [dc * (1.0 - f), du_f, du_r]
    dw = dh * (1.0 - r)
    if k == 4:
        parts.append(dw)
    out.update(du=torch.stack(parts, 2).view(B, L, k * H).to(dt), dx=dw.to(dt) if k == 3 else None, db_f=du_f.sum((0, 1)),
               db_r=du_r.sum((0, 1)), dc0=dc[:, 0] * f[:, 0])
    return out


def _back_plain(s):
    case = s["case"]
    T, k, E, dt = case["T"], case["k"], case["E"], DTYPES[case["dtype"]]
    inv, w, out = s["inv"].long(), s["weight"], s["out"]
    on = inv >= 0
    at = inv.clamp(min=0)
    dout = s["dout"].float()
    gathered = dout.clone() if case["residual"] else torch.where(on.any(0)[:, None], torch.zeros_like(dout), dout)
    for j in range(k):
        rows = on[j].nonzero()[:, 0]
        out["dy_perm"][at[j, rows]] = (w[j, rows, None] * dout[rows]).to(dt)
        out["dweight"][j] = torch.where(on[j], (dout * s["y_perm"][at[j]].float()).sum(1), torch.zeros_like(w[j]))
        gathered = gathered + torch.where(on[j][:, None], s["dx_perm"][at[j]].float(), torch.zeros_like(dout))
    idx = s["expert_idx"].long().t()
    dw = out["dweight"].t()
    p = torch.exp(s["logits"] - s["logits"].amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True)
    chosen = p.gather(1, idx)
    if case["renorm"]:
        chosen = chosen / chosen.sum(1, keepdim=True)
        dlogits = torch.zeros_like(p).scatter_(1, idx, chosen * (dw - (chosen * dw).sum(1, keepdim=True)))
    else:
        dlogits = (-p * (chosen * dw).sum(1, keepdim=True)).scatter_add_(1, idx, chosen * dw)
    return dict(dy_perm=out["dy_perm"], dweight=out["dweight"], dx=gathered.to(dt), dlogits=dlogits)


def _score_plain(s, train):
    case = s["case"]
    N, V, k = case["N"], case["V"], min(case["k"], case["V"])
    x = s["logits"].float()
    m = x.amax(1, keepdim=True)
    z = x - m
    p = torch.exp(z)
    total = p.sum(1, keepdim=True)
    logp = z - torch.log(total)
    p = p / total
    entropy = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    on = (s["target"] >= 0) & (s["target"] < V)
    at = s["target"].long().clamp(0, V - 1)[:, None]
    out = dict(logprob=torch.where(on, logp.gather(1, at)[:, 0], torch.zeros_like(entropy)), entropy=entropy,
               lse=(m + torch.log(total))[:, 0])
    if k:
        left, ids = x.clone(), torch.arange(V, device="cuda").expand(N, V).clone()
        best = []
        for _ in range(k):                              # the largest that is left, the lowest id among equals
            top = left.amax(1, keepdim=True)
            best.append(torch.where(left == top, ids, V).amin(1, keepdim=True))
            left.scatter_(1, best[-1], -math.inf)
            ids.scatter_(1, best[-1], V)
        top_idx = torch.cat(best, 1)
        out.update(top_idx=top_idx.to(torch.int32), top_logprob=logp.gather(1, top_idx))
    if train:
        g = torch.where(on, s["dlogprob"], torch.zeros_like(entropy))[:, None]
        d = -g * p - s["dentropy"][:, None] * torch.where(p > 0, p * (logp + entropy[:, None]), torch.zeros_like(p))
        d.scatter_add_(1, at, g)
        out["dlogits"] = d.to(DTYPES[case["dtype"]])
    return out


# ------------------------------------------------------------------------------------------------- the framework's calls
def _scan_own(s, train):
    import paper_2605_11537_amd as moe
    h, c_last, states = moe.sru_scan(s["u"], s["x"], s["b_f"], s["b_r"], s["c0"], s["lengths"], want_states=train)
    out = dict(h=h, c_last=c_last)
    if train:
        out.update(moe.sru_scan_backward(s["dh"], s["u"], states, s["x"], s["b_f"], s["b_r"], s["dc_last"], s["lengths"]))
    return out


def _back_own(s):
    import paper_2605_11537_amd as moe
    case = s["case"]
    g = moe.moe_combine_topk_backward(s["dout"], s["y_perm"], s["inv"], s["weight"], case["residual"], out=s["out"])
    dx = moe.moe_dispatch_topk_backward(s["dx_perm"], s["inv"], dx_add=g["dx"])
    dlogits = moe.moe_route_topk_backward(s["logits"], s["expert_idx"], g["dweight"], case["renorm"])
    return dict(dy_perm=g["dy_perm"], dweight=g["dweight"], dx=dx, dlogits=dlogits)


def _score_own(s, train):
    import paper_2605_11537_amd as moe
    k = min(s["case"]["k"], s["case"]["V"])
    out = moe.moe_token_logprobs(s["logits"], s["target"], k)
    if not k:
        out.pop("top_idx"), out.pop("top_logprob")
    if train:
        out["dlogits"] = moe.moe_token_logprobs_backward(s["logits"], s["target"], out["lse"], out["entropy"], s["dlogprob"],
                                                         s["dentropy"])
    return out


def run(state):
    kind = state["case"]["kind"]
    if kind == "back":
        return _back_own(state) if own else _back_plain(state)
    train = kind.endswith("_train")
    if kind.startswith("scan"):
        return _scan_own(state, train) if own else _scan_plain(state, train)
    return _score_own(state, train) if own else _score_plain(state, train)


# ------------------------------------------------------------------------------------------------- work
def work(case):
    z = SIZE[case["dtype"]]
    if case["kind"].startswith("scan"):
        B, L, H, k = case["B"], case["L"], case["H"], case["k"]
        n = B * L * H
        read = k + (k == 3)
        nbytes = n * z * (read + 1) + (2 * B + 2) * H * 4
        flops = n * 25
        if case["kind"] == "scan_train":
            nbytes += n * z * (2 * read + 1) + (2 * B + 4) * H * 4
            flops += n * 50
        return dict(bytes=nbytes, flops=flops)
    if case["kind"] == "back":
        T, k, d, E = case["T"], case["k"], case["d"], case["E"]
        K = int(_kept(case).sum())
        rows = (T + K + K + T) + (K + T + T)            # combine: dout, y | dy, dx; dispatch: dx_perm, dx | dx
        return dict(bytes=rows * d * z + 2 * T * E * 4 + 6 * k * T * 4, flops=4 * K * d + 5 * T * E)
    N, V, k = case["N"], case["V"], case["k"]
    train = case["kind"] == "score_train"
    return dict(bytes=N * V * z * (3 if train else 1) + N * (16 + 8 * k + (20 if train else 0)), flops=N * V * (12 if train else 6))


# ------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"scan": _scan_exact, "back": _back_exact, "scor": _score_exact}[case["kind"][:4]](s, case)


def _scan_exact(s, case):
    """Token by token."""
    B, L, H, k = case["B"], case["L"], case["H"], case["k"]
    blocks = s["u"].view(B, L, k, H)
    n = s["lengths"].tolist() if s["lengths"] is not None else [L] * B
    n = torch.tensor(n, device="cuda")
    train = case["kind"] == "scan_train"
    bf, br = s["b_f"].double(), s["b_r"].double()
    c = s["c0"].double()
    hs, cs = [], [c]

    def token(t):
        z, a, b = (blocks[:, t, i].double() for i in range(3))
        w = s["x"][:, t].double() if k == 3 else blocks[:, t, 3].double()
        return z, w, torch.sigmoid(a + bf), torch.sigmoid(b + br), (t < n)[:, None]

    for t in range(L):
        z, w, f, r, on = token(t)
        c = torch.where(on, f * c + (1 - f) * z, c)
        hs.append(torch.where(on, r * torch.tanh(c) + (1 - r) * w, 0.0))
        if train:
            cs.append(c)
    out = dict(h=torch.stack(hs, 1), c_last=c)
    if not train:
        return out
    du = torch.zeros(B, L, k, H, dtype=torch.float64, device="cuda")
    dx = torch.zeros(B, L, H, dtype=torch.float64, device="cuda")
    dc = s["dc_last"].double()
    for t in reversed(range(L)):
        z, w, f, r, on = token(t)
        g = torch.tanh(cs[t + 1])
        dh = torch.where(on, s["dh"][:, t].double(), 0.0)
        dw = dh * (1 - r)
        (du[:, t, 3] if k == 4 else dx[:, t]).copy_(dw)
        du[:, t, 2] = dh * (g - w) * r * (1 - r)
        full = dc + dh * r * (1 - g * g)
        du[:, t, 0] = torch.where(on, full * (1 - f), 0.0)
        du[:, t, 1] = torch.where(on, full * (cs[t] - z) * f * (1 - f), 0.0)
        dc = torch.where(on, full * f, dc)
    out.update(du=du.view(B, L, k * H), dx=dx if k == 3 else None, db_f=du[:, :, 1].sum((0, 1)), db_r=du[:, :, 2].sum((0, 1)), dc0=dc)
    return out


def _back_exact(s, case):
    """Assignment by assignment, scattered from the permuted rows' side; the gate's gradient through the softmax's Jacobian."""
    T, k, d, E = case["T"], case["k"], case["d"], case["E"]
    inv = s["inv"].reshape(-1).long()
    a = (inv >= 0).nonzero()[:, 0]
    row, token = inv[a], a % T
    dout, w = s["dout"].double(), s["weight"].double().reshape(-1)
    dy = torch.zeros(k * T, d, dtype=torch.float64, device="cuda")
    dy[row] = w[a, None] * dout[token]
    dweight = torch.zeros(k * T, dtype=torch.float64, device="cuda")
    dweight[a] = (s["y_perm"][row].double() * dout[token]).sum(1)
    dx = torch.zeros(T, d, dtype=torch.float64, device="cuda")
    dx.index_add_(0, token, s["dx_perm"][row].double())
    lone = torch.ones(T, dtype=torch.bool, device="cuda")
    lone[token] = False
    dx += dout if case["residual"] else dout * lone[:, None]
    dweight = dweight.view(k, T)
    ids = s["expert_idx"].long()
    chosen = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, ids.t().contiguous(), 1.0)
    p = torch.softmax(s["logits"].double() + (torch.log(chosen) if case["renorm"] else 0.0), 1)
    dp = torch.zeros(T, E, dtype=torch.float64, device="cuda").scatter_(1, ids.t().contiguous(), dweight.t().contiguous())
    return dict(dy_perm=dy, dweight=dweight, dx=dx, dlogits=p * (dp - (p * dp).sum(1, keepdim=True)))


def _score_exact(s, case):
    """Rows in blocks; alternatives by sorting."""
    N, V, k = case["N"], case["V"], min(case["k"], case["V"])
    parts = []
    step = max(1, 50_000_000 // V)
    for lo in range(0, N, step):
        x = s["logits"][lo:lo + step].double()
        target = s["target"][lo:lo + step].long()
        lse = torch.logsumexp(x, 1)
        logp = x - lse[:, None]
        p = torch.exp(logp)
        entropy = torch.special.entr(p).sum(1)
        on = target >= 0
        at = target.clamp(min=0)[:, None]
        o = dict(logprob=torch.where(on, logp.gather(1, at)[:, 0], 0.0), entropy=entropy, lse=lse)
        if k:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]
            o.update(top_idx=ids.to(torch.int32), top_logprob=logp.gather(1, ids))
        if case["kind"] == "score_train":
            g = torch.where(on, s["dlogprob"][lo:lo + step].double(), 0.0)[:, None]
            q = s["dentropy"][lo:lo + step].double()[:, None]
            o["dlogits"] = g * (torch.zeros_like(x).scatter_(1, at, 1.0) - p) - q * (torch.xlogy(p, p) + p * entropy[:, None])
        parts.append(o)
    return {key: torch.cat([o[key] for o in parts]) for key in parts[0]}
