"""Answers from whole tables, and training beyond the plain cross entropy, as cases that can be timed and compared.

Three operators that stand beside the full softmax's: log probabilities of given ids against a whole table, with the
entropy of every row and its best ids (what a trained model answers with); their gradients, for objectives that hold
the entropy up; and an update whose singular values are brought near 1 by Newton-Schulz products, alone and as the
step of an optimizer with momentum (Muon).

Where `own` is true the passes go through this library's entry points; where it is false they are elementary torch
operations in 32 bits, with what decides between neighbours (which of two nearly equal scores is larger) and the norm of
a whole matrix in 64.  Ids are skewed as nodes of graphs are, a share of them is padding (-1), scores of unrelated rows
spread by about 1, and updates have a few strong directions over many weak ones.
"""
from __future__ import annotations

import math

import torch

own = False

A, B, C = 3.4445, -4.7750, 2.0315       # of a step X <- A X + (B G + C G^2) X, G = X X^T
STEPS = 5
LR, MU, DECAY = 1e-3, 0.95, 0.01
MORE = 32               # candidates beside the best k whose scores are taken again in 64 bits


def listed():
    return [
        # The smallest call: one node's ten most likely neighbours, as a program that answers queries asks.  Latency counts.
        {"name": "answers 1 bf16 d256", "kind": "answers", "V": 200_003, "d": 256, "n": 1, "k": 10, "type": "bf16", "given": False},
        # An interactive batch against a small table.
        {"name": "answers 48 f32 d128", "kind": "answers", "V": 10_000, "d": 128, "n": 48, "k": 20, "type": "f32", "given": False},
        # A held-out batch of odd sizes: probabilities of its pairs, and the alternatives for hits among the first ten.
        {"name": "answers 10k f32 d100", "kind": "answers", "V": 10_000, "d": 100, "n": 10_007, "k": 10, "type": "f32", "given": True},
        # The same of a ragged batch against a larger table of odd width.
        {"name": "answers 1.5k bf16 d200", "kind": "answers", "V": 100_003, "d": 200, "n": 1500, "k": 50, "type": "bf16", "given": True},
        # The largest: wide embeddings, a large batch, a large table.
        {"name": "answers 8k bf16 d512", "kind": "answers", "V": 200_003, "d": 512, "n": 8192, "k": 16, "type": "bf16", "given": True},
        # A training step's probabilities, entropies and gradients on few rows of a wide table.
        {"name": "entropy step 16 f32 d256", "kind": "step", "V": 200_003, "d": 256, "n": 16, "type": "f32"},
        # The same of a batch on a small graph.
        {"name": "entropy step 4k f32 d128", "kind": "step", "V": 10_000, "d": 128, "n": 4096, "type": "f32"},
        # The same of a large batch on a large table.
        {"name": "entropy step 8k bf16 d512", "kind": "step", "V": 200_003, "d": 512, "n": 8192, "type": "bf16"},
        # The update of a small projection, alone.
        {"name": "orthogonal 1000 x 100 f32", "kind": "orthogonal", "rows": 1000, "cols": 100, "type": "f32"},
        # The update of a small graph's table, of odd sizes, in bf16.
        {"name": "orthogonal 10k x 300 bf16", "kind": "orthogonal", "rows": 10_007, "cols": 300, "type": "bf16"},
        # The optimizer's step on the table of a graph of a million nodes.
        {"name": "muon 1M x 128 f32", "kind": "muon", "rows": 1_000_000, "cols": 128, "type": "f32", "copy": False},
        # The same on a table of wide embeddings, with gradients and a copy of the parameters in bf16.
        {"name": "muon 200k x 512 bf16", "kind": "muon", "rows": 200_003, "cols": 512, "type": "bf16", "copy": True},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["answers", "answers", "answers", "step", "step", "orthogonal", "orthogonal", "muon"])
    case = {"kind": kind, "type": rng.choice(["f32", "bf16"])}
    if kind in ("orthogonal", "muon"):
        cols = log(16, 1024)
        rows = log(100, min(1_000_000, 128_000_000 // cols, 52_000_000_000 // (cols * cols)))
        if kind == "muon":
            return {**case, "rows": rows, "cols": cols, "copy": rng.random() < 0.5}
        return {**case, "rows": cols, "cols": rows} if rng.random() < 0.25 else {**case, "rows": rows, "cols": cols}
    d = log(32, 1024)
    V = log(10_000, 200_003)
    most = min(16_384, int((2e11 if case["type"] == "f32" else 8e11) / (V * d)), 1_600_000_000 // V)
    if kind == "step":
        return {**case, "V": V, "d": d, "n": log(1, max(2, most))}
    k = log(1, 64)
    return {**case, "V": V, "d": d, "n": log(1, max(2, min(most, 400_000_000 // ((k + MORE) * d)))), "k": k, "given": rng.random() < 0.5}


# ---------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------
def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _ids(V, n, gen):
    """int32 [n]: density of id rank r about r^(-2/3), ranks scattered over the ids; 3 of 100 positions are padding."""
    a = 2654435761 % V
    while math.gcd(a, V) != 1:
        a += 1
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    ids = ((u * u * u * V).to(torch.int64).clamp_(max=V - 1) * a + 40503 % V) % V
    if n > 1:
        ids[torch.rand(n, generator=gen, device="cuda") < 0.03] = -1
    return ids.to(torch.int32)


def _normal(shape, sd, gen):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, sd, generator=gen)


def _update(rows, cols, gen):
    """A gradient of a table: up to 16 directions that many rows share, of falling strength, over what is each row's own;
    rows of hubs are larger than others."""
    r = min(16, rows, cols)
    strong = (_normal((rows, r), 1.0, gen) * torch.arange(1, r + 1, device="cuda") ** -0.5) @ _normal((r, cols), 1.0, gen)
    return (strong.mul_(0.3) + _normal((rows, cols), 1.0, gen)) * (torch.exp(_normal((rows, 1), 0.5, gen)) * 1e-4)


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, dt, s = case["kind"], _type(case["type"]), {"case": case}
    if kind == "orthogonal":
        s["x"] = _update(case["rows"], case["cols"], gen).to(dt)
        return s
    if kind == "muon":
        s["g"] = _update(case["rows"], case["cols"], gen).to(dt)
        s["m"] = _update(case["rows"], case["cols"], gen) * 8.0
        s["p"] = _normal((case["rows"], case["cols"]), 0.1, gen)
        if case["copy"]:
            s["copy"] = s["p"].bfloat16()
        return s
    V, d, n = case["V"], case["d"], case["n"]
    sd = d ** -0.25
    ids = _ids(V, n, gen)
    w = _normal((V, d), sd, gen)
    s["h"] = (_normal((n, d), sd, gen) + 0.3 * w[ids.long().clamp(min=0)]).to(dt)       # rows that lean to their targets
    s["w"] = w.to(dt)
    s["ids"] = ids if kind == "step" or case["given"] else None
    return s


def _handles(case, s):
    """Outputs and workspaces that a program on this library keeps."""
    import paper_2005_13789_amd as ne
    kind = case["kind"]
    empty = lambda *shape, dtype=torch.float32: torch.empty(shape, dtype=dtype, device="cuda")  # noqa: E731
    if kind in ("orthogonal", "muon"):
        s["work"] = empty(ne.ne_orthogonalize_workspace_bytes(case["rows"], case["cols"]), dtype=torch.uint8)
        if kind == "orthogonal":
            s["out"] = torch.empty_like(s["x"])
        return
    n, V, d = case["n"], case["V"], case["d"]
    s["lse"], s["entropy"] = empty(n), empty(n)
    if s["ids"] is not None:
        s["logp"] = empty(n)
    k = case.get("k", 0)
    if k:
        s["top_ids"], s["top_logp"] = empty(n, k, dtype=torch.int32), empty(n, k)
    size = ne.ne_logprob_workspace_bytes(n, V, d, _type(case["type"]), k=k)
    if kind == "step":
        s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
        size = max(size, ne.ne_logprob_workspace_bytes(n, V, d, _type(case["type"]), grad=True))
    s["work"] = empty(size, dtype=torch.uint8)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handles(case, s)
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
ENTROPY = 0.05          # the weight of the entropy in what a training step maximises


def _answers_of(case):
    return [name for name, there in (("logp", case["kind"] == "step" or case["given"]), ("entropy", True), ("top_ids", "k" in case),
                                     ("top_logp", "k" in case), ("dh", case["kind"] == "step"), ("dw", case["kind"] == "step")) if there]


def _step_size(case):
    """Of the largest side: what makes an update's elements about as large as Adam's."""
    return 0.2 * math.sqrt(max(case["rows"], case["cols"]))


def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2005_13789_amd as ne
    case, kind = s["case"], s["case"]["kind"]
    if kind == "orthogonal":
        ne.ne_orthogonalize(s["x"], s["out"], s["work"], steps=STEPS)
        return s["out"]
    if kind == "muon":
        ne.ne_muon_step(s["p"], s["g"], s["m"], s["work"], LR, momentum=MU, nesterov=True, weight_decay=DECAY, scale=_step_size(case),
                        steps=STEPS, param_bf16=s.get("copy"))
        return {k: s[k] for k in ("p", "m", "copy") if k in s}
    ne.ne_logprob(s["h"], s["w"], s["ids"], s["lse"], s["work"], logp=s.get("logp"), entropy=s["entropy"], top_ids=s.get("top_ids"),
                  top_logp=s.get("top_logp"))
    if kind == "step":
        n = case["n"]
        ne.ne_logprob_grad(s["h"], s["w"], s["ids"], s["lse"], s["entropy"], s["dh"], s["dw"], s["work"], logp_scale=-1.0 / n,
                           entropy_scale=-ENTROPY / n)
    return {k: s[k] for k in _answers_of(case)}


def _orthogonal_plain(x):
    wide = x.shape[0] < x.shape[1]
    x = x.t() if wide else x
    norm = torch.sqrt(x.double().square().sum()).float()
    x = x / norm.clamp(min=1e-30)
    for _ in range(STEPS):
        g = x.t() @ x
        x = A * x + x @ (B * g + C * (g @ g))
    return x.t() if wide else x


def _run_plain(s):
    case, kind, dt = s["case"], s["case"]["kind"], _type(s["case"]["type"])
    if kind == "orthogonal":
        return _orthogonal_plain(s["x"].float()).to(dt)
    if kind == "muon":
        g = s["g"].float()
        s["m"] = s["m"] * MU + g
        o = _orthogonal_plain(g + s["m"] * MU)
        s["p"] = s["p"] * (1.0 - LR * DECAY) - o * (LR * _step_size(case))
        if "copy" in s:
            s["copy"] = s["p"].bfloat16()
        return {k: s[k] for k in ("p", "m", "copy") if k in s}
    n, ids, k = case["n"], s["ids"], case.get("k", 0)
    h, w = s["h"].float(), s["w"].float()
    logits = h @ w.t()
    top = logits.amax(1, keepdim=True)
    logits -= top
    p = torch.exp(logits)
    total = p.sum(1, keepdim=True)
    log_total = torch.log(total)
    p /= total
    entropy = (log_total - (p * logits).sum(1, keepdim=True))
    found = {}
    if k:       # the best by 32 bits and some more, in the order of their scores in 64, the lower id first
        some = torch.topk(logits, min(k + MORE, case["V"]), dim=1, sorted=False)[1].sort(dim=1)[0]
        score = (w[some].double() * h[:, None, :].double()).sum(2)
        order = torch.sort(score, dim=1, descending=True, stable=True)
        found["top_ids"] = some.gather(1, order[1][:, :k]).to(torch.int32)
        found["top_logp"] = ((order[0][:, :k] - top.double()) - log_total.double()).float()
    if ids is not None:
        at = ids.long().clamp(min=0)[:, None]
        named = (ids >= 0)[:, None]
        found["logp"] = torch.where(named, logits.gather(1, at) - log_total, 0.0)[:, 0]
    if kind == "step":      # p (1 + e (log p + entropy)) - [target], over n
        g = (logits - log_total + entropy) * (ENTROPY / n) + 1.0 / n
        g *= p
        g.scatter_add_(1, at, torch.full_like(at, -1.0 / n, dtype=torch.float32))
        g *= named
        found |= {"dh": (g @ w).to(dt), "dw": (g.t() @ h).to(dt)}
    found["entropy"] = entropy[:, 0]
    if ids is not None:     # padding has no answers
        found["entropy"] = torch.where(named[:, 0], found["entropy"], 0.0)
        if k:
            found["top_ids"] = torch.where(named, found["top_ids"], -1)
            found["top_logp"] = torch.where(named, found["top_logp"], -math.inf)
    return {k: found[k] for k in _answers_of(case)}


def work(case):
    """Inputs once, outputs once; the scores computed once, and one product for each gradient; of Newton-Schulz products one symmetric
    matrix of the small side, and one product with a polynomial of it."""
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind in ("orthogonal", "muon"):
        size, small = float(case["rows"]) * case["cols"], float(min(case["rows"], case["cols"]))
        per = 2 * e if kind == "orthogonal" else 16 + e + (2 if case["copy"] else 0)
        return {"bytes": per * size, "flops": 3 * size * small}
    V, d, n, k = float(case["V"]), float(case["d"]), float(case["n"]), case.get("k", 0)
    rows = (n + V) * d * e
    if kind == "step":
        return {"bytes": 2 * rows + 16 * n, "flops": 6 * n * V * d}
    return {"bytes": rows + n * (4 + 8 * k + (8 if case["given"] else 0)), "flops": 2 * n * V * d}


# ---------------------------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_orthogonal(x):
    """By Horner's rule on the smaller side's matrix."""
    x = x.double()
    small_first = x.shape[0] <= x.shape[1]
    y = (x if small_first else x.t()).contiguous()
    y = y / torch.linalg.vector_norm(y)
    one = torch.eye(y.shape[0], dtype=torch.float64, device=y.device)
    for _ in range(STEPS):
        g = torch.mm(y, y.t())
        y = torch.mm(A * one + torch.mm(g, B * one + C * g), y)
    return y if small_first else y.t()


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "orthogonal":
        return _exact_orthogonal(s["x"])
    if kind == "muon":
        g = s["g"].double()
        m = MU * s["m"].double() + g
        p = s["p"].double()
        p = p - LR * DECAY * p - LR * _step_size(case) * _exact_orthogonal(g + MU * m)
        return {"p": p, "m": m, **({"copy": p} if case["copy"] else {})}
    n, V, d, k = case["n"], case["V"], case["d"], case.get("k", 0)
    W = s["w"].double()
    out = {"logp": torch.zeros(n, dtype=torch.float64, device="cuda"), "entropy": torch.zeros(n, dtype=torch.float64, device="cuda"),
           "top_ids": torch.full((n, k), -1, dtype=torch.int32, device="cuda"),
           "top_logp": torch.full((n, k), -math.inf, dtype=torch.float64, device="cuda"),
           "dh": torch.zeros((n, d), dtype=torch.float64, device="cuda")}
    if kind == "step":
        out["dw"] = torch.zeros_like(W)
    for lo in range(0, n, 1024):        # rows that count, a share of the batch at a time
        rows = torch.arange(lo, min(lo + 1024, n), device="cuda")
        if s["ids"] is not None:
            rows = rows[s["ids"][rows] >= 0]
        H = s["h"][rows].double()
        L = torch.log_softmax(torch.mm(H, W.t()), dim=1)
        P = torch.exp(L)
        out["entropy"][rows] = E = -(P * L).sum(1)
        if s["ids"] is not None:
            mine, t = torch.arange(rows.numel(), device="cuda"), s["ids"][rows].long()
            out["logp"][rows] = L[mine, t]
        if k:
            best, ids = torch.topk(L, k, dim=1)
            out["top_ids"][rows], out["top_logp"][rows] = ids.to(torch.int32), best
        if kind == "step":      # of -(log p_target + ENTROPY entropy) / n
            D = P * (1.0 + ENTROPY * (L + E[:, None]))
            D[mine, t] -= 1.0
            out["dh"][rows] = torch.mm(D, W) / n
            out["dw"] += torch.mm(D.t(), H) / n
    return {name: out[name] for name in _answers_of(case)}
