"""The operators of full-softmax training, as cases that can be timed and compared.

A table's rows are looked up and scaled, scored against every row of a second table (softmax cross entropy over a
large vocabulary, logits never kept), the gradients come back to both tables, and AdamW moves them with states in 32
or in 8 bits.  Every case is one operator, or for the loss in training the pair of calls that a step makes.

Where `own` is true the passes go through this library's entry points; where it is false they are elementary torch
operations in 32 bits.  Ids are skewed as nodes of graphs and words of texts are (a few ids name a large share of the
positions), a share of them is padding (-1), and values are those of trained embeddings: scores of unrelated rows
spread by about 1.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

LR, B1, B2, EPS = 1e-3, 0.9, 0.999, 1e-8
BLOCK = 256             # elements that share a scale where AdamW's states have 8 bits


def listed():
    return [
        # The smallest call: the row of one node, as a program that answers queries fetches it.  Latency counts.
        {"name": "lookup 1 f32 d128", "kind": "lookup", "V": 1_000_000, "d": 128, "n": 1, "type": "f32"},
        # The rows of a large batch.
        {"name": "lookup 262k bf16 d256", "kind": "lookup", "V": 1_000_000, "d": 256, "n": 262_144, "type": "bf16"},
        # The gradient of a small interactive batch into a small table.
        {"name": "embed grad 4k f32 d128", "kind": "embed_grad", "V": 10_000, "d": 128, "n": 4096, "type": "f32",
         "accumulate": False},
        # The gradient of a large batch into a dense gradient that the optimizer reads whole.
        {"name": "embed grad 65k bf16 d512", "kind": "embed_grad", "V": 200_003, "d": 512, "n": 65_536, "type": "bf16",
         "accumulate": False},
        # Odd sizes, added to what another part of the model left there (a table used on both sides).
        {"name": "embed grad add 10k f32 d100", "kind": "embed_grad", "V": 1_000_000, "d": 100, "n": 10_007, "type": "f32",
         "accumulate": True},
        # One position scored against the whole table: serving.
        {"name": "loss 1 bf16 d256", "kind": "loss", "V": 200_003, "d": 256, "n": 1, "type": "bf16"},
        # Loss of a held-out batch of odd sizes, as the loss curve is taken.
        {"name": "loss 10k f32 d100", "kind": "loss", "V": 10_000, "d": 100, "n": 10_007, "type": "f32"},
        # A training step's loss and gradients on a small graph, in the tables' own type.
        {"name": "xent 4k f32 d128", "kind": "xent", "V": 10_000, "d": 128, "n": 4096, "type": "f32"},
        # A ragged batch against a larger table of odd width.
        {"name": "xent 1.5k bf16 d200", "kind": "xent", "V": 100_003, "d": 200, "n": 1500, "type": "bf16"},
        # The largest: wide embeddings, a large batch, a large table.
        {"name": "xent 8k bf16 d512", "kind": "xent", "V": 200_003, "d": 512, "n": 8192, "type": "bf16"},
        # Both tables of a graph of a million nodes, states in 32 bits.
        {"name": "adamw32 2 x 1M d128", "kind": "adamw", "bits": 32, "tensors": 2, "largest": 128_000_000, "ragged": False,
         "grad": "f32"},
        # Many tensors of all sizes, states in 8 bits, gradients and a copy of the parameters in bf16.
        {"name": "adamw8 64 ragged", "kind": "adamw", "bits": 8, "tensors": 64, "largest": 4_000_000, "ragged": True,
         "grad": "bf16"},
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["lookup", "embed_grad", "embed_grad", "loss", "loss", "xent", "xent", "adamw"])
    if kind == "adamw":
        tensors = log(1, 64)
        return {"kind": kind, "bits": rng.choice([8, 32]), "tensors": tensors, "largest": log(1000, 256_000_000 // tensors),
                "ragged": rng.random() < 0.7, "grad": rng.choice(["f32", "bf16"])}
    kind_of = {"kind": kind, "type": rng.choice(["f32", "bf16"])}
    if kind in ("lookup", "embed_grad"):
        d = log(16, 1024)
        case = {**kind_of, "V": log(10_000, min(1_000_000, 256_000_000 // d)), "d": d, "n": log(1, min(262_144, 100_000_000 // d))}
        return {**case, "accumulate": rng.random() < 0.4} if kind == "embed_grad" else case
    d = log(32, 1024)
    V = log(10_000, 200_003)
    most = 2e11 if kind_of["type"] == "f32" else 8e11
    return {**kind_of, "V": V, "d": d, "n": log(1, max(2, min(16_384, int(most / (V * d)), 1_600_000_000 // V)))}


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


def _numels(case):
    """Elements of each tensor: all of the largest size, or falling by a factor each to a single element."""
    T, largest = case["tensors"], case["largest"]
    if not case["ragged"]:
        return [largest] * T
    return [max(1, int(largest ** (1 - i / max(T - 1, 1)))) for i in range(T)]


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    kind, s = case["kind"], {"case": case, "seed": int(seed)}
    if kind == "adamw":     # the tensors lie in one buffer each, every one from a multiple of a block on
        numels = _numels(case)
        first = np.concatenate([[0], np.cumsum([-(-n // BLOCK) * BLOCK for n in numels])]).astype(np.int64)
        total = int(first[-1])
        real = torch.zeros(total, dtype=torch.float32, device="cuda")
        decay = torch.zeros(total // BLOCK, dtype=torch.float32, device="cuda")
        tensor = torch.zeros(total // BLOCK, dtype=torch.int64, device="cuda")
        for t, n in enumerate(numels):
            real[int(first[t]):int(first[t]) + n] = 1.0
            decay[int(first[t]) // BLOCK:int(first[t + 1]) // BLOCK] = 0.01 if n > 4096 else 0.0
            tensor[int(first[t]) // BLOCK:int(first[t + 1]) // BLOCK] = t
        s |= {"numels": numels, "first": first, "decay": decay, "tensor": tensor}
        s["first_block"] = torch.from_numpy(first[:-1] // BLOCK).cuda()[tensor]
        # gradients whose size differs from block to block, as those of layers and of rare rows do
        size = torch.exp(_normal(total // BLOCK, 1.0, gen)).repeat_interleave(BLOCK) * 1e-3
        s["p"] = _normal(total, 0.1, gen) * real
        s["g"] = (_normal(total, 1.0, gen) * size * real).to(_type(case["grad"]))
        m, r = _normal(total, 0.3, gen) * size * real, (_normal(total, 0.2, gen) + 1.0).abs_() * size * real
        s["step"] = 1000
        if case["bits"] == 32:
            s["m"], s["v"] = m, r.square_()
        else:
            for name, x in (("m", m), ("v", r)):
                scale = x.view(-1, BLOCK).abs().amax(1).clamp_(min=2.0 ** -100) / 448.0
                s[name] = (x.view(-1, BLOCK) / scale[:, None]).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn).view(-1)
                s[name + "_scale"] = scale
            s["copy"] = s["p"].bfloat16()
        return s
    V, d, n, dt = case["V"], case["d"], case["n"], _type(case["type"])
    sd = d ** -0.25
    s["ids"] = _ids(V, n, gen)
    if kind == "lookup":
        s["table"] = _normal((V, d), sd, gen).to(dt)
        s["out"] = torch.empty((n, d), dtype=dt, device="cuda")
    elif kind == "embed_grad":
        s["grad"] = _normal((n, d), 1e-3, gen).to(dt)
        s["table_grad"] = _normal((V, d), 1e-3, gen).to(dt) if case["accumulate"] else torch.empty((V, d), dtype=dt, device="cuda")
    else:       # rows that already lean to their targets
        w = _normal((V, d), sd, gen)
        s["h"] = (_normal((n, d), sd, gen) + 0.3 * w[s["ids"].long().clamp(min=0)]).to(dt)
        s["w"] = w.to(dt)
    return s


def _handles(case, s):
    """Outputs, workspaces and handles that a program on this library keeps."""
    import paper_2005_13789_amd as ne
    kind = case["kind"]
    if kind == "adamw":
        first, numels = s["first"], s["numels"]
        split = lambda x, unit=1: [x[int(f) // unit:int(f) // unit + -(-n // unit)] for f, n in zip(first, numels)]  # noqa: E731
        more = {}
        if case["bits"] == 8:
            more = {"m_scale": split(s["m_scale"], BLOCK), "v_scale": split(s["v_scale"], BLOCK), "params_bf16": split(s["copy"])}
        s["opt"] = ne.ne_create_adamw(split(s["p"]), split(s["g"]), split(s["m"]), split(s["v"]),
                                      torch.empty(ne.ne_adamw_workspace_bytes(numels), dtype=torch.uint8, device="cuda"),
                                      weight_decay=[0.01 if n > 4096 else 0.0 for n in numels], seed=s["seed"], **more)
    elif kind == "embed_grad":
        s["work"] = torch.empty(ne.ne_embed_workspace_bytes(case["V"], case["d"], case["n"]), dtype=torch.uint8, device="cuda")
    elif kind in ("loss", "xent"):
        s["loss"], s["lse"] = (torch.empty(case["n"], dtype=torch.float32, device="cuda") for _ in range(2))
        if kind == "xent":
            s["dh"], s["dw"] = torch.empty_like(s["h"]), torch.empty_like(s["w"])
        size = ne.ne_xent_workspace_bytes(case["n"], case["V"], case["d"], _type(case["type"]), grad=kind == "xent")
        s["work"] = torch.empty(size, dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        _handles(case, s)
    return s


# ---------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    import paper_2005_13789_amd as ne
    case, kind = s["case"], s["case"]["kind"]
    if kind == "lookup":
        ne.ne_embed_lookup(s["table"], s["ids"], s["out"], scale=math.sqrt(case["d"]))
        return s["out"]
    if kind == "embed_grad":
        ne.ne_embed_grad(s["ids"], s["grad"], s["table_grad"], s["work"], scale=math.sqrt(case["d"]), accumulate=case["accumulate"])
        return s["table_grad"]
    if kind == "adamw":
        s["step"] += 1
        ne.ne_adamw_step(s["opt"], s["step"], LR, B1, B2, EPS)
        return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if k in s}
    ne.ne_xent_loss(s["h"], s["w"], s["ids"], s["loss"], s["lse"], s["work"])
    if kind == "loss":
        return {"loss": s["loss"], "lse": s["lse"]}
    ne.ne_xent_grad(s["h"], s["w"], s["ids"], s["lse"], s["dh"], s["dw"], s["work"], scale=1.0 / case["n"])
    return {"loss": s["loss"], "lse": s["lse"], "dh": s["dh"], "dw": s["dw"]}


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "adamw":
        return _adamw_plain(s)
    V, d, dt, ids = case["V"], case["d"], _type(case["type"]), s["ids"].long()
    named = ids >= 0
    if kind == "lookup":
        x = s["table"][ids.clamp(min=0)].float() * math.sqrt(d)
        return (x * named[:, None]).to(dt)
    if kind == "embed_grad":
        old = s["table_grad"].float() if case["accumulate"] else torch.zeros((V, d), dtype=torch.float32, device="cuda")
        g = s["grad"].float() * math.sqrt(d) * named[:, None]
        # (32-bit gradients that are added to are added to in place, as the entry point does)
        new = old.index_add_(0, ids.clamp(min=0), g)
        if case["accumulate"] and dt != torch.float32:
            s["table_grad"].copy_(new)
            return s["table_grad"]
        return new.to(dt)
    h, w = s["h"].float(), s["w"].float()
    logits = h @ w.t()
    top = logits.amax(1)
    e = torch.exp(logits - top[:, None])
    total = e.sum(1)
    lse = top + torch.log(total)
    at = ids.clamp(min=0)[:, None]
    loss = torch.where(named, lse - logits.gather(1, at)[:, 0], 0.0)
    lse = torch.where(named, lse, 0.0)
    if kind == "loss":
        return {"loss": loss, "lse": lse}
    e *= (named / (total * case["n"]))[:, None]
    e.scatter_add_(1, at, -(named.float() / case["n"])[:, None])
    return {"loss": loss, "lse": lse, "dh": (e @ w).to(dt), "dw": (e.t() @ h).to(dt)}


M32 = 0xFFFFFFFF


def _philox(c, seed):
    """Philox4x32-10 words for counters of four int64 tensors that hold 32 bits each."""
    k0, k1 = seed & M32, (seed >> 32) & M32
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [((p1 >> 32) & M32) ^ c[1] ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c[3] ^ k1, p0 & M32]
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    return torch.stack(c, dim=1)


def _round_words(s):
    """int64 [elements]: word e % 4 of counter (e / 4, tensor, step, 3), e counted inside its tensor."""
    blocks = torch.arange(s["tensor"].numel(), device="cuda")
    group = (((blocks - s["first_block"]) * (BLOCK // 4))[:, None] + torch.arange(BLOCK // 4, device="cuda")).reshape(-1)
    tensor = s["tensor"].repeat_interleave(BLOCK // 4)
    return _philox([group, tensor, torch.full_like(group, s["step"]), torch.full_like(group, 3)], s["seed"]).reshape(-1)


def _e4m3_at_random(x, r16, keep):
    """x [blocks][BLOCK] over its block's largest magnitude, as e4m3, rounded up with the probability that keeps its
    expectation; keep: a value above 0 does not become 0.  Returns (float8 values, scales)."""
    top = x.abs().amax(1).clamp(min=2.0 ** -100)
    y = x * (448.0 / top)[:, None]
    a = y.abs().clamp(max=448.0)
    r16 = r16.view_as(x)
    big = ((a.view(torch.int32) + (r16 << 4).to(torch.int32)) & -0x100000).view(torch.float32)
    small = torch.floor(a * 512.0 + r16.float() * 2.0 ** -16)
    if keep:
        small = torch.where(a > 0, small.clamp(min=1.0), small)
    a = torch.where(a < 2.0 ** -6, small * 2.0 ** -9, big)
    return torch.copysign(a, y).to(torch.float8_e4m3fn).view(-1), top / 448.0


def _adamw_plain(s):
    s["step"] += 1
    bits, t = s["case"]["bits"], s["step"]
    f32 = lambda x: float(np.float32(x))  # noqa: E731
    b1, b2, c1, c2 = f32(B1), f32(B2), f32(1.0 - f32(B1)), f32(1.0 - f32(B2))
    size, root, eps = f32(f32(LR) / (1.0 - b1 ** t)), f32(1.0 / math.sqrt(1.0 - b2 ** t)), f32(EPS)
    g = s["g"].float()
    if bits == 8:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        r = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        v = r * r
    else:
        m, v = s["m"], s["v"]
    m = m * b1 + g * c1
    v = v * b2 + (g * g) * c2
    r = torch.sqrt(v)
    kept = (1.0 - s["decay"] * f32(LR)).repeat_interleave(BLOCK)
    p = s["p"] * kept - (m / (r * root + eps)) * size
    s["p"] = p
    if bits == 32:
        s["m"], s["v"] = m, v
        return {"p": p, "m": m, "v": v}
    words = _round_words(s)
    s["m"], s["m_scale"] = _e4m3_at_random(m.view(-1, BLOCK), words & 0xFFFF, False)
    s["v"], s["v_scale"] = _e4m3_at_random(r.view(-1, BLOCK), words >> 16, True)
    s["copy"] = p.bfloat16()
    return {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy")}


def work(case):
    """Inputs once, outputs once; the scores of a training step computed once, and one product for each gradient."""
    kind = case["kind"]
    if kind == "adamw":
        n = float(sum(_numels(case)))
        g = 4 if case["grad"] == "f32" else 2
        per = 8 + g + 16 if case["bits"] == 32 else 8 + g + 4 + 16 / BLOCK + 2
        return {"bytes": per * n, "flops": 15 * n}
    V, d, n, e = float(case["V"]), float(case["d"]), float(case["n"]), 4 if case["type"] == "f32" else 2
    if kind == "lookup":
        return {"bytes": 4 * n + 2 * n * d * e, "flops": n * d}
    if kind == "embed_grad":
        rows = 2 * min(n, V) if case["accumulate"] else V
        return {"bytes": 4 * n + n * d * e + rows * d * e, "flops": 2 * n * d}
    if kind == "loss":
        return {"bytes": (n + V) * d * e + 12 * n, "flops": 2 * n * V * d}
    return {"bytes": 2 * (n + V) * d * e + 12 * n, "flops": 6 * n * V * d}


# ---------------------------------------------------------------------------------------------
# the same in 64 bits
# ---------------------------------------------------------------------------------------------
def _exact_xent(s, case, train):
    n, V, d = case["n"], case["V"], case["d"]
    W = s["w"].double()
    loss, lse = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    dH, dW = torch.zeros((n, d), dtype=torch.float64, device="cuda"), torch.zeros_like(W)
    for lo in range(0, n, 1024):        # rows that have a target, a share of the batch at a time
        rows = torch.nonzero(s["ids"][lo:lo + 1024] >= 0)[:, 0] + lo
        t = s["ids"][rows].long()
        H = s["h"][rows].double()
        S = torch.mm(H, W.t())
        z = torch.logsumexp(S, dim=1)
        lse[rows], loss[rows] = z, z - S[torch.arange(rows.numel(), device="cuda"), t]
        if train:
            P = torch.exp(S.sub_(z[:, None]))
            P[torch.arange(rows.numel(), device="cuda"), t] -= 1.0
            dH[rows] = torch.mm(P, W) / n
            dW += torch.mm(P.t(), H) / n
    return {"loss": loss, "lse": lse, "dh": dH, "dw": dW} if train else {"loss": loss, "lse": lse}


def _exact_e4m3(x, r16, keep):
    top = torch.clamp(x.abs().amax(1, keepdim=True), min=2.0 ** -100)
    a = torch.clamp(x.abs() * (448.0 / top), max=448.0)
    e = torch.clamp(torch.floor(torch.log2(torch.clamp(a, min=2.0 ** -30))), min=-6.0)
    unit = torch.exp2(e - 3.0)
    q = torch.floor(a / unit + r16.view_as(x).double() / 65536.0)
    if keep:
        q = torch.where((q == 0) & (a > 0), 1.0, q)
    return (torch.sign(x) * q * unit).view(-1), (top / 448.0).view(-1)


def _exact_adamw(s, case):
    t = s["step"] + 1
    s["step"] = t
    g, p, m, v = (s[k].double() for k in ("g", "p", "m", "v"))
    if case["bits"] == 8:
        m = m * s["m_scale"].double().repeat_interleave(BLOCK)
        v = (v * s["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    b1, b2, lr, eps = (float(np.float32(x)) for x in (B1, B2, LR, EPS))
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    p = p - lr * s["decay"].double().repeat_interleave(BLOCK) * p
    p = p - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + eps)
    if case["bits"] == 32:
        return {"p": p, "m": m, "v": v}
    words = _round_words(s)
    m, ms = _exact_e4m3(m.view(-1, BLOCK), words % 65536, False)
    v, vs = _exact_e4m3(torch.sqrt(v).view(-1, BLOCK), words // 65536, True)
    return {"p": p, "m": m, "v": v, "m_scale": ms, "v_scale": vs, "copy": p}


def exact(case, seed):
    s, kind = _inputs(case, seed), case["kind"]
    if kind == "adamw":
        return _exact_adamw(s, case)
    if kind in ("loss", "xent"):
        return _exact_xent(s, case, kind == "xent")
    V, d, ids = case["V"], case["d"], s["ids"].long()
    root = float(np.float32(math.sqrt(d)))
    if kind == "lookup":
        out = torch.zeros((case["n"], d), dtype=torch.float64, device="cuda")
        out[ids >= 0] = s["table"][ids[ids >= 0]].double() * root
        return out
    out = s["table_grad"].double() if case["accumulate"] else torch.zeros((V, d), dtype=torch.float64, device="cuda")
    out.index_add_(0, ids[ids >= 0], s["grad"][ids >= 0].double() * root)
    return out
