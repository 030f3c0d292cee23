"""The operators in front of an expert layer's queues, as they are measured:
the dense product with its epilogue and the routing by scores.

A case is a dict of plain values.  ``op`` says which operator a pass runs:

* ``linear``: y = act(scale * (x W^T) + bias) + residual.  x [M][K] and the
  residual bf16 or f32; W [N][K] bf16, fp8 (e4m3 codes with a bf16 scale per
  output channel) or f32; bias f32; y of the activations' type or f32.
* ``route``: gate logits [T][E] f32 to expert ids [T][k] and weights [T][k].
  Scores are softmax or sigmoid; a bias may be added to them for the choice
  only; experts are limited to the best groups; weights are the chosen experts'
  scores, renormalised or not, times a scale.
* ``queue``: the same rule in front of a layer's queues: a fragment of tokens is
  routed and queued, and the layer re-batched.  Outputs: rows per expert, each
  (token, slot)'s row, the rows' weights and the rows themselves.

With ``own`` false, ``run`` computes them in elementary torch operations.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

LINEAR = dict(op="linear", act="bf16", wdt="bf16", out="bf16", bias=False, residual=False, fn="none")
ROUTE = dict(op="route", score="softmax", bias=False, n_groups=1, top_groups=1, group_top=1, renorm=True, scale=1.0,
             masked=0.0)


def listed():
    return [
        # gate logits of a decode step of the fine-grained layer: all latency
        dict(LINEAR, name="gate_decode_32", M=32, N=64, K=2048, out="f32"),
        # gate logits of a prefill batch of that layer: one pass over the tokens
        dict(LINEAR, name="gate_prefill_8192", M=8192, N=64, K=2048, out="f32"),
        # attention output back to the residual stream in a decode step of the
        # Mixtral-style layer: the weights' stream
        dict(LINEAR, name="proj_decode_32", M=32, N=4096, K=4096, residual=True),
        # one token through the first product of a dense feed-forward block, fp8 weights
        dict(LINEAR, name="up_fp8_1", M=1, N=14336, K=4096, wdt="fp8", bias=True, fn="silu"),
        # a ragged batch of mixed prefill and decode with everything in the epilogue
        dict(LINEAR, name="proj_777", M=777, N=4096, K=4096, bias=True, fn="gelu", residual=True),
        # sizes off every tile, rows that start at any two bytes
        dict(LINEAR, name="odd_101", M=101, N=1531, K=1027, bias=True, fn="gelu_tanh", residual=True),
        # the tiny f32 layer's sizes
        dict(LINEAR, name="tiny_f32_256", M=256, N=512, K=256, act="f32", wdt="f32", out="f32", bias=True, fn="relu",
             residual=True),
        # the second product of a dense feed-forward block, a prefill batch, fp8 weights
        dict(LINEAR, name="down_fp8_2048", M=2048, N=4096, K=14336, wdt="fp8", residual=True),
        # the first product of that block for a full prefill batch: the matrix cores
        dict(LINEAR, name="up_4096", M=4096, N=14336, K=4096, bias=True, fn="silu"),
        # a decode step's tokens over 256 experts: sigmoid scores, a balance bias, 4 of 8 groups
        dict(ROUTE, name="route_64", T=64, E=256, k=8, score="sigmoid", bias=True, n_groups=8, top_groups=4,
             group_top=2, scale=2.5),
        # a prefill batch under the same rule
        dict(ROUTE, name="route_8192", T=8192, E=256, k=8, score="sigmoid", bias=True, n_groups=8, top_groups=4,
             group_top=2, scale=2.5),
        # a ragged fragment routed into the queues: softmax scores, 3 of 8 groups by their best expert
        dict(ROUTE, name="queue_777", op="queue", T=777, E=160, k=6, d=2048, n_groups=8, top_groups=3, group_top=1,
             renorm=False, scale=16.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["gate", "dense", "dense", "dense", "dense_f32", "route", "route", "queue"])
    if kind == "gate":
        return dict(LINEAR, M=_log(rng, 1, 8192), N=_log(rng, 8, 512), K=64 * rng.randint(16, 112), out="f32",
                    bias=rng.random() < 0.2)
    if kind.startswith("dense"):
        f32 = kind == "dense_f32"
        M = _log(rng, 1, 512 if f32 else 4096)
        N = _log(rng, 64, 2048) if f32 else _log(rng, 256, 14336)
        K = _log(rng, 64, 2048) if f32 else _log(rng, 256, 14336)
        if rng.random() < 0.85:  # most rows are aligned
            K = (K + 15) // 16 * 16
        K = max(64, min(K, 4096 * 14336 * 4096 // (M * N)))
        if f32:
            t = dict(act="f32", wdt="f32", out="f32")
        else:
            t = dict(wdt=rng.choice(["bf16", "bf16", "fp8"]), out=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        return dict(LINEAR, M=M, N=N, K=K, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                    fn=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]), **t)
    groups = rng.choice([1, 1, 4, 8])
    E = groups * rng.randint(*{1: (8, 256), 4: (4, 64), 8: (2, 48)}[groups])
    top = 1 if groups == 1 else rng.randint(2, groups - 1)
    k = rng.randint(1, min(8, top * E // groups))
    c = dict(ROUTE, E=E, k=k, n_groups=groups, top_groups=top, group_top=rng.choice([1, 2]),
             score=rng.choice(["softmax", "sigmoid"]), bias=rng.random() < 0.6, renorm=rng.random() < 0.7,
             scale=rng.choice([1.0, 2.5, 16.0]), masked=rng.choice([0.0, 0.0, 0.1, 0.6]))
    if kind == "route":
        return dict(c, T=_log(rng, 1, 16384))
    return dict(c, op="queue", T=_log(rng, 1, 4096), d=64 * rng.randint(8, 64))


# ------------------------------------------------------------------ inputs
_TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _linear_inputs(c, seed):
    gen, act = _gen(seed), _TYPES[c["act"]]

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, device="cuda", generator=gen, dtype=dtype)

    w = randn(c["N"], c["K"], dtype=torch.float32 if c["wdt"] == "f32" else torch.bfloat16).mul_(0.02)
    scale = None
    if c["wdt"] == "fp8":
        scale = (w.abs().amax(1).float() / 448.0).to(torch.bfloat16)
        w = (w.float() / scale.float()[:, None]).clamp_(-448.0, 448.0).to(torch.float8_e4m3fn)
    return {"x": randn(c["M"], c["K"], dtype=act), "w": w, "scale": scale,
            "bias": randn(c["N"]).mul_(0.1) if c["bias"] else None,
            "residual": randn(c["M"], c["N"], dtype=act) if c["residual"] else None}


def _route_inputs(c, seed):
    gen, T, E = _gen(seed), c["T"], c["E"]
    # experts differ in popularity, and some may be away (their logits are masked)
    rank = torch.randperm(E, device="cuda", generator=gen).float() + 1.0
    logits = torch.randn(T, E, device="cuda", generator=gen) - 0.5 * torch.log(rank)
    if c["masked"]:
        away = torch.rand(E, device="cuda", generator=gen) < c["masked"]
        logits.masked_fill_(away[None, :], float("-inf"))
    bias = None
    if c["bias"]:
        bias = torch.rand(E, device="cuda", generator=gen) * (0.2 if c["score"] == "sigmoid" else 0.02)
    x = None
    if c["op"] == "queue":
        x = torch.randn(T, c["d"], device="cuda", generator=gen, dtype=torch.bfloat16)
    return {"logits": logits, "bias": bias, "x": x}


def prepare(case, seed):
    c = case
    if c["op"] == "linear":
        st = dict(_linear_inputs(c, seed), case=c)
        if own:
            import paper_2505_08944_amd as aep
            st["lin"] = aep.Linear(st["w"], scale=st["scale"], bias=st["bias"], activation=c["fn"],
                                   out_dtype=_TYPES[c["out"]])
        return st
    st = dict(_route_inputs(c, seed), case=c)
    if own:
        import paper_2505_08944_amd as aep
        st["router"] = aep.Router(c["E"], c["k"], score=c["score"], n_groups=c["n_groups"], top_groups=c["top_groups"],
                                  group_top=c["group_top"], renorm=c["renorm"], scale=c["scale"])
        if c["op"] == "queue":
            ctx = aep.Context(1, c["E"], c["d"], 64, c["k"], renorm=c["renorm"], max_tokens_per_layer=c["T"])
            up = torch.zeros(64, c["d"], device="cuda", dtype=torch.bfloat16)
            down = torch.zeros(c["d"], 64, device="cuda", dtype=torch.bfloat16)
            for e in range(c["E"]):
                ctx.set_expert_weights(0, e, up, up, down)
            ctx.set_router(0, st["router"], st["bias"])
            st["ctx"] = ctx
    return st


# -------------------------------------------------------------- plain forms
def _plain_linear(st):
    c = st["case"]
    w = st["w"].float()
    if st["scale"] is not None:
        w = w * st["scale"].float()[:, None]
    y = torch.matmul(st["x"].float(), w.T)
    if st["bias"] is not None:
        y = y + st["bias"]
    if c["fn"] == "relu":
        y = torch.maximum(y, torch.zeros_like(y))
    elif c["fn"] == "silu":
        y = y / (1.0 + torch.exp(-y))
    elif c["fn"] == "gelu":
        y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
    elif c["fn"] == "gelu_tanh":
        y = 0.5 * y * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (y + 0.044715 * y * y * y)))
    if st["residual"] is not None:
        y = y + st["residual"].float()
    return y.to(_TYPES[c["out"]])


def _plain_route(st):
    # in 64 bits, as neighbours in the order may be closer than 32 bits tell apart
    c, k, G = st["case"], st["case"]["k"], st["case"]["n_groups"]
    lo = float("-inf")
    logits = st["logits"].double()
    T, E = logits.shape
    masked = torch.isinf(logits)
    if c["score"] == "softmax":
        m = logits.amax(1, keepdim=True)
        e = torch.exp(logits - torch.where(torch.isinf(m), torch.zeros_like(m), m))
        total = e.sum(1, keepdim=True)
        score = e / torch.where(total > 0, total, torch.ones_like(total))
    else:
        score = 1.0 / (1.0 + torch.exp(-logits))
    choice = score
    if st["bias"] is not None:
        choice = score + st["bias"].double()
    choice = torch.where(masked, torch.full_like(choice, lo), choice)
    # without a bias experts are compared by their logits, which order them as their scores do
    key = choice if st["bias"] is not None else logits
    if G > 1:
        per = E // G
        n = min(c["group_top"], per)
        if n == 1:
            value = key.view(T, G, per).amax(2)
        else:
            best = torch.sort(choice.view(T, G, per), dim=2, descending=True, stable=True).values[:, :, :n]
            value = torch.where(torch.isinf(best), torch.zeros_like(best), best).sum(2)
            value = torch.where(torch.isinf(best[:, :, 0]), torch.full_like(value, lo), value)
        kept = torch.sort(value, dim=1, descending=True, stable=True).indices[:, :c["top_groups"]]
        stays = torch.zeros(T, G, device=logits.device, dtype=torch.bool).scatter_(1, kept, True)
        stays = stays[:, :, None].expand(T, G, per).reshape(T, E)
        # masked experts of the groups that stay come before those of the others
        key = torch.where(masked, torch.full_like(key, -1e300), key)
        key = torch.where(stays, key, torch.full_like(key, lo))
    idx = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :k]
    w = torch.gather(score, 1, idx)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = w / torch.where(total > 0, total, torch.ones_like(total))
    return idx.to(torch.int32), (w * c["scale"]).float()


def _plain_queue(st):
    c = st["case"]
    idx, w = _plain_route(st)
    flat = idx.flatten().long()
    order = torch.sort(flat, stable=True).indices
    pos = torch.empty_like(order)
    pos[order] = torch.arange(order.numel(), device=order.device)
    counts = (flat[:, None] == torch.arange(c["E"], device=flat.device)[None, :]).sum(0)
    return {"counts": counts.to(torch.int32), "token_pos": pos.view(idx.shape).to(torch.int32),
            "row_weight": w.flatten()[order], "rows": st["x"][order // c["k"]]}


def run(state):
    st = state
    op = st["case"]["op"]
    if not own:
        return {"linear": _plain_linear, "route": _plain_route, "queue": _plain_queue}[op](st)
    if op == "linear":
        return st["lin"](st["x"], residual=st["residual"])
    if op == "route":
        import paper_2505_08944_amd as aep
        return aep.route(st["router"], st["logits"], st["bias"])
    ctx = st["ctx"]
    ctx.route_enqueue(0, st["x"], st["logits"])
    b = ctx.rebatch(0)
    out = {"counts": b.counts(), "token_pos": b.token_pos(), "row_weight": b.row_weight(), "rows": b.x_perm()}
    ctx.release(b)
    return out


# ---------------------------------------------------------------- reference
def work(case):
    c = case
    if c["op"] == "linear":
        M, N, K = c["M"], c["N"], c["K"]
        size = {"f32": 4, "bf16": 2, "fp8": 1}
        nbytes = M * K * size[c["act"]] + N * K * size[c["wdt"]] + M * N * size[c["out"]]
        nbytes += (M * N * size[c["act"]] if c["residual"] else 0) + (4 * N if c["bias"] else 0)
        nbytes += 2 * N if c["wdt"] == "fp8" else 0
        return {"bytes": nbytes, "flops": 2 * M * N * K}
    T, E, k = c["T"], c["E"], c["k"]
    nbytes = 4 * T * E + (4 * E if c["bias"] else 0)
    # a score, and k comparisons, for each expert
    flops = T * E * (4 + k)
    if c["op"] == "route":
        return {"bytes": nbytes + 8 * T * k, "flops": flops}
    return {"bytes": nbytes + 2 * T * c["d"] + 2 * T * k * c["d"] + 8 * T * k + 4 * E, "flops": flops}


def _exact_linear(c, seed):
    st = _linear_inputs(c, seed)
    w = st["w"].float().double()
    if st["scale"] is not None:
        w.mul_(st["scale"].double()[:, None])
    out = []
    for rows in torch.split(torch.arange(c["M"], device="cuda"), 2048):
        y = torch.nn.functional.linear(st["x"][rows].double(), w, None if st["bias"] is None else st["bias"].double())
        F = torch.nn.functional
        y = {"none": lambda v: v, "relu": F.relu, "silu": F.silu, "gelu": F.gelu,
             "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}[c["fn"]](y)
        if st["residual"] is not None:
            y = y + st["residual"][rows].double()
        out.append(y)
    return torch.cat(out)


def _exact_choice(c, logits, bias):
    """Expert ids and weights by their definition, one token's selection after another's rounds."""
    T, E = logits.shape
    k, G, per = c["k"], c["n_groups"], c["E"] // c["n_groups"]
    live = np.isfinite(logits)
    with np.errstate(over="ignore", invalid="ignore"):
        if c["score"] == "sigmoid":
            s = np.where(live, 1.0 / (1.0 + np.exp(-np.where(live, logits, 0.0))), 0.0)
        else:
            top = np.where(live, logits, -np.inf).max(1, keepdims=True)
            s = np.where(live, np.exp(np.where(live, logits, 0.0) - np.where(np.isfinite(top), top, 0.0)), 0.0)
            s = s / np.maximum(s.sum(1, keepdims=True), 1e-300)
    pick = s + bias if bias is not None else logits
    pick = np.where(live, pick, -np.inf)
    open_ = np.ones((T, E), bool)
    if G > 1:
        worth = s + bias if bias is not None else (pick if c["group_top"] == 1 or per == 1 else s)
        left = np.where(live, worth, -np.inf).reshape(T, G, per).copy()
        value = left.max(2)
        if c["group_top"] == 2 and per > 1:
            np.put_along_axis(left, left.argmax(2)[:, :, None], -np.inf, 2)
            second = left.max(2)
            value = value + np.where(np.isfinite(second), second, 0.0)
        group_open = np.zeros((T, G), bool)
        at = np.arange(T)
        for _ in range(c["top_groups"]):
            v = np.where(group_open, -np.inf, value)
            # -inf means taken or empty: among equal ones the first that is still free
            first = np.where(np.isfinite(v).any(1), v.argmax(1), (~group_open).argmax(1))
            group_open[at, first] = True
        open_ = np.repeat(group_open, per, 1)
    idx = np.zeros((T, k), np.int32)
    at = np.arange(T)
    for j in range(k):
        v = np.where(open_, pick, -np.inf)
        idx[:, j] = np.where(np.isfinite(v).any(1), v.argmax(1), open_.argmax(1))
        open_[at, idx[:, j]] = False
    w = np.take_along_axis(s, idx.astype(np.int64), 1)
    if c["renorm"]:
        w = w / np.maximum(w.sum(1, keepdims=True), 1e-300)
    return idx, w * c["scale"]


def exact(case, seed):
    c = case
    if c["op"] == "linear":
        return _exact_linear(c, seed)
    st = _route_inputs(c, seed)
    bias = None if st["bias"] is None else st["bias"].cpu().numpy().astype(np.float64)
    idx, w = _exact_choice(c, st["logits"].cpu().numpy().astype(np.float64), bias)
    if c["op"] == "route":
        return idx, w
    flat = idx.reshape(-1)
    rows = [np.flatnonzero(flat == e) for e in range(c["E"])]
    order = np.concatenate(rows)
    pos = np.empty(flat.size, np.int32)
    pos[order] = np.arange(flat.size)
    return {"counts": np.array([len(r) for r in rows], np.int32), "token_pos": pos.reshape(idx.shape),
            "row_weight": w.reshape(-1)[order],
            "rows": st["x"].double()[torch.from_numpy(order // c["k"]).cuda()]}
