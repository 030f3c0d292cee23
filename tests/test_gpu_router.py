"""Routing by scores against a 64-bit form of the rule: ids equal, weights
within a few roundings of f32 (they are rounded once from 64 bits: half a step,
2^-24 relative, and 2^-40 for the 64-bit steps before it; a softmax that is not
renormalised divides by a sum of f32 exponentials, each off by at most 2^-22,
added up in at most 20 steps of 2^-24 each: 2^-19.5)."""

import numpy as np
import pytest
import torch

import ops_ref
import oracle
import paper_2505_08944_amd as aep
from gpu_helpers import assert_close, log, to_host

pytestmark = pytest.mark.gpu

W_TOL = 2.0 ** -24 + 2.0 ** -40

RULES = [
    dict(E=1, k=1), dict(E=8, k=2), dict(E=8, k=8, renorm=False), dict(E=60, k=4, score="sigmoid", scale=2.5),
    dict(E=64, k=6, renorm=False), dict(E=65, k=5, bias=True), dict(E=100, k=16, bias=True, score="sigmoid"),
    dict(E=160, k=6, n_groups=8, top_groups=3, renorm=False, scale=16.0),
    dict(E=256, k=8, n_groups=8, top_groups=4, group_top=2, score="sigmoid", bias=True, scale=2.5),
    dict(E=256, k=8, n_groups=8, top_groups=4, group_top=2, score="softmax"),
    dict(E=256, k=16, n_groups=64, top_groups=4, group_top=1, score="sigmoid", bias=True),
    dict(E=64, k=3, n_groups=64, top_groups=5, group_top=2, bias=True),  # groups of one
    dict(E=30, k=8, n_groups=3, top_groups=2, group_top=2, score="sigmoid"),
    dict(E=36, k=4, n_groups=4, top_groups=4, group_top=1, bias=True), dict(E=511, k=9, bias=True),
    dict(E=512, k=16, n_groups=4, top_groups=2, group_top=2, score="sigmoid", bias=True, renorm=False),
    dict(E=384, k=8, score="sigmoid", bias=True),
    dict(E=512, k=8, n_groups=64, top_groups=6, group_top=2, bias=True),
]


def rule(c):
    return {k: v for k, v in c.items() if k not in ("E", "k", "bias")}


def inputs(c, T, seed, mode="plain"):
    g = torch.Generator().manual_seed(seed)
    E = c["E"]
    l = torch.randn(T, E, generator=g) * 1.5
    b = torch.rand(E, generator=g) * (0.2 if c.get("score") == "sigmoid" else 0.02) if c.get("bias") else None
    if mode == "ties":  # few distinct values: experts and groups tie
        l = torch.randint(-2, 3, (T, E), generator=g).float()
        b = None if b is None else torch.randint(0, 2, (E,), generator=g).float() * 0.25
    elif mode == "masked":
        l.masked_fill_(torch.rand(T, E, generator=g) < torch.rand(T, 1, generator=g), float("-inf"))
        l[0] = float("-inf")  # nothing left
        if T > 1:
            l[1] = float("-inf")
            l[1, E // 2] = 1.0
    elif mode == "close":  # neighbours that 32 bits do not tell apart once the bias is added
        l = 8.0 + torch.randn(T, E, generator=g) * 1e-2
    elif mode == "offset":  # a bias so large that f32 sums keep little of the scores
        b = None if b is None else b + 50.0
    elif mode == "wide":
        l = l * 200.0
    return l, b


def check(c, l, b, idx, w):
    ri, rw = ops_ref.route(l.numpy(), c["k"], None if b is None else b.numpy(), **rule(c))
    gi, gw = to_host(idx), to_host(w).astype(np.float64)
    bad = np.argwhere((gi != ri).any(1)).ravel()
    assert not bad.size, (c, bad[:3], gi[bad[:2]], ri[bad[:2]])
    # results below f32's normal range are rounded to its fixed step there
    tol = W_TOL + (2.0 ** -19.5 if c.get("score", "softmax") == "softmax" and not c.get("renorm", True) else 0.0)
    assert np.all(np.abs(gw - rw) <= tol * rw + 2.0 ** -149), (c, np.abs(gw - rw).max())


@pytest.mark.parametrize("c", RULES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("mode", ["plain", "ties", "masked", "close", "offset", "wide"])
def test_rules(c, mode):
    r = aep.Router(c["E"], c["k"], **rule(c))
    for T in (1, 2, 33, 130):
        l, b = inputs(c, T, 3 * T + 1, mode)
        idx, w = aep.route(r, l.cuda(), None if b is None else b.cuda())
        assert idx.dtype == torch.int32 and w.dtype == torch.float32 and idx.shape == w.shape == (T, c["k"])
        check(c, l, b, idx, w)


def test_large_and_strided():
    c = RULES[8]
    r = aep.Router(c["E"], c["k"], **rule(c))
    l, b = inputs(c, 4099, 5)
    wide = torch.full((4099, 300), float("nan"))
    wide[:, 7:263] = l
    idx, w = aep.route(r, wide.cuda()[:, 7:263], b.cuda())
    check(c, l, b, idx, w)
    assert aep.route(r, l.cuda()[:0], b.cuda())[0].shape == (0, 8)


def test_reported_values():
    c = dict(E=40, k=4, bias=True)
    r = aep.Router(40, 4)
    l, b = inputs(c, 20, 9)
    flag = torch.zeros(1, dtype=torch.int32, device="cuda")
    l[2, 5] = float("-inf")
    aep.route(r, l.cuda(), b.cuda(), flag=flag)
    assert flag.item() == 0
    l[3, 7], l[4, 39] = float("nan"), float("inf")
    idx, w = aep.route(r, l.cuda(), b.cuda(), flag=flag)
    assert flag.item() == 1
    check(c, l, b, idx, w)
    flag.zero_()
    b[11] = float("nan")
    l, _ = inputs(c, 20, 10)
    idx, w = aep.route(r, l.cuda(), b.cuda(), flag=flag)
    assert flag.item() == 1
    check(c, l, b, idx, w)
    idx, w = aep.route(r, l.cuda(), b.cuda())  # nowhere to report to
    check(c, l, b, idx, w)


def test_streams_and_graphs():
    c = RULES[8]
    r = aep.Router(c["E"], c["k"], **rule(c))
    l, b = inputs(c, 100, 12)
    dl, db = l.cuda(), b.cuda()
    ref = aep.route(r, dl, db)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = aep.route(r, dl, db)
    for i in range(3):
        out[0].fill_(-1)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], ref[0]) and torch.equal(out[1], ref[1])
        l2, _ = inputs(c, 100, 20 + i)
        dl.copy_(l2)
        gr.replay()
        torch.cuda.synchronize()
        check(c, l2, b, *out)
        dl.copy_(l)


def test_refusals():
    r = aep.Router(8, 2)
    l = torch.zeros(4, 8, device="cuda")
    for bad in (dict(logits=l.double()), dict(logits=l[:, :7]), dict(logits=l.cpu()), dict(logits=l.t().contiguous().t()),
                dict(bias=torch.zeros(7, device="cuda")), dict(logits=l[:1].expand(4, 8)),
                dict(flag=torch.zeros(1, device="cuda")), dict(idx=torch.zeros(4, 2, device="cuda"))):
        a = dict(logits=l)
        a.update(bad)
        with pytest.raises(ValueError):
            aep.route(r, **a)
    with pytest.raises(ValueError):
        aep.Router(8, 2, score="tanh")
    with pytest.raises(aep.AEPError):
        aep.Router(8, 9)


# ------------------------------------------------------------------- queues
def ctx_for(c, T, d=64, S=0, pool=False, renorm=True):
    ctx = aep.Context(2, c["E"], d, 64, c["k"], n_shared=S, renorm=renorm, max_tokens_per_layer=T, token_pool=pool)
    up = torch.zeros(64, d, device="cuda", dtype=torch.bfloat16)
    down = torch.zeros(d, 64, device="cuda", dtype=torch.bfloat16)
    for layer in range(2):
        for e in range(c["E"] + S):
            ctx.set_expert_weights(layer, e, up, up, down)
    return ctx


def queue_ref(idx, w, x, E):
    flat = idx.reshape(-1)
    order = np.argsort(flat, kind="stable")
    pos = np.empty(flat.size, np.int32)
    pos[order] = np.arange(flat.size)
    return np.bincount(flat, minlength=E), pos.reshape(idx.shape), w.reshape(-1)[order], x[order // idx.shape[1]]


@pytest.mark.parametrize("i,frags", [(1, (5,)), (4, (1, 31, 40)), (7, (777,)), (8, (64, 33, 3)), (8, (2500, 1, 40)),
                                     (12, (4100,)), (13, (32, 32)), (14, (70, 1)),
                                     (17, (32, 45))])
@pytest.mark.parametrize("S", [0, 1])
def test_queues(i, frags, S):
    c = RULES[i]
    if c["k"] > 8:
        c = dict(c, k=8)
    T = sum(frags)
    log(f"queues E={c['E']} k={c['k']} fragments {frags}")
    ctx = ctx_for(c, T, S=S)
    parts = [inputs(c, t, 31 + j, "masked" if j == 1 else "plain") for j, t in enumerate(frags)]
    b = parts[0][1]
    ctx.set_router(1, aep.Router(c["E"], c["k"], **rule(c)), None if b is None else b.cuda())
    for rep in range(2):  # queues empty again after a drain
        x = torch.randn(T, 64).to(torch.bfloat16).cuda()
        at, routing = 0, []
        for l, _ in parts:
            routing.append(ctx.route_enqueue(1, x[at:at + l.shape[0]], l.cuda(), routing_out=True))
            at += l.shape[0]
        for (l, _), (gi, gw) in zip(parts, routing):
            check(c, l, b, gi, gw)
        idx, w = (torch.cat([r[j] for r in routing]) for j in (0, 1))
        counts, pos, rw, rows = queue_ref(to_host(idx), to_host(w), to_host(x), c["E"])
        assert np.array_equal(ctx.expert_counts(1), counts)
        bt = ctx.rebatch(1)
        assert np.array_equal(to_host(bt.counts())[:c["E"]], counts)
        assert np.array_equal(to_host(bt.token_pos()), pos)
        assert np.array_equal(to_host(bt.row_weight()), rw)
        assert np.array_equal(to_host(bt.token_weight()), to_host(w))
        assert np.array_equal(to_host(bt.x_perm())[:len(rows)], rows)
        ctx.release(bt)
        ctx.sync()


def test_layers_keep_their_own_rule():
    """Layer 0 by the context's rule, layer 1 by its router; and back again."""
    c = dict(E=16, k=2, score="sigmoid", bias=True, scale=3.0)
    ctx = ctx_for(c, 40)
    l, b = inputs(c, 40, 41)
    x = torch.randn(40, 64).to(torch.bfloat16).cuda()
    plain = aep.route(aep.Router(16, 2), l.cuda())
    ctx.set_router(1, aep.Router(16, 2, **rule(c)), b.cuda())
    own = ctx.route_enqueue(0, x, l.cuda(), routing_out=True)
    assert torch.equal(own[0], plain[0]) and torch.allclose(own[1], plain[1], rtol=4e-6, atol=0)
    check(c, l, b, *ctx.route_enqueue(1, x, l.cuda(), routing_out=True))
    for layer in (0, 1):
        ctx.release(ctx.rebatch(layer))
    ctx.set_router(1, None)
    again = ctx.route_enqueue(1, x, l.cuda(), routing_out=True)
    assert torch.equal(again[0], own[0]) and torch.equal(again[1], own[1])
    ctx.sync()


def test_non_finite_logits_are_reported_by_sync():
    c = dict(E=80, k=3)
    ctx = ctx_for(c, 50)
    ctx.set_router(0, aep.Router(80, 3))
    l, _ = inputs(c, 50, 43)
    l[0, 3] = float("-inf")
    x = torch.zeros(50, 64, dtype=torch.bfloat16, device="cuda")
    ctx.route_enqueue(0, x, l.cuda())
    ctx.release(ctx.rebatch(0))
    ctx.sync()
    l[9, 9] = float("nan")
    got = ctx.route_enqueue(0, x, l.cuda(), routing_out=True)
    check(c, l, None, *got)
    ctx.release(ctx.rebatch(0))
    with pytest.raises(aep.AEPError):
        ctx.sync()
    ctx.sync()


def test_pool_ids():
    """Caller ids and single-expert drains with a layer's router."""
    c = dict(E=72, k=3, score="sigmoid", bias=True)
    ctx = ctx_for(c, 64, pool=True)
    l, b = inputs(c, 40, 47)
    ctx.set_router(0, aep.Router(72, 3, **rule(c)), b.cuda())
    x = torch.randn(40, 64).to(torch.bfloat16).cuda()
    ids = torch.randperm(64)[:40].to(torch.int32).cuda()
    idx, w = ctx.route_enqueue_ids(0, x, l.cuda(), ids, routing_out=True)
    check(c, l, b, idx, w)
    want = np.bincount(to_host(idx).ravel(), minlength=72)
    assert np.array_equal(ctx.expert_counts(0), want)
    out, ready = torch.zeros(64, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(64, dtype=torch.int32, device="cuda")
    for e in range(72):
        bt = ctx.rebatch_expert(0, e)
        n = int(bt.counts()[e])
        assert n == want[e]
        rows = to_host(bt.row_token())[:n]
        assert np.array_equal(rows, to_host(ids)[np.argwhere((to_host(idx) == e).any(1)).ravel()])
        ctx.pool_accumulate(bt, ctx.expert_ffn(bt))
        ctx.release(bt)
    ctx.pool_release(0, out, ready)
    assert int(ready.sum()) == 40 and set(torch.nonzero(ready).ravel().tolist()) == set(ids.tolist())
    ctx.sync()


def test_enqueue_in_a_graph():
    c = RULES[8]
    T = 90
    ctx = ctx_for(c, T)
    l, b = inputs(c, T, 51)
    dl, x = l.cuda(), torch.randn(T, 64).to(torch.bfloat16).cuda()
    ctx.set_router(0, aep.Router(c["E"], c["k"], **rule(c)), b.cuda())

    def step():
        ctx.route_enqueue(0, x, dl)
        bt = ctx.rebatch(0)
        res = [t.clone() for t in (bt.counts(), bt.token_pos(), bt.row_weight(), bt.x_perm())]
        ctx.release(bt)
        return res

    ref = step()
    torch.cuda.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        out = step()
    for i in range(4):
        for o in out:
            o.zero_()
        gr.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, r) for a, r in zip(out, ref)), i
        assert all(torch.equal(a, r) for a, r in zip(step(), ref)), i
    ctx.sync()


# -------------------------------------------------------- all of it together
@pytest.mark.parametrize("T", [5, 200])
def test_layer_from_attention_output_to_experts(T):
    """Projection with its residual, gate product, routing by scores, experts, combine."""
    d, f, E, k = 256, 192, 96, 4
    g = torch.Generator().manual_seed(61)

    def rnd(*s, scale=1.0):
        return (torch.randn(*s, generator=g) * scale).to(torch.bfloat16).cuda()

    attn, h0, wo, wg = rnd(T, d), rnd(T, d), rnd(d, d, scale=d ** -0.5), rnd(E, d, scale=d ** -0.5)
    bias = (torch.rand(E, generator=g) * 0.2).cuda()
    ctx = aep.Context(1, E, d, f, k, max_tokens_per_layer=T)
    ws = []
    for e in range(E):
        w = (rnd(f, d, scale=d ** -0.5), rnd(f, d, scale=d ** -0.5), rnd(d, f, scale=f ** -0.5))
        ctx.set_expert_weights(0, e, *w)
        ws.append([t.double().cpu().numpy() for t in w])
    c = dict(E=E, k=k, score="sigmoid", n_groups=8, top_groups=4, group_top=2, scale=2.5)
    ctx.set_router(0, aep.Router(E, k, **rule(c)), bias)
    h = aep.linear(attn, wo, residual=h0)
    logits = aep.linear(h, wg, out_dtype=torch.float32)
    idx, w = ctx.route_enqueue(0, h, logits, routing_out=True)
    out = ctx.run_layer(0)
    ctx.sync()
    # each step against 64 bits on the inputs that it was given
    href = (attn.double() @ wo.double().T + h0.double()).cpu().numpy()
    assert_close(h.double().cpu().numpy(), href, 2.0 ** -7, "projection")
    hn = h.double().cpu().numpy()
    assert_close(logits.double().cpu().numpy(), hn @ wg.double().cpu().numpy().T, 1e-5, "gate logits")
    check(c, logits.cpu(), bias.cpu(), idx, w)
    ref = np.zeros((T, d))
    for t in range(T):
        for e, a in zip(to_host(idx)[t], to_host(w)[t]):
            gate, up, down = ws[e]
            v = gate @ hn[t]
            ref[t] += float(a) * (down @ (v / (1 + np.exp(-v)) * (up @ hn[t])))
    assert_close(out.double().cpu().numpy(), ref, 2e-2, "layer")
