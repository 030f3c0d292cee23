"""A layer's decode steps on 4-bit data, as a server runs them: the projection of queries, keys and values with 4-bit
weights, the new tokens into the cache, the attention, the output projection with the residual, gate, routing and
experts.  Every stage is checked on the inputs that it got, with the tolerances of its own tests."""

import numpy as np
import pytest
import torch

import mx4_ref
import paper_2505_08944_amd as aep
from gpu_helpers import BF16_RTOL, assert_close, log
from test_gpu_cache4 import i32, table
from test_gpu_linear import f64
from test_gpu_linear4 import check as check_linear

pytestmark = pytest.mark.gpu

D, HQ, HKV, HD, E, K, F, PAGE = 512, 8, 2, 64, 8, 2, 256, 32
WIDTH = (HQ + 2 * HKV) * HD


class Layer:
    def __init__(self, longest):
        g = torch.Generator(device="cuda").manual_seed(1)

        def rnd(*s, scale=1.0):
            return torch.randn(*s, device="cuda", generator=g) * scale

        self.wq, self.wo = (aep.quantize_mx4(rnd(n, k, scale=k ** -0.5)) for n, k in ((WIDTH, D), (D, HQ * HD)))
        self.values = [aep.dequantize_mx4(*w, k, dtype=torch.float32) for w, k in ((self.wq, D), (self.wo, HQ * HD))]
        self.qkv, self.out = aep.Linear4(*self.wq), aep.Linear4(*self.wo)
        self.gate_w = rnd(E, D, scale=D ** -0.5).to(torch.bfloat16)
        self.gate = aep.Linear(self.gate_w, out_dtype=torch.float32)
        self.router = aep.Router(E, K)
        self.cache = aep.Cache4(sum(-(-l // PAGE) for l in longest) + 1, HKV, HD, page_size=PAGE)
        self.pages = table(longest, PAGE, self.cache.n_pages)
        self.experts = [[rnd(*s, scale=0.05).to(torch.bfloat16) for s in ((F, D), (F, D), (D, F))] for _ in range(E)]
        self.ctx = aep.Context(1, E, D, F, K, max_tokens_per_layer=256)
        for e, w in enumerate(self.experts):
            self.ctx.set_expert_weights(0, e, *w)

    def attention(self, h, lens, rows=None):
        qkv = self.qkv(h).view(h.shape[0], HQ + 2 * HKV, HD)
        q, k, v = qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:]
        self.cache.append(k, v, self.pages, lens, rows)
        a = self.cache.attend(q, self.pages, lens, rows)
        return qkv, a, self.out(a.view(h.shape[0], HQ * HD), residual=h)

    def step(self, h, lens, rows=None):
        qkv, a, h2 = self.attention(h, lens, rows)
        logits = self.gate(h2)
        self.ctx.route_enqueue(0, h2, logits)
        return qkv, a, h2, logits, self.ctx.run_layer(0)


def check_step(layer, h, got, lens, n, history, what):
    """history: the kept keys and values of each sequence, float64 [l][heads][d], which this step's are added to."""
    qkv, a, h2, logits, out = got
    T = h.shape[0]
    check_linear(qkv.reshape(T, WIDTH), h, f64(layer.values[0]), None, None, "none", what)
    x, av = f64(qkv), f64(a)
    r = 0
    for b, m in enumerate(n):
        for part, lo in ((0, HQ), (1, HQ + HKV)):
            kept = mx4_ref.quantize(x[r:r + m, lo:lo + HKV])[2]
            history[b][part] = np.concatenate([history[b][part], kept])
        k, v = history[b]
        assert len(k) == lens[b]
        for i in range(m):
            for head in range(HQ):
                kv = head * HKV // HQ
                ref, _, spread, size, s = mx4_ref.attend(x[r + i, head], k[:, kv], v[:, kv], lens[b] - m + i, HD ** -0.5, 0)
                # (test_gpu_attend4.py)
                e = (HD + 8) * 2.0 ** -23 * s + 2.0 ** -23 * (2 * s + 12) + 2.0 ** -22
                tol = 1.02 * (e + 2.0 ** -8) * spread + (lens[b] / 32 + 256) * 2.0 ** -23 * size
                tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
                assert (np.abs(av[r + i, head] - ref) <= tol).all(), (what, b, i, head)
        r += m
    check_linear(h2, a.reshape(T, HQ * HD), f64(layer.values[1]), None, h, "none", what)
    check_linear(logits, h2, f64(layer.gate_w), None, None, "none", what)
    idx, w = (t.cpu().numpy() for t in aep.route(layer.router, logits))
    x2, want = f64(h2), np.zeros((T, D))
    for t in range(T):
        for j in range(K):
            g, u, d = (f64(m) for m in layer.experts[idx[t, j]])
            s = g @ x2[t]
            want[t] += w[t, j] * (d @ (s / (1 + np.exp(-s)) * (u @ x2[t])))
    assert_close(f64(out), want, BF16_RTOL, f"{what}: layer's output")


def test_prompts_then_single_tokens_then_a_captured_step():
    prompts = [70, 1, 33, 128, 5]
    longest = [p + 12 for p in prompts]
    layer = Layer(longest)
    B = len(prompts)
    g = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn(sum(prompts), D, device="cuda", generator=g).to(torch.bfloat16)
    history = [[np.zeros((0, HKV, HD)), np.zeros((0, HKV, HD))] for _ in range(B)]
    rows = i32(*np.concatenate([[0], np.cumsum(prompts)]).tolist())
    log("prompts")
    got = layer.step(h, i32(*prompts), rows)
    check_step(layer, h, got, prompts, prompts, history, "prompts")
    lens = list(prompts)
    for step in range(3):
        log(f"step {step}")
        h = torch.randn(B, D, device="cuda", generator=g).to(torch.bfloat16)
        lens = [l + 1 for l in lens]
        check_step(layer, h, layer.step(h, i32(*lens)), lens, [1] * B, history, f"step {step}")
    # the step once more, captured; between its replays the same step in eager mode, one token further
    log("captured steps")
    dev_lens, h = i32(*lens), torch.zeros(B, D, dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):  # (what the first call of each allocates)
        layer.step(h, i32(*[l + 1 for l in lens]))
    torch.cuda.current_stream().wait_stream(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dev_lens.add_(1)
        got = layer.step(h, dev_lens)
    dev_lens.copy_(i32(*lens))
    for step in range(3):
        h.copy_(torch.randn(B, D, device="cuda", generator=g))
        graph.replay()
        torch.cuda.synchronize()
        lens = [l + 1 for l in lens]
        assert dev_lens.tolist() == lens
        check_step(layer, h, got, lens, [1] * B, history, f"replay {step}")
        h1 = torch.randn(B, D, device="cuda", generator=g).to(torch.bfloat16)
        lens = [l + 1 for l in lens]
        check_step(layer, h1, layer.step(h1, i32(*lens)), lens, [1] * B, history, f"eager step after replay {step}")
        dev_lens.copy_(i32(*lens))
    layer.ctx.sync()
