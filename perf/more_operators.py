"""The operators of a decode step on 4-bit data, as they are measured: the dense
product with 4-bit weights, the quantiser, and the attention's paged cache of
keys and values in 4 bits, written and read.

All of them hold values in one format (OCP MXFP4): blocks of 32 consecutive
values share a power of two, and a value is a code of 4 bits, sign and one of 0,
0.5, 1, 1.5, 2, 3, 4, 6.  A block's power is the smallest at which its largest
value is at most 7 times it; a value goes to the nearest code, in the middle to
the even one.

A case is a dict of plain values.  ``op`` says which operator a pass runs:

* ``linear4``: y = act(x W^T + bias) + residual.  x [M][K] bf16, W [N][K] in 4
  bits, bias f32, y and the residual bf16, or y f32.
* ``quantize``: a matrix [N][K], bf16 or f32, to 4 bits.  Output: the values.
* ``append``: the newest n rows of keys and values of each of B sequences go
  into their pages, and are read back.  Outputs: the values that were kept.
* ``attend``: each of the newest n rows of queries of each sequence attends to
  the tokens up to its own (the last ``window`` of them where it is not 0), Hq
  heads over Hkv heads of the cache.  Output: [B n][Hq][D] bf16; zeros where a
  sequence has no token for a row.

Sequences are as long as ``lengths`` says, whatever the seed.  With ``own`` false,
``run`` computes them in elementary torch operations.
"""

from __future__ import annotations

import math

import torch

own = False

LINEAR = dict(op="linear4", out="bf16", bias=False, residual=False, fn="none")
CACHE = dict(Hkv=8, D=128, page=64, n=1, empty=False)
ATTEND = dict(CACHE, op="attend", Hq=32, window=0)


def listed():
    return [
        # one token through the first product of a dense feed-forward block: the weights' stream
        dict(LINEAR, name="up4_1", M=1, N=14336, K=4096, bias=True, fn="silu"),
        # attention output back to the residual stream in a decode step of the
        # Mixtral-style layer
        dict(LINEAR, name="proj4_32", M=32, N=4096, K=4096, residual=True),
        # a few rows, sizes off every tile, a last block that is not whole
        dict(LINEAR, name="odd4_13", M=13, N=1531, K=1027, bias=True, fn="gelu", residual=True, out="f32"),
        # a ragged batch of mixed prefill and decode: the matrix cores
        dict(LINEAR, name="proj4_777", M=777, N=4096, K=4096, residual=True),
        # the fine-grained layer's narrow matrix, odd rows
        dict(op="quantize", name="quant_1408", N=1408, K=2045, x="f32"),
        # the first matrix of a dense feed-forward block at load time: the copy's rate
        dict(op="quantize", name="quant_14336", N=14336, K=4096, x="bf16"),
        # a decode step's keys and values of 64 sequences: latency
        dict(CACHE, op="append", name="append_64", B=64, longest=8192),
        # prompts of 8 sequences behind what they have already
        dict(CACHE, op="append", name="append_8x1021", B=8, n=1021, longest=4096),
        # draft tokens of 16 sequences, a head of the cache for each head, a window: small work
        dict(ATTEND, name="draft_16", B=16, n=5, Hq=16, Hkv=16, D=64, longest=2048, window=1024, page=32),
        # one sequence, one token, a long context: few rows, the split over the context
        dict(ATTEND, name="long_1", B=1, longest=100003),
        # a decode step of 64 sequences of any length up to 16384, 4 heads to a head of the cache
        dict(ATTEND, name="decode_64", B=64, longest=16384, empty=True),
        # a piece of 4 prompts against what they have already: the matrix cores
        dict(ATTEND, name="chunk_4", B=4, n=509, longest=8192),
    ]


def lengths(c):
    """Tokens that the cache holds of each sequence, the newest n among them."""
    B, longest, n = c["B"], c["longest"], c["n"]
    if B == 1:
        return [longest]
    out = []
    for b in range(B):
        share = math.modf((b + 1) * 0.6180339887498949)[0]
        out.append(max(n, min(longest, 1 + int(longest * share))))
    if c["empty"]:  # a padded batch: slots without a sequence
        out = [0 if b % 8 == 5 else l for b, l in enumerate(out)]
    return out


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear4", "linear4", "quantize", "append", "attend", "attend", "attend"])
    if kind == "linear4":
        M, N, K = _log(rng, 1, 777), _log(rng, 256, 14336), _log(rng, 256, 14336)
        if rng.random() < 0.75:  # most rows are whole blocks
            K = (K + 31) // 32 * 32
        if M > 16:
            K = max(64, min(K, 777 * 4096 * 4096 // (M * N)))
        return dict(LINEAR, M=M, N=N, K=K, bias=rng.random() < 0.5, residual=rng.random() < 0.5,
                    fn=rng.choice(["none", "relu", "silu", "gelu", "gelu_tanh"]),
                    out=rng.choice(["bf16", "bf16", "bf16", "f32"]))
    if kind == "quantize":
        N, K = _log(rng, 16, 14336), _log(rng, 64, 4096)
        return dict(op="quantize", N=N, K=K, x=rng.choice(["bf16", "bf16", "f32"]))
    c = dict(CACHE, Hkv=rng.choice([1, 2, 4, 8, 8, 16]), D=rng.choice([64, 128, 128, 256]),
             page=rng.choice([32, 64, 128, 256]), empty=rng.random() < 0.3)
    per = c["Hkv"] * c["D"]
    if kind == "append":
        c.update(op="append", B=_log(rng, 1, 64), longest=_log(rng, 64, 8192))
        most = min(c["longest"], 8 * 1021 * 1024 // (per * c["B"]))
        c["n"] = rng.choice([1, _log(rng, 1, max(1, most))])
        return dict(c, n=max(1, min(c["n"], most)))
    heads = rng.choice([1, 2, 4, 4, 5, 7, 8, 16])
    c.update(op="attend", Hq=c["Hkv"] * heads, B=_log(rng, 1, 96), n=rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 8, 509)]))
    # no more rows of queries than chunk_4 has, nor operations, and no more bytes than decode_64
    rows = c["B"] * heads * per
    c["n"] = max(1, min(c["n"], 4 * 509 * 32 * 128 // rows))
    c["longest"] = min(_log(rng, max(64, c["n"]), 100003), 64 * 12000 * 1024 // (per * c["B"]),
                       4 * 509 * 32 * 128 * 4000 // (c["n"] * rows))
    c["longest"] = max(c["longest"], c["n"])
    return dict(c, window=rng.choice([0, 0, 0, _log(rng, 16, 4096)]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _randn(gen, *shape):
    return torch.empty(*shape, device="cuda", dtype=torch.bfloat16).normal_(generator=gen)


def _linear_inputs(c, seed):
    gen = _gen(seed)
    w = _randn(gen, c["N"], c["K"]).mul_(0.02)
    return {"w": w, "x": _randn(gen, c["M"], c["K"]),
            "bias": torch.randn(c["N"], device="cuda", generator=gen).mul_(0.1) if c["bias"] else None,
            "residual": _randn(gen, c["M"], c["N"]) if c["residual"] else None}


def _quantize_inputs(c, seed):
    x = _randn(_gen(seed), c["N"], c["K"]).mul_(0.02)
    return x.float() if c["x"] == "f32" else x


def _cache_inputs(c, seed):
    """Keys and values of all tokens, sequence behind sequence, the pages of each, and queries."""
    gen, lens = _gen(seed), lengths(c)
    total, Hkv, D = sum(lens), c["Hkv"], c["D"]
    k, v = _randn(gen, total, Hkv, D), _randn(gen, total, Hkv, D)
    k[:, :, ::16] *= 4  # (channels of keys differ in size)
    per = [(l + c["page"] - 1) // c["page"] for l in lens]
    n_pages = max(1, sum(per))
    order = torch.randperm(n_pages, device="cuda", generator=gen).to(torch.int32)
    widest = max(1, max(per))
    first = torch.tensor([sum(per[:b]) for b in range(c["B"])], device="cuda")
    count = torch.tensor(per, device="cuda")
    at = torch.arange(widest, device="cuda")[None, :]
    table = torch.where(at < count[:, None], order[(first[:, None] + at).clamp_(max=n_pages - 1)], 0)
    st = {"k": k, "v": v, "pages": table.to(torch.int32), "n_pages": n_pages,
          "lens": torch.tensor(lens, device="cuda", dtype=torch.int32)}
    if c["op"] == "attend":
        st["q"] = _randn(gen, c["B"] * c["n"], c["Hq"], D)
    return st


def _spans(c):
    """Each sequence's first token in the inputs, and its tokens."""
    at, out = 0, []
    for l in lengths(c):
        out.append((at, l))
        at += l
    return out


def _newest(c, t):
    """The newest n tokens of each sequence (none of one that is empty: zeros in their place)."""
    n, pad = c["n"], torch.zeros_like(t[:1]).expand(c["n"], -1, -1)
    return torch.cat([t[at + l - n:at + l] if l else pad for at, l in _spans(c)])


def prepare(case, seed):
    c = case
    if c["op"] == "linear4":
        st = dict(_linear_inputs(c, seed), case=c)
        st["codes"], st["scale"] = _encode(st.pop("w"))
        if own:
            import paper_2505_08944_amd as aep
            st["lin"] = aep.Linear4(st["codes"], st["scale"], c["K"], bias=st["bias"], activation=c["fn"],
                                    out_dtype=torch.float32 if c["out"] == "f32" else torch.bfloat16)
        return st
    if c["op"] == "quantize":
        return {"case": c, "x": _quantize_inputs(c, seed)}
    inp = _cache_inputs(c, seed)
    st = {"case": c, "pages": inp["pages"], "lens": inp["lens"], "q": inp.get("q")}
    n = c["n"] if c["op"] == "append" else 0
    if n:
        st["k"], st["v"] = _newest(c, inp["k"]), _newest(c, inp["v"])
    # what the cache holds already: all that a pass does not append
    kept = [max(0, l - n) for l in lengths(c)]
    if own:
        import paper_2505_08944_amd as aep
        st["cache"] = aep.Cache4(inp["n_pages"], c["Hkv"], c["D"], page_size=c["page"])
        if not n:
            rows = torch.tensor([0] + [at + l for at, l in _spans(c)], device="cuda", dtype=torch.int32)
            if sum(kept):
                st["cache"].append(inp["k"], inp["v"], st["pages"], st["lens"], rows)
        return st
    shape = (inp["n_pages"], c["page"], c["Hkv"])
    st["store"] = {}
    for name in ("k", "v"):
        st["store"][name] = torch.zeros(*shape, c["D"] // 2, device="cuda", dtype=torch.uint8)
        st["store"][name + "_scale"] = torch.zeros(*shape, c["D"] // 32, device="cuda", dtype=torch.uint8)
        if not n:
            for b, (at, l) in enumerate(_spans(c)):
                if l:
                    _put(st, name, b, 0, inp[name][at:at + l])
    return st


# -------------------------------------------------------------- plain forms
_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _power(e):
    """2^e, for e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x):
    """4-bit codes, two to a byte, and scales (2^(byte - 127)) of blocks of 32 along the last dimension."""
    K = x.shape[-1]
    pad = -K % 32
    v = x.float()
    if pad:
        v = torch.cat([v, torch.zeros(*v.shape[:-1], pad, device=v.device)], -1)
    v = v.reshape(*v.shape[:-1], -1, 32)
    big = v.abs().amax(-1, keepdim=True)
    # the exponent of big / 7, rounded up: big = f 2^e with f in [0.5, 1), and 7 2^(e - 3) = 0.875 2^e
    f, e = torch.frexp(big)
    e = torch.where(f <= 0.875, e - 3, e - 2)
    e = torch.where(big == 0, torch.zeros_like(e), e).clamp_(-126, 127)
    a = v.abs() * _power(-e)
    # codes by the middles between them; a value in the middle goes to the even code
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a > mid) if i % 2 == 0 else (a >= mid)
    code += 8 * torch.signbit(v).to(torch.uint8)
    code = code.reshape(*code.shape[:-2], -1)
    code = code[..., :K + (K & 1)]
    return (code[..., 0::2] | code[..., 1::2] << 4).contiguous(), (e[..., 0] + 127).to(torch.uint8)


def _decode(codes, scale, K):
    table = torch.tensor(_VALUES + [-v for v in _VALUES], device=codes.device)
    v = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], -1)[..., :K]
    power = _power(scale.to(torch.int32) - 127)[..., None].expand(*scale.shape, 32)
    return table[v.to(torch.int32)] * power.reshape(*scale.shape[:-1], -1)[..., :K]


def _places(st, b, first, n):
    """(page, place in it) of tokens first .. first + n of sequence b."""
    page = st["case"]["page"]
    pos = torch.arange(first, first + n, device="cuda")
    return st["pages"][b, pos // page].long(), pos % page


def _put(st, name, b, first, x):
    page, at = _places(st, b, first, x.shape[0])
    codes, scale = _encode(x)
    st["store"][name][page, at] = codes
    st["store"][name + "_scale"][page, at] = scale


def _get(st, name, b, first, n):
    page, at = _places(st, b, first, n)
    return _decode(st["store"][name][page, at], st["store"][name + "_scale"][page, at], st["case"]["D"])


def _plain_linear(st):
    c = st["case"]
    w = _decode(st["codes"], st["scale"], c["K"])
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
    return y if c["out"] == "f32" else y.to(torch.bfloat16)


def _plain_append(st):
    c, n = st["case"], st["case"]["n"]
    live = [b for b, l in enumerate(lengths(c)) if l]
    pos = st["lens"][:, None].long() + torch.arange(-n, 0, device="cuda")
    pages = st["pages"]
    if len(live) < c["B"]:
        live = torch.tensor(live, device="cuda")
        pos, pages = pos[live], pages[live]
    page, at = torch.gather(pages, 1, pos // c["page"]).long().flatten(), (pos % c["page"]).flatten()
    out = []
    for name in ("k", "v"):
        new, store, scales = st[name], st["store"][name], st["store"][name + "_scale"]
        rows = new.view(c["B"], n, c["Hkv"], c["D"])
        if len(live) < c["B"]:
            rows = rows[live]
        store[page, at], scales[page, at] = _encode(rows.reshape(-1, c["Hkv"], c["D"]))
        kept = _decode(store[page, at], scales[page, at], c["D"]).to(torch.bfloat16)
        if len(live) < c["B"]:
            t = torch.zeros_like(new)
            t.view(c["B"], n, c["Hkv"], c["D"])[live] = kept.view(-1, n, c["Hkv"], c["D"])
            kept = t
        out.append(kept)
    return tuple(out)


def _plain_attend(st):
    c, n, D = st["case"], st["case"]["n"], st["case"]["D"]
    heads = c["Hq"] // c["Hkv"]
    out = torch.zeros_like(st["q"])
    for b, l in enumerate(lengths(c)):
        if not l:
            continue
        # the earliest row's window says which tokens any row can see
        first = max(0, l - n - c["window"] + 1) if c["window"] else 0
        k = _get(st, "k", b, first, l - first).transpose(0, 1)
        v = _get(st, "v", b, first, l - first).transpose(0, 1).contiguous()
        q = st["q"][b * n:b * n + n].float().reshape(n, c["Hkv"], heads, D).permute(1, 0, 2, 3).reshape(c["Hkv"], n * heads, D)
        pos = torch.arange(first, l, device="cuda")[None, :]
        row = (l - n + torch.arange(n, device="cuda"))[:, None]
        away = pos > row
        if c["window"]:
            away = away | (pos <= row - c["window"])
        away = away[:, None, :].expand(n, heads, -1).reshape(1, n * heads, -1)
        s = torch.matmul(q, k.transpose(1, 2).contiguous()) * D ** -0.5
        s = torch.where(away, float("-inf"), s)
        s = torch.exp(s - s.amax(2, keepdim=True))
        o = torch.matmul(s, v) / s.sum(2, keepdim=True)
        o = o.reshape(c["Hkv"], n, heads, D).permute(1, 0, 2, 3).reshape(n, c["Hq"], D)
        out[b * n:b * n + n] = o.to(torch.bfloat16)
    return out


def run(state):
    st = state
    c = st["case"]
    if not own:
        if c["op"] == "quantize":
            return _decode(*_encode(st["x"]), c["K"]).to(torch.bfloat16)  # (exact)
        return {"linear4": _plain_linear, "append": _plain_append, "attend": _plain_attend}[c["op"]](st)
    if c["op"] == "linear4":
        return st["lin"](st["x"], residual=st["residual"])
    if c["op"] == "attend":
        return st["cache"].attend(st["q"], st["pages"], st["lens"], window=c["window"])
    if c["op"] == "append":
        st["cache"].append(st["k"], st["v"], st["pages"], st["lens"])
        return st["cache"].read(st["pages"], st["lens"], c["B"] * c["n"])
    import paper_2505_08944_amd as aep
    codes, scale = aep.quantize_mx4(st["x"])
    return aep.dequantize_mx4(codes, scale, c["K"])


# ---------------------------------------------------------------- reference
def work(case):
    c = case
    if c["op"] == "linear4":
        M, N, K = c["M"], c["N"], c["K"]
        nbytes = 2 * M * K + N * ((K + 1) // 2 + (K + 31) // 32) + (4 if c["out"] == "f32" else 2) * M * N
        return {"bytes": nbytes + (2 * M * N if c["residual"] else 0) + (4 * N if c["bias"] else 0), "flops": 2 * M * N * K}
    if c["op"] == "quantize":
        # the matrix, and its values, which are the output
        return {"bytes": c["N"] * c["K"] * ((4 if c["x"] == "f32" else 2) + 2), "flops": 4 * c["N"] * c["K"]}
    lens, n, per = lengths(c), c["n"], c["Hkv"] * c["D"]
    held = per // 2 + per // 32  # bytes of a token's keys, or values
    if c["op"] == "append":
        rows = sum(n for l in lens if l)
        return {"bytes": 2 * rows * (2 * per + held) + 4 * n * c["B"] * per, "flops": 8 * rows * per}
    seen = pairs = 0
    for l in lens:
        if l:
            seen += min(l, n + c["window"] - 1) if c["window"] else l
            pairs += sum(min(l - n + i + 1, c["window"] or l) for i in range(n))
    nbytes = 2 * seen * held + 4 * c["B"] * n * c["Hq"] * c["D"] + 4 * sum((l + c["page"] - 1) // c["page"] for l in lens)
    return {"bytes": nbytes, "flops": 4 * pairs * c["Hq"] * c["D"]}


def _nearest(x):
    """The values that 4 bits keep of x, in 64 bits: of the 15 multiples of each block's power the nearest, of two as near
    the one with the even code."""
    K = x.shape[-1]
    out = []
    for at in range(0, K, 32):
        v = x[..., at:at + 32].double()
        big = v.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(big > 0, big, 7.0) / 7.0)).long()
        power = (e + 1023 << 52).view(torch.float64)
        # (a logarithm that is off by a little at a border)
        power = torch.where(7.0 * power < big, power * 2, torch.where(7.0 * power / 2 >= big, power / 2, power))
        power = torch.where(big > 0, power.clamp(2.0 ** -126, 2.0 ** 127), 1.0)
        best, off = torch.zeros_like(v), v.abs()
        for i in (2, 4, 6, 1, 3, 5, 7):  # even codes first, and odd ones only where they are nearer
            value = _VALUES[i] * power
            nearer = (v.abs() - value).abs() < off
            off = torch.where(nearer, (v.abs() - value).abs(), off)
            best = torch.where(nearer, value.expand_as(best), best)
        out.append(torch.where(v < 0, -best, best))
    return torch.cat(out, -1)


def _exact_attend(c, seed):
    inp, n, D = _cache_inputs(c, seed), c["n"], c["D"]
    heads = c["Hq"] // c["Hkv"]
    out = torch.zeros(c["B"], n, c["Hq"], D, device="cuda", dtype=torch.float64)
    q = inp["q"].double().view(c["B"], n, c["Hq"], D)
    for b, (at, l) in enumerate(_spans(c)):
        if not l:
            continue
        for h in range(c["Hkv"]):
            k, v = _nearest(inp["k"][at:at + l, h]), _nearest(inp["v"][at:at + l, h])
            for i in range(0, n, 64):
                m = min(64, n - i)
                s = torch.einsum("nhd,ld->hnl", q[b, i:i + m, h * heads:(h + 1) * heads], k) / math.sqrt(D)
                row = torch.arange(l - n + i, l - n + i + m, device="cuda")[:, None]
                col = torch.arange(l, device="cuda")[None, :]
                see = (col <= row) & ((row - col < c["window"]) if c["window"] else (col >= 0))
                p = torch.softmax(s.masked_fill(~see, float("-inf")), -1)
                out[b, i:i + m, h * heads:(h + 1) * heads] = torch.einsum("hnl,ld->nhd", p, v)
    return out.view(c["B"] * n, c["Hq"], D)


def exact(case, seed):
    c = case
    if c["op"] == "quantize":
        return _nearest(_quantize_inputs(c, seed))
    if c["op"] == "append":
        inp = _cache_inputs(c, seed)
        return _nearest(_newest(c, inp["k"])), _nearest(_newest(c, inp["v"]))
    if c["op"] == "attend":
        return _exact_attend(c, seed)
    st = _linear_inputs(c, seed)
    F = torch.nn.functional
    y = F.linear(st["x"].double(), _nearest(st["w"]), None if st["bias"] is None else st["bias"].double())
    y = {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu,
         "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[c["fn"]](y)
    return y if st["residual"] is None else y + st["residual"].double()
