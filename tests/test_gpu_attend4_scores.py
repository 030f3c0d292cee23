"""Attention over the cache in 4 bits with large scores: from 2^20 to near the end of f32, of both signs.

Scores are f32 there as everywhere, so tokens of nearly equal ones are weighed by chance; the inputs have
tokens whose scores are the largest by a wide margin, one or several with equal keys, and the premise is asserted: with
S = scale sum |q| |k| of a token, its f32 score is off by at most e = (D + 8) 2^-23 S, and every other score is below the
largest by more than twice its own e and theirs, and 200 (e^-200 is nothing).  Then the result is the mean of the values of the largest: equal keys give equal bits of their
scores, so that weights under one reference are equal; under two (blocks, waves and parts have one each) each weight is rounded to
bf16 by itself, 2^-8, with 2^-20 for exponent and exponential.  Tolerance per value, with the spread and size of the mean as in
test_gpu_attend4.py: 1.02 (2^-8 + 2^-20) spread + (L / 32 + 256) 2^-23 size + L 2^-120 max |v|, and rounding to bf16.
lse: the score, (D + 8) 2^-23 S; its product with log2 e, the reference's distance from it, the sum's logarithm added and
the product with log 2, each rounded to f32, and that factor itself: 5 2^-24 |lse|, below 2^-21; and 2^-8 + 2^-20 for the sum.
"""

import numpy as np
import pytest
import torch

import mx4_ref
from gpu_helpers import log
from test_gpu_attend4 import Case, mx4_ref_values

pytestmark = pytest.mark.gpu

# lens, rows, heads of the cache, heads of queries to one, D, wide table
SHAPES = [([90, 7], 1, 2, 4, 128, False), ([90, 40], 1, 1, 8, 256, False), ([77, 300], 5, 2, 4, 64, False),
          ([2100], 1, 1, 4, 128, False), ([1700], 7, 1, 4, 256, False), ([1500, 300], 40, 2, 4, 128, True),
          ([700], 130, 1, 1, 64, True), ([500, 81], 40, 2, 2, 256, True), ([1300, 300], [200, 1], 1, 2, 128, True)]


def winners(l, n):
    """Tokens that every row sees, one per block, wave, unit and half of the sequence."""
    last = l - n
    return sorted({t for t in (0, 31, 33, 40, 127, 128, 260, last // 2, last) if 0 <= t <= last})


def check(c, out, lse, scale, what, heads=None):
    f = lambda t: t.double().cpu().numpy()
    got, glse, q = f(out), f(lse), f(c.q)
    wk, wv = mx4_ref_values(c.k), mx4_ref_values(c.v)
    r = 0
    for b, (l, n) in enumerate(zip(c.lens, c.n)):
        k, v = wk[c.at[b]:c.at[b] + l], wv[c.at[b]:c.at[b] + l]
        for i in range(n):
            if i in (0, 1, 31, 32, 64, 127, 128, n - 1):
                for h in heads or range(c.Hkv * c.group):
                    kk, vv, pos = k[:l - n + i + 1, h // c.group], v[:l - n + i + 1, h // c.group], l - n + i
                    s = scale * (kk @ q[r, h])
                    top = s.max()
                    errs = (c.D + 8) * 2.0 ** -23 * scale * (np.abs(kk) @ np.abs(q[r, h]))
                    err = errs[s == top].max()
                    assert ((s == top) | (s + 2 * errs < top - 2 * err - 200)).all()  # (the premise)
                    ref, ref_lse, spread, size, _ = mx4_ref.attend(q[r, h], k[:, h // c.group], v[:, h // c.group], pos, scale, 0)
                    tol = 1.02 * (2.0 ** -8 + 2.0 ** -20) * spread + (l / 32 + 256) * 2.0 ** -23 * size
                    tol = tol + l * 2.0 ** -120 * np.abs(vv).max()
                    tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
                    bad = ~(np.abs(got[r, h] - ref) <= tol)
                    assert not bad.any(), (what, b, i, h, got[r, h][bad][:4], ref[bad][:4], tol[bad][:4])
                    near = err + 2.0 ** -21 * abs(ref_lse) + 2.0 ** -8 + 2.0 ** -20
                    assert abs(glse[r, h] - ref_lse) <= near, (what, b, i, h, glse[r, h], ref_lse)
            r += 1


def fill(c, seed, negative, one):
    """Keys of 1 .. 2 and, of the winners, 6 (the least: of -6 .. -4 and -1); queries of 0.5 .. 1.5."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.rand(c.k.shape, generator=g, device="cuda")
    c.k.copy_(-4 - 2 * x if negative else 1 + x)
    for b, (l, n) in enumerate(zip(c.lens, c.n)):
        if l:
            at = winners(l, n)
            for t in (at[seed % len(at):][:1] if one else at):
                c.k[c.at[b] + t] = -1.0 if negative else 6.0
    c.q.copy_(0.5 + torch.rand(c.q.shape, generator=g, device="cuda"))


@pytest.mark.parametrize("i", range(len(SHAPES)))
@pytest.mark.parametrize("power", [20, 25, 28, 32, 33, 36, 60, 118])
def test_large_scale(i, power):
    *shape, many = SHAPES[i]
    c = Case(*shape, seed=40 + i)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for negative in (False, True):
        for one in (False, True):
            log(f"attend4 scores of 2^{power} shape {i} negative {negative} one {one}")
            fill(c, power + i, negative, one)
            c.write()
            # (the largest score is about 2^power, in powers of two)
            scale = float(np.float32(2.0 ** power / (6.0 * c.D * 1.4427)))
            out = c.attend(many, scale=scale, lse=lse)
            check(c, out, lse, scale, (i, power, negative, one))


@pytest.mark.parametrize("i", [0, 2, 3, 5, 7])
@pytest.mark.parametrize("qp,kp", [(20, 20), (0, 60), (60, 0), (55, 60), (-60, 100)])
def test_large_queries_and_keys(i, qp, kp):
    """The same with the default scale."""
    *shape, many = SHAPES[i]
    c = Case(*shape, seed=60 + i)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for negative in (False, True):
        log(f"attend4 queries of 2^{qp} keys of 2^{kp} shape {i} negative {negative}")
        fill(c, qp + i, negative, False)
        c.k.mul_(2.0 ** kp)
        c.q.mul_(2.0 ** qp)
        c.write()
        out = c.attend(many, lse=lse)
        check(c, out, lse, c.D ** -0.5, (i, qp, kp, negative))


@pytest.mark.parametrize("i", [0, 3, 4, 5, 6, 7])
def test_scores_that_double(i):
    """Powers of the keys that grow from some tokens to the next: references go from small to large ones, and a wave, a
    workgroup or a block has seen others than its neighbour."""
    *shape, many = SHAPES[i]
    c = Case(*shape, seed=80 + i)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for sign in (1.0, -1.0):
        log(f"attend4 scores that double, shape {i} sign {sign}")
        for b, (l, n) in enumerate(zip(c.lens, c.n)):
            t = torch.arange(l, device="cuda")
            # (rows of the first tokens too: the power falls where scores are negative)
            p = torch.div(t * 80, max(l, 1), rounding_mode="floor") * sign
            c.k[c.at[b]:c.at[b] + l] = (sign * torch.exp2(p.float() + (8.0 if sign > 0 else 100.0)))[:, None, None].to(c.k.dtype)
        c.q.copy_(0.5 + torch.rand(c.q.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)))
        c.write()
        out = c.attend(many, lse=lse)
        check(c, out, lse, c.D ** -0.5, (i, sign))


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_large_scores_beside_small_ones(i):
    """Columns of one wave with and without them: heads' queries of 1 and of 2^40 in turn, or rows'.  The small ones are held
    to their own tolerance (not to the bits of a call of their own: a wave's references rise together)."""
    *shape, many = SHAPES[i]
    c = Case(*shape, seed=100 + i)
    lse, scale = torch.empty(c.q.shape[:2], device="cuda"), 1.0 / (2 * c.D)
    log(f"attend4 scores large and small, shape {i}")
    fill(c, i, False, False)
    c.write()
    rows, H = {0, 1, 30, 31, 32, 64, -1}, c.Hkv * c.group
    c.check(c.attend(many, scale=scale, lse=lse), lse, scale=scale, what=i, rows=rows)
    large = list(range(1, H, 2))
    if H > 1:
        c.q[:, large] *= 2.0 ** 40
    else:
        c.q[1::2] *= 2.0 ** 40
    out = c.attend(many, scale=scale, lse=lse)
    c.check(out, lse, scale=scale, what=i, rows=rows)
    if H > 1:
        check(c, out, lse, scale, i, large)
    else:
        c.q[::2] *= 2.0 ** 40
        all_lse = torch.empty_like(lse)
        every = c.attend(many, scale=scale, lse=all_lse)
        check(c, every, all_lse, scale, i)
        every[1::2], all_lse[1::2] = out[1::2], lse[1::2]
        check(c, every, all_lse, scale, i)


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_the_end_of_f32(i):
    """Largest scores of about 2^127 in powers of two, the last that are f32; behind it NaN, for the columns that have such scores."""
    *shape, many = SHAPES[i]
    c = Case(*shape, seed=120 + i)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    scale = float(np.float32(2.0 ** 127 / (6.0 * c.D * 1.4427)))
    for negative in (False, True):
        log(f"attend4 scores of 2^127 shape {i} negative {negative}")
        fill(c, i, negative, False)
        c.write()
        out = c.attend(many, scale=scale, lse=lse)
        check(c, out, lse, scale, (i, negative))
    fill(c, i, False, False)
    c.write()
    c.q[-1, -1] *= 16.0
    last = c.attend(many, scale=scale)
    assert bool(torch.isnan(last[-1, -1]).all()) and int(torch.isnan(last).sum()) == c.D
