"""Attention over the cache in 4 bits against its formula in 64 bits, on the values that the cache keeps.

Tolerance, per value.  A score is an f32 sum of D exact products (size S = scale sum |q| |k|), off by at
most (D + 8) 2^-23 S; its exponent in powers of two and the exponential add 2^-23 of the exponent's size (at most the
scores' spread and the 8 by which the reference may lag, both below 2 S + 12) and 2^-22.  Each p_t is
rounded to bf16 (2^-8).  All of that scales p_t by 1 + e_t, in both sums, so that out moves by sum p e (v - out) /
sum p: at most max |e| sum p |v - out| / sum p.  A p_t below 2^-126 is lost, as f32 and bf16 have no
smaller normal values; it is relative to a reference that is at most 6 powers of two above the largest score, so that the
largest p_t is at least 2^-6 and what is lost at most L 2^-120 max |v|.  The f32 sums of up to L / 32 + 64 terms, each exact to
2^-23, and the joining of parts add (L / 32 + 256) 2^-23 sum p |v| / sum p, and rounding out to bf16 2^-8 of it.
lse: max |e| without the last rounding's 2^-8 of single p (their mean is no larger), and 2^-20 for the logarithm.
"""

import threading

import numpy as np
import pytest
import torch

import mx4_ref
import paper_2505_08944_amd as aep
from gpu_helpers import log
from test_gpu_cache4 import i32, rows_of, table

pytestmark = pytest.mark.gpu


class Case:
    def __init__(self, lens, n, Hkv, group, D, page=64, seed=0, spare=2):
        """n: rows of each sequence, a number or a list."""
        self.lens, self.D, self.Hkv, self.group = lens, D, Hkv, group
        self.uniform = isinstance(n, int)
        self.n = [n] * len(lens) if self.uniform else n
        n_pages = sum(-(-l // page) for l in lens) + spare
        self.cache = aep.Cache4(n_pages, Hkv, D, page_size=page)
        # what no token was written to is NaN
        self.cache.data.fill_(255)
        self.pages = table(lens, page, n_pages, seed)
        total, at = sum(lens), np.concatenate([[0], np.cumsum(lens)]).tolist()
        self.at = at
        k, v = rows_of(total, Hkv, D, 2 * seed, False), rows_of(total, Hkv, D, 2 * seed + 1, False)
        k[:, :, ::16] *= 4
        self.k, self.v = k, v
        self.write()
        T = sum(self.n)
        self.q = rows_of(T, Hkv * group, D, 3 * seed + 7, False)
        self.rows = None if self.uniform else i32(*np.concatenate([[0], np.cumsum(self.n)]).tolist())
        self.dev_lens = i32(*lens)

    def write(self):
        if sum(self.lens):
            self.cache.append(self.k, self.v, self.pages, i32(*self.lens), i32(*self.at))

    def attend(self, many=False, **kw):
        """many: with a table padded so far that the kernel for many columns takes the sequences that have them."""
        pages = self.pages
        if many:
            need = 8 * 512 * 128 // (self.Hkv * len(self.lens)) // self.cache.page_size + 1
            pages = torch.nn.functional.pad(pages, (0, max(0, need - pages.shape[1])), value=-7)
        return self.cache.attend(self.q, pages, self.dev_lens, self.rows, **kw)

    def check(self, out, lse=None, window=0, scale=None, what=None, rows=None):
        scale = self.D ** -0.5 if scale is None else scale
        f = lambda t: t.double().cpu().numpy()
        got, q = f(out), f(self.q)
        glse = None if lse is None else f(lse)
        wk, wv = (mx4_ref_values(t) for t in (self.k, self.v))
        r = 0
        for b, (l, n) in enumerate(zip(self.lens, self.n)):
            k, v = wk[self.at[b]:self.at[b] + l], wv[self.at[b]:self.at[b] + l]
            for i in range(n):
                if rows is None or i in rows or i - n in rows:
                    for h in range(self.Hkv * self.group):
                        kv = h // self.group
                        ref, ref_lse, spread, size, s = mx4_ref.attend(q[r, h], k[:, kv], v[:, kv], l - n + i, scale, window)
                        e = (self.D + 8) * 2.0 ** -23 * s + 2.0 ** -23 * (2 * s + 12) + 2.0 ** -22
                        tol = 1.02 * (e + 2.0 ** -8) * spread + (l / 32 + 256) * 2.0 ** -23 * size
                        tol = tol + l * 2.0 ** -120 * np.nan_to_num(np.abs(v[:, kv])).max(initial=0.0)
                        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
                        bad = ~((np.abs(got[r, h] - ref) <= tol) | (np.isnan(got[r, h]) & np.isnan(ref)))
                        assert not bad.any(), (what, b, i, h, got[r, h][bad][:4], ref[bad][:4], tol[bad][:4])
                        if glse is not None:
                            if np.isinf(ref_lse):
                                assert glse[r, h] == ref_lse
                            else:
                                assert abs(glse[r, h] - ref_lse) <= e + 2.0 ** -8 + 2.0 ** -20 * (1 + abs(ref_lse)), (what, b, i, h)
                r += 1


def mx4_ref_values(x):
    """The kept values (exact: test_gpu_mx4.py)."""
    T, H, D = x.shape
    if T == 0:
        return np.zeros((0, H, D))
    return aep.dequantize_mx4(*aep.quantize_mx4(x.reshape(T * H, D)), D).double().cpu().numpy().reshape(T, H, D)


CASES = [
    ([1], 1, 1, 1, 64, 32), ([1], 1, 1, 1, 128, 64), ([2, 1, 3], 1, 2, 4, 256, 32), ([31, 32, 33], 1, 2, 1, 128, 32),
    ([127, 128, 129, 1], 1, 1, 8, 128, 64), ([0, 5, 0, 700], 1, 3, 5, 64, 64), ([1000], 1, 8, 4, 128, 64),
    ([513, 64], 1, 2, 16, 128, 128), ([300, 77], 1, 1, 17, 128, 64), ([90], 1, 2, 40, 64, 32), ([2049], 1, 1, 2, 256, 256),
    ([7, 5], 5, 2, 4, 128, 64), ([40, 9, 200], 9, 1, 4, 256, 32), ([130], 130, 1, 1, 128, 64), ([65, 200], 64, 2, 3, 64, 64),
    ([50, 257], 33, 2, 2, 256, 64), ([100, 0, 33, 500], [1, 3, 0, 20], 2, 4, 128, 64), ([70, 300], [70, 1], 1, 4, 64, 32),
    ([3, 2], 6, 2, 4, 128, 64), ([0, 0], 1, 1, 1, 128, 64), ([33] * 70, 1, 1, 4, 128, 32), ([5] * 130, [b % 3 for b in range(130)], 1, 2, 64, 32),
    ([b % 5 for b in range(600)], [(b * 3) % 4 for b in range(600)], 1, 1, 64, 32), ([40, 0, 1] * 86, 1, 1, 2, 128, 32),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_cases(i):
    """Lengths at the edges of blocks, units and pages; rows without tokens; groups of any size; with and without a window."""
    c = Case(*CASES[i], seed=i)
    for window in (0, 1, 50, 10 ** 6):
        log(f"attend4 case {i} {CASES[i]} window {window}")
        for many in (False, True):
            flag, lse = i32(0), torch.full(c.q.shape[:2], 5.0, device="cuda")
            out = c.attend(many, window=window, flag=flag, lse=lse)
            c.check(out, lse, window, what=(i, window, many))
            assert int(flag) == 0


@pytest.mark.parametrize("lens,n,Hkv,group,D,window", [
    ([20011], 1, 2, 4, 128, 0), ([9001, 3, 30000, 600], 1, 1, 8, 64, 0), ([12345], 3, 1, 4, 256, 5000),
    ([5000, 1, 2600], 7, 2, 4, 128, 0), ([4096, 700], 200, 1, 4, 128, 0), ([8200], 65, 2, 8, 64, 777),
    ([6000, 100], [300, 1], 1, 2, 128, 0)])
def test_long_and_shared(lens, n, Hkv, group, D, window):
    """Tiles of columns that many workgroups share."""
    log(f"attend4 {lens} {n} {Hkv}x{group} d {D} window {window}")
    c = Case(lens, n, Hkv, group, D, seed=3)
    lse = torch.empty(c.q.shape[:2], device="cuda")
    for many in (False, True):
        out = c.attend(many, window=window, lse=lse)
        c.check(out, lse, window, rows={0, 1, 2, 3, 15, 16, 31, 63, 64, 100, 199, -1, -2}, what=many)


def test_scores_that_grow_and_fall():
    """The reference follows: scores that grow from block to block, one token that outweighs all others at
    each place, scores far below 0."""
    for grow, n in ((0.01, 4), (-0.01, 4), (0.3, 4), (-0.3, 4), (0.02, 33), (-0.3, 33), (0.3, 33)):
        c = Case([1500], n, 1, 4, 128, seed=5)
        c.k.copy_(((torch.arange(1500, device="cuda")[:, None, None] * grow).expand(1500, 1, 128)) / 128)
        c.q.copy_(torch.rand_like(c.q) * 8)
        c.write()
        c.check(c.attend(n > 16, scale=1.0), scale=1.0, what=(grow, n), rows={0, 1, 16, -1})
    c = Case([700], 1, 1, 1, 64, seed=6)
    for at in (0, 1, 31, 32, 127, 128, 500, 699):
        c.k.fill_(-1.0)
        c.k[at] = 6.0
        c.q.fill_(2.0)
        c.write()
        out = c.attend()
        c.check(out, what=at)
        assert torch.equal(out[0, 0].cpu(), torch.from_numpy(mx4_ref_values(c.v)[at, 0]).to(torch.bfloat16))


def test_equal_scores_are_a_mean():
    c = Case([333, 4096], 1, 2, 4, 128, seed=8)
    c.q.zero_()
    c.check(c.attend())


def test_values_that_are_not_finite():
    """What a row sees is NaN where the formula is; what it does not see does not count: later tokens, tokens before the window,
    what lies behind the last token of a page."""
    for n, window, D in ((9, 0, 128), (9, 40, 64), (40, 0, 256), (40, 33, 128)):
        c = Case([100, 50], n, 2, 4, D, seed=9)
        c.k[100 - n // 2, 0, 3] = float("inf")        # a token in the middle of the rows
        c.v[100 - n // 3, 1, 40] = float("nan")
        c.v[100 + 3, 0, 1] = float("inf")             # an early one of the second sequence
        c.write()
        lse = torch.empty(c.q.shape[:2], device="cuda")
        for many in (False, True):
            out = c.attend(many, window=window, lse=lse)
            c.check(out, None, window, what=(n, window, D, many))
            assert not bool(torch.isnan(out[:n - n // 2 - 1]).any())
            assert bool(torch.isnan(out[n - 1]).any())
    c = Case([200], 2, 1, 4, 128, seed=10)
    c.q[0, 1, 0] = float("nan")
    out = c.attend()
    assert bool(torch.isnan(out[0, 1]).all()) and int(torch.isnan(out).sum()) == 128


@pytest.mark.parametrize("byte", [0x7f, 0xfc, 0xfd, 0xfe])
def test_unwritten_places_hold_any_byte(byte):
    """Behind the last token, scales of 2^125 and more and codes of -6: beyond bf16 with the two largest."""
    for lens, n, Hkv, group, D in (([1, 40, 33], 1, 2, 4, 128), ([45, 7], 5, 1, 8, 64), ([70, 130], 40, 1, 2, 256),
                                   ([75], 70, 2, 2, 64), ([35, 161], 30, 1, 8, 128)):
        c = Case(lens, n, Hkv, group, D, seed=11)
        c.cache.data.fill_(byte)
        c.write()
        for window in (0, 20):
            for many in (False, True):
                lse = torch.full(c.q.shape[:2], 5.0, device="cuda")
                c.check(c.attend(many, window=window, lse=lse), lse, window, what=(byte, lens, window, many))


def test_scale():
    c = Case([300, 20], 2, 2, 4, 128, seed=11)
    for scale in (1e-30, 0.01, 1.0, 30.0):
        c.check(c.attend(scale=scale), scale=scale, what=scale)


def test_strides_and_places():
    """Queries as a slice of a product's rows, heads in front of rows, at an odd address; out strided: what lies between stays."""
    c = Case([300, 20, 64], 3, 2, 4, 128, seed=12)
    want = c.attend()
    T, H, D = c.q.shape
    wide = torch.full((T, H * D + 2 * 128 + 1), 3.0, dtype=torch.bfloat16, device="cuda")
    q = torch.as_strided(wide, (T, H, D), (wide.stride(0), D, 1), 1)
    q.copy_(c.q)
    buf = torch.full((H, T + 1, D + 4), 77.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :T, 2:D + 2].transpose(0, 1)
    got = c.cache.attend(q, c.pages, c.dev_lens, out=out)
    assert got is out and torch.equal(out, want)
    assert bool((buf[:, T] == 77).all()) and bool((buf[:, :, :2] == 77).all()) and bool((buf[:, :, D + 2:] == 77).all())
    assert torch.equal(c.cache.attend(c.q.transpose(0, 1).contiguous().transpose(0, 1), c.pages, c.dev_lens), want)
    # the pages' rows apart
    t = torch.full((3, c.pages.shape[1] + 5), -9, dtype=torch.int32, device="cuda")
    t[:, 2:2 + c.pages.shape[1]] = c.pages
    assert torch.equal(c.cache.attend(c.q, t[:, 2:2 + c.pages.shape[1]], c.dev_lens), want)


def test_rows_of_no_sequence_stay():
    c = Case([300, 20], [2, 3], 2, 4, 128, seed=13)
    want = c.attend()
    q = torch.cat([c.q, c.q])
    out, lse = torch.full_like(q, 9.0), torch.full(q.shape[:2], 9.0, device="cuda")
    c.cache.attend(q, c.pages, c.dev_lens, c.rows, out=out, lse=lse)
    assert torch.equal(out[:5], want) and bool((out[5:] == 9).all()) and bool((lse[5:] == 9).all())
    assert not bool((lse[:5] == 9).any())


def test_what_only_the_device_sees_is_held_to_bounds_and_reported():
    c = Case([300, 20], 2, 2, 4, 64, seed=14)
    want = c.attend()
    P = c.pages.shape[1]
    for pages, lens, rows in (((0, 0, 99), None, None), ((0, 1, -1), None, None), (None, (64 * P + 1, 20), None),
                              (None, (-1, 20), None), (None, None, (0, 5, 4)), (None, None, (0, 2, 400)), (None, None, (-2, 2, 4)),
                              (None, (2 ** 31 - 1, -2 ** 31), (2 ** 31 - 1, -2 ** 31, 0))):
        t, flag = c.pages.clone(), i32(0)
        if pages:
            t[pages[0], pages[1]] = pages[2]
        c.cache.attend(c.q, t, c.dev_lens if lens is None else i32(*lens), None if rows is None else i32(*rows), flag=flag)
        assert int(flag) == 1, (pages, lens, rows)
    assert torch.equal(c.attend(), want)


def test_rows_that_descend_make_more_work_than_is_counted():
    """Every other sequence has all rows, 65536 times: 4.4 10^9 units, more than 32 bits.  Nobody has a share of them."""
    B, T, H, D, P = 1 << 17, 1 << 15, 8, 64, 66
    assert (B // 2) * H * (T // 128) * -(-P * 64 // 128) > 1 << 32
    cache = aep.Cache4(P, H, D)
    pages = torch.arange(P, dtype=torch.int32, device="cuda").expand(B, P).contiguous()
    lens = torch.full((B,), P * 64, dtype=torch.int32, device="cuda")
    rows = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    rows[1::2] = T
    q = torch.zeros(T, H, D, dtype=torch.bfloat16, device="cuda")
    out, flag = torch.full((T + 2, H, D), 77.0, dtype=torch.bfloat16, device="cuda"), i32(0)
    log("attend4 rows that descend")
    cache.attend(q, pages, lens, rows, out=out[1:-1], flag=flag)
    assert int(flag) == 1 and bool((out == 77).all())
    log("attend4 rows that descend, fewer")
    rows = i32(0, 5, 0, 5, 0, 5, 0, 5)
    flag = i32(0)
    cache.attend(q[:5], pages[:7, :2], lens[:7], rows, out=out[1:6], flag=flag)
    assert int(flag) == 1 and bool((out[0] == 77).all()) and bool((out[6:] == 77).all())
    # and rows that ascend, with the same lengths
    rows = torch.clamp(torch.arange(B + 1, device="cuda"), max=T).to(torch.int32)
    flag = i32(0)
    cache.attend(q[:64], pages[:100, :2], i32(*[128] * 100), torch.clamp(rows[:101], max=64), out=out[1:65], flag=flag)
    assert int(flag) == 0 and bool((out[1:65] == 0).all()) and bool((out[0] == 77).all()) and bool((out[65:] == 77).all())


def test_prompts_beside_single_tokens():
    """Sequences of many and of few columns in one call, with the most rows known and not; the same bits again and again."""
    c = Case([700, 90, 0, 2000, 300, 1], [200, 1, 1, 3, 40, 1], 2, 4, 128, seed=18)
    for many in (False, True):
        out = c.attend(many)
        c.check(out, what=many, rows={0, 1, 2, 31, 32, 33, 127, -1})
        for max_rows in (200, 10 ** 6):
            assert torch.equal(c.attend(many, max_rows=max_rows), out)
        c.check(c.attend(many, max_rows=3), what="a bound that does not hold", rows={0, 1, -1})
        for i in range(5):
            assert torch.equal(c.attend(many), out)


def test_nothing_to_do():
    c = Case([30], 1, 2, 4, 64, seed=15)
    assert c.cache.attend(c.q[:0], c.pages, c.dev_lens).shape == (0, 8, 64)
    assert c.cache.attend(c.q[:0], c.pages[:0], c.dev_lens[:0]).shape == (0, 8, 64)
    out = torch.full_like(c.q, 4.0)
    c.cache.attend(c.q, c.pages[:0], c.dev_lens[:0], i32(0), out=out)
    assert bool((out == 4).all())
    # a table without pages: no sequence has a token
    assert bool((c.cache.attend(c.q, c.pages[:, :0], i32(0)) == 0).all())


def test_lengths_change_under_a_captured_call():
    """A decode step captured once: queries, lengths and the cache change between its replays."""
    c = Case([500, 70, 129, 1], 1, 2, 4, 128, seed=16)
    new_k, new_v = rows_of(4, 2, 128, 50, False), rows_of(4, 2, 128, 51, False)
    lens, out = c.dev_lens.clone(), torch.empty_like(c.q)
    lens.copy_(i32(499, 69, 128, 0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(1)
        c.cache.append(new_k, new_v, c.pages, lens)
        c.cache.attend(c.q, c.pages, lens, out=out)
    for i in range(4):
        lens.copy_(i32(499 - i, 69 - 7 * i, 128 - i, 0))
        new_k.normal_()
        c.q.normal_()
        graph.replay()
        torch.cuda.synchronize()
        now = [500 - i, 70 - 7 * i, 129 - i, 1]
        assert lens.tolist() == now
        want = c.cache.attend(c.q, c.pages, i32(*now))
        assert torch.equal(out, want), i
        k, _ = c.cache.read(c.pages, i32(*now), 4)
        codes = aep.quantize_mx4(new_k.view(8, 128))
        assert torch.equal(k.view(8, 128), aep.dequantize_mx4(*codes, 128))


def test_a_captured_call_with_many_columns():
    c = Case([700, 90, 300], [100, 1, 40], 2, 4, 64, seed=19)
    want, out = c.attend(True), torch.empty_like(c.q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.attend(True, out=out)
    for i in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(c.attend(True), want), i


def test_threads_on_streams_of_their_own():
    c = Case([3000, 70, 129, 1, 0, 900], 2, 2, 4, 128, seed=17)
    qs = [c.q, c.q * 2, c.q + 1]
    torch.cuda.synchronize()
    want = [c.cache.attend(q, c.pages, c.dev_lens) for q in qs]
    torch.cuda.synchronize()
    bad = []

    def work(k):
        try:
            st = torch.cuda.Stream()
            with torch.cuda.stream(st):
                for i in range(40):
                    y = c.cache.attend(qs[(i + k) % 3], c.pages, c.dev_lens)
                    st.synchronize()
                    if not torch.equal(y, want[(i + k) % 3]):
                        bad.append((k, i))
        except Exception as e:  # (a thread's own would be lost)
            bad.append((k, repr(e)))

    threads = [threading.Thread(target=work, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad, bad[:4]


def test_pages_behind_4_gib():
    page, H, D = 4096, 16, 256
    log("attend4 behind 4 GiB")
    cache = aep.Cache4(600, H, D, page_size=page)
    cache.data.fill_(255)
    pages = i32(599, 300, 0).view(1, 3)
    T = 2 * page + 100
    k, v = rows_of(T, H, D, 11, False), rows_of(T, H, D, 12, False)
    cache.append(k, v, pages, i32(T))
    small = aep.Cache4(3, H, D, page_size=page)
    near = i32(0, 1, 2).view(1, 3)
    small.append(k, v, near, i32(T))
    q = rows_of(3, H * 2, D, 13, False)
    assert torch.equal(cache.attend(q, pages, i32(T)), small.attend(q, near, i32(T)))


def test_numbers_in_tensors_count_by_their_value():
    """A scale or a window in a tensor whose value changes between two calls."""
    c = Case([100, 30], 2, 2, 4, 64, seed=23)
    scale, window, most = torch.tensor(0.25, dtype=torch.float64), torch.tensor(0), torch.tensor(4)
    for s, w, m in ((0.25, 0, 4), (0.5, 20, 2), (0.125, 3, 0)):
        scale.fill_(s), window.fill_(w), most.fill_(m)
        want = c.attend(scale=s, window=w, max_rows=m)
        assert torch.equal(c.attend(scale=scale, window=window, max_rows=most), want)
        c.check(want, window=w, scale=s, what=(s, w))
    for kw in (dict(window=1.0), dict(max_rows=1.0), dict(window=1 << 40), dict(max_rows=-1), dict(scale=float("nan")), dict(scale="x")):
        for _ in range(2):
            with pytest.raises((TypeError, ValueError, aep.AEPError)):
                c.attend(**kw)


@pytest.mark.parametrize("n,group,D", [(70, 2, 128), (130, 1, 64), (33, 4, 256), (9, 2, 128), (1, 4, 64)])
def test_pages_before_the_window_may_be_gone(n, group, D):
    """Entries of pages that lie wholly before every row's window are out of range: nothing of them is needed, or reported."""
    c = Case([1000, 600], n, 2, group, D, page=32, seed=24)
    for window in (1, 16, 31, 32, 33, 50, 64, 65, 96, 97):
        log(f"attend4 window {window} of {n} x {group} d {D}")
        pages = c.pages.clone()
        for b, l in enumerate(c.lens):
            c.pages[b, :max(0, l - n - window + 1) // 32] = -7
        for many in (False, True):
            flag, lse = i32(0), torch.empty(c.q.shape[:2], device="cuda")
            out = c.attend(many, window=window, flag=flag, lse=lse)
            c.check(out, lse, window, what=(window, many), rows={0, 1, 31, 32, 63, 64, 65, -1})
            assert int(flag) == 0, (window, many)
        c.pages.copy_(pages)


def test_lengths_of_sequences_without_rows_do_not_count():
    c = Case([300, 70], [2, 70], 2, 4, 64, seed=25)
    pages = torch.nn.functional.pad(c.pages, (0, 0, 1, 1), value=-7)
    for many in (False, True):
        want, flag = c.attend(many), i32(0)
        need = 8 * 512 * 128 // (2 * 2) // 64 + 1 if many else 0
        t = torch.nn.functional.pad(pages, (0, max(0, need - pages.shape[1])), value=-7)
        for lens in ((-5, 2 ** 31 - 1), (2 ** 31 - 1, -2 ** 31)):
            got = c.cache.attend(c.q, t, i32(lens[0], 300, 70, lens[1]), i32(0, 0, 2, 72, 72), flag=flag)
            assert torch.equal(got, want) and int(flag) == 0, (many, lens)


def test_rows_of_no_sequence_are_zeros_without_out():
    """New tensors hold nothing that was in their memory before."""
    c = Case([300, 20], [2, 3], 2, 4, 128, seed=26)
    want = c.attend()
    q = torch.cat([c.q, c.q])
    for rows, own, none in ((c.rows, slice(0, 5), slice(5, 10)), (c.rows + 3, slice(3, 8), [0, 1, 2, 8, 9])):
        x = torch.zeros_like(q)
        x[own] = c.q
        for _ in range(3):
            junk = [torch.full_like(q, float("nan")) for _ in range(4)]
            torch.cuda.synchronize()
            del junk  # (whose memory a new tensor of its size gets)
            out = c.cache.attend(x, c.pages, c.dev_lens, rows)
            assert torch.equal(out[own], want) and bool((out[none] == 0).all())


def test_rows_of_no_sequence_are_zeros_in_a_captured_call():
    """A padded batch captured once: who has rows changes between replays, and the rows that had an owner before are zeros."""
    c = Case([300, 20, 64], [2, 3, 1], 2, 4, 128, seed=27)
    q, rows = torch.cat([c.q, c.q]), c.rows.clone()
    ends = (c.rows, i32(0, 2, 2, 2), i32(0, 0, 3, 4), c.rows + 6, c.rows)
    want = [c.cache.attend(q, c.pages, c.dev_lens, e) for e in ends]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = c.cache.attend(q, c.pages, c.dev_lens, rows)
        k, v = c.cache.read(c.pages, c.dev_lens, 12, rows)
    for e, w in zip(ends, want):
        rows.copy_(e)
        graph.replay()
        torch.cuda.synchronize()
        own = torch.zeros(12, dtype=torch.bool)
        own[int(e[0]):int(e[-1])] = True
        assert torch.equal(out, w) and bool((out[~own.cuda()] == 0).all())
        assert bool((k[~own.cuda()] == 0).all()) and bool((v[~own.cuda()] == 0).all())
        assert bool((k[own.cuda()] != 0).any(-1).all())
