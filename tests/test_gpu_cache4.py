"""The cache in 4 bits: rows written and read back against a 64-bit quantiser, every byte of the
cache that a call does not write left as it was, and what the calls do with rows, lengths and pages out of range."""

import numpy as np
import pytest
import torch

import mx4_ref
import paper_2505_08944_amd as aep
from gpu_helpers import log

pytestmark = pytest.mark.gpu


def i32(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def table(lens, page, n_pages, seed=0):
    """Pages in random order, each of one sequence; unused entries are out of range, which no call may mind."""
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).tolist()
    per = [-(-l // page) for l in lens]
    assert sum(per) <= n_pages
    t = torch.full((len(lens), max(1, max(per))), -7, dtype=torch.int32)
    for b, n in enumerate(per):
        for i in range(n):
            t[b, i] = order.pop()
    return t.cuda()


def rows_of(T, H, D, seed=0, scale=True):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, H, D, generator=g)
    if scale:
        x = x * torch.exp2(torch.randint(-8, 8, (T, H, 1), generator=g).float())
    return x.to(torch.bfloat16).cuda()


def kept(x):
    return mx4_ref.quantize(x.double().cpu().numpy())[2]


def equal(t, want):
    return np.array_equal(t.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("H,D,page", [(1, 64, 32), (8, 128, 64), (3, 256, 32), (2, 128, 256), (5, 64, 128), (16, 256, 64),
                                      (1, 128, 4096)])
def test_written_and_read(H, D, page):
    """Prompts of odd lengths, then single tokens, then several: all tokens read back, whole and in part."""
    log(f"cache4 heads {H} d {D} page {page}")
    lens = [1, 31, 33, 0, page, page + 1, 2 * page + 17]
    new = [1, 1, 1, 1, 1, 1, 1]
    more = [5, 40, 1, 0, 3, 2, 70]
    n_pages = sum(-(-(a + b + c) // page) for a, b, c in zip(lens, new, more)) + 3
    cache = aep.Cache4(n_pages, H, D, page_size=page)
    total = [a + b + c for a, b, c in zip(lens, new, more)]
    pages = table(total, page, n_pages)
    flag = i32(0)
    ks, vs = [[] for _ in lens], [[] for _ in lens]
    have = [0] * len(lens)
    for step, n in enumerate((lens, new, more)):
        T = sum(n)
        k, v = rows_of(T, H, D, 2 * step), rows_of(T, H, D, 2 * step + 1)
        k[0, 0, 5] = float("nan")
        have = [a + b for a, b in zip(have, n)]
        at = np.concatenate([[0], np.cumsum(n)])
        uniform = len(set(n)) == 1
        cache.append(k, v, pages, i32(*have), None if uniform else i32(*at.tolist()), flag=flag)
        kk, kv = kept(k), kept(v)
        for b in range(len(lens)):
            ks[b].append(kk[at[b]:at[b + 1]])
            vs[b].append(kv[at[b]:at[b + 1]])
        rk, rv = cache.read(pages, i32(*have), T, None if uniform else i32(*at.tolist()), flag=flag)
        assert equal(rk, kk) and equal(rv, kv), step
    at = np.concatenate([[0], np.cumsum(total)]).tolist()
    k, v = cache.read(pages, i32(*total), at[-1], i32(*at), flag=flag)
    assert equal(k, np.concatenate([np.concatenate(t) for t in ks]))
    assert equal(v, np.concatenate([np.concatenate(t) for t in vs]))
    assert int(flag) == 0


@pytest.mark.parametrize("D", [64, 128, 256])
def test_other_places_stay(D):
    """A token's bytes are its own: all others of the allocation stay as they were."""
    H, page = 3, 64
    cache = aep.Cache4(4, H, D, page_size=page)
    cache.data.random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(1))
    before = cache.data.clone()
    pages = i32(2, 0).view(1, 2)
    cache.append(rows_of(1, H, D), rows_of(1, H, D, 1), pages, i32(64 + 38))
    diff = int((cache.data != before).sum())
    assert diff <= 2 * H * (D // 2 + D // 32)
    # written again with what is there: nothing changes but that token's bytes
    after = cache.data.clone()
    cache.append(rows_of(1, H, D), rows_of(1, H, D, 1), pages, i32(64 + 38))
    assert torch.equal(cache.data, after)
    # every token written once: every byte is written
    other = aep.Cache4(4, H, D, page_size=page)
    other.data.fill_(0x5a)
    x = torch.full((256, H, D), 6.0, dtype=torch.bfloat16, device="cuda")
    other.append(x, x, i32(3, 1, 0, 2).view(1, 4), i32(256))
    assert not bool((other.data == 0x5a).any())


def test_strided_rows():
    """Keys and values as slices of one product's rows."""
    H, D, T = 4, 128, 37
    cache = aep.Cache4(3, H, D)
    qkv = rows_of(T, 3 * H, D, 3).view(T, 3 * H * D)
    k, v = qkv[:, H * D:2 * H * D].view(T, H, D), qkv[:, 2 * H * D:].view(T, H, D)
    pages = i32(2, 0).view(1, 2)
    cache.append(k, v, pages, i32(T))
    rk, rv = cache.read(pages, i32(T), T)
    assert equal(rk, kept(k)) and equal(rv, kept(v))
    # heads in front of rows, at an odd address
    buf = rows_of(1, 1, H * T * D + 1, 4).view(-1)[1:].view(H, T, D).transpose(0, 1)
    cache.append(buf, buf, pages, i32(T))
    rk, rv = cache.read(pages, i32(T), T)
    assert equal(rk, kept(buf)) and equal(rv, kept(buf))


def test_rows_without_tokens_and_behind_the_last_sequence():
    H, D = 2, 64
    cache = aep.Cache4(4, H, D, page_size=32)
    pages, flag = i32(0, 1, 2, 3).view(2, 2), i32(0)
    k, v = rows_of(12, H, D, 5), rows_of(12, H, D, 6)
    # 5 rows of a sequence of 3 tokens; 4 rows of one of 40; three rows of nobody
    cache.append(k, v, pages, i32(3, 40), i32(0, 5, 9), flag=flag)
    ok, ov = torch.full_like(k, 9.0), torch.full_like(v, 9.0)
    cache.read(pages, i32(3, 40), 12, i32(0, 5, 9), k=ok, v=ov, flag=flag)
    for got, x in ((ok, k), (ov, v)):
        want = kept(x)
        want[:2], want[9:] = 0.0, 9.0
        assert equal(got, want)
    assert int(flag) == 0
    # rows that begin behind the first
    cache.read(pages, i32(3, 40), 12, i32(3, 5, 9), k=ok.fill_(9.0), v=ov)
    assert bool((ok[:3] == 9).all()) and equal(ok[3:5], kept(k)[3:5])


def test_what_only_the_device_sees_is_held_to_bounds_and_reported():
    H, D = 2, 64
    k, v = rows_of(8, H, D, 7), rows_of(8, H, D, 8)
    for pages, lens, rows in (((0, 5), (40, 3), None), ((0, -1), (40, 3), None), ((0, 1), (65, 3), None), ((0, 1), (-4, 3), None),
                              ((0, 1), (40, 3), (0, 9, 8)), ((0, 1), (40, 3), (0, 4, 20)), ((0, 1), (40, 3), (-3, 4, 8)),
                              ((0, 1), (2 ** 31 - 1, -2 ** 31), (2 ** 31 - 1, -2 ** 31, 0))):
        cache, flag = aep.Cache4(4, H, D, page_size=32), i32(0)
        t = i32(*pages, 2, 3).view(2, 2)
        r = None if rows is None else i32(*rows)
        cache.append(k, v, t, i32(*lens), r, flag=flag)
        assert int(flag) == 1, (pages, lens, rows)
        flag.zero_()
        cache.read(t, i32(*lens), 8, r, flag=flag)
        assert int(flag) == 1, (pages, lens, rows)
        cache.append(k, v, t, i32(*lens), r)  # (reported to nobody)


def test_nothing_to_do():
    cache = aep.Cache4(1, 2, 64)
    e = torch.empty(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    cache.append(e, e, i32().view(0, 1), i32())
    cache.append(e, e, i32(0).view(1, 1), i32(5))
    k, v = cache.read(i32(0).view(1, 1), i32(5), 0)
    assert k.shape == (0, 2, 64) and v.shape == (0, 2, 64)


@pytest.mark.parametrize("B", [1, 63, 64, 65, 1000])
def test_many_sequences(B):
    """Sequences of no, one and several rows, found among many."""
    H, D = 1, 64
    n = [(b * 7) % 4 for b in range(B)]
    lens = [m + (b % 3) for b, m in enumerate(n)]
    cache = aep.Cache4(B, H, D, page_size=32)
    pages = torch.arange(B, dtype=torch.int32, device="cuda").view(B, 1)
    at = np.concatenate([[0], np.cumsum(n)]).tolist()
    k, v = rows_of(at[-1] + 2, H, D, 9), rows_of(at[-1] + 2, H, D, 10)
    cache.append(k, v, pages, i32(*lens), i32(*at))
    rk, rv = cache.read(pages, i32(*lens), at[-1], i32(*at))
    assert equal(rk, kept(k)[:at[-1]]) and equal(rv, kept(v)[:at[-1]])


def test_more_than_32_bits_of_bytes():
    """Pages that lie behind 4 GiB."""
    H, D, page = 16, 256, 4096
    n_pages = 600
    log(f"cache4 of {n_pages} pages")
    cache = aep.Cache4(n_pages, H, D, page_size=page)
    assert n_pages * page * H * D // 2 > 1 << 32  # (of keys alone)
    pages = i32(0, n_pages - 1, n_pages // 2).view(1, 3)
    T = 2 * page + 100
    k, v = rows_of(T, H, D, 11, False), rows_of(T, H, D, 12, False)
    cache.append(k, v, pages, i32(T))
    rk, rv = cache.read(pages, i32(T), T)
    for got, x in ((rk, k), (rv, v)):
        codes, scale = aep.quantize_mx4(x.view(T * H, D))
        assert torch.equal(got, aep.dequantize_mx4(codes, scale, D).view(T, H, D))


def test_a_number_of_rows_in_a_tensor_counts_by_its_value():
    cache = aep.Cache4(4, 1, 64)
    pages, lens = i32(0, 1)[None], i32(100)
    k, v = rows_of(100, 1, 64, 1), rows_of(100, 1, 64, 2)
    cache.append(k, v, pages, lens)
    n = torch.tensor(3)
    for rows in (3, 50, 1):
        n.fill_(rows)
        for got, x in zip(cache.read(pages, lens, n), (k, v)):
            assert got.shape == (rows, 1, 64) and equal(got, kept(x[100 - rows:]))
    for bad in (3.0, 1 << 40, -1, "3"):
        for _ in range(2):
            with pytest.raises((TypeError, ValueError, aep.AEPError)):
                cache.read(pages, lens, bad)


# sequences' pages (of 32 tokens, 4 in the cache), lens and rows of 8 rows; what of it has a place: (sequence, its
# pages, len, first row, rows) of calls that have nothing out of range
PLACES = [
    ([[0, -1], [2, 3]], (40, 3), None, [(1, [2, 3], 3, 4, 4)]),
    ([[0, 4], [2, 3]], (40, 36), None, [(1, [2, 3], 36, 4, 4)]),
    ([[1, 2 ** 31 - 1], [-2 ** 31, 3]], (34, 36), None, [(0, [1, 0], 32, 0, 2), (1, [0, 3], 36, 4, 4)]),
    ([[-1, 1], [99, -1]], (34, 1), None, [(0, [0, 1], 34, 2, 2)]),
    ([[0, 1], [2, 3]], (65, 3), None, [(0, [0, 1], 64, 0, 3), (1, [2, 3], 3, 4, 4)]),
    ([[0, 1], [2, 3]], (2 ** 31 - 1, 67), None, [(1, [2, 3], 64, 4, 1)]),
    ([[0, 1], [2, 3]], (-4, 68), None, []),
    ([[0, 1], [2, 3]], (40, 20), (0, 4, 20), [(0, [0, 1], 40, 0, 4)]),
    ([[0, 1], [2, 3]], (40, 20), (-3, 4, 8), [(1, [2, 3], 20, 4, 4)]),
    ([[0, 1], [2, 3]], (40, 20), (0, 3, 9), [(0, [0, 1], 40, 0, 3)]),
]


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("i", range(len(PLACES)))
def test_rows_without_a_place_are_left_out(i, D):
    """A page outside the cache, a token behind the last page, rows that are not there: nothing is written for them,
    into nobody's place; what has a place is written to it."""
    log(f"cache4 places {i} d {D}")
    pages, lens, rows, right = PLACES[i]
    H = 2
    k, v = rows_of(8, H, D, 7), rows_of(8, H, D, 8)
    cache, want, flag = aep.Cache4(4, H, D, page_size=32), aep.Cache4(4, H, D, page_size=32), i32(0)
    cache.data.random_(0, 256, generator=torch.Generator(device="cuda").manual_seed(i))
    want.data.copy_(cache.data)
    for _, p, l, at, n in right:
        want.append(k[at:at + n], v[at:at + n], i32(*p).view(1, 2), i32(l))
    t, r = i32(*pages[0], *pages[1]).view(2, 2), None if rows is None else i32(*rows)
    cache.append(k, v, t, i32(*lens), r, flag=flag)
    assert int(flag) == 1
    assert torch.equal(cache.data, want.data)
    cache.append(k, v, t, i32(*lens), r)  # (reported to nobody)
    assert torch.equal(cache.data, want.data)


def test_a_captured_step_grows_past_its_pages():
    """A step captured once: a slot without a sequence, and a sequence that has no page yet for its next token, leave all
    others' tokens as they are, until they have a page."""
    H, D, page = 2, 128, 32
    cache, flag = aep.Cache4(3, H, D, page_size=page), i32(0)
    pages, lens = i32(0, 2, 1, -1, -1, -1).view(3, 2), i32(62, 30, -1)
    k, v = rows_of(3, H, D, 20), rows_of(3, H, D, 21)
    old_k, old_v = rows_of(62, H, D, 22), rows_of(62, H, D, 23)
    cache.append(old_k, old_v, pages[:1], lens[:1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lens.add_(1)
        cache.append(k, v, pages, lens, flag=flag)
    for step, now in enumerate(((63, 31, 0), (64, 32, 1))):
        graph.replay()
        torch.cuda.synchronize()
        assert lens.tolist() == list(now) and int(flag) == step
    flag.zero_()
    lens[0] = 0  # (a sequence that is full: taken out)
    before = cache.data.clone()
    pages[0].fill_(-1)
    lens[0] = -1
    graph.replay()  # the second one's token 33 has no page
    torch.cuda.synchronize()
    assert lens.tolist() == [0, 33, 2] and int(flag) == 1 and torch.equal(cache.data, before)
    rk, rv = cache.read(i32(0, 2).view(1, 2), i32(62), 62)
    assert equal(rk, kept(old_k)) and equal(rv, kept(old_v))
    pages[1, 1] = 2
    lens[1] = 32
    graph.replay()
    torch.cuda.synchronize()
    rk, rv = cache.read(pages[1:2], lens[1:2], 1)
    assert equal(rk, kept(k[1:2])) and equal(rv, kept(v[1:2]))


def test_lengths_of_sequences_without_rows_do_not_count():
    H, D = 2, 64
    cache, flag = aep.Cache4(2, H, D, page_size=32), i32(0)
    pages, lens, rows = i32(0, 7, 1).view(3, 1), i32(-5, 2 ** 31 - 1, 20), i32(0, 0, 0, 4)
    k, v = rows_of(4, H, D, 24), rows_of(4, H, D, 25)
    cache.append(k, v, pages, lens, rows, flag=flag)
    rk, rv = cache.read(pages, lens, 4, rows, flag=flag)
    assert equal(rk, kept(k)) and equal(rv, kept(v)) and int(flag) == 0


def test_rows_of_no_sequence_read_as_zeros_where_there_is_no_tensor_for_them():
    H, D = 2, 128
    cache = aep.Cache4(2, H, D, page_size=32)
    k, v = rows_of(9, H, D, 26), rows_of(9, H, D, 27)
    pages, lens, rows = i32(1, 0).view(2, 1), i32(20, 4), i32(2, 4, 6)
    cache.append(k, v, pages, lens, rows)
    for _ in range(3):
        junk = [torch.full_like(k, float("nan")) for _ in range(4)]
        torch.cuda.synchronize()
        del junk  # (whose memory a new tensor of its size gets)
        for got, x in zip(cache.read(pages, lens, 9, rows), (k, v)):
            want = kept(x)
            want[:2], want[6:] = 0.0, 0.0
            assert equal(got, want)
