"""The order of the tiled dense product's LDS accesses, on the CPU, as
test_ffn_order_host.py has it for the FFN: whatever a wave reads has landed before
a barrier that precedes the read, and is read before a barrier that precedes its
refill, whatever the timing; all waves pass the same barriers."""

import ctypes

import pytest

import linear_host


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    return linear_host.load(tmp_path_factory.mktemp("linear"))


# whole rounds; tiles of the last one, halves, pieces; family, rows and pieces of the last rows' tiles
CHAINS = {
    "whole": (3, 0, 1, 1, 0, 0, 1),
    "rest": (1, 4, 1, 1, 0, 0, 1),
    "halves": (2, 7, 2, 1, 0, 0, 1),
    "halves_alone": (0, 7, 2, 1, 0, 0, 1),
    "pieces": (1, 6, 1, 3, 0, 0, 1),
    "halves_pieces": (0, 7, 2, 2, 0, 0, 1),
    "family1": (0, 0, 1, 1, 1, 4, 1),
    "family2": (0, 0, 1, 1, 2, 4, 1),
    "family1_pieces": (0, 0, 1, 1, 1, 2, 2),
    "family2_pieces": (0, 0, 1, 1, 2, 2, 2),
    "all": (1, 5, 2, 1, 1, 1, 1),
    "all_pieces": (2, 5, 2, 2, 2, 1, 2),
}


@pytest.mark.parametrize("fp8", [0, 1])
@pytest.mark.parametrize("chain", sorted(CHAINS))
def test_lds_reads_and_refills_are_ordered(lib, chain, fp8):
    c = CHAINS[chain]
    pieces = max(c[3], c[6])
    # K steps fewer than a ring's stages, as many and more, the last one whole or not
    for steps in (4 * pieces, 4 * pieces + 1, 13) if pieces > 1 else (1, 2, 3, 4, 5, 13, 14):
        for k in (64 * steps, 64 * steps - 48):
            for xcd in (0, 7):
                n, msg = ctypes.c_long(0), ctypes.create_string_buffer(256)
                bad = lib.linear_order_violations(fp8, k, (ctypes.c_int * 7)(*c), xcd, ctypes.byref(n), msg, 256)
                assert n.value > 0 or bad or xcd, (chain, k)
                assert bad != -1, f"{chain}, K = {k}: waves pass different numbers of barriers"
                assert bad == 0, f"{chain}, K = {k}: {bad} unordered accesses; {msg.value.decode()}"
