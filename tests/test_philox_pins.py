"""Dropout's generator against the known answers that are published with it (Salmon, Moraes,
Dror and Shaw, 2011: the vectors of Philox-4x32 with 10 rounds), which the oracle that the
kernels are compared with inherits."""
import pytest
import torch

import operators_oracle as ref

MASK = 0xFFFFFFFF


def philox(c, k):
    c, k = list(c), list(k)
    for r in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        key = [(k[0] + r * 0x9E3779B9) & MASK, (k[1] + r * 0xBB67AE85) & MASK]
        c = [(p1 >> 32) ^ c[1] ^ key[0], p1 & MASK, (p0 >> 32) ^ c[3] ^ key[1], p0 & MASK]
    return c


@pytest.mark.parametrize("counter,key,words", [
    ([0] * 4, [0] * 2, [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([MASK] * 4, [MASK] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
])
def test_published_answers(counter, key, words):
    assert philox(counter, key) == words


def oracle_numbers(n, seed, offset):
    """The 16-bit numbers behind keep_mask: the largest threshold that keeps the element."""
    r = torch.zeros(n, dtype=torch.int64)
    for bit in range(15, -1, -1):
        for i in range(n):
            t = int(r[i]) | 1 << bit
            r[i] = t if ref.keep_mask(n, t / 65536, seed, offset)[i] else r[i]
    return r.tolist()


@pytest.mark.parametrize("seed,offset", [(0, 0), (0x299F31D0A4093822, 0x0370734413198A2E),
                                         ((1 << 64) - 1, (1 << 64) - 1)])
def test_the_oracle_draws_from_it(seed, offset):
    n = 20   # three counters, the last one's numbers in part
    want = []
    for block in range(3):
        for w in philox([block, 0, offset & MASK, offset >> 32], [seed & MASK, seed >> 32]):
            want += [w & 0xFFFF, w >> 16]
    assert oracle_numbers(n, seed, offset) == want[:n]


def test_the_published_numbers_in_the_oracle():
    assert oracle_numbers(8, 0, 0) == [0xE8D5, 0x6627, 0xC58D, 0xE169, 0xAC4C, 0xBC57, 0xDBD8,
                                       0x9B00]
