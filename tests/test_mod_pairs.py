"""How the dropout decisions of keys j and j xor 1, which share two bytes, hang together: all 65536 pairs of bytes, through the oracle of these calls.  No GPU."""
import os
import re

import numpy as np
import pytest

import mod_oracle as M

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "sigmoid_attn.h")


@pytest.fixture
def falls(monkeypatch):
    """p -> [65536, 2] truth values of what falls of one pair of keys, for every value of their two bytes."""
    a, b = (x.ravel().astype(np.uint64) for x in np.meshgrid(np.arange(256), np.arange(256), indexing="ij"))
    words = []
    for w in range(4):                                          # keys 0 and 1 take bits 0 and 8, 16 and 24 of each word
        bit = lambda byte, s: (byte >> np.uint64(s)) & np.uint64(1)
        word = sum(bit(byte, 2 * w + odd) << np.uint64(at + 8 * odd) for byte, at in ((a, 0), (b, 16)) for odd in (0, 1))
        words.append(np.repeat(word[:, None], 2, axis=1))
    monkeypatch.setattr(M, "philox", lambda counter, key, rounds: words)
    return lambda p: ~M.mask(0, 0, 0, 65536, 2, p)


def stated():
    text = " ".join(re.sub(r"^ \*", "", line) for line in open(HEADER).read().split("\n"))
    text = re.sub(r"\s+", " ", text)
    number = r"(\d+(?:\.\d+)?(?:e-\d+)?)"
    bound = re.search(r"both fall has a probability of \(1 - keep\)\^2 to \(1 - keep\)\^2 \+ " + number, text)
    ratios = re.findall(number + r" times (?:as often as independent ones )?(?:at|from)(?: 1 - keep =)? " + number, text)
    return float(bound.group(1)), [(float(a), float(b)) for a, b in ratios]


@pytest.mark.parametrize("p", [1e-5, 0.0005, 0.001, 0.002, 0.004, 0.01, 0.02, 0.05, 0.1, 0.2, 0.33, 1 / 3, 0.4, 0.5, 0.7, 0.9, 0.999])
def test_both_of_a_pair(falls, p):
    bound, _ = stated()
    f = falls(p)
    out = 65536 - M.kept(p)
    assert f[:, 0].sum() == f[:, 1].sum() == out                # each alone: exactly its share
    over = f.all(axis=1).sum() / 65536 - (out / 65536) ** 2
    assert 0 <= over <= bound


def test_the_bound_for_every_share():
    # the larger of a pair's two numbers decides whether both fall
    reverse = np.array([int(f"{i:08b}"[::-1], 2) for i in range(256)])
    a, b = np.meshgrid(np.arange(256), np.arange(256), indexing="ij")
    both = np.bincount(np.maximum(256 * a + reverse[b], 256 * b + reverse[a]).ravel(), minlength=65536).cumsum() / 65536    # both below 1, 2, ..
    share = np.arange(1, 65537) / 65536
    bound, ratios = stated()
    assert 0 <= (both - share ** 2).min() and 0.98 * bound < (both - share ** 2).max() <= bound
    assert len(ratios) == 4
    for ratio, at in ratios:
        got = (both / share ** 2)[share >= at].max() if at >= 0.02 else (both / share ** 2)[int(at * 65536 + 0.5) - 1]
        assert 0.98 * ratio < got <= 1.01 * ratio, (at, got)
