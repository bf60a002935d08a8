"""How far dropout's mask is from independent where word numbers are far apart: the figures that
the header gives are those of the words."""
import os
import re
import sys

import numpy as np

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import moments_ref as M  # noqa: E402

HEADER = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "lmzipf.h")
SAMPLES = 1 << 18


def stated():
    """[(distances below 2^this, correlation at most)] from the header, the last without a limit."""
    with open(HEADER) as f:
        text = re.sub(r"\n \*\s*", " ", f.read())
    within = re.findall(r"(0\.\d+) within 2\^(\d+) words", text)
    beyond = re.search(r"(0\.\d+) beyond", text)
    assert len(within) >= 3 and beyond, "the header gives no figures"
    return [(int(b), float(c)) for c, b in within] + [(64, float(beyond.group(1)))]


def correlation(distance, seed, start, p):
    """The largest correlation, over the halves of words, of what is kept `distance` words apart."""
    e = np.random.default_rng(distance % 1_000_003).integers(0, 1 << 24, SAMPLES, dtype=np.uint64)
    e += np.uint64(start)
    T = round(65536 * p)
    most = 0.0
    for shift in (0, 16):
        a, b = ((((M.words(x, seed) >> np.uint32(shift)) & np.uint32(0xFFFF)) >= T) - (1 - p)
                for x in (e, e + np.uint64(distance)))
        most = max(most, abs(float((a * b).mean())) / (p * (1 - p)))
    return most


def test_correlations_are_those_of_the_header():
    """Powers of two, and the sums and multiples of them that correlate most."""
    figures = stated()
    far = [1 << b for b in range(36)] + [3 << b for b in range(0, 34, 3)]
    far += [496, 1920, 8448, 126_976, 135_168, 17 << 19, 31_457_280, 62_914_560, 71_303_168,
            1_006_632_960, 1_140_850_688, 65 << 32]
    found = {}
    for d in far:
        limit = next(c for b, c in figures if d < 1 << b)
        for seed, start in ((3, 0), (77, 1 << 25), (9, 1 << 20), (12345, 1 << 25)):
            for p in (0.1, 0.5, 0.9):
                c = correlation(d, seed, start, p)
                assert c <= limit + 6 / SAMPLES ** 0.5, (d, seed, p, c)
                found[limit] = max(found.get(limit, 0.0), c)
    # and no figure is far above what there is: the limits are real ones
    assert all(c >= 0.4 * limit for limit, c in found.items()), found


def test_neighbouring_words_are_independent():
    for d in range(1, 65):
        for p in (0.1, 0.5):
            assert correlation(d, 5, 0, p) < 6 / SAMPLES ** 0.5
