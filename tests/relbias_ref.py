"""The buckets of a relative position bias in whole numbers (no test functions here)."""
from __future__ import annotations

import functools


@functools.lru_cache(maxsize=None)
def far_borders(near, far, N):
    """first[t]: the smallest distance d >= near with d^N >= near^(N - t) far^t, that is
    floor(N log(d / near) / log(far / near)) >= t."""
    first, d = [], near
    for t in range(N):
        most = near ** (N - t) * far ** t
        while d ** N < most:
            d += 1
        first.append(d)
    return first


def bucket(rel, nb, far, mode):
    """The bucket of distance rel = key - query, -1 where it is masked."""
    if mode == "causal" and rel > 0:
        return -1
    n = nb // 2 if mode == "both" else nb
    near = n // 2
    d = abs(rel) if mode == "both" else max(-rel, 0)
    if d < near:
        b = d
    else:
        b = near - 1 + sum(d >= f for f in far_borders(near, far, n - near))
    return b + (n if mode == "both" and rel > 0 else 0)
