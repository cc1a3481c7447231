"""Plain forms of the expert layer in 64 bits, for its tests: from the definitions
in include/fastbfp.h, with no code of the library."""
from __future__ import annotations

import numpy as np


def routing(tokens, top, experts, seed, drop=0.0, skew=0.0, busy=None):
    """ids int64 [tokens, top]: distinct experts for each token (all of the first
    `busy` ones where given), -1 or an id past the end for dropped choices."""
    rng = np.random.Generator(np.random.PCG64(seed))
    n = experts if busy is None else busy
    score = rng.gumbel(size=(tokens, n)) - skew * np.log1p(rng.permutation(n))
    ids = np.argsort(-score, axis=1)[:, :top].astype(np.int64)
    gone = rng.random(ids.shape) < drop
    return np.where(gone, np.where(rng.random(ids.shape) < 0.5, -1, experts + 3), ids)


def plan(ids, experts):
    """(offsets, k_offsets, order, place) by a list for each expert."""
    lists = [[] for _ in range(experts + 1)]
    for slot, e in enumerate(ids.reshape(-1).tolist()):
        lists[e if 0 <= e < experts else experts].append(slot)
    order = np.array([s for part in lists for s in part], dtype=np.int64)
    place = np.empty_like(order)
    place[order] = np.arange(order.size)
    counts = [len(part) for part in lists[:experts]]
    offsets = np.concatenate([[0], np.cumsum(counts)]).astype(np.int64)
    k_offsets = np.concatenate([[0], np.cumsum([-(-n // 128) * 128 for n in counts])]).astype(np.int64)
    return offsets, k_offsets, order, place


def token_places(x, offsets, k_offsets, places):
    """Rows of x (in the experts' order) at their places in the token grouping."""
    out = np.zeros((places, x.shape[1]), dtype=x.dtype)
    for e in range(len(offsets) - 1):
        n = offsets[e + 1] - offsets[e]
        out[k_offsets[e]:k_offsets[e] + n] = x[offsets[e]:offsets[e + 1]]
    return out
