"""CPU oracle of the quantised, sampling actor: rows to 8-bit levels, the product of levels with scales, the draw of an
index from a row of scores.  TEST INFRASTRUCTURE ONLY.  Everything in 64 bits, one row at a time, from the definitions in
include/dqn_mi355.h."""
from __future__ import annotations

from collections import namedtuple

import numpy as np


def quantize_rows(x):
    """x [rows, cols] (fp64 values of the inputs) -> levels int64, exact scales fp64 (NaN for a row that is not finite)."""
    x = np.asarray(x, dtype=np.float64)
    levels = np.zeros(x.shape, np.int64)
    scales = np.zeros(x.shape[0])
    for r, row in enumerate(x):
        if not np.all(np.isfinite(row)):
            scales[r] = np.nan
            continue
        a = np.max(np.abs(row)) if row.size else 0.0
        if a > 0:
            # 127 |x| = level a + rest, 0 <= rest < a: exact (an input has at most 24 significant bits, a level 7)
            whole = np.floor(127.0 * np.abs(row) / a)
            rest = 127.0 * np.abs(row) - whole * a
            whole, rest = np.where(rest < 0, whole - 1, whole), np.where(rest < 0, rest + a, rest)
            up = (2 * rest > a) | ((2 * rest == a) & (whole % 2 == 1))
            levels[r] = np.sign(row).astype(np.int64) * (whole + up).astype(np.int64)
        scales[r] = a / 127.0
    return levels, scales


def linear(xq, sx, wq, sw, bias=None, relu=False):
    """act(sx sw (xq wq^T) + bias): the sums in whole numbers, the rest in fp64."""
    acc = np.asarray(xq).astype(np.float64) @ np.asarray(wq).astype(np.float64).T   # exact below 2^53
    y = acc * np.outer(np.asarray(sx, np.float64), np.asarray(sw, np.float64))
    if bias is not None:
        y = y + np.asarray(bias, np.float64)
    return np.where(y < 0, 0.0, y) if relu else y


Drawn = namedtuple("Drawn", "index logp low high filter_margin")
"""index, logp: the draw (-1 and NaN for a refused row).  low, high: the lowest and highest index that a shift of u by `slack`
(relative to the kept mass) reaches.  filter_margin: how near the nearest entry lies to top-p's border, relative to the mass."""


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, slack=0.0):
    x = np.asarray(x, dtype=np.float64)
    refused = Drawn(-1, np.nan, -1, -1, np.inf)
    t = float(temperature)
    if not (t >= 0 and t < np.inf) or np.isnan(top_p) or np.isnan(min_p) or np.isnan(u) or np.any(np.isnan(x)):
        return refused
    if x.size == 0 or np.max(x) == -np.inf:
        return refused
    top = np.max(x)
    if t == 0:
        i = int(np.argmax(x))
        return Drawn(i, 0.0, i, i, np.inf)
    with np.errstate(invalid="ignore", over="ignore"):
        w = np.where(x == top, 1.0, np.exp((x - top) / t))
    order = np.lexsort((np.arange(x.size), -x))
    margin = np.inf
    if 0 < top_k < x.size:
        order = order[:int(top_k)]
    if top_p < 1:
        mass = float(np.sum(w[order]))
        before = np.concatenate([[0.0], np.cumsum(w[order])[:-1]])
        keep = before < top_p * mass
        keep[0] = True
        if top_p > 0 and order.size > 1:
            margin = float(np.min(np.abs(before[1:] - top_p * mass))) / mass
        order = order[keep]
    order = np.sort(order[w[order] >= min(min_p, 1.0)])
    c = np.cumsum(w[order])
    u = min(max(float(u), 0.0), 1 - 2.0 ** -24)

    def at(share):
        i = int(np.searchsorted(c, share * c[-1], side="right"))
        return min(i, int(np.searchsorted(c, c[-1])))
    i = at(u)
    return Drawn(int(order[i]), float(np.log(w[order[i]] / c[-1])), int(order[at(max(0.0, u - slack))]), int(order[at(u + slack)]), margin)
