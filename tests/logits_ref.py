"""Plain 64-bit implementations of the calls on logits, for the tests: numpy on
the CPU, by the definitions, one row at a time."""
from __future__ import annotations

import math

import numpy as np

FREE, FINISHED, DEAD = -3, -2, -1
M64 = (1 << 64) - 1


def pack(allowed: np.ndarray) -> np.ndarray:
    """bool [R, V] as int32 mask rows [R, ceil(V/32)]."""
    R, V = allowed.shape
    bits = np.zeros((R, (V + 31) // 32 * 32), np.uint8)
    bits[:, :V] = allowed
    return np.packbits(bits, axis=1, bitorder="little").view(np.int32)


def allowed_row(allowed, state: int, V: int) -> np.ndarray:
    """bool [V]: what a row in `state` allows (allowed: bool [R, V] or None)."""
    if allowed is None or state == FREE:
        return np.ones(V, bool)
    if 0 <= state < len(allowed):
        return allowed[state]
    row = np.zeros(V, bool)
    row[V - 1] = True
    return row


def penalize(x, history, prompt, r, p, f, bias, ok):
    """(result, bound) of one row in 64 bits: x float [V], history a list of ids, bias a list of (id, value).
    The bound is on the error of the same steps in 32 bits: half a unit of the last place of each result."""
    V = len(x)
    y = x.astype(np.float64)
    bound = np.zeros(V)
    count, seen = {}, set()
    for i, t in enumerate(history):
        if 0 <= t < V:
            seen.add(t)
            if i >= prompt:
                count[t] = count.get(t, 0) + 1
    u = 2.0 ** -24
    total = {}

    def fit(v):  # past the largest number of 32 bits is infinite there
        return math.copysign(math.inf, v) if abs(v) > 3.4028235677973366e38 else v
    with np.errstate(all="ignore"):
        for t in seen:
            y[t] = fit(y[t] / r if y[t] > 0 else y[t] * r)
            bound[t] += abs(y[t]) * u
        for t, c in count.items():
            y[t] = fit(y[t] - f * c)
            bound[t] += (abs(f * c) + abs(y[t])) * u
            y[t] = fit(y[t] - p)
            bound[t] += abs(y[t]) * u
        for t, v in bias:
            if 0 <= t < V:
                total[t] = total.get(t, 0.0) + v
                bound[t] += abs(total[t]) * u
        for t, v in total.items():
            y[t] = fit(y[t] + v)
            bound[t] += abs(y[t]) * u
    y[~ok] = -math.inf
    bound[~ok] = 0
    return y, bound


def noise(seed: int, n: int) -> float:
    z = (seed + (n + 1) * 0x9E3779B97F4A7C15) & M64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    z ^= z >> 31
    return -math.log(-math.log((2 * (z >> 41) + 1) / 2 ** 24))


def kept(x, T, k, p, min_p, ok):
    """(ids in order, their weights, margin) of one row that top-k, top-p and min-p keep. The margin is how
    far, relative, the decisions of top-p and min-p are from the other way."""
    y = np.where(ok & ~np.isnan(x), x.astype(np.float64), -math.inf)
    top = y.max()
    if top == -math.inf:
        return np.zeros(0, int), np.zeros(0), math.inf
    with np.errstate(all="ignore"):
        w = np.where(y == top, 1.0, np.where(y > -math.inf, np.exp((y - top) / T), 0.0))
    order = np.argsort(-y, kind="stable")
    order = order[y[order] > -math.inf]
    if k > 0:
        order = order[:k]
    ws, n, margin = w[order], len(order), math.inf
    if p < 1:
        target = p * ws.sum()
        before = np.cumsum(ws) - ws
        n = max(1, int((before < target).sum()))
        near = np.abs(before[1:] - target) / ws.sum()
        margin = min(margin, near.min(initial=math.inf))
    if min_p > 0:
        n = max(1, min(n, int((ws >= min_p).sum())))
        margin = min(margin, float((np.abs(ws[1:] - min_p) / min_p).min(initial=math.inf)))
    return order[:n], ws[:n], margin


def sample(x, seed, T, k, p, min_p, ok):
    """(token, logprob, margin) of one row: the margin is how far the nearest decision is from the other way."""
    greedy = not T > 0
    T = 1.0 if greedy else T
    V = len(x)
    y = np.where(ok & ~np.isnan(x), x.astype(np.float64), -math.inf)
    top = y.max()
    if top == -math.inf:
        return -1, -math.inf, math.inf
    with np.errstate(all="ignore"):
        z = np.where(y == top, 0.0, (y - top) / T)
        log_sum = math.log(np.where(y > -math.inf, np.exp(z), 0.0).sum())
    if greedy:
        t = int(np.argmax(y))
        return t, float(z[t] - log_sum), math.inf
    ids, ws, margin = kept(x, T, k if 0 < k < V else 0, p, min_p, ok)
    mass = {}
    for i, w in zip(ids.tolist(), ws.tolist()):
        mass[i // 256] = mass.get(i // 256, 0.0) + w

    def draw(scores):
        nonlocal margin
        best = max(scores, key=lambda s: (s[0], -s[1]))
        for s, i in scores:
            if i != best[1]:
                margin = min(margin, best[0] - s)
        return best[1]

    group = draw([(math.log(m) + noise(seed, 2 ** 31 + j), j) for j, m in mass.items() if m > 0])
    t = draw([(float(z[i]) + noise(seed, i), i) for i, w in zip(ids.tolist(), ws.tolist()) if i // 256 == group])
    return t, float(z[t] - log_sum), margin
