"""trie_sample where its ranges end, against the definition in 64 bits (the rules of test_gpu_sample.py)."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as ref
from test_gpu_sample import _check, _logits, _run, cuda  # noqa: F401 (cuda: a fixture)

pytestmark = pytest.mark.gpu


def _full(B, T=1.0, k=0, p=1.0, min_p=0.0):
    return [np.full(B, v, t) for v, t in ((T, np.float32), (k, np.int32), (p, np.float32), (min_p, np.float32))]


def _seeds(rng, B):
    return rng.integers(-2 ** 63, 2 ** 63 - 1, B)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 40000])
@pytest.mark.parametrize("min_p", [1.0000001, 1.5, math.inf])
@pytest.mark.parametrize("k,p", [(0, 1.0), (0, 0.9), (50, 1.0), (300, 0.9)])
def test_min_p_above_one(cuda, V, k, p, min_p, dtype):  # noqa: F811
    """No weight reaches min_p: the first token is kept all the same, the lowest id of equal logits."""
    rng = np.random.default_rng([V, k])
    B = 6
    x = _logits(rng, B, V, dtype)
    x[1] = 0.5
    x[2, V // 2:] = 40.0
    allowed = rng.random((3, V)) < 0.01
    allowed[2] = False
    states = np.array([ref.FREE, ref.FREE, ref.FREE, 0, 1, 2], np.int32)
    seeds, ways = _seeds(rng, B), _full(B, 0.7, k, p, min_p)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways, allowed, states)
    with np.errstate(invalid="ignore"):  # how far weights are from an infinite min_p
        _check(x, seeds, *ways, allowed, states, tok, lp)
    assert tok[1] == 0 and tok[2] == V // 2 and tok[5] == -1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [700, 40001])
@pytest.mark.parametrize("k,p,min_p", [(0, 1.0, 0.0), (50, 1.0, 0.0), (0, 0.9, 0.0), (300, 0.9, 0.2)])
@pytest.mark.parametrize("temperature", [1e-45, 1e-39, 1e-38, 3e38, math.inf])
def test_extreme_temperatures(cuda, temperature, V, k, p, min_p, dtype):  # noqa: F811
    """Next to zero: the largest logits alone have weight. Next to infinity: all that are allowed and finite have
    the same. Rows with masked, -inf and NaN logits beside free ones."""
    rng = np.random.default_rng([V, k])
    B = 6
    x = _logits(rng, B, V, dtype)
    x[1, ::3] = -math.inf
    x[1, 1::3] = math.nan
    x[2, 5::97] = 41.0
    allowed = rng.random((3, V)) < 0.03
    allowed[2, :] = False
    states = np.array([ref.FREE, ref.FREE, ref.FREE, 0, 1, 2], np.int32)
    seeds, ways = _seeds(rng, B), _full(B, temperature, k, p, min_p)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways, allowed, states)
    _check(x, seeds, *ways, allowed, states, tok, lp)
    assert tok[5] == -1 and (tok[:5] >= 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,many,k", [(700, 4, 5), (700, 5, 5), (700, 9, 5), (700, 650, 600), (40000, 99, 100), (40000, 100, 100),
                                      (40000, 230, 100), (40000, 20000, 100), (40000, 230, 50), (40000, 7000, 6000)])
@pytest.mark.parametrize("p", [1.0, 0.6])
def test_infinities(cuda, p, V, many, k, dtype):  # noqa: F811
    """Fewer infinite logits than top_k, as many, and more: the first k in the order of their ids are kept, and finite
    ones weigh nothing beside them. (0.6 times a number of equal weights that is no whole number of them.)"""
    rng = np.random.default_rng([V, many, k])
    B = 8
    x = _logits(rng, B, V, dtype)
    for b in range(B):
        x[b, rng.permutation(V)[:many]] = math.inf
    seeds, ways = _seeds(rng, B), _full(B, 0.8, k, 0.6 + 1 / 700 if p < 1 else 1.0)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways)
    _check(x, seeds, *ways, None, None, tok, lp)


@pytest.mark.parametrize("B", [1, 5, 76, 120])
def test_first_word_to_the_cluster(cuda, B):  # noqa: F811
    """Rows whose CTAs share the pass and that have nothing to choose from, beside rows that have: the first CTA tells
    the others so as soon as it starts, again and again in a row of calls."""
    rng = np.random.default_rng(B)
    V = 300
    x = _logits(rng, B, V, "f32")
    x[::2] = -math.inf
    seeds, ways = _seeds(rng, B), _full(B, 0.9, 0, 0.8)
    dev = x.to(cuda)
    for _ in range(20):
        tok, lp = _run(cuda, dev, seeds, *ways)
        assert (tok[::2] == -1).all()
    _check(x, seeds, *ways, None, None, tok, lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [8192, 50001])
@pytest.mark.parametrize("k,p", [(40, 1.0), (100, 1.0), (6000, 1.0), (6000, 0.7001), (0, 0.6003)])
def test_minus_zero(cuda, k, p, V, dtype):  # noqa: F811
    """-0 is 0, also as the largest logit of its group: the lowest ids are kept."""
    rng = np.random.default_rng([V, k])
    B = 8
    x = _logits(rng, B, V, dtype)
    x[:4] = -0.0
    x[1, ::2] = 0.0
    x[2, ::300] = 0.0
    x[3, ::7] = -0.5
    x[4:] = x[4:].clamp(max=-0.0)
    allowed = np.ones((1, V), bool)
    allowed[0, 1::5] = False
    states = np.where(np.arange(B) % 4 == 3, 0, ref.FREE).astype(np.int32)
    seeds, ways = _seeds(rng, B), _full(B, 1.1, k, p)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways, allowed, states)
    _check(x, seeds, *ways, allowed, states, tok, lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k,p,min_p", [(2, 1.0, 0.0), (50, 1.0, 0.0), (64, 0.9, 0.0), (50, 1.0, 0.1)])
def test_tokens_of_one_group(cuda, k, p, min_p, dtype):  # noqa: F811
    """All that a row allows lies in one group of 256 ids (ten digits side by side), or in two whose largest logits are
    equal, or nearly so: fewer groups than top_k. Constrained rows, and free ones masked with -inf; infinite logits
    beside finite ones."""
    rng = np.random.default_rng([k, 1])
    V, B = 16640, 96
    x = _logits(rng, B, V, dtype)
    allowed = np.zeros((6, V), bool)
    allowed[0, 512:522] = True
    allowed[1, [600, 611, 900, 901]] = True
    allowed[2, 300:330] = allowed[2, 5000:5042] = True
    allowed[3, [16639]] = True
    allowed[4, 1024:1026] = True
    allowed[5, 256:512:5] = True
    x[:, [600, 900]] = 1.25
    x[:, [611, 901]] = 0.75
    x[:, 300] = x[:, 5000] = 30.0
    x[1::12, 5000] = 30.25
    x[:, 1024] = 1e-39
    x[:, 1025] = 0.0
    x[2::12, 16000] = math.inf
    states = (np.arange(B) % 6).astype(np.int32)
    for b in range(0, B, 4):  # the same by -inf
        x[b, np.nonzero(~allowed[states[b]])[0]] = -math.inf
        states[b] = ref.FREE
    states[2::12] = ref.FREE
    seeds, ways = _seeds(rng, B), _full(B, 1.3, k, p, min_p)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways, allowed, states)
    _check(x, seeds, *ways, allowed, states, tok, lp)
    if k == 50 and min_p == 0:
        assert len(set(tok[states == 0].tolist())) > 2


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("temperature,offset", [(1e-2, 0.0), (1e-3, 0.0), (1e-4, 0.0), (1e-5, 0.0), (1e-6, 0.0), (1e-7, 0.0),
                                                (1.0, 1e4), (1.0, -1e5), (0.7, 1e6), (30.0, 3e7)])
@pytest.mark.parametrize("k,p,min_p", [(0, 1.0, 0.0), (0, 0.7003, 0.0), (50, 0.7003, 0.0), (0, 1.0, 0.5)])
def test_large_over_temperature(cuda, temperature, offset, k, p, min_p, dtype):  # noqa: F811
    """Logits that are many temperatures away from 0: five equal largest ones, and others a few
    temperatures below, which 32 or 16 bits may make equal to them."""
    import torch
    rng = np.random.default_rng([int(1e7 * temperature), int(abs(offset))])
    V, B = 3000, 8
    x = _logits(rng, B, V, "f32") + offset
    x[:, 100::700] = 37.3 + offset
    for b in range(B):
        x[b, rng.integers(0, V, 50)] = torch.from_numpy((37.3 + offset - temperature * rng.random(50) * 6).astype(np.float32))
    x[:, 100::700] = 37.3 + offset
    x = x.to(torch.float32 if dtype == "f32" else torch.bfloat16)
    seeds, ways = _seeds(rng, B), _full(B, temperature, k, p, min_p)
    tok, lp = _run(cuda, x.to(cuda), seeds, *ways)
    _check(x, seeds, *ways, None, None, tok, lp)
    assert (lp <= 1e-5).all()


LEVELS = {
    "halves": (np.arange(400, 269, -1) + 0.45) * 2.0 ** -19,  # 19 bits lose nearly half a unit of each
    "close together": np.linspace(0.33, 0.25, 30),
    "far apart": np.exp(-np.linspace(4.0, 9.0, 30)),
}


# lift: how many temperatures the largest logit is above the end of the bin
@pytest.mark.parametrize("temperature,levels,lift,many", [(0.004, "halves", 1.8, 3900), (0.004, "close together", 1.8, 3000),
                                                          (0.06, "close together", 0.2, 3000), (0.004, "far apart", 1.8, 2500),
                                                          (1e-3, "far apart", 0.5, 2500)])
@pytest.mark.parametrize("k", [0, 4500])
def test_small_weights_of_one_bin(cuda, temperature, levels, lift, many, k):  # noqa: F811
    """Top-p ends among thousands of tokens of small weights that lie within 1/32 of one another. Over many seeds no
    token past the cut is drawn, and of those before it as many as their weight says. Sums of weights in 32 bits are
    within 2^-20 of the whole; chi-square of n degrees of freedom is above n + 6 sqrt(2 n) + 20 with a probability
    below 1e-7."""
    import torch
    rng = np.random.default_rng([many, k])
    V, B = 6000, 60000
    x = np.full(V, -5.0, np.float32)
    at = 300 + rng.permutation(V - 300)[:many]
    x[at] = 1.0 + temperature * np.log(rng.choice(LEVELS[levels], many))
    x[3] = 1.0  # the first group's largest logit is where a bin ends
    x[5000] = 1.0 + lift * temperature
    ok = np.ones(V, bool)
    T = float(np.float32(temperature))
    _, w, _ = ref.kept(x, T, k, 1.0, 0.0, ok)
    p = float(np.float32((w[0] + w[1] + 0.95 * w[2:many + 2].sum()) / w.sum()))
    ids, w, _ = ref.kept(x, T, k, p, 0.0, ok)
    seeds = _seeds(rng, B)
    tok, _ = _run(cuda, torch.from_numpy(x).to(cuda).repeat(B, 1), seeds, *_full(B, temperature, k, p))
    near = 2 + int(2.0 ** -20 * w.sum() / w[-1])  # tokens about the cut that rounding may let in or out
    later, _, _ = ref.kept(x, T, len(ids) + near, 1.0, 0.0, ok)
    got = np.bincount(tok, minlength=V)
    assert got.sum() == got[later].sum(), np.setdiff1d(np.nonzero(got)[0], later)
    part = np.array_split(np.arange(2, max(2, len(ids) - near)), 20)  # in the order of their logits
    want = np.array([w[i].sum() for i in part]) / w.sum() * B
    seen = np.array([got[ids[i]].sum() for i in part])
    chi = ((seen - want) ** 2 / want).sum()
    assert chi < 20 + 6 * math.sqrt(40) + 20, (chi, seen, want)


@pytest.mark.parametrize("seed", range(2))
def test_top_p_next_to_one(cuda, seed):  # noqa: F811
    """Top-p just below 1 and top-k at the end of a bin of 1/32: no rounding lets a token past the first k in."""
    import torch
    rng = np.random.default_rng(seed)
    V, B = 2000, 60000
    x = rng.normal(0, 1, (B, V)).astype(np.float32)
    edge = x[:, :256].max(axis=1) - (rng.integers(20, 50, B) / 32).astype(np.float32)
    k = np.maximum(12, (x > edge[:, None]).sum(axis=1) + rng.integers(-1, 2, B)).astype(np.int32)
    p = (1 - 2.0 ** -24 * rng.integers(1, 4, B)).astype(np.float32)
    ways = _full(B, 4.0)
    tok, _ = _run(cuda, torch.from_numpy(x).to(cuda), _seeds(rng, B), ways[0], k, p)
    drawn = x[np.arange(B), tok][:, None]
    before = (x > drawn).sum(axis=1) + ((x == drawn) & (np.arange(V) < tok[:, None])).sum(axis=1)
    assert (before < k).all(), int((before >= k).sum())


def _noise(seed, n):
    """ref.noise of an array of numbers."""
    with np.errstate(over="ignore"):
        z = np.uint64(seed % 2 ** 64) + (n.astype(np.uint64) + np.uint64(1)) * np.uint64(0x9E3779B97F4A7C15)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
        z ^= z >> np.uint64(31)
    return -np.log(-np.log((2 * (z >> np.uint64(41)).astype(np.float64) + 1) / 2 ** 24))


@pytest.mark.parametrize("k,p", [(0, 0.9), (0, 0.3), (20_000_000, 0.95), (17_000_000, 1.0)])
def test_equal_logits_of_a_huge_vocabulary(cuda, k, p):  # noqa: F811
    """25 million equal logits: weights of more than 2^24 tokens. A token is one of the first k, or of top-p of them;
    groups weigh the same, so the draw is the largest noise. (The two largest are about 1 apart; that the rounding of 32
    bits decides between them is let pass for one row.)"""
    import torch
    V, B = 3 << 23, 24
    x = torch.full((B, V), 0.75, dtype=torch.bfloat16, device=cuda)
    seeds = np.random.default_rng(7).integers(-2 ** 63, 2 ** 63 - 1, B)
    tok, lp = _run(cuda, x, seeds, *_full(B, 1.0, k, p))
    n = math.ceil(float(np.float32(p)) * (k or V)) if p < 1 else k
    groups = np.arange((n + 255) // 256)
    same = 0
    for b in range(B):
        group = int(np.argmax(np.log(np.minimum(256, n - 256 * groups)) + _noise(int(seeds[b]), groups + 2 ** 31)))
        ids = np.arange(256 * group, min(n, 256 * group + 256))
        same += int(ids[np.argmax(_noise(int(seeds[b]), ids))]) == tok[b]
    assert same >= B - 1 and np.abs(lp + math.log(V)).max() < 1e-4
