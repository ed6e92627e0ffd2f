"""trie_sample against the definition in 64 bits.

Tokens have to be equal, except where the 64-bit decision that made the token
(which group, which token, where top-p or min-p cuts) is closer than 2e-5 to
the other way: scores are sums of a logit (|x| <= 60 here), a logarithm and
noise below 17 in 32 bits, each within 2^-24 of values below 64, and weights
are relative to 2^-20 (an exponent up to 30 rounded to 24 bits, exp2 to 2 units).
Log-probabilities are within 1e-5 + 2^-22 |z|."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as ref
from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu
MARGIN = 2e-5


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_12574_gb300 import _build
    _build.build()
    return torch.device("cuda:0")


def _up(dev, a):
    import torch
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)


def _check(x, seeds, temp, k, p, min_p, allowed, states, tokens, logprobs):
    """x: CPU tensor; the others numpy."""
    B, V = x.shape
    x = x.float().numpy()
    exact = 0
    for b in range(B):
        ok = ref.allowed_row(allowed, ref.FREE if states is None else int(states[b]), V)
        t, lp, margin = ref.sample(x[b], int(seeds[b]), 1.0 if temp is None else float(temp[b]),
                                   0 if k is None else int(k[b]), 1.0 if p is None else float(p[b]),
                                   0.0 if min_p is None else float(min_p[b]), ok)
        if tokens[b] != t:
            assert margin < MARGIN, (b, tokens[b], t, margin)
            continue
        exact += 1
        if t < 0:
            assert logprobs[b] == -math.inf
        else:
            assert abs(logprobs[b] - lp) <= 1e-5 + 2.0 ** -22 * abs(lp), (b, logprobs[b], lp)
    assert exact >= B - max(1, B // 50)


def _run(dev, x, seeds, temp=None, k=None, p=None, min_p=None, allowed=None, states=None):
    tok, lp = T.trie_sample(x, _up(dev, seeds), _up(dev, temp), _up(dev, k), _up(dev, p), _up(dev, min_p),
                            None if allowed is None else _up(dev, ref.pack(allowed)), _up(dev, states))
    return tok.cpu().numpy(), lp.cpu().numpy()


def _logits(rng, B, V, dtype, peaks=20):
    import torch
    x = rng.normal(0, 2, (B, V))
    for b in range(B):
        x[b, rng.integers(0, V, peaks)] += rng.random(peaks) * rng.random() * 14
    return torch.from_numpy(x.astype(np.float32)).to(torch.float32 if dtype == "f32" else torch.bfloat16)


def _ways(rng, B, V):
    temp = rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 2.0], B).astype(np.float32)
    k = rng.choice([0, 0, 1, 5, 50, 700, 3000, V, V + 7, -2], B).astype(np.int32)
    p = rng.choice([1.0, 1.0, 0.9, 0.5, 0.99, 0.0, 1.5], B).astype(np.float32)
    m = rng.choice([0.0, 0.0, 0.02, 0.3, 1.0], B).astype(np.float32)
    return temp, k, p, m


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B", [(2, 8), (33, 16), (255, 16), (256, 16), (257, 16), (1001, 24), (8192, 24), (32000, 24),
                                 (50021, 16), (152064, 12), (262144, 6)])
def test_sample(cuda, V, B, dtype):
    rng = np.random.default_rng([V, B])
    x = _logits(rng, B, V, dtype)
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp, k, p, m = _ways(rng, B, V)
    tok, lp = _run(cuda, x.to(cuda), seeds, temp, k, p, m)
    _check(x, seeds, temp, k, p, m, None, None, tok, lp)
    tok, lp = _run(cuda, x.to(cuda), seeds)
    _check(x, seeds, None, None, None, None, None, None, tok, lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [2, 63, 300, 5001, 50021])
def test_sample_grammar(cuda, V, dtype):
    rng = np.random.default_rng(V)
    B, rows = 24, 9
    x = _logits(rng, B, V, dtype)
    allowed = rng.random((rows, V)) < np.array([0.0, 1 / V, 0.001, 0.01, 0.1, 0.5, 0.9, 1.0, 0.02])[:, None]
    allowed[0] = False
    states = rng.integers(-3, rows + 1, B).astype(np.int32)
    states[:5] = [0, ref.FREE, ref.FINISHED, ref.DEAD, rows]
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp, k, p, m = _ways(rng, B, V)
    tok, lp = _run(cuda, x.to(cuda), seeds, temp, k, p, m, allowed, states)
    _check(x, seeds, temp, k, p, m, allowed, states, tok, lp)
    assert tok[0] == -1 and tok[2] == tok[3] == tok[4] == V - 1


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [300, 40000])
def test_sample_ties(cuda, V, dtype):
    """Logits of few distinct values: which of the equal ones top-k and top-p keep (the lowest ids). Top-p here is
    taken so that its cut is never at a boundary (0.37 of counts that are whole numbers of equal weights is checked
    by the margin)."""
    import torch
    rng = np.random.default_rng(V)
    B = 30
    values = np.array([2.0, 1.5, 0.0, -0.0, -1.0, -4.0])
    x = torch.from_numpy(values[rng.integers(0, 6, (B, V))].astype(np.float32)).to(
        torch.float32 if dtype == "f32" else torch.bfloat16)
    x[0] = 1.25
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp = np.full(B, 1.0, np.float32)
    temp[::5] = 0
    k = rng.choice([0, 1, 3, 64, 65, 1024, 1025, 2049, V // 2], B).astype(np.int32)
    p = rng.choice([1.0, 0.37, 0.83], B).astype(np.float32)
    tok, lp = _run(cuda, x.to(cuda), seeds, temp, k, p)
    _check(x, seeds, temp, k, p, None, None, None, tok, lp)


@pytest.mark.parametrize("k,p,min_p", [(2048, 1.0, 0.0), (2049, 0.95, 0.0), (5000, 0.5, 0.01), (0, 0.999, 0.0),
                                       (0, 0.9999, 0.001), (1024, 0.7, 0.0), (1025, 0.7, 0.0)])
def test_sample_broad(cuda, k, p, min_p):
    """Kept sets that no short list holds."""
    rng = np.random.default_rng(k + 1)
    V, B = 70001, 8
    x = _logits(rng, B, V, "f32", peaks=1)
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    full = [np.full(B, v, t) for v, t in ((1.5, np.float32), (k, np.int32), (p, np.float32), (min_p, np.float32))]
    tok, lp = _run(cuda, x.to(cuda), seeds, *full)
    _check(x, seeds, *full, None, None, tok, lp)


def test_sample_special_values(cuda):
    """NaN, infinities, the lowest value, rows of nothing."""
    import torch
    V, B = 600, 9
    rng = np.random.default_rng(0)
    x = _logits(rng, B, V, "f32")
    x[0] = math.nan
    x[1] = -math.inf
    x[2, 100] = math.inf
    x[3, [5, 300, 599]] = math.inf
    x[4, ::2] = math.nan
    x[5] = -3.4028234e38
    x[6, :599] = -math.inf
    x[7] = -math.inf
    x[7, 13] = -3.4028234e38
    x[8, 10] = 3.4028234e38
    seeds = np.arange(B) * 77 - 3
    for k, p, m in ((0, 1.0, 0.0), (20, 0.9, 0.0), (0, 0.9, 0.1)):
        full = [np.full(B, v, t) for v, t in ((1.0, np.float32), (k, np.int32), (p, np.float32), (m, np.float32))]
        if p < 1:
            x5 = x[5].clone()
            x[5, 300:] = -math.inf   # 300 equal weights: no cut at a boundary for 0.9 would need a whole number
            x[5, 299] = -math.inf
        tok, lp = _run(cuda, x.to(cuda), seeds, *full)
        _check(x, seeds, *full, None, None, tok, lp)
        assert tok[0] == tok[1] == -1 and tok[2] == 100 and tok[3] in (5, 300, 599) and tok[6] == 599 and tok[7] == 13
        if p < 1:
            x[5] = x5


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 13), (5, 2), (8, 8), (7, 1)])
def test_sample_strides(cuda, offset, pad, dtype):
    """Rows at any distance and any alignment; the logits are not written."""
    import torch
    rng = np.random.default_rng([offset, pad])
    V, B = 3333, 12
    x = _logits(rng, B, V, dtype)
    buf = torch.full((B * (V + pad) + offset,), math.inf, dtype=x.dtype, device=cuda)
    view = buf[offset:].view(B, V + pad)[:, :V]
    view.copy_(x)
    before = buf.clone()
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp, k, p, m = _ways(rng, B, V)
    tok, lp = _run(cuda, view, seeds, temp, k, p, m)
    _check(x, seeds, temp, k, p, m, None, None, tok, lp)
    assert torch.equal(buf, before)


@pytest.mark.parametrize("k,p,min_p", [(0, 1.0, 0.0), (9, 1.0, 0.0), (0, 0.8, 0.0), (0, 1.0, 0.05)])
def test_sample_frequencies(cuda, k, p, min_p):
    """How often each token is drawn over many seeds, against its probability: chi-square of n degrees of freedom
    is above n + 6 sqrt(2 n) + 20 with a probability below 1e-7."""
    import torch
    rng = np.random.default_rng(3)
    V, B = 700, 60000
    x = rng.normal(0, 1.5, V).astype(np.float32)
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    full = [np.full(B, v, t) for v, t in ((0.9, np.float32), (k, np.int32), (p, np.float32), (min_p, np.float32))]
    tok, _ = _run(cuda, torch.from_numpy(x).to(cuda).repeat(B, 1), seeds, *full)
    ids, w, _ = ref.kept(x, 0.9, k, p, min_p, np.ones(V, bool))
    want = np.zeros(V)
    want[ids] = w / w.sum() * B
    got = np.bincount(tok, minlength=V)
    assert got[want == 0].sum() == 0
    n = len(ids) - 1
    chi = ((got - want)[ids] ** 2 / want[ids]).sum()
    assert chi < n + 6 * math.sqrt(2 * n) + 20, (chi, n)


def test_sample_repeats_and_graphs(cuda):
    """The same call twice gives the same bits; a captured call replayed on new logits gives theirs; the
    caller's outputs, workspace and stream are used."""
    import torch
    rng = np.random.default_rng(9)
    V, B = 40000, 10
    a, c = _logits(rng, B, V, "bf16"), _logits(rng, B, V, "bf16")
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp, k, p, m = _ways(rng, B, V)
    dev = [_up(cuda, v) for v in (seeds, temp, k, p, m)]
    x = a.to(cuda)
    tok, lp = T.trie_sample(x, *dev)
    tok2, lp2 = torch.full_like(tok, 9), torch.full_like(lp, 9)
    work = torch.zeros(T.trie_sample_workspace(B, V) // 4 + 2, dtype=torch.int32, device=cuda)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = T.trie_sample(x, *dev, tokens=tok2, logprobs=lp2, workspace=work, stream=side)
    side.synchronize()
    assert got[0] is tok2 and torch.equal(tok, tok2) and torch.equal(lp, lp2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.trie_sample(x, *dev, tokens=tok2, logprobs=lp2, workspace=work)
    x.copy_(c)
    graph.replay()
    _check(c, seeds, temp, k, p, m, None, None, tok2.cpu().numpy(), lp2.cpu().numpy())


def test_sample_refusals(cuda):
    import torch
    x = torch.zeros(2, 100, device=cuda)
    s = torch.zeros(2, dtype=torch.int64, device=cuda)
    i = torch.zeros(2, dtype=torch.int32, device=cuda)
    m = torch.zeros(3, 4, dtype=torch.int32, device=cuda)
    bad = [
        (ValueError, lambda: T.trie_sample(x, None)), (ValueError, lambda: T.trie_sample(x.t(), s)),
        (TypeError, lambda: T.trie_sample(x, i)), (ValueError, lambda: T.trie_sample(x, s[:1])),
        (TypeError, lambda: T.trie_sample(x.cpu(), s)), (TypeError, lambda: T.trie_sample(x, s, top_k=s)),
        (TypeError, lambda: T.trie_sample(x, s, temperature=i)), (ValueError, lambda: T.trie_sample(x, s, mask=m)),
        (ValueError, lambda: T.trie_sample(x, s, tokens=i[:1])), (TypeError, lambda: T.trie_sample(x, s, tokens=s)),
        (ValueError, lambda: T.trie_sample(x, s, workspace=i[:1])), (ValueError, lambda: T.trie_sample_workspace(-1, 5)),
        (ValueError, lambda: T.trie_sample(x, s, mask=m, states=i[:1])),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    work = torch.zeros(64, device=cuda)
    lib, p = T.load_library(), x.data_ptr()
    args = [p, 0, 100, 2, 100, s.data_ptr()] + [None] * 5 + [0, None, work.data_ptr(), i.data_ptr(), None, None]
    assert lib.trie_sample(*args) == T.TRIE_OK
    torch.cuda.synchronize()
    for at, value in [(0, None), (0, p + 1), (1, 2), (2, 99), (3, -1), (3, 65536), (4, 1), (5, None), (10, p), (12, p),
                      (13, None), (13, work.data_ptr() + 4), (14, None)]:
        wrong = list(args)
        wrong[at] = value
        assert lib.trie_sample(*wrong) == T.TRIE_EINVAL, (at, value)
    empty, _ = T.trie_sample(x[:0], s[:0])
    assert empty.numel() == 0
