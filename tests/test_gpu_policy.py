"""The policy loss and its gradient against the definition in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as lref
import rows_ref as ref
from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device")
    T.load_library()
    return torch.device("cuda:0")


def _type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _logits(rng, B, V, dtype):
    import torch
    x = rng.normal(0, 2, (B, V))
    x[np.arange(B)[:, None], rng.integers(0, V, (B, 8))] += rng.uniform(0, 10, (B, 8))
    return torch.from_numpy(x.astype(np.float32)).to(_type(dtype))


def _rows(rng, logits, temperature, allowed=None, states=None, padding=True):
    """Tokens of each row among its allowed ones, old log-probabilities that put the ratio well off the clips'
    borders, references, advantages, weights; as numpy arrays of 32 bits."""
    x = logits.double().numpy()
    B, V = x.shape
    ok = np.stack([lref.allowed_row(allowed, lref.FREE if states is None else int(states[b]), V) for b in range(B)])
    tokens, old, refs = np.full(B, -1, np.int32), np.zeros(B, np.float32), np.zeros(B, np.float32)
    for b in range(B):
        ids = np.flatnonzero(ok[b])
        if not len(ids):
            tokens[b] = rng.integers(0, V)
            continue
        tokens[b] = ids[x[b, ids].argmax()] if b % 3 == 0 else rng.choice(ids)
        _, lp, _, _ = ref.policy(x[b], tokens[b], 0, 0, None, 1, temperature[b], 0.2, 0.3, 0, ok[b])
        lp = lp if math.isfinite(lp) else 0.0
        old[b] = lp + [-0.6, -0.1, 0.0, 0.1, 0.5][b % 5]
        refs[b] = lp + rng.normal(0, 0.5)
    weights = rng.uniform(0.5, 2, B).astype(np.float32) / B
    if padding and B > 4:
        weights[4] = 0
        tokens[3] = [-1, V, 2 ** 31 - 1, -2 ** 31][B % 4]
    A = rng.normal(0, 1, B).astype(np.float32)
    return ok, tokens, old, refs, A, weights


def _check(x, got, grad, ok, tokens, old, refs, A, weights, temperature, low, high, kl):
    """Errors of 32 bits, u = 2^-24 each: an exponent's argument a (in bits) has three roundings, its value 4 u
    (the function) more; sums of V values 32 at a time and in trees; lp a logarithm and two roundings of its size."""
    losses, logprobs = (t.double().cpu().numpy() for t in got)
    B, V = x.shape
    half = 2.0 ** -8 if grad is not None and str(grad.dtype) == "torch.bfloat16" else U
    g = None if grad is None else grad.double().cpu().numpy()
    for b in range(B):
        r = None if refs is None else float(refs[b])
        loss, lp, slope, want = ref.policy(x[b], int(tokens[b]), float(old[b]), float(A[b]), r, float(weights[b]),
                                           float(temperature[b]), low, high, kl, ok[b])
        if not math.isfinite(lp):
            for value, other in ((lp, logprobs[b]), (loss, losses[b])):
                assert value == other or (math.isnan(value) and math.isnan(other)), (b, value, other)
            if g is not None:
                assert np.array_equal(g[b], want, equal_nan=True) or (np.isnan(want[ok[b]]).all() and np.isnan(g[b][ok[b]]).all()
                                                                      and (g[b][~ok[b]] == 0).all()), b
            continue
        off = (60 + 4 * math.log2(V) + V / 128) * U + 4 * U * abs(lp)
        assert abs(logprobs[b] - lp) <= off, (b, logprobs[b], lp)
        rho, w = math.exp(lp - float(old[b])), float(weights[b])
        d = 0.0 if r is None else r - lp
        reach = w * (abs(rho * A[b]) + (kl * (math.exp(d) + 1) if r is not None else 0))
        assert abs(losses[b] - loss) <= reach * (off + (8 + abs(lp - old[b]) + abs(d)) * U) + kl * w * 8 * U * abs(d), (b, losses[b], loss)
        if g is None:
            continue
        assert (g[b][~ok[b]] == 0).all()
        T_ = temperature[b] if temperature[b] > 0 else 1.0
        bits = np.where(want != 0, np.abs(np.minimum(x[b] - x[b][ok[b]].max(), 0)) / T_ * 1.45, 0)
        at = int(tokens[b])
        rel = off + (20 + 4 * bits) * U
        bound = np.abs(want) * (rel + half) + reach / T_ * (off + 16 * U) * np.where(slope != 0, np.abs(want / (slope / T_ or 1)), 0) + 2.0 ** -133
        bound[at] += reach / T_ * off  # 1 - p
        worst = (np.abs(g[b] - want) - bound).max()
        assert worst <= 0, (b, worst, slope)


def _run(cuda, logits, tokens, old, refs, A, weights, temperature, grad, **more):
    import torch
    put = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(cuda)  # noqa: E731
    return T.trie_policy_loss(logits, put(tokens), put(old), put(A), ref_logprobs=put(refs), weights=put(weights),
                              temperature=put(temperature), grad=grad, **more)


@pytest.mark.parametrize("with_grad", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(1, 2), (3, 3), (1, 7), (5, 31), (9, 33), (17, 1000), (40, 4097), (8, 32000), (6, 50021),
                                 (2, 262144), (1, 700001)])
def test_policy(cuda, B, V, dtype, with_grad):
    import torch
    rng = np.random.default_rng([B, V])
    logits = _logits(rng, B, V, dtype)
    temperature = rng.choice([0.5, 1.0, 1.3, 0.0], B).astype(np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, temperature)
    x = logits.double().numpy()
    there = logits.to(cuda)
    grad = torch.full_like(there, math.nan) if with_grad else None
    for low, high, kl in ((0.2, 0.3, 0.0), (0.2, 0.3, 0.1)):
        got = _run(cuda, there, tokens, old, refs, A, weights, temperature, grad, clip=(low, high), kl=kl)
        _check(x, got, grad, ok, tokens, old, refs, A, weights, temperature, low, high, kl)
    assert torch.equal(there.cpu(), logits)


def test_policy_defaults(cuda):
    """Without reference, weights and temperatures: no KL term, 1 and 1."""
    import torch
    rng = np.random.default_rng(3)
    B, V = 12, 500
    logits = _logits(rng, B, V, "f32")
    one = np.ones(B, np.float32)
    ok, tokens, old, refs, A, _ = _rows(rng, logits, one, padding=False)
    grad = torch.empty(B, V, device=cuda)
    got = _run(cuda, logits.to(cuda), tokens, old, None, A, None, None, grad, kl=0.3)
    _check(logits.double().numpy(), got, grad, ok, tokens, old, None, A, one, one, 0.2, 0.2, 0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(20, 65), (33, 1000), (24, 8191), (16, 50021)])
def test_policy_grammar(cuda, B, V, dtype):
    """Rows that allow nothing, one token, few, half, all; free, finished and dead rows; NaN, infinities and the
    type's ends where no token is allowed; bits of the mask behind V."""
    import torch
    rng = np.random.default_rng([B, V, 1])
    allowed = rng.random((8, V)) < np.array([0, 0, 0.01, 0.5, 1.0, 30 / V, 2 / V, 0.9])[:, None]
    allowed[1, V // 2] = True
    allowed[5, V - 1] = True
    states = np.array([0, 1, 2, 3, 4, 5, 6, 7, -1, -2, -3, 8, 2 ** 31 - 1, -2 ** 31, 3, 5] * 3, np.int32)[:B]
    packed = lref.pack(allowed)
    if V % 32:
        packed[:, -1] |= np.int32(-1) << np.int32(V % 32)
    logits = _logits(rng, B, V, dtype)
    temperature = rng.choice([0.7, 1.0], B).astype(np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, temperature, allowed, states)
    for value in (math.nan, math.inf, -math.inf, torch.finfo(logits.dtype).max, torch.finfo(logits.dtype).min):
        wild = torch.where(torch.from_numpy(ok), logits, torch.full_like(logits, value))
        grad = torch.full_like(wild, math.nan, device=cuda)
        got = _run(cuda, wild.to(cuda), tokens, old, refs, A, weights, temperature, grad, kl=0.05,
                   mask=torch.from_numpy(packed).to(cuda), states=torch.from_numpy(states).to(cuda))
        _check(wild.double().numpy(), got, grad, ok, tokens, old, refs, A, weights, temperature, 0.2, 0.2, 0.05)
    tokens = rng.integers(0, V, B).astype(np.int32)  # most are not allowed
    got = _run(cuda, logits.to(cuda), tokens, old, refs, A, weights, temperature, grad, kl=0.05,
               mask=torch.from_numpy(packed).to(cuda), states=torch.from_numpy(states).to(cuda))
    bad = ~ok[np.arange(B), tokens]
    assert bool((got[1].cpu()[torch.from_numpy(bad)] == -math.inf).all()) and bool((got[0].cpu()[torch.from_numpy(bad)] == 0).all())
    assert bool((grad.cpu()[torch.from_numpy(bad)] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,in_place", [(2049, False), (4999, True), (36000, False)])
def test_policy_numbers_of_tokens(cuda, V, in_place, dtype):
    """Rows of few to several hundred allowed tokens: anywhere, in one piece at either end, 1,024 apart, and every
    other one, which are all of some words."""
    import torch
    rng = np.random.default_rng([V, 7])
    rows = []
    for n in (1, 31, 32, 33, 64, 65, 127, 128, 129, 300):
        for ids in (rng.choice(V, n, replace=False), np.arange(n), np.arange(V - n, V), (np.arange(n) * 1024 + 5) % V, 2 * np.arange(n)):
            row = np.zeros(V, bool)
            row[ids] = True
            rows.append(row)
    allowed = np.stack(rows)
    B = len(rows) + 110  # enough for a CTA a row
    states = np.concatenate([np.arange(len(rows)), rng.integers(-3, len(rows), 110)]).astype(np.int32)
    logits = _logits(rng, B, V, dtype)
    temperature = rng.choice([0.7, 1.0], B).astype(np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, temperature, allowed, states)
    there = logits.to(cuda)
    grad = there if in_place else torch.full_like(there, math.nan)
    got = _run(cuda, there, tokens, old, refs, A, weights, temperature, grad, kl=0.05,
               mask=torch.from_numpy(lref.pack(allowed)).to(cuda), states=torch.from_numpy(states).to(cuda))
    _check(logits.double().numpy(), got, grad, ok, tokens, old, refs, A, weights, temperature, 0.2, 0.2, 0.05)


@pytest.mark.parametrize("with_grad", [False, True])
@pytest.mark.parametrize("B,V,dtype", [(40, 100001, "bf16"), (60, 160001, "bf16"), (40, 240003, "bf16"), (60, 110001, "f32"),
                                       (30, 190001, "f32"), (20, 220001, "f32")])
def test_policy_shares(cuda, B, V, dtype, with_grad):
    """Rows shared by 4, 6, 8, 10 and 16 CTAs, more of them than are at work at once, some constrained."""
    import torch
    rng = np.random.default_rng([B, V, 2])
    allowed = rng.random((4, V)) < np.array([3 / V, 40 / V, 900 / V, 0.5])[:, None]
    allowed[:, V // 3] = True
    states = rng.choice([0, 1, 2, 3, -3, -3, -3, -2], B).astype(np.int32)
    logits = _logits(rng, B, V, dtype)
    temperature = rng.choice([0.7, 1.0], B).astype(np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, temperature, allowed, states)
    there = logits.to(cuda)
    grad = torch.full_like(there, math.nan) if with_grad else None
    got = _run(cuda, there, tokens, old, refs, A, weights, temperature, grad, kl=0.05,
               mask=torch.from_numpy(lref.pack(allowed)).to(cuda), states=torch.from_numpy(states).to(cuda))
    _check(logits.double().numpy(), got, grad, ok, tokens, old, refs, A, weights, temperature, 0.2, 0.2, 0.05)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 5003, 300001])
def test_policy_special_values(cuda, V, dtype):
    """Rows with a NaN, an infinity, only -inf, one token of any weight, the type's ends; weight 0 beside a NaN."""
    import torch
    rng = np.random.default_rng(V)
    B = 12
    logits = _logits(rng, B, V, dtype)
    logits[0, V - 3] = math.nan
    logits[1, 5] = math.inf
    logits[2] = -math.inf
    logits[3] = -math.inf
    logits[3, 7] = -5.0
    logits[4, 11] = math.nan
    logits[5, 1::2] = -math.inf
    logits[6] = 0
    logits[7] = torch.finfo(logits.dtype).min
    logits[8, 9] = torch.finfo(logits.dtype).max
    logits[9, :] = -math.inf
    logits[9, 3] = torch.finfo(logits.dtype).min
    logits[10, 0] = math.nan
    tokens = np.array([1, 6, 3, 7, 2, 4, 39, 0, 9, 3, 0, 13], np.int32)
    one = np.ones(B, np.float32)
    A, weights = rng.normal(0, 1, B).astype(np.float32), np.full(B, 0.5, np.float32)
    weights[4] = 0
    ok = np.ones((B, V), bool)
    x = logits.double().numpy()
    old = np.zeros(B, np.float32)
    for b in (5, 6, 7, 11):
        old[b] = ref.policy(x[b], int(tokens[b]), 0, 0, None, 1, 1.0, 0.2, 0.2, 0, ok[b])[1] + 0.1
    refs = old - np.float32(0.2)
    grad = torch.full_like(logits, 7.0, device=cuda)
    got = _run(cuda, logits.to(cuda), tokens, old, refs, A, weights, one, grad, kl=0.05)
    losses, lp = got[0].cpu(), got[1].cpu()
    assert bool(losses[[0, 1, 10]].isnan().all()) and bool(lp[[0, 1, 10]].isnan().all())
    assert bool(grad[[0, 1, 10]].isnan().all())
    assert losses[4] == 0 and bool((grad[4] == 0).all())
    keep = [2, 3, 5, 6, 7, 8, 9, 11]
    _check(x[keep], (got[0][keep], got[1][keep]), grad[keep], ok[keep], tokens[keep], old[keep], refs[keep], A[keep], weights[keep],
           one[keep], 0.2, 0.2, 0.05)


@pytest.mark.parametrize("temperature", [math.nan, -1.0, 0.0, 1e-45, 1e-38, 1e-3, 1e3, 3e38, math.inf])
def test_policy_temperatures(cuda, temperature):
    import torch
    rng = np.random.default_rng(11)
    B, V = 10, 300
    logits = _logits(rng, B, V, "f32")
    t = np.full(B, temperature, np.float32)
    given = np.full(B, temperature if temperature > 0 else 1.0)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, given)
    grad = torch.empty(B, V, device=cuda)
    got = _run(cuda, logits.to(cuda), tokens, old, refs, A, weights, t, grad)
    if temperature < 1e-30 and temperature > 0:  # probabilities are 0 or 1
        assert not bool(got[0].isnan().any()) and not bool(grad.isnan().any())
        return
    _check(logits.double().numpy(), got, grad, ok, tokens, old, refs, A, weights, np.minimum(given, 3.4028234e38), 0.2, 0.2, 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1001, 40000])
@pytest.mark.parametrize("offset,pad,g_offset,g_pad", [(0, 0, 0, 0), (1, 0, 1, 0), (1, 0, 2, 3), (3, 13, 3, 13), (4, 64, 0, 8), (8, 23, 7, 1)])
def test_policy_strides(cuda, offset, pad, g_offset, g_pad, V, dtype):
    """Rows at any distance and alignment, of the logits and of the gradient; what lies between is not written."""
    import torch
    rng = np.random.default_rng([offset, pad])
    B = 7
    logits = _logits(rng, B, V, dtype)
    one = np.ones(B, np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, logits, one)

    def placed(offset, pad):
        buf = torch.full((B * (V + pad) + offset + 8,), 7.0, dtype=logits.dtype, device=cuda)
        return buf, buf[offset:offset + B * (V + pad)].view(B, V + pad)
    _, x = placed(offset, pad)
    x[:, :V] = logits.to(cuda)
    buf, g = placed(g_offset, g_pad)
    got = _run(cuda, x[:, :V], tokens, old, refs, A, weights, one, g[:, :V], kl=0.05)
    _check(logits.double().numpy(), got, g[:, :V], ok, tokens, old, refs, A, weights, one, 0.2, 0.2, 0.05)
    assert bool((g[:, V:] == 7).all()) and bool((buf[:g_offset] == 7).all()) and bool((buf[-8:] == 7).all())
    # in place
    apart = g[:, :V].clone()
    again = _run(cuda, x[:, :V], tokens, old, refs, A, weights, one, x[:, :V], kl=0.05)
    assert torch.equal(x[:, :V], apart) and torch.equal(again[0], got[0]) and torch.equal(again[1], got[1])
    assert bool((x[:, V:] == 7).all())


@pytest.mark.parametrize("dtype,V", [("bf16", 3100), ("bf16", 30011), ("f32", 70001), ("f32", 280001), ("bf16", 700003)])
@pytest.mark.parametrize("in_place", [False, True])
def test_policy_many_rows(cuda, dtype, V, in_place):
    """More rows than are at work at a time, free rows and rows that allow few and many tokens one after the other."""
    import torch
    rng = np.random.default_rng([V, in_place])
    B = 3000 if V < 4000 else 700 if V < 100000 else 40
    allowed = np.zeros((6, V), bool)
    allowed[0, rng.choice(V, 7, replace=False)] = True
    allowed[1, rng.choice(V, 500, replace=False)] = True
    allowed[2, rng.choice(V, 3000, replace=False)] = True
    allowed[3] = rng.random(V) < 0.7
    allowed[4, V - 9:] = True
    allowed[5, :3] = True
    states = rng.choice([-3, -3, 0, 1, 2, 3, 4, 5, -1], B).astype(np.int32)
    logits = (torch.from_numpy(rng.normal(0, 2, (64 if B > 64 else B, V)).astype(np.float32)).to(_type(dtype)).to(cuda))
    logits = logits.repeat((B + len(logits) - 1) // len(logits), 1)[:B].contiguous()
    ok = torch.from_numpy(np.stack([lref.allowed_row(allowed, s, V) for s in range(-3, 6)])).to(cuda)
    ok = ok[torch.from_numpy(states).to(cuda).long() + 3]
    g = torch.Generator(device=cuda)
    g.manual_seed(V)
    tokens = torch.where(ok, torch.rand(B, V, generator=g, device=cuda), -1.0).argmax(dim=1)
    A, weights = torch.randn(B, generator=g, device=cuda), torch.rand(B, generator=g, device=cuda) + 0.5
    # in 64 bits
    y = torch.where(ok, logits.double(), -math.inf)
    y = y - torch.logsumexp(y, dim=1, keepdim=True)
    lp = y.gather(1, tokens[:, None])[:, 0]
    old = (lp - 0.1).float()  # rho = exp(0.1): within the clips
    rho = torch.exp(lp - old.double())
    want = torch.exp(y) * (weights * A * rho)[:, None]
    want.scatter_add_(1, tokens[:, None], -(weights * A * rho)[:, None])
    grad = logits if in_place else torch.full_like(logits, math.nan)
    losses, logprobs = T.trie_policy_loss(logits, tokens.int(), old, A, weights=weights, clip=(0.5, 0.5), grad=grad,
                                          mask=torch.from_numpy(lref.pack(allowed)).to(cuda), states=torch.from_numpy(states).to(cuda))
    # the bounds of _check for |lp| < 20 and |x| < 40
    off = (60 + 4 * math.log2(V) + V / 128 + 80) * U
    assert float((logprobs - lp).abs().max()) <= off
    assert float((losses + weights * A * rho).abs().max()) <= float((weights * A * rho).abs().max()) * (off + 16 * U)
    assert bool((grad[~ok] == 0).all())
    half = 2.0 ** -8 if dtype == "bf16" else U
    reach = (weights * A * rho).abs()[:, None].double()
    bound = want.abs() * (2 * off + 260 * U + half) + 2.0 ** -133
    bound.scatter_add_(1, tokens[:, None], reach * off)
    assert float(((grad.double() - want).abs() - bound).max()) <= 0


def test_policy_far_rows(cuda):
    """Logits and gradients more than 2^31 values behind the first."""
    import torch
    B, V = 16500, 131072
    rng = np.random.default_rng(1)
    n = 24
    logits = torch.zeros(B, V, dtype=torch.bfloat16, device=cuda)
    tail = _logits(rng, n, V, "bf16")
    logits[-n:] = tail.to(cuda)
    one = np.ones(n, np.float32)
    ok, tokens, old, refs, A, weights = _rows(rng, tail, one)
    put = lambda a, fill: torch.cat([torch.full((B - n,), fill, dtype=torch.from_numpy(a).dtype), torch.from_numpy(a)]).to(cuda)  # noqa: E731
    grad = torch.full_like(logits, math.nan)
    losses, logprobs = T.trie_policy_loss(logits, put(tokens, 7), put(old, -math.log(V)), put(A, 0.0), ref_logprobs=put(refs, -math.log(V)),
                                          weights=put(weights, 1.0), kl=0.05, grad=grad)
    _check(tail.double().numpy(), (losses[-n:], logprobs[-n:]), grad[-n:], ok, tokens, old, refs, A, weights, one, 0.2, 0.2, 0.05)
    assert float((logprobs[:-n] + math.log(V)).abs().max()) <= 1e-4
    assert bool(grad[::97].isfinite().all())


def test_policy_repeats_and_graphs(cuda):
    """The same bits every time, on a side stream and replayed from a graph on new logits; given outputs."""
    import torch
    rng = np.random.default_rng(4)
    B, V = 50, 30011
    one = np.ones(B, np.float32)
    logits, other = _logits(rng, B, V, "bf16"), _logits(rng, B, V, "bf16")
    ok, tokens, old, refs, A, weights = _rows(rng, logits, one)
    dev = {k: torch.from_numpy(v).to(cuda) for k, v in dict(t=tokens, o=old, a=A, w=weights).items()}
    x = logits.to(cuda)
    grads = [torch.empty_like(x) for _ in range(3)]

    def loss(grad, stream=None, **out):
        return T.trie_policy_loss(x, dev["t"], dev["o"], dev["a"], weights=dev["w"], grad=grad, stream=stream, **out)
    first = loss(grads[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = loss(grads[1], side)
    side.synchronize()
    assert torch.equal(grads[0], grads[1]) and torch.equal(first[0], second[0]) and torch.equal(first[1], second[1])
    out = dict(losses=torch.empty(B, device=cuda), logprobs=torch.empty(B, device=cuda))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss(grads[2], **out)
    x.copy_(other)
    graph.replay()
    want = loss(grads[1])
    assert torch.equal(grads[1], grads[2]) and torch.equal(out["losses"], want[0]) and torch.equal(out["logprobs"], want[1])


def test_policy_refusals(cuda):
    import torch
    B, V = 3, 64
    x, f, t = torch.zeros(B, V, device=cuda), torch.zeros(B, device=cuda), torch.zeros(B, dtype=torch.int32, device=cuda)
    m = torch.zeros(2, 2, dtype=torch.int32, device=cuda)
    call = T.trie_policy_loss
    bad = [
        (TypeError, lambda: call(x.half(), t, f, f)), (TypeError, lambda: call(x.cpu(), t, f, f)), (ValueError, lambda: call(x[0], t, f, f)),
        (ValueError, lambda: call(x, None, f, f)), (ValueError, lambda: call(x, t, None, f)), (ValueError, lambda: call(x, t, f, None)),
        (TypeError, lambda: call(x, t.long(), f, f)), (ValueError, lambda: call(x, t[:2], f, f)), (TypeError, lambda: call(x, t, f.double(), f)),
        (ValueError, lambda: call(x, t, f, f, ref_logprobs=f[:1])), (ValueError, lambda: call(x, t, f, f, weights=x)),
        (ValueError, lambda: call(x, t, f, f, grad=x[:2])), (ValueError, lambda: call(x, t, f, f, grad=x.bfloat16())),
        (ValueError, lambda: call(x, t, f, f, grad=x.t().contiguous().t())), (ValueError, lambda: call(x, t, f, f, mask=m)),
        (ValueError, lambda: call(x, t, f, f, states=t)), (ValueError, lambda: call(x, t, f, f, mask=m[:, :1], states=t)),
        (T.TrieError, lambda: call(x, t, f, f, clip=(-0.1, 0.2))), (T.TrieError, lambda: call(x, t, f, f, clip=(1.1, 0.2))),
        (T.TrieError, lambda: call(x, t, f, f, clip=(0.1, math.nan))), (T.TrieError, lambda: call(x, t, f, f, kl=-1.0)),
        (T.TrieError, lambda: call(x, t, f, f, kl=math.inf)), (ValueError, lambda: call(x[:, ::2], t, f, f)),
    ]
    for kind, run in bad:
        with pytest.raises(kind):
            run()
    losses, logprobs = call(x[:0], t[:0], f[:0], f[:0], grad=x[:0])
    assert losses.shape == logprobs.shape == (0,)
