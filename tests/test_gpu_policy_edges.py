"""The policy loss where a ratio, a slope or a temperature's reciprocal leaves the range of 32 bits, and rows without a
token beside a NaN."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as lref
from paper_2608_12574_gb300 import triemask as T
from test_gpu_policy import _type, cuda  # noqa: F401

pytestmark = pytest.mark.gpu
SIZES = [300, 5003, 300001]  # rows held by one CTA and by several, and rows read again


def _run(dev, x, tokens, old, A, weights=None, temperature=None, refs=None, **more):
    import torch
    put = lambda a, t=torch.float32: None if a is None else torch.tensor(a, dtype=t, device=dev)  # noqa: E731
    grad = torch.full_like(x, 7.0)
    losses, lp = T.trie_policy_loss(x, put(tokens, torch.int32), put(old), put(A), ref_logprobs=put(refs), weights=put(weights),
                                    temperature=put(temperature), grad=grad, **more)
    return losses.cpu(), lp.cpu(), grad


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_tiny_temperature(cuda, V, dtype):  # noqa: F811
    """A probability of 0 has a gradient of 0, however large slope / temperature is; one of 1 as well; two tokens of a half
    each have as much of it as 32 bits hold."""
    import torch
    x = torch.from_numpy(np.random.default_rng(V).normal(0, 1, (3, V)).astype(np.float32)).clamp(max=4).to(_type(dtype)).to(cuda)
    x[0, 5] = x[1, V - 1] = 6.0
    x[2, 7] = x[2, V - 2] = 6.0
    losses, lp, grad = _run(cuda, x, [5, V - 1, 7], [0.0] * 3, [3.0, -3.0, 3.0], [50.0] * 3, [1e-38, 2.0 ** -126, 1e-38])
    # rho is 1, and a half in the last row
    assert losses.tolist()[:2] == [-150.0, 150.0] and abs(float(losses[2]) + 75) < 1e-4
    assert lp.tolist()[:2] == [0.0, 0.0] and abs(float(lp[2]) - math.log(0.5)) < 1e-6
    assert bool((grad[:2] == 0).all())
    assert grad[2, 7] == -math.inf and grad[2, V - 2] == math.inf
    grad[2, 7] = grad[2, V - 2] = 0
    assert bool((grad[2] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_ratio_beyond_32_bits(cuda, V, dtype):  # noqa: F811
    """An old log-probability 190 below the new one: an advantage of 0 has no surrogate at all, a positive one the clipped,
    a negative one an infinite loss, and no NaN beside it."""
    import torch
    x = torch.zeros(4, V, dtype=_type(dtype), device=cuda)
    x[:, 1::3] = -200.0  # so far below that their probabilities are 0 in 32 bits
    x[3, 2] = 200.0
    n = V - len(range(1, V, 3))
    lp_want = -math.log(n)
    refs = [lp_want + 0.5] * 3 + [0.5]
    losses, lp, grad = _run(cuda, x, [0, 0, 0, 2], [-200.0] * 4, [0.0, 2.0, -2.0, -2.0], refs=refs, kl=0.25, clip=(0.2, 0.3))
    assert float((lp - torch.tensor([lp_want] * 3 + [0.0])).abs().max()) < 1e-4
    kl, slope = 0.25 * (math.exp(0.5) - 1.5), 0.25 * (1 - math.exp(0.5))
    assert abs(float(losses[0]) - kl) < 1e-4 and abs(float(losses[1]) - (kl - 2.0 * 1.3)) < 1e-4
    assert losses[2] == math.inf and losses[3] == math.inf
    want = torch.full((V,), -slope / n)
    want[1::3] = 0.0
    want[0] += slope
    for b in (0, 1):  # one of the clip's border has the KL term's gradient
        assert float((grad[b].float().cpu() - want).abs().max()) <= abs(slope) * (1e-4 + (2.0 ** -8 if dtype == "bf16" else 0))
    assert grad[2, 0] == math.inf and bool((grad[2, 3::3] == -math.inf).all()) and bool((grad[2, 1::3] == 0).all())
    assert not bool(grad[3].isnan().any())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("V", SIZES)
def test_no_token_beside_nan(cuda, V, value, dtype):  # noqa: F811
    """A row without a token (outside the vocabulary, not allowed, of logit -inf) has the loss 0 and zeros whatever its allowed
    logits hold; one with a token has NaN, and with weight 0 the log-probability alone."""
    import torch
    allowed = np.ones((2, V), bool)
    allowed[1] = False
    allowed[1, [3, 9, V - 1]] = True
    allowed[0, 6] = False
    tokens = [-1, V, 6, 8, 4, 2 ** 31 - 1, 6, 8, 8, 9, 4, 3]
    states = [0, 0, 0, 0, -3, 1, 1, 1, 0, 1, -3, 1]
    weights = [1.0] * 10 + [0.0] * 2
    x = torch.from_numpy(np.random.default_rng(V).normal(0, 1, (12, V)).astype(np.float32)).to(_type(dtype)).to(cuda)
    x[:, V - 1] = value
    x[3, 8] = x[4, 4] = -math.inf
    x[10, 4] = 1.0
    losses, lp, grad = _run(cuda, x, tokens, [-3.0] * 12, [1.0] * 12, weights, refs=[-3.0] * 12, kl=0.1,
                            mask=torch.from_numpy(lref.pack(allowed)).to(cuda), states=torch.tensor(states, dtype=torch.int32, device=cuda))
    none = [0, 1, 2, 3, 4, 5, 6, 7]
    assert bool((losses[none] == 0).all()) and bool((lp[none] == -math.inf).all()) and bool((grad[none] == 0).all())
    assert bool(losses[8:10].isnan().all()) and bool(lp[8:].isnan().all())
    for b, s in ((8, 0), (9, 1)):
        ok = torch.from_numpy(allowed[s]).to(cuda)
        assert bool(grad[b][ok].isnan().all()) and bool((grad[b][~ok] == 0).all())
    assert bool((losses[10:] == 0).all()) and bool((grad[10:] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", SIZES)
def test_nan_beside_zero(cuda, V, dtype):  # noqa: F811
    """A NaN is none of the values that 32 bits do not hold: beside an advantage of 0, or a probability of 1, it stays."""
    import torch
    x = torch.from_numpy(np.random.default_rng(V).normal(0, 1, (5, V)).astype(np.float32)).to(_type(dtype)).to(cuda)
    x[0, V - 2] = math.nan          # a logit
    x[2] = -300.0
    x[2, 5] = 300.0                 # the token's probability is 1
    losses, lp, grad = _run(cuda, x, [5] * 5, [-3.0, math.nan, 0.0, -3.0, -3.0], [0.0, 0.0, math.nan, math.nan, 0.0], clip=(0.2, 0.2))
    assert bool(losses[:4].isnan().all()) and bool(grad[:4].isnan().all())
    assert bool(lp[0].isnan()) and bool(lp[1:].isfinite().all())
    assert losses[4] == 0 and bool((grad[4] == 0).all())
