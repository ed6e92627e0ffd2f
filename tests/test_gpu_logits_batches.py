"""The calls on logits at batch sizes and lists on both sides of where their kernels are
cut differently: rows shared by one, two and four CTAs, crowds of equal logits, histories
on one and several CTAs, more constrained rows than a block has threads.

Tolerances are those of test_gpu_sample.py and test_gpu_penalize.py."""
from __future__ import annotations

import numpy as np
import pytest

import logits_ref as ref
import test_gpu_penalize as penalize
import test_gpu_sample as sample

pytestmark = pytest.mark.gpu
cuda = sample.cuda


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("B", [76, 77, 152, 153, 304, 305])
def test_sample_batches(cuda, B, masked, dtype):
    rng = np.random.default_rng([B, masked])
    V = 5003
    x = sample._logits(rng, B, V, dtype)
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp, k, p, m = sample._ways(rng, B, V)
    allowed = states = None
    if masked:
        allowed = rng.random((6, V)) < np.array([0.0, 0.001, 0.05, 0.5, 0.9, 1.0])[:, None]
        states = rng.integers(-3, 7, B).astype(np.int32)
    tok, lp = sample._run(cuda, x.to(cuda), seeds, temp, k, p, m, allowed, states)
    sample._check(x, seeds, temp, k, p, m, allowed, states, tok, lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1500, 9001, 20000])
def test_sample_crowds(cuda, V, dtype):
    """Crowds of some hundred to some thousand equal logits, cut by count, by weight and by both."""
    import torch
    rng = np.random.default_rng(V)
    B = 40
    values = np.array([1.75, 1.5, 1.0, 0.25, -1.0, -2.0, -3.5])
    x = torch.from_numpy(values[rng.integers(0, 7, (B, V))].astype(np.float32)).to(
        torch.float32 if dtype == "f32" else torch.bfloat16)
    seeds = rng.integers(-2 ** 63, 2 ** 63 - 1, B)
    temp = rng.choice([0.5, 1.0, 3.0], B).astype(np.float32)
    k = rng.choice([0, 65, 129, 200, 700, 1400], B).astype(np.int32)
    p = rng.choice([1.0, 0.37, 0.83, 0.61], B).astype(np.float32)
    tok, lp = sample._run(cuda, x.to(cuda), seeds, temp, k, p)
    sample._check(x, seeds, temp, k, p, None, None, None, tok, lp)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B,H,n_bias,rows", [
    (200, 700, 9, 3, 5), (1023, 1100, 0, 0, 4), (40000, 2, 6000, 9, 3), (40000, 2, 6001, 9, 3), (90000, 2, 12000, 9, 3),
    (90000, 3, 12001, 9, 3), (90000, 160, 6100, 0, 2)])
def test_penalize_batches(cuda, V, B, H, n_bias, rows, dtype):
    rng = np.random.default_rng([V, B, H])
    case = penalize._case(rng, V, B, H, n_bias, rows, dtype)
    out = penalize._run(cuda, V, *case)
    penalize._check(case[0][:, :V], out, *case[1:])
