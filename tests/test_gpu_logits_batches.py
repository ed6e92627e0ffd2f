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
from paper_2608_12574_gb300 import triemask as T

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


@pytest.mark.parametrize("V", [33, 257, 1001, 5003])
def test_mask_bits_past_the_vocabulary(cuda, V):
    """A mask's last word may have bits past V: they name no token."""
    import torch
    rng = np.random.default_rng(V)
    B, D = 6, 64
    allowed = rng.random((4, V)) < np.array([0.0, 3 / V, 0.5, 1.0])[:, None]
    states = torch.tensor([0, 1, 2, 3, 1, ref.FINISHED], dtype=torch.int32, device=cuda)
    clean = torch.from_numpy(ref.pack(allowed)).to(cuda)
    dirty = clean.clone()
    dirty[:, -1] |= torch.tensor(np.uint32((0xFFFFFFFF << (V % 32)) & 0xFFFFFFFF).view(np.int32).item(), device=cuda)
    w, ws = T.trie_head_quantize_weight(torch.from_numpy(rng.normal(0, 0.1, (V, D)).astype(np.float32)).to(cuda))
    q, s = T.trie_head_quantize(torch.from_numpy(rng.normal(0, 1, (B, D)).astype(np.float32)).to(cuda))
    seeds = torch.arange(B, device=cuda)
    for rows in (slice(0, B), slice(0, 2), slice(1, 3)):  # with and without rows that allow many
        got = []
        for mask in (clean, dirty):
            n = rows.stop - rows.start
            whole = torch.full((n + 1, V + 3), 7.0, device=cuda)
            out = whole[:n, :V]
            st = states[rows].contiguous()
            qn, sn = T.trie_head_quantize(torch.from_numpy(np.ones((n, D), np.float32)).to(cuda)) if n != B else (q, s)
            T.trie_head_logits(qn, sn, w, ws, out, mask, st)
            head = out.clone()
            T.trie_penalize(out, mask=mask, states=st)
            tok, lp = T.trie_sample(out, seeds[:n], mask=mask, states=st)
            assert bool((whole[n:] == 7).all()) and bool((whole[:, V:] == 7).all())
            got.append((head, out.clone(), tok, lp))
        for a, b in zip(*got):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset", [0, 1, 2, 4, 8])
def test_weights_at_any_boundary(cuda, offset, dtype):
    """Rows of weights on and off 16-byte boundaries are the same numbers."""
    import torch
    rng = np.random.default_rng(offset)
    V, D = 300, 272
    w = torch.from_numpy(rng.normal(0, 1, (V, D)).astype(np.float32)).to(getattr(torch, dtype)).to(cuda)
    want = T.trie_head_quantize_weight(w)
    wide = torch.zeros(V, D + 16, dtype=w.dtype, device=cuda)
    wide[:, offset:offset + D] = w
    got = T.trie_head_quantize_weight(wide[:, offset:offset + D])
    assert torch.equal(want[0].view(torch.uint8), got[0].view(torch.uint8)) and torch.equal(want[1], got[1])
