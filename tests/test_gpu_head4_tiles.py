"""The 4-bit head where a CTA, or a pair of CTAs, takes several tiles: the ring's phases, accumulators used again and scales
read ahead go on from one tile to the next."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as lref
from paper_2608_12574_gb300 import triemask as T
from test_gpu_head4 import _check, _inputs, _type, cuda  # noqa: F401

pytestmark = pytest.mark.gpu


def _rows(M, V, pad, dtype, dev):
    import torch
    return torch.full((M, V + pad), math.nan, dtype=_type(dtype), device=dev)[:, :V]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 15])  # of odd V: rows at any two or four bytes; all on 32-byte boundaries
@pytest.mark.parametrize("M,V,D", [(5, 40001, 200), (40, 60001, 656), (64, 40001, 256), (128, 60001, 400), (200, 40001, 256),
                                   (256, 60001, 528), (300, 20001, 272)])
def test_head4_tiles(cuda, M, V, D, pad, dtype):  # noqa: F811
    x, w = _inputs(np.random.default_rng([M, V, D]), M, V, D, cuda)
    out = _rows(M, V, pad, dtype, cuda)
    T.trie_head4_logits(*x, *w, out)
    _check(x, w, D, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad", [0, 15])
@pytest.mark.parametrize("M,V,D", [(64, 40001, 256), (200, 40001, 256), (300, 40001, 144)])
def test_head4_tiles_grammar(cuda, M, V, D, pad, dtype):  # noqa: F811
    """Free rows, rows of few tokens and of many, so that some of a CTA's tiles are left out and others are not."""
    import torch
    rng = np.random.default_rng([M, V, 1])
    x, w = _inputs(rng, M, V, D, cuda)
    allowed = rng.random((8, V)) < np.array([0, 3 / V, 40 / V, 0.3, 0.9, 0, 0, 0])[:, None]
    allowed[5, 11000:11400] = True      # more than a list's length, in few tiles
    allowed[6, V - 300:] = True
    allowed[7, ::97] = True
    mask = torch.from_numpy(lref.pack(allowed)).to(cuda)
    for choice in ([-3, 0, 1, 2, 3, 4, -1], [5, 6, 0, 1], [5], [7, 2, -2]):
        states = rng.choice(choice, M).astype(np.int32)
        ok = torch.from_numpy(np.stack([lref.allowed_row(allowed, int(s), V) for s in states])).to(cuda)
        out = _rows(M, V, pad, dtype, cuda)
        T.trie_head4_logits(*x, *w, out, mask, torch.from_numpy(states).to(cuda))
        _check(x, w, D, out, ok)
