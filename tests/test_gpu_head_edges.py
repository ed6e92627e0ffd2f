"""trie_head_logits on batches and vocabularies that take a CTA through many tiles, or past the sizes up to which
something is looked up ahead (the rules of test_gpu_head.py)."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as ref
from paper_2608_12574_gb300 import triemask as T
from test_gpu_head import _check, _inputs, _type, cuda  # noqa: F401 (cuda: a fixture)

pytestmark = pytest.mark.gpu


def _grammar(allowed, states, V, dev):
    """(mask, states, what is allowed) on the device."""
    import torch
    ok = torch.from_numpy(np.stack([ref.allowed_row(allowed, int(s), V) for s in states])).to(dev)
    return torch.from_numpy(ref.pack(allowed)).to(dev), torch.from_numpy(states).to(dev), ok


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(129, 20001, 16), (256, 50021, 128), (200, 39000, 1168), (300, 20480, 400),
                                   (600, 15001, 272), (1, 60000, 16), (128, 41000, 144), (33, 50021, 1296)])
def test_many_tiles_a_cta(cuda, M, V, D, dtype):  # noqa: F811
    """More tiles than there are CTAs, or pairs of them, with fewer blocks of columns than the rings have places and
    with more; with a grammar some tiles between them are left out."""
    import torch
    rng = np.random.default_rng([M, V, D])
    x, w = _inputs(rng, M, V, D, dtype, cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
    T.trie_head_logits(q, scales, wq, ws, out)
    _check(q, scales, wq, ws, out)
    allowed = np.zeros((4, V), bool)
    allowed[0, :V // 3] = True
    allowed[1, ::700] = True
    allowed[2, V // 2:V // 2 + 400] = True
    allowed[3, rng.choice(V, 30, replace=False)] = True
    for choice in ([0, 3], [1, 2, 3], [2, 3, -2]):
        mask, states, ok = _grammar(allowed, rng.choice(choice, M).astype(np.int32), V, cuda)
        out.fill_(math.nan)
        T.trie_head_logits(q, scales, wq, ws, out, mask, states)
        _check(q, scales, wq, ws, out, ok)


@pytest.mark.parametrize("dense", [[], [16399], [0, 9000]])
def test_many_rows(cuda, dense):  # noqa: F811
    """More rows than every CTA looks through for one that is left to the tiles: none, the last, some."""
    import torch
    rng = np.random.default_rng(16400)
    M, V, D = 16400, 700, 144
    x, w = _inputs(rng, M, V, D, "bf16", cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    allowed = rng.random((5, V)) < 0.02
    allowed[4] = rng.random(V) < 0.7
    states = rng.integers(-2, 4, M).astype(np.int32)
    states[dense] = 4
    mask, states, ok = _grammar(allowed, states, V, cuda)
    out = torch.full((M, V), math.nan, dtype=torch.bfloat16, device=cuda)
    T.trie_head_logits(q, scales, wq, ws, out, mask, states)
    _check(q, scales, wq, ws, out, ok)


def test_many_tiles_ahead(cuda):  # noqa: F811
    """A vocabulary of more tiles than a CTA looks up the need of (2,048 for each of 152)."""
    import torch
    M, V, D = 2, 2049 * 152 * 128 + 77, 16
    g = torch.Generator(device=cuda)
    g.manual_seed(5)
    w = torch.randn(V, D, generator=g, device=cuda)
    x = torch.randn(M, D, generator=g, device=cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    del w
    allowed = np.zeros((2, V), bool)
    allowed[0, ::5001] = True
    allowed[0, -300:] = True
    allowed[1, V // 7:V // 2] = True
    for choice in ([0, 1], [0, ref.FREE]):
        mask, states, ok = _grammar(allowed, np.array(choice, np.int32), V, cuda)
        out = torch.full((M, V), math.nan, dtype=torch.bfloat16, device=cuda)
        T.trie_head_logits(q, scales, wq, ws, out, mask, states)
        _check(q, scales, wq, ws, out, ok)


def test_long_hidden_states(cuda):  # noqa: F811
    """Hidden states longer than what the kernel for rows of few tokens holds: the tiles write such rows too."""
    import torch
    rng = np.random.default_rng(32784)
    for M, D in ((5, 32768), (5, 32784), (140, 33040)):
        V = 700
        x, w = _inputs(rng, M, V, D, "f32", cuda)
        q, scales = T.trie_head_quantize(x)
        wq, ws = T.trie_head_quantize_weight(w)
        allowed = rng.random((3, V)) < 0.01
        mask, states, ok = _grammar(allowed, rng.choice([0, 1, 2, -1], M).astype(np.int32), V, cuda)
        out = torch.full((M, V), math.nan, device=cuda)
        T.trie_head_logits(q, scales, wq, ws, out, mask, states)
        _check(q, scales, wq, ws, out, ok)
