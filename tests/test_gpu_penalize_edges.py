"""trie_penalize where its ranges end, against the definition in 64 bits (the rules of test_gpu_penalize.py)."""
from __future__ import annotations

import numpy as np
import pytest

import logits_ref as ref
from paper_2608_12574_gb300 import triemask as T
from test_gpu_penalize import _case, _check, _run, cuda  # noqa: F401 (cuda: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B", [1, 64])
@pytest.mark.parametrize("H", [700, 1500, 5900])
def test_full_queues(cuda, H, B):  # noqa: F811
    """Tables filled as far as they get, by distinct tokens: every warp writes its queue out several times and keeps
    a rest of any length."""
    rng = np.random.default_rng([H, B])
    V = 40000
    case = list(_case(rng, V, B, H, 9, 0, "bf16"))
    for b in range(B):
        case[1][b] = rng.permutation(V)[:H]
    case[2][:] = H - np.arange(B)
    out = _run(cuda, V, *case)
    _check(case[0], out, *case[1:])


@pytest.mark.parametrize("max_length", [-5, 8, 70000, 2 ** 28 + 9, 2 ** 31 - 1])
def test_no_history(cuda, max_length):  # noqa: F811
    """Without a history its length says nothing: biases and the grammar as ever."""
    import torch
    rng = np.random.default_rng(3)
    V, B = 20000, 5
    case = list(_case(rng, V, B, 0, 700, 4, "f32"))
    x = case[0].to(cuda)
    off, tok, val, mask, states = (torch.from_numpy(np.ascontiguousarray(a)).to(cuda)
                                   for a in (*case[7], ref.pack(case[8]), case[9]))
    rc = T.load_library().trie_penalize(
        x.data_ptr(), 0, V, B, V, None, 0, max_length, None, None, None, None, None, off.data_ptr(), tok.data_ptr(),
        val.data_ptr(), mask.data_ptr(), mask.shape[0], states.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == T.TRIE_OK, T.trie_last_error()
    _check(case[0], x.cpu(), None, None, None, None, None, None, *case[7:])
