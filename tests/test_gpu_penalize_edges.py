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
