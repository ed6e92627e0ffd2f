"""What the norm, the 4-bit head and the policy loss refuse, without a GPU (the C ABI's checks come before any
launch: addresses here are numbers that nothing reads), and the tests' own reference of the loss against
differences."""
from __future__ import annotations

import math

import numpy as np
import pytest

import rows_ref as ref
from paper_2608_12574_gb300 import triemask as T

AT = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def lib():
    from paper_2608_12574_gb300 import _build
    _build.build()
    return T.load_library()


ROWS = dict(x=AT, dtype=0, stride=64)
NORM = dict(ROWS, residual=AT, r_dtype=1, r_stride=64, gain=AT, g_dtype=0, eps=1e-6)
LOGITS = dict(logits=AT, l_dtype=0, l_stride=64)
GRAMMAR = dict(mask=None, mask_rows=0, states=None)
CALLS = {
    "trie_head_norm_quantize": dict(NORM, M=4, D=64, q=AT, scales=AT, pitch=4, stream=None),
    "trie_head4_quantize": dict(ROWS, M=4, D=64, q=AT, scales=AT, row_scales=AT, stream=None),
    "trie_head4_norm_quantize": dict(NORM, M=4, D=64, q=AT, scales=AT, row_scales=AT, stream=None),
    "trie_head4_logits": dict(q=AT, scales=AT, row_scales=AT, w=AT, w_scales=AT, w_row_scales=AT, M=4, V=64, D=64, **LOGITS,
                              **GRAMMAR, space=AT, stream=None),
    "trie_policy_loss": dict(**LOGITS, B=4, V=64, tokens=AT, old=AT, advantages=AT, ref=AT, weights=AT, temperature=AT,
                             low=0.2, high=0.2, kl=0.1, **GRAMMAR, losses=AT, logprobs=AT, grad=AT, g_stride=64, stream=None),
}
ON_ROWS = [dict(dtype=2), dict(M=-1), dict(D=0), dict(D=2 ** 24 + 1, stride=2 ** 25, r_stride=2 ** 25), dict(stride=63), dict(x=None),
           dict(q=None), dict(scales=None), dict(x=AT + 2), dict(x=AT + 1, dtype=1)]
ON_NORM = [*ON_ROWS, dict(r_dtype=7), dict(g_dtype=-1), dict(r_stride=63), dict(gain=None), dict(gain=AT + 2), dict(residual=AT + 1),
           dict(eps=0.0), dict(eps=-1.0), dict(eps=math.nan), dict(eps=math.inf), dict(eps=1e-31)]
ON_4 = [dict(q=AT + 8), dict(scales=AT + 4), dict(row_scales=None), dict(row_scales=AT + 2)]
ON_LOGITS = [dict(l_dtype=7), dict(V=1), dict(V=2 ** 31 - 1000, l_stride=2 ** 31), dict(l_stride=63), dict(logits=None),
             dict(logits=AT + 2), dict(logits=AT + 1, l_dtype=1), dict(mask=AT), dict(states=AT),
             dict(mask=AT + 2, states=AT, mask_rows=1), dict(mask=AT, states=AT, mask_rows=-1)]
BAD = {
    "trie_head_norm_quantize": [*ON_NORM, dict(pitch=3), dict(scales=AT + 2)],
    "trie_head4_quantize": [{k: v for k, v in c.items() if k != "r_stride"} for c in ON_ROWS] + ON_4,
    "trie_head4_norm_quantize": [*ON_NORM, *ON_4],
    "trie_head4_logits": [*ON_LOGITS, dict(M=-1), dict(M=2 ** 20 + 1), dict(D=0), dict(D=2 ** 24 + 1), dict(q=None), dict(scales=None),
                          dict(row_scales=None), dict(w=None), dict(w_scales=None), dict(w_row_scales=None), dict(q=AT + 8),
                          dict(w=AT + 4), dict(scales=AT + 8), dict(w_scales=AT + 1), dict(row_scales=AT + 2),
                          dict(w_row_scales=AT + 1), dict(mask=AT, states=AT, mask_rows=1, space=None),
                          dict(mask=AT, states=AT, mask_rows=1, space=AT + 8)],
    "trie_policy_loss": [*ON_LOGITS, dict(B=-1), dict(B=2 ** 30 + 1), dict(tokens=None), dict(old=None), dict(advantages=None), dict(losses=None),
                         dict(logprobs=None), dict(tokens=AT + 2), dict(old=AT + 1), dict(advantages=AT + 2), dict(ref=AT + 2),
                         dict(weights=AT + 2), dict(temperature=AT + 2), dict(losses=AT + 2), dict(logprobs=AT + 2), dict(low=-0.1),
                         dict(low=1.5), dict(low=math.nan), dict(high=-0.1), dict(high=math.inf), dict(high=math.nan), dict(kl=-1.0),
                         dict(kl=math.inf), dict(kl=math.nan), dict(g_stride=63), dict(grad=AT + 2), dict(grad=AT + 1, l_dtype=1),
                         dict(l_stride=65)],
}


@pytest.mark.parametrize("which,change", [(w, c) for w, cs in BAD.items() for c in cs],
                         ids=lambda x: x if isinstance(x, str) else ",".join(f"{k}={v}" for k, v in x.items()))
def test_refusals(lib, which, change):
    assert set(change) <= set(CALLS[which])
    assert getattr(lib, which)(*{**CALLS[which], **change}.values()) == T.TRIE_EINVAL
    assert T.trie_last_error()


@pytest.mark.parametrize("which", sorted(CALLS))
def test_nothing_to_do(lib, which):
    """No rows: no pointer is needed and nothing is launched."""
    good = CALLS[which]
    none = {k: None for k, v in good.items() if v == AT}
    empty = {k: 0 for k in ("M", "B") if k in good}
    assert getattr(lib, which)(*{**good, **none, **empty}.values()) == T.TRIE_OK


def test_sizes(lib):
    assert [lib.trie_head4_row_bytes(d) for d in (1, 32, 33, 4096)] == [16, 16, 32, 2048]
    assert [lib.trie_head4_scale_bytes(*s) for s in ((0, 64), (1, 1), (128, 64), (129, 65))] == [0, 512, 512, 2048]
    assert lib.trie_head4_row_bytes(0) == lib.trie_head4_row_bytes(2 ** 24 + 1) == -1
    assert lib.trie_head4_scale_bytes(-1, 64) == lib.trie_head4_scale_bytes(1, 0) == -1
    assert lib.trie_head4_scale_bytes(2 ** 31 - 1, 2 ** 24) > 2 ** 31


def test_binding_refuses_host_tensors(lib):
    import torch
    x, g, i = torch.zeros(4, 64), torch.ones(64), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: T.trie_head_norm_quantize(x, g), lambda: T.trie_head4_norm_quantize(x, g), lambda: T.trie_head4_quantize(x),
                 lambda: T.trie_policy_loss(x, i, g[:4], g[:4])):
        with pytest.raises(TypeError):
            call()
    q, s, r = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(1, 1, 32, 4, 4).to(torch.float8_e4m3fn), torch.zeros(4)
    with pytest.raises(TypeError):
        T.trie_head4_logits(q, s, r, q, s, r, torch.zeros(4, 4))


@pytest.mark.parametrize("kl", [0.0, 0.3])
def test_reference_gradient(kl):
    """The reference's gradient against differences of its loss."""
    rng = np.random.default_rng(1)
    V, step = 12, 1e-6
    for old, A in ((-2.0, 1.0), (-2.0, -1.0), (-3.5, 0.7), (-3.5, -0.7), (-1.0, 0.4), (-1.0, -0.4)):
        x, ok = rng.normal(0, 1, V), rng.random(V) < 0.8
        ok[3] = True
        args = (3, old, A, -1.5, 0.7, 1.3, 0.2, 0.3, kl, ok)
        _, _, _, grad = ref.policy(x, *args)
        for v in range(V):
            up, down = x.copy(), x.copy()
            up[v] += step
            down[v] -= step
            slope = (ref.policy(up, *args)[0] - ref.policy(down, *args)[0]) / (2 * step)
            assert abs(slope - grad[v]) <= 1e-8, (old, A, v)


def test_reference_codes():
    u = np.array([0, 0.2, 0.25, 0.26, 0.75, 1.2, 1.25, 1.75, 2.5, 2.6, 3.5, 5.0, 5.1, 6, 7])
    assert ref.nearest4(u).tolist() == [0, 0, 0, 1, 2, 2, 2, 4, 4, 5, 6, 6, 7, 7, 7]
