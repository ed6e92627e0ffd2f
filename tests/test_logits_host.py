"""What the calls on logits refuse, without a GPU: the C ABI's checks come before any launch
(addresses here are numbers that nothing reads), the binding's before the library."""
from __future__ import annotations

import pytest

from paper_2608_12574_gb300 import triemask as T

AT = 1 << 20  # an aligned address


@pytest.fixture(scope="module")
def lib():
    from paper_2608_12574_gb300 import _build
    _build.build()
    return T.load_library()


def _call(f, names, good, **change):
    assert set(change) <= set(names)
    return f(*[{**good, **change}[n] for n in names])


QUANTIZE = ["x", "dtype", "stride", "M", "D", "q", "scales", "pitch", "stream"]
WEIGHT = ["x", "dtype", "stride", "V", "D", "q", "scales", "stream"]
HEAD = ["q", "scales", "pitch", "w", "w_scales", "M", "V", "D", "logits", "dtype", "stride", "mask", "rows", "states",
        "space", "stream"]
PENALIZE = ["logits", "dtype", "stride", "B", "V", "history", "h_stride", "H", "length", "prompt", "repetition",
            "presence", "frequency", "offsets", "tokens", "values", "mask", "rows", "states", "stream"]
SAMPLE = ["logits", "dtype", "stride", "B", "V", "seeds", "temperature", "top_k", "top_p", "min_p", "mask", "rows",
          "states", "space", "tokens", "logprobs", "stream"]
LOGITS = dict(logits=AT, dtype=0, stride=64, V=64, mask=None, rows=0, states=None, stream=None)
GOOD = {
    "quantize": dict(x=AT, dtype=0, stride=64, M=4, D=64, q=AT, scales=AT, pitch=4, stream=None),
    "weight": dict(x=AT, dtype=0, stride=64, V=4, D=64, q=AT, scales=AT, stream=None),
    "head": dict(LOGITS, q=AT, scales=AT, pitch=4, w=AT, w_scales=AT, M=4, D=64, space=AT),
    "penalize": dict(LOGITS, B=4, history=AT, h_stride=8, H=8, length=AT, prompt=None, repetition=None, presence=None,
                     frequency=None, offsets=None, tokens=None, values=None),
    "sample": dict(LOGITS, B=4, seeds=AT, temperature=None, top_k=None, top_p=None, min_p=None, space=AT, tokens=AT,
                   logprobs=None),
}
ON_LOGITS = [dict(dtype=7), dict(V=1), dict(V=2 ** 31 - 1000, stride=2 ** 31), dict(stride=63), dict(logits=None),
             dict(logits=AT + 2), dict(logits=AT + 1, dtype=1), dict(mask=AT), dict(states=AT),
             dict(mask=AT + 2, states=AT, rows=1), dict(mask=AT, states=AT, rows=-1)]
BAD = {
    "quantize": [dict(dtype=2), dict(M=-1), dict(D=0), dict(stride=63), dict(x=None), dict(q=None), dict(scales=None),
                 dict(pitch=3), dict(x=AT + 2), dict(scales=AT + 2)],
    "weight": [dict(dtype=-1), dict(V=-1), dict(D=0), dict(stride=1), dict(x=None), dict(q=None), dict(scales=None),
               dict(x=AT + 1, dtype=1)],
    "head": [*ON_LOGITS, dict(M=-1), dict(M=2 ** 20 + 1, pitch=2 ** 21), dict(D=8), dict(D=72), dict(D=0), dict(pitch=0),
             dict(pitch=6), dict(q=None), dict(scales=None), dict(w=None), dict(w_scales=None), dict(q=AT + 8),
             dict(w=AT + 8), dict(scales=AT + 4), dict(w_scales=AT + 2), dict(mask=AT, states=AT, rows=1, space=None),
             dict(mask=AT, states=AT, rows=1, space=AT + 8)],
    "penalize": [*ON_LOGITS, dict(B=-1), dict(B=65536), dict(length=None), dict(H=-1), dict(H=2 ** 28 + 1, h_stride=2 ** 29),
                 dict(h_stride=7), dict(offsets=AT), dict(offsets=AT, tokens=AT)],
    "sample": [*ON_LOGITS, dict(B=-1), dict(B=65536), dict(seeds=None), dict(space=None), dict(space=AT + 8),
               dict(tokens=None)],
}
NAMES = {"quantize": ("trie_head_quantize", QUANTIZE), "weight": ("trie_head_quantize_weight", WEIGHT),
         "head": ("trie_head_logits", HEAD), "penalize": ("trie_penalize", PENALIZE), "sample": ("trie_sample", SAMPLE)}


@pytest.mark.parametrize("which,change", [(w, c) for w, cs in BAD.items() for c in cs],
                         ids=lambda x: x if isinstance(x, str) else ",".join(f"{k}={v}" for k, v in x.items()))
def test_refusals(lib, which, change):
    name, names = NAMES[which]
    assert _call(getattr(lib, name), names, GOOD[which], **change) == T.TRIE_EINVAL
    assert T.trie_last_error()


@pytest.mark.parametrize("which", ["quantize", "weight", "head", "penalize", "sample"])
def test_nothing_to_do(lib, which):
    """No rows: no pointer is needed and nothing is launched."""
    name, names = NAMES[which]
    none = {k: None for k in GOOD[which] if k in ("x", "q", "scales", "w", "w_scales", "logits", "history", "seeds", "space", "tokens")}
    empty = {k: 0 for k in ("B", "M") if k in GOOD[which]} or {"V": 0}
    assert _call(getattr(lib, name), names, GOOD[which], **none, **empty) == T.TRIE_OK


def test_workspaces(lib):
    assert lib.trie_sample_workspace(65536, 64) == lib.trie_sample_workspace(4, 1) == lib.trie_sample_workspace(-1, 64) == -1
    assert lib.trie_head_workspace(2 ** 20 + 1, 64) == lib.trie_head_workspace(4, 1) == lib.trie_head_workspace(-1, 64) == -1
    assert lib.trie_sample_workspace(0, 64) >= 0 and lib.trie_head_workspace(0, 64) >= 0
    small, large = lib.trie_sample_workspace(1, 32000), lib.trie_sample_workspace(256, 262144)
    assert 0 < small < large < 2 ** 31
    with pytest.raises(ValueError):
        T.trie_sample_workspace(4, 1)
    with pytest.raises(ValueError):
        T.trie_head_workspace(-1, 64)


def test_binding_refuses_host_tensors(lib):
    import torch
    x, v = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: T.trie_head_quantize(x), lambda: T.trie_head_quantize_weight(x),
                 lambda: T.trie_penalize(x), lambda: T.trie_sample(x, v)):
        with pytest.raises(TypeError):
            call()
    q = torch.zeros(4, 64, dtype=torch.float8_e4m3fn)
    with pytest.raises(TypeError):
        T.trie_head_logits(q, torch.zeros(1, 4), torch.zeros(64, 64, dtype=torch.float8_e4m3fn), torch.zeros(1, 1), x)
    with pytest.raises(TypeError):
        T.trie_head_quantize(x.to(torch.float16))
    with pytest.raises(ValueError):
        T.trie_head_quantize(torch.zeros(4))
