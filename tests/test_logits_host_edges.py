"""What else the calls on logits refuse, without a GPU (the rules of test_logits_host.py)."""
from __future__ import annotations

import pytest

from paper_2608_12574_gb300 import triemask as T
from test_logits_host import AT, GOOD, NAMES, _call, lib  # noqa: F401 (lib: a fixture)

BIAS = dict(offsets=AT, tokens=AT, values=AT)
GRAMMAR = dict(mask=AT, states=AT, rows=1)
OFF = {
    "head": [dict(GRAMMAR, states=AT + 2)],
    "penalize": [dict(GRAMMAR, states=AT + 1), *(dict(BIAS, **{n: AT + 2}) for n in BIAS),
                 *({n: AT + 1} for n in ("history", "length", "prompt", "repetition", "presence", "frequency"))],
    "sample": [dict(GRAMMAR, states=AT + 2), dict(seeds=AT + 4),
               *({n: AT + 2} for n in ("temperature", "top_k", "top_p", "min_p", "tokens", "logprobs"))],
}


@pytest.mark.parametrize("which,change", [(w, c) for w, cs in OFF.items() for c in cs],
                         ids=lambda x: x if isinstance(x, str) else ",".join(f"{k}={v}" for k, v in x.items()))
def test_arrays_off_their_elements(lib, which, change):  # noqa: F811
    name, names = NAMES[which]
    assert _call(getattr(lib, name), names, GOOD[which], **change) == T.TRIE_EINVAL
    assert "aligned" in T.trie_last_error()
