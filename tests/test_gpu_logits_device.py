"""The calls on logits and tensors of a device that is not the current one."""
from __future__ import annotations

import pytest

from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu


def test_other_device_refused(monkeypatch):
    """With another device current the calls are refused before the library is called (the current device is a
    stand-in: no second one is needed)."""
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_12574_gb300 import _build
    _build.build()
    dev = torch.device("cuda:0")
    x = torch.zeros(4, 256, device=dev)
    q, s = T.trie_head_quantize(x)
    w, ws = T.trie_head_quantize_weight(x)
    out, seeds = torch.zeros(4, 4, device=dev), torch.zeros(4, dtype=torch.int64, device=dev)
    h = torch.zeros(4, 8, dtype=torch.int32, device=dev)
    calls = [lambda: T.trie_head_quantize(x), lambda: T.trie_head_quantize_weight(x),
             lambda: T.trie_head_logits(q, s, w, ws, out), lambda: T.trie_penalize(out),
             lambda: T.trie_penalize(out, h, h[:, 0].contiguous()), lambda: T.trie_sample(out, seeds)]
    for call in calls:
        call()
    torch.cuda.synchronize()
    lib = T.load_library()
    names = ("trie_head_quantize", "trie_head_quantize_weight", "trie_head_logits", "trie_penalize", "trie_sample")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for name in names:
        monkeypatch.setattr(lib, name, lambda *a, name=name: pytest.fail(f"{name} was launched"))
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()
