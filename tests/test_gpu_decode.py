"""The decode loop that runs the head, the penalties, the sampler and the trie's states together."""
from __future__ import annotations

import numpy as np
import pytest

from paper_2608_12574_gb300 import decode
from paper_2608_12574_gb300 import triemask as T
from paper_2608_12574_gb300 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def built():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device")
    T.load_library()


@pytest.mark.parametrize("batch,constrained", [(16, 8), (5, 5), (3, 0), (1, 1)])
def test_decode_loop(batch, constrained):
    """Constrained rows spell strings of the set, free ones go on; a second run says the same."""
    steps = 48
    loop, w, texts = decode.example(batch, constrained, steps)
    names = set(W.unpack(w.set_bytes, w.set_offsets))
    states = loop.states.cpu().numpy()
    assert int(loop.err.item()) == 0
    assert bool((states[:constrained] == T.TRIE_STATE_FINISHED).all())
    assert bool((states[constrained:] == T.TRIE_STATE_FREE).all())
    for text in texts[:constrained]:
        assert text in names
    for row in loop.outputs()[constrained:]:
        assert len(row) == steps and w.V - 1 not in row and min(row) >= 0
    assert bool((loop.logprobs <= 0).all()) and bool(loop.logprobs.isfinite().all())
    again, _, same = decode.example(batch, constrained, steps)
    assert same == texts and again.outputs() == loop.outputs()


def test_decode_loop_captured():
    """The captured step gives what the same step gives launch by launch."""
    import torch
    loop, _, _ = decode.example(12, 6, 20)
    other, _, _ = decode.example(12, 6, 1)
    wide = torch.zeros_like(loop.history)
    wide[:, :other.history.shape[1]] = other.history
    other.history = wide
    for _ in range(19):
        other.step()
    assert np.array_equal(loop.history.cpu().numpy(), other.history.cpu().numpy())
    assert np.array_equal(loop.states.cpu().numpy(), other.states.cpu().numpy())


def test_decode_loop_refusals():
    import torch
    w = torch.zeros(64, 16, device="cuda")
    prompts = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        decode.DecodeLoop(None, None, w, prompts, 3, 8)
    with pytest.raises(ValueError):
        decode.DecodeLoop(None, None, w, prompts, 0, 3)


@pytest.mark.parametrize("bits", [8, 4])
def test_head_weights(bits):
    """A loop's quantized weights can be read, and others put in their place."""
    import torch
    loop, w, _ = decode.example(4, 2, 4, D=128, head_bits=bits)
    assert loop.w.shape == (w.V, 128 if bits == 8 else 64) and loop.w_scales.dtype is (torch.float32 if bits == 8 else torch.float8_e4m3fn)
    assert len(loop.weight) == (2 if bits == 8 else 3) and loop.weight[0] is loop.w and loop.weight[1] is loop.w_scales
    loop.head()
    assert bool((loop.logits[2:, :-1] != 0).any())
    loop.w = torch.zeros_like(loop.w)
    loop.head()
    assert bool((loop.logits[2:, :-1] == 0).all())
