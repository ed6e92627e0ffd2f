"""The norm, the 4-bit head, the sampler and the policy loss one after the other, as they are used together."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as lref
from paper_2608_12574_gb300 import decode
from paper_2608_12574_gb300 import triemask as T
from paper_2608_12574_gb300 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device")
    T.load_library()
    return torch.device("cuda:0")


@pytest.mark.parametrize("bits,norm", [(4, False), (4, True), (8, True)])
@pytest.mark.parametrize("batch,constrained", [(16, 8), (150, 140), (1, 1)])
def test_decode_loop(cuda, bits, norm, batch, constrained):
    """Constrained rows spell strings of the set, free ones go on; the captured step says what step() does."""
    import torch
    steps = 48
    loop, w, texts = decode.example(batch, constrained, steps, head_bits=bits, norm=norm)
    names = set(W.unpack(w.set_bytes, w.set_offsets))
    assert int(loop.err.item()) == 0
    assert bool((loop.states[:constrained] == T.TRIE_STATE_FINISHED).all())
    assert all(text in names for text in texts[:constrained])
    for row in loop.outputs()[constrained:]:
        assert len(row) == steps and w.V - 1 not in row and min(row) >= 0
    other, _, _ = decode.example(batch, constrained, 1, head_bits=bits, norm=norm)
    wide = torch.zeros_like(loop.history)
    wide[:, :other.history.shape[1]] = other.history
    other.history = wide
    for _ in range(steps - 1):
        other.step()
    assert torch.equal(loop.history, other.history) and torch.equal(loop.states, other.states)


def test_decode_loop_refuses_bits(cuda):
    import torch
    w = torch.zeros(64, 16, device=cuda)
    with pytest.raises(ValueError):
        decode.DecodeLoop(None, None, w, torch.zeros(2, 3, dtype=torch.int32, device=cuda), 0, 8, head_bits=6)


class Chain:
    """Hidden states, a residual, 4-bit weights, a grammar for half of the rows."""

    def __init__(self, dev, M, V, D, dtype, seed):
        import torch
        rng = np.random.default_rng([M, V, seed])
        put = lambda a, t=torch.float32: torch.from_numpy(np.ascontiguousarray(a)).to(t).to(dev)  # noqa: E731
        self.x, self.start = put(rng.normal(0, 1, (M, D)), dtype), put(rng.normal(0, 3, (M, D)))
        self.residual = self.start.clone()
        self.gain = put(rng.uniform(0.5, 1.5, D))
        self.w = T.trie_head4_quantize(put(rng.normal(0, 1, (V, D)) / math.sqrt(D) * 3))
        allowed = rng.random((5, V)) < np.array([0.002, 0.3, 3 / V, 1, 0.9])[:, None]
        allowed[:, 5] = True
        self.allowed = allowed
        self.state_ids = rng.choice([-3, -3, -3, 0, 1, 2, 3, 4, -1], M).astype(np.int32)
        self.mask, self.states = put(lref.pack(allowed), torch.int32), put(self.state_ids, torch.int32)
        self.logits = torch.empty(M, V, dtype=dtype, device=dev)
        self.temperature = put(rng.choice([0.7, 1.0, 1.3], M))
        self.seeds = put(rng.integers(-2 ** 62, 2 ** 62, M), torch.int64)
        self.A = put(rng.normal(0, 1, M))
        self.weights = put(rng.uniform(0.5, 1.5, M) / M)
        self.grad = torch.empty_like(self.logits)

    def run(self, stream=None):
        self.residual.copy_(self.start)
        on = dict(mask=self.mask, states=self.states, stream=stream)
        q = T.trie_head4_norm_quantize(self.x, self.gain, self.residual, stream=stream)
        T.trie_head4_logits(*q, *self.w, self.logits, **on)
        tokens, sampled = T.trie_sample(self.logits, self.seeds, temperature=self.temperature, **on)
        losses, logprobs = T.trie_policy_loss(self.logits, tokens, sampled, self.A, weights=self.weights,
                                              temperature=self.temperature, kl=0.1, grad=self.grad, **on)
        return tokens, sampled, losses, logprobs


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(1, 500, 128), (40, 3001, 400), (200, 5000, 512)])
def test_chain(cuda, M, V, D, dtype):
    """A token's log-probability is the sampler's, so the ratio is 1, the loss minus the weighted advantage, and the
    gradient's rows add up to 0."""
    import torch
    c = Chain(cuda, M, V, D, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], 1)
    tokens, sampled, losses, logprobs = c.run()
    ok = torch.from_numpy(np.stack([lref.allowed_row(c.allowed, int(s), V) for s in c.state_ids])).to(cuda)
    assert bool(ok[torch.arange(M), tokens.long()].all())
    # both are within 1e-5 of the log-probability in 64 bits (test_gpu_sample.py, test_gpu_policy.py)
    assert float((logprobs - sampled).abs().max()) <= 2e-5
    want = -c.weights * c.A
    assert float((losses - want).abs().max()) <= float(want.abs().max()) * 3e-5
    assert bool((c.grad[~ok] == 0).all())
    # a row's entries: half a step each (of 2^-8 or 2^-24) and p's own error, 1e-4 of it at most; and the token's
    # entry is slope (1 - exp(lp)) / T with lp off by up to 2e-5, so by slope exp(lp) 2e-5 / T, |slope| = |weight A|,
    # however small 1 - exp(lp) is
    size = c.grad.double().abs().sum(dim=1)
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    off = size * (half + 1e-4) + (want.abs() / c.temperature).double() * 2e-5
    assert bool((c.grad.double().sum(dim=1).abs() <= off).all())


def test_chain_captured(cuda):
    """Two captured chains replayed in turn and on two streams at once give what the calls give launch by launch."""
    import torch
    chains = [Chain(cuda, 30 + 110 * i, 2003, 256, torch.bfloat16, i) for i in range(2)]
    want = [[t.clone() for t in (*c.run(), c.logits, c.grad, c.residual)] for c in chains]
    graphs, outs = [], []
    for c in chains:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(c.run())
        for t in (c.logits, c.grad, *outs[-1]):
            t.zero_()
    side = [torch.cuda.Stream() for _ in chains]
    for i in range(6):
        for g, s in zip(graphs, side):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for c, out, ref in zip(chains, outs, want):
            for a, b in zip((*out, c.logits, c.grad, c.residual), ref):
                assert torch.equal(a, b)
    for c, ref in zip(chains, want):  # and on given streams
        s = side[0]
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            out = c.run(stream=s)
        s.synchronize()
        for a, b in zip((*out, c.logits, c.grad), ref):
            assert torch.equal(a, b)


def test_first_calls_are_captured(cuda):
    """A process whose first calls are made under capture (what a call asks the runtime once is asked there)."""
    import os
    import subprocess
    import sys
    code = """
import sys, torch
sys.path[:0] = [%r, %r]
import test_gpu_policy_chain as C
dev = torch.device("cuda:0")
c = C.Chain(dev, 20, 2003, 4096, torch.bfloat16, 1)
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    out = c.run()
graph.replay()
torch.cuda.synchronize()
got = [t.clone() for t in (*out, c.logits, c.grad)]
want = [*c.run(), c.logits, c.grad]
assert all(torch.equal(a, b) for a, b in zip(got, want))
print("same")
""" % (os.path.dirname(os.path.dirname(os.path.abspath(__file__))), os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]
