"""A decode loop over the library's calls, from hidden states to sampled tokens.

    python -m paper_2608_12574_gb300.decode [--batch 16] [--constrained 8] [--steps 48] [--bits 8|4] [--norm]

Some rows of the batch are constrained to a set of strings (a trie's mask, states
advanced by the sampled tokens), the others are free; they share every call:

    trie_head_quantize, trie_head_logits   hidden states -> logits, -inf off the grammar
        (or trie_head_norm_quantize in front of it; in 4 bits the trie_head4_ calls)
    trie_penalize                          repetition, presence, frequency, biases
    trie_sample                            temperature, top-k, top-p, min-p -> tokens
    trie_advance                           the constrained rows' states

The step is captured once in a CUDA graph and replayed. The model in front of it is a
stand-in with random weights (an embedding and a rotation): what comes before the head
is the user's own.
"""
from __future__ import annotations

import argparse

from . import triemask as T
from . import workloads as W


class DecodeLoop:
    """A batch of `batch` rows, of which the first `constrained` follow the trie `h` and its mask.

    prompts: int32 [batch, P] token ids. weight: [V, D]. head_bits: 8 or 4, of the head's weights and
    hidden states. gain: [D], the last norm's, which the head's call then includes. The sampling settings
    are one value for all rows here; the calls take one for each."""

    def __init__(self, h, mask, weight, prompts, constrained: int, max_length: int, *, head_bits=8, gain=None,
                 temperature=0.8, top_k=50, top_p=0.95, min_p=0.0, repetition=1.1, presence=0.0, frequency=0.0, seed=0):
        import torch
        B, (V, D), dev = prompts.shape[0], weight.shape, weight.device
        P = prompts.shape[1]
        if not 0 <= constrained <= B:
            raise ValueError("constrained must be in [0, batch]")
        if max_length <= P:
            raise ValueError("max_length must leave room after the prompts")
        if head_bits not in (4, 8):
            raise ValueError("head_bits must be 4 or 8")
        self.h, self.mask, self.constrained, self.P = h, mask, constrained, P

        def every(value, dtype=torch.float32):
            return torch.full((B,), value, dtype=dtype, device=dev)
        self.gain, self.head_bits = gain, head_bits
        if head_bits == 8:
            self.w, self.w_scales = T.trie_head_quantize_weight(weight)
        else:
            self.w, self.w_scales, self.w_row_scales = T.trie_head4_quantize(weight)
        self.embedding = weight.to(torch.float32) * D ** 0.5
        self.hidden = torch.zeros(B, D, device=dev)
        self.logits = torch.empty(B, V, dtype=torch.bfloat16, device=dev)
        self.head_space = torch.empty(T.trie_head_workspace(B, V), dtype=torch.uint8, device=dev)
        self.sample_space = torch.empty(T.trie_sample_workspace(B, V), dtype=torch.uint8, device=dev)
        self.history = torch.zeros(B, max_length, dtype=torch.int32, device=dev)
        self.history[:, :P] = prompts
        self.prompt = every(P, torch.int32)
        self.length = every(P, torch.int32)
        self.tokens = self.history[:, P - 1].clone()
        self.logprobs = every(0.0)
        self.states = every(T.TRIE_STATE_FREE, torch.int32)
        self.states[:constrained] = h.root(0)
        self.err = torch.zeros(1, dtype=torch.int32, device=dev)
        self.seeds = torch.arange(seed, seed + B, dtype=torch.int64, device=dev) << 32  # plus the step
        self.ways = dict(temperature=every(temperature), top_k=every(top_k, torch.int32), top_p=every(top_p),
                         min_p=every(min_p))
        self.penalties = dict(repetition=every(repetition), presence=every(presence), frequency=every(frequency))
        # free rows may not stop here: a bias of -inf on the last token, none for the constrained rows
        free = torch.arange(B + 1, device=dev, dtype=torch.int32) - constrained
        self.bias = (free.clamp_(min=0), every(V - 1, torch.int32), every(-float("inf")))
        self.graph = None

    @property
    def weight(self):
        """The head's weights as its call takes them."""
        return (self.w, self.w_scales) if self.head_bits == 8 else (self.w, self.w_scales, self.w_row_scales)

    def head(self) -> None:
        """self.logits of self.hidden under the grammar."""
        rows = (self.logits, self.mask, self.states, self.head_space)
        if self.head_bits == 8:
            x = T.trie_head_quantize(self.hidden) if self.gain is None else T.trie_head_norm_quantize(self.hidden, self.gain)
            T.trie_head_logits(*x, *self.weight, *rows)
        else:
            x = T.trie_head4_quantize(self.hidden) if self.gain is None else T.trie_head4_norm_quantize(self.hidden, self.gain)
            T.trie_head4_logits(*x, *self.weight, *rows)

    def step(self) -> None:
        """One token for every row. Only the stream's work: nothing is read back."""
        import torch
        # the stand-in model
        last = self.embedding.index_select(0, self.tokens.clamp(min=0))
        self.hidden.copy_(torch.nn.functional.normalize(self.hidden.roll(1, dims=1) * 0.5 + last, dim=1) * 8.0)
        # the head under the grammar, penalties, the draw
        self.head()
        T.trie_penalize(self.logits, self.history, self.length, self.prompt, bias=self.bias, **self.penalties)
        T.trie_sample(self.logits, self.seeds, mask=self.mask, states=self.states, tokens=self.tokens,
                      logprobs=self.logprobs, workspace=self.sample_space, **self.ways)
        # what was said, and where the constrained rows are now
        at = self.length.clamp(max=self.history.shape[1] - 1).long()
        self.history.scatter_(1, at[:, None], self.tokens[:, None])
        self.length.add_(1).clamp_(max=self.history.shape[1])
        if self.constrained:
            T.trie_advance(self.h, self.states[:self.constrained], self.tokens[:self.constrained], self.err)
        self.seeds.add_(1)

    def run(self, steps: int) -> None:
        """`steps` tokens a row: the first by step(), which also records what a capture may not, the others by a graph of it."""
        import torch
        for _ in range(min(1, steps)):
            self.step()
        if steps > 1 and self.graph is None:
            self.graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(self.graph):
                self.step()
        for _ in range(steps - 1):
            self.graph.replay()

    def outputs(self):
        """Token ids after the prompt, one list a row (a constrained row's up to its last token's id V - 1)."""
        V = self.logits.shape[1]
        rows = []
        for b, row in enumerate(self.history.cpu().tolist()):
            said = row[self.P:int(self.length[b])]
            rows.append(said[:said.index(V - 1)] if b < self.constrained and V - 1 in said else said)
        return rows


def example(batch: int = 16, constrained: int = 8, steps: int = 48, D: int = 512, seed: int = 0, head_bits: int = 8,
            norm: bool = False):
    """Decodes with the tool names as the set. Returns (loop, the workload, texts of the rows)."""
    import torch
    w = W.config(1)
    h = T.trie_build(w.set_bytes, w.set_offsets)
    mask = T.alloc_mask(h, w.V)
    T.trie_compile_masks(h, w.vocab_bytes, w.vocab_offsets, w.V, mask)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    weight = (torch.randn(w.V, D, generator=g, device="cuda") / D ** 0.5).to(torch.bfloat16)
    prompts = torch.randint(0, w.V - 1, (batch, 4), generator=g, device="cuda", dtype=torch.int32)
    gain = torch.rand(D, generator=g, device="cuda") + 0.5 if norm else None
    loop = DecodeLoop(h, mask, weight, prompts, constrained, 4 + steps, head_bits=head_bits, gain=gain, seed=seed)
    loop.run(steps)
    vocab = W.unpack(w.vocab_bytes, w.vocab_offsets)
    return loop, w, [b"".join(vocab[t] for t in row) for row in loop.outputs()]


def main() -> None:
    p = argparse.ArgumentParser(description=__doc__.split("\n", 1)[0])
    p.add_argument("--batch", type=int, default=16)
    p.add_argument("--constrained", type=int, default=8)
    p.add_argument("--steps", type=int, default=48)
    p.add_argument("--bits", type=int, choices=(4, 8), default=8)
    p.add_argument("--norm", action="store_true")
    a = p.parse_args()
    loop, _, texts = example(a.batch, a.constrained, a.steps, head_bits=a.bits, norm=a.norm)
    for b, text in enumerate(texts):
        kind = "constrained" if b < a.constrained else "free"
        print(f"{b:3d} {kind:11s} {text[:60]!r}")


if __name__ == "__main__":
    main()
