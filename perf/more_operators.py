"""The cases that the operators before the logits head and after the sampler are measured on.

norm      root-mean-square norm of hidden states, with the residual's addition, into the 8-bit floating point
          (e4m3, a scale for each row and 128 columns) that the 8-bit logits head reads.
head4     logits from hidden states by a weight matrix in microscaled 4-bit floating point: e2m1 values, an
          e4m3 scale for each 16 columns of a row, a 32-bit scale for each row. The hidden states are
          quantized the same way within the call, by themselves or by the norm in front of it. With a
          grammar, only tokens that a row's state allows get a logit, the others -inf.
policy    the clipped policy loss with a KL term of sampled tokens, from their logits at the temperature and
          under the grammar that they were sampled with, and its gradient by the logits.

A grammar is a mask (a row of bits for every state, token v in bit v % 32 of word v / 32) and a state for
each row of the batch: a row of the mask, FREE (no grammar: every token), or anything else (only the end
of the sequence, token V - 1).
"""
from __future__ import annotations

import math

import torch

own = False

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2, "none": 0}
_FREE, _FINISHED, _DEAD = -3, -2, -1
_EPS = 1e-6
_CLIP, _KL = (0.2, 0.28), 0.05
_TINY = 2.0**-100  # the smallest scale of a row in 4 bits


def listed():
    return [
        # one request's next token
        dict(name="norm-M1-D4096-bf16", op="norm", M=1, D=4096, dtype="bf16", residual="bf16"),
        # a full batch of a decode step, the residual kept in 32 bits
        dict(name="norm-M256-D4096-bf16-f32", op="norm", M=256, D=4096, dtype="bf16", residual="f32"),
        # every position of a prompt is scored, all in 32 bits; the hidden size is not a multiple of 128
        dict(name="norm-M1000-D4112-f32", op="norm", M=1000, D=4112, dtype="f32", residual="f32"),
        # the positions of many prompts
        dict(name="norm-M16384-D5120-bf16", op="norm", M=16384, D=5120, dtype="bf16", residual="bf16"),
        # one request's next token, small model: the latency of the smallest head
        dict(name="head4-M1-V32000-D2048-bf16", op="head4", M=1, V=32000, D=2048, dtype="bf16", grammar=0.0, norm=False),
        # a full batch, the model's last norm in front of the head
        dict(name="head4-M256-V152064-D4096-norm", op="head4", M=256, V=152064, D=4096, dtype="bf16", grammar=0.0, norm=True),
        # the same batch where every request is constrained: few tokens are possible
        dict(name="head4-M256-V152064-D4096-grammar", op="head4", M=256, V=152064, D=4096, dtype="bf16", grammar=1.0,
             norm=True),
        # every position of a prompt is scored, logits kept in 32 bits, a vocabulary with added tokens and no padding
        dict(name="head4-M1000-V128011-D4112-f32", op="head4", M=1000, V=128011, D=4112, dtype="f32", grammar=0.0, norm=False),
        # the loss alone, to watch a small run
        dict(name="policy-B64-V32000-f32", op="policy", B=64, V=32000, dtype="f32", grammar=0.0, grad=False, ref=True),
        # a micro-batch of long answers, with the gradient
        dict(name="policy-B4096-V152064-bf16-grad", op="policy", B=4096, V=152064, dtype="bf16", grammar=0.0, grad=True, ref=True),
        # answers of which half the tokens were sampled under a grammar; rows at any two-byte boundary
        dict(name="policy-B1024-V128011-grammar-grad", op="policy", B=1024, V=128011, dtype="bf16", grammar=0.5, grad=True,
             ref=False),
        # logits kept in 32 bits, a large vocabulary
        dict(name="policy-B300-V262144-f32-grad", op="policy", B=300, V=262144, dtype="f32", grammar=0.0, grad=True, ref=True),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of lo..hi."""
    return min(hi, int(lo * (hi / lo) ** rng.random()))


def _hidden_size(rng, hi):
    if rng.random() < 0.6:
        return rng.choice([d for d in (512, 1024, 1536, 2048, 2560, 4096, 5120, 8192) if d <= hi])
    return _spread(rng, 512, hi) | 1 if rng.random() < 0.5 else _spread(rng, 512, hi) // 16 * 16


def draw(rng):
    op = rng.choice(["norm", "head4", "policy"])
    case = dict(op=op, dtype=rng.choice(["f32", "bf16"]))
    if op == "norm":
        D = _hidden_size(rng, 8192)
        case["residual"] = rng.choice(["none", "bf16", "f32"])
        per_value = 1 + _SIZE[case["dtype"]] + 2 * _SIZE[case["residual"]]
        case.update(M=min(_spread(rng, 1, 16384), 16384 * 5120 * 7 // (D * per_value)), D=D)
        return case
    V = _spread(rng, 32000, 262144)
    if rng.random() < 0.6:  # most vocabularies are padded to a multiple of 64, the others are of any size
        V = max(32000, V // 64 * 64)
    case.update(V=V, grammar=rng.choice([0.0, 0.0, 0.5, 1.0]))
    if op == "head4":
        D = _hidden_size(rng, 5120)
        D = min(D, 152064 * 4096 // V)
        M = _spread(rng, 1, 1000)
        case.update(M=max(1, min(M, 1000 * 128000 * 4096 // (V * D), int(512e6 / (V * _SIZE[case["dtype"]])))), D=D,
                    norm=rng.random() < 0.5)
        return case
    B = _spread(rng, 1, 4096)
    case.update(B=max(1, min(B, int(1.24e9 / (V * _SIZE[case["dtype"]])))), grad=rng.random() < 0.7, ref=rng.random() < 0.7)
    return case


# ------------------------------------------------------------------- inputs

def _grammar(g, rows, V, share):
    """The masks of 4,096 trie nodes and a state for each row. A node allows 1 to 72 tokens out of the
    3,000 that a set's strings are spelled with, some nodes allow the end of the sequence; of the
    constrained rows one in 16 has finished or left its set."""
    dev, nodes = "cuda", 4096
    words = (V + 31) // 32
    pool = torch.randint(0, V - 1, (3000,), generator=g, device=dev)
    many = torch.exp(torch.rand(nodes, generator=g, device=dev) * math.log(72.0)).long().clamp(1, 72)
    pick = pool[torch.randint(0, 3000, (nodes, 72), generator=g, device=dev)]
    node = torch.arange(nodes, device=dev)[:, None].expand(nodes, 72)
    used = torch.arange(72, device=dev)[None, :] < many[:, None]
    ends = torch.nonzero(torch.rand(nodes, generator=g, device=dev) < 0.3)[:, 0]
    bit = torch.unique(torch.cat([(node * (words * 32) + pick)[used], ends * (words * 32) + V - 1]))
    mask = torch.zeros(nodes * words, dtype=torch.int64, device=dev)
    mask.index_add_(0, bit // 32, torch.ones_like(bit) << (bit % 32))
    mask = (mask - ((mask >> 31) << 32)).to(torch.int32).view(nodes, words)
    states = torch.randint(0, nodes, (rows,), generator=g, device=dev)
    kind = torch.rand(rows, generator=g, device=dev)
    states = torch.where(kind < 1 / 32, torch.full_like(states, _FINISHED), states)
    states = torch.where(kind > 31 / 32, torch.full_like(states, _DEAD), states)
    free = torch.rand(rows, generator=g, device=dev) >= share
    return mask, torch.where(free, torch.full_like(states, _FREE), states).to(torch.int32)


def _choose(g, n, values, dtype):
    of = torch.tensor(values, dtype=dtype, device="cuda")
    return of[torch.randint(0, len(values), (n,), generator=g, device="cuda")]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(17000 + seed)
    rows = case["B"] if case["op"] == "policy" else case["M"]
    st = {"op": case["op"], "mask": None, "states": None}
    if case["op"] != "norm":
        st["V"] = case["V"]
        if case["grammar"] > 0:
            st["mask"], st["states"] = _grammar(g, rows, case["V"], case["grammar"])
    if case["op"] == "policy":
        return _prepare_policy(case, g, st)
    D, dtype = case["D"], _TYPE[case["dtype"]]
    # a few channels of a model's hidden states are much larger than the others
    channel = torch.exp(torch.randn(D, generator=g, device="cuda") * 0.7)
    st["x"] = (torch.randn(rows, D, generator=g, device="cuda") * channel).to(dtype)
    st["D"], st["residual"], st["gain"] = D, None, None
    if case["op"] == "norm" or case["norm"]:
        kind = case.get("residual", case["dtype"])
        if kind != "none":
            st["residual"] = (torch.randn(rows, D, generator=g, device="cuda") * channel * 4.0).to(_TYPE[kind])
        st["gain"] = (1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(dtype)
    if case["op"] == "head4":
        w = torch.randn(case["V"], D, generator=g, device="cuda", dtype=torch.bfloat16)
        w *= torch.exp(torch.randn(case["V"], 1, generator=g, device="cuda") * 0.25) / math.sqrt(D)
        st["w"], st["w_scales"], st["w_row_scales"] = _packed_weight(w)
        st["logits"] = torch.empty(rows, case["V"], device="cuda", dtype=dtype)
    return st


def _packed_weight(w):
    """Weights as a program keeps them: two 4-bit codes a byte, the even column's in the low half, rows filled
    up with zeros to 32 columns; scales of 128 rows x 64 columns together, as [row / 128][column / 64][row % 32]
    [row % 128 / 32][column % 64 / 16]."""
    V, D = w.shape
    value, block, row = _quantized4(w.float())
    size = value.abs()
    code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8)
    code += (torch.signbit(value) & (size > 0)) * 8
    code = torch.nn.functional.pad(code, (0, -D % 32))
    pv, pk = -V % 128, -block.shape[1] % 4
    block = torch.nn.functional.pad(block, (0, pk, 0, pv))
    block = block.view((V + pv) // 128, 4, 32, (D + 63) // 64, 4).permute(0, 3, 2, 1, 4)
    return code[:, ::2] | (code[:, 1::2] << 4), block.to(torch.float8_e4m3fn).contiguous(), row


def _prepare_policy(case, g, st):
    B, V, dtype = case["B"], case["V"], _TYPE[case["dtype"]]
    # a broad bulk, and in each row up to 64 tokens that stand out
    x = torch.randn(B, V, generator=g, device="cuda") * 2.0
    at = torch.randint(0, V, (B, 64), generator=g, device="cuda")
    lift = torch.rand(B, 64, generator=g, device="cuda") * torch.rand(B, 1, generator=g, device="cuda") * 14.0
    st["logits"] = x.scatter_add_(1, at, lift).to(dtype)
    del x, at, lift
    st["temperature"] = _choose(g, B, [0.7, 1.0, 1.0, 1.2], torch.float32)
    # tokens as sampled from these logits, log-probabilities of a slightly older policy and of a reference
    noise = torch.rand(B, V, generator=g, device="cuda").clamp_(min=2.0**-25)
    score = st["logits"].float() / st["temperature"][:, None]
    ok = _allowed(st)
    if ok is not None:
        score = torch.where(ok, score, -math.inf)
    best = (score - torch.log_(-torch.log_(noise))).argmax(dim=1, keepdim=True)
    lp = (score.gather(1, best) - torch.logsumexp(score, dim=1, keepdim=True))[:, 0]
    del noise, score, ok
    st["old"] = lp + 0.15 * torch.randn(B, generator=g, device="cuda")
    st["ref"] = lp + 0.4 * torch.randn(B, generator=g, device="cuda") if case["ref"] else None
    st["advantages"] = torch.randn(B, generator=g, device="cuda")
    # one row in 32 is behind the end of its answer
    padding = torch.rand(B, generator=g, device="cuda") < 1 / 32
    st["tokens"] = torch.where(padding, -1, best[:, 0]).to(torch.int32)
    st["weights"] = torch.where(padding, 0.0, 1.0 / B)
    st["grad"] = torch.empty_like(st["logits"]) if case["grad"] else None
    return st


# ---------------------------------------------------------------------- run

def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "norm":
        return _norm(st)
    if st["op"] == "head4":
        return _head4(st)
    return _policy(st)


def _run_own(st):
    from paper_2608_12574_gb300 import triemask as T
    if st["op"] == "norm":
        q, scales = T.trie_head_norm_quantize(st["x"], st["gain"], st["residual"], eps=_EPS)
        return [q, scales[:, :q.shape[0]], st["residual"]]
    grammar = dict(mask=st["mask"], states=st["states"])
    if st["op"] == "head4":
        if st["gain"] is None:
            x = T.trie_head4_quantize(st["x"])
        else:
            x = T.trie_head4_norm_quantize(st["x"], st["gain"], st["residual"], eps=_EPS)
        T.trie_head4_logits(*x, st["w"], st["w_scales"], st["w_row_scales"], st["logits"], **grammar)
        return [st["logits"], st["residual"]]
    losses, logprobs = T.trie_policy_loss(
        st["logits"], st["tokens"], st["old"], st["advantages"], ref_logprobs=st["ref"], weights=st["weights"],
        temperature=st["temperature"], clip=_CLIP, kl=_KL, grad=st["grad"], **grammar)
    return [losses, logprobs, st["grad"]]


def _allowed(st):
    """bool [rows, V]: which tokens each row's state allows; None without a grammar."""
    mask, states, V = st["mask"], st["states"], st["V"]
    if mask is None:
        return None
    bits = mask[states.clamp(0, mask.shape[0] - 1).long()][:, :, None] >> torch.arange(32, device="cuda", dtype=torch.int32)
    bits = (bits & 1).bool().flatten(1)[:, :V]
    node = (states >= 0) & (states < mask.shape[0])
    end = torch.arange(V, device="cuda") == V - 1
    return torch.where(node[:, None], bits, end) | (states == _FREE)[:, None]


def _normalized(st):
    """The normed rows in 32 bits; the residual is brought up to date."""
    h = st["x"].float()
    if st["residual"] is not None:
        h = st["residual"].copy_(h + st["residual"].float()).float()
    # the values lie next to the borders of 8 and 4 bits: the mean in 64
    r = (1.0 / torch.sqrt(h.double().square().mean(dim=1, keepdim=True) + _EPS)).float()
    return h * r * st["gain"].float()


def _norm(st):
    y = _normalized(st)
    M, D = y.shape
    blocks = torch.nn.functional.pad(y, (0, -D % 128)).view(M, -1, 128)
    scale = blocks.abs().amax(dim=2, keepdim=True) * (1.0 / 448.0)
    scale = torch.where(scale > 0, scale, 1.0)
    q = (blocks / scale).to(torch.float8_e4m3fn).view(M, -1)[:, :D].contiguous()
    return [q, scale[:, :, 0].T.contiguous(), st["residual"]]


def _quantized4(x):
    """(e2m1 values, e4m3 scales of 16 columns, scales of the rows) of x in 32 bits."""
    M, D = x.shape
    row = (x.abs().amax(dim=1) * (1.0 / 2688.0)).clamp(min=_TINY)
    x = torch.nn.functional.pad(x, (0, -D % 16)).view(M, -1, 16)
    block = x.abs().amax(dim=2) / row[:, None] * (1.0 / 6.0)
    block = block.clamp(max=448.0).to(torch.float8_e4m3fn).float()
    step = block * row[:, None]
    x = x * torch.where(step > 0, 1.0 / step, 0.0)[:, :, None]
    size = x.abs()
    value = 0.5 * (size > 0.25) + 0.5 * (size >= 0.75) + 0.5 * (size > 1.25) + 0.5 * (size >= 1.75)
    value = value + 1.0 * (size > 2.5) + 1.0 * (size >= 3.5) + 2.0 * (size > 5.0)
    return torch.where(x < 0, -value, value).view(M, -1)[:, :D], block, row


def _head4(st):
    V, D = st["V"], st["D"]
    x = st["x"].float() if st["gain"] is None else _normalized(st)
    value, block, row = _quantized4(x)
    x = value * block.repeat_interleave(16, dim=1)[:, :D] * row[:, None]
    of = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    code = st["w"]
    w = of[torch.stack([code & 15, code >> 4], dim=2).flatten(1)[:, :D].int()]
    scale = st["w_scales"].float().permute(0, 3, 2, 1, 4).flatten(0, 2).flatten(1)[:V]
    w = w * scale.repeat_interleave(16, dim=1)[:, :D] * st["w_row_scales"][:, None]
    y = x @ w.T
    ok = _allowed(st)
    if ok is not None:
        y = torch.where(ok, y, -math.inf)
    return [st["logits"].copy_(y), st["residual"]]


def _policy(st):
    V, x = st["V"], st["logits"].float()
    ok = _allowed(st)
    if ok is not None:
        x = torch.where(ok, x, -math.inf)
    T = st["temperature"][:, None]
    y = (x - x.amax(dim=1, keepdim=True)) / T
    y = y - torch.log(torch.exp(y).sum(dim=1, keepdim=True))
    token = st["tokens"].clamp(min=0).long()[:, None]
    lp = y.gather(1, token)[:, 0]
    known = (st["tokens"] >= 0) & (st["tokens"] < V) & (lp != -math.inf)
    A, w = st["advantages"], st["weights"]
    rho = torch.exp(lp - st["old"])
    free, held = rho * A, rho.clamp(1.0 - _CLIP[0], 1.0 + _CLIP[1]) * A
    loss, slope = -torch.minimum(free, held), -torch.where(free <= held, free, 0.0)
    if st["ref"] is not None:
        d = st["ref"] - lp
        loss = loss + _KL * (torch.exp(d) - d - 1.0)
        slope = slope + _KL * (1.0 - torch.exp(d))
    there = known & (w != 0)
    loss = torch.where(there, w * loss, 0.0)
    lp = torch.where(known, lp, -math.inf)
    if st["grad"] is None:
        return [loss, lp, None]
    slope = torch.where(there, w * slope, 0.0)[:, None] / T
    grad = -slope * torch.exp(y)
    grad = grad.scatter_add_(1, token, slope)
    return [loss, lp, st["grad"].copy_(grad)]


# --------------------------------------------------------------------- work

def _possible():
    """Tokens that a constrained row allows, about (the mean of 1 to 72 spread over the logarithm)."""
    return 17


def work(case):
    size = _SIZE[case["dtype"]]
    if case["op"] == "norm":
        M, D = case["M"], case["D"]
        n_bytes = M * D * (size + 2 * _SIZE[case["residual"]] + 1) + D * size + 4 * M * ((D + 127) // 128)
        return {"bytes": n_bytes, "flops": 8.0 * M * D}
    V, share = case["V"], case["grammar"]
    rows = case["B"] if case["op"] == "policy" else case["M"]
    masks = share * rows * ((V + 31) // 32) * 4
    if case["op"] == "head4":
        D = case["D"]
        # with a grammar in every row: the weights of the tokens that some row allows
        tokens = V if share < 1 else min(V, int(3000 * (1 - math.exp(-rows * _possible() / 3000))))
        per_row = (1 - share) * V + share * _possible()
        n_bytes = tokens * (D * 9 // 16 + 4) + rows * D * size + rows * V * size
        if case["norm"]:
            n_bytes += 2 * rows * D * size
        return {"bytes": n_bytes + masks, "flops": 2.0 * rows * per_row * D}
    seen = (1 - share) * V + share * _possible()
    n_bytes = rows * seen * size + masks + 28 * rows + (rows * V * size if case["grad"] else 0)
    return {"bytes": n_bytes, "flops": (8.0 if case["grad"] else 4.0) * rows * seen}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """By the definitions, in 64 bits (but for the roundings that a definition names)."""
    st = prepare(case, seed)
    if case["op"] == "policy":
        return _exact_policy(st)
    x, residual = st["x"].double(), None
    if st["residual"] is not None:
        residual = x + st["residual"].double()
        x = residual.float().to(st["residual"].dtype).double()
    if st["gain"] is not None:
        x = _exact_rounded(x * _exact_rounded(torch.rsqrt((x * x).mean(1) + _EPS))[:, None])
        x = _exact_rounded(x * st["gain"].double())
    if case["op"] == "norm":
        return [*_exact_e4m3(x), residual]
    x, w = _exact_e2m1(x), _exact_weight(st)
    y = x @ w.T
    if st["mask"] is not None:
        for b in range(len(y)):
            tokens = _exact_row(st, b)
            if tokens is not None:
                row = torch.full_like(y[b], -math.inf)
                row[tokens] = y[b, tokens]
                y[b] = row
    return [y, residual]


def _exact_rounded(v):
    return v.float().double()


def _exact_row(st, b):
    """The tokens that row b allows, ascending; None for all."""
    if st["mask"] is None or int(st["states"][b]) == _FREE:
        return None
    s, V = int(st["states"][b]), st["V"]
    if not 0 <= s < st["mask"].shape[0]:
        return torch.tensor([V - 1], device="cuda")
    words = st["mask"][s].long() & 0xFFFFFFFF
    full = torch.nonzero(words)[:, 0]
    bits = (words[full][:, None] // 2 ** torch.arange(32, device="cuda")) % 2
    tokens = (full[:, None] * 32 + torch.arange(32, device="cuda"))[bits == 1]
    return tokens[tokens < V]


def _exact_e4m3(y):
    M, D = y.shape
    q, scales = torch.zeros_like(y), []
    for k in range(0, D, 128):
        part = y[:, k:k + 128].float()
        s = part.abs().amax(dim=1) * torch.tensor(1 / 448, dtype=torch.float32, device="cuda")
        s[s == 0] = 1.0
        q[:, k:k + 128] = (part / s[:, None]).to(torch.float8_e4m3fn).double()
        scales.append(s.double())
    return [q, torch.stack(scales)]


def _exact_e2m1(y):
    """Dequantized rows: each value the nearest of the grid, of two as near the one with an even code."""
    M, D = y.shape
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64, device="cuda")
    border = (grid[1:] + grid[:-1]) / 2
    f32 = dict(dtype=torch.float32, device="cuda")
    row = torch.maximum(y.float().abs().amax(dim=1) * torch.tensor(1 / 2688, **f32), torch.tensor(_TINY, **f32))
    out = torch.zeros_like(y)
    for k in range(0, D, 16):
        part = y[:, k:k + 16].float()
        t = part.abs().amax(dim=1) / row * torch.tensor(1 / 6, **f32)
        s = t.clamp(max=448).to(torch.float8_e4m3fn).float()
        step = s * row
        u = (part * torch.where(step > 0, 1 / step, torch.zeros_like(step))[:, None]).double()
        below = torch.bucketize(u.abs(), border)               # borders below |u|
        above = torch.bucketize(u.abs(), border, right=True)   # borders not above |u|
        code = torch.where((below != above) & (above % 2 == 0), above, below)
        out[:, k:k + 16] = grid[code] * u.sign() * s[:, None].double() * row[:, None].double()
    return out


def _exact_weight(st):
    V, D = st["V"], st["D"]
    code = torch.stack([st["w"] & 15, st["w"] >> 4], dim=2).view(V, -1)[:, :D]
    part = code & 1
    power = ((code >> 1) & 3).double()
    w = torch.where(power > 0, (1 + part * 0.5) * 2 ** (power - 1), part * 0.5) * (1 - 2 * (code >> 3).double())
    v = torch.arange(V, device="cuda")[:, None]
    k = torch.arange((D + 15) // 16, device="cuda")[None, :] * 16
    scale = st["w_scales"].view(torch.uint8)[v // 128, k // 64, v % 32, v % 128 // 32, k % 64 // 16]
    scale = scale.view(torch.float8_e4m3fn).double() * st["w_row_scales"].double()[:, None]
    return w * scale[:, torch.arange(D, device="cuda") // 16]


def _exact_policy(st):
    B, V = st["logits"].shape
    loss, logprob = [], []
    grad = None if st["grad"] is None else torch.zeros(B, V, dtype=torch.float64, device="cuda")
    column = {k: (st[k].tolist() if st[k] is not None else None) for k in
              ("tokens", "old", "ref", "advantages", "weights", "temperature")}
    for b in range(B):
        ids = _exact_row(st, b)
        y = st["logits"][b].double() / column["temperature"][b]
        y = y if ids is None else y[ids]
        lse = torch.logsumexp(y, 0)
        t = column["tokens"][b]
        at = None
        if t >= 0:
            at = t if ids is None else (ids == t).nonzero().flatten().tolist()
            at = (at[0] if at else None) if isinstance(at, list) else at
        if at is None:
            loss.append(0.0)
            logprob.append(-math.inf)
            continue
        lp = float(y[at] - lse)
        logprob.append(lp)
        w, A = column["weights"][b], column["advantages"][b]
        rho = math.exp(lp - column["old"][b])
        free, held = rho * A, min(max(rho, 1 - _CLIP[0]), 1 + _CLIP[1]) * A
        value, slope = -min(free, held), -free if free <= held else 0.0
        if column["ref"] is not None:
            d = column["ref"][b] - lp
            value += _KL * (math.expm1(d) - d)
            slope -= _KL * math.expm1(d)
        loss.append(w * value)
        if grad is not None and w != 0:
            slope = w * slope / column["temperature"][b]
            p = -slope * torch.exp(y - lse)
            p[at] += slope
            if ids is None:
                grad[b] = p
            else:
                grad[b, ids] = p
    return [torch.tensor(loss, dtype=torch.float64), torch.tensor(logprob, dtype=torch.float64), grad]
