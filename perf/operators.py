"""The cases that the operators around a grammar mask are measured on: from a model's last hidden
states to the sampled token.

head      logits from hidden states by a weight matrix in 8-bit floating point (e4m3) with a scale for
          each block of 128 x 128 weights; the hidden states arrive in 16 or 32 bits and are quantized
          within the call, a scale for each row and 128 columns. With a grammar, only tokens that a
          row's state allows get a logit, the others -inf.
penalize  repetition, presence and frequency penalties, biases and the grammar mask, on logits in place.
sample    temperature, top-k, top-p, min-p and the draw of a token, with its log-probability.

A grammar is a mask (a row of bits for every state, token v in bit v % 32 of word v / 32) and a state for
each row of the batch: a row of the mask, FREE (no grammar: every token), or anything else (only the end
of the sequence, token V - 1). Random numbers are a function of a seed for each row, which is an input.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_FREE, _FINISHED, _DEAD = -3, -2, -1
_BLOCK = 128   # columns (and, for weights, rows) that share a scale
_GROUP = 256   # tokens whose group is drawn before the token is
_FP8_MAX = 448.0


def listed():
    return [
        # one request's next token, small model: the latency of the smallest head
        dict(name="head-M1-V32000-D2048-bf16", op="head", M=1, V=32000, D=2048, dtype="bf16", grammar=0.0),
        # a mid-sized batch, a vocabulary with added tokens and no padding
        dict(name="head-M64-V128011-D4096-bf16", op="head", M=64, V=128011, D=4096, dtype="bf16", grammar=0.0),
        # a full batch
        dict(name="head-M256-V152064-D4096-bf16", op="head", M=256, V=152064, D=4096, dtype="bf16", grammar=0.0),
        # the same batch where every request is constrained: few tokens are possible
        dict(name="head-M256-V152064-D4096-grammar", op="head", M=256, V=152064, D=4096, dtype="bf16", grammar=1.0),
        # every position of a prompt is scored, logits kept in 32 bits; hidden size not a multiple of 128
        dict(name="head-M1000-V128000-D4112-f32", op="head", M=1000, V=128000, D=4112, dtype="f32", grammar=0.0),
        # one chat request early in its answer
        dict(name="penalize-B1-V32000-H300-f32", op="penalize", B=1, V=32000, H=300, bias=8, dtype="f32", grammar=0.0),
        # a full batch, half of it constrained, ordinary prompts
        dict(name="penalize-B256-V152064-H2000", op="penalize", B=256, V=152064, H=2000, bias=16, dtype="bf16",
             grammar=0.5),
        # long documents in the prompts, long lists of banned tokens, rows at any two-byte boundary
        dict(name="penalize-B48-V128011-H32768", op="penalize", B=48, V=128011, H=32768, bias=300, dtype="bf16",
             grammar=0.25),
        # one chat request: top-k and top-p, the latency of the smallest call
        dict(name="sample-B1-V32000-f32", op="sample", B=1, V=32000, dtype="f32", grammar=0.0, ways="chat"),
        # a full batch of chat requests
        dict(name="sample-B256-V152064-bf16", op="sample", B=256, V=152064, dtype="bf16", grammar=0.0, ways="chat"),
        # rollouts and requests of every kind side by side, logits kept in 32 bits
        dict(name="sample-B64-V262144-f32", op="sample", B=64, V=262144, dtype="f32", grammar=0.0, ways="mixed"),
        # most requests constrained, an odd vocabulary
        dict(name="sample-B200-V128011-grammar", op="sample", B=200, V=128011, dtype="bf16", grammar=0.75, ways="mixed"),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread over the logarithm of lo..hi."""
    return min(hi, int(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["head", "penalize", "sample"])
    V = _spread(rng, 32000, 262144)
    if rng.random() < 0.6:  # most vocabularies are padded to a multiple of 64, the others are of any size
        V = max(32000, V // 64 * 64)
    case = dict(op=op, V=V, dtype=rng.choice(["f32", "bf16"]), grammar=rng.choice([0.0, 0.0, 0.5, 1.0]))
    if op == "head":
        D = rng.choice([1024, 1536, 2048, 2560, 4096, 5120]) if rng.random() < 0.6 else _spread(rng, 1024, 5120) | 15
        if D % 128 or V * D > 152064 * 4096:  # an odd multiple of 16
            D = min(D, 152064 * 4096 // V) // 32 * 32 - 16
        M = _spread(rng, 1, 1000)
        case.update(M=max(1, min(M, 1000 * 128000 * 4096 // (V * D), int(512e6 / (V * _SIZE[case["dtype"]])))), D=D)
    else:
        B = _spread(rng, 1, 256)
        case["B"] = max(1, min(B, int(78e6 / (V * _SIZE[case["dtype"]]))))
    if op == "penalize":
        case.update(H=_spread(rng, 16, min(32768, 48 * 32768 // case["B"])) | 1, bias=rng.choice([0, 8, 300]))
    if op == "sample":
        case["ways"] = rng.choice(["chat", "mixed"])
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


def _logits(g, B, V, dtype):
    """Logits as a model's are: a broad bulk, and in each row up to 64 tokens that stand out."""
    x = torch.randn(B, V, generator=g, device="cuda") * 2.0
    at = torch.randint(0, V, (B, 64), generator=g, device="cuda")
    lift = torch.rand(B, 64, generator=g, device="cuda") * torch.rand(B, 1, generator=g, device="cuda") * 14.0
    return x.scatter_add_(1, at, lift).to(_TYPE[dtype])


def _choose(g, n, values, dtype):
    of = torch.tensor(values, dtype=dtype, device="cuda")
    return of[torch.randint(0, len(values), (n,), generator=g, device="cuda")]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(9000 + seed)
    op, V = case["op"], case["V"]
    st = {"op": op, "V": V, "mask": None, "states": None}
    rows = case["M"] if op == "head" else case["B"]
    if case["grammar"] > 0:
        st["mask"], st["states"] = _grammar(g, rows, V, case["grammar"])
    if op == "head":
        D = case["D"]
        w = torch.randn(V, D, generator=g, device="cuda", dtype=torch.bfloat16)
        w *= torch.exp(torch.randn(V, 1, generator=g, device="cuda") * 0.25) / math.sqrt(D)
        st["w"], st["w_scales"] = _quantized_weight(w)
        x = torch.randn(rows, D, generator=g, device="cuda")
        x *= torch.exp(torch.randn(D, generator=g, device="cuda") * 0.5) * 2.0
        st["x"] = x.to(_TYPE[case["dtype"]])
        st["logits"] = torch.empty(rows, V, device="cuda", dtype=_TYPE[case["dtype"]])
        return st
    st["logits"] = _logits(g, rows, V, case["dtype"])
    if op == "penalize":
        H = case["H"]
        # words of a text repeat as Zipf's law says; a prompt is most of a history
        tok = torch.exp(torch.rand(rows, H, generator=g, device="cuda") * math.log(V)).long() - 1
        st["history"] = ((tok * 7919 + 13) % V).to(torch.int32)
        st["length"] = torch.randint(max(1, H // 2), H + 1, (rows,), generator=g, device="cuda", dtype=torch.int32)
        st["prompt"] = (st["length"] * (0.5 + 0.5 * torch.rand(rows, generator=g, device="cuda"))).to(torch.int32)
        st["repetition"] = _choose(g, rows, [1.0, 1.05, 1.1, 1.3], torch.float32)
        st["presence"] = _choose(g, rows, [0.0, 0.2, 1.0, -0.5], torch.float32)
        st["frequency"] = _choose(g, rows, [0.0, 0.1, 0.5], torch.float32)
        st["bias"] = None
        if case["bias"]:
            n = case["bias"]
            tok = (torch.arange(n, device="cuda")[None, :] * (V // n)
                   + torch.randint(0, V // n, (rows, n), generator=g, device="cuda"))
            value = torch.randn(rows, n, generator=g, device="cuda") * 4.0
            value[:, ::4] = -math.inf  # banned
            st["bias"] = (torch.arange(0, rows * n + 1, n, device="cuda", dtype=torch.int32),
                          tok.to(torch.int32).flatten(), value.flatten())
    else:
        st["seeds"] = torch.randint(-2**62, 2**62, (rows,), generator=g, device="cuda")
        if case["ways"] == "chat":
            st["temperature"] = _choose(g, rows, [0.6, 0.7, 0.8, 1.0], torch.float32)
            st["top_k"] = _choose(g, rows, [20, 40, 50, 64], torch.int32)
            st["top_p"] = _choose(g, rows, [0.8, 0.9, 0.95], torch.float32)
            st["min_p"] = None
        else:
            st["temperature"] = _choose(g, rows, [0.0, 0.7, 1.0, 1.0, 1.2], torch.float32)
            st["top_k"] = _choose(g, rows, [0, 0, 0, 40, 1000], torch.int32)
            st["top_p"] = _choose(g, rows, [1.0, 1.0, 0.9, 0.95], torch.float32)
            st["min_p"] = _choose(g, rows, [0.0, 0.0, 0.05], torch.float32)
    return st


def _quantized_weight(w):
    """e4m3 weights with a scale for each block of 128 x 128, as a checkpoint holds them."""
    V, D = w.shape
    pv, pd = -V % _BLOCK, -D % _BLOCK
    blocks = torch.nn.functional.pad(w, (0, pd, 0, pv)).view((V + pv) // _BLOCK, _BLOCK, (D + pd) // _BLOCK, _BLOCK)
    scale = blocks.abs().amax(dim=(1, 3)).float() / _FP8_MAX
    q = (blocks / scale[:, None, :, None]).to(torch.float8_e4m3fn).view(V + pv, D + pd)
    return q[:V, :D].contiguous(), scale.contiguous()


# ---------------------------------------------------------------------- run

def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "head":
        return _head(st)
    if st["op"] == "penalize":
        return _penalize(st)
    return _sample(st)


def _run_own(st):
    from paper_2608_12574_gb300 import triemask as T
    grammar = dict(mask=st["mask"], states=st["states"])
    if st["op"] == "head":
        q, scales = T.trie_head_quantize(st["x"])
        T.trie_head_logits(q, scales, st["w"], st["w_scales"], st["logits"], **grammar)
        return st["logits"]
    if st["op"] == "penalize":
        T.trie_penalize(st["logits"], st["history"], st["length"], st["prompt"], repetition=st["repetition"],
                        presence=st["presence"], frequency=st["frequency"], bias=st["bias"], **grammar)
        return st["logits"]
    return T.trie_sample(st["logits"], st["seeds"], temperature=st["temperature"], top_k=st["top_k"],
                         top_p=st["top_p"], min_p=st["min_p"], **grammar)


def _allowed(st):
    """bool [rows, V]: which tokens each row's state allows; None without a grammar."""
    mask, states, V = st["mask"], st["states"], st["V"]
    if mask is None:
        return None
    bits = mask[states.clamp(0, mask.shape[0] - 1).long()][:, :, None] >> torch.arange(32, device="cuda")
    bits = (bits & 1).bool().flatten(1)[:, :V]
    node = (states >= 0) & (states < mask.shape[0])
    end = torch.arange(V, device="cuda") == V - 1
    return torch.where(node[:, None], bits, end) | (states == _FREE)[:, None]


def _head(st):
    x, w, V = st["x"].float(), st["w"], st["V"]
    M, D = x.shape
    pad = -D % _BLOCK
    x = torch.nn.functional.pad(x, (0, pad)).view(M, -1, _BLOCK)
    scale = x.abs().amax(dim=2, keepdim=True) / _FP8_MAX
    scale = torch.where(scale > 0, scale, torch.ones_like(scale))
    x = ((x / scale).to(torch.float8_e4m3fn).float() * scale).view(M, -1)[:, :D]
    by_row = st["w_scales"].repeat_interleave(_BLOCK, dim=0)[:V]
    w = w.float() * by_row.repeat_interleave(_BLOCK, dim=1)[:, :D]
    y = x @ w.T
    ok = _allowed(st)
    if ok is not None:
        y = torch.where(ok, y, -math.inf)
    return st["logits"].copy_(y)


def _penalize(st):
    V, history = st["V"], st["history"].long()
    B, H = history.shape
    at = torch.arange(H, device="cuda")[None, :]
    there = (at < st["length"][:, None]) & (history >= 0) & (history < V)
    where = torch.where(there, history, V)
    count = torch.zeros(B, V + 1, device="cuda")
    seen = count.scatter_add(1, where, there.float())[:, :V] > 0
    count = count.scatter_add(1, where, (there & (at >= st["prompt"][:, None])).float())[:, :V]
    x, r = st["logits"].float(), st["repetition"][:, None]
    x = torch.where(seen, torch.where(x > 0, x / r, x * r), x)
    x = x - st["frequency"][:, None] * count
    x = x - torch.where(count > 0, st["presence"][:, None], 0.0)
    if st["bias"] is not None:
        offsets, token, value = st["bias"]
        row = torch.searchsorted(offsets[1:], torch.arange(len(token), device="cuda"), right=True)
        x = x.index_put((row, token.long()), value, accumulate=True)
    ok = _allowed(st)
    if ok is not None:
        x = torch.where(ok, x, -math.inf)
    return st["logits"].copy_(x)


def _gumbel(seeds, n):
    """Gumbel noise number n of each seed: 23 bits of splitmix64."""
    def shifted(z, by):
        return (z >> by) & ((1 << (64 - by)) - 1)
    z = seeds[:, None] + (n + 1)[None, :] * -0x61C8864680B583EB
    z = (z ^ shifted(z, 30)) * -0x40A7B892E31B1A47
    z = (z ^ shifted(z, 27)) * -0x6B2FB644ECCEEE15
    z = z ^ shifted(z, 31)
    u = (2 * shifted(z, 41) + 1).float() * 2.0**-24
    return -torch.log(-torch.log(u))


def _sample(st):
    V, x = st["V"], st["logits"].float()
    B = x.shape[0]
    ok = _allowed(st)
    x = torch.where(torch.isnan(x) if ok is None else torch.isnan(x) | ~ok, -math.inf, x)
    greedy = (st["temperature"] == 0)[:, None]
    T = torch.where(greedy, 1.0, st["temperature"][:, None])
    top = x.amax(dim=1, keepdim=True)
    y = torch.where(x == top, torch.zeros_like(x), (x - top) / T)
    w = torch.where(x > -math.inf, torch.exp(y), 0.0)
    order = torch.sort(x, dim=1, descending=True, stable=True).indices
    k = torch.where(st["top_k"] > 0, st["top_k"], V)[:, None]
    first_k = torch.arange(V, device="cuda")[None, :] < k
    sorted_w = w.gather(1, order) * first_k
    total, before = sorted_w.sum(dim=1, keepdim=True), sorted_w.cumsum(dim=1) - sorted_w
    top_p = st["top_p"][:, None]
    keep = first_k & ((top_p >= 1) | (before < top_p * total))
    if st["min_p"] is not None:
        keep &= sorted_w >= st["min_p"][:, None]
    keep[:, 0] = True
    kept = torch.zeros_like(keep).scatter_(1, order, keep) & (w > 0)
    groups = (V + _GROUP - 1) // _GROUP
    mass = torch.nn.functional.pad(torch.where(kept, w, 0.0), (0, groups * _GROUP - V)).view(B, groups, _GROUP).sum(2)
    score = torch.log(mass) + _gumbel(st["seeds"], torch.arange(groups, device="cuda") + 2**31)
    group = score.argmax(dim=1, keepdim=True)
    ids = torch.arange(V, device="cuda")
    score = torch.where(kept & (ids[None, :] // _GROUP == group), y + _gumbel(st["seeds"], ids), -math.inf)
    token = torch.where(greedy, x.argmax(dim=1, keepdim=True), score.argmax(dim=1, keepdim=True))
    logprob = y.gather(1, token) - torch.log(w.sum(dim=1, keepdim=True))
    none = top == -math.inf
    return [torch.where(none, -1, token)[:, 0].to(torch.int32), torch.where(none, -math.inf, logprob)[:, 0]]


# --------------------------------------------------------------------- work

def _possible(case):
    """Tokens that a constrained row allows, about (the mean of 1 to 72 spread over the logarithm)."""
    return 17


def work(case):
    V, size, share = case["V"], _SIZE[case["dtype"]], case["grammar"]
    rows = case["M"] if case["op"] == "head" else case["B"]
    masks = share * rows * ((V + 31) // 32) * 4
    if case["op"] == "head":
        D = case["D"]
        # with a grammar in every row: the weights of the tokens that some row allows
        tokens = V if share < 1 else min(V, int(3000 * (1 - math.exp(-rows * _possible(case) / 3000))))
        per_row = (1 - share) * V + share * _possible(case)
        n_bytes = tokens * D + rows * D * size + rows * V * size + 4 * (tokens + 127) // 128 * ((D + 127) // 128)
        return {"bytes": n_bytes + masks, "flops": 2.0 * rows * per_row * D}
    if case["op"] == "penalize":
        H = 0.75 * case["H"]
        distinct = V / math.log(V) * math.log(1 + H * math.log(V) / V) + H / 2
        touched = min(V, min(H, distinct) + case["bias"])
        n_bytes = rows * (4 * H + 8 * case["bias"]) + (1 - share) * rows * 2 * size * touched + share * rows * V * size
        return {"bytes": n_bytes + masks, "flops": 4 * rows * touched}
    seen = (1 - share) * V + share * _possible(case)
    return {"bytes": rows * seen * size + masks + 40 * rows, "flops": 4 * rows * seen}


# -------------------------------------------------------------------- exact

def exact(case, seed):
    """By the definitions, in 64 bits."""
    st = prepare(case, seed)
    if case["op"] == "head":
        return _exact_head(st)
    if case["op"] == "penalize":
        return _exact_penalize(st)
    return _exact_sample(st)


def _exact_rows(st, b):
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


def _exact_head(st):
    x = st["x"].double()
    M, D = x.shape
    V = st["V"]
    out = torch.zeros(M, V, dtype=torch.float64, device="cuda")
    for i, k in enumerate(range(0, D, _BLOCK)):
        part = st["x"][:, k:k + _BLOCK].float()
        scale = part.abs().amax(dim=1) / _FP8_MAX  # the scale and the 8-bit values are 32-bit roundings by definition
        scale[scale == 0] = 1.0
        q = (part / scale[:, None]).to(torch.float8_e4m3fn).double() * scale[:, None].double()
        column = st["w_scales"][:, i].double().repeat_interleave(_BLOCK)[:V]
        out += q @ (st["w"][:, k:k + _BLOCK].double() * column[:, None]).T
    for b in range(M):
        tokens = _exact_rows(st, b)
        if tokens is not None:
            row = torch.full_like(out[b], -math.inf)
            row[tokens] = out[b, tokens]
            out[b] = row
    return out


def _exact_penalize(st):
    out = st["logits"].double()
    for b in range(out.shape[0]):
        n, p = int(st["length"][b]), int(st["prompt"][b])
        said = st["history"][b, :n].long()
        for tokens, count in [torch.unique(said, return_counts=True)]:
            v = out[b, tokens]
            r = st["repetition"][b].double()
            out[b, tokens] = torch.where(v > 0, v / r, v * r)
        tokens, count = torch.unique(said[p:], return_counts=True)
        out[b, tokens] -= st["frequency"][b].double() * count.double() + st["presence"][b].double()
        if st["bias"] is not None:
            lo, hi = int(st["bias"][0][b]), int(st["bias"][0][b + 1])
            out[b, st["bias"][1][lo:hi].long()] += st["bias"][2][lo:hi].double()
        tokens = _exact_rows(st, b)
        if tokens is not None:
            row = torch.full_like(out[b], -math.inf)
            row[tokens] = out[b, tokens]
            out[b] = row
    return out


def _exact_noise(seed, numbers):
    """Gumbel noise of one seed by splitmix64, in Python's whole numbers."""
    out, m = [], (1 << 64) - 1
    for n in numbers:
        z = (seed + (n + 1) * 0x9E3779B97F4A7C15) & m
        z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & m
        z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & m
        z ^= z >> 31
        out.append(-math.log(-math.log((2 * (z >> 41) + 1) / 2**24)))
    return torch.tensor(out, dtype=torch.float64, device="cuda")


def _exact_sample(st):
    V, B = st["V"], st["logits"].shape[0]
    token, logprob = [], []
    for b in range(B):
        ids = _exact_rows(st, b)
        ids = torch.arange(V, device="cuda") if ids is None else ids
        x = st["logits"][b].double()[ids]
        ids, x = ids[x > -math.inf], x[x > -math.inf]  # NaN is not above either
        if not len(ids):
            token.append(-1)
            logprob.append(-math.inf)
            continue
        T = float(st["temperature"][b])
        y = (x - x.max()) / (T or 1.0)
        order = torch.sort(-x, stable=True).indices
        n = int(st["top_k"][b])
        order = order[:n] if n > 0 else order
        w = torch.exp(y[order])
        n, p = len(order), float(st["top_p"][b])
        if p < 1:
            n = max(1, int(((w.cumsum(0) - w) < p * w.sum()).sum()))
        if st["min_p"] is not None:
            n = max(1, min(n, int((w >= float(st["min_p"][b])).sum())))
        kept = torch.sort(order[:1] if T == 0 else order[:n]).values
        group = ids[kept] // _GROUP
        there, at = torch.unique(group, return_inverse=True)
        mass = torch.zeros(len(there), dtype=torch.float64, device="cuda").index_add_(0, at, torch.exp(y[kept]))
        seed = int(st["seeds"][b])
        best = int((torch.log(mass) + _exact_noise(seed, [2**31 + j for j in there.tolist()])).argmax())
        last = kept[group == there[best]]
        pick = last[int((y[last] + _exact_noise(seed, ids[last].tolist())).argmax())]
        token.append(int(ids[pick]))
        logprob.append(float(y[pick] - torch.log(torch.exp(y).sum())))
    return [torch.tensor(token, dtype=torch.int32), torch.tensor(logprob, dtype=torch.float64)]
