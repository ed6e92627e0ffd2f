"""The logits head in 4 bits, under a grammar, against the sums in 64 bits."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as lref
import rows_ref as ref
from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device")
    T.load_library()
    return torch.device("cuda:0")


def _type(name):
    import torch
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def _inputs(rng, M, V, D, dev):
    import torch
    x = rng.normal(0, 1, (M, D)) * np.exp(rng.normal(0, 1, (1, D)))
    w = rng.normal(0, 1, (V, D)) / math.sqrt(D) * np.exp(rng.normal(0, 0.5, (V, 1)))
    x, w = (torch.from_numpy(t.astype(np.float32)).to(dev) for t in (x, w))
    return T.trie_head4_quantize(x), T.trie_head4_quantize(w)


def _check(x, w, D, out, ok=None):
    """A block of 64 columns is one addition to the sums: of its 64 products and the sum before, each taken exactly
    or cut at 2^-23 of the largest, so at most 2 units of 2^-23 of the terms' magnitudes for each block; four
    roundings more for the scales of the rows; half a step of the logits' type."""
    import torch
    a, b = ref.values4(*x, D), ref.values4(*w, D)
    want, size, got = a @ b.T, a.abs() @ b.abs().T, out.double()
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    if ok is not None:
        assert bool((got[~ok] == -math.inf).all())
        want, size, got = want[ok], size[ok], got[ok]
    assert bool(torch.isfinite(got).all())
    if not got.numel():
        return
    bound = ((D + 63) // 64 * 2 + 4) * 2.0 ** -23 * size + half * want.abs()
    worst = ((got - want).abs() - bound).max()
    assert float(worst) <= 0, float(worst)
    if got.numel() > 1000:
        rel = float((got - want).norm() / want.norm())
        assert rel <= 1e-5 + (2.0 ** -8 if out.dtype == torch.bfloat16 else 0), rel


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [
    (1, 2, 1), (1, 2, 16), (1, 1000, 128), (2, 129, 144), (7, 128, 2048), (16, 4097, 1040), (17, 333, 256), (31, 1024, 512),
    (32, 777, 640), (33, 640, 1023), (64, 2049, 400), (65, 1001, 384), (100, 515, 4096), (128, 1300, 272),
    (129, 900, 512), (255, 1111, 1168), (256, 2048, 2048), (257, 1027, 128), (300, 5003, 641), (1000, 1500, 528),
    (513, 700, 5120), (3, 300, 33), (128, 383, 65), (130, 40001, 100)])
def test_head4(cuda, M, V, D, dtype):
    import torch
    x, w = _inputs(np.random.default_rng([M, V, D]), M, V, D, cuda)
    out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
    T.trie_head4_logits(*x, *w, out)
    _check(x, w, D, out)


def test_head4_places(cuda):
    """Single ones at every column and row, so that a value or a scale taken from another's place shows."""
    import torch
    M, V, D = 140, 300, 200
    x, w = torch.zeros(M, D, device=cuda), torch.zeros(V, D, device=cuda)
    x[torch.arange(M), torch.arange(M) * 7 % D] = 2.0 ** (torch.arange(M, device=cuda) % 9)
    w[:] = 1.0 + torch.arange(V, device=cuda)[:, None] % 5 + 8 * (torch.arange(D, device=cuda)[None, :] % 3)
    x, w = T.trie_head4_quantize(x), T.trie_head4_quantize(w)
    out = torch.empty(M, V, device=cuda)
    T.trie_head4_logits(*x, *w, out)
    _check(x, w, D, out)
    # rows' blocks of very different size
    g = torch.Generator(device=cuda)
    g.manual_seed(1)
    x = torch.randn(M, D, generator=g, device=cuda) * 2.0 ** torch.randint(-8, 8, (M, 1), generator=g, device=cuda)
    w = torch.randn(V, D, generator=g, device=cuda) * 2.0 ** (torch.arange(D, device=cuda) // 16 % 7 - 3.0)
    x, w = T.trie_head4_quantize(x), T.trie_head4_quantize(w)
    T.trie_head4_logits(*x, *w, out)
    _check(x, w, D, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(1, 1000, 256), (5, 50021, 256), (40, 8191, 400), (256, 4099, 1024), (300, 3000, 130)])
def test_head4_grammar(cuda, M, V, D, dtype):
    """Rows that allow nothing, one token, all; free, finished and dead rows; tiles that nobody allows."""
    import torch
    rng = np.random.default_rng([M, V])
    rows = 12
    x, w = _inputs(rng, M, V, D, cuda)
    allowed = rng.random((rows, V)) < np.array([0, 1 / V, 0.001, 0.0003, 0.01, 1.0] * 2)[:, None]
    allowed[0] = False
    allowed[1, :128] = True
    mask = torch.from_numpy(lref.pack(allowed)).to(cuda)
    for choice in ([0], [0, 1, 2, 3, -1, -2, rows], [2, 3, 4], [-3, 0, 2], [5, 1]):
        states = rng.choice(choice, M).astype(np.int32)
        ok = torch.from_numpy(np.stack([lref.allowed_row(allowed, int(s), V) for s in states])).to(cuda)
        out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
        T.trie_head4_logits(*x, *w, out, mask, torch.from_numpy(states).to(cuda))
        _check(x, w, D, out, ok)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D,few", [(3, 2, 16, 2), (33, 5000, 144, 255), (33, 5000, 144, 256), (33, 5000, 144, 257),
                                       (130, 9001, 2048, 40), (300, 4100, 273, 72), (4, 1000, 70000, 9)])
def test_head4_few_tokens(cuda, M, V, D, few, dtype):
    """Rows that allow up to a list's length of tokens, exactly that, and one more, beside dense ones; a given
    workspace; bits of the mask behind V."""
    import torch
    rng = np.random.default_rng([M, V, few])
    rows = 16
    x, w = _inputs(rng, M, V, D, cuda)
    allowed = np.zeros((rows, V), bool)
    for r in range(rows):
        allowed[r, rng.choice(V, min(V, few if r % 2 else max(1, few - r)), replace=False)] = True
    allowed[3] = rng.random(V) < 0.6
    packed = lref.pack(allowed)
    if V % 32:
        packed[:, -1] |= np.int32(-1) << np.int32(V % 32)
    mask = torch.from_numpy(packed).to(cuda)
    work = torch.full((T.trie_head_workspace(M, V) // 4 + 4,), 0x5A5A5A5A, dtype=torch.int32, device=cuda)
    for choice in ([1, 5, 2], [0, 1, 2, 3, -1, -2]):
        states = rng.choice(choice, M).astype(np.int32)
        ok = torch.from_numpy(np.stack([lref.allowed_row(allowed, int(s), V) for s in states])).to(cuda)
        out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
        T.trie_head4_logits(*x, *w, out, mask, torch.from_numpy(states).to(cuda), workspace=work)
        _check(x, w, D, out, ok)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M", [21, 140])
@pytest.mark.parametrize("offset,pad", [(0, 7), (1, 0), (3, 13), (4, 64), (7, 1), (16, 32)])
def test_head4_strides(cuda, M, offset, pad, dtype):
    """Rows of logits at any distance and any alignment; what lies between them is not written."""
    import torch
    V, D = 1001, 272
    x, w = _inputs(np.random.default_rng([offset, pad]), M, V, D, cuda)
    buf = torch.full((M * (V + pad) + offset + 8,), 7.0, dtype=_type(dtype), device=cuda)
    whole = buf[offset:offset + M * (V + pad)].view(M, V + pad)
    T.trie_head4_logits(*x, *w, whole[:, :V])
    _check(x, w, D, whole[:, :V])
    assert bool((whole[:, V:] == 7).all()) and bool((buf[:offset] == 7).all()) and bool((buf[-8:] == 7).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V", [(20, 700), (130, 64), (130, 127), (130, 323), (260, 1100)])
def test_head4_row_starts(cuda, M, V, dtype):
    """Rows that start anywhere between two 32-byte boundaries are those of aligned ones, with a grammar too, and
    nothing beside them is written. The sums are the same ones, so all bits are."""
    import torch
    rng = np.random.default_rng([M, V])
    D = 200
    x, w = _inputs(rng, M, V, D, cuda)
    # free rows among the others (-3), so that these are not dot products
    mask = torch.from_numpy(lref.pack(rng.random((4, V)) < 0.7)).to(cuda)
    states = torch.from_numpy(rng.choice([0, 1, 2, 3, -3], M).astype(np.int32)).to(cuda)
    stride = (V + 15) // 16 * 16 + 16
    for extra in ({}, {"mask": mask, "states": states}):
        want = torch.empty(M, stride, dtype=_type(dtype), device=cuda)[:, :V]
        T.trie_head4_logits(*x, *w, want, **extra)
        for start in range(32 // want.element_size()):
            buf = torch.full((M * stride + 32,), 7.0, dtype=_type(dtype), device=cuda)
            rows = buf[start:start + M * stride].view(M, stride)
            T.trie_head4_logits(*x, *w, rows[:, :V], **extra)
            assert torch.equal(rows[:, :V], want), start
            assert bool((rows[:, V:] == 7).all()) and bool((buf[:start] == 7).all()) and bool((buf[start + M * stride:] == 7).all())


@pytest.mark.parametrize("M", [70, 200])
def test_head4_special_values(cuda, M):
    """A row, or a token's weights, with NaN or an infinity has NaN logits and leaves the others alone; zeros give
    zeros; scales of rows behind the last and what lies behind D are not looked at."""
    import torch
    rng = np.random.default_rng(2)
    V, D = 500, 400
    x = torch.from_numpy(rng.normal(0, 1, (M, D)).astype(np.float32)).to(cuda)
    w = torch.from_numpy(rng.normal(0, 1, (V, D)).astype(np.float32)).to(cuda)
    x[5] = 0
    want = torch.empty(M, V, device=cuda)
    T.trie_head4_logits(*T.trie_head4_quantize(x), *T.trie_head4_quantize(w), want)
    x[3, 17], x[40, 399], x[69, 0], w[7, 3], w[499, 1] = math.nan, math.inf, -math.inf, math.nan, math.inf
    out = torch.empty(M, V, device=cuda)
    q, s, r = T.trie_head4_quantize(x)
    flat = s.view(torch.uint8).permute(0, 3, 2, 1, 4).flatten(0, 2)
    flat[M:] = 0x7F
    s = flat.view((M + 127) // 128, 4, 32, -1, 4).permute(0, 3, 2, 1, 4).contiguous().view(torch.float8_e4m3fn)
    T.trie_head4_logits(q, s, r, *T.trie_head4_quantize(w), out)
    bad = torch.zeros(M, V, dtype=torch.bool, device=cuda)
    bad[[3, 40, 69]] = True
    bad[:, [7, 499]] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], want[~bad]) and bool((out[5][~bad[5]] == 0).all())


def test_head4_far_rows(cuda):
    """Logits more than 2^31 values behind the first, free and under a grammar."""
    import torch
    M, V, D = 16500, 131072, 64
    g = torch.Generator(device=cuda)
    g.manual_seed(3)
    x = T.trie_head4_quantize(torch.randn(M, D, generator=g, device=cuda))
    w = T.trie_head4_quantize(torch.randn(V, D, generator=g, device=cuda))
    out = torch.empty(M, V, dtype=torch.bfloat16, device=cuda)
    T.trie_head4_logits(*x, *w, out)
    first = M // 128 * 128
    last = (x[0][first:], x[1][first // 128:], x[2][first:])
    _check(last, w, D, out[first:])
    allowed = np.zeros((2, V), bool)
    allowed[0, 5::9999] = True
    mask = torch.from_numpy(lref.pack(allowed)).to(cuda)
    states = torch.zeros(M, dtype=torch.int32, device=cuda)
    T.trie_head4_logits(*x, *w, out, mask, states)
    _check(last, w, D, out[first:], torch.from_numpy(allowed[0]).to(cuda).expand(M - first, V))


def test_head4_repeats_and_graphs(cuda):
    """The same bits every time, alone, on a side stream and replayed from a graph on new hidden states."""
    import torch
    rng = np.random.default_rng(4)
    M, V, D = 48, 3001, 1024
    x = torch.from_numpy(rng.normal(0, 1, (M, D)).astype(np.float32)).to(cuda)
    y = torch.from_numpy(rng.normal(0, 1, (M, D)).astype(np.float32)).to(cuda)
    w = T.trie_head4_quantize(torch.from_numpy(rng.normal(0, 1, (V, D)).astype(np.float32)).to(cuda))

    def head(out, stream=None):
        T.trie_head4_logits(*T.trie_head4_quantize(x, stream=stream), *w, out, stream=stream)
    outs = [torch.empty(M, V, dtype=torch.bfloat16, device=cuda) for _ in range(3)]
    head(outs[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    head(outs[1], side)
    side.synchronize()
    assert torch.equal(outs[0], outs[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        head(outs[2])
    x.copy_(y)
    graph.replay()
    head(outs[1])
    assert torch.equal(outs[1], outs[2]) and not torch.equal(outs[0], outs[1])


def test_head4_refusals(cuda):
    import torch
    M, V, D = 3, 200, 256
    q, s, r = T.trie_head4_quantize(torch.zeros(M, D, device=cuda))
    w, ws, wr = T.trie_head4_quantize(torch.zeros(V, D, device=cuda))
    out = torch.zeros(M, V, device=cuda)
    i = torch.zeros(M, dtype=torch.int32, device=cuda)
    m = torch.zeros(3, 7, dtype=torch.int32, device=cuda)
    bad = [
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out[:, :-1])),
        (ValueError, lambda: T.trie_head4_logits(q[:2], s, r, w, ws, wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s[:, :3], r, w, ws, wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r[:2], w, ws, wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w[:, :120], ws, wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws[:1], wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w[0], ws, wr, out)),
        (TypeError, lambda: T.trie_head4_logits(q.view(torch.int8), s, r, w, ws, wr, out)),
        (TypeError, lambda: T.trie_head4_logits(q, s.view(torch.uint8), r, w, ws, wr, out)),
        (TypeError, lambda: T.trie_head4_logits(q, s, r.double(), w, ws, wr, out)),
        (TypeError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out.half())),
        (TypeError, lambda: T.trie_head4_logits(q.cpu(), s, r, w, ws, wr, out)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out, mask=m)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out, states=i)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out, mask=m, states=i, workspace=i)),
        (ValueError, lambda: T.trie_head4_logits(q, s, r, w, ws, wr, out, mask=m[:, :6], states=i)),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    T.trie_head4_logits(q[:0], s[:0], r[:0], w, ws, wr, out[:0])
