"""trie_head_quantize, trie_head_quantize_weight and trie_head_logits against
their definitions.

Quantized values and scales are compared bit for bit (a product with 1/448, a
division, a rounding to e4m3, by torch on the CPU). Logits are compared with sums in 64 bits of the
quantized values: a block's 128 products are exact, and adding them up in 32
bits is off by at most 128 units of 2^-23 of the sum of their magnitudes, even
where an adder truncates; scaling and adding the blocks adds a few units of
2^-24 a block of the same sum. So |error| <= 2^-16 sum |x w| for each logit,
and, errors of many terms being independent, 1e-5 of the whole in the 2-norm.
bf16 adds half a unit of its 8 bits (2^-8 relative)."""
from __future__ import annotations

import math

import numpy as np
import pytest

import logits_ref as ref
from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2608_12574_gb300 import _build
    _build.build()
    return torch.device("cuda:0")


def _type(dtype):
    import torch
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _quantized(x, rows):
    """(e4m3 values as float64, scales [row blocks, column blocks]) of x by blocks of rows x 128, on the CPU."""
    import torch
    n, d = x.shape
    x = x.float()
    q, scales = torch.zeros(n, d, dtype=torch.float8_e4m3fn), torch.zeros((n + rows - 1) // rows, (d + 127) // 128)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            block = x[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128]
            s = block.abs().max() * torch.tensor(1 / 448, dtype=torch.float32)
            scales[i, j] = s if s > 0 else 1
            q[i * rows:(i + 1) * rows, j * 128:(j + 1) * 128] = (block / scales[i, j]).to(torch.float8_e4m3fn)
    return q, scales


def _inputs(rng, M, V, D, dtype, dev):
    import torch
    x = rng.normal(0, 1, (M, D)) * np.exp(rng.normal(0, 1, (1, D)))
    w = rng.normal(0, 1, (V, D)) / math.sqrt(D) * np.exp(rng.normal(0, 0.5, (V, 1)))
    x = torch.from_numpy(x.astype(np.float32)).to(_type(dtype)).to(dev)
    return x, torch.from_numpy(w.astype(np.float32)).to(dev)


def _check(q, scales, w, w_scales, out, ok=None):
    """out against the sums in 64 bits (on the device: the largest of these are 10^10 products)."""
    import torch
    M, D = q.shape
    V = w.shape[0]
    want = torch.zeros(M, V, dtype=torch.float64, device=q.device)
    size = torch.zeros_like(want)
    for j in range((D + 127) // 128):
        a = q[:, j * 128:(j + 1) * 128].double() * scales[j, :M, None].double()
        b = w[:, j * 128:(j + 1) * 128].double() * w_scales[:, j].double().repeat_interleave(128)[:V, None]
        want += a @ b.T
        size += a.abs() @ b.abs().T
    got = out.double()
    half = 2.0 ** -8 if out.dtype == torch.bfloat16 else 2.0 ** -24
    if ok is not None:
        assert bool((got[~ok] == -math.inf).all())
        want, size, got = want[ok], size[ok], got[ok]
    assert bool(torch.isfinite(got).all())
    worst = ((got - want).abs() - 2.0 ** -16 * size - half * want.abs()).max() if got.numel() else torch.zeros(())
    assert float(worst) <= 0, float(worst)
    if got.numel() > 1000:
        rel = float((got - want).norm() / want.norm())
        assert rel <= 1e-5 + (2.0 ** -8 if out.dtype == torch.bfloat16 else 0), rel


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", [(1, 1), (1, 16), (3, 127), (5, 128), (4, 129), (2, 300), (33, 1040), (256, 4096)])
def test_quantize(cuda, M, D, dtype):
    import torch
    rng = np.random.default_rng([M, D])
    x = torch.from_numpy((rng.normal(0, 1, (M, D)) * np.exp(rng.normal(0, 3, (M, D)))).astype(np.float32))
    x[0, ::3] = 0
    if M > 2:
        x[1] = 0
        x[2] *= 1e-38          # scales below the normal range
    x = x.to(_type(dtype))
    q, scales = T.trie_head_quantize(x.to(cuda))
    wq, ws = _quantized(x, 1)
    assert q.shape == (M, D) and torch.equal(q.cpu().view(torch.uint8), wq.view(torch.uint8))
    assert torch.equal(scales.cpu()[:, :M], ws.T)
    wide = torch.zeros(M, D + 5, dtype=x.dtype, device=cuda)
    wide[:, 2:D + 2] = x.to(cuda)
    q2, s2 = T.trie_head_quantize(wide[:, 2:D + 2])
    assert torch.equal(q.view(torch.uint8), q2.view(torch.uint8)) and torch.equal(scales[:, :M], s2[:, :M])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,D", [(2, 16), (127, 130), (128, 128), (129, 272), (515, 1040)])
def test_quantize_weight(cuda, V, D, dtype):
    import torch
    rng = np.random.default_rng([V, D])
    w = torch.from_numpy(rng.normal(0, 1, (V, D)).astype(np.float32)).to(_type(dtype))
    q, scales = T.trie_head_quantize_weight(w.to(cuda))
    wq, ws = _quantized(w, 128)
    assert torch.equal(q.cpu().view(torch.uint8), wq.view(torch.uint8)) and torch.equal(scales.cpu(), ws)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [
    (1, 2, 16), (1, 1000, 128), (2, 129, 144), (7, 128, 2048), (16, 4097, 1040), (17, 333, 256), (31, 1024, 512),
    (32, 777, 640), (33, 640, 1024), (64, 2049, 400), (65, 1001, 384), (100, 515, 4096), (128, 1300, 272),
    (129, 900, 512), (255, 1111, 1168), (256, 2048, 2048), (257, 1027, 128), (300, 5003, 640), (1000, 1500, 528),
    (513, 700, 5120)])
def test_head(cuda, M, V, D, dtype):
    import torch
    rng = np.random.default_rng([M, V, D])
    x, w = _inputs(rng, M, V, D, dtype, cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
    T.trie_head_logits(q, scales, wq, ws, out)
    _check(q, scales, wq, ws, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D", [(1, 1000, 256), (5, 50021, 256), (40, 8191, 400), (256, 4099, 1024), (300, 3000, 128)])
def test_head_grammar(cuda, M, V, D, dtype):
    """Rows that allow nothing, one token, all; free, finished and dead rows; tiles that nobody allows."""
    import torch
    rng = np.random.default_rng([M, V])
    rows = 12
    x, w = _inputs(rng, M, V, D, dtype, cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    allowed = rng.random((rows, V)) < np.array([0, 1 / V, 0.001, 0.0003, 0.01, 1.0] * 2)[:, None]
    allowed[0] = False
    allowed[1, :128] = True
    mask = torch.from_numpy(ref.pack(allowed)).to(cuda)
    for choice in ([0], [0, 1, 2, 3, -1, -2, rows], [2, 3, 4], [-3, 0, 2], [5, 1]):
        states = rng.choice(choice, M).astype(np.int32)
        ok = torch.from_numpy(np.stack([ref.allowed_row(allowed, int(s), V) for s in states])).to(cuda)
        out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
        T.trie_head_logits(q, scales, wq, ws, out, mask, torch.from_numpy(states).to(cuda))
        _check(q, scales, wq, ws, out, ok)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,V,D,few", [(3, 2, 16, 2), (33, 5000, 144, 255), (33, 5000, 144, 256), (33, 5000, 144, 257),
                                       (130, 9001, 2048, 40), (300, 4100, 272, 72)])
def test_head_few_tokens(cuda, M, V, D, few, dtype):
    """Rows that allow up to a list's length of tokens, exactly that, and one more, beside dense ones; a given
    workspace."""
    import torch
    rng = np.random.default_rng([M, V, few])
    rows = 16
    x, w = _inputs(rng, M, V, D, dtype, cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    allowed = np.zeros((rows, V), bool)
    for r in range(rows):
        allowed[r, rng.choice(V, min(V, few if r % 2 else max(1, few - r)), replace=False)] = True
    allowed[3] = rng.random(V) < 0.6
    mask = torch.from_numpy(ref.pack(allowed)).to(cuda)
    work = torch.full((T.trie_head_workspace(M, V) // 4 + 4,), 0x5A5A5A5A, dtype=torch.int32, device=cuda)
    for choice in ([1, 5, 2], [0, 1, 2, 3, -1, -2]):
        states = rng.choice(choice, M).astype(np.int32)
        ok = torch.from_numpy(np.stack([ref.allowed_row(allowed, int(s), V) for s in states])).to(cuda)
        out = torch.full((M, V), math.nan, dtype=_type(dtype), device=cuda)
        T.trie_head_logits(q, scales, wq, ws, out, mask, torch.from_numpy(states).to(cuda), workspace=work)
        _check(q, scales, wq, ws, out, ok)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 13), (4, 64), (7, 1)])
def test_head_strides(cuda, offset, pad, dtype):
    """Rows of logits at any distance and any alignment; what lies between them is not written."""
    import torch
    rng = np.random.default_rng([offset, pad])
    M, V, D = 21, 1001, 272
    x, w = _inputs(rng, M, V, D, dtype, cuda)
    q, scales = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    buf = torch.full((M * (V + pad) + offset + 8,), 7.0, dtype=_type(dtype), device=cuda)
    whole = buf[offset:offset + M * (V + pad)].view(M, V + pad)
    T.trie_head_logits(q, scales, wq, ws, whole[:, :V])
    _check(q, scales, wq, ws, whole[:, :V])
    assert bool((whole[:, V:] == 7).all()) and bool((buf[:offset] == 7).all()) and bool((buf[-8:] == 7).all())


def test_head_special_values(cuda):
    """A row with NaN or an infinity has NaN logits and leaves the others alone; a row of zeros gives zeros."""
    import torch
    rng = np.random.default_rng(2)
    M, V, D = 70, 500, 400
    x, w = _inputs(rng, M, V, D, "f32", cuda)
    clean = x.clone()
    x[3, 17], x[40, 399], x[69, 0] = math.nan, math.inf, -math.inf
    x[5] = clean[5] = 0
    wq, ws = T.trie_head_quantize_weight(w)
    out, want = torch.empty(M, V, device=cuda), torch.empty(M, V, device=cuda)
    T.trie_head_logits(*T.trie_head_quantize(x), wq, ws, out)
    T.trie_head_logits(*T.trie_head_quantize(clean), wq, ws, want)
    bad = torch.zeros(M, dtype=torch.bool, device=cuda)
    bad[[3, 40, 69]] = True
    assert bool(out[bad].isnan().all()) and torch.equal(out[~bad], want[~bad]) and bool((out[5] == 0).all())


def test_head_repeats_and_graphs(cuda):
    """The same bits every time, alone, on a side stream and replayed from a graph on new hidden states."""
    import torch
    rng = np.random.default_rng(4)
    M, V, D = 48, 3001, 1024
    x, w = _inputs(rng, M, V, D, "bf16", cuda)
    y, _ = _inputs(rng, M, V, D, "bf16", cuda)
    wq, ws = T.trie_head_quantize_weight(w)

    def head(out, stream=None):
        T.trie_head_logits(*T.trie_head_quantize(x, stream=stream), wq, ws, out, stream=stream)
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


def test_head_refusals(cuda):
    import torch
    M, V, D = 3, 200, 256
    x, w = torch.zeros(M, D, device=cuda), torch.zeros(V, D, device=cuda)
    q, s = T.trie_head_quantize(x)
    wq, ws = T.trie_head_quantize_weight(w)
    out = torch.zeros(M, V, device=cuda)
    i = torch.zeros(M, dtype=torch.int32, device=cuda)
    m = torch.zeros(3, 7, dtype=torch.int32, device=cuda)
    bad = [
        (TypeError, lambda: T.trie_head_quantize(x.half())), (TypeError, lambda: T.trie_head_quantize(x.cpu())),
        (ValueError, lambda: T.trie_head_quantize(x[0])), (ValueError, lambda: T.trie_head_quantize(x.t())),
        (ValueError, lambda: T.trie_head_quantize_weight(w[:, ::2])),
        (ValueError, lambda: T.trie_head_logits(q, s, wq, ws, out[:, :-1])),
        (ValueError, lambda: T.trie_head_logits(q[:2], s, wq, ws, out)),
        (ValueError, lambda: T.trie_head_logits(q, s[:1], wq, ws, out)),
        (ValueError, lambda: T.trie_head_logits(q, s[:, :3].contiguous(), wq, ws, out)),
        (ValueError, lambda: T.trie_head_logits(q, s, wq, ws[:1], out)),
        (TypeError, lambda: T.trie_head_logits(q.view(torch.uint8), s, wq, ws, out)),
        (TypeError, lambda: T.trie_head_logits(q, s, wq, ws, out.half())),
        (TypeError, lambda: T.trie_head_logits(q, s.half(), wq, ws, out)),
        (ValueError, lambda: T.trie_head_logits(q, s, wq, ws, out, mask=m)),
        (ValueError, lambda: T.trie_head_logits(q, s, wq, ws, out, mask=m, states=i, workspace=i)),
        (ValueError, lambda: T.trie_head_workspace(-1, 5)),
        (ValueError, lambda: T.trie_head_logits(q, s, wq, ws, out, mask=m[:, :6], states=i)),
        (T.TrieError, lambda: T.trie_head_logits(q[:, :24].contiguous(), s[:1], wq[:, :24].contiguous(),
                                                 ws[:, :1].contiguous(), out)),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    lib = T.load_library()
    args = [q.data_ptr(), s.data_ptr(), 4, wq.data_ptr(), ws.data_ptr(), M, V, D, out.data_ptr(), 0, V, None, 0, None,
            None, None]
    assert lib.trie_head_logits(*args) == T.TRIE_OK
    torch.cuda.synchronize()
    for at, value in [(0, None), (0, q.data_ptr() + 8), (1, None), (1, s.data_ptr() + 4), (2, 2), (2, 6), (3, None),
                      (3, wq.data_ptr() + 4), (4, None), (4, ws.data_ptr() + 2), (5, -1), (6, 1), (7, 0), (7, 24),
                      (8, None), (8, out.data_ptr() + 2), (9, 5), (10, V - 1), (11, i.data_ptr()), (13, i.data_ptr()),
                      (14, out.data_ptr() + 4)]:
        wrong = list(args)
        wrong[at] = value
        assert lib.trie_head_logits(*wrong) == T.TRIE_EINVAL, (at, value)
    T.trie_head_logits(q[:0], s, wq, ws, out[:0])
    e, _ = T.trie_head_quantize(x[:0])
    assert e.shape == (0, D)
