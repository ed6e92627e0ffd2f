"""Rows for the logits heads: the norm with the residual's addition into 8 and 4 bits, and the quantization to
4 bits, bit for bit (r is the only value from a sum, which both sides keep far beyond its 24 bits)."""
from __future__ import annotations

import math

import numpy as np
import pytest

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


def _rows(rng, M, D, dtype, spread=1.0):
    import torch
    x = rng.normal(0, 1, (M, D)) * np.exp(rng.normal(0, spread, (1, D)))
    return torch.from_numpy(x.astype(np.float32)).to(_type(dtype))


def _same8(got, y):
    import torch
    q, scales = got
    wq, ws = ref.rows8(y)
    assert torch.equal(scales.cpu()[:, :y.shape[0]], ws)
    assert torch.equal(q.cpu().view(torch.uint8), wq.view(torch.uint8))


def _same4(got, y):
    import torch
    code, s, behind = ref.unpack4(*got, y.shape[1])
    wcode, ws, wrow = ref.rows4(y)
    assert torch.equal(got[2].cpu(), wrow) and torch.equal(s, ws)
    # the sign of a value that rounds to 0 is kept
    assert np.array_equal(code, wcode)
    assert all(bool((b == 0).all()) for b in behind)


CASES = [(1, 1), (1, 16), (3, 127), (5, 128), (4, 129), (2, 300), (33, 1040), (7, 2047), (130, 64), (256, 4096), (3, 8192),
         (2, 8200), (2, 20000), (1, 70001)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("residual", [None, "f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", CASES)
def test_norm(cuda, M, D, dtype, residual, bits):
    import torch
    rng = np.random.default_rng([M, D, bits])
    x = _rows(rng, M, D, dtype)
    res = None if residual is None else _rows(rng, M, D, residual) * 3
    gain = torch.from_numpy((1 + 0.3 * rng.normal(0, 1, D)).astype(np.float32)).to(_type("bf16" if D % 2 else dtype))
    eps = 1e-5 if D % 3 else 1e-6
    y, h = ref.normed(x, res, gain, eps)
    there = None if res is None else res.to(cuda)
    f, same = (T.trie_head_norm_quantize, _same8) if bits == 8 else (T.trie_head4_norm_quantize, _same4)
    got = f(x.to(cuda), gain.to(cuda), there, eps=eps)
    if res is not None:
        assert torch.equal(there.cpu(), h)
    same(got, y)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "f32"), ("f32", None)])
@pytest.mark.parametrize("M,D", [(5000, 64), (3000, 1040), (1500, 4096), (700, 8192), (700, 8200)])
def test_norm_many_rows(cuda, M, D, dtype, residual, bits):
    """More rows than CTAs: each goes over several."""
    import torch
    rng = np.random.default_rng([M, D, bits])
    x = _rows(rng, M, D, dtype)
    res = None if residual is None else _rows(rng, M, D, residual) * 3
    gain = torch.from_numpy((1 + 0.3 * rng.normal(0, 1, D)).astype(np.float32))
    y, h = ref.normed(x, res, gain, 1e-6)
    there = None if res is None else res.to(cuda)
    f, same = (T.trie_head_norm_quantize, _same8) if bits == 8 else (T.trie_head4_norm_quantize, _same4)
    got = f(x.to(cuda), gain.to(cuda), there)
    if res is not None:
        assert torch.equal(there.cpu(), h)
    same(got, y)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dtype,residual", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32"), ("bf16", None),
                                            ("f32", None)])
@pytest.mark.parametrize("M,D", [(700, 1), (400, 7), (400, 25), (500, 41), (400, 1001), (330, 2050), (320, 4100), (350, 8), (350, 520),
                                 (310, 6152)])
def test_norm_many_odd_rows(cuda, M, D, dtype, residual, bits):
    """More rows than twice the SMs, at every distance from a 16-byte boundary or at none."""
    rng = np.random.default_rng([M, D])
    x, res = _rows(rng, M, D, dtype), None if residual is None else _rows(rng, M, D, residual)
    gain = _rows(rng, 1, D, dtype)[0]
    y, h = ref.normed(x, res, gain, 1e-6)
    there = None if res is None else res.to(cuda)
    f, same = (T.trie_head_norm_quantize, _same8) if bits == 8 else (T.trie_head4_norm_quantize, _same4)
    same(f(x.to(cuda), gain.to(cuda), there), y)
    if res is not None:
        import torch
        assert torch.equal(there.cpu(), h)


def test_norm_far_rows(cuda):
    """Rows more than 2^31 values behind the first."""
    import torch
    M, D = 526000, 4096
    x = torch.zeros(M, D, dtype=torch.bfloat16, device=cuda)
    res = torch.zeros(M, D, dtype=torch.bfloat16, device=cuda)
    tail, rest = _rows(np.random.default_rng(1), 40, D, "bf16"), _rows(np.random.default_rng(2), 40, D, "bf16")
    gain = torch.ones(D, device=cuda)
    y, h = ref.normed(tail, rest, gain.cpu(), 1e-6)
    for f in (T.trie_head_norm_quantize, T.trie_head4_norm_quantize):
        x[-40:], res[-40:] = tail.to(cuda), rest.to(cuda)
        got = f(x, gain, res)
        assert torch.equal(res[-40:].cpu(), h)
        if len(got) == 2:
            _same8((got[0][-40:], got[1][:, M - 40:M]), y)
        else:
            code, s, row = ref.rows4(y)
            assert torch.equal(got[2][-40:].cpu(), row)
            first = (M - 40) // 128  # whole blocks of 128 rows from here on
            mine, scales, _ = ref.unpack4(got[0][first * 128:], got[1][first:], got[2], D)
            assert np.array_equal(mine[-40:], code) and torch.equal(scales[-40:], s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D", CASES)
def test_quantize4(cuda, M, D, dtype):
    import torch
    rng = np.random.default_rng([M, D, 7])
    x = _rows(rng, M, D, dtype, 3.0)
    x[0, ::3] = 0
    if M > 2:
        x[1] = 0
        x[2] = (x[2].double() * 1e-34).to(x.dtype)  # steps below the smallest row scale
    _same4(T.trie_head4_quantize(x.to(cuda)), x.float())


def test_quantize4_borders(cuda):
    """Every border between two codes and its neighbours, both signs; a scale of a block at its ends."""
    import torch
    u = np.array([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6], np.float32)
    u = np.concatenate([u, np.nextafter(u, np.float32(9)), np.nextafter(u, np.float32(-9))])
    u = np.concatenate([u, -u])
    u = np.pad(u, (0, -len(u) % 15)).reshape(-1, 15)
    rows = np.concatenate([u, np.full((len(u), 1), 6, np.float32)], axis=1).reshape(1, -1)
    rows = np.concatenate([rows, np.full((1, 16), 2688, np.float32)], axis=1)  # the row's scale is 1, the blocks' too
    x = torch.from_numpy(np.concatenate([rows, rows * 2.0 ** 20, rows * 2.0 ** -60]).astype(np.float32))
    _same4(T.trie_head4_quantize(x.to(cuda)), x)
    small = torch.from_numpy(np.geomspace(1e-7, 1, 40 * 16).astype(np.float32)[None, :])  # block scales down to 0
    _same4(T.trie_head4_quantize(small.to(cuda)), small)


@pytest.mark.parametrize("eps", [1e-30, 1e-6, 1e30])
@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e-20, 1e-14, 1e-10, 1e10, 1e18, 1e19, 1e25, 1e37])
def test_norm_range(cuda, size, eps):
    """Squares beyond the range of 32 bits."""
    import torch
    rng = np.random.default_rng(5)
    x = torch.from_numpy((rng.normal(0, 1, (3, 400)) * size).astype(np.float32))
    x[1] = 0
    gain = torch.ones(400)
    y, _ = ref.normed(x, None, gain, eps)
    _same8(T.trie_head_norm_quantize(x.to(cuda), gain.to(cuda), eps=eps), y)
    _same4(T.trie_head4_norm_quantize(x.to(cuda), gain.to(cuda), eps=eps), y)


def test_not_numbers(cuda):
    """A row with a NaN or an infinity gets NaNs (8 bits) or a NaN scale (4 bits) and leaves the others alone."""
    import torch
    rng = np.random.default_rng(6)
    clean = _rows(rng, 9, 300, "f32")
    x = clean.clone()
    x[1, 17], x[4, 299], x[8, 0] = math.nan, math.inf, -math.inf
    bad = torch.zeros(9, dtype=torch.bool)
    bad[[1, 4, 8]] = True
    gain = torch.ones(300, device=cuda)
    for norm in (True, False):
        got = T.trie_head4_norm_quantize(x.to(cuda), gain) if norm else T.trie_head4_quantize(x.to(cuda))
        want = T.trie_head4_norm_quantize(clean.to(cuda), gain) if norm else T.trie_head4_quantize(clean.to(cuda))
        assert bool(got[2].cpu()[bad].isnan().all())
        for a, b in zip(got, want):
            a, b = (t.cpu().view(torch.uint8) if t.dtype is not torch.float32 else t.cpu() for t in (a, b))
            if a.dim() == 5:
                a, b = (t.permute(0, 3, 2, 1, 4).flatten(0, 2).flatten(1)[:9] for t in (a, b))
            assert torch.equal(a[~bad], b[~bad])
    q, scales = T.trie_head_norm_quantize(x.to(cuda), gain)
    wq, ws = T.trie_head_norm_quantize(clean.to(cuda), gain)
    q, wq = q.float().cpu(), wq.float().cpu()
    assert bool(q[bad].isnan().any(dim=1).all())
    assert torch.equal(q[~bad], wq[~bad]) and torch.equal(scales[:, :9].cpu()[:, ~bad], ws[:, :9].cpu()[:, ~bad])


@pytest.mark.parametrize("offset,pad", [(0, 8), (1, 0), (3, 13), (4, 64), (8, 8), (2, 6)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_norm_strides(cuda, dtype, offset, pad):
    """Rows at any distance and any alignment; what lies between the residual's rows is not written."""
    import torch
    rng = np.random.default_rng([offset, pad])
    M, D = 5, 264

    def placed(t):
        buf = torch.full((M * (D + pad) + offset + 8,), 7.0, dtype=t.dtype, device=cuda)
        whole = buf[offset:offset + M * (D + pad)].view(M, D + pad)
        whole[:, :D] = t.to(cuda)
        return buf, whole
    x, res = _rows(rng, M, D, dtype), _rows(rng, M, D, dtype)
    gain = _rows(rng, 1, D + 3, dtype)[0]
    y, h = ref.normed(x, res, gain[3:], 1e-6)
    for f, same in ((T.trie_head_norm_quantize, _same8), (T.trie_head4_norm_quantize, _same4)):
        _, wx = placed(x)
        buf, wr = placed(res)
        same(f(wx[:, :D], gain.to(cuda)[3:], wr[:, :D]), y)
        assert torch.equal(wr[:, :D].cpu(), h)
        assert bool((wr[:, D:] == 7).all()) and bool((buf[:offset] == 7).all()) and bool((buf[-8:] == 7).all())
    _, wx = placed(x)
    _same4(T.trie_head4_quantize(wx[:, :D]), x.float())


def test_norm_is_quantize_of_normed(cuda):
    """The 8-bit norm gives what trie_head_quantize gives of the normed rows."""
    import torch
    rng = np.random.default_rng(8)
    x, gain = _rows(rng, 40, 1000, "bf16"), torch.from_numpy(rng.normal(1, 0.2, 1000).astype(np.float32))
    y, _ = ref.normed(x, None, gain, 1e-6)
    q, s = T.trie_head_norm_quantize(x.to(cuda), gain.to(cuda))
    wq, ws = T.trie_head_quantize(y.to(cuda))
    assert torch.equal(q.view(torch.uint8), wq.view(torch.uint8)) and torch.equal(s[:, :40], ws[:, :40])


def test_norm_streams_and_graphs(cuda):
    """On a side stream and replayed from a graph on new hidden states; the residual goes on in place."""
    import torch
    rng = np.random.default_rng(9)
    M, D = 20, 1536
    x, other = _rows(rng, M, D, "bf16").to(cuda), _rows(rng, M, D, "bf16").to(cuda)
    res, gain = _rows(rng, M, D, "f32").to(cuda), torch.ones(D, device=cuda)
    mine = [res.clone() for _ in range(3)]
    first = T.trie_head4_norm_quantize(x, gain, mine[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    second = T.trie_head4_norm_quantize(x, gain, mine[1], stream=side)
    side.synchronize()
    assert torch.equal(first[0], second[0]) and torch.equal(mine[0], mine[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        third = T.trie_head4_norm_quantize(x, gain, mine[2])
    graph.replay()
    assert torch.equal(first[0], third[0]) and torch.equal(mine[0], mine[2])
    x.copy_(other)
    graph.replay()
    again = T.trie_head4_norm_quantize(other, gain, mine[0])
    assert torch.equal(again[0], third[0]) and torch.equal(again[2], third[2]) and torch.equal(mine[0], mine[2])


def test_norm_refusals(cuda):
    import torch
    x, gain = torch.zeros(3, 64, device=cuda), torch.ones(64, device=cuda)
    for f in (T.trie_head_norm_quantize, T.trie_head4_norm_quantize):
        bad = [
            (TypeError, lambda: f(x.half(), gain)), (TypeError, lambda: f(x.cpu(), gain)), (ValueError, lambda: f(x[0], gain)),
            (ValueError, lambda: f(x.t(), gain)), (ValueError, lambda: f(x, gain[:-1])), (TypeError, lambda: f(x, gain.half())),
            (ValueError, lambda: f(x, x)), (ValueError, lambda: f(x, gain, x[:2])), (TypeError, lambda: f(x, gain, x.half())),
            (ValueError, lambda: f(x, torch.ones(128, device=cuda)[::2])), (TypeError, lambda: f(x, gain.cpu())),
            (T.TrieError, lambda: f(x, gain, eps=0.0)), (T.TrieError, lambda: f(x, gain, eps=math.nan)),
            (T.TrieError, lambda: f(x, gain, eps=math.inf)),
            (ValueError, lambda: f(x, gain, torch.zeros(1, 64, device=cuda).expand(3, 64))),
        ]
        for kind, call in bad:
            with pytest.raises(kind):
                call()
        assert f(x[:0], gain)[0].shape[0] == 0
    assert T.trie_head4_quantize(x[:0])[0].shape == (0, 32)
    with pytest.raises(TypeError):
        T.trie_head4_quantize(x.half())
