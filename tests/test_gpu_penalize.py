"""trie_penalize against the definition in 64 bits.

Tolerance: every step is rounded to nearest in 32 bits, so a result is within
the sum of half a unit in the last place of each step's value
(logits_ref.penalize), doubled for the steps' errors passing through later
steps with a factor of at most max(r, 1/r) <= 2; bf16 adds half a unit of its
8 bits (2^-8 relative). Untouched logits and masked ones are compared bit for bit."""
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


def _bits(t):
    import torch
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16).cpu().numpy()


def _check(before, after, history, length, prompt, r, p, f, bias, allowed, states):
    """Every row of `after` against the definition; before / after CPU tensors."""
    import torch
    B, V = before.shape
    raw0, raw1 = _bits(before), _bits(after)
    x, got = before.float().numpy(), after.float().numpy()
    for b in range(B):
        n = 0 if history is None else max(0, min(int(length[b]), history.shape[1]))
        said = [] if history is None else history[b, :n].tolist()
        pr = 0 if prompt is None else int(prompt[b])
        of = [] if bias is None else list(zip(bias[1][bias[0][b]:bias[0][b + 1]].tolist(),
                                              bias[2][bias[0][b]:bias[0][b + 1]].tolist()))
        ok = ref.allowed_row(allowed, FREE if states is None else int(states[b]), V)
        want, bound = ref.penalize(x[b], said, pr, 1.0 if r is None else float(r[b]), 0.0 if p is None else float(p[b]),
                                   0.0 if f is None else float(f[b]), of, ok)
        touched = np.zeros(V, bool)
        touched[[t for t in said + [t for t, _ in of] if 0 <= t < V]] = True
        same = ok & ~touched
        assert np.array_equal(raw0[b][same], raw1[b][same]), b
        assert np.all(got[b][~ok] == -math.inf), b
        at = ok & touched
        w, g = want[at], got[b][at].astype(np.float64)
        assert np.array_equal(np.isnan(w), np.isnan(g)) and np.array_equal(np.isinf(w), np.isinf(g)), b
        fin = np.isfinite(w)
        assert np.array_equal(w[~fin & ~np.isnan(w)], g[~fin & ~np.isnan(w)]), b
        tol = 2 * bound[at][fin] + (2.0 ** -8 * np.abs(w[fin]) + 2.0 ** -126 if before.dtype == torch.bfloat16 else 2.0 ** -148)
        worst = np.abs(w[fin] - g[fin]) - tol
        assert worst.size == 0 or worst.max() <= 0, (b, worst.max())


FREE = ref.FREE


def _case(rng, V, B, H, n_bias, rows, dtype, stride=None, hot=None):
    import torch
    tdtype = torch.float32 if dtype == "f32" else torch.bfloat16
    stride = stride or V
    whole = torch.from_numpy(rng.normal(0, 4, (B, stride)).astype(np.float32)).to(tdtype)
    history = rng.integers(0, hot or V, (B, H)).astype(np.int32) if H else None
    length = rng.integers(0, H + 1, B).astype(np.int32)
    prompt = rng.integers(0, H + 1, B).astype(np.int32)
    r = rng.choice([0.5, 1.0, 1.2, 2.0], B).astype(np.float32)
    p = rng.choice([0.0, 0.3, -0.7], B).astype(np.float32)
    f = rng.choice([0.0, 0.1, 1.5], B).astype(np.float32)
    bias = None
    if n_bias:
        many = rng.integers(0, n_bias + 1, B)
        off = np.concatenate([[0], np.cumsum(many)]).astype(np.int32)
        tok = rng.integers(0, hot or V, max(1, off[-1])).astype(np.int32)
        val = rng.normal(0, 3, max(1, off[-1])).astype(np.float32)
        val[rng.random(len(val)) < 0.2] = -math.inf
        bias = (off, tok, val)
    allowed = states = None
    if rows:
        allowed = rng.random((rows, V)) < rng.choice([0.0, 0.002, 0.5, 1.0], (rows, 1))
        allowed[0] = False
        states = rng.integers(0, rows, B).astype(np.int32)
        states[rng.random(B) < 0.3] = FREE
        states[:4] = [0, ref.FINISHED, ref.DEAD, rows + 5][:min(4, B)]
    return whole, history, length, prompt, r, p, f, bias, allowed, states


def _run(dev, V, whole, history, length, prompt, r, p, f, bias, allowed, states, offset=0):
    """The call on a view of `whole` that starts `offset` elements into a buffer."""
    import torch

    def up(a):
        return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev)
    B, stride = whole.shape
    buf = torch.zeros(B * stride + offset + 16, dtype=whole.dtype, device=dev)
    buf[offset:offset + B * stride] = whole.reshape(-1).to(dev)
    view = buf[offset:offset + B * stride].view(B, stride)
    T.trie_penalize(view[:, :V], up(history), up(length) if history is not None else None,
                    up(prompt) if history is not None and prompt is not None else None, up(r), up(p), up(f),
                    None if bias is None else tuple(up(x) for x in bias),
                    None if allowed is None else up(ref.pack(allowed)), up(states))
    torch.cuda.synchronize()
    out = buf.cpu()
    assert bool((out[:offset] == 0).all()) and bool((out[offset + B * stride:] == 0).all())
    out = out[offset:offset + B * stride].view(B, stride)
    assert np.array_equal(_bits(out[:, V:]), _bits(whole[:, V:]))  # between the rows
    return out[:, :V]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,B,H,n_bias,rows", [
    (2, 3, 4, 2, 2), (31, 5, 1, 0, 3), (33, 6, 70, 5, 4), (1001, 7, 300, 20, 6), (8192, 4, 64, 3, 0),
    (8193, 5, 5000, 40, 5), (16391, 9, 257, 0, 7), (32000, 1, 300, 8, 0), (50021, 6, 9001, 300, 8),
    (152064, 3, 2048, 16, 4)])
def test_penalize(cuda, V, B, H, n_bias, rows, dtype):
    rng = np.random.default_rng([V, B, H])
    case = _case(rng, V, B, H, n_bias, rows, dtype)
    out = _run(cuda, V, *case)
    _check(case[0][:, :V], out, *case[1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("offset,pad", [(0, 1), (1, 0), (3, 13), (5, 2), (7, 64)])
def test_penalize_strides(cuda, offset, pad, dtype):
    """Rows at any distance and any alignment, and histories that are columns of a wider array."""
    import torch
    rng = np.random.default_rng([offset, pad])
    V = 9001
    case = list(_case(rng, V, 6, 40, 6, 5, dtype, stride=V + pad))
    out = _run(cuda, V, *case, offset=offset)
    _check(case[0][:, :V], out, *case[1:])
    wide = torch.from_numpy(np.concatenate([case[1], case[1][::-1]], axis=1)).to(cuda)
    x = case[0][:, :V].to(cuda).contiguous()
    T.trie_penalize(x, wide[:, 3:33], torch.from_numpy(case[2]).to(cuda))
    _check(case[0][:, :V], x.cpu(), wide[:, 3:33].cpu().numpy(), case[2], None, None, None, None, None, None, None)


@pytest.mark.parametrize("H", [1, 100, 20000, 70001])
def test_penalize_counts(cuda, H):
    """One token said over and over, ids outside the vocabulary, a token biased many times: counts and sums."""
    rng = np.random.default_rng(H)
    V, B = 40000, 4
    case = list(_case(rng, V, B, H, 60, 0, "f32", hot=7))
    case[1][0, :] = 5
    case[1][1, ::2] = -1
    case[1][1, 1::3] = V
    case[1][2, ::5] = 2 ** 31 - 1
    case[2][:] = [H, H, H + 9, -4]      # longer than the array: all of it; negative: none
    case[3][:] = [0, H // 2, 0, 0]
    case[7][1][::4] = -2 ** 31
    out = _run(cuda, V, *case)
    _check(case[0], out, *case[1:])


@pytest.mark.parametrize("stride", [4, 64, 1024, 8192])
def test_penalize_crowded_histories(cuda, stride):
    """Distinct tokens that are all multiples of one number, more of them than any table's fair share."""
    rng = np.random.default_rng(stride)
    V = 262144
    n = V // stride
    case = list(_case(rng, V, 2, n, 12, 0, "bf16"))
    case[1][:] = (np.arange(n) * stride)[None, :]
    case[2][:] = n
    out = _run(cuda, V, *case)
    _check(case[0], out, *case[1:])


@pytest.mark.parametrize("n", [4090, 20000])
def test_penalize_long_bias_lists(cuda, n):
    """Rows with more biased tokens than a table holds, beside rows with few and with none."""
    rng = np.random.default_rng(n)
    V, B = 33001, 4
    case = list(_case(rng, V, B, 500, 5, 4, "f32"))
    many = [n, 0, 7, 3]
    off = np.concatenate([[0], np.cumsum(many)]).astype(np.int32)
    tok = rng.integers(0, V, off[-1]).astype(np.int32)   # some twice
    tok[:2 * V // 3:3][:n // 3] = rng.permutation(V)[:len(tok[:2 * V // 3:3][:n // 3])]
    case[7] = (off, tok, rng.normal(0, 3, off[-1]).astype(np.float32))
    case[9][:] = [FREE, FREE, 1, 3]
    out = _run(cuda, V, *case)
    _check(case[0], out, *case[1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_penalize_special_values(cuda, dtype):
    """Infinities, NaN, zeros and the type's lowest value, touched and untouched, allowed and not."""
    import torch
    V, B = 640, 4
    rng = np.random.default_rng(5)
    case = list(_case(rng, V, B, 400, 90, 3, dtype))
    special = torch.tensor([math.inf, -math.inf, math.nan, 0.0, -0.0, -3.3895e38, 3.3895e38, 1e-45])
    case[0] = special[torch.from_numpy(rng.integers(0, 8, (B, V)))].to(case[0].dtype)
    case[7][2][::7] = math.inf
    case[9][:] = [FREE, 1, 2, FREE]
    out = _run(cuda, V, *case)
    _check(case[0], out, *case[1:])


def test_penalize_nothing(cuda):
    """No history, no bias, no grammar, empty histories, no rows: nothing changes."""
    import torch
    x = torch.randn(3, 1000, device=cuda)
    y = x.clone()
    T.trie_penalize(y)
    T.trie_penalize(y, torch.zeros(3, 0, dtype=torch.int32, device=cuda), torch.zeros(3, dtype=torch.int32, device=cuda))
    none = torch.zeros(0, dtype=torch.int32, device=cuda)
    T.trie_penalize(y, bias=(torch.zeros(4, dtype=torch.int32, device=cuda), none, none.float()))
    T.trie_penalize(y[:0])
    assert torch.equal(x, y)


def test_penalize_streams_and_graphs(cuda):
    """On a side stream, and captured in a graph that is replayed on new inputs."""
    import torch
    rng = np.random.default_rng(1)
    V, B = 5000, 3
    case = list(_case(rng, V, B, 50, 4, 3, "bf16"))
    up = [None if c is None else torch.from_numpy(np.ascontiguousarray(c)).to(cuda) for c in case[1:7]]
    bias = tuple(torch.from_numpy(c).to(cuda) for c in case[7])
    mask, states = torch.from_numpy(ref.pack(case[8])).to(cuda), torch.from_numpy(case[9]).to(cuda)
    x = case[0].to(cuda)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    T.trie_penalize(x, *up, bias, mask, states, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    _check(case[0], x.cpu(), *case[1:])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        T.trie_penalize(x, *up, bias, mask, states)
    for _ in range(2):
        fresh = torch.from_numpy(rng.normal(0, 4, (B, V)).astype(np.float32)).to(torch.bfloat16)
        x.copy_(fresh)
        graph.replay()
        _check(fresh, x.cpu(), *case[1:])


def test_penalize_refusals(cuda):
    import torch
    x = torch.zeros(2, 100, device=cuda)
    i = torch.zeros(2, dtype=torch.int32, device=cuda)
    h = torch.zeros(2, 5, dtype=torch.int32, device=cuda)
    m = torch.zeros(3, 4, dtype=torch.int32, device=cuda)
    bad = [
        (ValueError, lambda: T.trie_penalize(x.t())), (ValueError, lambda: T.trie_penalize(x[:, ::2])),
        (ValueError, lambda: T.trie_penalize(x[:1].expand(2, 100))), (TypeError, lambda: T.trie_penalize(x.half())),
        (TypeError, lambda: T.trie_penalize(x.cpu())), (ValueError, lambda: T.trie_penalize(x, h)),
        (ValueError, lambda: T.trie_penalize(x, h[:1], i)), (TypeError, lambda: T.trie_penalize(x, h.long(), i)),
        (ValueError, lambda: T.trie_penalize(x, h, i[:1])), (ValueError, lambda: T.trie_penalize(x, length=i)),
        (ValueError, lambda: T.trie_penalize(x, repetition=x[0, :3])),
        (TypeError, lambda: T.trie_penalize(x, presence=i)),
        (ValueError, lambda: T.trie_penalize(x, bias=(i, i, x[0, :2]))),
        (ValueError, lambda: T.trie_penalize(x, mask=m)), (ValueError, lambda: T.trie_penalize(x, states=i)),
        (ValueError, lambda: T.trie_penalize(x, mask=m[:, :3], states=i)),
        (T.TrieError, lambda: T.trie_penalize(x[:, :1])),
    ]
    for kind, call in bad:
        with pytest.raises(kind):
            call()
    lib = T.load_library()
    p = x.data_ptr()
    args = [p, 0, 100, 2, 100, h.data_ptr(), 5, 5, i.data_ptr()] + [None] * 8 + [0, None, None]
    assert lib.trie_penalize(*args) == T.TRIE_OK
    for at, value in [(0, None), (0, p + 2), (1, 7), (2, 99), (3, -1), (3, 65536), (4, 1), (6, 4), (7, -1), (8, None),
                      (13, p), (16, p), (18, p)]:
        wrong = list(args)
        wrong[at] = value
        assert lib.trie_penalize(*wrong) == T.TRIE_EINVAL, (at, value)
        assert T.trie_last_error()
