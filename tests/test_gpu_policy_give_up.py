"""The policy loss where a wait within it gives up (a stalled GPU): what it writes is right or NaN, nothing else is
written, and it ends; and on a device of any number. Built from the library's source with waits that a plan ends
(policy_give_up.cu)."""
from __future__ import annotations

import ctypes
import math
import os
import shutil
import subprocess

import numpy as np
import pytest

import logits_ref as lref
from paper_2608_12574_gb300 import _build
from paper_2608_12574_gb300 import triemask as T

pytestmark = pytest.mark.gpu
WORKERS, SENDER, FINISHER, BRINGERS = 15, 15, 16, 17  # warps of a CTA


@pytest.fixture(scope="module")
def cuda():
    import torch
    if not torch.cuda.is_available():
        pytest.fail("no CUDA device")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def planned(cuda, tmp_path_factory):
    """A library of trie_policy_loss and plan_give_up."""
    out = str(tmp_path_factory.mktemp("policy") / "policy_give_up.so")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "policy_give_up.cu")
    subprocess.run([_build.NVCC, "-shared", "-cudart", "shared", source, "-o", out, "-I", _build.CSRC, *_build.CUDA_FLAGS], check=True)
    return _load(out)


def _load(path):
    lib = ctypes.CDLL(str(path))
    lib.trie_policy_loss.restype, lib.trie_policy_loss.argtypes = T.SIGNATURES["trie_policy_loss"]
    return lib


class Case:
    def __init__(self, dev, B, V, dtype, in_place):
        import torch
        rng = np.random.default_rng([B, V])
        allowed = rng.random((4, V)) < np.array([3 / V, 40 / V, 0.5, 0.002])[:, None]
        allowed[:, V // 3] = True
        self.B, self.V, self.in_place = B, V, in_place
        put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dev)  # noqa: E731
        self.mask = put(lref.pack(allowed))
        self.states = put(rng.choice([0, 1, 2, 3, -3, -3, -3], B).astype(np.int32))
        self.logits = put(rng.normal(0, 2, (B, V)).astype(np.float32)).to(dtype)
        self.tokens = torch.full((B,), V // 3, dtype=torch.int32, device=dev)
        self.old = torch.full((B,), -math.log(V), device=dev)
        self.A = put(rng.normal(0, 1, B).astype(np.float32))

    def run(self, lib):
        """(losses, log-probabilities, gradient), of which 64 more entries than it has are looked at."""
        import torch
        B, V, dev = self.B, self.V, self.logits.device
        losses, logprobs = torch.full((2, B + 64), 7.0, device=dev)
        buf = torch.full((B + 1, V + 7), 7.0, dtype=self.logits.dtype, device=dev)
        x = self.logits
        if self.in_place:
            buf[:B, :V] = x
            x = buf
        got = lib.trie_policy_loss(
            x.data_ptr(), 0 if x.dtype is torch.float32 else 1, x.stride(0), B, V, self.tokens.data_ptr(), self.old.data_ptr(),
            self.A.data_ptr(), self.old.data_ptr(), None, None, 0.2, 0.2, 0.1, self.mask.data_ptr(), self.mask.shape[0],
            self.states.data_ptr(), losses.data_ptr(), logprobs.data_ptr(), buf.data_ptr(), buf.stride(0),
            torch.cuda.current_stream().cuda_stream)
        assert got == 0
        torch.cuda.synchronize()
        assert bool((losses[B:] == 7).all()) and bool((logprobs[B:] == 7).all())
        assert bool((buf[B] == 7).all()) and bool((buf[:, V:] == 7).all())
        return losses[:B], logprobs[:B], buf[:B, :V]


def test_any_device(cuda, planned, tmp_path):
    """A device whose number is beyond the library's tables: in a library of its own, which has not been called before."""
    import torch
    c = Case(cuda, 300, 60003, torch.bfloat16, False)
    assert planned.plan_give_up(-1, 0, 0) == 0
    want = c.run(planned)
    lib = _load(shutil.copy(planned._name, tmp_path / "another.so"))
    lib.pretend_device(16)
    for _ in range(2):
        for t, ref in zip(c.run(lib), want):
            assert torch.equal(t, ref)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,V,dtype,ctas,clusters", [(700, 9001, "bf16", 1, 152), (400, 60003, "bf16", 2, 76), (100, 131071, "f32", 8, 18),
                                                     (40, 220001, "f32", 16, 7)])
def test_give_up(cuda, planned, B, V, dtype, ctas, clusters, in_place):
    """clusters: about so many are at work, so that each takes some rows."""
    import torch
    c = Case(cuda, B, V, {"f32": torch.float32, "bf16": torch.bfloat16}[dtype], in_place)
    assert planned.plan_give_up(-1, 0, 0) == 0
    want = c.run(planned)
    assert not any(bool(t.isnan().any()) for t in want)
    for warp in (0, WORKERS - 1, SENDER, FINISHER, BRINGERS, BRINGERS + 2):
        for rank in {0, ctas - 1}:
            for after in (0, 1, 2, 3, 5):
                if after > {SENDER: 3, FINISHER: 3, BRINGERS: 1, BRINGERS + 2: 0}.get(warp, 5):
                    continue  # it has no such wait
                assert planned.plan_give_up(ctas + rank, warp, after) == 0  # in the second cluster
                got = c.run(planned)
                bad = [t.isnan() for t in got]
                rows = (bad[0] | bad[1] | bad[2].any(dim=1)).nonzero()[:, 0]
                assert len(rows) and len(rows) <= (B + clusters // 2 - 1) // (clusters // 2), (warp, rank, after)
                for t, nan, ref in zip(got, bad, want):
                    assert torch.equal(t[~nan], ref[~nan]), (warp, rank, after)
    assert planned.plan_give_up(-1, 0, 0) == 0
    for t, ref in zip(c.run(planned), want):
        assert torch.equal(t, ref)
