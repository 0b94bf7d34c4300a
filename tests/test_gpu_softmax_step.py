"""The prefix kernel's softmax step by itself: what it computes, and what it leaves alone when the product that it has to wait for
never ends."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_00097_b200 import build

pytestmark = pytest.mark.gpu

M, L = 0.5, 3.0


@pytest.fixture(scope="module")
def step(tmp_path_factory):
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    path = str(tmp_path_factory.mktemp("step") / "step.so")
    source = os.path.join(os.path.dirname(os.path.abspath(__file__)), "softmax_step_harness.cu")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), *build.NVCC_FLAGS, "-o", path, source])
    f = ctypes.CDLL(path).run_step
    p, fl, i = ctypes.c_void_p, ctypes.c_float, ctypes.c_int
    f.argtypes, f.restype = [i, p, p, fl, fl, i, p, p, p], i

    def call(pieces, scores, o, ready):
        out, ml, arrived = torch.full_like(o, -1.0), torch.zeros(32, 2, device="cuda"), torch.full((2,), -1, dtype=torch.int32, device="cuda")
        torch.cuda.synchronize()
        assert f(pieces, scores.data_ptr(), o.data_ptr(), M, L, ready, out.data_ptr(), ml.data_ptr(), arrived.data_ptr()) == 0
        return out, ml, arrived.tolist()
    return call


def inputs():
    g = torch.Generator(device="cuda").manual_seed(11)
    scores = torch.randn(32, 128, generator=g, device="cuda")
    scores[5:17, 64:] += 40.0            # some rows' second half exceeds the reference by 2^8 and more
    return scores, torch.randn(32, 128, generator=g, device="cuda")


@pytest.mark.parametrize("pieces", [1, 2])
def test_a_raise_in_the_second_half(step, pieces):
    """Each factor 2^x is off by 2^-22 relative and |x| 2^-23 from its argument (|x| < 64); sums of 128 add 2^-17 at most."""
    scores, o = inputs()
    out, ml, arrived = step(pieces, scores, o, 1)
    assert arrived == [1, 1]
    s = scores.double()
    m = torch.maximum(s[:, 64:].amax(-1), torch.tensor(M, device="cuda").double())     # the first halves stay below M + 8
    assert torch.equal(ml[:, 0], m.float())
    want = L * torch.exp2(M - m) + torch.exp2(s - m[:, None]).sum(-1)
    assert ((ml[:, 1].double() / want - 1).abs() <= 2.0 ** -16).all()
    scaled = o.double() * torch.exp2(M - m)[:, None]
    assert ((out.double() - scaled).abs() <= 2.0 ** -16 * scaled.abs()).all()


@pytest.mark.parametrize("pieces", [1, 2])
def test_a_wait_that_runs_out_is_reported_and_changes_nothing(step, pieces):
    scores, o = inputs()
    out, ml, arrived = step(pieces, scores, o, 0)
    assert ml[:, 0].isnan().all()              # what the kernel takes for the failure
    assert arrived == [1, 0]                   # the second half's weights are not announced
    assert torch.equal(out, o)                 # O, to which the product may still be adding, was not written
