"""Which rows belong to which sequence, where some sequences have no new tokens or none that exist."""
import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import Chunk
from tests.test_gpu_rotate import Rotate

pytestmark = pytest.mark.gpu

# sequences without new tokens may begin at any row between their neighbours' beginnings
LAYOUTS = {
    "behind": ([(0, 5), (7, 0)], [0, 0]),
    "in front": ([(7, 0), (0, 5)], [0, 0]),
    "inside": ([(60, 9), (3, 0), (0, 0), (64, 4), (100, 0)], [1, 4, 9, 11, 12]),
    "many": ([(3, 70), *[(9, 0)] * 200, (0, 6), *[(1, 0)] * 31], [2, *[2 + i // 4 for i in range(200)], 80, *[83] * 31]),
    "gap": ([(3, 4), (5, 0), (5, 2)], [0, 6, 9]),
}


def laid_out(name):
    pairs, starts = LAYOUTS[name]
    c = Chunk(pairs, 6, 2, seed=len(pairs))
    c.starts, c.rows = starts, max(s + n for s, (_, n) in zip(starts, pairs)) + 3
    c.row_start = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.q = c.randn(c.rows, 6, 128).to(torch.bfloat16)
    return c


@pytest.mark.parametrize("name", LAYOUTS)
def test_sequences_without_new_tokens(name):
    c = laid_out(name)
    Rotate(c).run().check()
    c.check(*c.attend())
    assert ffd.ffd_read_device_status(c.workspace) == 0
