"""A step in which no sequence has a new token goes through all functions on new tokens alike."""
import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import PAGE, Chunk
from tests.test_gpu_rotate import Rotate

pytestmark = pytest.mark.gpu


def test_adding_nothing():
    c = Chunk([(30, 0), (5, 0)], 4, 2, seed=10, gap=0)
    Rotate(c, fused=False).run()
    _, lse = c.attend()
    weight = torch.rand(c.pages, 2, PAGE, device="cuda")
    old = weight.clone()
    ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, weight, c.table, c.lens, add=True, **c.row_args())
    assert torch.equal(weight, old) and ffd.ffd_read_device_status(c.workspace) == 0
    with pytest.raises(ffd.FfdError):        # without rows, `add` has to be given in its range all the same
        ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, weight, c.table, c.lens, add=2, **c.row_args())
