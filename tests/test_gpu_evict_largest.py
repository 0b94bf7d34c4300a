"""Eviction where counts are next to what an int32 holds."""
import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE

pytestmark = pytest.mark.gpu

LARGEST = 2147483647


@pytest.mark.parametrize("budget", [LARGEST, LARGEST - 63])
def test_the_largest_budget(budget):
    """A sequence that is shorter is kept whole; all the places behind it are marked as empty, and nothing else is written."""
    cfg, n = ffd.Config(1, 1), 100
    k, v = (torch.randn(2, 1, PAGE, D, device="cuda").to(torch.bfloat16) for _ in range(2))
    weight, lens = torch.rand(2, 1, PAGE, device="cuda"), torch.tensor([n], dtype=torch.int32, device="cuda")
    k_out, v_out, w_out = torch.full_like(k, 7.0), torch.full_like(v, 7.0), torch.full_like(weight, 7.0)
    margin = 1 << 20
    buffer = torch.full((margin + budget + margin,), -7, dtype=torch.int32, device="cuda")
    kept, out_lens = buffer[margin:margin + budget].view(1, 1, budget), torch.zeros_like(lens)
    ws = ffd.new_workspace_chunk(cfg, 1, 1, 2)
    ffd.ffd_evict_kv(cfg, k, v, weight, None, lens, k_out, v_out, w_out, None, out_lens, kept, max_blocks_per_seq=2, max_out_blocks=2, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0 and out_lens.tolist() == [n]
    assert kept[0, 0, :n].tolist() == list(range(n))
    for begin in range(n, budget, 1 << 28):
        assert int(kept[0, 0, begin:begin + (1 << 28)].max()) == -1 and int(kept[0, 0, begin:begin + (1 << 28)].min()) == -1
    assert bool((buffer[:margin] == -7).all()) and bool((buffer[margin + budget:] == -7).all())
    for got, want in ((k_out, k), (v_out, v), (w_out, weight)):
        flat, source = got.flatten(0, 2), want.flatten(0, 2)
        assert torch.equal(flat[:n], source[:n]) and bool((flat[n:] == 7.0).all())
