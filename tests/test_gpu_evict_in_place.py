"""Eviction whose new lengths go where the old ones are, in a pool that is read and written."""
import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import PAGE, Chunk
from tests.test_gpu_weigh_evict import Evict, lengths

pytestmark = pytest.mark.gpu

LENGTHS = [(40000,), (9000, 30, 1, 0, 200, 201, 5000), tuple(150 + 97 * i for i in range(40))]


@pytest.mark.parametrize("n", LENGTHS, ids=len)
@pytest.mark.parametrize("heads", [1, 8])
def test_lengths_in_place(n, heads):
    for seed in range(5):
        c = Chunk(lengths(*n), heads, heads, seed=seed)
        e = Evict(c, 200, 3, 30)
        e.lens = c.lens
        e.run().check()


def test_one_pool_and_one_array_of_lengths():
    """As a serving loop would: kept tokens to free pages of the same pool, then tables and lengths are the sequences' new ones."""
    c = Chunk(lengths(700, 64, 1999, 130), 4, 4, seed=1)
    own = Evict(c, 128, 3, 30)
    own.run()                                                        # in pools and lengths of their own
    k, v = (torch.cat([x, torch.full((9, *x.shape[1:]), 7.0, dtype=x.dtype, device="cuda")]) for x in (c.k_cache, c.v_cache))
    w = torch.cat([own.weight, torch.full((9, 4, PAGE), 7.0, device="cuda")])
    table = (torch.randperm(9, generator=c.gen, device="cuda")[:8].view(4, 2) + c.pages).to(torch.int32).contiguous()
    kept, lens, before = torch.empty_like(own.kept), c.lens.clone(), w[:c.pages].clone()
    ffd.ffd_evict_kv(c.cfg, k, v, w, c.table, lens, k, v, w, table, lens, kept, n_sink=3, n_local=30, max_blocks_per_seq=c.blocks,
                     max_out_blocks=2, workspace=c.workspace)
    assert torch.equal(kept, own.kept) and lens.tolist() == [128, 64, 128, 128]
    assert torch.equal(k[:c.pages], c.k_cache) and torch.equal(v[:c.pages], c.v_cache) and torch.equal(w[:c.pages], before)
    for b, n in enumerate(lens.tolist()):
        slot = torch.arange(n, device="cuda")
        here, there = table[b].long()[slot // PAGE], own.where[b][slot // PAGE]
        for got, want in ((k, own.k), (v, own.v), (w, own.w)):
            assert torch.equal(got[here, :, slot % PAGE], want[there, :, slot % PAGE])
    assert ffd.ffd_read_device_status(c.workspace) == 0
