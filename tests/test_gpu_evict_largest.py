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


@pytest.mark.parametrize("more", [0, 40])
def test_the_longest_sequence(more):
    """2^31 - 64 tokens.  All blocks but a few are one page, whose weights are 0; the others' are positive, and all of theirs are kept, with
    `more` of the first zeros."""
    cfg, blocks, sink, local = ffd.Config(1, 1), (1 << 25) - 1, 3, 70
    n = blocks * PAGE
    special = sorted({1, 2, 4097, 5 << 20, (1 << 24) + 1, blocks // 2, blocks - 3, blocks - 2, blocks - 1})
    pages = len(special) + 1
    gen = torch.Generator(device="cuda").manual_seed(more)
    k, v = (torch.randn(pages, 1, PAGE, D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    weight = torch.rand(pages, 1, PAGE, generator=gen, device="cuda") + 0.5
    weight[0] = 0.0
    table = torch.zeros(1, blocks, dtype=torch.int32, device="cuda")
    table[0, special] = torch.arange(1, pages, dtype=torch.int32, device="cuda")
    stays = {t for x in special for t in range(x * PAGE, (x + 1) * PAGE)} | set(range(sink)) | set(range(sink, sink + more)) | set(range(n - local, n))
    stays = sorted(stays)
    budget = len(stays)
    out_blocks = (budget + PAGE - 1) // PAGE
    k_out, v_out = (torch.zeros(out_blocks, 1, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lens, out_lens = torch.tensor([n], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    kept = torch.full((1, 1, budget), -7, dtype=torch.int32, device="cuda")
    ws = ffd.new_workspace_chunk(cfg, 1, 1, blocks)
    ffd.ffd_evict_kv(cfg, k, v, weight, table, lens, k_out, v_out, None, None, out_lens, kept, n_sink=sink, n_local=local, max_blocks_per_seq=blocks,
                     max_out_blocks=out_blocks, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0 and out_lens.tolist() == [budget]
    assert kept[0, 0].tolist() == stays
    token = torch.tensor(stays, device="cuda")
    page, at = table[0, token // PAGE].long(), token % PAGE
    assert torch.equal(k_out.flatten(0, 2)[:budget], k[page, 0, at]) and torch.equal(v_out.flatten(0, 2)[:budget], v[page, 0, at])
