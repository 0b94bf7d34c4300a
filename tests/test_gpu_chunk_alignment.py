"""Every buffer of the functions on new tokens at 16 bytes behind a 32-byte boundary, which is all the alignment they ask for: the same
bits as from buffers at a 256-byte boundary."""
import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE, Chunk
from tests.test_gpu_rotate import Rotate
from tests.test_gpu_weigh_evict import Evict, lengths, lse_of

pytestmark = pytest.mark.gpu


def shifted(t):
    """A copy of `t`, 16 bytes behind a 32-byte boundary."""
    if t is None:
        return None
    skip = 16 // t.element_size()
    buffer = torch.empty(t.numel() + skip, dtype=t.dtype, device=t.device)
    assert buffer.data_ptr() % 32 == 0
    copy = buffer[skip:].view(t.shape)
    copy.copy_(t)
    assert copy.data_ptr() % 32 == 16
    return copy


def shift(o, *names):
    for name in names:
        setattr(o, name, shifted(getattr(o, name)))


# tiles that are all one share's and tiles in several parts; pairs of warpgroups and joined ones
@pytest.mark.parametrize("pairs", [[(0, 300), (64, 9)], [(9000, 1), (3, 40)], [(5000, 150)], [(300, 400)] * 6, [(0, 1)]], ids=str)
@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("buffers", [("out",), ("workspace",), ("out", "workspace", "q", "k_cache", "v_cache", "table", "lens", "row_start", "first")],
                         ids=len)
def test_attention(pairs, out_dtype, buffers):
    c = Chunk(pairs, 8, 2, seed=1, out_dtype=out_dtype)
    out, lse = c.attend()
    again, again_lse = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    shift(c, *(b for b in buffers if b != "out"))
    if "out" in buffers:
        again, again_lse = shifted(again), shifted(again_lse)
    c.attend(again, again_lse)
    assert torch.equal(again, out) and torch.equal(again_lse, lse)
    assert ffd.ffd_read_device_status(c.workspace) == 0


def test_rotation():
    r = Rotate(Chunk([(0, 90), (64, 3)], 6, 2, seed=2), fused=False, given=True)
    shift(r.c, "table", "lens", "row_start", "first", "workspace")
    shift(r, "q", "k", "v", "q_out", "k_cache", "v_cache", "q_norm", "k_norm", "table", "positions")
    r.run().check()


def test_weights():
    c = Chunk([(700, 40), (64, 3)], 8, 2, seed=3)
    lse, weight = lse_of(c), torch.zeros(c.pages, 2, PAGE, device="cuda")
    ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, weight, c.table, c.lens, **c.row_args())
    again, lse = shifted(torch.zeros_like(weight)), shifted(lse)
    shift(c, "q", "k_cache", "table", "lens", "row_start", "first", "workspace")
    ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, again, c.table, c.lens, **c.row_args())
    assert torch.equal(again, weight)


def test_eviction():
    e = Evict(Chunk(lengths(500, 30, 900), 2, 2, seed=4), 200, 3, 30)
    shift(e.c, "k_cache", "v_cache", "table", "lens", "workspace")
    shift(e, "weight", "k", "v", "w", "table", "lens", "kept")
    assert e.k.shape[-1] == D
    e.run().check()
