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


@pytest.mark.parametrize("change", [lambda c: c.row_start.__setitem__(2, c.rows), lambda c: c.row_start.__setitem__(2, c.rows + 40),
                                    lambda c: c.row_start.__setitem__(0, -200), lambda c: c.lens.__setitem__(2, -1),
                                    lambda c: c.lens.__setitem__(2, 2 ** 31 - 1), lambda c: c.first.__setitem__(1, -3)],
                         ids=["behind the last", "far behind", "before the first", "negative length", "long", "negative first token"])
def test_every_bad_sequence_is_reported(change):
    """Rows that do not exist are left out; the others' are written."""
    c = Chunk([(100, 20), (64, 30), (5, 7)], 4, 2, seed=7)
    change(c)
    r = Rotate(c).run()
    assert ffd.ffd_read_device_status(c.workspace) & ffd.DEV_BAD_SEQ_LEN
    for b in range(3):
        if int(c.row_start[b]) == c.starts[b] and int(c.lens[b]) == c.length[b] and int(c.first[b]) == c.pairs[b][0]:
            rows = slice(c.starts[b], c.starts[b] + c.pairs[b][1])
            assert (r.q_out[rows] != 7.0).any(-1).all()


def test_a_bad_sequence_among_many():
    """More sequences than the rows' CTAs have threads, a bad one among those without rows."""
    for where in (0, 4321, 8999):
        c = Chunk([(2, 1), *[(1, 0)] * 9000], 2, 1, seed=8, gap=0, room=0)
        c.row_start[where] = 0
        c.lens[where] = -1
        Rotate(c).run()
        assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_SEQ_LEN
