"""Attention of a chunk of new tokens over a paged cache, against its definition in 64 bits."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE, Chunk

pytestmark = pytest.mark.gpu

SHAPES = [
    [(0, 1)],                                   # one token that sees itself only
    [(0, 2)], [(1, 1)], [(62, 1)], [(63, 1)], [(64, 1)], [(126, 3)],
    [(5, 17)], [(127, 31)], [(0, 64)], [(0, 65)], [(0, 127)], [(1, 128)], [(0, 129)],
    [(3, 255)], [(0, 256)], [(130, 257)], [(700, 33)], [(1000, 300)], [(0, 777)],
    [(0, 0), (5, 3), (0, 0)],                   # sequences without tokens
    [(100, 0), (64, 5), (17, 0), (0, 1)],       # and without new ones
    [(0, 100), (2000, 1), (333, 70), (0, 1), (64, 64)],
]


@pytest.mark.parametrize("pairs", SHAPES, ids=str)
@pytest.mark.parametrize("heads", [(4, 1), (8, 2), (3, 3)], ids=str)
def test_lengths(pairs, heads):
    c = Chunk(pairs, *heads, seed=len(pairs))
    c.check(*c.attend())


@pytest.mark.parametrize("group", range(1, 9))
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_groups(group, out_dtype):
    c = Chunk([(70, 150), (0, 3), (500, 1), (31, 129 // group)], 2 * group, 2, seed=group, out_dtype=out_dtype)
    c.check(*c.attend())


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("pairs", [[(9000, 1)], [(9000, 40)], [(9000, 100)], [(20000, 1), (3, 5)]], ids=str)
def test_one_long_sequence_is_divided(pairs, out_dtype):
    c = Chunk(pairs, 8, 2, seed=3, out_dtype=out_dtype)
    c.check(*c.attend())


@pytest.mark.parametrize("out_dtype", [0, 1])
def test_many_tiles(out_dtype):
    c = Chunk([(1000, 1500), (0, 1100), (77, 900)], 16, 8, seed=4, out_dtype=out_dtype)
    c.check(*c.attend())


def test_many_short_sequences():
    c = Chunk([((i * 37) % 190, (i * 11) % 9) for i in range(300)], 4, 2, seed=5)
    c.check(*c.attend())


@pytest.mark.parametrize("paged", [False, True])
def test_one_token_each(paged):
    c = Chunk([(0, 1), (63, 1), (64, 1), (999, 1), (4095, 1)], 8, 2, one=True, paged=paged)
    c.check(*c.attend())


def test_one_token_each_and_a_sequence_without_any():
    c = Chunk([(0, 1), (0, 0), (64, 1)], 8, 2, one=True)
    out, lse = c.attend()
    c.check(out, lse)


def test_scale_and_a_table_with_pages_in_place():
    c = Chunk([(100, 90)], 4, 2, sm_scale=0.3, paged=False)
    c.check(*c.attend())


@pytest.mark.parametrize("pairs", [[(20000, 60)], [(2000, 300), (2048, 1), (2049, 1)], [(0, 5000)], [(2150, 30), (4096, 9)]], ids=str)
def test_binary32_results_over_many_keys(pairs):
    """The tensor cores' sums cut off, so their error grows with their length: the runs keep it where that of short ones is."""
    c = Chunk(pairs, 8, 2, seed=6, out_dtype=1)
    out, lse = c.attend()
    c.check(out, lse)
    want = c.expected()[0]
    mine = c.owned()
    # two pieces of a weight are off by up to 2^-18 of it; a run's 256 additions, each cut off by up to 2^-23, by 2^-16 of the
    # sum's size at most and, the sizes growing, by a quarter of that on average
    assert (out.double() - want)[mine].norm() <= (2.0 ** -18 + 2.0 ** -18) * want[mine].norm()
