"""Values that are no numbers, where a CTA's share has many tiles: they reach the rows that see them, and no other sequence, head or
earlier row, bit for bit.  A share holds notes of such values for its last eight segments; here it has more of them."""
import math

import pytest
import torch

from tests.chunk_cases import Chunk

pytestmark = pytest.mark.gpu

HEADS = (32, 8)
BATCHES = {
    "prompt-on-long": [(100, 512), (16000, 512)] * 2,
    "two": [(100, 512), (16000, 512)],
    "chunks": [(700 + 40 * i, 512) for i in range(32)],
    "drafts": [(1000 + 13 * i, 5) for i in range(256)],
}
CHANNEL = 5


def compare(c, clean, spots):
    """`spots`: {(sequence, KV head): token whose value in CHANNEL is no number}.  A call on it against the clean call's results."""
    kept = {}
    for (b, g), t in spots.items():
        page, at = c.place(b, t)
        kept[b, g] = c.v_cache[page, g, at, CHANNEL].clone()
        c.v_cache[page, g, at, CHANNEL] = (math.inf, -math.inf, math.nan)[t % 3]
    out, lse = c.attend()
    assert torch.equal(lse, clean[1])
    touched = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    for (b, g), t in spots.items():
        first, n = c.pairs[b]
        touched[c.starts[b] + t - first:c.starts[b] + n, g * c.group:(g + 1) * c.group] = True
    assert not out[touched][:, CHANNEL].isfinite().any()
    same = torch.ones(out.shape, dtype=torch.bool, device="cuda")
    same[..., CHANNEL] = ~touched
    wrong = (out != clean[0]) & same
    assert not wrong.any(), wrong.nonzero()[:5].tolist()
    for (b, g), t in spots.items():
        page, at = c.place(b, t)
        c.v_cache[page, g, at, CHANNEL] = kept[b, g]


@pytest.mark.parametrize("name,out_dtype,where", [("prompt-on-long", 1, (0, 7, 560)), ("two", 1, (0, 0, 300)), ("chunks", 0, (1, 1, 810)),
                                                  ("drafts", 0, (2, 6, 1028))])
def test_one_value(name, out_dtype, where):
    c = Chunk(BATCHES[name], *HEADS, seed=1, out_dtype=out_dtype)
    compare(c, c.attend(), {where[:2]: where[2]})


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_many_values(name, out_dtype):
    """Every second KV head of every sequence has one, in its first, middle or last new token."""
    c = Chunk(BATCHES[name], *HEADS, seed=2, out_dtype=out_dtype)
    clean = c.attend()
    for odd in (0, 1):
        for part in (0.3, 0.5, 1.0):
            compare(c, clean, {(b, g): f + max(1, int(part * n) - 1) for b, (f, n) in enumerate(c.pairs) for g in range(odd, HEADS[1], 2)})
    again = c.attend()
    assert torch.equal(again[0], clean[0]) and torch.equal(again[1], clean[1])
