"""Binary32 results of a chunk's attention are as near to 64 bits as the formula in plain binary32 operations is."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import Chunk

pytestmark = pytest.mark.gpu


def plain(c):
    """The results and log-sum-exps in binary32 operations."""
    out, lse = torch.zeros(c.rows, c.q_heads, 128, device="cuda"), torch.zeros(c.rows, c.q_heads, device="cuda")
    allowed = torch.backends.cuda.matmul.allow_tf32
    torch.backends.cuda.matmul.allow_tf32 = False
    for b, (f, n) in enumerate(c.pairs):
        rows = slice(c.starts[b], c.starts[b] + n)
        for h in range(c.q_heads if n else 0):
            k, v = (c.tokens(x, b, h // c.group).float() for x in (c.k_cache, c.v_cache))
            score = c.q[rows, h].float() @ k.T * c.sm
            score.masked_fill_(torch.arange(f + n, device="cuda")[None, :] > f + torch.arange(n, device="cuda")[:, None], -math.inf)
            top = score.amax(-1, keepdim=True)
            w = torch.exp(score - top)
            out[rows, h] = w @ v / w.sum(-1, keepdim=True)
            lse[rows, h] = (top + torch.log(w.sum(-1, keepdim=True)))[:, 0]
    torch.backends.cuda.matmul.allow_tf32 = allowed
    return out, lse


@pytest.mark.parametrize("scale", [0.3, 1.0, 3.0])
@pytest.mark.parametrize("pairs,heads", [([(0, 64)], (8, 2)), ([(0, 300), (500, 70)], (8, 2)), ([(0, 2047)], (4, 4)), ([(4000, 64)], (6, 2)),
                                         ([(20000, 5)], (8, 1)), ([(65000, 1)], (8, 2)), ([(0, 1)], (5, 1)),
                                         ([(63, 1), (64, 2), (65, 1), (127, 130)], (8, 2))], ids=str)
def test_error(pairs, heads, scale):
    c = Chunk(pairs, *heads, seed=3, out_dtype=1, q_scale=scale)
    out, lse = c.attend()
    c.check(out, lse)
    want, _, want_lse, _ = c.expected()
    near, near_lse = plain(c)
    mine = c.owned()

    def error(x, y):
        return float((x.double() - y)[mine].norm() / y[mine].norm())

    # Both sides round every weight, logit and sum to 24 bits, in another order, and the tensor cores' sums of eight terms cut off, which
    # is twice a rounding: up to twice the error, and for results of a few keys a few roundings, 2^-22, more
    assert error(out, want) <= 2 * error(near, want) + 2.0 ** -22
    assert error(lse, want_lse) <= 2 * error(near_lse, want_lse) + 2.0 ** -22


def test_one_large_logit_among_many():
    """Weights far below the largest one keep their bits: a token that has much of the weight and a value of 0 takes nothing of the
    others' result."""
    c = Chunk([(3000, 1)], 4, 1, seed=4, out_dtype=1)
    page, at = c.place(0, 1234)
    c.k_cache[page, 0, at] = (c.q[c.starts[0]].float().mean(0) * 3).to(torch.bfloat16)
    c.v_cache[page, 0, at] = 0.0
    out, lse = c.attend()
    c.check(out, lse)
    want, _, _, _ = c.expected()
    row = c.starts[0]
    assert float((out.double() - want)[row].norm() / want[row].norm()) < 2.0 ** -19      # logits of up to 30, off by 2^-21 of that
    assert ffd.ffd_read_device_status(c.workspace) == 0


def test_a_graph_replays_other_lengths_and_calls_overlap():
    c = Chunk([(700, 140), (64, 3), (0, 330)], 8, 2, seed=9, out_dtype=1)
    out, lse = c.attend()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.attend(out, lse)
    other = Chunk([(5000, 40), (9, 300)], 8, 2, seed=10, out_dtype=1)
    want, want_lse = other.attend()
    got, got_lse = torch.empty_like(want), torch.empty_like(want_lse)
    for pairs in ([(700, 140), (64, 3), (0, 330)], [(300, 11), (0, 2), (60, 270)], [(0, 0), (0, 1), (0, 0)]):
        c.pairs, c.length = pairs, [f + n for f, n in pairs]
        c.lens.copy_(torch.tensor(c.length, device="cuda"))
        c.first.copy_(torch.tensor([f for f, _ in pairs], device="cuda"))
        out.fill_(7.0), lse.fill_(7.0), got.fill_(7.0), got_lse.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(3):                       # replays on one stream, calls with another workspace on a second
            graph.replay()
            with torch.cuda.stream(side):
                other.attend(got, got_lse)
        torch.cuda.synchronize()
        c.check(out, lse)
        rows = other.owned()
        assert torch.equal(got[rows], want[rows]) and torch.equal(got_lse[rows], want_lse[rows])


def test_the_same_call_gives_the_same_bits():
    c = Chunk([(3000, 70), (0, 300), (17, 1)], 8, 2, seed=8, out_dtype=1)
    a = c.attend()
    for _ in range(5):
        b = c.attend()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("group", [3, 8])
def test_bad_pages(group):
    """A bad page in the middle of a context, and one at its end, leave their tokens out and are reported."""
    for where in (1, 5, 8):
        c = Chunk([(400, 150), (0, 40)], group, 1, seed=group, out_dtype=1)
        c.table[0, where] = -1
        out, lse = c.attend()
        assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
        gone = torch.arange(550, device="cuda") // 64 == where
        logits = c.logits

        def without(b, h):
            score, size = logits(b, h)
            return (score.masked_fill(gone, -math.inf), size) if b == 0 else (score, size)

        c.logits = without
        c.check(out, lse)
