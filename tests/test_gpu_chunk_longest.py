"""One new token behind 2^31 - 65 cached ones: rotation, attention and weighing where a token's number is next to what an int32 holds.
All blocks but a few are one page of zeros, so that most logits are 0 and most values too."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE
from tests.test_gpu_rotate import cos_sin

pytestmark = pytest.mark.gpu

BLOCKS = (1 << 25) - 1
N = BLOCKS * PAGE
SPECIAL = [1, 4097, (1 << 24) + 1, BLOCKS // 2, BLOCKS - 5, BLOCKS - 2, BLOCKS - 1]
HEADS = 2


@pytest.fixture(scope="module")
def cache():
    gen = torch.Generator(device="cuda").manual_seed(1)
    pages = len(SPECIAL) + 1
    k, v = (torch.randn(pages, 1, PAGE, D, generator=gen, device="cuda").to(torch.bfloat16) for _ in range(2))
    k[0], v[0] = 0.0, 0.0
    table = torch.zeros(1, BLOCKS, dtype=torch.int32, device="cuda")
    table[0, SPECIAL] = torch.arange(1, pages, dtype=torch.int32, device="cuda")
    q = (4.0 * torch.randn(1, HEADS, D, generator=gen, device="cuda")).to(torch.bfloat16)
    return k, v, table, torch.tensor([N], dtype=torch.int32, device="cuda"), q


def in_64_bits(k, v, q):
    """(special tokens' weights, the log-sum-exp, the result, its sum of magnitudes, the logits' own sums of magnitudes), zeros counted."""
    keys, values = k[1:, 0].flatten(0, 1).double(), v[1:, 0].flatten(0, 1).double()
    score = q[0].double() @ keys.T / math.sqrt(D)
    lse = torch.logaddexp(torch.logsumexp(score, -1), torch.full((HEADS,), math.log(N - len(keys)), dtype=torch.float64, device="cuda"))
    w = torch.exp(score - lse[:, None])
    return w, lse, w @ values, w @ values.abs(), q[0].double().abs() @ keys.abs().T / math.sqrt(D)


@pytest.mark.parametrize("rows", [True, False])
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_attention_and_weights(cache, rows, out_dtype):
    k, v, table, lens, q = cache
    cfg = ffd.Config(HEADS, 1, out_dtype=out_dtype)
    listed = dict(row_start=torch.zeros_like(lens), first_token=lens - 1) if rows else {}
    args = dict(max_blocks_per_seq=BLOCKS, workspace=ffd.new_workspace_chunk(cfg, 1, 1, BLOCKS), **listed)
    out, lse = torch.zeros(1, HEADS, D, dtype=torch.float32 if out_dtype else torch.bfloat16, device="cuda"), torch.zeros(1, HEADS, device="cuda")
    ffd.ffd_attend_chunk(cfg, q, k, v, table, lens, out, lse=lse, **args)
    w, want_lse, want, mass, size = in_64_bits(k, v, q)
    # A share is 2^31 / 148 keys in steps of 128 of which either warpgroup takes every second one and adds a step's weights in two halves:
    # 2^17 additions of a rounding each, 2^-24 of the sum; as much again for the values' sums, which cut off (2^-23)
    # and the logits' errors, 128 additions that may cut off, with a few roundings of the exponents' size
    logit = size * 128 * 2.0 ** -23 + 2.0 ** -20 * 34
    slack = 2.0 ** 17 * (2.0 ** -24 + 2.0 ** -23) + 2 * float(logit.max())
    own = 0.0 if out_dtype else 2.0 ** -8
    assert ((out[0].double() - want).abs() <= (slack + 2.0 ** -8 + own) * mass).all()
    assert ((lse[0].double() - want_lse).abs() <= slack).all()
    weight = torch.zeros(k.shape[0], 1, PAGE, device="cuda")
    ffd.ffd_weigh_kv(cfg, q, lse, k, weight, table, lens, **args)
    got = weight[1:, 0].flatten().double()
    exact = w * torch.exp(want_lse - lse[0].double())[:, None]                    # for the log-sum-exp that was given
    assert ((got - exact.sum(0)).abs() <= (exact * (logit + 2.0 ** -22)).sum(0)).all()
    assert ffd.ffd_read_device_status(args["workspace"]) == 0


def test_rotation(cache):
    k, v, table, lens, _ = cache
    cfg = ffd.Config(HEADS, 1)
    k, v, turn = k.clone(), v.clone(), cos_sin(D)
    old_k, old_v = k.clone(), v.clone()
    new_q, new_k, new_v = (torch.randn(1, h, D, device="cuda").to(torch.bfloat16) for h in (HEADS, 1, 1))
    q_out, ws = torch.zeros_like(new_q), ffd.new_workspace_chunk(cfg, 1, 1, BLOCKS)
    ffd.ffd_rotate_write_kv(cfg, new_q, new_k, new_v, q_out, k, v, table, lens, cos_sin=turn, positions=torch.tensor([0], dtype=torch.int32, device="cuda"),
                            row_start=torch.zeros_like(lens), first_token=lens - 1, max_blocks_per_seq=BLOCKS, workspace=ws)
    assert torch.equal(q_out, new_q) and torch.equal(k[-1, 0, -1], new_k[0, 0]) and torch.equal(v[-1, 0, -1], new_v[0, 0])   # turned by 0
    old_k[-1, 0, -1], old_v[-1, 0, -1] = new_k[0, 0], new_v[0, 0]
    assert torch.equal(k, old_k) and torch.equal(v, old_v) and ffd.ffd_read_device_status(ws) == 0
