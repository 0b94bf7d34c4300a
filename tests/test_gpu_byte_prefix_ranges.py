"""The byte cache and the shared prefix over more of their range, against 64 bits: other scales of the logits, batches of very uneven
lengths, long shares of a warp, own tokens that outweigh the prefix, pools beyond 32-bit offsets.  The tolerances are those of
test_gpu_byte_prefix.py, whose docstring derives them for any length, scale and batch."""
import math

import pytest
import torch

from tests.test_gpu_byte_prefix import (BLK, D, DTYPE, FORMATS, Cache, Shared, check, decode, ffd, gen,   # noqa: F401
                                        joined_values, normal, quantise, raw, with_prefix)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sm", [0.3, 1.0, 2.0 ** -9, 2.0 ** -40])
@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
def test_other_scales_of_the_logits(ffd, fmt, sm):
    for batch in (3, 40):
        g = gen(190 + batch)
        pre, c = Shared(g, 333, 2), Cache(g, fmt, [(50 * b) % 131 for b in range(batch)], 2)
        q = normal(g, batch, 8, D).to(torch.bfloat16)
        cfg = ffd.Config(8, 2, sm_scale=sm)
        out, lse, ws = with_prefix(ffd, cfg, q, pre, c)
        assert ffd.ffd_read_device_status(ws) == 0
        check(out, lse, q, joined_values(pre, c), fmt, sm=cfg.c().sm_scale)
        if fmt != "bf16":
            out, lse, ws = decode(ffd, cfg, q, c)
            check(out, lse, q, list(zip(*c.values)), fmt, sm=cfg.c().sm_scale)


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
def test_results_without_their_log_sum_exp(ffd, fmt, out_dtype):
    g = gen(191)
    pre, c = Shared(g, 200, 2), Cache(g, fmt, [0, 5, 129], 2)
    q = normal(g, 3, 6, D).to(torch.bfloat16)
    cfg = ffd.Config(6, 2, out_dtype=out_dtype)
    want, _, ws = with_prefix(ffd, cfg, q, pre, c)
    out = torch.full_like(want, math.nan)
    shared = dict(max_prefix_blocks=pre.most, max_blocks_per_seq=c.most, workspace=ws)
    if fmt == "bf16":
        k, v = torch.cat([pre.pools[0], c.k]), torch.cat([pre.pools[1], c.v])
        table = (c.index + pre.pools[0].shape[0]).to(torch.int32).contiguous()
        ffd.ffd_decode_prefix(cfg, q, k, v, pre.table, pre.len, table, c.seq_lens, out, **shared)
    else:
        ffd.ffd_decode_prefix_byte(cfg, q, *pre.pools, pre.table, pre.len, *c.byte, c.table, c.seq_lens, out, **shared)
    assert torch.equal(out, want)
    if fmt != "bf16":
        want, _, ws = decode(ffd, cfg, q, c)
        out.fill_(math.nan)
        ffd.ffd_decode_byte(cfg, q, *c.byte, c.table, c.seq_lens, out, max_blocks_per_seq=c.most, workspace=ws)
        assert torch.equal(out, want)


def ramped(c, b, lo, hi):
    """Sequence b's keys grow along it, so that each partial's sum outweighs those before it."""
    n = c.lens[b]
    t = torch.arange(n, device="cuda")
    page = c.index[b][t // BLK]
    scale = c.k_scale[page, :, t % BLK] * torch.linspace(lo, hi, n, device="cuda")[:, None]
    c.k_scale[page, :, t % BLK] = scale
    codes = raw(c.k)[page, :, t % BLK].view(c.k.dtype)
    c.values[0][b] = codes.double() * scale.double()[..., None]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,lens", [
    ((8, 8), [9000] + [1] * 63),              # 72 partials for one warp
    ((32, 8), [1] * 40 + [9000] + [0] * 23),
    ((4, 1), [131072] + [64] * 63),           # 429 partials for four warps, in several rounds
    ((1, 1), [70, 131072] + [3] * 62),
    ((6, 1), [64] * 63 + [131072])])
def test_one_long_sequence_among_short_ones(ffd, fmt, heads, lens):
    """Many more partials for some heads than for the others: the merge goes over them in rounds."""
    g = gen(192)
    c = Cache(g, fmt, lens, heads[1])
    q = normal(g, len(lens), heads[0], D).to(torch.bfloat16)
    long = lens.index(max(lens))
    for lo, hi in ((1.0, 1.0), (0.02, 4.0), (3.0, 0.01)):
        if lo != hi:
            ramped(c, long, lo, hi)
        for out_dtype in (0, 1):
            out, lse, ws = decode(ffd, ffd.Config(*heads, out_dtype=out_dtype), q, c)
            assert ffd.ffd_read_device_status(ws) == 0
            check(out, lse, q, list(zip(*c.values)), fmt)


@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
def test_a_warp_whose_share_is_longer_than_its_window_of_pages(ffd, fmt):
    """147 KV heads leave one CTA for the own tokens: a warp goes over several heads of 79 pages each, 32 of them at a time."""
    g = gen(193)
    pre, c = Shared(g, 130, 147), Cache(g, fmt, [5000], 147)
    q = normal(g, 1, 147, D).to(torch.bfloat16)
    out, lse, ws = with_prefix(ffd, ffd.Config(147, 147), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), fmt)


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
@pytest.mark.parametrize("batch,heads,prefix,own", [(64, (8, 2), 4000, 3000), (16, (16, 4), 2500, 6001)])
def test_own_tokens_that_outweigh_the_prefix(ffd, fmt, batch, heads, prefix, own, out_dtype):
    """The prefix could have many chunks, and gets few."""
    g = gen(194)
    pre, c = Shared(g, prefix, heads[1]), Cache(g, fmt, [own - 37 * b for b in range(batch)], heads[1])
    q = normal(g, batch, heads[0], D).to(torch.bfloat16)
    out, lse, ws = with_prefix(ffd, ffd.Config(*heads, out_dtype=out_dtype), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), fmt, one_piece=batch * heads[0] // heads[1] > 128 and out_dtype == 0)


def test_reading_back_beyond_32_bit_offsets(ffd):
    """Pages behind the 4 GB mark of the byte pools and of the 16-bit ones."""
    g = gen(195)
    kv, pages, cache_pages = 8, 68000, 34000          # 4.46 GB per pool each
    pool = [torch.zeros(pages, kv, BLK, D, dtype=torch.int8, device="cuda") for _ in "kv"]
    scale = [torch.zeros(pages, kv, BLK, device="cuda") for _ in "kv"]
    cache = [torch.zeros(cache_pages, kv, BLK, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    i32 = dict(dtype=torch.int32, device="cuda")
    table, to = torch.tensor([[pages - 1, 3]], **i32), torch.tensor([[cache_pages - 2, cache_pages - 1]], **i32)
    lens, ws = torch.tensor([100], **i32), torch.zeros(256, dtype=torch.uint8, device="cuda")
    t = torch.arange(100, device="cuda")
    page, dst = table[0].long()[t // BLK], to[0].long()[t // BLK]
    want = []
    for p, s in zip(pool, scale):
        code, sc = quantise(normal(g, 100, kv, D).to(torch.bfloat16), "int8")
        p[page, :, t % BLK], s[page, :, t % BLK] = code, sc
        want.append((code.float() * sc[..., None]).to(torch.bfloat16))
    ffd.ffd_read_kv_byte(ffd.Config(kv, kv), *pool, *scale, table, lens, *cache, cache_table=to, max_blocks_per_seq=2, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0
    for x, w in zip(cache, want):
        assert torch.equal(x[dst, :, t % BLK], w)
        assert not x[:-2].any() and not x[-1, :, 36:].any()


@pytest.mark.parametrize("batch", [2, 40])
def test_a_prefix_beyond_32_bit_offsets(ffd, batch):
    """The prefix's pages and the sequences' own lie behind the 4 GB mark of a 16-bit pool."""
    g = gen(196)
    kv, pages = 8, 36000                               # 4.7 GB per pool
    pools = [torch.zeros(pages, kv, BLK, D, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    at = pages - 4 - 2 * batch                         # three pages of prefix, then two for each sequence
    assert at * kv * BLK * D * 2 > 2 ** 32
    i32 = dict(dtype=torch.int32, device="cuda")
    pre_table, table = torch.arange(at, at + 3, **i32), torch.arange(at + 3, at + 3 + 2 * batch, **i32).view(batch, 2)
    lens = [(31 * b) % 129 for b in range(batch)]
    values = [[], []]
    for i, p in enumerate(pools):
        shared = normal(g, 150, kv, D).to(torch.bfloat16)
        t = torch.arange(150, device="cuda")
        p[pre_table.long()[t // BLK], :, t % BLK] = shared
        for b, n in enumerate(lens):
            mine = normal(g, n, kv, D).to(torch.bfloat16)
            if n:
                t = torch.arange(n, device="cuda")
                p[table[b].long()[t // BLK], :, t % BLK] = mine
            values[i].append(torch.cat([shared, mine]).double())
    q = normal(g, batch, 4 * kv, D).to(torch.bfloat16)
    cfg = ffd.Config(4 * kv, kv)
    out, lse = torch.full(q.shape, math.nan, device="cuda"), torch.full(q.shape[:2], math.nan, device="cuda")
    ws = ffd.new_workspace_prefix(cfg, batch, 2, 3)
    ffd.ffd_decode_prefix(cfg, q, *pools, pre_table, torch.tensor([150], **i32), table, torch.tensor(lens, **i32), out, lse=lse,
                          max_prefix_blocks=3, max_blocks_per_seq=2, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, list(zip(*values)), "bf16")
