"""The largest batches that the byte cache and the shared prefix accept, against 64 bits for all sequences at once.

A sequence has no token or one, so that its result is a softmax over the prefix's few tokens and that one.  The tolerances are those
of test_gpu_byte_prefix.py for these few tokens: with A the largest sm sum |q k|,  dS <= pieces sm max|q| max sum|k| + 13 2^-22 A,
the result is off by W (2 (dS + 2^-22 + 2^-16) + 2^-19) with W <= max |v|, and a bf16 piece of P or a bf16 result by 2^-8 W each."""
import math

import pytest
import torch

from tests.test_gpu_byte_prefix import BLK, D, FORMATS, PIECES, DTYPE, Shared, ffd, gen, normal, quantise, raw   # noqa: F401

pytestmark = pytest.mark.gpu


def one_token_each(g, fmt, batch, kv):
    """Page b holds sequence b's token, if it has one; its other rows hold NaN."""
    lens = (torch.rand(batch, generator=g, device="cuda") < 0.7).to(torch.int32)
    lens[0], lens[-1] = 0, 1
    byte, values = [], []
    for _ in "kv":
        code, scale = quantise(normal(g, batch, kv, D).to(torch.bfloat16), fmt)
        pool = torch.full((batch, kv, BLK, D), -1, dtype=torch.int8, device="cuda")
        pool[:, :, 0] = raw(code)
        scales = torch.full((batch, kv, BLK), math.nan, device="cuda")
        scales[:, :, 0] = scale
        byte.append((pool.view(DTYPE[fmt]), scales))
        values.append(code.double() * scale.double()[..., None])
    (k, ks), (v, vs) = byte
    return lens, (k, v, ks, vs), values


def compare(out, lse, q, own, lens, shared, fmt, one_piece):
    """q [B, Hq, D]; own: (k, v) [B, Hkv, D]; shared: (k, v) [n, Hkv, D]; in 64 bits."""
    kv = own[0].shape[1]
    qd = q.double().view(q.shape[0], kv, -1, D)
    sm = 1 / math.sqrt(D)
    s = [torch.einsum("bhgd,nhd->bhgn", qd, shared[0]) * sm, torch.einsum("bhgd,bhd->bhg", qd, own[0])[..., None] * sm]
    s[1].masked_fill_((lens == 0)[:, None, None, None], -math.inf)
    s = torch.cat(s, -1)
    want_lse = torch.logsumexp(s, -1)
    p = torch.exp(s - torch.where(want_lse == -math.inf, 0.0, want_lse)[..., None])
    n = shared[0].shape[0]
    want = torch.einsum("bhgn,nhd->bhgd", p[..., :n], shared[1]) + p[..., n:] * own[1][:, :, None]
    k1 = max([x.abs().sum(-1).max().item() for x in (shared[0], own[0]) if x.numel()])
    vmax = max([x.abs().max().item() for x in (shared[1], own[1]) if x.numel()])
    qmax = q.double().abs().max().item()
    ds = (PIECES[fmt] + 13 * 2.0 ** -22) * sm * qmax * k1
    tol = vmax * (2 * (ds + 2.0 ** -22 + 2.0 ** -16) + 2.0 ** -19 + (2.0 ** -8 if one_piece else 0))
    if out.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * vmax
    assert ((out.double().view(want.shape) - want).abs() <= tol).all()
    empty = (want_lse == -math.inf).view(lse.shape)
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()
    assert ((lse.double() - want_lse.view(lse.shape)).abs()[~empty] <= ds + 2.0 ** -19).all()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("batch,heads", [(65535, (1, 1)), (8191, (64, 8)), (21845, (9, 3))])
def test_the_most_sequences(ffd, fmt, batch, heads):
    g = gen(200)
    lens, byte, values = one_token_each(g, fmt, batch, heads[1])
    q = normal(g, batch, heads[0], D).to(torch.bfloat16)
    for out_dtype in (0, 1):
        cfg = ffd.Config(*heads, out_dtype=out_dtype)
        ws = ffd.new_workspace_prefix(cfg, batch, 1)
        out = torch.full(q.shape, math.nan, dtype=torch.float32 if out_dtype else torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:2], math.nan, device="cuda")
        ffd.ffd_decode_byte(cfg, q, *byte, None, lens, out, lse=lse, max_blocks_per_seq=1, workspace=ws)
        assert ffd.ffd_read_device_status(ws) == 0
        none = torch.zeros(0, heads[1], D, dtype=torch.float64, device="cuda")
        compare(out, lse, q, values, lens, (none, none), fmt, False)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("batch,heads,prefix", [(65535, (1, 1), 5), (8191, (64, 8), 3), (21845, (9, 3), 130)])
def test_the_most_sequences_on_a_prefix(ffd, fmt, batch, heads, prefix):
    g = gen(201)
    lens, byte, values = one_token_each(g, fmt, batch, heads[1])
    pre = Shared(g, prefix, heads[1])
    q = normal(g, batch, heads[0], D).to(torch.bfloat16)
    for out_dtype in (0, 1):
        cfg = ffd.Config(*heads, out_dtype=out_dtype)
        ws = ffd.new_workspace_prefix(cfg, batch, 1, pre.most)
        out = torch.full(q.shape, math.nan, dtype=torch.float32 if out_dtype else torch.bfloat16, device="cuda")
        lse = torch.full(q.shape[:2], math.nan, device="cuda")
        ffd.ffd_decode_prefix_byte(cfg, q, *pre.pools, pre.table, pre.len, *byte, None, lens, out, lse=lse, max_prefix_blocks=pre.most,
                                   max_blocks_per_seq=1, workspace=ws)
        assert ffd.ffd_read_device_status(ws) == 0
        compare(out, lse, q, values, lens, pre.values, fmt, out_dtype == 0)


@pytest.mark.parametrize("fmt", FORMATS)
def test_writing_and_reading_the_most_sequences(ffd, fmt):
    g = gen(202)
    batch, kv = 65535, 1
    lens = (torch.rand(batch, generator=g, device="cuda") < 0.7).to(torch.int32)
    new = [normal(g, batch, kv, D).to(torch.bfloat16) for _ in "kv"]
    pools = [torch.full((batch, kv, BLK, D), 1, dtype=torch.int8, device="cuda").view(DTYPE[fmt]) for _ in "kv"]
    scales = [torch.full((batch, kv, BLK), 0.5, device="cuda") for _ in "kv"]
    caches = [torch.full((batch, kv, BLK, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    cfg, ws = ffd.Config(1, 1), torch.zeros(256, dtype=torch.uint8, device="cuda")
    start = (lens.cumsum(0) - lens).to(torch.int32)
    first = torch.zeros_like(lens)
    for ragged in (False, True):
        for p in pools:
            raw(p).fill_(1)
        extra = dict(row_start=start, first_token=first) if ragged else {}
        ffd.ffd_write_kv_byte(cfg, *new, *pools, *scales, None, lens, max_blocks_per_seq=1, workspace=ws, **extra)
        ffd.ffd_read_kv_byte(cfg, *pools, *scales, None, lens, *caches, max_blocks_per_seq=1, workspace=ws)
        assert ffd.ffd_read_device_status(ws) == 0
        rows = start.long() if ragged else torch.arange(batch, device="cuda")
        has = lens > 0
        for x, p, s, c in zip(new, pools, scales, caches):
            code, scale = quantise(x[rows[has]], fmt)
            assert torch.equal(raw(p)[has, :, 0], raw(code)) and torch.equal(s[has, :, 0], scale)
            assert (raw(p)[~has] == 1).all() and (raw(p)[:, :, 1:] == 1).all()
            assert torch.equal(c[has, :, 0], (code.float() * scale[..., None]).to(torch.bfloat16))
            assert (c[~has] == 7.0).all() and (c[:, :, 1:] == 7.0).all()
