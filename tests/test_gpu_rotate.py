"""Norm, rotation and storing of new tokens, against the definition in 64 bits."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE, Chunk

pytestmark = pytest.mark.gpu

PLACES = 5000


def cos_sin(rotary):
    half = rotary // 2
    angle = torch.arange(PLACES, device="cuda", dtype=torch.float64)[:, None] / 10000.0 ** (torch.arange(half, device="cuda", dtype=torch.float64) / half)
    return torch.stack([torch.cos(angle), torch.sin(angle)], 1).float().contiguous()


class Rotate:
    def __init__(self, c, *, rotary=D, interleaved=False, norm=True, fused=True, given=False, eps=1e-6):
        self.c, self.rotary, self.interleaved, self.eps = c, rotary, interleaved, eps
        rows, hq, hkv = c.rows, c.q_heads, c.kv_heads
        if fused:
            both = (c.randn(rows, (hq + 2 * hkv) * D) * torch.exp(c.randn(rows, 1))).to(torch.bfloat16)
            cut = (hq * D, (hq + hkv) * D)
            self.q, self.k, self.v = (x.view(rows, -1, D) for x in (both[:, :cut[0]], both[:, cut[0]:cut[1]], both[:, cut[1]:]))
        else:
            self.q, self.k, self.v = (c.randn(rows, h, D).to(torch.bfloat16) for h in (hq, hkv, hkv))
        self.q_norm, self.k_norm = ((1 + 0.3 * c.randn(D)).to(torch.bfloat16) if norm else None for _ in range(2))
        self.table = cos_sin(rotary) if rotary else None
        self.positions = torch.randint(0, PLACES, (rows,), generator=c.gen, device="cuda", dtype=torch.int32) if given else None
        self.q_out = torch.full((rows, hq, D), 7.0, dtype=torch.bfloat16, device="cuda")
        self.k_cache, self.v_cache = (torch.full_like(c.k_cache, 7.0) for _ in range(2))

    def run(self, **more):
        c = self.c
        ffd.ffd_rotate_write_kv(c.cfg, self.q, self.k, self.v, self.q_out, self.k_cache, self.v_cache, c.table, c.lens, cos_sin=self.table,
                                interleaved=self.interleaved, q_norm=self.q_norm, k_norm=self.k_norm, eps=self.eps,
                                positions=self.positions, **(c.row_args() | more))
        return self

    def turned(self, x, weight, place):
        """(what it should be, the bound of the error in 64 bits) of rows x."""
        y = x.double()
        if weight is not None:
            y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + self.eps) * weight.double()
        half = self.rotary // 2
        size = y.abs().clone()
        if half:
            i = torch.arange(half, device="cuda")
            a, b = (2 * i, 2 * i + 1) if self.interleaved else (i, i + half)
            c, s = self.table[place, 0].double()[:, None], self.table[place, 1].double()[:, None]
            z = y.clone()
            z[..., a], z[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
            size[..., a] = size[..., b] = y[..., a].abs() + y[..., b].abs()
            y = z
        # one rounding to bf16, and a few roundings in binary32 of the terms (the norm: 2^-21 with its square root)
        return y, 2.0 ** -8 * y.abs() + 2.0 ** -20 * size + 1e-40

    def check(self, left_out=()):
        c = self.c
        q, k, v = torch.full_like(self.q_out, 7.0).double(), torch.full_like(self.k_cache, 7.0).double(), torch.full_like(self.v_cache, 7.0)
        q_tol, k_tol = torch.zeros_like(q), torch.zeros_like(k)
        for b, (f, n) in enumerate(c.pairs):
            rows = torch.tensor([c.starts[b] + i for i in range(n) if c.starts[b] + i not in left_out], device="cuda", dtype=torch.long)
            if not len(rows):
                continue
            token = f + rows - c.starts[b]
            place = token if self.positions is None else self.positions[rows].long()
            q[rows], q_tol[rows] = self.turned(self.q[rows], self.q_norm, place)
            page, at = c.place(b, token)
            k[page, :, at], k_tol[page, :, at] = self.turned(self.k[rows], self.k_norm, place)
            v[page, :, at] = self.v[rows]
        assert ((self.q_out.double() - q).abs() <= q_tol).all()
        assert ((self.k_cache.double() - k).abs() <= k_tol).all()
        assert torch.equal(self.v_cache, v)


PAIRS = [(0, 1), (63, 2), (10, 0), (64, 130), (4000, 3)]


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [0, 16, 48, 64, 112, 128])
def test_rotation(rotary, interleaved, norm):
    Rotate(Chunk(PAIRS, 6, 2, seed=rotary), rotary=rotary, interleaved=interleaved, norm=norm).run().check()


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (8, 1), (15, 3), (56, 8), (7, 7)], ids=str)
@pytest.mark.parametrize("fused", [False, True])
def test_heads(heads, fused):
    c = Chunk(PAIRS, *heads, seed=3)
    Rotate(c, fused=fused, given=True).run().check()
    assert ffd.ffd_read_device_status(c.workspace) == 0


@pytest.mark.parametrize("which", ["q_norm", "k_norm"])
def test_one_norm_only(which):
    r = Rotate(Chunk(PAIRS, 3, 1, seed=5))
    setattr(r, which, None)
    r.run().check()


def test_many_rows():
    Rotate(Chunk([(0, 5000), (37, 4901)], 8, 2, seed=6), given=True).run().check()       # a warp has all heads of a token
    Rotate(Chunk([(0, 2000)], 32, 8, seed=7)).run().check()                              # a part of them


@pytest.mark.parametrize("paged", [False, True])
def test_one_token_each(paged):
    c = Chunk([(0, 1), (0, 0), (64, 1), (999, 1)], 4, 2, one=True, paged=paged)
    c.pairs[1] = (0, 0)
    Rotate(c).run().check()


def test_a_position_without_cosines():
    c = Chunk([(0, 40), (5, 9)], 4, 2, seed=8)
    r = Rotate(c, given=True)
    r.positions[c.starts[0] + 3], r.positions[c.starts[1] + 8] = -1, PLACES
    r.run().check(left_out=(c.starts[0] + 3, c.starts[1] + 8))
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_POSITION


def test_a_row_that_is_all_zero_and_one_that_is_huge():
    c = Chunk([(0, 2)], 2, 1)
    r = Rotate(c, fused=False)
    r.q[c.starts[0]] = 0.0
    r.q[c.starts[0] + 1] = 1e15
    r.run().check()
