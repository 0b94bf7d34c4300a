"""Chunks of new tokens over a paged cache, and what the functions on them should give, in 64 bits and plain torch operations."""
import math

import torch

from paper_2609_00097_b200 import ffd

D, PAGE = 128, 64


class Chunk:
    """Sequences with `first` cached and `n` new tokens each, the new ones in the cache too; `gap` rows belong to nobody in front
    of every sequence's and behind the last.  Pages are in random order, and what belongs to no token is NaN."""

    def __init__(self, pairs, q_heads, kv_heads, *, seed=0, out_dtype=0, paged=True, gap=1, one=False, sm_scale=0.0, room=1, q_scale=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.gen, self.pairs, self.q_heads, self.kv_heads = gen, pairs, q_heads, kv_heads
        self.group = q_heads // kv_heads
        self.batch = len(pairs)
        self.cfg = ffd.Config(q_heads, kv_heads, out_dtype=out_dtype, sm_scale=sm_scale)
        self.sm = sm_scale or 1.0 / math.sqrt(D)
        self.length = [f + n for f, n in pairs]
        self.blocks = max(1, max((x + PAGE - 1) // PAGE for x in self.length)) + room
        if paged:
            self.pages = self.batch * self.blocks + 3
            order = torch.randperm(self.pages, generator=gen, device="cuda")[:self.batch * self.blocks]
            self.where = order.view(self.batch, self.blocks)
            self.table = self.where.to(torch.int32).contiguous()
        else:
            self.pages = self.batch * self.blocks
            self.where = torch.arange(self.pages, device="cuda").view(self.batch, self.blocks)
            self.table = None
        self.lens = torch.tensor(self.length, dtype=torch.int32, device="cuda")
        starts, at = [], 0
        for _, n in pairs:
            at += 0 if one else gap
            starts.append(at)
            at += 1 if one else n
        self.starts = starts
        self.rows = at if one else at + gap
        self.one = one
        self.row_start = None if one else torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.first = None if one else torch.tensor([f for f, _ in pairs], dtype=torch.int32, device="cuda")
        self.q = (self.randn(max(self.rows, 1), q_heads, D) * q_scale).to(torch.bfloat16)[:self.rows]
        self.k_cache = torch.full((self.pages, kv_heads, PAGE, D), math.nan, dtype=torch.bfloat16, device="cuda")
        self.v_cache = self.k_cache.clone()
        for b, n in enumerate(self.length):
            page, at = self.place(b, torch.arange(n, device="cuda"))
            self.k_cache[page, :, at] = self.randn(n, kv_heads, D).to(torch.bfloat16)
            self.v_cache[page, :, at] = self.randn(n, kv_heads, D).to(torch.bfloat16)
        self.workspace = ffd.new_workspace_chunk(self.cfg, self.batch, max(self.rows, 1), self.blocks)

    def randn(self, *shape):
        return torch.randn(*shape, generator=self.gen, device="cuda")

    def place(self, b, token):
        return self.where[b][token // PAGE], token % PAGE

    def tokens(self, pool, b, g):
        """[tokens, ...] of sequence b and KV head g, in 64 bits."""
        page, at = self.place(b, torch.arange(self.length[b], device="cuda"))
        return pool[page, g, at].double()

    def row_args(self):
        return dict(row_start=self.row_start, first_token=self.first, max_blocks_per_seq=self.blocks, workspace=self.workspace)

    def attend(self, out=None, lse=None):
        dtype = torch.float32 if self.cfg.out_dtype else torch.bfloat16
        out = torch.full((self.rows, self.q_heads, D), 7.0, dtype=dtype, device="cuda") if out is None else out
        lse = torch.full((self.rows, self.q_heads), 7.0, device="cuda") if lse is None else lse
        ffd.ffd_attend_chunk(self.cfg, self.q, self.k_cache, self.v_cache, self.table, self.lens, out, lse=lse, **self.row_args())
        return out, lse

    def logits(self, b, h):
        """([n, tokens] logits of head h, -inf where a token is not seen; the sums of the products' magnitudes)."""
        f, n = self.pairs[b]
        q = self.q[self.starts[b]:self.starts[b] + n, h].double()
        k = self.tokens(self.k_cache, b, h // self.group)
        hidden = torch.arange(f + n, device="cuda")[None, :] > f + torch.arange(n, device="cuda")[:, None]
        return (q @ k.T * self.sm).masked_fill(hidden, -math.inf), (q.abs() @ k.abs().T * self.sm).masked_fill(hidden, 0.0)

    def owned(self):
        """Rows that belong to a sequence."""
        mine = torch.zeros(self.rows, dtype=torch.bool, device="cuda")
        for s, (f, n) in zip(self.starts, self.pairs):
            mine[s:s + n] = True
        return mine

    def expected(self):
        """(out, sums of weight * |value|, lse, bound of a logit's error) in 64 bits."""
        out = torch.full((self.rows, self.q_heads, D), 7.0, dtype=torch.float64, device="cuda")
        mass, lse = torch.zeros_like(out), torch.full((self.rows, self.q_heads), 7.0, dtype=torch.float64, device="cuda")
        slack = torch.zeros_like(lse)
        for b, (f, n) in enumerate(self.pairs):
            if n == 0:
                continue
            rows = slice(self.starts[b], self.starts[b] + n)
            for h in range(self.q_heads):
                score, size = self.logits(b, h)
                v = self.tokens(self.v_cache, b, h // self.group)
                w = torch.softmax(score, -1)
                out[rows, h], mass[rows, h] = w @ v, w @ v.abs()
                lse[rows, h] = torch.logsumexp(score, -1)
                # 128 products, exact in binary32, in binary32 sums that may cut off instead of rounding: 2^-23 of the magnitudes
                # for each addition; scaling and the power of two add a few 2^-24 of the result's own size
                slack[rows, h] = (size.amax(-1) * 128 * 2.0 ** -23) + 2.0 ** -20 * (1 + lse[rows, h].abs())
        return out, mass, lse, slack

    def check(self, out, lse):
        want, mass, want_lse, slack = self.expected()
        mine = self.owned()
        assert (out[~mine] == 7.0).all() and (lse[~mine] == 7.0).all()
        # weights rounded to 8 or 16 bits, the result to its type, weights off by the logits' errors
        piece = 2.0 ** -16 if self.cfg.out_dtype else 2.0 ** -8
        own = 2.0 ** -24 if self.cfg.out_dtype else 2.0 ** -8
        bound = own * want.abs() + (piece + 2.0 * slack[..., None]) * mass + 1e-30
        off = (out.double() - want).abs()
        assert (off <= bound).all(), (off / bound).max().item()
        lse_off = (lse.double() - want_lse).abs()
        assert (lse_off <= slack + 1e-30)[mine].all(), (lse_off / slack)[mine].max().item()
        assert ffd.ffd_read_device_status(self.workspace) == 0
