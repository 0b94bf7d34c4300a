"""The attention weight of cached tokens, and eviction by it, against their definitions."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE, Chunk

pytestmark = pytest.mark.gpu


def lse_of(c):
    lse = torch.full((c.rows, c.q_heads), math.nan, device="cuda")
    for b, (f, n) in enumerate(c.pairs):
        for h in range(c.q_heads if n else 0):
            lse[c.starts[b]:c.starts[b] + n, h] = torch.logsumexp(c.logits(b, h)[0], -1).float()
    return lse


def weigh(c, lse, add=False):
    weight = torch.rand(c.pages, c.kv_heads, PAGE, generator=c.gen, device="cuda")
    old = weight.clone()
    ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, weight, c.table, c.lens, add=add, **c.row_args())
    want, tol = old.double(), torch.zeros_like(old).double()
    for b, (f, n) in enumerate(c.pairs):
        token = torch.arange(f + n, device="cuda")
        page, at = c.place(b, token)
        for g in range(c.kv_heads if f + n else 0):
            total, slack = torch.zeros(f + n, dtype=torch.float64, device="cuda"), torch.zeros(f + n, dtype=torch.float64, device="cuda")
            for h in range(g * c.group, (g + 1) * c.group):
                score, size = c.logits(b, h)
                w = torch.exp(score - lse[c.starts[b]:c.starts[b] + n, h].double()[:, None])
                w = torch.where(torch.isnan(w), 0.0, w) if n else w
                total += w.sum(0)
                # a weight is off by its logit's error, by roundings of the exponent's size and of the sum
                slack += (w * (size * 128 * 2.0 ** -23 + 2.0 ** -20 * (1 + score.abs().clamp(max=1e4)))).sum(0)
            kept = old[page, g, at].double() * (token < f) if add else 0.0
            want[page, g, at] = total + kept
            tol[page, g, at] = slack + (n * c.group + 2) * 2.0 ** -24 * (total + kept)
    off = (weight.double() - want).abs()
    assert (off <= tol).all(), (off - tol).max().item()
    return weight


PAIRS = [[(0, 1)], [(0, 5), (127, 1), (128, 3), (0, 0), (40, 0)], [(255, 1), (256, 1), (257, 2)], [(300, 64)], [(100, 200), (0, 129), (900, 33)],
         [(0, 700)], [(3000, 2)]]


@pytest.mark.parametrize("pairs", PAIRS, ids=str)
@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("heads", [(4, 1), (6, 2)], ids=str)
def test_weigh(pairs, add, heads):
    c = Chunk(pairs, *heads, seed=len(pairs))
    weigh(c, lse_of(c), add)
    assert ffd.ffd_read_device_status(c.workspace) == 0


@pytest.mark.parametrize("group", range(1, 9))
def test_weigh_groups(group):
    c = Chunk([(200, 131), (700, 3), (0, 300)], 2 * group, 2, seed=group)
    weigh(c, lse_of(c), True)


def test_weigh_many():
    c = Chunk([((i * 97) % 900, (i * 7) % 5) for i in range(120)], 4, 2, seed=9)
    weigh(c, lse_of(c), True)
    c = Chunk([(6000, 64), (100, 900)], 16, 8, seed=10)
    weigh(c, lse_of(c))


@pytest.mark.parametrize("paged", [False, True])
def test_weigh_one_token_each(paged):
    c = Chunk([(0, 1), (0, 0), (64, 1), (999, 1)], 4, 2, one=True, paged=paged)
    weigh(c, lse_of(c), True)


def test_weigh_heads_without_tokens_and_repeated():
    c = Chunk([(70, 30)], 4, 2, seed=11)
    lse = lse_of(c)
    lse[c.starts[0] + 4, 1] = -math.inf
    for h in (1,):
        c.logits_of = c.logits
    want = c.logits

    def without(b, h):
        score, size = want(b, h)
        if h == 1:
            score[4] = -math.inf
        return score, size

    c.logits = without
    a = weigh(c, lse)
    again = torch.rand_like(a)
    ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, again, c.table, c.lens, **c.row_args())
    page, at = c.place(0, torch.arange(100, device="cuda"))
    assert torch.equal(a[page, :, at], again[page, :, at])


# ---- eviction ------------------------------------------------------------------------------------------------------------


def chosen(w, budget, sink, local):
    """Tokens that stay, by the definition."""
    n = len(w)
    if n <= budget:
        return list(range(n))
    key = [-math.inf if math.isnan(x) else x for x in w]
    nan = [math.isnan(x) for x in w]
    middle = sorted(range(sink, n - local), key=lambda t: (nan[t], -key[t], t))[:budget - sink - local]
    return sorted(list(range(sink)) + middle + list(range(n - local, n)))


class Evict:
    def __init__(self, c, budget, sink=0, local=0, weight=None, out_paged=True):
        self.c, self.budget, self.sink, self.local = c, budget, sink, local
        c.k_cache.nan_to_num_(nan=3.0)
        c.v_cache.nan_to_num_(nan=3.0)
        self.weight = c.randn(c.pages, c.kv_heads, PAGE) if weight is None else weight
        self.blocks = (budget + PAGE - 1) // PAGE + 1
        pages = c.batch * self.blocks + 2
        order = torch.randperm(pages, generator=c.gen, device="cuda")[:c.batch * self.blocks].view(c.batch, self.blocks)
        self.where = order if out_paged else torch.arange(c.batch * self.blocks, device="cuda").view(c.batch, self.blocks)
        self.table = self.where.to(torch.int32).contiguous() if out_paged else None
        self.k, self.v = (torch.full((pages, c.kv_heads, PAGE, D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        self.w = torch.full((pages, c.kv_heads, PAGE), 7.0, device="cuda")
        self.lens = torch.full((c.batch,), -5, dtype=torch.int32, device="cuda")
        self.kept = torch.full((c.batch, c.kv_heads, budget), -7, dtype=torch.int32, device="cuda")

    def run(self):
        c = self.c
        ffd.ffd_evict_kv(c.cfg, c.k_cache, c.v_cache, self.weight, c.table, c.lens, self.k, self.v, self.w, self.table, self.lens, self.kept,
                         n_sink=self.sink, n_local=self.local, max_blocks_per_seq=c.blocks, max_out_blocks=self.blocks, workspace=c.workspace)
        return self

    def check(self):
        c = self.c
        k, v, w = torch.full_like(self.k, 7.0), torch.full_like(self.v, 7.0), torch.full_like(self.w, 7.0)
        for b, n in enumerate(c.length):
            assert self.lens[b] == min(n, self.budget)
            for g in range(c.kv_heads):
                page, at = c.place(b, torch.arange(n, device="cuda"))
                stays = chosen(self.weight[page, g, at].tolist(), self.budget, self.sink, self.local)
                got = self.kept[b, g].tolist()
                assert got == stays + [-1] * (self.budget - len(stays)), (b, g)
                slot, token = torch.arange(len(stays), device="cuda"), torch.tensor(stays, device="cuda", dtype=torch.long)
                to, (source, row) = self.where[b][slot // PAGE], c.place(b, token)
                k[to, g, slot % PAGE], v[to, g, slot % PAGE] = c.k_cache[source, g, row], c.v_cache[source, g, row]
                w[to, g, slot % PAGE] = self.weight[source, g, row]
        assert torch.equal(self.k, k) and torch.equal(self.v, v)
        assert torch.equal(self.w.nan_to_num(nan=99.0), w.nan_to_num(nan=99.0))
        assert ffd.ffd_read_device_status(c.workspace) == 0


def lengths(*n):
    return [(x, 0) for x in n]


@pytest.mark.parametrize("budget,sink,local", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (64, 4, 20), (65, 0, 65), (100, 60, 40), (130, 0, 0), (500, 1, 300)])
def test_evict(budget, sink, local):
    c = Chunk(lengths(0, 1, 63, 64, 65, 129, 500, 501, 1300), 4, 2, seed=budget)
    Evict(c, budget, sink, local).run().check()


@pytest.mark.parametrize("paged", [False, True])
def test_evict_long(paged):
    c = Chunk(lengths(20001, 4096, 17), 2, 1, seed=1, paged=paged)
    Evict(c, 3000, 7, 100, out_paged=paged).run().check()


def test_evict_one_long_sequence_in_a_cluster():
    c = Chunk(lengths(70013), 1, 1, seed=2)
    Evict(c, 5003, 64, 999).run().check()


def test_evict_more_tokens_than_shared_memory_holds():
    c = Chunk(lengths(50000, *[3] * 160), 1, 1, seed=3)     # a CTA for each sequence: the longest is read again
    Evict(c, 700, 3, 30).run().check()


@pytest.mark.parametrize("values", ["zeros", "few", "special"])
def test_evict_ties_and_special_weights(values):
    c = Chunk(lengths(1000, 3333), 4, 2, seed=4)
    shape = (c.pages, c.kv_heads, PAGE)
    if values == "zeros":
        w = torch.zeros(shape, device="cuda")
        w[..., ::2] = -0.0                                     # equal to 0
    elif values == "few":
        w = torch.randint(0, 3, shape, generator=c.gen, device="cuda").float()
    else:
        pick = torch.tensor([math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-45, -1e-45, 3.4e38, -3.4e38, 1.0], device="cuda")
        w = pick[torch.randint(0, 10, shape, generator=c.gen, device="cuda")]
    for budget in (10, 333, 950):
        Evict(c, budget, 3, 5, weight=w).run().check()


def test_evict_without_weights_out():
    c = Chunk(lengths(300), 2, 2, seed=5)
    e = Evict(c, 100, 4, 4)
    full, e.w = e.w, None
    e.run()
    e.w = full
    page, at = c.place(0, torch.arange(300, device="cuda"))
    assert e.kept[0, 1].tolist() == chosen(e.weight[page, 1, at].tolist(), 100, 4, 4)


def test_evict_with_a_budget_beyond_the_table():
    c = Chunk(lengths(90, 40), 2, 1, seed=7)
    e = Evict(c, 500, 4, 4)
    e.blocks = 2
    e.where = e.where[:, :2].contiguous()
    e.table = e.where.to(torch.int32).contiguous()
    e.run().check()                                            # the sequences fit: kept whole
    e.blocks, e.where, e.table = 1, e.where[:, :1].contiguous(), e.table[:, :1].contiguous()
    e.k.fill_(7.0), e.v.fill_(7.0), e.w.fill_(7.0)
    e.run()                                                    # 26 of the first one's tokens have no place
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_SEQ_LEN
    assert e.lens.tolist() == [90, 40] and e.kept[0, 0, :90].tolist() == list(range(90))
    page, at = c.place(0, torch.arange(64, device="cuda"))
    assert torch.equal(e.k[e.where[0, 0], 0], c.k_cache[page, 0, at])
