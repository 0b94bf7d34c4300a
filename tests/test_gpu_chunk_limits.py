"""What the functions on a chunk of new tokens do with values that are no numbers, bad pages and lengths, other streams, captured
graphs, pools beyond 32 bits, and one after the other as they are used."""
import math

import pytest
import torch

from paper_2609_00097_b200 import ffd
from tests.chunk_cases import D, PAGE, Chunk
from tests.test_gpu_rotate import PLACES, Rotate, cos_sin
from tests.test_gpu_weigh_evict import Evict, chosen, lengths, lse_of

pytestmark = pytest.mark.gpu


# ---- values that are no numbers --------------------------------------------------------------------------------------------


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("group", [1, 4, 5])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_tokens_that_a_row_does_not_see_have_no_influence(bad, group, out_dtype):
    """Token t's key and value are no numbers: rows before t get what they get without it, rows from t on something that is none."""
    for first, n, where in ((0, 300, (0, 1, 63, 64, 130, 255, 256, 299)), (1000, 90, (1000, 1031, 1032, 1089))):
        c = Chunk([(first, n), (20, 5)], 2 * group, 2, seed=n, out_dtype=out_dtype)
        clean, clean_lse = c.attend()
        for t in where:
            page, at = c.place(0, t)
            k, v = c.k_cache[page, 0, at].clone(), c.v_cache[page, 0, at].clone()
            c.v_cache[page, 0, at, 5] = bad
            c.k_cache[page, 0, at, 7] = math.nan if t % 2 else 0.0
            out, lse = c.attend()
            before = slice(0, c.starts[0] + t - first)
            assert torch.equal(out[before], clean[before]) and torch.equal(lse[before], clean_lse[before]), t
            after = slice(c.starts[0] + t - first, c.starts[0] + n)
            assert not out[after, :group, 5].isfinite().any(), t
            if t % 2 == 0:                                     # the key is a number: other channels are untouched by the value
                mask = torch.arange(D, device="cuda") != 5
                assert out[after, :group][..., mask].isfinite().all()
            else:
                assert out[after, :group].isnan().all() and lse[after, :group].isnan().all()
            assert torch.equal(out[:, group:], clean[:, group:])          # the other KV head
            rest = slice(c.starts[1], c.rows)
            assert torch.equal(out[rest], clean[rest])                    # the other sequence
            c.k_cache[page, 0, at], c.v_cache[page, 0, at] = k, v
        again, _ = c.attend()
        assert torch.equal(again, clean)
        assert ffd.ffd_read_device_status(c.workspace) == 0


def test_queries_and_logits_that_are_no_numbers():
    c = Chunk([(100, 40)], 4, 2, seed=1)
    clean, clean_lse = c.attend()
    r = c.starts[0]
    c.q[r + 3, 1, 0] = math.nan
    c.q[r + 8] = torch.finfo(torch.bfloat16).max        # products beyond binary32: infinities of either sign
    out, lse = c.attend()
    assert out[r + 3, 1].isnan().all() and lse[r + 3, 1].isnan()
    other = torch.ones(c.rows, 4, dtype=torch.bool, device="cuda")
    other[r + 3, 1] = other[r + 8] = False
    other[r + 8] = False
    assert torch.equal(out[other], clean[other]) and torch.equal(lse[other], clean_lse[other])


def test_large_and_small_logits():
    for scale in (0.0, 1e-3, 30.0):
        c = Chunk([(500, 100), (0, 33)], 8, 2, seed=2, q_scale=scale)
        c.check(*c.attend())


# ---- bad pages and lengths ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("page", [-1, 10 ** 6])
def test_bad_pages_are_left_out_and_reported(page):
    c = Chunk([(200, 150), (0, 40)], 4, 2, seed=3)
    c.table[0, 2] = page
    out, lse = c.attend()
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
    want, gone = c.logits, torch.arange(350, device="cuda") // PAGE == 2

    def without(b, h):
        score, size = want(b, h)
        return (score.masked_fill(gone, -math.inf), size) if b == 0 else (score, size)

    c.logits = without
    c.check(out, lse)
    weight = torch.full((c.pages, 2, PAGE), 7.0, device="cuda")
    ffd.ffd_weigh_kv(c.cfg, c.q, lse_of(c), c.k_cache, weight, c.table, c.lens, **c.row_args())
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
    assert (weight[c.where[0, 2]] == 7.0).all() and (weight[c.where[0, 1]] != 7.0).all()


def test_all_pages_bad():
    c = Chunk([(10, 30)], 4, 2, seed=4)
    c.table.fill_(-1)
    out, lse = c.attend()
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
    mine = c.owned()
    assert (out[mine] == 0).all() and (lse[mine] == -math.inf).all() and (out[~mine] == 7.0).all()


def test_bad_pages_of_writing_and_evicting():
    c = Chunk([(60, 200), (0, 9)], 4, 2, seed=5)
    r = Rotate(c)
    c.table[0, 2] = -7
    r.run()
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
    assert (r.k_cache[c.where[0, 2]] == 7.0).all() and (r.k_cache[c.where[0, 3], :, 0] != 7.0).any()
    assert (r.q_out[c.owned()] != 7.0).any(-1).all()                     # the queries are there all the same

    c = Chunk(lengths(300, 300), 2, 1, seed=6)
    e = Evict(c, 100, 3, 5)
    c.table[0, 1], e.table[1, 0] = 1 << 20, -1
    e.run()
    assert ffd.ffd_read_device_status(c.workspace) == ffd.DEV_BAD_PAGE
    weights = [e.weight[c.place(b, torch.arange(300, device="cuda"))[0], 0, torch.arange(300, device="cuda") % PAGE].tolist() for b in range(2)]
    weights[0][64:128] = [math.nan] * 64                                 # tokens that cannot be read are kept last
    for b in range(2):
        assert e.kept[b, 0].tolist() == chosen(weights[b], 100, 3, 5)
    assert (e.k[e.where[1, 0]] == 7.0).all() and (e.k[e.where[1, 1], :, 0] != 7.0).any()


def test_lengths_and_rows_out_of_range():
    c = Chunk([(100, 20), (64, 30), (5, 7)], 4, 2, seed=7)
    good, good_lse = c.attend()
    lens, first, start = c.lens.clone(), c.first.clone(), c.row_start.clone()
    weight = torch.zeros(c.pages, 2, PAGE, device="cuda")
    r = Rotate(c)
    lse = lse_of(c).nan_to_num(nan=0.0)
    for change in (lambda: c.lens.__setitem__(0, -5), lambda: c.first.__setitem__(0, -1), lambda: c.row_start.__setitem__(0, -3),
                   lambda: c.row_start.__setitem__(0, 2 ** 31 - 5), lambda: c.row_start.__setitem__(2, c.rows - 2),
                   lambda: c.lens.__setitem__(0, 2 ** 31 - 1), lambda: c.first.__setitem__(1, 2 ** 31 - 1)):
        change()
        out, l = c.attend()
        seen = ffd.ffd_read_device_status(c.workspace)
        assert seen in (0, ffd.DEV_BAD_SEQ_LEN, ffd.DEV_BAD_SEQ_LEN | ffd.DEV_BAD_PAGE)
        assert seen or c.first[1] == 2 ** 31 - 1                         # (a first token behind the end: no new tokens)
        ffd.ffd_weigh_kv(c.cfg, c.q, lse, c.k_cache, weight, c.table, c.lens, **c.row_args())
        r.run()
        ffd.ffd_read_device_status(c.workspace)
        c.lens.copy_(lens), c.first.copy_(first), c.row_start.copy_(start)
    out, l = c.attend()
    assert torch.equal(out, good) and torch.equal(l, good_lse)


# ---- streams, graphs, repetition -----------------------------------------------------------------------------------------------


def test_the_same_call_gives_the_same_bits():
    c = Chunk([(3000, 70), (0, 300), (17, 1)], 8, 2, seed=8)
    a = c.attend()
    for _ in range(5):
        b = c.attend()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_graphs_replay_other_lengths():
    pairs = [(700, 40), (64, 3), (0, 130)]
    c = Chunk(pairs, 8, 2, seed=9)
    lse_in = lse_of(c).nan_to_num(nan=0.0)
    weight, out, lse = torch.zeros(c.pages, 2, PAGE, device="cuda"), torch.full((c.rows, 8, D), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((c.rows, 8), 7.0, device="cuda")
    r, e = Rotate(c), Evict(c, 90, 4, 20, weight=c.randn(c.pages, 2, PAGE))
    side = torch.cuda.Stream()

    def run():
        c.attend(out, lse)
        ffd.ffd_weigh_kv(c.cfg, c.q, lse_in, c.k_cache, weight, c.table, c.lens, **c.row_args())
        e.run()
        r.run()

    with torch.cuda.stream(side):
        run()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for pairs in ([(700, 40), (64, 3), (0, 130)], [(300, 11), (0, 2), (60, 70)], [(0, 0), (0, 1), (0, 0)]):
        c.pairs, c.length = pairs, [f + n for f, n in pairs]
        c.lens.copy_(torch.tensor(c.length, device="cuda"))
        c.first.copy_(torch.tensor([f for f, _ in pairs], device="cuda"))
        out.fill_(7.0), lse.fill_(7.0), e.k.fill_(7.0), e.v.fill_(7.0), e.w.fill_(7.0), r.q_out.fill_(7.0), r.k_cache.fill_(7.0), r.v_cache.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        c.check(out, lse)
        e.check()
        r.check()


def test_calls_on_several_streams_at_once():
    jobs = []
    for i in range(4):
        c = Chunk([(2000 + 100 * i, 30 + i), (0, 200)], 8, 2, seed=20 + i)
        jobs.append((c, torch.cuda.Stream(), c.attend()))
    torch.cuda.synchronize()
    got = []
    for _ in range(10):
        for c, stream, _ in jobs:
            with torch.cuda.stream(stream):
                got.append(c.attend())
    torch.cuda.synchronize()
    for x, (out, lse) in enumerate(got):
        want = jobs[x % 4][2]
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    c = jobs[0][0]                                        # a stream that is named is taken, whatever the current one
    out = torch.full_like(jobs[0][2][0], 7.0)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    ffd.ffd_attend_chunk(c.cfg, c.q, c.k_cache, c.v_cache, c.table, c.lens, out, **c.row_args(), stream=stream)
    stream.synchronize()
    assert torch.equal(out, jobs[0][2][0])


def test_no_rows_at_all():
    c = Chunk([(30, 0), (5, 0)], 4, 2, seed=10, gap=0)
    assert c.rows == 0
    c.attend()
    Rotate(c, fused=False).run()
    with pytest.raises(ffd.FfdError):
        ffd.ffd_weigh_kv(c.cfg, c.q, torch.zeros(0, 4, device="cuda"), c.k_cache, torch.zeros(c.pages, 2, PAGE, device="cuda"), c.table, c.lens,
                         **c.row_args())
    assert ffd.ffd_read_device_status(c.workspace) == 0


def test_a_large_batch_of_short_sequences():
    c = Chunk([(i % 5, 1 + i % 3) for i in range(9000)], 2, 1, seed=11, gap=0, room=0)
    out, lse = c.attend()
    # every sequence fits a page: all of them at once
    k, v = (x[c.where[:, 0], 0].double() for x in (c.k_cache, c.v_cache))
    first = torch.tensor([f for f, _ in c.pairs], device="cuda")
    for i in range(3):
        has = torch.tensor([n > i for _, n in c.pairs], device="cuda")
        rows = torch.tensor(c.starts, device="cuda")[has] + i
        for h in range(2):
            hidden = torch.arange(PAGE, device="cuda")[None, :] > (first[has] + i)[:, None]
            score = torch.einsum("bd,btd->bt", c.q[rows, h].double(), k[has]).masked_fill(hidden, -math.inf) * c.sm
            want = torch.einsum("bt,btd->bd", torch.softmax(score, -1), v[has].nan_to_num(nan=0.0))
            # a rounding of the result and of the weights, both 2^-8, of values that are seldom beyond 5
            assert (out[rows, h].double() - want).abs().max() < 2 * 2.0 ** -8 * 6
            assert (lse[rows, h].double() - torch.logsumexp(score, -1)).abs().max() < 1e-4
    assert ffd.ffd_read_device_status(c.workspace) == 0


def test_pools_beyond_32_bits():
    """Pages whose elements lie 2^32 and more behind the pool's beginning."""
    c = Chunk([(90, 60), (0, 5)], 2, 1, seed=12)
    pages = (1 << 32) // (PAGE * D) + 400
    far = torch.arange(pages - c.batch * c.blocks, pages, device="cuda").view(c.batch, c.blocks)
    old = c.where
    k, v = (torch.empty(pages, 1, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[far], v[far] = c.k_cache[old], c.v_cache[old]
    c.k_cache, c.v_cache, c.where, c.table, c.pages = k, v, far, far.to(torch.int32).contiguous(), pages
    out, lse = c.attend()
    c.check(out, lse)
    weight = torch.zeros(pages, 1, PAGE, device="cuda")
    ffd.ffd_weigh_kv(c.cfg, c.q, lse_of(c), k, weight, c.table, c.lens, **c.row_args())
    assert weight[far[0, 0]].min() > 0 and weight[: pages - c.batch * c.blocks].max() == 0
    kept, lens = torch.zeros(2, 1, 64, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    to = torch.tensor([[pages - 300], [pages - 200]], dtype=torch.int32, device="cuda")
    ffd.ffd_evict_kv(c.cfg, k, v, weight, c.table, c.lens, k, v, weight, to, lens, kept, n_local=10, max_blocks_per_seq=c.blocks, max_out_blocks=1,
                     workspace=c.workspace)
    page, at = c.place(0, kept[0, 0].long())
    assert torch.equal(k[pages - 300, 0], k[page, 0, at]) and torch.equal(v[pages - 300, 0], v[page, 0, at]) and lens.tolist() == [64, 5]
    fresh = torch.randn(c.rows, 2, D, device="cuda").to(torch.bfloat16)
    ffd.ffd_rotate_write_kv(c.cfg, fresh, fresh[:, :1].contiguous(), fresh[:, 1:].contiguous(), torch.empty_like(fresh), k, v, c.table, c.lens, **c.row_args())
    page, at = c.place(0, torch.arange(90, 150, device="cuda"))
    assert torch.equal(v[page, 0, at], fresh[c.starts[0]:c.starts[0] + 60, 1])
    assert ffd.ffd_read_device_status(c.workspace) == 0


# ---- one after the other ---------------------------------------------------------------------------------------------------------


def test_a_prompt_in_chunks_its_eviction_and_the_decode_behind_it():
    """Two prompts come in chunks; their last 32 tokens say what is kept; the cut caches serve the sparse and the dense decode; a
    new token goes behind them at its own position.  The whole against the same steps in 64 bits."""
    hq, hkv, total, budget, sink, local = 8, 2, (700, 333), 256, 8, 64
    gen = torch.Generator(device="cuda").manual_seed(13)
    q, k, v = (torch.randn(2, 701, h, D, generator=gen, device="cuda").to(torch.bfloat16) for h in (hq, hkv, hkv))
    norm = (1 + 0.1 * torch.randn(D, generator=gen, device="cuda")).to(torch.bfloat16)
    table, blocks = torch.randperm(24, generator=gen, device="cuda")[:22].view(2, 11).to(torch.int32).contiguous(), 11
    cfg = ffd.Config(hq, hkv, out_dtype=0)
    turn = cos_sin(D)
    k_cache, v_cache = (torch.zeros(24, hkv, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ws = ffd.new_workspace_chunk(cfg, 2, 400, blocks)
    done, q_all, lse_all = [0, 0], torch.zeros_like(q), torch.zeros(2, 701, hq, device="cuda")
    outs = torch.zeros(2, 701, hq, D, dtype=torch.bfloat16, device="cuda")
    for step in ((300, 100), (250, 233), (150, 0)):
        lens = torch.tensor([done[b] + step[b] for b in range(2)], dtype=torch.int32, device="cuda")
        first, start = torch.tensor(done, dtype=torch.int32, device="cuda"), torch.tensor([0, step[0]], dtype=torch.int32, device="cuda")
        rows = [torch.cat([x[b, done[b]:done[b] + step[b]] for b in range(2)]).contiguous() for x in (q, k, v)]
        q_rot, out, lse = torch.empty_like(rows[0]), torch.empty_like(rows[0]), torch.empty(sum(step), hq, device="cuda")
        args = dict(row_start=start, first_token=first, max_blocks_per_seq=blocks, workspace=ws)
        ffd.ffd_rotate_write_kv(cfg, *rows, q_rot, k_cache, v_cache, table, lens, cos_sin=turn, q_norm=norm, k_norm=norm, **args)
        ffd.ffd_attend_chunk(cfg, q_rot, k_cache, v_cache, table, lens, out, lse=lse, **args)
        for b in range(2):
            here = slice(sum(step[:b]), sum(step[:b + 1]))
            there = slice(done[b], done[b] + step[b])
            q_all[b, there], lse_all[b, there], outs[b, there] = q_rot[here], lse[here], out[here]
            done[b] += step[b]
    # the last 32 tokens' weights, and the eviction
    lens = torch.tensor(total, dtype=torch.int32, device="cuda")
    first, start = lens - 32, torch.tensor([0, 32], dtype=torch.int32, device="cuda")
    q_seen, lse_seen = (torch.cat([x[b, total[b] - 32:total[b]] for b in range(2)]).contiguous() for x in (q_all, lse_all))
    weight = torch.empty(24, hkv, PAGE, device="cuda")
    ffd.ffd_weigh_kv(cfg, q_seen, lse_seen, k_cache, weight, table, lens, row_start=start, first_token=first, max_blocks_per_seq=blocks, workspace=ws)
    out_blocks = budget // PAGE + 1
    small_k, small_v = (torch.zeros(2 * out_blocks, hkv, PAGE, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small_w = torch.zeros(2 * out_blocks, hkv, PAGE, device="cuda")
    kept, small_lens = torch.zeros(2, hkv, budget, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    ffd.ffd_evict_kv(cfg, k_cache, v_cache, weight, table, lens, small_k, small_v, small_w, None, small_lens, kept, n_sink=sink, n_local=local,
                     max_blocks_per_seq=blocks, max_out_blocks=out_blocks, workspace=ws)
    assert small_lens.tolist() == [budget, budget]
    # a new token behind each, at the position that it has in its sequence
    new = [torch.stack([x[b, total[b]] for b in range(2)]).contiguous() for x in (q, k, v)]
    q_new, places = torch.empty_like(new[0]), lens.clone()
    now = small_lens + 1
    ffd.ffd_rotate_write_kv(cfg, *new, q_new, small_k, small_v, None, now, cos_sin=turn, q_norm=norm, k_norm=norm, positions=places,
                            max_blocks_per_seq=out_blocks, workspace=ws)
    step_out, step_lse = torch.empty_like(q_new), torch.empty(2, hq, device="cuda")
    ffd.ffd_attend_chunk(cfg, q_new, small_k, small_v, None, now, step_out, lse=step_lse, max_blocks_per_seq=out_blocks, workspace=ws)
    ffd.ffd_weigh_kv(cfg, q_new, step_lse, small_k, small_w, None, now, add=True, max_blocks_per_seq=out_blocks, workspace=ws)
    # the library's own decodes read the same cache
    full = ffd.Config(hq, hkv, out_dtype=1)
    ws2 = ffd.new_workspace(full, 2, out_blocks)
    dense, dense_lse, sparse = torch.empty(2, hq, D, device="cuda"), torch.empty(2, hq, device="cuda"), torch.empty(2, hq, D, device="cuda")
    ffd.ffd_decode_dense(full, q_new, small_k, small_v, None, now, dense, lse=dense_lse, max_blocks_per_seq=out_blocks, workspace=ws2)
    codes, scales = torch.zeros(2 * out_blocks, hkv, 2048, dtype=torch.uint8, device="cuda"), torch.zeros(2 * out_blocks, hkv, D, dtype=torch.float16, device="cuda")
    ffd.ffd_quantize_keys(full, small_k, codes, scales, None, now, max_blocks_per_seq=out_blocks)
    ffd.ffd_decode(full, q_new, small_k, small_v, codes, scales, None, now, math.inf, sparse, max_blocks_per_seq=out_blocks, workspace=ws2)
    assert ffd.ffd_read_device_status(ws) == 0 and ffd.ffd_read_device_status(ws2) == 0

    # ---- in 64 bits, from the rotated rows as they were stored
    def turned(x, place):
        y = x.double()
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * norm.double()
        a, b, c, s = y[..., :64], y[..., 64:], turn[place, 0].double()[:, None], turn[place, 1].double()[:, None]
        return torch.cat([a * c - b * s, b * c + a * s], -1)

    for b in range(2):
        place = torch.arange(total[b] + 1, device="cuda")
        q_want, k_want = turned(q[b, :total[b] + 1], place), turned(k[b, :total[b] + 1], place)
        token = place[:-1]
        k_here, v_here = (x[table[b].long()[token // PAGE], :, token % PAGE] for x in (k_cache, v_cache))
        assert ((k_here.double() - k_want[:-1]).abs() <= 2.0 ** -8 * k_want[:-1].abs() + 1e-5).all()
        assert torch.equal(v_here, v[b, :total[b]])
        for h in range(hq):
            g = h // 4
            score = q_all[b, :total[b], h].double() @ k_here[:, g].double().T / math.sqrt(D)
            score = score + torch.triu(torch.full_like(score, -math.inf), 1)
            p = torch.softmax(score, -1)
            want, mass = p @ v_here[:, g].double(), p @ v_here[:, g].double().abs()
            # roundings to bf16 of the result and of the weights
            assert ((outs[b, :total[b], h].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * mass).all()
            assert (lse_all[b, :total[b], h].double() - torch.logsumexp(score, -1)).abs().max() < 1e-4
        for g in range(hkv):
            got = weight[table[b].long()[token // PAGE], g, token % PAGE]
            w = torch.zeros(total[b], dtype=torch.float64, device="cuda")
            for h in range(4 * g, 4 * g + 4):
                score = q_all[b, total[b] - 32:total[b], h].double() @ k_here[:, g].double().T / math.sqrt(D)
                score = score + torch.triu(torch.full_like(score, -math.inf), total[b] - 31)
                w += torch.exp(score - lse_all[b, total[b] - 32:total[b], h].double()[:, None]).sum(0)
            assert (got.double() - w).abs().max() < 1e-4 * w.max()
            assert kept[b, g].tolist() == chosen(got.tolist(), budget, sink, local)
            # the new token over what is kept
            stays = kept[b, g].long()
            page = b * out_blocks + torch.arange(budget + 1, device="cuda") // PAGE
            k_new, v_new = (x[page, g, torch.arange(budget + 1, device="cuda") % PAGE].double() for x in (small_k, small_v))
            assert torch.equal(k_new[:budget], k_here[stays, g].double()) and torch.equal(v_new[:budget], v_here[stays, g].double())
            assert ((k_new[budget] - k_want[total[b], g]).abs() <= 2.0 ** -8 * k_want[total[b], g].abs() + 1e-5).all()
            w_now = torch.cat([got[stays].double(), torch.zeros(1, dtype=torch.float64, device="cuda")])
            for h in range(4 * g, 4 * g + 4):
                assert ((q_new[b, h].double() - q_want[total[b], h]).abs() <= 2.0 ** -8 * q_want[total[b], h].abs() + 1e-5).all()
                score = k_new @ q_new[b, h].double() / math.sqrt(D)
                p = torch.softmax(score, -1)
                want, mass = p @ v_new, p @ v_new.abs()
                assert ((step_out[b, h].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -12) * mass).all()
                assert ((dense[b, h].double() - want).abs() <= 2.0 ** -12 * mass).all()
                assert ((sparse[b, h].double() - want).abs() <= 2.0 ** -12 * mass).all()
                assert abs(float(step_lse[b, h] - dense_lse[b, h])) < 1e-4
                w_now += torch.exp(score - step_lse[b, h].double())
            got_now = small_w[page, g, torch.arange(budget + 1, device="cuda") % PAGE].double()
            assert (got_now - w_now).abs().max() < 1e-4 * w_now.max()
