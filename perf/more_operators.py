"""What is measured of the way of a chunk of new tokens into a paged cache, of its attention, and of keeping the cache small.

Four kinds of case, one for each operator:

``rotate``  ``ffd_rotate_write_kv``: the rows of a projection are normalised per head, rotated by their positions and stored:
            queries as rows, keys and values in the cache's pages.
``chunk``   ``ffd_attend_chunk``: the new tokens of every sequence attend to the sequence's cache, themselves included (causal).
``weigh``   ``ffd_weigh_kv``: the attention weight that every cached token receives from some queries is summed up.
``evict``   ``ffd_evict_kv``: per KV head the tokens with the largest sums are kept and stored again in other pages.

Pages hold 64 tokens of every KV head, head_dim is 128, query head h uses KV head h // (q_heads // kv_heads).  A sequence has
`old` tokens in its cache and `new` ones behind them; both are spread evenly over their ranges and paired in a fixed way, so that
the work of a case does not depend on the seed, and dealt to the sequences by the seed.  Rows past a sequence's end and pages
that nobody owns hold values too, which belong to no result.
"""
import math

import torch

own = False

D = 128          # head_dim
PAGE = 64        # tokens in a page
EXTRA = 3        # rows behind the last sequence's
POISON = 1.0e4   # what rows past a sequence's end hold


def listed():
    return [
        # a serving step stores one new token for each of 16 running sequences: a latency
        dict(name="rotate-step-b16", kind="rotate", batch=16, q_heads=32, kv_heads=8, old_lo=0, old_hi=4095, new_lo=1, new_hi=1,
             norm=True, rotary=128, interleaved=False, given=False),
        # a prefill batch of ragged prompts, rows out of a fused projection
        dict(name="rotate-prompts-b8", kind="rotate", batch=8, q_heads=32, kv_heads=8, old_lo=0, old_hi=0, new_lo=1, new_hi=8191,
             norm=True, rotary=128, interleaved=False, given=False),
        # one token for each of 16 running sequences attends densely: the latency of a serving step
        dict(name="chunk-step-b16", kind="chunk", batch=16, q_heads=32, kv_heads=8, old_lo=255, old_hi=4095, new_lo=1, new_hi=1,
             out="bf16"),
        # five drafted tokens of eight users are checked at once, contexts of 4 K to 32 K behind a random page table
        dict(name="chunk-draft-b8", kind="chunk", batch=8, q_heads=32, kv_heads=8, old_lo=4096, old_hi=32763, new_lo=5, new_hi=5,
             out="bf16"),
        # a chunked prefill's scheduler: chunks of up to 512 tokens on contexts of up to 16 K
        dict(name="chunk-512-b4", kind="chunk", batch=4, q_heads=32, kv_heads=8, old_lo=0, old_hi=16000, new_lo=129, new_hi=512,
             out="bf16"),
        # a batch of ragged prompts of a model without grouped heads, results in 32 bits
        dict(name="chunk-prompts-b6-fp32", kind="chunk", batch=6, q_heads=8, kv_heads=8, old_lo=0, old_hi=0, new_lo=1,
             new_hi=2047, out="fp32"),
        # one whole prompt of 8 K
        dict(name="chunk-8k-b1", kind="chunk", batch=1, q_heads=32, kv_heads=8, old_lo=0, old_hi=0, new_lo=8192, new_hi=8192,
             out="bf16"),
        # a chunk of 2 K deep in a document of 64 K: the largest
        dict(name="chunk-2k-on-62k", kind="chunk", batch=1, q_heads=32, kv_heads=8, old_lo=63488, old_hi=63488, new_lo=2048,
             new_hi=2048, out="bf16"),
        # each decode step adds its token's weights for 16 sequences
        dict(name="weigh-step-b16", kind="weigh", batch=16, q_heads=32, kv_heads=8, old_lo=1024, old_hi=16383, new_lo=1, new_hi=1,
             add=True),
        # the last 64 tokens of a 32 K prompt say what is worth keeping
        dict(name="weigh-window-32k", kind="weigh", batch=1, q_heads=32, kv_heads=8, old_lo=32704, old_hi=32704, new_lo=64,
             new_hi=64, add=False),
        # that prompt is cut down to 4 K
        dict(name="evict-32k-to-4k", kind="evict", batch=1, q_heads=32, kv_heads=8, old_lo=32768, old_hi=32768, new_lo=0, new_hi=0,
             budget=4096, sink=64, local=1024, zeros=0.0),
        # a serving batch's ragged caches are cut down to 2 K, much of them never looked at
        dict(name="evict-ragged-b16", kind="evict", batch=16, q_heads=32, kv_heads=8, old_lo=512, old_hi=16384, new_lo=0, new_hi=0,
             budget=2048, sink=4, local=256, zeros=0.5),
    ]


def draw(rng):
    """A case of the ranges above; the products are capped so that none costs more than the largest listed one."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))

    kind = rng.choice(["rotate", "chunk", "chunk", "weigh", "evict"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
    batch = between(1, 64)
    case = dict(kind=kind, batch=batch, q_heads=kv_heads * group, kv_heads=kv_heads)
    tokens = max(64, (1 << 22) // (batch * kv_heads))                       # of a sequence: at most 2 GB of keys and values
    if kind == "rotate":
        new = between(1, min(8192, max(1, (1 << 21) // (batch * (kv_heads * group + 2 * kv_heads)))))
        old = rng.choice([0, between(1, min(16384, tokens))])
        case |= dict(norm=rng.choice([False, True]), rotary=rng.choice([0, 32, 64, 128, 128]), interleaved=rng.choice([False, True]),
                     given=rng.choice([False, True]))
    elif kind == "chunk":
        new = between(1, min(8192, tokens))
        most = (1 << 31) // (batch * case["q_heads"] * new)
        while most < 2 * new:                                               # a square of new tokens fits as well
            new = max(1, new // 2)
            most = (1 << 31) // (batch * case["q_heads"] * new)
        old = rng.choice([0, between(1, max(1, min(65536, tokens, most - new)))])
        case |= dict(out=rng.choice(["bf16", "bf16", "fp32"]))
    elif kind == "weigh":
        new = between(1, min(512, tokens))
        most = max(new + 1, (1 << 30) // (batch * case["q_heads"] * new))
        old = rng.choice([0, between(1, max(1, min(65536, tokens, most - new)))])
        case |= dict(add=rng.choice([False, True]))
    else:
        new, old = 0, between(1, min(65536, tokens))
        sink, local = rng.choice([0, 4, 64]), between(1, 1024) - 1
        case |= dict(budget=max(1, sink + local + between(1, max(1, old)) - 1), sink=sink, local=local, zeros=rng.choice([0.0, 0.5, 0.9]))
    low_new = new if rng.random() < 0.5 else min(new, rng.randint(0, new))
    low_old = old if rng.random() < 0.5 else rng.randint(0, old)
    return case | dict(old_lo=low_old, old_hi=old, new_lo=low_new, new_hi=new)


# ---- inputs -------------------------------------------------------------------------------------------------------


def spread(lo, hi, n):
    return [hi if n == 1 else lo + (hi - lo) * i // (n - 1) for i in range(n)]


def lengths(case):
    """(old, new) tokens of every sequence, before the seed deals them out: the range of one is run through in another order
    than the other's."""
    b = case["batch"]
    old, new = spread(case["old_lo"], case["old_hi"], b), spread(case["new_lo"], case["new_hi"], b)
    step = next(x for x in (7, 5, 3, 11, 13, 1) if math.gcd(x, b) == 1)
    return [(old[i], new[i * step % b]) for i in range(b)]


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def keys(gen, *shape):
    """Keys as caches hold them: a few channels are several times larger than the rest."""
    channel = 1.0 + 3.0 * (torch.rand(shape[-1], generator=gen, device="cuda") > 0.96)
    return (normal(gen, *shape) * channel).to(torch.bfloat16)


def values(gen, *shape):
    """Values as caches hold them: tokens differ in size."""
    return (normal(gen, *shape) * torch.exp(0.5 * normal(gen, *shape[:-1], 1))).to(torch.bfloat16)


def pool(gen, make, pages, kv_heads):
    """A pool of 16-bit pages, made a part at a time."""
    t = torch.empty(pages, kv_heads, PAGE, D, dtype=torch.bfloat16, device="cuda")
    part = max(1, (1 << 25) // (kv_heads * PAGE * D))
    for p in range(0, pages, part):
        n = min(part, pages - p)
        t[p:p + n] = make(gen, n, kv_heads, PAGE, D)
    return t


def tables(gen, lens, spare=5):
    """(block table, number of pages, longest block count): pages in random order, a few of them nobody's."""
    nb = (lens + PAGE - 1) // PAGE
    most, total = max(1, int(nb.max())), int(nb.sum()) + spare
    order = torch.randperm(total, generator=gen, device="cuda")
    at = torch.arange(most, device="cuda")[None, :] + (nb.cumsum(0) - nb)[:, None]
    table = torch.where(torch.arange(most, device="cuda")[None, :] < nb[:, None], order[at.clamp(max=total - 1)], 0)
    return table.to(torch.int32).contiguous(), total, most


def prepare(case, seed):
    torch.cuda.init()
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
    kind, batch, kv_heads, q_heads = case["kind"], case["batch"], case["kv_heads"], case["q_heads"]
    both = torch.tensor(lengths(case), device="cuda")[torch.randperm(batch, generator=gen, device="cuda")]
    first, count = both[:, 0].contiguous(), both[:, 1].contiguous()
    lens = first + count
    s = dict(case=case, lens=lens.to(torch.int32))
    s["table"], s["pages"], s["most"] = tables(gen, lens)
    one = case["new_lo"] == case["new_hi"] == 1
    s["rows"] = batch if one else int(count.sum()) + EXTRA
    s["first"] = None if one else first.to(torch.int32)
    s["start"] = None if one else (count.cumsum(0) - count).to(torch.int32)
    s["first_of"], s["count"] = first, count
    s["most_new"] = max(case["new_hi"], 1)
    if kind == "rotate":
        qkv = torch.zeros(s["rows"], (q_heads + 2 * kv_heads) * D, dtype=torch.bfloat16, device="cuda")
        cut = (q_heads * D, (q_heads + kv_heads) * D)
        s["q"] = qkv[:, :cut[0]].view(s["rows"], q_heads, D)
        s["k_new"] = qkv[:, cut[0]:cut[1]].view(s["rows"], kv_heads, D)
        s["v_new"] = qkv[:, cut[1]:].view(s["rows"], kv_heads, D)
        s["q"].copy_(normal(gen, s["rows"], q_heads, D) * torch.exp(0.5 * normal(gen, s["rows"], q_heads, 1)))
        s["k_new"].copy_(keys(gen, s["rows"], kv_heads, D))
        s["v_new"].copy_(values(gen, s["rows"], kv_heads, D))
        for x in ("q_norm", "k_norm"):
            s[x] = (1.0 + 0.2 * normal(gen, D)).to(torch.bfloat16) if case["norm"] else None
        places = max(1, int(lens.max())) + 100
        half = case["rotary"] // 2
        s["cos_sin"] = None
        if half:   # the cosines and the sines of every position, made once when a model is loaded
            angle = torch.arange(places, device="cuda", dtype=torch.float64)[:, None] / 10000.0 ** (
                torch.arange(half, device="cuda", dtype=torch.float64) / half)
            s["cos_sin"] = torch.stack([torch.cos(angle), torch.sin(angle)], 1).float().contiguous()
        s["positions"] = torch.randint(0, places, (s["rows"],), generator=gen, device="cuda", dtype=torch.int32) if case["given"] else None
        s["q_out"] = torch.full((s["rows"], q_heads, D), 0.25, dtype=torch.bfloat16, device="cuda")
        for x in "kv":   # what the pool held before: to be left alone where nothing is written
            s[x + "_cache"] = torch.full((s["pages"], kv_heads, PAGE, D), 0.25, dtype=torch.bfloat16, device="cuda")
    else:
        s["k_cache"] = pool(gen, keys, s["pages"], kv_heads)
        if kind != "weigh":
            s["v_cache"] = pool(gen, values, s["pages"], kv_heads)
        at = (lens - 1).clamp(min=0)
        page = s["table"].long().gather(1, (at // PAGE)[:, None]).squeeze(1)
        past = torch.arange(PAGE, device="cuda")[None, :] > (at % PAGE)[:, None]     # rows of the last page past the end
        seq, row = torch.nonzero(past & (lens > 0)[:, None], as_tuple=True)
        for x in "kv":
            if x + "_cache" in s:
                s[x + "_cache"][page[seq], :, row] = POISON
    if kind in ("chunk", "weigh"):
        s["q"] = normal(gen, s["rows"], q_heads, D).to(torch.bfloat16)
    if kind == "chunk":
        s["out"] = torch.full((s["rows"], q_heads, D), 0.25, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")
        s["lse"] = torch.full((s["rows"], q_heads), 0.25, dtype=torch.float32, device="cuda")
    if kind == "weigh":   # the log-sum-exp of every query's logits, as attention left it
        s["lse"] = torch.zeros(s["rows"], q_heads, dtype=torch.float32, device="cuda")
        inside, rows = rows_of(s)
        lse = torch.logsumexp(scores_of(s, torch.float32), -1)
        s["lse"][rows[inside]] = lse.view(batch, q_heads, -1).transpose(1, 2)[inside]
        s["weight"] = torch.rand(s["pages"], kv_heads, PAGE, generator=gen, device="cuda") * 0.01
    if kind == "evict":   # sums of weights: a few tokens have most of it; what was never looked at has none
        w = torch.exp(2.0 * normal(gen, s["pages"], kv_heads, PAGE) - 6.0)
        s["weight"] = torch.where(torch.rand(w.shape, generator=gen, device="cuda") < case["zeros"], 0.0, w)
        new_lens = lens.clamp(max=case["budget"])
        s["out_table"], s["out_pages"], s["out_most"] = tables(gen, new_lens)
        for x in "kv":
            s[x + "_out"] = torch.full((s["out_pages"], kv_heads, PAGE, D), 0.25, dtype=torch.bfloat16, device="cuda")
        s["weight_out"] = torch.full((s["out_pages"], kv_heads, PAGE), 0.25, device="cuda")
        s["out_lens"] = torch.zeros(batch, dtype=torch.int32, device="cuda")
        s["kept"] = torch.zeros(batch, kv_heads, case["budget"], dtype=torch.int32, device="cuda")
    if own:   # the workspace that a user's program allocates once for its geometry
        from paper_2609_00097_b200 import ffd
        s["cfg"] = ffd.Config(q_heads, kv_heads, out_dtype=0 if case.get("out", "bf16") == "bf16" else 1)
        s["workspace"] = ffd.new_workspace_chunk(s["cfg"], batch, s["rows"], s["most"])
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if own:
        return OWN[case["kind"]](s)
    return PLAIN[case["kind"]](s)


def own_rotate(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_rotate_write_kv(s["cfg"], s["q"], s["k_new"], s["v_new"], s["q_out"], s["k_cache"], s["v_cache"], s["table"], s["lens"],
                            cos_sin=s["cos_sin"], interleaved=s["case"]["interleaved"], q_norm=s["q_norm"], k_norm=s["k_norm"],
                            eps=1e-6, positions=s["positions"], row_start=s["start"], first_token=s["first"],
                            max_blocks_per_seq=s["most"], workspace=s["workspace"])
    return dict(q=s["q_out"], k=s["k_cache"], v=s["v_cache"])


def own_chunk(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_attend_chunk(s["cfg"], s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["out"], lse=s["lse"],
                         row_start=s["start"], first_token=s["first"], max_blocks_per_seq=s["most"], workspace=s["workspace"])
    return dict(out=s["out"], lse=s["lse"])


def own_weigh(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_weigh_kv(s["cfg"], s["q"], s["lse"], s["k_cache"], s["weight"], s["table"], s["lens"], add=s["case"]["add"],
                     row_start=s["start"], first_token=s["first"], max_blocks_per_seq=s["most"], workspace=s["workspace"])
    return dict(weight=s["weight"])


def own_evict(s):
    from paper_2609_00097_b200 import ffd
    c = s["case"]
    ffd.ffd_evict_kv(s["cfg"], s["k_cache"], s["v_cache"], s["weight"], s["table"], s["lens"], s["k_out"], s["v_out"],
                     s["weight_out"], s["out_table"], s["out_lens"], s["kept"], n_sink=c["sink"], n_local=c["local"],
                     max_blocks_per_seq=s["most"], max_out_blocks=s["out_most"], workspace=s["workspace"])
    return dict(k=s["k_out"], v=s["v_out"], weight=s["weight_out"], lens=s["out_lens"], kept=s["kept"])


OWN = dict(rotate=own_rotate, chunk=own_chunk, weigh=own_weigh, evict=own_evict)


def rows_of(s):
    """For every sequence and every i up to the longest chunk: whether it has a new token i, and that token's row."""
    i = torch.arange(s["most_new"], device="cuda")[None, :]
    inside = i < s["count"][:, None]
    start = s["count"].cumsum(0) - s["count"]
    return inside, torch.where(inside, start[:, None] + i, 0)


def gathered(s, x):
    """[batch, kv_heads, tokens, D] of the sequences' pages in 32 bits; zero past their ends."""
    t = s[x + "_cache"][s["table"].long()].float()
    t = t.permute(0, 2, 1, 3, 4).reshape(t.shape[0], t.shape[2], -1, D)
    inside = torch.arange(t.shape[2], device="cuda")[None, :] < s["lens"][:, None]
    return t.masked_fill_(~inside[:, None, :, None], 0.0)


def scores_of(s, dtype):
    """The logits [batch, kv_heads, heads of a group * most_new, tokens] of the new tokens; -infinity where a token is not seen."""
    inside, rows = rows_of(s)
    batch, kv_heads, most = s["lens"].numel(), s["case"]["kv_heads"], s["most_new"]
    q = s["q"][rows].to(dtype).permute(0, 2, 1, 3).reshape(batch, kv_heads, -1, D)
    score = q @ gathered(s, "k").to(dtype).transpose(-1, -2)
    score.mul_(1.0 / math.sqrt(D))
    token = torch.arange(score.shape[-1], device="cuda")
    hidden = token[None, None, :] > (s["first_of"][:, None] + torch.arange(most, device="cuda")[None, :])[:, :, None]
    hidden |= token[None, None, :] >= s["lens"][:, None, None]
    score.view(batch, kv_heads, -1, most, score.shape[-1]).masked_fill_(hidden[:, None, None], -math.inf)
    return score


def plain_rotate(s):
    case = s["case"]
    inside, rows = rows_of(s)
    seq, i = torch.nonzero(inside, as_tuple=True)
    row = rows[seq, i]
    token = s["first_of"][seq] + i
    place = token if s["positions"] is None else s["positions"].long()[row]

    def turned(x, weight):
        x = x[row].float()
        if weight is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
        if s["cos_sin"] is None:
            return x.to(torch.bfloat16)
        half = s["cos_sin"].shape[-1]
        cos, sin = s["cos_sin"][place, 0][:, None], s["cos_sin"][place, 1][:, None]
        if case["interleaved"]:
            a, b = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
            both = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = x[..., :half], x[..., half:2 * half]
            both = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([both, x[..., 2 * half:]], -1).to(torch.bfloat16)

    s["q_out"][row] = turned(s["q"], s["q_norm"])
    page, at = s["table"].long()[seq, token // PAGE], token % PAGE
    s["k_cache"][page, :, at] = turned(s["k_new"], s["k_norm"])
    s["v_cache"][page, :, at] = s["v_new"][row]
    return dict(q=s["q_out"], k=s["k_cache"], v=s["v_cache"])


def plain_chunk(s):
    inside, rows = rows_of(s)
    batch, q_heads = s["lens"].numel(), s["case"]["q_heads"]
    score = scores_of(s, torch.float32)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)      # (a sequence without any token)
    weight = score.sub_(top).exp_()
    total = weight.sum(-1, keepdim=True)
    out = (weight @ gathered(s, "v")) / total
    lse = torch.log(total) + top
    s["out"][rows[inside]] = out.view(batch, q_heads, -1, D).transpose(1, 2)[inside].to(s["out"].dtype)
    s["lse"][rows[inside]] = lse.view(batch, q_heads, -1).transpose(1, 2)[inside]
    return dict(out=s["out"], lse=s["lse"])


def plain_weigh(s):
    inside, rows = rows_of(s)
    batch, kv_heads = s["lens"].numel(), s["case"]["kv_heads"]
    lse = s["lse"][rows].masked_fill(~inside[..., None], math.inf).transpose(1, 2).reshape(batch, kv_heads, -1)
    got = scores_of(s, torch.float32).sub_(lse[..., None]).exp_().sum(2)                # [batch, kv_heads, tokens]
    token = torch.arange(got.shape[-1], device="cuda")
    seq, token = torch.nonzero(token[None, :] < s["lens"][:, None], as_tuple=True)
    page, at = s["table"].long()[seq, token // PAGE], token % PAGE
    got = got[seq, :, token]
    if s["case"]["add"]:
        got = torch.where((token < s["first_of"][seq])[:, None], s["weight"][page, :, at] + got, got)
    s["weight"][page, :, at] = got
    return dict(weight=s["weight"])


def plain_evict(s):
    c, lens = s["case"], s["lens"].long()
    batch, kv_heads, budget = lens.numel(), c["kv_heads"], c["budget"]
    page = s["table"].long()
    weight = s["weight"][page].permute(0, 2, 1, 3).reshape(batch, kv_heads, -1)
    token = torch.arange(weight.shape[-1], device="cuda")
    safe = (token[None, :] < c["sink"]) | (token[None, :] >= (lens - c["local"])[:, None])
    key = weight.masked_fill(safe[:, None], math.inf).masked_fill((token[None, :] >= lens[:, None])[:, None], -math.inf)
    n = min(budget, key.shape[-1])
    best = key.sort(dim=-1, descending=True, stable=True).indices[..., :n]                  # ties to the lowest index
    best = torch.where(torch.arange(n, device="cuda") < lens[:, None, None], best, key.shape[-1]).sort(-1).values
    s["kept"].fill_(-1)
    s["kept"][..., :n] = torch.where(best < key.shape[-1], best, -1)
    s["out_lens"].copy_(lens.clamp(max=budget))
    seq, head, slot = torch.nonzero(s["kept"] >= 0, as_tuple=True)
    token = s["kept"][seq, head, slot].long()
    to, here, source, at = s["out_table"].long()[seq, slot // PAGE], slot % PAGE, page[seq, token // PAGE], token % PAGE
    s["weight_out"][to, head, here] = s["weight"][source, head, at]
    s["k_out"][to, head, here] = s["k_cache"][source, head, at]
    s["v_out"][to, head, here] = s["v_cache"][source, head, at]
    return dict(k=s["k_out"], v=s["v_out"], weight=s["weight_out"], lens=s["out_lens"], kept=s["kept"])


PLAIN = dict(rotate=plain_rotate, chunk=plain_chunk, weigh=plain_weigh, evict=plain_evict)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    pairs, kv_heads, q_heads, batch = lengths(case), case["kv_heads"], case["q_heads"], case["batch"]
    new, tokens = sum(n for _, n in pairs), sum(f + n for f, n in pairs if n)
    seen = sum(n * f + n * (n + 1) // 2 for f, n in pairs)              # (query, key) pairs of a head
    if case["kind"] == "rotate":
        row = (q_heads + 2 * kv_heads) * D * 2
        places = min(new, max(f + n for f, n in pairs) + 100)
        return dict(bytes=2 * new * row + 4 * case["rotary"] * places + 12 * batch, flops=new * (q_heads + kv_heads) * D * 8)
    if case["kind"] == "chunk":
        heads = new * q_heads * (2 * D + (2 if case["out"] == "bf16" else 4) * D + 4)
        return dict(bytes=heads + tokens * kv_heads * 4 * D + 12 * batch, flops=4 * D * q_heads * seen)
    if case["kind"] == "weigh":
        heads = new * q_heads * (2 * D + 4)
        return dict(bytes=heads + tokens * kv_heads * (2 * D + (8 if case["add"] else 4)) + 12 * batch, flops=2 * D * q_heads * seen)
    length = [f + n for f, n in pairs]
    kept = sum(min(n, case["budget"]) for n in length)
    return dict(bytes=kv_heads * (4 * sum(length) + kept * (2 * 4 * D + 4 + 4)) + 12 * batch, flops=kv_heads * sum(length))


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    kind, group, kv_heads = case["kind"], case["q_heads"] // case["kv_heads"], case["kv_heads"]
    firsts, counts, table = s["first_of"].tolist(), s["count"].tolist(), s["table"].long()
    starts = [sum(counts[:b]) for b in range(len(counts))]

    def pages(pool, b, g, n):
        """Tokens 0 .. n - 1 of sequence b and KV head g."""
        return pool[table[b, :(n + PAGE - 1) // PAGE], g].flatten(0, 1)[:n].double()

    if kind == "rotate":
        outs = dict(q=s["q_out"].double(), k=s["k_cache"].double(), v=s["v_cache"].double())
        for b, (f, n) in enumerate(zip(firsts, counts)):
            rows, token = slice(starts[b], starts[b] + n), torch.arange(f, f + n, device="cuda")
            place = token if s["positions"] is None else s["positions"][rows].long()
            for x, source, weight in (("q", s["q"], s["q_norm"]), ("k", s["k_new"], s["k_norm"])):
                y = source[rows].double()
                if weight is not None:
                    y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / D + 1e-6) * weight.double()
                half = case["rotary"] // 2
                if half:
                    turn = torch.complex(s["cos_sin"][place, 0].double(), s["cos_sin"][place, 1].double())[:, None]
                    pair = y[..., :2 * half].unflatten(-1, (half, 2) if case["interleaved"] else (2, half))
                    pair = pair if case["interleaved"] else pair.transpose(-1, -2)
                    z = torch.view_as_real(torch.complex(pair[..., 0].contiguous(), pair[..., 1].contiguous()) * turn)
                    y = torch.cat([(z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2), y[..., 2 * half:]], -1)
                if x == "q":
                    outs["q"][rows] = y
                else:
                    outs["k"][table[b][token // PAGE], :, token % PAGE] = y
            outs["v"][table[b][token // PAGE], :, token % PAGE] = s["v_new"][rows].double()
        return outs
    if kind == "evict":   # copies, of the rows that the definition names
        outs = dict(k=s["k_out"].double(), v=s["v_out"].double(), weight=s["weight_out"].double(), lens=None, kept=None)
        for b, n in enumerate(firsts):
            middle = range(case["sink"], n - case["local"])
            for g in range(kv_heads):
                stays = list(range(n))
                if n > case["budget"]:
                    w = pages(s["weight"], b, g, n).tolist()
                    best = sorted(middle, key=lambda t: (-w[t], t))[:case["budget"] - case["sink"] - case["local"]]
                    stays = sorted(set(stays) - set(middle) | set(best))
                token, slot = torch.tensor(stays, device="cuda", dtype=torch.long), torch.arange(len(stays), device="cuda")
                source, to = table[b][token // PAGE], s["out_table"][b].long()[slot // PAGE]
                for x, pool in (("k", s["k_cache"]), ("v", s["v_cache"]), ("weight", s["weight"])):
                    outs[x][to, g, slot % PAGE] = pool[source, g, token % PAGE].double()
        return outs
    outs = dict(out=s["out"].double(), lse=s["lse"].double()) if kind == "chunk" else dict(weight=s["weight"].double())
    for b, (f, n) in enumerate(zip(firsts, counts)):
        for h in range(case["q_heads"]):
            g = h // group
            k = pages(s["k_cache"], b, g, f + n)
            if kind == "weigh" and h % group == 0:
                total = torch.zeros(f + n, dtype=torch.float64, device="cuda")
            for i in range(0, n, 2048):
                rows = slice(starts[b] + i, starts[b] + min(n, i + 2048))
                logit = s["q"][rows, h].double() @ k.T / math.sqrt(D)
                logit += torch.triu(torch.full_like(logit, -math.inf), f + i + 1)
                if kind == "chunk":
                    outs["lse"][rows, h] = torch.logsumexp(logit, -1)
                    outs["out"][rows, h] = torch.softmax(logit, -1) @ pages(s["v_cache"], b, g, f + n)
                else:
                    total += torch.exp(logit - s["lse"][rows, h].double()[:, None]).sum(0)
            if kind == "weigh" and h % group == group - 1 and f + n:
                token = torch.arange(f + n, device="cuda")
                at = (table[b][token // PAGE], g, token % PAGE)
                old = outs["weight"][at] * (token < f) if case["add"] else 0.0
                outs["weight"][at] = total + old
    return outs
