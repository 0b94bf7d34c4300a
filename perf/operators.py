"""What is measured of the byte cache (keys and values in 8 bits, written and read back), of the decode attention that
reads it, and of the decode attention of a batch that shares a prefix.

Four kinds of case, one for each operator:

``write``   ``ffd_write_kv_byte``: new keys and values are quantised into the pages of a byte cache, one scale for each
            token and KV head: int8 (scale = absmax / 127) or e4m3 (scale = absmax / 448).
``read``    ``ffd_read_kv_byte``: the byte cache is turned back into 16-bit pages.
``decode``  ``ffd_decode_byte``: one query token per sequence attends to its whole byte cache.
``prefix``  ``ffd_decode_prefix`` / ``ffd_decode_prefix_byte``: one query token per sequence attends to a prefix that all
            sequences share (16-bit pages, stored once) and then to the sequence's own tokens (16-bit or byte pages).

Pages hold 64 tokens of every KV head, head_dim is 128, query head h uses KV head h // (q_heads // kv_heads).  Lengths are
spread evenly over [len_lo, len_hi] and dealt to the sequences by the seed, so that the work of a case does not depend on
the seed.  Rows past a sequence's end and pages that nobody owns hold values too, which belong to no result.
"""
import math

import torch

own = False

D = 128          # head_dim
PAGE = 64        # tokens in a page
POISON = 1.0e4   # what 16-bit rows past the prefix's end hold
LIMIT = {"int8": 127.0, "e4m3": 448.0}
CODE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}


def listed():
    return [
        # a serving step writes one new token for each of 16 running sequences: a latency
        dict(name="write-step-b16-int8", kind="write", fmt="int8", batch=16, q_heads=32, kv_heads=8, len_lo=1, len_hi=4096,
             new="one", fused=False),
        # a prefill batch of ragged prompts, the rows taken out of a fused qkv projection
        dict(name="write-prompts-b8-e4m3", kind="write", fmt="e4m3", batch=8, q_heads=32, kv_heads=8, len_lo=1, len_hi=8191,
             new="all", fused=True),
        # one 32 K context brought back into 16-bit pages, e.g. to share it as a prefix or to build its thumbnails
        dict(name="read-32k-int8", kind="read", fmt="int8", batch=1, q_heads=32, kv_heads=8, len_lo=32768, len_hi=32768,
             paged=False),
        # ragged sequences brought back through page tables, e.g. when a batch moves to another worker
        dict(name="read-ragged-b16-e4m3", kind="read", fmt="e4m3", batch=16, q_heads=32, kv_heads=8, len_lo=1, len_hi=16383,
             paged=True),
        # the smallest decode of the repository's workloads: one 4 K sequence, 8 query and 2 KV heads
        dict(name="decode-4k-b1-int8", kind="decode", fmt="int8", batch=1, q_heads=8, kv_heads=2, len_lo=4096, len_hi=4096,
             paged=False, out="bf16"),
        # a single user's 32 K context
        dict(name="decode-32k-b1-e4m3", kind="decode", fmt="e4m3", batch=1, q_heads=32, kv_heads=8, len_lo=32768,
             len_hi=32768, paged=False, out="bf16"),
        # the repository's benchmark geometry: four sequences of 128 K
        dict(name="decode-128k-b4-int8", kind="decode", fmt="int8", batch=4, q_heads=32, kv_heads=8, len_lo=131072,
             len_hi=131072, paged=False, out="bf16"),
        # a serving batch of ragged lengths behind a random page table
        dict(name="decode-ragged-b16-e4m3", kind="decode", fmt="e4m3", batch=16, q_heads=32, kv_heads=8, len_lo=16384,
             len_hi=65536, paged=True, out="bf16"),
        # a few chats that have just started on a system prompt of odd length: a latency
        dict(name="prefix-4k-b4-bf16", kind="prefix", fmt="bf16", batch=4, q_heads=32, kv_heads=8, prefix=4133, len_lo=1,
             len_hi=61, out="bf16"),
        # sampling 16 answers to one 32 K document, each answer in the byte cache
        dict(name="prefix-32k-b16-int8", kind="prefix", fmt="int8", batch=16, q_heads=32, kv_heads=8, prefix=32768, len_lo=1,
             len_hi=1021, out="bf16"),
        # 64 users of one 128 K corpus: the largest
        dict(name="prefix-128k-b64-e4m3", kind="prefix", fmt="e4m3", batch=64, q_heads=32, kv_heads=8, prefix=131072,
             len_lo=1, len_hi=509, out="bf16"),
        # a wide batch, 8 query heads per KV head, on a long few-shot prompt: bound by arithmetic
        dict(name="prefix-8k-b128-bf16", kind="prefix", fmt="bf16", batch=128, q_heads=64, kv_heads=8, prefix=8203, len_lo=1,
             len_hi=255, out="bf16"),
    ]


def draw(rng):
    """A case of the ranges above; the token counts are capped so that none costs more than the largest listed one."""
    def between(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["write", "read", "decode", "prefix"])
    kv_heads = rng.choice([1, 2, 3, 4, 8])
    group = rng.choice([1, 2, 3, 4, 6, 8])
    case = dict(kind=kind, q_heads=kv_heads * group, kv_heads=kv_heads)
    if kind == "prefix":
        case["batch"] = between(1, 128)
        most = min(131072, (1 << 28) // (case["batch"] * case["q_heads"]))
        case["prefix"] = between(1, most)
        hi = between(1, min(4096, max(1, (1 << 18) // (case["batch"] * kv_heads))))
        case |= dict(fmt=rng.choice(["bf16", "int8", "e4m3"]), len_lo=rng.randint(0, hi), len_hi=hi, out="bf16")
    else:
        case["batch"] = between(1, 64)
        most = (1 << 22 if kind == "decode" else 1 << 20) // (case["batch"] * kv_heads)
        hi = between(1, min(131072, max(2, most)))
        case |= dict(fmt=rng.choice(["int8", "e4m3"]), len_lo=rng.randint(0, hi), len_hi=hi)
        if kind == "write":
            case |= dict(new=rng.choice(["one", "all"]), fused=rng.choice([False, True]))
        else:
            case |= dict(paged=rng.choice([False, True]))
        if kind == "decode":
            case["out"] = "bf16"
    return case


# ---- inputs -------------------------------------------------------------------------------------------------------


def lengths(case):
    """The sequences' lengths, before the seed deals them out."""
    b, lo, hi = case["batch"], case["len_lo"], case["len_hi"]
    return [lo + (hi - lo) * i // max(1, b - 1) for i in range(b)] if b > 1 else [hi]


def quantise(x, fmt):
    """(codes, scales) of the last axis of x, each step one operation in binary32; a row below 2^-100 is all zero."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    tiny = top < 2.0 ** -100
    limit, safe = torch.full_like(top, LIMIT[fmt]), torch.where(tiny, torch.ones_like(top), top)   # tensors: true divisions
    scale = torch.where(tiny, torch.zeros_like(top), top / limit)
    y = torch.where(tiny, torch.zeros_like(x), x * (limit / safe))
    code = y.round().clamp(-127, 127).to(torch.int8) if fmt == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn)
    return code, scale.squeeze(-1)


def pages_of(gen, lens, paged):
    """(block table or None, number of pages, longest block count) of these lengths."""
    dev = "cuda"
    batch, most = lens.numel(), max(1, (int(lens.max()) + PAGE - 1) // PAGE)
    if not paged:
        return None, batch * most, most
    nb = (lens + PAGE - 1) // PAGE
    total = int(nb.sum()) + 5
    order = torch.randperm(total, generator=gen, device=dev)
    at = torch.arange(most, device=dev)[None, :] + (nb.cumsum(0) - nb)[:, None]
    table = torch.where(torch.arange(most, device=dev)[None, :] < nb[:, None], order[at.clamp(max=total - 1)], 0)
    return table.to(torch.int32).contiguous(), total, most


def normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def keys(gen, *shape):
    """Keys as caches hold them: a few channels are several times larger than the rest."""
    channel = 1.0 + 3.0 * (torch.rand(shape[-1], generator=gen, device="cuda") > 0.96)
    return (normal(gen, *shape) * channel).to(torch.bfloat16)


def values(gen, *shape):
    """Values as caches hold them: tokens differ in size."""
    return (normal(gen, *shape) * torch.exp(0.5 * normal(gen, *shape[:-1], 1))).to(torch.bfloat16)


def byte_pages(gen, make, fmt, pages, kv_heads):
    """(codes, scales) of a pool of pages, quantised a part at a time."""
    code = torch.empty(pages, kv_heads, PAGE, D, dtype=CODE[fmt], device="cuda")
    scale = torch.empty(pages, kv_heads, PAGE, dtype=torch.float32, device="cuda")
    part = max(1, (1 << 25) // (kv_heads * PAGE * D))
    for p in range(0, pages, part):
        n = min(part, pages - p)
        code[p:p + n], scale[p:p + n] = quantise(make(gen, n, kv_heads, PAGE, D), fmt)
    return code, scale


def prepare(case, seed):
    torch.cuda.init()
    gen = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 17)
    kind, fmt, batch, kv_heads, q_heads = case["kind"], case["fmt"], case["batch"], case["kv_heads"], case["q_heads"]
    lens = torch.tensor(lengths(case), device="cuda")[torch.randperm(batch, generator=gen, device="cuda")]
    s = dict(case=case, lens=lens.to(torch.int32))
    s["table"], s["pages"], s["most"] = pages_of(gen, lens, case.get("paged", True))
    if kind == "write":
        first = torch.zeros_like(lens) if case["new"] == "all" else (lens - 1).clamp(min=0)
        count = lens - first
        s["rows"] = batch if case["new"] == "one" else max(1, int(count.sum()))
        width = (q_heads + 2 * kv_heads) * D if case["fused"] else kv_heads * D
        at_k, at_v = (q_heads * D, (q_heads + kv_heads) * D) if case["fused"] else (0, 0)
        qkv = torch.zeros(s["rows"], width, dtype=torch.bfloat16, device="cuda")
        s["k_new"] = qkv[:, at_k:at_k + kv_heads * D].view(s["rows"], kv_heads, D)
        other = qkv if case["fused"] else torch.zeros_like(qkv)
        s["v_new"] = other[:, at_v:at_v + kv_heads * D].view(s["rows"], kv_heads, D)
        s["k_new"].copy_(keys(gen, s["rows"], kv_heads, D))
        s["v_new"].copy_(values(gen, s["rows"], kv_heads, D))
        one = case["new"] == "one"
        s["first"] = None if one else first.to(torch.int32)
        s["start"] = None if one else (count.cumsum(0) - count).to(torch.int32)
        for x in "kv":   # what the pool held before: recognisable, and to be left alone where nothing is written
            s[x + "_code"] = torch.full((s["pages"], kv_heads, PAGE, D), 3.0, device="cuda").to(CODE[fmt])
            s[x + "_scale"] = torch.full((s["pages"], kv_heads, PAGE), 0.5, device="cuda")
    elif fmt != "bf16":
        s["k_code"], s["k_scale"] = byte_pages(gen, keys, fmt, s["pages"], kv_heads)
        s["v_code"], s["v_scale"] = byte_pages(gen, values, fmt, s["pages"], kv_heads)
    if kind == "read":   # what the 16-bit pages held before: to be left alone past the sequences' ends
        for x in "kv":
            s[x + "_cache"] = torch.full((batch * s["most"], kv_heads, PAGE, D), 0.25, dtype=torch.bfloat16, device="cuda")
    if kind in ("decode", "prefix"):
        s["q"] = normal(gen, batch, q_heads, D).to(torch.bfloat16)
        s["out"] = torch.zeros(batch, q_heads, D, dtype=torch.bfloat16 if case["out"] == "bf16" else torch.float32, device="cuda")
        s["lse"] = torch.zeros(batch, q_heads, dtype=torch.float32, device="cuda")
    if kind == "prefix":
        s["prefix_len"] = torch.tensor([case["prefix"]], dtype=torch.int32, device="cuda")
        s["prefix_most"] = (case["prefix"] + PAGE - 1) // PAGE
        # 16-bit sequences live in the same pool as the prefix, behind the prefix's pages
        pool = s["prefix_most"] + 3 + (s["pages"] if fmt == "bf16" else 0)
        order = torch.randperm(pool, generator=gen, device="cuda").to(torch.int32)
        s["prefix_table"] = order[:s["prefix_most"]].contiguous()
        if fmt == "bf16":
            s["table"] = order[s["prefix_most"] + s["table"].long()].contiguous()
        s["prefix_pages"] = pool
        s["k_cache"] = torch.empty(pool, kv_heads, PAGE, D, dtype=torch.bfloat16, device="cuda")
        s["v_cache"] = torch.empty_like(s["k_cache"])
        part = max(1, (1 << 25) // (kv_heads * PAGE * D))
        for p in range(0, pool, part):
            n = min(part, pool - p)
            s["k_cache"][p:p + n] = keys(gen, n, kv_heads, PAGE, D)
            s["v_cache"][p:p + n] = values(gen, n, kv_heads, PAGE, D)
        if case["prefix"] % PAGE:
            s["k_cache"][s["prefix_table"][-1].long(), :, case["prefix"] % PAGE:] = POISON
            s["v_cache"][s["prefix_table"][-1].long(), :, case["prefix"] % PAGE:] = POISON
    if own:   # the workspace that a user's program allocates once for its geometry
        from paper_2609_00097_b200 import ffd
        s["cfg"] = ffd.Config(q_heads, kv_heads, out_dtype=0 if case.get("out", "bf16") == "bf16" else 1)
        s["workspace"] = ffd.new_workspace_prefix(s["cfg"], batch, s["most"], s.get("prefix_most", 0))
    return s


# ---- one pass -----------------------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if own:
        return OWN[case["kind"]](s)
    return PLAIN[case["kind"]](s)


def own_write(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_write_kv_byte(s["cfg"], s["k_new"], s["v_new"], s["k_code"], s["v_code"], s["k_scale"], s["v_scale"], s["table"],
                          s["lens"], row_start=s["start"], first_token=s["first"], max_blocks_per_seq=s["most"],
                          workspace=s["workspace"])
    return dict(k=s["k_code"], v=s["v_code"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def own_read(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_read_kv_byte(s["cfg"], s["k_code"], s["v_code"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["k_cache"],
                         s["v_cache"], max_blocks_per_seq=s["most"], workspace=s["workspace"])
    return dict(k=s["k_cache"], v=s["v_cache"])


def own_decode(s):
    from paper_2609_00097_b200 import ffd
    ffd.ffd_decode_byte(s["cfg"], s["q"], s["k_code"], s["v_code"], s["k_scale"], s["v_scale"], s["table"], s["lens"],
                        s["out"], lse=s["lse"], max_blocks_per_seq=s["most"], workspace=s["workspace"])
    return dict(out=s["out"], lse=s["lse"])


def own_prefix(s):
    from paper_2609_00097_b200 import ffd
    shared = dict(lse=s["lse"], max_prefix_blocks=s["prefix_most"], max_blocks_per_seq=s["most"], workspace=s["workspace"])
    if s["case"]["fmt"] == "bf16":
        ffd.ffd_decode_prefix(s["cfg"], s["q"], s["k_cache"], s["v_cache"], s["prefix_table"], s["prefix_len"], s["table"],
                              s["lens"], s["out"], **shared)
    else:
        ffd.ffd_decode_prefix_byte(s["cfg"], s["q"], s["k_cache"], s["v_cache"], s["prefix_table"], s["prefix_len"],
                                   s["k_code"], s["v_code"], s["k_scale"], s["v_scale"], s["table"], s["lens"], s["out"],
                                   **shared)
    return dict(out=s["out"], lse=s["lse"])


OWN = dict(write=own_write, read=own_read, decode=own_decode, prefix=own_prefix)


def page_table(s):
    if s["table"] is not None:
        return s["table"].long()
    return torch.arange(s["lens"].numel() * s["most"], device="cuda").view(-1, s["most"])


def plain_write(s):
    fmt, lens = s["case"]["fmt"], s["lens"].long()
    if s["start"] is None:   # row b is the last token of sequence b
        rows = torch.nonzero(lens > 0).squeeze(1)
        seq, token = rows, lens[rows] - 1
    else:
        rows = torch.arange(s["rows"], device="cuda")
        seq = torch.searchsorted(s["start"].long(), rows, right=True) - 1
        token = s["first"].long()[seq] + rows - s["start"].long()[seq]
        rows, seq, token = rows[token < lens[seq]], seq[token < lens[seq]], token[token < lens[seq]]
    page, at = page_table(s)[seq, token // PAGE], token % PAGE
    for x in "kv":
        code, scale = quantise(s[x + "_new"][rows], fmt)
        s[x + "_code"].view(torch.int8)[page, :, at] = code.view(torch.int8)
        s[x + "_scale"][page, :, at] = scale
    return dict(k=s["k_code"], v=s["v_code"], k_scale=s["k_scale"], v_scale=s["v_scale"])


def plain_read(s):
    token = torch.arange(s["most"] * PAGE, device="cuda")
    seq, token = torch.nonzero(token[None, :] < s["lens"].long()[:, None], as_tuple=True)
    page, to, at = page_table(s)[seq, token // PAGE], seq * s["most"] + token // PAGE, token % PAGE
    for x in "kv":
        value = s[x + "_code"].view(torch.int8)[page, :, at].view(s[x + "_code"].dtype).float() * s[x + "_scale"][page, :, at][..., None]
        s[x + "_cache"][to, :, at] = value.to(torch.bfloat16)
    return dict(k=s["k_cache"], v=s["v_cache"])


def gathered(s, x):
    """[batch, kv_heads, tokens, D] in 32 bits, whatever the sequences' pages hold; zero past their ends."""
    page = page_table(s)
    if s["case"]["fmt"] == "bf16":
        t = s[x + "_cache"][page].float()
    else:
        t = s[x + "_code"].view(torch.int8)[page].view(s[x + "_code"].dtype).float() * s[x + "_scale"][page][..., None]
    t = t.permute(0, 2, 1, 3, 4).reshape(page.shape[0], t.shape[2], -1, D)
    inside = torch.arange(t.shape[2], device="cuda")[None, :] < s["lens"][:, None]
    return t.masked_fill_(~inside[:, None, :, None], 0.0), inside


def joined(parts):
    """Attention over several lists of scored tokens: (scores [.., tokens], product of the weights with the values)."""
    top = parts[0][0].amax(-1)
    if len(parts) > 1:
        top = torch.maximum(top, parts[1][0].amax(-1))
    safe = torch.where(top == -math.inf, 0.0, top)[..., None]
    weights = [torch.exp(score - safe) for score, _ in parts]
    total, out = weights[0].sum(-1, keepdim=True), parts[0][1](weights[0])
    if len(parts) > 1:
        total, out = total + weights[1].sum(-1, keepdim=True), out + parts[1][1](weights[1])
    out = torch.where(total > 0, out / total, 0.0)
    return out, torch.log(total.squeeze(-1)) + safe.squeeze(-1)


def own_tokens(s):
    k, inside = gathered(s, "k")
    batch, kv_heads = k.shape[:2]
    q = s["q"].float().view(batch, kv_heads, -1, D)
    score = (q @ k.transpose(-1, -2)) / math.sqrt(D)
    score = score.masked_fill(~inside[:, None, None, :], -math.inf)
    del k
    v = gathered(s, "v")[0]
    return score, lambda w: w @ v


def finish(s, out, lse):
    batch, q_heads = s["q"].shape[:2]
    return dict(out=out.reshape(batch, q_heads, D).to(s["out"].dtype), lse=lse.reshape(batch, q_heads))


def plain_decode(s):
    return finish(s, *joined([own_tokens(s)]))


def plain_prefix(s):
    n = s["case"]["prefix"]
    batch, kv_heads = s["lens"].numel(), s["case"]["kv_heads"]
    k, v = (s[x + "_cache"][s["prefix_table"].long()].permute(1, 0, 2, 3).reshape(kv_heads, -1, D)[:, :n].float() for x in "kv")
    q = s["q"].float().view(batch, kv_heads, -1, D)
    flat = q.transpose(0, 1).reshape(kv_heads, -1, D)
    score = (flat @ k.transpose(-1, -2)) / math.sqrt(D)

    def back(t):
        return t.view(kv_heads, batch, -1, t.shape[-1]).transpose(0, 1)

    def product(w):
        return back(w.transpose(0, 1).reshape(kv_heads, -1, n) @ v)

    return finish(s, *joined([(back(score), product), own_tokens(s)]))


PLAIN = dict(write=plain_write, read=plain_read, decode=plain_decode, prefix=plain_prefix)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------


def work(case):
    lens, kv_heads, q_heads, batch = lengths(case), case["kv_heads"], case["q_heads"], case["batch"]
    row = kv_heads * D
    byte = 2 * (row + 4 * kv_heads)          # a token's key and value in 8 bits with their scales
    half = 2 * 2 * row                       # the same in 16 bits
    tokens = sum(lens)
    if case["kind"] == "write":
        new = tokens if case["new"] == "all" else sum(n > 0 for n in lens)
        return dict(bytes=new * (half + byte) + 12 * batch, flops=new * 2 * row * 3)
    if case["kind"] == "read":
        return dict(bytes=tokens * (half + byte) + 4 * batch, flops=tokens * 2 * row)
    heads = batch * q_heads * (2 * D + (2 if case["out"] == "bf16" else 4) * D + 4)
    total = tokens * (half if case["fmt"] == "bf16" else byte) + heads + 4 * batch
    flops = 4 * D * q_heads * tokens
    if case["kind"] == "prefix":
        total += case["prefix"] * half
        flops += 4 * D * q_heads * batch * case["prefix"]
    return dict(bytes=total, flops=flops)


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    kind, fmt = case["kind"], case["fmt"]
    lens = s["lens"].tolist()
    table = s["table"].tolist() if s["table"] is not None else [[b * s["most"] + i for i in range(s["most"])] for b in range(len(lens))]

    def tokens(x, b):
        """The keys or values of sequence b: [kv_heads, tokens, D]."""
        pages = torch.tensor(table[b][:(lens[b] + PAGE - 1) // PAGE], dtype=torch.long, device="cuda")
        if fmt == "bf16":
            t = s[x + "_cache"][pages].double()
        else:
            t = s[x + "_code"].view(torch.int8)[pages].view(s[x + "_code"].dtype).double() * s[x + "_scale"][pages].double()[..., None]
        return t.transpose(0, 1).reshape(case["kv_heads"], -1, D)[:, :lens[b]]

    if kind == "write":
        outs = {}
        for x in "kv":
            code, scale = s[x + "_code"].double(), s[x + "_scale"].double()
            for b, n in enumerate(lens):
                first = 0 if case["new"] == "all" else n - 1
                if n == 0:
                    continue
                row0 = b if s["start"] is None else int(s["start"][b])
                new = s[x + "_new"][row0:row0 + n - first].double()                       # [tokens, kv_heads, D]
                top = new.abs().amax(-1)
                token = torch.arange(first, n, device="cuda")
                page, at = torch.tensor(table[b], device="cuda")[token // PAGE], token % PAGE
                scale[page, :, at] = top / LIMIT[fmt]
                grid = new * (LIMIT[fmt] / top.clamp(min=1e-300))[..., None]
                if fmt == "e4m3":
                    step = torch.exp2(torch.floor(torch.log2(grid.abs().clamp(min=2.0 ** -6))) - 3)
                    grid = torch.round(grid / step) * step
                    code[page, :, at] = grid
            outs[x] = code if fmt == "e4m3" else None
            outs[x + "_scale"] = scale
        return outs
    if kind == "read":
        outs = {}
        for x in "kv":
            cache = s[x + "_cache"].double()
            for b, n in enumerate(lens):
                if n:
                    t = tokens(x, b).transpose(0, 1)
                    at = torch.arange(n, device="cuda")
                    cache[b * s["most"] + at // PAGE, :, at % PAGE] = t
            outs[x] = cache
        return outs
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(case["batch"], case["q_heads"], D, dtype=torch.float64, device="cuda")
    lse = torch.full((case["batch"], case["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    if kind == "prefix":
        shared = {x: s[x + "_cache"][s["prefix_table"].long()].transpose(0, 1).reshape(case["kv_heads"], -1, D)[:, :case["prefix"]]
                  for x in "kv"}
    for b, n in enumerate(lens):
        mine = {x: tokens(x, b) for x in "kv"}
        for g in range(case["kv_heads"]):
            heads = slice(g * group, (g + 1) * group)
            k, v = (torch.cat([shared[x][g].double(), mine[x][g]]) if kind == "prefix" else mine[x][g] for x in "kv")
            if not k.shape[0]:
                continue
            score = s["q"][b, heads].double() @ k.T / math.sqrt(D)
            lse[b, heads] = torch.logsumexp(score, -1)
            out[b, heads] = torch.softmax(score, -1) @ v
    return dict(out=out, lse=lse)
