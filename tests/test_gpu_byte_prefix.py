"""The byte cache (write, read back, attend) and the shared prefix on the GPU, against plain 64-bit computations.

Tolerances of the attention results.  Let W = sum_t p_t |v_t| / sum_t p_t (per channel) and A = max_t sm sum_c |q_c k_tc|.
 * A logit is a chain of at most 9 tensor-core accumulations of exact products (8 steps of 16 channels) with binary32
   results, each off by at most 2^-22 of the terms' magnitude, and two binary32 products: |dS| <= 11 * 2^-22 * A.
 * Over a byte cache q is a sum of pieces.  e4m3: scaled by a power of two to a largest element in [128, 256), its 8 bits are
   two e4m3 numbers of 4 bits; elements below 2^-2 meet the grid's end, 2^-9, and are off by 2^-10 at most, 2^-17 of the
   largest.  int8: scaled by a power of two to a largest element in [2^21, 2^22) and rounded to an integer, which three
   digits hold: off by 2^-1, at most 2^-22 of the largest.
   dS grows by (2^-17 or 2^-22) sm max|q_c| max_t sum_c |k_tc|.
 * A weight 2^x has |dx| / |x| <= 2^-22 from its argument, 2^-22 from ex2 and keeps 16 bits or more in two pieces
   (2^-16): |dp| / p <= dS + |x| 2^-22 + 2^-22 + 2^-16, |x| <= 2 A / ln 2.
 * The sums over n tokens: at most n / 16 chained accumulations of 2^-22 each, the merges 2^-20.
 * The quotient doubles what the weights are off by:  tol_out = W * (2 * dp + (n / 16) * 2^-22 + 2^-20).
 * Over a byte cache a weight meets the codes as p_t s_t (s_t the value's scale) relative to about the largest of them, in two
   f16 pieces of which the second is scaled by 2^11: f16 numbers are multiples of 2^-24, so the pieces are multiples of
   2^-35 and a weight is off by 2^-36 of the largest p s, however small it is itself.  A channel in which the heavy tokens
   have code 0 shows it.  |code_t| s_t <= max_c |v_tc|, so the n weights add  n 2^-36 max_t (p_t max_c |v_tc|) / sum_t p_t.
 * One bf16 piece of P (a prefix under more than 128 rows and a bf16 result) adds 2^-8 W; a bf16 result 2^-8 |out|.
 * lse: dS + |x| 2^-22 + n / 16 * 2^-22 + 2^-20 + 2^-23 |lse|.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

D, BLK = 128, 64
LIMIT = {"int8": 127.0, "e4m3": 448.0}
DTYPE = {"int8": torch.int8, "e4m3": torch.float8_e4m3fn}
FORMATS = ["int8", "e4m3"]


@pytest.fixture(scope="module")
def ffd():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_00097_b200 import ffd as m
    m.load_library()
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def quantise(x, fmt):
    """The documented operations, one binary32 operation each."""
    x = x.float()
    x = torch.where(x.isnan(), torch.zeros_like(x), x).clamp(-torch.finfo(torch.bfloat16).max, torch.finfo(torch.bfloat16).max)
    top = x.abs().amax(-1, keepdim=True)
    tiny = top < 2.0 ** -100
    # tensors on both sides: with a number on one side torch multiplies by a rounded reciprocal instead
    limit, safe = torch.full_like(top, LIMIT[fmt]), torch.where(tiny, torch.ones_like(top), top)
    scale = torch.where(tiny, torch.zeros_like(top), top / limit).squeeze(-1)
    y = torch.where(tiny, torch.zeros_like(x), x * (limit / safe))
    return (y.round().to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)), scale


def raw(t):
    return t.view(torch.int8)


def table_for(g, lens, spare=3):
    """A random page table of these lengths: (table [B, most], pages)."""
    nb = [(n + BLK - 1) // BLK for n in lens]
    most, total = max(1, max(nb)), sum(nb) + spare
    order = torch.randperm(total, generator=g, device="cuda").to(torch.int32)
    table = torch.full((len(lens), most), -7, dtype=torch.int32, device="cuda")    # entries behind a sequence's end are not used
    at = 0
    for b, n in enumerate(nb):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


class Cache:
    """Sequences in a byte cache or in 16-bit pages; everything that is no sequence's holds NaN."""

    def __init__(self, g, fmt, lens, kv_heads, k_gain=1.0, v_gain=1.0, paged=True):
        self.lens, self.fmt = list(lens), fmt
        if paged:
            self.table, self.pages = table_for(g, lens)
            self.most = self.table.shape[1]
            t = self.table.long()
        else:
            self.most = max(1, max((n + BLK - 1) // BLK for n in lens))
            self.pages, self.table = len(lens) * self.most, None
            t = torch.arange(self.pages, device="cuda").view(len(lens), -1)
        self.index = t
        self.seq_lens = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.values = []
        for x, gain in (("k", k_gain), ("v", v_gain)):
            if fmt == "bf16":
                pool = torch.full((self.pages, kv_heads, BLK, D), float("nan"), dtype=torch.bfloat16, device="cuda")
                scale = None
            else:
                pool = torch.full((self.pages, kv_heads, BLK, D), -1, dtype=torch.int8, device="cuda")   # e4m3: NaN
                pool = pool if fmt == "int8" else pool.view(torch.float8_e4m3fn)
                scale = torch.full((self.pages, kv_heads, BLK), float("nan"), device="cuda")
            vals = []
            for b, n in enumerate(self.lens):
                data = (gain * normal(g, n, kv_heads, D) * torch.exp(normal(g, n, kv_heads, 1))).to(torch.bfloat16)
                at = torch.arange(n, device="cuda")
                page = t[b][at // BLK] if n else at
                if fmt == "bf16":
                    pool[page, :, at % BLK] = data
                    vals.append(data.double())
                else:
                    code, sc = quantise(data, fmt)
                    raw(pool)[page, :, at % BLK] = raw(code)
                    scale[page, :, at % BLK] = sc
                    vals.append(code.double() * sc.double()[..., None])
            setattr(self, x, pool)
            setattr(self, x + "_scale", scale)
            self.values.append(vals)

    @property
    def byte(self):
        return self.k, self.v, self.k_scale, self.v_scale


def reference(q, ks, vs, sm):
    """q [Hq, D]; ks, vs [n, Hkv, D] in 64 bits -> out, lse, W [Hq, D], A [Hq] and what the grain of f16 adds [Hq]."""
    hq, hkv, n = q.shape[0], ks.shape[1], ks.shape[0]
    if n == 0:
        z = torch.zeros(hq, D, dtype=torch.float64, device="cuda")
        return z, torch.full((hq,), -math.inf, dtype=torch.float64, device="cuda"), z, z[:, 0], z[:, 0]
    q = q.double().view(hkv, hq // hkv, D)
    k, v = ks.permute(1, 0, 2), vs.permute(1, 0, 2)
    s = q @ k.transpose(1, 2) * sm
    a = (q.abs() @ k.abs().transpose(1, 2) * sm).amax(-1)
    p = torch.softmax(s, -1)
    grain = n * 2.0 ** -36 * (p * v.abs().amax(-1)[:, None, :]).amax(-1)
    return (p @ v).reshape(hq, D), torch.logsumexp(s, -1).reshape(hq), (p @ v.abs()).reshape(hq, D), a.reshape(hq), grain.reshape(hq)


PIECES = {"bf16": 0.0, "e4m3": 2.0 ** -17, "int8": 2.0 ** -22}


def check(out, lse, q, caches, fmt, sm=1 / math.sqrt(D), one_piece=False):
    """caches: per sequence (k values, v values) in 64 bits; fmt: the format of the sequences' own tokens."""
    assert not out.float().isnan().any()
    for b, (k, v) in enumerate(caches):
        want, want_lse, w, a, grain = reference(q[b], k, v, sm)
        n = k.shape[0]
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -math.inf).all()
            continue
        group = q.shape[1] // k.shape[1]
        k1 = k.abs().sum(-1).amax(0).repeat_interleave(group)
        ds = PIECES[fmt] * sm * q[b].double().abs().amax(-1) * k1 + 11 * 2.0 ** -22 * a + 2 * a / math.log(2) * 2.0 ** -22
        dp = ds + 2.0 ** -22 + 2.0 ** -16
        tol = w * (2 * dp + n / 16 * 2.0 ** -22 + 2.0 ** -20 + (2.0 ** -8 if one_piece else 0))[:, None] + grain[:, None]
        if out.dtype == torch.bfloat16:
            tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs()
        err = (out[b].double() - want).abs()
        assert (err <= tol + 1e-37).all(), (b, n, (err / (tol + 1e-37)).max().item())
        tol_lse = ds + n / 16 * 2.0 ** -22 + 2.0 ** -20 + 2.0 ** -23 * want_lse.abs()
        assert ((lse[b].double() - want_lse).abs() <= tol_lse).all(), (b, n, (lse[b].double() - want_lse).abs().max().item())


def decode(ffd, cfg, q, c, ws=None, stream=None):
    ws = ffd.new_workspace_prefix(cfg, len(c.lens), c.most) if ws is None else ws
    out = torch.full(q.shape, float("nan"), dtype=torch.float32 if cfg.out_dtype else torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    ffd.ffd_decode_byte(cfg, q, *c.byte, c.table, c.seq_lens, out, max_blocks_per_seq=c.most, workspace=ws, lse=lse,
                        stream=stream)
    return out, lse, ws


# ---- writing and reading back --------------------------------------------------------------------------------------


def write_case(g, fmt, kv_heads, spans, fused, scale=1.0):
    """spans: (first, length with the new tokens) per sequence."""
    lens = [n for _, n in spans]
    counts = [max(0, n - f) for f, n in spans]
    table, pages = table_for(g, lens)
    rows = max(1, sum(counts)) + 2                        # two rows behind the last sequence
    width = kv_heads * D * (3 if fused else 1)
    data = torch.zeros(2, rows, width, dtype=torch.bfloat16, device="cuda")
    at = kv_heads * D if fused else 0
    k_new, v_new = (data[i][:, at:at + kv_heads * D].view(rows, kv_heads, D) for i in (0, 1))
    for t in (k_new, v_new):
        t.copy_((scale * normal(g, rows, kv_heads, D) * torch.exp(2 * normal(g, rows, kv_heads, 1))).to(torch.bfloat16))
    starts = [sum(counts[:b]) for b in range(len(counts))]
    pool = {x: torch.full((pages, kv_heads, BLK, D), 5, dtype=torch.int8, device="cuda") for x in "kv"}
    pool = {x: t if fmt == "int8" else t.view(torch.float8_e4m3fn) for x, t in pool.items()}
    scales = {x: torch.full((pages, kv_heads, BLK), 0.25, device="cuda") for x in "kv"}
    return dict(lens=lens, counts=counts, starts=starts, table=table, k_new=k_new, v_new=v_new, pool=pool, scales=scales)


def expect_written(c, fmt, spans):
    want = {x: raw(c["pool"][x]).clone() for x in "kv"}, {x: c["scales"][x].clone() for x in "kv"}
    for x in "kv":
        code, scale = quantise(c[x + "_new"], fmt)
        for b, (first, n) in enumerate(spans):
            if n > first:
                token = torch.arange(first, n, device="cuda")
                page, new = c["table"][b].long()[token // BLK], slice(c["starts"][b], c["starts"][b] + n - first)
                want[0][x][page, :, token % BLK] = raw(code)[new]
                want[1][x][page, :, token % BLK] = scale[new]
    return want


def write(ffd, cfg, c, spans, one=False):
    i32 = dict(dtype=torch.int32, device="cuda")
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    lens = torch.tensor(c["lens"], **i32)
    extra = {} if one else dict(row_start=torch.tensor(c["starts"], **i32), first_token=torch.tensor([f for f, _ in spans], **i32))
    batch = len(spans)
    k_new, v_new = (c["k_new"][:batch], c["v_new"][:batch]) if one else (c["k_new"], c["v_new"])
    ffd.ffd_write_kv_byte(cfg, k_new, v_new, c["pool"]["k"], c["pool"]["v"], c["scales"]["k"], c["scales"]["v"], c["table"], lens,
                          max_blocks_per_seq=c["table"].shape[1], workspace=ws, **extra)
    return ffd.ffd_read_device_status(ws)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kv_heads,fused,spans", [
    (1, False, [(0, 1)]),
    (2, True, [(0, 64), (0, 0), (3, 5), (63, 65), (10, 10)]),
    (3, False, [(0, 130), (128, 129), (64, 128)]),
    (8, True, [(0, 700), (511, 1025), (0, 1), (0, 0), (0, 333)]),
    (9, False, [(5, 200)]),
    (17, False, [(0, 700), (1, 70)]),
    # enough rows for the kernel that streams them
    (8, True, [(0, 2500), (3, 4), (0, 0), (100, 900), (77, 77)]),
    (9, False, [(0, 2000), (64, 65)]),
    (1, True, [(0, 9600)]),
    (19, False, [(1, 64), (0, 1300)]),
])
def test_write_is_exactly_the_documented_quantizer(ffd, fmt, kv_heads, fused, spans):
    g = gen(100 + kv_heads)
    c = write_case(g, fmt, kv_heads, spans, fused)
    want = expect_written(c, fmt, spans)
    assert write(ffd, ffd.Config(kv_heads, kv_heads), c, spans) == 0
    for x in "kv":    # every byte of the pool: what was not written is as it was
        assert torch.equal(raw(c["pool"][x]), want[0][x])
        assert torch.equal(c["scales"][x], want[1][x])
    # against the definition in 64 bits: an int8 value is within half a step (and its rounding) of x, an e4m3 value within
    # 2^-4 of x or half of the smallest step
    for x in "kv":
        code, scale = quantise(c[x + "_new"], fmt)
        value, true = code.double() * scale.double()[..., None], c[x + "_new"].double()
        step = scale.double()[..., None]
        tol = 0.5 * step if fmt == "int8" else torch.maximum(2.0 ** -4 * true.abs(), 2.0 ** -10 * step)
        assert ((value - true).abs() <= tol + 2.0 ** -21 * true.abs()).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_write_of_one_token_per_sequence(ffd, fmt):
    g = gen(7)
    lens = [1, 0, 64, 65, 700, 129]
    spans = [(max(0, n - 1), n) for n in lens]
    c = write_case(g, fmt, 5, spans, False)
    c["starts"] = list(range(len(lens)))
    c["k_new"], c["v_new"] = (torch.cat([c[x], c[x]])[:len(lens)].contiguous() for x in ("k_new", "v_new"))
    want = expect_written(c, fmt, spans)
    assert write(ffd, ffd.Config(5, 5), c, spans, one=True) == 0
    for x in "kv":
        assert torch.equal(raw(c["pool"][x]), want[0][x])
        assert torch.equal(c["scales"][x], want[1][x])


def test_write_of_one_token_for_each_of_many_sequences(ffd):
    g = gen(77)
    lens = [(b * 37) % 200 for b in range(9600)]
    spans = [(max(0, n - 1), n) for n in lens]
    c = write_case(g, "e4m3", 2, [(0, 9598)], False)     # 9600 rows
    c["table"], pages = table_for(g, lens)
    c["lens"], c["starts"] = lens, list(range(len(lens)))
    c["pool"] = {x: torch.full((pages, 2, BLK, D), 5, dtype=torch.int8, device="cuda").view(torch.float8_e4m3fn) for x in "kv"}
    c["scales"] = {x: torch.full((pages, 2, BLK), 0.25, device="cuda") for x in "kv"}
    lt = torch.tensor(lens, device="cuda")
    assert write(ffd, ffd.Config(2, 2), c, spans, one=True) == 0
    some = torch.nonzero(lt > 0).squeeze(1)
    page, row = c["table"].long()[some, (lt[some] - 1) // BLK], (lt[some] - 1) % BLK
    for x in "kv":
        code, scale = quantise(c[x + "_new"], "e4m3")
        want, want_scale = torch.full_like(raw(c["pool"][x]), 0), torch.full_like(c["scales"][x], 0.25)
        want.copy_(raw(torch.full((1,), 5, dtype=torch.int8, device="cuda")))
        want[page, :, row], want_scale[page, :, row] = raw(code)[some], scale[some]
        assert torch.equal(raw(c["pool"][x]), want) and torch.equal(c["scales"][x], want_scale)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("rows", [12, 3000])
def test_write_of_extreme_rows(ffd, fmt, rows):
    """Zero rows, rows around the smallest and largest magnitudes, infinities and NaN."""
    g = gen(8)
    spans = [(0, rows)]
    c = write_case(g, fmt, 2 if rows == 12 else 7, spans, False)
    k = c["k_new"]
    k[0] = 0.0
    k[1] *= 2.0 ** -120
    k[2, 0] = 2.0 ** -100
    k[3, 0] = -(2.0 ** -101)
    k[4] = torch.finfo(torch.bfloat16).max
    k[5, 1, 3] = float("inf")
    k[6, 0, 127] = float("-inf")
    k[7, 1] = float("nan")
    k[8, 0, 5] = float("nan")
    k[9, 0, 0], k[9, 0, 1] = float("nan"), float("inf")
    k[10] = 0.0
    k[10, 1, 77] = -3.0
    want = expect_written(c, fmt, spans)
    heads = c["k_new"].shape[1]
    assert write(ffd, ffd.Config(heads, heads), c, spans) == 0
    for x in "kv":
        got, exp = (torch.where(codes == -128, 0, codes) for codes in (raw(c["pool"][x]), want[0][x]))   # e4m3's -0 as +0
        assert torch.equal(got, exp)
        assert torch.equal(c["scales"][x], want[1][x])


def test_write_with_many_sequences(ffd):
    """The search for a row's sequence: more than 32^2 sequences, most of them with nothing new."""
    g = gen(9)
    spans = [(0, (b * 7) % 3 if b % 5 else 0) for b in range(1500)]
    c = write_case(g, "int8", 1, spans, False)
    want = expect_written(c, "int8", spans)
    assert write(ffd, ffd.Config(1, 1), c, spans) == 0
    for x in "kv":
        assert torch.equal(raw(c["pool"][x]), want[0][x])
        assert torch.equal(c["scales"][x], want[1][x])


def test_write_reports_bad_pages_and_lengths(ffd):
    g = gen(10)
    spans = [(0, 130), (0, 70)]
    c = write_case(g, "int8", 2, spans, False)
    want = expect_written(c, "int8", spans)
    pages = c["pool"]["k"].shape[0]
    hidden = int(c["table"][0, 1])
    for x in "kv":
        want[0][x][hidden], want[1][x][hidden] = 5, 0.25
    for bad in (-1, pages, 2 ** 31 - 1):
        c["table"][0, 1] = bad
        assert write(ffd, ffd.Config(2, 2), c, spans) == ffd.DEV_BAD_PAGE
    for x in "kv":
        assert torch.equal(raw(c["pool"][x]), want[0][x])
    c["table"][0, 1] = hidden
    c["lens"][1] = 1000        # beyond the table: clamped to its 192 tokens; rows 0 .. 69 still are tokens 0 .. 69
    c["table"][1, 2] = c["table"][0, 2]
    assert write(ffd, ffd.Config(2, 2), c, spans) == ffd.DEV_BAD_SEQ_LEN
    c["lens"][1] = -5
    assert write(ffd, ffd.Config(2, 2), c, spans) == ffd.DEV_BAD_SEQ_LEN


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("kv_heads,lens,first", [
    (1, [1], None), (2, [64, 0, 65, 130], None), (8, [700, 1, 0, 333], [63, 0, 0, 64]), (3, [200, 129], [128, 129]),
    (2, [100, 100], [200, -4])])
def test_read_back_is_the_rounded_product_and_touches_nothing_else(ffd, fmt, kv_heads, lens, first):
    g = gen(20 + kv_heads)
    c = Cache(g, fmt, lens, kv_heads)
    cfg = ffd.Config(kv_heads, kv_heads)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    out_table, out_pages = table_for(g, lens, spare=1)
    k, v = (torch.full((out_pages, kv_heads, BLK, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    want = []
    for x, pool, scale in (("k", c.k, c.k_scale), ("v", c.v, c.v_scale)):
        w = torch.full_like(k, 9.0)
        for b, n in enumerate(lens):
            lo = max(0, first[b]) if first else 0
            for t in range(lo, n):
                page, to = int(c.table[b, t // BLK]), int(out_table[b, t // BLK])
                w[to, :, t % BLK] = (pool[page, :, t % BLK].float() * scale[page, :, t % BLK][:, None]).to(torch.bfloat16)
        want.append(w)
    ft = None if first is None else torch.tensor(first, dtype=torch.int32, device="cuda")
    ffd.ffd_read_kv_byte(cfg, *c.byte, c.table, c.seq_lens, k, v, cache_table=out_table, first_token=ft,
                         max_blocks_per_seq=c.most, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_read_back_reports_bad_pages_on_both_sides(ffd):
    g = gen(30)
    c = Cache(g, "int8", [200, 130], 2, paged=False)
    cfg = ffd.Config(2, 2)
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    k, v = (torch.full((c.pages, 2, BLK, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv")
    ffd.ffd_read_kv_byte(cfg, *c.byte, None, c.seq_lens, k, v, max_blocks_per_seq=c.most, workspace=ws)
    good = k.clone()
    assert ffd.ffd_read_device_status(ws) == 0
    for side in ("block", "cache"):
        table = torch.arange(c.pages, dtype=torch.int32, device="cuda").view(2, -1).contiguous()
        table[0, 2] = c.pages if side == "block" else -1
        k.fill_(9.0)
        ffd.ffd_read_kv_byte(cfg, *c.byte, table if side == "block" else None, c.seq_lens, k, v, max_blocks_per_seq=c.most,
                             cache_table=table if side == "cache" else None, workspace=ws)
        assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_PAGE
        assert (k[2] == 9.0).all()
        keep = [i for i in range(c.pages) if i != 2]
        assert torch.equal(k[keep], good[keep])


# ---- attention over the byte cache ------------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group", range(1, 9))
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_decode_of_small_ragged_batches(ffd, fmt, group, out_dtype):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 0, 127, 128, 129, 1000]
    g = gen(40 + group)
    c = Cache(g, fmt, lens, 2)
    q = normal(g, len(lens), 2 * group, D).to(torch.bfloat16)
    out, lse, ws = decode(ffd, ffd.Config(2 * group, 2, out_dtype=out_dtype), q, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, list(zip(*c.values)), c.fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("heads,lens", [((8, 2), [4096]), ((32, 8), [5001, 77, 1]), ((8, 1), [20011]), ((3, 3), [9000, 2, 700])])
def test_decode_of_longer_contexts(ffd, fmt, heads, lens):
    g = gen(60 + heads[0])
    c = Cache(g, fmt, lens, heads[1], paged=len(lens) > 1)
    q = normal(g, len(lens), heads[0], D).to(torch.bfloat16)
    out, lse, ws = decode(ffd, ffd.Config(*heads), q, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, list(zip(*c.values)), c.fmt)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("q_gain,k_gain,v_gain", [(2.0 ** -60, 1.0, 1.0), (2.0 ** 40, 2.0 ** -40, 1.0), (8.0, 1.0, 2.0 ** 100),
                                                  (1.0, 3.0, 2.0 ** -90), (0.0, 1.0, 1.0)])
def test_decode_of_extreme_magnitudes(ffd, fmt, q_gain, k_gain, v_gain):
    g = gen(70)
    c = Cache(g, fmt, [500, 65], 2, k_gain=k_gain, v_gain=v_gain)
    q = (q_gain * normal(g, 2, 8, D)).to(torch.bfloat16)
    out, lse, ws = decode(ffd, ffd.Config(8, 2), q, c)
    check(out, lse, q, list(zip(*c.values)), c.fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_of_very_different_sizes(ffd, fmt):
    """One token's value is 2^60 times the others' while its weight is negligible, and another's value is zero."""
    g = gen(71)
    c = Cache(g, fmt, [300], 1)
    q = torch.zeros(1, 4, D, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 16.0
    page, row = int(c.table[0, 1]), 7
    raw(c.k)[page, 0, row] = 0
    c.k_scale[page, 0, row] = 1.0
    one = raw(torch.tensor([-100.0], device="cuda").to(DTYPE[fmt]))
    raw(c.k)[page, 0, row, 0] = one[0]                  # its logit: -1600 / sqrt(128)
    c.v_scale[page, 0, row] = 2.0 ** 60
    raw(c.v)[int(c.table[0, 0]), 0, 3] = 0
    c.v_scale[int(c.table[0, 0]), 0, 3] = 0.0
    values = []
    for pool, scale in ((c.k, c.k_scale), (c.v, c.v_scale)):
        t = torch.arange(300, device="cuda")
        p = c.table[0].long()[t // BLK]
        values.append(pool.double()[p, :, t % BLK] * scale.double()[p, :, t % BLK][..., None])
    out, lse, _ = decode(ffd, ffd.Config(4, 1), q, c)
    check(out, lse, q, [tuple(values)], fmt)


def test_decode_reports_and_skips_bad_pages(ffd):
    g = gen(72)
    c = Cache(g, "int8", [300, 200, 64], 2)
    cfg = ffd.Config(8, 2)
    q = normal(g, 3, 8, D).to(torch.bfloat16)
    for bad in (-1, c.pages, 2 ** 31 - 1, -2 ** 31):
        c.table[0, 2] = bad
        c.table[2, 0] = bad              # a sequence of which nothing is left
        out, lse, ws = decode(ffd, cfg, q, c)
        assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_PAGE
        keep = torch.tensor([t for t in range(300) if t // BLK != 2], device="cuda")
        none = c.values[0][2][:0]
        check(out, lse, q, [(c.values[0][0][keep], c.values[1][0][keep]), (c.values[0][1], c.values[1][1]), (none, none)], "int8")


def test_decode_clamps_bad_lengths(ffd):
    g = gen(73)
    c = Cache(g, "e4m3", [192, 130], 2)
    q = normal(g, 2, 4, D).to(torch.bfloat16)
    c.seq_lens[0], c.seq_lens[1] = 100000, -3
    out, lse, ws = decode(ffd, ffd.Config(4, 2), q, c)
    assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_SEQ_LEN
    check(out, lse, q, [(c.values[0][0], c.values[1][0]), (c.values[0][1][:0], c.values[1][1][:0])], "e4m3")


# ---- shared prefix ------------------------------------------------------------------------------------------------------


class Shared:
    """A prefix in 16-bit pages whose unused rows hold NaN."""

    def __init__(self, g, n, kv_heads, spare=2, gain=1.0):
        self.n, self.most = n, max(1, (n + BLK - 1) // BLK)
        pages = self.most + spare
        self.table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[:self.most].contiguous()
        self.len = torch.tensor([n], dtype=torch.int32, device="cuda")
        self.pools, self.values = [], []
        for _ in "kv":
            pool = torch.full((pages, kv_heads, BLK, D), float("nan"), dtype=torch.bfloat16, device="cuda")
            data = (gain * normal(g, n, kv_heads, D) * torch.exp(0.5 * normal(g, n, kv_heads, 1))).to(torch.bfloat16)
            at = torch.arange(n, device="cuda")
            pool[self.table.long()[at // BLK], :, at % BLK] = data
            self.pools.append(pool)
            self.values.append(data.double())


def with_prefix(ffd, cfg, q, pre, c, ws=None, stream=None):
    ws = ffd.new_workspace_prefix(cfg, len(c.lens), c.most, pre.most) if ws is None else ws
    out = torch.full(q.shape, float("nan"), dtype=torch.float32 if cfg.out_dtype else torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    kw = dict(max_prefix_blocks=pre.most, max_blocks_per_seq=c.most, workspace=ws, lse=lse, stream=stream)
    if c.fmt == "bf16":   # one pool: the sequences' pages behind the prefix's
        at = pre.pools[0].shape[0]
        k, v = torch.cat([pre.pools[0], c.k]), torch.cat([pre.pools[1], c.v])
        table = (c.index + at).to(torch.int32).contiguous()
        ffd.ffd_decode_prefix(cfg, q, k, v, pre.table, pre.len, table, c.seq_lens, out, **kw)
    else:
        ffd.ffd_decode_prefix_byte(cfg, q, *pre.pools, pre.table, pre.len, *c.byte, c.table, c.seq_lens, out, **kw)
    return out, lse, ws


def joined_values(pre, c):
    return [tuple(torch.cat([pre.values[i], c.values[i][b]]) for i in (0, 1)) for b in range(len(c.lens))]


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("fmt", ["bf16", "int8", "e4m3"])
@pytest.mark.parametrize("prefix", [0, 1, 63, 64, 65, 128, 129, 300, 2011])
def test_prefix_lengths(ffd, fmt, prefix, out_dtype):
    g = gen(80 + prefix)
    lens = [0, 1, 17, 64, 200]
    pre, c = Shared(g, prefix, 2), Cache(g, fmt, lens, 2)
    q = normal(g, len(lens), 6, D).to(torch.bfloat16)
    out, lse, ws = with_prefix(ffd, ffd.Config(6, 2, out_dtype=out_dtype), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), c.fmt)


@pytest.mark.parametrize("out_dtype", [0, 1])
@pytest.mark.parametrize("batch,group,kv_heads,prefix", [
    (1, 1, 1, 700), (20, 5, 2, 700), (9, 3, 1, 300), (18, 7, 2, 90), (11, 6, 3, 2000), (128, 1, 1, 515), (129, 1, 2, 515), (40, 5, 2, 1000), (37, 7, 1, 333), (64, 8, 1, 130), (70, 8, 2, 1025),
    (43, 3, 4, 4133)])
def test_prefix_rows(ffd, batch, group, kv_heads, prefix, out_dtype):
    """Row tiles: one row, one full tile, one row in the second tile, several groups of two tiles, odd groups."""
    g = gen(90 + batch)
    lens = [(13 * b) % 70 for b in range(batch)]
    pre, c = Shared(g, prefix, kv_heads), Cache(g, "int8", lens, kv_heads)
    q = normal(g, batch, group * kv_heads, D).to(torch.bfloat16)
    out, lse, ws = with_prefix(ffd, ffd.Config(group * kv_heads, kv_heads, out_dtype=out_dtype), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), c.fmt, one_piece=batch * group > 128 and out_dtype == 0)


@pytest.mark.parametrize("batch", [4, 48])
def test_prefix_with_growing_logits(ffd, batch):
    """Keys that grow along the prefix: the running maximum is raised, and the accumulators rescaled, again and again."""
    g = gen(95)
    pre, c = Shared(g, 3001, 2), Cache(g, "bf16", [5 + b for b in range(batch)], 2)
    q = normal(g, batch, 8, D).to(torch.bfloat16)
    ramp = torch.linspace(0.01, 6.0, 3001, device="cuda")
    for x in (0,):
        at = torch.arange(3001, device="cuda")
        data = (pre.values[x] * ramp[:, None, None].double()).to(torch.bfloat16)
        pre.pools[x][pre.table.long()[at // BLK], :, at % BLK] = data
        pre.values[x] = data.double()
    out, lse, ws = with_prefix(ffd, ffd.Config(8, 2), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), c.fmt)


@pytest.mark.parametrize("batch", [3, 48])
def test_prefix_with_bad_pages_and_lengths(ffd, batch):
    g = gen(96)
    pre, c = Shared(g, 500, 2), Cache(g, "int8", [20] * batch, 2)
    cfg = ffd.Config(8, 2)
    q = normal(g, batch, 8, D).to(torch.bfloat16)
    good = pre.table.clone()
    for blk in (0, 3, 7):
        for bad in (-1, pre.pools[0].shape[0], 2 ** 31 - 1):
            pre.table[blk] = bad
            out, lse, ws = with_prefix(ffd, cfg, q, pre, c)
            assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_PAGE
            keep = torch.tensor([t for t in range(500) if t // BLK != blk], device="cuda")
            check(out, lse, q, [(torch.cat([pre.values[0][keep], k]), torch.cat([pre.values[1][keep], v])) for k, v in zip(*c.values)], c.fmt)
            pre.table.copy_(good)
    pre.table.fill_(-1)                   # nothing of the prefix is left
    out, lse, ws = with_prefix(ffd, cfg, q, pre, c)
    assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_PAGE
    check(out, lse, q, list(zip(*c.values)), c.fmt)
    pre.table.copy_(good)
    pre.len.fill_(-8)
    out, lse, ws = with_prefix(ffd, cfg, q, pre, c)
    assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_SEQ_LEN
    check(out, lse, q, list(zip(*c.values)), c.fmt)
    full = Shared(g, 512, 2)
    full.len.fill_(10 ** 9)
    out, lse, ws = with_prefix(ffd, cfg, q, full, c)
    assert ffd.ffd_read_device_status(ws) == ffd.DEV_BAD_SEQ_LEN
    check(out, lse, q, joined_values(full, c), c.fmt)


# ---- together, captured, on other streams ---------------------------------------------------------------------------------


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_serving_run(ffd, fmt):
    """A prompt is written to the byte cache and read back into 16-bit pages, where it becomes the shared prefix of a batch;
    every sequence then grows in the byte cache by one token per step, each step writing and attending."""
    g = gen(110)
    batch, kv, group, prompt, steps = 5, 2, 4, 333, 70
    cfg = ffd.Config(kv * group, kv)
    i32 = dict(dtype=torch.int32, device="cuda")
    ws = ffd.new_workspace_prefix(cfg, batch, 2, (prompt + BLK - 1) // BLK)

    def pool(pages):
        return [torch.zeros(pages, kv, BLK, D, dtype=torch.int8, device="cuda").view(DTYPE[fmt]) for _ in "kv"] + \
               [torch.zeros(pages, kv, BLK, device="cuda") for _ in "kv"]

    blocks = (prompt + BLK - 1) // BLK
    first = pool(blocks)
    new = [normal(g, prompt, kv, D).to(torch.bfloat16) for _ in "kv"]
    zero, n = torch.zeros(1, **i32), torch.tensor([prompt], **i32)
    ffd.ffd_write_kv_byte(cfg, *new, *first, None, n, row_start=zero, first_token=zero, max_blocks_per_seq=blocks, workspace=ws)
    caches = [torch.full((blocks, kv, BLK, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    ffd.ffd_read_kv_byte(cfg, *first, None, n, *caches, max_blocks_per_seq=blocks, workspace=ws)
    shared = []
    for x in new:
        code, scale = quantise(x, fmt)
        shared.append((code.float() * scale[..., None]).to(torch.bfloat16).double())
    own = pool(batch * 2)
    lens, table = torch.zeros(batch, **i32), torch.arange(blocks, **i32)
    kept = [[torch.zeros(0, kv, D, dtype=torch.float64, device="cuda") for _ in range(batch)] for _ in "kv"]
    out, lse = torch.zeros(batch, kv * group, D, device="cuda"), torch.zeros(batch, kv * group, device="cuda")
    for step in range(steps):
        rows = [normal(g, batch, kv, D).to(torch.bfloat16) for _ in "kv"]
        q = normal(g, batch, kv * group, D).to(torch.bfloat16)
        lens += 1
        ffd.ffd_write_kv_byte(cfg, *rows, *own, None, lens, max_blocks_per_seq=2, workspace=ws)
        ffd.ffd_decode_prefix_byte(cfg, q, *caches, table, n, *own, None, lens, out, lse=lse, max_prefix_blocks=blocks,
                                   max_blocks_per_seq=2, workspace=ws)
        for i in (0, 1):
            code, scale = quantise(rows[i], fmt)
            value = code.double() * scale.double()[..., None]
            kept[i] = [torch.cat([kept[i][b], value[b:b + 1]]) for b in range(batch)]
        if step % 9 == 0 or step == steps - 1:
            check(out, lse, q, [tuple(torch.cat([shared[i], kept[i][b]]) for i in (0, 1)) for b in range(batch)], fmt)
    assert ffd.ffd_read_device_status(ws) == 0
    # without the prefix the same cache serves ffd_decode_byte
    ffd.ffd_decode_byte(cfg, q, *own, None, lens, out, lse=lse, max_blocks_per_seq=2,
                        workspace=ffd.new_workspace_prefix(cfg, batch, 2))
    check(out, lse, q, [(kept[0][b], kept[1][b]) for b in range(batch)], fmt)


def test_results_do_not_depend_on_the_run_and_graphs_replay_new_lengths(ffd):
    g = gen(120)
    pre, c = Shared(g, 1000, 2), Cache(g, "int8", [130, 128, 70], 2)
    cfg = ffd.Config(8, 2)
    q = normal(g, 3, 8, D).to(torch.bfloat16)
    out1, lse1, ws = with_prefix(ffd, cfg, q, pre, c)
    for _ in range(3):
        out2, lse2, _ = with_prefix(ffd, cfg, q, pre, c, ws=ws)
        assert torch.equal(out1, out2) and torch.equal(lse1, lse2)
    out, lse = torch.zeros_like(out1), torch.zeros_like(lse1)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        ffd.ffd_decode_prefix_byte(cfg, q, *pre.pools, pre.table, pre.len, *c.byte, c.table, c.seq_lens, out, lse=lse,
                                   max_prefix_blocks=pre.most, max_blocks_per_seq=c.most, workspace=ws)
    torch.cuda.current_stream().wait_stream(side)
    graph.replay()
    assert torch.equal(out, out1) and torch.equal(lse, lse1)
    pre.len.fill_(77)
    c.seq_lens.copy_(torch.tensor([0, 65, 1]))
    graph.replay()
    values = [tuple(torch.cat([pre.values[i][:77], c.values[i][b][:n]]) for i in (0, 1)) for b, n in enumerate([0, 65, 1])]
    check(out, lse, q, values, "int8")


def test_calls_on_two_streams_with_their_own_workspaces(ffd):
    g = gen(130)
    jobs = []
    for i in range(2):
        pre, c = Shared(g, 2000 + 500 * i, 4), Cache(g, FORMATS[i], [300, 5, 129, 64], 4)
        q = normal(g, 4, 16, D).to(torch.bfloat16)
        cfg = ffd.Config(16, 4)
        jobs.append((pre, c, q, cfg, ffd.new_workspace_prefix(cfg, 4, c.most, pre.most), torch.cuda.Stream()))
    want = [with_prefix(ffd, cfg, q, pre, c)[:2] for pre, c, q, cfg, _, _ in jobs]
    torch.cuda.synchronize()
    got = []
    for _ in range(5):
        for pre, c, q, cfg, ws, s in jobs:
            with torch.cuda.stream(s):
                got.append(with_prefix(ffd, cfg, q, pre, c, ws=ws, stream=s)[:2])
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0]) and torch.equal(lse, want[i % 2][1])


def test_a_cache_beyond_32_bit_offsets(ffd):
    """Pages whose bytes lie behind the 4 GB mark of the pool."""
    g = gen(140)
    kv, pages = 8, 68000                                  # 68000 * 8 * 8192 B = 4.46 GB per pool
    k = torch.zeros(pages, kv, BLK, D, dtype=torch.int8, device="cuda")
    v, ks = torch.zeros_like(k), torch.zeros(pages, kv, BLK, device="cuda")
    vs = torch.zeros_like(ks)
    cfg = ffd.Config(8, 8)
    table = torch.tensor([[pages - 1, 3], [pages - 2, pages - 3]], dtype=torch.int32, device="cuda")
    lens, ws = torch.tensor([100, 70], dtype=torch.int32, device="cuda"), ffd.new_workspace_prefix(cfg, 2, 2)
    starts, zero = torch.tensor([0, 100], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    new = [normal(g, 170, kv, D).to(torch.bfloat16) for _ in "kv"]
    ffd.ffd_write_kv_byte(cfg, *new, k, v, ks, vs, table, lens, row_start=starts, first_token=zero, max_blocks_per_seq=2,
                          workspace=ws)
    q = normal(g, 2, 8, D).to(torch.bfloat16)
    out, lse = torch.zeros(2, 8, D, device="cuda"), torch.zeros(2, 8, device="cuda")
    ffd.ffd_decode_byte(cfg, q, k, v, ks, vs, table, lens, out, lse=lse, max_blocks_per_seq=2, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0
    values = []
    for lo, hi in ((0, 100), (100, 170)):
        pair = []
        for x in new:
            code, scale = quantise(x[lo:hi], "int8")
            pair.append(code.double() * scale.double()[..., None])
        values.append(tuple(pair))
    check(out, lse, q, values, "int8")


# ---- numbers that are not finite, large geometries, one workspace for many calls ----------------------------------------------

@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("fmt", FORMATS)
def test_a_query_that_is_not_finite_spoils_its_own_head_only(ffd, fmt, bad):
    g = gen(150)
    for lens in ([40, 3000, 64], [9000, 700, 1]):
        c = Cache(g, fmt, lens, 2)
        cfg = ffd.Config(12, 2)
        q = normal(g, 3, 12, D).to(torch.bfloat16)
        clean, clean_lse, ws = decode(ffd, cfg, q, c)
        spoilt = q.clone()
        spoilt[1, 7, 100] = bad
        out, lse, _ = decode(ffd, cfg, spoilt, c, ws=ws)
        assert out[1, 7].isnan().all() and lse[1, 7].isnan()
        out[1, 7], lse[1, 7] = clean[1, 7], clean_lse[1, 7]
        check(out, lse, q, list(zip(*c.values)), fmt)


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("fmt", ["bf16"] + FORMATS)
@pytest.mark.parametrize("batch,out_dtype", [(3, 0), (48, 0), (48, 1)])
def test_what_is_not_finite_beside_a_prefix_spoils_what_it_meets(ffd, fmt, batch, out_dtype, bad):
    g = gen(151)
    pre, c = Shared(g, 1500, 2), Cache(g, fmt, [90 + b for b in range(batch)], 2)
    cfg = ffd.Config(8, 2, out_dtype=out_dtype)
    q = normal(g, batch, 8, D).to(torch.bfloat16)
    clean, clean_lse, ws = with_prefix(ffd, cfg, q, pre, c)
    spoilt = q.clone()
    spoilt[1, 6, 3] = bad
    out, lse, _ = with_prefix(ffd, cfg, spoilt, pre, c, ws=ws)
    assert out[1, 6].isnan().all() and lse[1, 6].isnan()
    out[1, 6], lse[1, 6] = clean[1, 6], clean_lse[1, 6]
    check(out, lse, q, joined_values(pre, c), fmt, one_piece=batch * 4 > 128 and out_dtype == 0)
    # a NaN among the prefix's keys: every row of that KV head
    pre.pools[0][pre.table[4].item(), 1, 33, 9] = math.nan
    out, lse, _ = with_prefix(ffd, cfg, q, pre, c, ws=ws)
    assert out[:, 4:].isnan().all() and lse[:, 4:].isnan().all()
    out[:, 4:], lse[:, 4:] = clean[:, 4:], clean_lse[:, 4:]
    check(out, lse, q, joined_values(pre, c), fmt, one_piece=batch * 4 > 128 and out_dtype == 0)


@pytest.mark.parametrize("fmt", FORMATS)
def test_decode_of_many_sequences(ffd, fmt):
    """More sequences than a CTA has threads: a thread sums several, some of them empty."""
    g = gen(160)
    lens = [(37 * b) % 101 if b % 3 else 0 for b in range(1100)]
    c = Cache(g, fmt, lens, 1)
    q = normal(g, len(lens), 3, D).to(torch.bfloat16)
    out, lse, ws = decode(ffd, ffd.Config(3, 1), q, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, list(zip(*c.values)), fmt)


@pytest.mark.parametrize("heads,batch,prefix", [((160, 160), 2, 300), ((75, 75), 300, 200), ((2, 1), 700, 1000), ((150, 150), 3, 0)])
@pytest.mark.parametrize("out_dtype", [0, 1])
def test_prefix_of_many_heads_and_sequences(ffd, heads, batch, prefix, out_dtype):
    """As many (KV head, group of row tiles) pairs as SMs or more, and more sequences than threads."""
    g = gen(161)
    pre, c = Shared(g, prefix, heads[1]), Cache(g, "e4m3", [(29 * b) % 67 for b in range(batch)], heads[1])
    q = normal(g, batch, heads[0], D).to(torch.bfloat16)
    out, lse, ws = with_prefix(ffd, ffd.Config(*heads, out_dtype=out_dtype), q, pre, c)
    assert ffd.ffd_read_device_status(ws) == 0
    check(out, lse, q, joined_values(pre, c), c.fmt, one_piece=batch * (heads[0] // heads[1]) > 128 and out_dtype == 0)


def test_the_workspace_of_the_largest_call_serves_smaller_ones(ffd):
    """And nothing that a call left in it matters to the next: it is filled with NaN in between."""
    g = gen(162)
    cfg = ffd.Config(8, 2, out_dtype=0)
    ws = ffd.new_workspace_prefix(cfg, 70, 4, 40)
    for batch, prefix, own in ((70, 2500, 200), (33, 2500, 1), (32, 1200, 256), (31, 130, 64), (7, 2560, 100), (1, 2000, 30), (64, 0, 65)):
        ws[256 + 65536 * 4:].fill_(0xff)
        pre, c = Shared(g, prefix, 2), Cache(g, "int8", [own - b % 2 for b in range(batch)], 2)
        q = normal(g, batch, 8, D).to(torch.bfloat16)
        out, lse, _ = with_prefix(ffd, cfg, q, pre, c, ws=ws)
        assert ffd.ffd_read_device_status(ws) == 0
        check(out, lse, q, joined_values(pre, c), c.fmt, one_piece=batch * 4 > 128)
        out, lse, _ = decode(ffd, cfg, q, c, ws=ws)
        assert ffd.ffd_read_device_status(ws) == 0
        check(out, lse, q, list(zip(*c.values)), c.fmt)


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_captured_step_writes_its_token_and_attends_to_it(ffd, fmt):
    g = gen(163)
    c = Cache(g, fmt, [60, 120, 3], 2)          # six more tokens: the first sequence goes on to a page of its own
    c.table[0, 1] = next(p for p in range(c.pages) if p not in c.table.flatten().tolist())
    cfg = ffd.Config(8, 2)
    ws = ffd.new_workspace_prefix(cfg, 3, c.most)
    q, new = normal(g, 3, 8, D).to(torch.bfloat16), [normal(g, 3, 2, D).to(torch.bfloat16) for _ in "kv"]
    out, lse = torch.zeros(3, 8, D, device="cuda"), torch.zeros(3, 8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ffd.ffd_write_kv_byte(cfg, *new, *c.byte, c.table, c.seq_lens, max_blocks_per_seq=c.most, workspace=ws)
        ffd.ffd_decode_byte(cfg, q, *c.byte, c.table, c.seq_lens, out, lse=lse, max_blocks_per_seq=c.most, workspace=ws)
    values = [list(zip(*c.values))[b] for b in range(3)]
    for _ in range(6):
        c.seq_lens += 1
        for x in (q, *new):
            x.copy_(normal(g, *x.shape))
        graph.replay()
        for b in range(3):
            pair = []
            for x, old in zip(new, values[b]):
                code, scale = quantise(x[b], fmt)
                pair.append(torch.cat([old, (code.double() * scale.double()[:, None])[None]]))
            values[b] = tuple(pair)
        assert ffd.ffd_read_device_status(ws) == 0
        check(out, lse, q, values, fmt)
