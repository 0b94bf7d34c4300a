"""Host-side checks of the byte cache's and the shared prefix's entry points: refusals before any launch, workspace sizes,
and the binding's own checks.  No GPU."""
import ctypes

import pytest
import torch

from paper_2609_00097_b200 import build, ffd

FAKE, ODD = 0x1000, 0x1008      # aligned / misaligned addresses that no call may dereference


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return ffd.load_library()


def config(**kw):
    return ffd.Config(kw.pop("num_q_heads", 32), kw.pop("num_kv_heads", 8), **kw)


CALLS = {
    "ffd_write_kv_byte": dict(format=0, k_new=FAKE, v_new=FAKE, row_stride=1024, num_rows=4, row_start=FAKE, k_byte=FAKE,
                              v_byte=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=None, first_token=FAKE, seq_lens=FAKE,
                              batch=2, max_blocks=16, num_pages=32, workspace=FAKE, workspace_bytes=1 << 30, stream=None),
    "ffd_read_kv_byte": dict(format=0, k_byte=FAKE, v_byte=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=None,
                             first_token=None, seq_lens=FAKE, batch=2, max_blocks=16, num_pages=32, k_cache=FAKE,
                             v_cache=FAKE, cache_table=None, num_cache_pages=32, workspace=FAKE, workspace_bytes=1 << 30,
                             stream=None),
    "ffd_decode_byte": dict(format=0, q=FAKE, k_byte=FAKE, v_byte=FAKE, k_scale=FAKE, v_scale=FAKE, block_table=None,
                            seq_lens=FAKE, batch=2, max_blocks=16, num_pages=32, out=FAKE, lse=FAKE, workspace=FAKE,
                            workspace_bytes=1 << 30, stream=None),
    "ffd_decode_prefix": dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, prefix_table=FAKE, prefix_len=FAKE, max_prefix_blocks=8,
                              block_table=None, seq_lens=FAKE, batch=2, max_blocks=16, num_pages=32, out=FAKE, lse=FAKE,
                              workspace=FAKE, workspace_bytes=1 << 30, stream=None),
    "ffd_decode_prefix_byte": dict(format=1, q=FAKE, k_cache=FAKE, v_cache=FAKE, prefix_table=FAKE, prefix_len=FAKE,
                                   max_prefix_blocks=8, num_prefix_pages=8, k_byte=FAKE, v_byte=FAKE, k_scale=FAKE,
                                   v_scale=FAKE, block_table=None, seq_lens=FAKE, batch=2, max_blocks=16, num_pages=32,
                                   out=FAKE, lse=FAKE, workspace=FAKE, workspace_bytes=1 << 30, stream=None),
}
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
OPTIONAL = {"block_table", "cache_table", "lse", "stream"}


def call(lib, name, cfg=None, **changed):
    args = {**CALLS[name], **changed}
    c = (cfg or config()).c()
    return getattr(lib, name)(ctypes.byref(c), *args.values())


def cases():
    for name, args in CALLS.items():
        for key, value in args.items():
            if value == FAKE and key not in OPTIONAL:
                yield name, {key: None}, NULL
            if value == FAKE:
                yield name, {key: ODD}, ALIGN
        if "format" in args:
            yield name, {"format": 2}, UNSUPPORTED
            yield name, {"format": -1}, UNSUPPORTED
        for key in ("batch", "max_blocks", "num_pages"):
            yield name, {key: 0}, SHAPE
            yield name, {key: -3}, SHAPE
        yield name, {"batch": 65536}, SHAPE
        yield name, {"batch": 8192}, SHAPE            # batch * KV heads = 65536
        yield name, {"max_blocks": 1 << 26}, SHAPE    # more tokens than an int32 counts
        yield name, {"workspace_bytes": 255}, WORKSPACE
    for key in ("row_start", "first_token"):
        yield "ffd_write_kv_byte", {key: None}, NULL                                        # one without the other
    yield "ffd_write_kv_byte", {"row_start": None, "first_token": None}, SHAPE              # 4 rows for 2 sequences
    yield "ffd_write_kv_byte", {"num_rows": 0}, SHAPE
    yield "ffd_write_kv_byte", {"row_stride": 1016}, SHAPE                                  # rows that overlap
    yield "ffd_write_kv_byte", {"row_stride": 1028}, SHAPE                                  # rows off the 16-byte grid
    yield "ffd_read_kv_byte", {"num_cache_pages": 0}, SHAPE
    for name in ("ffd_decode_prefix", "ffd_decode_prefix_byte"):
        yield name, {"max_prefix_blocks": 0}, SHAPE
        yield name, {"max_prefix_blocks": -1}, SHAPE
        yield name, {"max_prefix_blocks": 1 << 26}, SHAPE
        yield name, {"workspace_bytes": 1 << 18}, WORKSPACE
    yield "ffd_decode_prefix", {"num_pages": 1 << 22}, SHAPE          # 2^31 rows: beyond a TMA coordinate
    yield "ffd_decode_prefix_byte", {"num_prefix_pages": 1 << 22}, SHAPE
    yield "ffd_decode_prefix_byte", {"num_prefix_pages": 0}, SHAPE


@pytest.mark.parametrize("name,changed,status", list(cases()))
def test_bad_arguments_are_refused_before_any_launch(lib, name, changed, status):
    assert call(lib, name, **changed) == status


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("field,value,status", [
    ("head_dim", 64, UNSUPPORTED), ("block_tokens", 32, UNSUPPORTED), ("num_kv_heads", 5, SHAPE), ("num_kv_heads", 0, SHAPE),
    ("num_q_heads", 72, UNSUPPORTED), ("out_dtype", 2, UNSUPPORTED), ("sm_scale", -1.0, SHAPE),
    ("sm_scale", float("nan"), SHAPE), ("sm_scale", float("inf"), SHAPE)])
def test_bad_configurations_are_refused(lib, name, field, value, status):
    cfg = config()
    setattr(cfg, field, value)
    assert call(lib, name, cfg) == status
    assert getattr(lib, name)(None, *CALLS[name].values()) == NULL


def test_workspace_sizes():
    cfg = config()
    plain = ffd.ffd_workspace_bytes_prefix(cfg, 4, 64)
    assert plain % 256 == 0 and plain >= 256 + 65536 * 4       # what ffd_workspace_init writes
    with_prefix = ffd.ffd_workspace_bytes_prefix(cfg, 4, 64, 512)
    assert with_prefix > plain
    assert ffd.ffd_workspace_bytes_prefix(cfg, 64, 64, 512) > with_prefix
    for group in range(1, 9):                                  # every group size is served
        assert ffd.ffd_workspace_bytes_prefix(ffd.Config(2 * group, 2), 3, 5, 7) > 0
    for bad in ((0, 64, 0), (4, 0, 0), (4, 64, -1), (4, 64, 1 << 26)):
        with pytest.raises(ffd.FfdError) as e:
            ffd.ffd_workspace_bytes_prefix(cfg, *bad)
        assert e.value.status == SHAPE
    # thumbnail settings are not looked at
    cfg.quant_bits, cfg.n_sink_blocks, cfg.n_local_blocks = 3, 0, 0
    assert ffd.ffd_workspace_bytes_prefix(cfg, 4, 64) == plain


def test_a_workspace_for_the_largest_call_serves_all_smaller_ones(lib):
    for heads in ((32, 8), (8, 1), (16, 16), (300, 300), (7, 7)):
        cfg = ffd.Config(*heads)
        for axis, rest in ((0, (5, 70)), (1, (33, 70)), (2, (33, 5)), (2, (3, 900)), (0, (900, 3)), (0, (5, 0))):
            last = 0
            for x in list(range(1, 300, 3)) + [400, 1000, 2000]:
                if axis == 0 and x * heads[1] >= 65536:
                    break
                args = list(rest)
                args.insert(axis, x if axis != 2 else x - 1)
                now = ffd.ffd_workspace_bytes_prefix(cfg, *args)
                assert now >= last, (heads, args)
                last = now


def test_a_workspace_one_byte_short_is_refused(lib):
    need = ffd.ffd_workspace_bytes_prefix(config(), 2, 16)
    assert call(lib, "ffd_decode_byte", workspace_bytes=need - 1) == WORKSPACE
    need = ffd.ffd_workspace_bytes_prefix(config(), 2, 16, 8)
    assert call(lib, "ffd_decode_prefix_byte", workspace_bytes=need - 1) == WORKSPACE


def test_binding_checks_what_the_library_cannot_see(lib):
    """Everything is looked at before the workspace's device is found to be no GPU: a call in which all else fits gets there."""
    cfg = ffd.Config(4, 2, out_dtype=0)
    bf, i32, i8 = torch.bfloat16, torch.int32, torch.int8

    def z(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=torch.float32).to(dtype)

    cache = dict(k_byte=z(6, 2, 64, 128, dtype=i8), v_byte=z(6, 2, 64, 128, dtype=i8), k_scale=z(6, 2, 64), v_scale=z(6, 2, 64))
    own = dict(block_table=z(3, 2, dtype=i32), seq_lens=z(3, dtype=i32), max_blocks_per_seq=2)
    half = dict(k_cache=z(4, 2, 64, 128, dtype=bf), v_cache=z(4, 2, 64, 128, dtype=bf))
    results = dict(q=z(3, 4, 128, dtype=bf), out=z(3, 4, 128, dtype=bf), lse=z(3, 4))
    prefix = dict(prefix_table=z(5, dtype=i32), prefix_len=z(1, dtype=i32), max_prefix_blocks=5)
    end = dict(workspace=z(512, dtype=torch.uint8))
    calls = {
        ffd.ffd_write_kv_byte: dict(k_new=z(9, 2, 128, dtype=bf), v_new=z(9, 2, 128, dtype=bf), **cache, **own,
                                    row_start=z(3, dtype=i32), first_token=z(3, dtype=i32), **end),
        ffd.ffd_read_kv_byte: dict(**cache, **own, **half, cache_table=z(3, 2, dtype=i32), first_token=z(3, dtype=i32), **end),
        ffd.ffd_decode_byte: dict(**results, **cache, **own, **end),
        ffd.ffd_decode_prefix: dict(**results, **half, **prefix, **own, **end),
        ffd.ffd_decode_prefix_byte: dict(**results, **half, **prefix, **cache, **own, **end),
    }
    wrong = {
        "q": [z(3, 4, 128), z(3, 2, 128, dtype=bf), z(3, 128, 4, dtype=bf).transpose(1, 2), z(4, 128, dtype=bf), None],
        "out": [z(3, 4, 128), z(2, 4, 128, dtype=bf)],
        "lse": [z(4, 4), z(3, 4, dtype=bf), z(12)],
        "k_byte": [z(6, 2, 64, 128, dtype=torch.uint8), z(6, 64, 2, 128, dtype=i8), z(6, 2, 64, 64, dtype=i8), z(6, dtype=i8)],
        "v_byte": [z(5, 2, 64, 128, dtype=i8), z(6, 2, 64, 128, dtype=torch.float8_e4m3fn), z(6, 2, 64, 256, dtype=i8)[..., ::2]],
        "k_scale": [z(6, 2, 64, dtype=bf), z(6, 64, 2), z(6, 2)],
        "v_scale": [z(7, 2, 64), torch.zeros(6, 2, 64, dtype=torch.float64)],
        "k_cache": [z(4, 2, 64, 128), z(4, 1, 64, 128, dtype=bf)],
        "v_cache": [z(3, 2, 64, 128, dtype=bf)],
        "block_table": [z(3, 3, dtype=i32), torch.zeros(3, 2, dtype=torch.int64), z(3, 4, dtype=i32)[:, ::2]],
        "cache_table": [z(3, 1, dtype=i32)],
        "first_token": [z(2, dtype=i32)],
        "row_start": [z(4, dtype=i32)],
        "prefix_table": [z(4, dtype=i32), None],
        "prefix_len": [z(2, dtype=i32), torch.zeros(1, dtype=torch.int64)],
        "k_new": [z(9, 2, 128), z(9, 128, 2, dtype=bf).transpose(1, 2), z(9, 4, 128, dtype=bf)[:, ::2], z(9, 256, dtype=bf)],
        "v_new": [z(8, 2, 128, dtype=bf), z(9, 4, 128, dtype=bf)[:, :2]],
        "workspace": [z(512, 2, dtype=torch.uint8)[:, 0], None],
    }
    for function, good in calls.items():
        with pytest.raises(ValueError, match="workspace: a CUDA tensor"):
            function(cfg, **good)
        for name in wrong.keys() & good.keys():
            for value in wrong[name]:
                with pytest.raises(ValueError, match=name):
                    function(cfg, **{**good, name: value})
    with pytest.raises(ValueError, match="seq_lens|block_table"):
        ffd.ffd_decode_byte(cfg, **{**calls[ffd.ffd_decode_byte], "seq_lens": z(2, dtype=i32)})
    with pytest.raises(ValueError, match="32 bits"):
        ffd.ffd_decode_byte(cfg, **{**calls[ffd.ffd_decode_byte], "max_blocks_per_seq": 1 << 40})
    # rows of a fused projection, and tables that are left out, are fine
    fused = z(9, 3 * 256, dtype=bf)
    with pytest.raises(ValueError, match="workspace: a CUDA tensor"):
        ffd.ffd_write_kv_byte(cfg, **{**calls[ffd.ffd_write_kv_byte], "k_new": fused[:, 256:512].view(9, 2, 128),
                                      "v_new": fused[:, 512:].view(9, 2, 128), "block_table": None})


def test_a_configuration_can_be_changed_between_calls(lib):
    cfg = config()
    first = ffd.ffd_workspace_bytes_prefix(cfg, 4, 64)
    address = cfg.address()
    assert address == cfg.address()
    cfg.num_q_heads = 8
    assert cfg.c().num_q_heads == 8
    assert ffd.ffd_workspace_bytes_prefix(cfg, 4, 64) < first
    assert cfg == ffd.Config(8, 8)
