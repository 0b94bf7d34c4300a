"""Host-side checks of the functions on a chunk of new tokens: refusals before any launch, the workspace's size, the binding's own
checks.  No GPU."""
import ctypes

import pytest
import torch

from paper_2609_00097_b200 import build, ffd

FAKE, ODD = 0x10000, 0x10008      # aligned / misaligned addresses that no call may dereference
NULL, SHAPE, UNSUPPORTED, ALIGN, WORKSPACE = 1, 2, 3, 4, 5
ROWS = dict(row_start=FAKE, first_token=FAKE, seq_lens=FAKE)
END = dict(workspace=FAKE, workspace_bytes=1 << 30, stream=None)
CALLS = {
    "ffd_rotate_write_kv": dict(rotation="rotation", q=FAKE, q_stride=4096, k_new=FAKE, v_new=FAKE, kv_stride=1024, num_rows=4,
                                positions=FAKE, q_out=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=None, **ROWS, batch=2,
                                max_blocks=16, num_pages=32, **END),
    "ffd_attend_chunk": dict(q=FAKE, k_cache=FAKE, v_cache=FAKE, block_table=None, **ROWS, num_rows=4, batch=2, max_blocks=16,
                             num_pages=32, out=FAKE, lse=FAKE, **END),
    "ffd_weigh_kv": dict(q=FAKE, lse=FAKE, k_cache=FAKE, weight=FAKE, add=1, block_table=None, **ROWS, num_rows=4, batch=2,
                         max_blocks=16, num_pages=32, **END),
    "ffd_evict_kv": dict(k_cache=FAKE, v_cache=FAKE, weight=FAKE, block_table=None, seq_lens=FAKE, batch=2, max_blocks=16, num_pages=32,
                         budget=200, n_sink=4, n_local=64, k_out=FAKE, v_out=FAKE, weight_out=FAKE, out_table=None,
                         max_out_blocks=4, num_out_pages=8, out_lens=FAKE, kept=FAKE, **END),
}
OPTIONAL = {("ffd_attend_chunk", "lse"), ("ffd_rotate_write_kv", "positions"), ("ffd_evict_kv", "weight_out")}


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return ffd.load_library()


def config(**kw):
    return ffd.Config(kw.pop("num_q_heads", 32), kw.pop("num_kv_heads", 8), **kw)


def rotation(cos_sin=FAKE, num_positions=100, rotary_dim=128, interleaved=0, q_norm=FAKE, k_norm=FAKE, eps=1e-6):
    return ffd.ffd_rotation(cos_sin, num_positions, rotary_dim, interleaved, q_norm, k_norm, eps)


def call(lib, name, cfg=None, turn=None, **changed):
    args = {**CALLS[name], **changed}
    c = (cfg or config()).c()
    values = [ctypes.byref(turn or rotation()) if v == "rotation" else v for v in args.values()]
    return getattr(lib, name)(ctypes.byref(c), *values)


def cases():
    for name, args in CALLS.items():
        for key, value in args.items():
            if value == FAKE and (name, key) not in OPTIONAL:
                yield name, {key: None}, NULL
            if value == FAKE or key in ("block_table", "out_table"):
                yield name, {key: ODD}, ALIGN
        for key in ("batch", "max_blocks", "num_pages"):
            yield name, {key: 0}, SHAPE
            yield name, {key: -3}, SHAPE
        yield name, {"batch": 65536}, SHAPE
        yield name, {"batch": 8192}, SHAPE            # batch * KV heads = 65536
        yield name, {"max_blocks": 1 << 26}, SHAPE    # more tokens than an int32 counts
        yield name, {"num_pages": 1 << 22}, SHAPE     # 2^31 rows: beyond a TMA coordinate
        yield name, {"workspace_bytes": 255}, WORKSPACE
        if "num_rows" in args:
            yield name, {"num_rows": 0}, SHAPE
            yield name, {"num_rows": -1}, SHAPE
            yield name, {"row_start": None, "first_token": None}, SHAPE       # 4 rows for 2 sequences
    yield "ffd_rotate_write_kv", {"rotation": None}, NULL
    for key, width in (("q_stride", 4096), ("kv_stride", 1024)):
        yield "ffd_rotate_write_kv", {key: width - 8}, SHAPE                  # rows that overlap
        yield "ffd_rotate_write_kv", {key: width + 4}, SHAPE                  # rows off the 16-byte grid
    yield "ffd_attend_chunk", {"workspace_bytes": 1 << 20}, WORKSPACE
    for add in (2, -1):
        yield "ffd_weigh_kv", {"add": add}, UNSUPPORTED
    for changed in ({"budget": 0}, {"budget": -5}, {"n_sink": -1}, {"n_local": -1}, {"n_sink": 137}, {"n_local": 197},
                    {"max_out_blocks": 0}, {"num_out_pages": 0}, {"num_out_pages": 1 << 22},
                    {"n_sink": 2147483647, "n_local": 2147483647}):
        yield "ffd_evict_kv", changed, SHAPE


@pytest.mark.parametrize("name,changed,status", list(cases()))
def test_bad_arguments_are_refused_before_any_launch(lib, name, changed, status):
    assert call(lib, name, **changed) == status


@pytest.mark.parametrize("changed,status", [
    (dict(cos_sin=None), NULL), (dict(cos_sin=ODD), ALIGN), (dict(q_norm=ODD), ALIGN), (dict(k_norm=ODD), ALIGN),
    (dict(num_positions=0), SHAPE), (dict(num_positions=-1), SHAPE), (dict(rotary_dim=8), UNSUPPORTED), (dict(rotary_dim=-16), UNSUPPORTED),
    (dict(rotary_dim=120), UNSUPPORTED), (dict(rotary_dim=144), UNSUPPORTED), (dict(interleaved=2), UNSUPPORTED),
    (dict(eps=-1e-6), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(eps=float("inf")), SHAPE)])
def test_bad_rotations_are_refused(lib, changed, status):
    assert call(lib, "ffd_rotate_write_kv", turn=rotation(**changed)) == status


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("field,value,status", [
    ("head_dim", 64, UNSUPPORTED), ("block_tokens", 32, UNSUPPORTED), ("num_kv_heads", 5, SHAPE), ("num_kv_heads", 0, SHAPE),
    ("num_q_heads", 72, UNSUPPORTED), ("out_dtype", 2, UNSUPPORTED), ("sm_scale", -1.0, SHAPE),
    ("sm_scale", float("nan"), SHAPE), ("sm_scale", float("inf"), SHAPE)])
def test_bad_configurations_are_refused(lib, name, field, value, status):
    cfg = config()
    setattr(cfg, field, value)
    assert call(lib, name, cfg) == status
    values = [ctypes.byref(rotation()) if v == "rotation" else v for v in CALLS[name].values()]
    assert getattr(lib, name)(None, *values) == NULL


def test_workspace_size(lib):
    size = ffd.ffd_workspace_bytes_chunk(config(), 4, 100, 64)
    assert size % 256 == 0 and size >= 256 + 65536 * 4       # what ffd_workspace_init writes
    for group in range(1, 9):                                # one size for every geometry
        assert ffd.ffd_workspace_bytes_chunk(ffd.Config(2 * group, 2), 300, 1 << 20, 7) == size
    for bad in ((0, 1, 64), (4, 0, 64), (4, 1, 0), (4, 1, 1 << 26)):
        with pytest.raises(ffd.FfdError) as e:
            ffd.ffd_workspace_bytes_chunk(config(), *bad)
        assert e.value.status == SHAPE
    assert call(lib, "ffd_attend_chunk", workspace_bytes=size - 1) == WORKSPACE


def z(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=torch.float32).to(dtype)


def test_binding_checks_what_the_library_cannot_see(lib):
    """Everything is looked at before the workspace's device is found to be no GPU: a call in which all else fits gets there."""
    cfg = ffd.Config(4, 2, out_dtype=0)
    bf, i32 = torch.bfloat16, torch.int32
    half = dict(k_cache=z(4, 2, 64, 128, dtype=bf), v_cache=z(4, 2, 64, 128, dtype=bf))
    own = dict(block_table=z(3, 2, dtype=i32), seq_lens=z(3, dtype=i32), max_blocks_per_seq=2)
    rows = dict(row_start=z(3, dtype=i32), first_token=z(3, dtype=i32))
    end = dict(workspace=z(512, dtype=torch.uint8))
    calls = {
        ffd.ffd_rotate_write_kv: dict(q=z(9, 4, 128, dtype=bf), k_new=z(9, 2, 128, dtype=bf), v_new=z(9, 2, 128, dtype=bf),
                                      q_out=z(9, 4, 128, dtype=bf), **half, **own, cos_sin=z(7, 2, 32), q_norm=z(128, dtype=bf),
                                      k_norm=z(128, dtype=bf), positions=z(9, dtype=i32), **rows, **end),
        ffd.ffd_attend_chunk: dict(q=z(9, 4, 128, dtype=bf), **half, **own, out=z(9, 4, 128, dtype=bf), lse=z(9, 4), **rows, **end),
        ffd.ffd_weigh_kv: dict(q=z(9, 4, 128, dtype=bf), lse=z(9, 4), k_cache=half["k_cache"], weight=z(4, 2, 64), **own, **rows, **end),
        ffd.ffd_evict_kv: dict(**half, weight=z(4, 2, 64), **own, k_out=z(5, 2, 64, 128, dtype=bf), v_out=z(5, 2, 64, 128, dtype=bf),
                               weight_out=z(5, 2, 64), out_table=z(3, 1, dtype=i32), out_lens=z(3, dtype=i32), kept=z(3, 2, 50, dtype=i32),
                               max_out_blocks=1, **end),
    }
    wrong = {
        "q": [z(9, 4, 128), z(9, 2, 128, dtype=bf), z(9, 128, 4, dtype=bf).transpose(1, 2), z(9, 512, dtype=bf), None],
        "k_new": [z(9, 2, 128), z(8, 2, 128, dtype=bf), z(9, 4, 128, dtype=bf)[:, ::2]],
        "v_new": [z(8, 2, 128, dtype=bf), z(9, 4, 128, dtype=bf)[:, :2]],       # rows other than the keys' ones
        "q_out": [z(9, 4, 128), z(9, 8, 128, dtype=bf)[:, :4]],
        "out": [z(9, 4, 128), z(8, 4, 128, dtype=bf)],
        "lse": [z(4, 9), z(9, 4, dtype=bf), z(36)],
        "k_cache": [z(4, 2, 64, 128), z(4, 1, 64, 128, dtype=bf), z(4, 2, 64, 64, dtype=bf)],
        "v_cache": [z(3, 2, 64, 128, dtype=bf)],
        "weight": [z(5, 2, 64), z(4, 64, 2), z(4, 2, 64, dtype=bf)],
        "block_table": [z(3, 3, dtype=i32), torch.zeros(3, 2, dtype=torch.int64), z(3, 4, dtype=i32)[:, ::2]],
        "first_token": [z(2, dtype=i32)],
        "row_start": [z(4, dtype=i32), torch.zeros(3, dtype=torch.int64)],
        "positions": [z(8, dtype=i32), torch.zeros(9, dtype=torch.int64)],
        "cos_sin": [z(7, 1, 32), z(7, 64), z(7, 2, 32, dtype=bf), z(7, 2, 256), z(7, 2, 64)[..., ::2]],
        "q_norm": [z(64, dtype=bf), z(128)],
        "k_norm": [z(256, dtype=bf)[::2]],
        "k_out": [z(5, 2, 64, 128), z(5, 1, 64, 128, dtype=bf)],
        "v_out": [z(4, 2, 64, 128, dtype=bf)],
        "weight_out": [z(4, 2, 64)],
        "out_table": [z(3, 2, dtype=i32)],
        "out_lens": [z(4, dtype=i32)],
        "kept": [z(3, 1, 50, dtype=i32), torch.zeros(3, 2, 50, dtype=torch.int64), z(3, 100, dtype=i32)],
        "workspace": [z(512, 2, dtype=torch.uint8)[:, 0], None],
    }
    seen = set()
    for function, good in calls.items():
        with pytest.raises(ValueError, match="workspace: a CUDA tensor"):
            function(cfg, **good)
        for name in wrong.keys() & good.keys():
            seen.add(name)
            for value in wrong[name]:
                with pytest.raises(ValueError, match=name):
                    function(cfg, **{**good, name: value})
    assert seen == set(wrong)
    # what may be left out, and rows of a fused projection
    fused = z(9, 8 * 128, dtype=bf)
    with pytest.raises(ValueError, match="workspace: a CUDA tensor"):
        ffd.ffd_rotate_write_kv(cfg, **{**calls[ffd.ffd_rotate_write_kv], "q": fused[:, :512].view(9, 4, 128),
                                        "k_new": fused[:, 512:768].view(9, 2, 128), "v_new": fused[:, 768:].view(9, 2, 128),
                                        "cos_sin": None, "q_norm": None, "k_norm": None, "positions": None, "block_table": None})
    with pytest.raises(ValueError, match="workspace: a CUDA tensor"):
        ffd.ffd_evict_kv(cfg, **{**calls[ffd.ffd_evict_kv], "weight_out": None, "out_table": None, "block_table": None})
