"""A configuration is a plain value: copied, pickled, sent to another process or changed by another thread, every call uses the
fields that its own Config has at that moment.  No GPU."""
import copy
import ctypes
import dataclasses
import gc
import os
import pickle
import subprocess
import sys
import threading

import pytest
import torch

from paper_2609_00097_b200 import build, ffd

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build_library()
    return ffd.load_library()


def heads_of_a_call(cfg):
    """The query heads that a call with this configuration works with: the binding names the shape it wants."""
    with pytest.raises(ValueError, match="q: a contiguous BFloat16 tensor") as e:
        ffd.ffd_decode_byte(cfg, torch.zeros(3, 5, 7, dtype=torch.bfloat16), *[None] * 4, None, None, None,
                            max_blocks_per_seq=2, workspace=torch.zeros(512, dtype=torch.uint8))
    return int(str(e.value).split("[3, ")[1].split(",")[0])


def used(**kw):
    cfg = ffd.Config(kw.pop("num_q_heads", 32), kw.pop("num_kv_heads", 8), **kw)
    cfg.c(), cfg.address()
    assert heads_of_a_call(cfg) == cfg.num_q_heads
    return cfg


COPIES = {"copy": copy.copy, "deepcopy": copy.deepcopy, "pickle": lambda c: pickle.loads(pickle.dumps(c)),
          "replace": dataclasses.replace}


@pytest.mark.parametrize("how", COPIES)
@pytest.mark.parametrize("dropped", [False, True])
def test_a_copy_stands_by_itself(how, dropped):
    cfg = used(sm_scale=0.25)
    other = COPIES[how](cfg)
    assert other == cfg
    cfg.num_q_heads = 8
    if dropped:
        del cfg
    gc.collect()
    junk = [ffd.ffd_config(*range(7, 14), 7.0, 7) for _ in range(1000)]    # takes the place of what was freed
    assert heads_of_a_call(other) == 32 and other.c().num_q_heads == 32
    at = ffd.ffd_config.from_address(other.address())
    assert (at.num_q_heads, at.num_kv_heads, at.sm_scale) == (32, 8, 0.25)
    other.num_q_heads = 16
    assert heads_of_a_call(other) == 16
    if not dropped:
        assert heads_of_a_call(cfg) == 8
    del junk


def test_a_copy_carries_the_fields_only():
    cfg = used()
    names = {f.name for f in dataclasses.fields(cfg)}
    for other in (copy.copy(cfg), copy.deepcopy(cfg), pickle.loads(pickle.dumps(cfg))):
        assert set(vars(other)) == names


def test_a_used_configuration_serves_another_process(tmp_path):
    path = tmp_path / "cfg"
    path.write_bytes(pickle.dumps(used(num_q_heads=24)))
    code = f"""
import pickle, torch
from paper_2609_00097_b200 import ffd
cfg = pickle.load(open({str(path)!r}, "rb"))
try:
    ffd.ffd_decode_byte(cfg, torch.zeros(3, 5, 7, dtype=torch.bfloat16), *[None] * 4, None, None, None, max_blocks_per_seq=2,
                        workspace=torch.zeros(512, dtype=torch.uint8))
except ValueError as e:
    print(e)
"""
    got = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert got.returncode == 0, got
    assert "[3, 24, 128]" in got.stdout


def test_a_structure_that_was_handed_out_is_the_callers_own():
    cfg = used()
    held = cfg.c()
    held.num_q_heads = 7
    assert cfg.num_q_heads == 32 and cfg.c().num_q_heads == 32 and heads_of_a_call(cfg) == 32
    address = cfg.address()
    cfg.num_q_heads = 16
    assert held.num_q_heads == 7
    assert cfg.address() == address and ffd.ffd_config.from_address(address).num_q_heads == 16


def test_another_thread_may_change_a_configuration():
    """A call sees all the fields that one moment had, or another's; once the changes have ended, the last ones."""
    cfg, stop, wrong = used(), threading.Event(), []

    def change():
        while not stop.is_set():
            for n in (16, 24, 32):
                cfg.num_q_heads = n

    interval = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    threads = [threading.Thread(target=change) for _ in range(2)]
    try:
        for t in threads:
            t.start()
        for _ in range(3000):
            n = heads_of_a_call(cfg)
            if n not in (16, 24, 32):
                wrong.append(n)
    finally:
        stop.set()
        for t in threads:
            t.join()
        sys.setswitchinterval(interval)
    assert not wrong
    cfg.num_q_heads = 8
    assert heads_of_a_call(cfg) == 8 and cfg.c().num_q_heads == 8


@pytest.mark.parametrize("name", [f.name for f in dataclasses.fields(ffd.Config)])
def test_a_field_that_is_no_number_is_refused(name):
    cfg = ffd.Config(4, 2)
    for bad in (None, "8", 8.5, 1 << 40) if name != "sm_scale" else (None, "8"):
        setattr(cfg, name, bad)
        with pytest.raises(ValueError, match="cfg." + name):
            ffd.ffd_decode_byte(cfg, *[None] * 8, max_blocks_per_seq=2, workspace=torch.zeros(512, dtype=torch.uint8))


def test_what_is_no_configuration_is_refused():
    for bad in (None, 0, 4096, object()):
        with pytest.raises(AttributeError):
            ffd.ffd_decode_byte(bad, *[None] * 8, max_blocks_per_seq=2, workspace=torch.zeros(512, dtype=torch.uint8))


def test_every_field_reaches_the_library(lib):
    """Through the binding, the structure has what ffd_config says, field by field."""
    cfg = ffd.Config(6, 2, 128, 64, 4, 2, 3, 0.5, 0)
    assert [getattr(cfg.c(), n) for n, _ in ffd.ffd_config._fields_] == [6, 2, 128, 64, 4, 2, 3, 0.5, 0]
    assert [n for n, _ in ffd.ffd_config._fields_] == [f.name for f in dataclasses.fields(cfg)]
    assert ctypes.sizeof(ffd.ffd_config) == 36
