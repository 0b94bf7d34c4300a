"""A step in which no sequence has a new token."""
import pytest
import torch

from tests.test_gpu_byte_prefix import D, FORMATS, Cache, ffd, gen, raw   # noqa: F401 (ffd: a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
def test_no_rows_write_nothing(ffd, fmt):
    c = Cache(gen(180), fmt, [70, 0, 64], 2)
    before = [x.clone() for x in c.byte]
    ws = torch.zeros(256, dtype=torch.uint8, device="cuda")
    none = torch.zeros(0, 2, D, dtype=torch.bfloat16, device="cuda")
    start = torch.zeros(3, dtype=torch.int32, device="cuda")
    cfg = ffd.Config(4, 2)
    ffd.ffd_write_kv_byte(cfg, none, none, *c.byte, c.table, c.seq_lens, row_start=start, first_token=c.seq_lens.clone(),
                          max_blocks_per_seq=c.most, workspace=ws)
    assert ffd.ffd_read_device_status(ws) == 0
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(before, c.byte))
    with pytest.raises(ffd.FfdError):          # one row per sequence is what the other form means
        ffd.ffd_write_kv_byte(cfg, none, none, *c.byte, c.table, c.seq_lens, max_blocks_per_seq=c.most, workspace=ws)
