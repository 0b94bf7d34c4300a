"""Queries of the largest finite magnitudes over the byte cache, against 64 bits.  The tolerances are those of
test_gpu_byte_prefix.py: they are relative to the head's largest element, so its size changes nothing."""
import pytest
import torch

from tests.test_gpu_byte_prefix import BLK, D, FORMATS, Cache, check, decode, ffd, gen, normal   # noqa: F401 (ffd: a fixture)

pytestmark = pytest.mark.gpu

SM = 2.0 ** -19


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("group", [3, 6])
@pytest.mark.parametrize("largest", [1.0, 1.5, 2.0 - 2.0 ** -7])     # times 2^127: the last is the largest bf16 number
@pytest.mark.parametrize("sign", [1, -1])
def test_queries_from_2_to_the_127(ffd, fmt, group, largest, sign):
    """Keys of about 2^-112 bring the logits back to the size of 1."""
    g = gen(170 + group)
    lens = [1, 64, 300]
    c = Cache(g, fmt, lens, 2)
    c.k_scale *= 2.0 ** -112
    c.values[0] = [k * 2.0 ** -112 for k in c.values[0]]       # exact: no scale becomes subnormal
    q = (2.0 ** 124 * normal(g, len(lens), 2 * group, D)).to(torch.bfloat16)
    q[:, ::2, 5] = sign * largest * 2.0 ** 127                  # every other head; the rest stay below 2^127
    assert q.isfinite().all() and c.k_scale[~c.k_scale.isnan()].min() >= 2.0 ** -126
    for out_dtype in (0, 1):
        out, lse, ws = decode(ffd, ffd.Config(2 * group, 2, sm_scale=SM, out_dtype=out_dtype), q, c)
        assert ffd.ffd_read_device_status(ws) == 0
        check(out, lse, q, list(zip(*c.values)), fmt, sm=SM)
