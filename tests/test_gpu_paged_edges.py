"""keep_paged_attention at the ends of its arguments' ranges, against the 64-bit oracle."""
import pytest
import torch

from test_gpu_paged_attention import FORMATS, RAGGED, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt,dh", [("f32", "f32", 64), ("f32", "int8", 80), ("bf16", "bf16", 128), ("bf16", "fp8", 128),
                                          ("bf16", "int8", 64), ("bf16", "bf16", 256)])
@pytest.mark.parametrize("extra", [[], [(300, 7), (200, 900)]])
def test_windows_that_hide_nothing(dtype, fmt, dh, extra):
    """rows before the first token beside windows as long as the table, longer, and of the largest number: as without one"""
    b = Batch(RAGGED + extra, 4, 2, dh, FORMATS[dtype], fmt, 16, seed=dh)
    want = b.check()
    capacity = b.table.shape[1] * 16
    for window in (capacity - 1, capacity, 2 ** 31 - 1025, 2 ** 31 - 1):
        got = b.check(window=window)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
