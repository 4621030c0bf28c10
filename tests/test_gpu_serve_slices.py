"""Inputs and outputs of the serving calls as slices of the same wide rows."""
import pytest
import torch

from paper_2602_23592_amd import binding as kb
from test_gpu_paged_attention import FORMATS, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("out_first", [False, True])
@pytest.mark.parametrize("rows", [1, 5])
def test_rotation_into_other_columns(dtype, out_first, rows):
    """queries and keys of a fused row to columns beside them, behind or before"""
    hq, hkv, dh = 4, 2, 64
    g = torch.Generator().manual_seed(rows)
    buf = torch.randn(rows, 2 * (hq + hkv), dh, generator=g).to(dtype).cuda()
    before = buf.clone()
    i, o = (hq + hkv, 0) if out_first else (0, hq + hkv)
    parts = lambda t, at: (t[:, at:at + hq], t[:, at + hq:at + hq + hkv])
    pos = torch.arange(7, 7 + rows, dtype=torch.int32, device="cuda")
    freq = torch.from_numpy(kb.rope_frequencies(dh)[0]).cuda()
    want = kb.rope_rows(*(t.clone() for t in parts(before, i)), pos, freq)
    (q, k), (qo, ko) = parts(buf, i), parts(buf, o)
    kb.rope_rows(q, k, pos, freq, q_out=qo, k_out=ko)
    assert torch.equal(qo, want[0]) and torch.equal(ko, want[1])
    assert torch.equal(buf[:, i:i + hq + hkv], before[:, i:i + hq + hkv])


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "int8")])
def test_attention_into_other_columns(dtype, fmt):
    b = Batch([(33, 190), (2, 70)], 4, 2, 128, FORMATS[dtype], fmt, 10)
    want, _ = b.run()
    end = int(b.start[-1])
    args = (b.cache, torch.from_numpy(b.start).cuda(), torch.tensor(b.total, dtype=torch.int32, device="cuda"), b.table)
    for at, to in ((0, 4), (5, 1)):
        wide = torch.zeros(b.q.shape[0], 9, 128, dtype=FORMATS[dtype], device="cuda")
        wide[:, at:at + 4] = b.q
        kb.paged_attention(wide[:, at:at + 4], *args, out=wide[:, to:to + 4])
        assert torch.equal(wide[:end, to:to + 4], want[:end]) and torch.equal(wide[:, at:at + 4], b.q)
        with pytest.raises(kb.KeepError):
            kb.paged_attention(wide[:, at:at + 4], *args, out=wide[:, 3:7])
