"""keep_paged_attention at the ends of its arguments' ranges, against the 64-bit oracle."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb
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


def check_signs(b, power, scale):
    g = torch.Generator().manual_seed(power)
    sign = lambda t: (torch.randint(0, 2, t.shape, generator=g) * 2 - 1).float().cuda()
    b.q.copy_(sign(b.q))
    if b.cache.k_scale is None:
        b.cache.k.copy_(sign(b.cache.k) * 2.0 ** power)
    else:
        b.cache.k.copy_(sign(b.cache.k).to(b.cache.k.dtype))
        b.cache.k_scale.fill_(2.0 ** power)
    out, lse = b.run(scale=scale)
    k, v = b.numbers()
    dh, end = b.q.shape[2], int(b.start[-1])
    want, wl, absum = (t[:end] for t in so.paged_attention(b.q.double().cpu().numpy(), k, v, b.start, b.total,
                                                           b.table.cpu().numpy(), 0, scale))
    # From 2^14 on a row's scores lie 4096 or more apart or are equal: the largest share the row, with equal weights.  Below, a
    # score is off by 2^-24 of its size three times (log2(e), its product with the scale, the product with the score), a
    # probability by twice that (its own and the norm's).  Then the rounded probability, the sum, the result; of the log-sum-exp
    # three roundings of the largest score's place, the sum with the logarithm, and two of ln 2.
    err = 3 * 2.0 ** -24 * dh * 2.0 ** power * 0.125 if power < 14 else 0.0
    half = torch.finfo(b.dtype).eps / 2
    o, l = out.double().cpu().numpy()[:end], lse.double().cpu().numpy()[:end]
    assert np.isfinite(o).all() and np.isfinite(l).all(), b.new
    assert (np.abs(o - want) <= (2 * err + 2.0 ** -8 + 2.0 ** -13) * absum + half * np.abs(want)).all(), b.new
    assert (np.abs(l - wl) <= 6 * 2.0 ** -24 * np.abs(wl) + err + 2.0 ** -13).all(), b.new


@pytest.mark.parametrize("dtype,fmt,dh", [("f32", "f32", 64), ("f32", "fp8", 80), ("bf16", "bf16", 64), ("bf16", "bf16", 128),
                                          ("bf16", "fp8", 128), ("bf16", "int8", 64), ("bf16", "bf16", 256)])
@pytest.mark.parametrize("power", [3, 14, 17, 18, 19, 21, 26, 31, 36, 60, 100, 116])
@pytest.mark.parametrize("scale", [0.125, -0.125])
def test_scores_of_any_finite_size(dtype, fmt, dh, power, scale):
    """Queries of ones and keys of 2^power, signs at random: scores are whole multiples of 2^power, so binary32 sums them exactly,
    tells different ones apart and keeps equal ones equal, and the largest of a row share it, however large they are.  Chunks
    (tiles of 128, 32 and 16 query rows) and single tokens."""
    for seqs in ([(70, 300), (200, 333), (1, 77), (3, 500)], [(12, 300), (12, 90)], [(7, 300), (1, 40)]):
        check_signs(Batch(seqs, 4, 2, dh, FORMATS[dtype], fmt, 16, seed=power), power, scale)


@pytest.mark.parametrize("dtype,fmt,dh", [("f32", "f32", 64), ("f32", "int8", 128), ("bf16", "bf16", 128), ("bf16", "fp8", 64),
                                          ("bf16", "bf16", 256)])
def test_what_the_order_of_sums_depends_on(dtype, fmt, dh):
    """Other page numbers: the same bits.  A wider table, padding rows, empty sequences: the same results."""
    b = Batch([(1, 900), (20, 333), (3, 3)], 4, 2, dh, FORMATS[dtype], fmt, 16, seed=2)
    want = b.check()
    pages = b.cache.k.shape[0]
    to = torch.randperm(pages, generator=torch.Generator().manual_seed(9)).cuda()
    moved = [None if t is None else torch.empty_like(t) for t in (b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale)]
    for t, m in zip((b.cache.k, b.cache.v, b.cache.k_scale, b.cache.v_scale), moved):
        if t is not None:
            (m.view(torch.uint8) if m.element_size() == 1 else m)[to] = t.view(torch.uint8) if t.element_size() == 1 else t
    old, b.cache, table = b.cache, kb.PagedCache(*moved), b.table
    b.table = torch.where(table < pages, to[table.clamp(max=pages - 1).long()].int(), table)
    got = b.run()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    b.cache = old
    b.table = torch.cat([table, torch.full((3, 5000), 1 << 30, dtype=torch.int32, device="cuda")], 1)
    b.check()
    b.table = torch.cat([b.table, b.table[:2]])
    b.total, b.start = b.total + [40, 0], np.concatenate([b.start, b.start[-1:], b.start[-1:]])
    b.q = torch.cat([b.q] + [b.q[:2]] * 100)
    b.check()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16")])
def test_the_most_sequences_of_a_call(dtype, fmt):
    r = np.random.default_rng(5)
    b = Batch([(int(r.integers(0, 3)), int(r.integers(0, 40))) for _ in range(kb.KEEP_PAGED_MAX_SEQS)], 2, 1, 64, FORMATS[dtype], fmt, 8)
    b.check()


@pytest.mark.parametrize("dtype,fmt,dh", [("f32", "f32", 16), ("bf16", "bf16", 128), ("bf16", "int8", 64), ("bf16", "fp8", 256)])
@pytest.mark.parametrize("hq,hkv", [(64, 1), (71, 1), (300, 2)])
def test_many_heads_share_one(dtype, fmt, dh, hq, hkv):
    """a token's rows fill several tiles, or end inside one"""
    b = Batch([(1, 300), (3, 3), (2, 1), (0, 9), (5, 77)], hq, hkv, dh, FORMATS[dtype], fmt, 20, seed=hq)
    b.check()
    b.check(window=30)
