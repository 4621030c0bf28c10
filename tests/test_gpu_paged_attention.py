"""keep_paged_attention against the 64-bit oracle: types, formats, head layouts, lengths from nothing to long, windows, pages that
end inside a tile, strides, values that are not finite, rows of no sequence, and that equal calls give equal bits."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb
from test_gpu_paged_cache import FORMATS, as_numbers

pytestmark = pytest.mark.gpu


class Batch:
    """Sequences of (new tokens, tokens in all) over pages in random order, filled through keep_cache_write."""

    def __init__(self, seqs, hq, hkv, dh, dtype, fmt, size, seed=0, tail=2, tokens_first=False):
        g = torch.Generator().manual_seed(seed)
        self.new, self.total = [n for n, _ in seqs], [t for _, t in seqs]
        per = [-(-t // size) for t in self.total]
        pages, width = sum(per) + 2, max(per + [1])
        order = torch.randperm(pages, generator=g).tolist()
        table = np.full((len(seqs), width), 1 << 30, np.int32)       # (what is not read may hold anything)
        for s, p in enumerate(per):
            for i in range(p):
                table[s, i] = order.pop()
        self.table = torch.from_numpy(table).cuda()
        self.start = np.concatenate([[0], np.cumsum(self.new)]).astype(np.int32)
        rows = int(self.start[-1]) + tail
        self.q = torch.randn(rows, hq, dh, generator=g).to(dtype).cuda()
        shape = (pages, size, hkv, dh) if tokens_first else (pages, hkv, size, dh)
        k, v = (torch.zeros(shape, device="cuda").to(FORMATS[fmt]) for _ in range(2))
        for t in (k, v):                                              # what no token was written to is NaN, or a wild code
            (t.view(torch.uint8).fill_(0x7f) if t.element_size() == 1 else t.fill_(float("nan")))
        if tokens_first:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        ks, vs = (torch.full((pages, hkv, size), float("nan"), device="cuda") if k.element_size() == 1 else None for _ in range(2))
        self.cache = kb.PagedCache(k, v, ks, vs)
        for s, t in enumerate(self.total):
            if t:
                pos = np.arange(t)
                slots = torch.from_numpy((table[s, pos // size] * size + pos % size).astype(np.int32)).cuda()
                self.cache.write(torch.randn(t, hkv, dh, generator=g).to(dtype).cuda(),
                                 torch.randn(t, hkv, dh, generator=g).to(dtype).cuda(), slots)
        self.size, self.dtype, self.fmt = size, dtype, fmt

    def numbers(self):
        r = []
        for t, s in ((self.cache.k, self.cache.k_scale), (self.cache.v, self.cache.v_scale)):
            x = as_numbers(t).astype(np.float64)
            r.append(x if s is None else x * s.double().cpu().numpy()[..., None])
        return r

    def run(self, **kw):
        out, lse = torch.full_like(self.q, 5.0), torch.full(self.q.shape[:2], 5.0, device="cuda")
        kb.paged_attention(self.q, self.cache, torch.from_numpy(self.start).cuda(),
                           torch.tensor(self.total, dtype=torch.int32, device="cuda"), self.table, out=out, lse=lse, **kw)
        torch.cuda.synchronize()
        return out, lse

    def check(self, **kw):
        out, lse = self.run(**kw)
        end = int(self.start[-1])
        assert (out[end:] == 5).all() and (lse[end:] == 5).all()
        k, v = self.numbers()
        q = self.q.double().cpu().numpy()
        want, wl, absum = so.paged_attention(q, k, v, self.start, self.total, self.table.cpu().numpy(), kw.get("window", 0),
                                             kw.get("scale") or None)
        o, l = out.double().cpu().numpy()[:end], lse.double().cpu().numpy()[:end]
        want, wl, absum = want[:end], wl[:end], absum[:end]
        dh, n = q.shape[2], max(self.total + [1])
        # A score is off by ds: dh products and sums of binary32 (2^-24 each, of sums of |q k| <= |q| |k|), the scale, the
        # 8-bit scale and the exponent's argument a few more.  A probability is off by 2 ds (its own and the norm's), 2^-22 of
        # the exponential; n of them are added (2^-24 each).
        scale = abs(kw.get("scale") or dh ** -0.5)
        qk = np.linalg.norm(q[:end], axis=-1).max(initial=0) * np.sqrt(np.nanmax(np.nansum(k * k, -1), initial=0)) * scale
        ds = (dh + 8) * 2.0 ** -24 * qk
        rel = 2 * ds + 2.0 ** -22 + (n + 64) * 2.0 ** -24
        half = torch.finfo(self.dtype).eps / 2
        # on the bf16 matrix instruction the probabilities (with the values' scales) are rounded to bf16: 2^-8 each
        low = 2.0 ** -8 if self.dtype == torch.bfloat16 and dh in (64, 128, 256) and self.fmt != "f32" else 0.0
        assert (np.abs(o - want) <= (rel + low) * absum + half * np.abs(want) + 1e-30).all(), \
            (np.abs(o - want) - ((rel + low) * absum + half * np.abs(want))).max()
        some = np.isfinite(wl)
        assert np.array_equal(l[~some], wl[~some])
        assert (np.abs(l[some] - wl[some]) <= ds + 2.0 ** -22 + (n + 64) * 2.0 ** -24 + 2.0 ** -23 * np.abs(wl[some])).all()
        return out, lse


TYPES = [("f32", "f32"), ("f32", "fp8"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("bf16", "f32")]
RAGGED = [(1, 1), (1, 200), (0, 50), (3, 3), (2, 129), (5, 2), (0, 0), (4, 0), (1, 64), (70, 300)]


@pytest.mark.parametrize("dtype,fmt", TYPES)
@pytest.mark.parametrize("hq,hkv,dh", [(5, 1, 128), (8, 2, 64), (3, 3, 80), (2, 1, 256), (6, 2, 16)])
def test_ragged_batches(dtype, fmt, hq, hkv, dh):
    Batch(RAGGED, hq, hkv, dh, FORMATS[dtype], fmt, 16).check()


@pytest.mark.parametrize("dtype,fmt,dh", [("f32", "int8", 64), ("bf16", "bf16", 128), ("bf16", "fp8", 128), ("bf16", "int8", 64)])
@pytest.mark.parametrize("size", [1, 7, 20, 64, 100, 256])
def test_page_sizes_and_windows(dtype, fmt, dh, size):
    b = Batch([(1, 257), (40, 41), (3, 700), (90, 400)], 4, 2, dh, FORMATS[dtype], fmt, size, seed=size)
    b.check()
    for window in (1, 17, 64, 100000):
        b.check(window=window)


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8")])
@pytest.mark.parametrize("new,total", [(1, 4097), (1, 20000), (2, 9000), (300, 5000), (1030, 1030)])
def test_long_sequences_are_cut_and_joined(dtype, fmt, new, total):
    Batch([(new, total)], 5, 1, 128, FORMATS[dtype], fmt, 64).check()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("f32", "int8"), ("bf16", "f32"), ("bf16", "bf16"), ("bf16", "fp8")])
@pytest.mark.parametrize("dh", [16, 48, 96, 112, 144, 240])
def test_widths_between_the_kernels_own(dtype, fmt, dh):
    b = Batch(RAGGED + [(33, 150)], 6, 2, dh, FORMATS[dtype], fmt, 12, seed=dh)
    b.check()
    b.check(window=40)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8"), ("f32", "bf16")])
@pytest.mark.parametrize("seqs", [[(1, 5000)], [(2, 4000), (1, 1)], [(20, 900), (7, 2000)], [(300, 2000), (41, 41), (0, 9)]])
def test_heads_of_256(dtype, fmt, seqs):
    b = Batch(seqs, 8, 2, 256, FORMATS[dtype], fmt, 20, seed=3)
    b.check()
    b.check(window=333)


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
@pytest.mark.parametrize("seqs", [[(701, 1500)], [(200, 333), (199, 4100)]])
def test_long_chunks_with_heads_of_256(fmt, seqs):
    b = Batch(seqs, 6, 1, 256, torch.bfloat16, fmt, 24, seed=4)
    b.check()
    b.check(window=100)
    new, total = seqs[0]
    key = total - 130                                    # not finite: only the rows that see it may show that
    (b.cache.v if fmt == "bf16" else b.cache.v_scale)[int(b.table[0, key // 24]), 0, key % 24] = float("nan")
    out, _ = b.run(window=100)
    sees = torch.zeros(out.shape[0], dtype=torch.bool, device="cuda")
    sees[new - 130:new - 30] = True
    end = int(b.start[-1])
    assert torch.isnan(out[:end][sees[:end]]).all() and torch.isfinite(out[:end][~sees[:end]]).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", "bf16"), ("bf16", "bf16"), ("bf16", "int8")])
def test_many_sequences(dtype, fmt):
    r = np.random.default_rng(5)
    Batch([(int(r.integers(0, 3)), int(r.integers(0, 90))) for _ in range(700)], 4, 2, 64, FORMATS[dtype], fmt, 16).check()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "int8")])
def test_the_joined_cache_as_pages_and_wide_rows(dtype, fmt):
    """[tokens][heads] pages, as a prefill leaves them; queries and output as part of wider rows"""
    b = Batch([(33, 190), (2, 70)], 4, 2, 128, FORMATS[dtype], fmt, 10, tokens_first=True)
    out, _ = b.check(scale=0.3)
    wide = torch.randn(b.q.shape[0], 10, 128, device="cuda").to(FORMATS[dtype])
    wide[:, 3:7] = b.q
    o = torch.zeros_like(wide)
    kb.paged_attention(wide[:, 3:7], b.cache, torch.from_numpy(b.start).cuda(),
                       torch.tensor(b.total, dtype=torch.int32, device="cuda"), b.table, scale=0.3, out=o[:, 1:5])
    end = int(b.start[-1])
    assert torch.equal(o[:end, 1:5], out[:end]) and (o[:, 5:] == 0).all() and (o[:, 0] == 0).all() and (o[end:] == 0).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8")])
@pytest.mark.parametrize("seqs", [[(60, 130)], [(3, 66)], [(64, 64), (1, 300)]])
@pytest.mark.parametrize("what", ["k", "v"])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(dtype, fmt, seqs, what):
    b = Batch(seqs, 4, 2, 64, FORMATS[dtype], fmt, 16, seed=9)
    clean, clean_lse = b.run()
    new, total = seqs[0]
    at = total - 2                                       # seen by the first sequence's last two rows
    page, off = int(b.table[0, at // 16]), at % 16
    t, scale = (b.cache.k, b.cache.k_scale) if what == "k" else (b.cache.v, b.cache.v_scale)
    if scale is not None:
        scale[page, 1, off] = float("nan")
    else:
        t[page, 1, off, 5] = float("inf") if what == "v" else float("nan")
    out, lse = b.run()
    hit = torch.zeros_like(out, dtype=torch.bool)
    hit[new - 2:new, 2:] = True
    if what == "v" and scale is None:
        hit[..., :5] = hit[..., 6:] = False
        assert torch.isinf(out[hit]).all()
        assert torch.equal(lse, clean_lse)
    else:
        assert torch.isnan(out[hit]).all()
    # (the few keys of a tile with such values may be added in another order: a rounding more of the probabilities each)
    a, c = out[~hit].float(), clean[~hit].float()
    assert torch.isfinite(a[~torch.isnan(c)]).all()
    assert ((a - c).abs() <= 2.0 ** -7 * (c.abs() + 4.0)).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16")])
def test_lowest_scores_and_large_ones(dtype, fmt):
    """Scores near the type's lowest value still make a softmax; equal ones weigh the same."""
    b = Batch([(1, 70), (2, 3)], 2, 1, 64, FORMATS[dtype], fmt, 16)
    b.q.fill_(1.0)
    b.cache.k.fill_(-1e36)
    out, lse = b.run()
    for r, n, first in ((0, 70, 0), (1, 2, 1), (2, 3, 1)):
        s = 0 if r == 0 else 1
        v = torch.stack([b.cache.v[b.table[s, t // 16], 0, t % 16].double() for t in range(n)])
        want = v.mean(0)
        assert ((out[r].double() - want).abs() <= 2.0 ** -7 * v.abs().mean(0) + 1e-6).all()
    assert (lse[:3] < -7e36).all() and torch.isfinite(lse[:3]).all()


def test_starts_and_pages_out_of_range_stay_inside_the_buffers():
    b = Batch([(4, 40), (4, 40)], 2, 2, 64, torch.float32, "f32", 16)
    start = torch.tensor([-5, 6, 99], dtype=torch.int32, device="cuda")       # clamped to 0, 6, rows
    lens = torch.tensor([40, 1 << 30], dtype=torch.int32, device="cuda")      # the second to 3 pages
    table = b.table.clone()
    table[0, 1] = -7
    table[1] = 1 << 30
    out, lse = torch.zeros_like(b.q), torch.zeros(b.q.shape[:2], device="cuda")
    kb.paged_attention(b.q, b.cache, start, lens, table, out=out, lse=lse)
    b.cache.k.nan_to_num_()
    b.cache.v.nan_to_num_()
    kb.paged_attention(b.q, b.cache, start, lens, table, out=out, lse=lse)
    k, v = b.numbers()
    want, wl, _ = so.paged_attention(b.q.double().cpu().numpy(), k, v, [0, 6, 10], [40, 48], table.cpu().numpy())
    assert np.allclose(out.cpu().numpy(), want, atol=1e-5) and np.allclose(lse.cpu().numpy(), wl, atol=1e-5)
    # a start that falls: the sequence has no rows
    lse.fill_(5)
    kb.paged_attention(b.q, b.cache, torch.tensor([8, 2, 2], dtype=torch.int32, device="cuda"), lens, table, out=out, lse=lse)
    assert (lse == 5).all()


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "fp8")])
def test_equal_calls_give_equal_bits_whatever_the_workspace_holds(dtype, fmt):
    b = Batch([(1, 3000), (200, 900), (1, 5)], 4, 2, 128, FORMATS[dtype], fmt, 32)
    need = kb.paged_attention_workspace_bytes(4, b.cache, 3)
    ref = None
    for fill in (0, 255, 0x7f):
        ws = torch.full((need,), fill, dtype=torch.uint8, device="cuda")
        got = b.run(workspace=ws)
        ref = ref or got
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])


def test_binding_refuses():
    b = Batch([(1, 5)], 2, 1, 64, torch.float32, "f32", 16, tail=0)
    one = torch.tensor([5], dtype=torch.int32, device="cuda")
    start = torch.from_numpy(b.start).cuda()
    for args, kw in (((b.q[:, :, :32], b.cache, start, one, b.table), {}), ((b.q, b.cache, start[:1], one, b.table), {}),
                     ((b.q, b.cache, start, one.long(), b.table), {}), ((b.q, b.cache, start, one, b.table[0]), {}),
                     ((b.q, b.cache, start, one, b.table), {"out": b.q[:, :1]}), ((b.q, b.cache, start, one, b.table), {"out": b.q}),
                     ((b.q.double(), b.cache, start, one, b.table), {}),
                     ((b.q, b.cache, start, one, b.table), {"lse": torch.zeros(1, device="cuda")}),
                     ((b.q, b.cache, start, one, b.table), {"workspace": torch.zeros(512, dtype=torch.uint8, device="cuda")})):
        with pytest.raises(kb.KeepError):
            kb.paged_attention(*args, **kw)


@pytest.mark.parametrize("dtype,fmt", [("f32", "f32"), ("f32", "fp8"), ("bf16", "bf16"), ("bf16", "fp8"), ("bf16", "int8")])
@pytest.mark.parametrize("dh", [64, 80, 128, 256])
def test_negative_scales(dtype, fmt, dh):
    """a negative factor on every tile, where the largest product is not the largest score"""
    for new in (1, 7, 20, 300):
        Batch([(new, 700), (min(new, 4), 33)], 4, 2, dh, FORMATS[dtype], fmt, 16, seed=new).check(scale=-0.07)
