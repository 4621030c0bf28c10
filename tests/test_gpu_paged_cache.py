"""keep_cache_write and keep_cache_read against the oracle, bit for bit: formats, types, head widths, layouts, odd values,
slots outside the cache."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb

pytestmark = pytest.mark.gpu

FORMATS = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "int8": torch.int8}


def make(fmt, pages, size, heads, dh, tokens_first=False):
    """A cache whose every byte is set, so that what a call must not touch shows; tokens_first: [tokens][heads] like a prefill's"""
    c = kb.PagedCache.empty(FORMATS[fmt], pages, size, heads, dh)
    if tokens_first:
        k, v = (torch.empty((pages, size, heads, dh), dtype=FORMATS[fmt], device="cuda").transpose(1, 2) for _ in range(2))
        c = kb.PagedCache(k, v, c.k_scale, c.v_scale)
    for t in (c.k, c.v):
        (t.view(torch.uint8) if t.element_size() == 1 else t).fill_(3)
    for t in (c.k_scale, c.v_scale):
        if t is not None:
            t.fill_(-5.0)
    return c


def as_numbers(t):
    return t.to(torch.float32).cpu().numpy() if t.dtype != torch.float8_e4m3fn else t.cpu().float().numpy()


def expected(x, fmt):
    """(stored values as numbers, scales or None) of rows x [n, heads, dh], float32 numpy"""
    if fmt in so.TOP:
        return so.quantise(x, fmt)
    return (torch.from_numpy(x).to(FORMATS[fmt]).float().numpy(), None)


def check(fmt, dtype, n, heads, dh, size, tokens_first=False, seed=0, spread=8, odd=False):
    g = torch.Generator().manual_seed(seed + n + dh)
    pages = n // size + 3
    x = [(torch.randn(n, heads, dh, generator=g) * torch.randint(-spread, spread + 1, (n, heads, 1), generator=g).float().exp2())
         .to(dtype) for _ in range(2)]
    if odd:         # (row, head) pairs with values that are not finite, zeros, numbers near the smallest
        x[0][0, 0, 3], x[0][1, 0, 0], x[1][0, 1, dh - 1], x[1][2] = float("nan"), float("inf"), -float("inf"), 0.0
        x[0][3] *= 1e-38
        x[0][4], x[1][5] = 1e-40, -3e38
    slots = torch.randperm(pages * size, generator=g)[:n].to(torch.int32)
    slots[n // 2:n // 2 + 1] = -1
    if n > 3:
        slots[n - 1], slots[1] = pages * size, -(1 << 31)
    ok = ((slots >= 0) & (slots < pages * size)).numpy()
    c = make(fmt, pages, size, heads, dh, tokens_first)
    c.write(x[0].cuda(), x[1].cuda(), slots.cuda())
    back = [torch.full_like(t, 9.0, device="cuda") for t in x]
    c.read(slots.cuda(), back[0], back[1])
    torch.cuda.synchronize()
    p, o = slots.numpy()[ok] // size, slots.numpy()[ok] % size
    for t, pages_t, scale_t, got in ((x[0], c.k, c.k_scale, back[0]), (x[1], c.v, c.v_scale, back[1])):
        want, scale = expected(t.float().numpy(), fmt)
        stored = as_numbers(pages_t)
        assert np.array_equal(stored[p, :, o], want[ok], equal_nan=True)
        rest = np.ones((pages, size), bool)
        rest[p, o] = False
        raw = (pages_t.view(torch.uint8) if pages_t.element_size() == 1 else pages_t).float().cpu().numpy()
        assert (raw.transpose(0, 2, 1, 3)[rest] == 3).all()
        if scale is not None:
            s = scale_t.cpu().numpy()
            assert np.array_equal(s[p, :, o], scale[ok], equal_nan=True) and (s.transpose(0, 2, 1)[rest] == -5).all()
            with np.errstate(all="ignore"):
                want = so.dequantise(want, scale)
        want = torch.from_numpy(np.ascontiguousarray(want)).to(dtype).float().numpy()
        assert np.array_equal(got.float().cpu().numpy()[ok], want[ok], equal_nan=True)
        assert (got.float().cpu().numpy()[~ok] == 9).all()


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("dh", [16, 64, 80, 128, 208, 256])
def test_write_and_read_back(fmt, dtype, dh):
    check(fmt, dtype, 37, 3, dh, 16)


@pytest.mark.parametrize("fmt", list(FORMATS))
@pytest.mark.parametrize("n,heads,size", [(1, 1, 1), (1, 8, 16), (5, 1, 7), (64, 8, 100), (513, 2, 256), (1000, 5, 1)])
def test_sizes(fmt, n, heads, size):
    check(fmt, torch.bfloat16, n, heads, 128, size)
    check(fmt, torch.float32, n, heads, 48, size, tokens_first=True)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_values_that_are_not_finite_and_tiny_ones(fmt, dtype):
    check(fmt, dtype, 40, 4, 64, 8, odd=True)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_ties_round_to_even(fmt):
    # amax = Q makes the scale 1, so values are codes: every grid point, every midpoint and their neighbours
    top = float(so.TOP[fmt])
    grid = np.r_[so.FP8] if fmt == "fp8" else np.arange(128.0)
    mid = (grid[1:] + grid[:-1]) / 2
    v = np.concatenate([grid, mid, np.nextafter(mid.astype(np.float32), 0), np.nextafter(mid.astype(np.float32), 1e9)])
    v = np.concatenate([v, -v]).astype(np.float32)
    v = np.concatenate([v, np.zeros(-len(v) % 15, np.float32)]).reshape(-1, 1, 15)
    x = np.concatenate([np.full((len(v), 1, 1), top, np.float32), v], 2)
    c = make(fmt, len(x), 1, 1, 16)
    t = torch.from_numpy(x).cuda()
    slots = torch.arange(len(x), dtype=torch.int32, device="cuda")
    c.write(t, t, slots)
    a, b = torch.empty_like(t), torch.empty_like(t)
    c.read(slots, a, b)
    want, scale = so.quantise(x, fmt)
    assert (scale == 1).all() and np.array_equal(a.cpu().numpy(), want) and torch.equal(a, b)


def test_rows_of_a_wider_buffer_and_offsets_past_32_bits():
    fused = torch.randn(20, 10 * 64, generator=torch.Generator().manual_seed(3)).cuda()
    k, v = fused[:, 128:256].unflatten(1, (2, 64)), fused[:, 512:].unflatten(1, (2, 64))
    # pages of 2^33 bytes and more in all: the last ones lie past 32-bit offsets of elements
    pages, size = 4200, 128
    c = kb.PagedCache.empty(torch.bfloat16, pages, size, 64, 128)
    wide = kb.PagedCache(c.k[:, :2, :, :64], c.v[:, :2, :, :64])
    slots = (pages * size - 1 - 97 * torch.arange(20, device="cuda")).to(torch.int32)
    assert int(slots[0]) * 64 * 128 > 1 << 32
    wide.write(k, v, slots)
    a, b = torch.empty(20, 2, 64, device="cuda"), torch.empty(20, 2, 64, device="cuda")
    wide.read(slots, a, b)
    assert torch.equal(a, k.bfloat16().float()) and torch.equal(b, v.bfloat16().float())


def test_binding_refuses():
    z = torch.zeros
    k = z(2, 2, 16, 64, device="cuda")
    with pytest.raises(kb.KeepError):
        kb.PagedCache(k, k[:1])
    with pytest.raises(kb.KeepError):
        kb.PagedCache(k.half(), k.half())
    with pytest.raises(kb.KeepError):
        kb.PagedCache(k.to(torch.int8), k.to(torch.int8))
    with pytest.raises(kb.KeepError):
        kb.PagedCache(k, k.clone(), z(2, 2, 16, device="cuda"), z(2, 2, 16, device="cuda"))
    with pytest.raises(kb.KeepError):
        kb.PagedCache(k.cpu(), k.cpu())
    c, s = kb.PagedCache(k, k.clone()), z(3, dtype=torch.int32, device="cuda")
    rows = z(3, 2, 64, device="cuda")
    for bad in ((rows[:2], rows[:2], s), (rows, rows[:, :1], s), (rows, rows.bfloat16(), s), (rows.double(), rows.double(), s),
                (rows[:, :, :32], rows[:, :, :32], s), (rows, rows, s.long()), (rows.cpu(), rows.cpu(), s)):
        with pytest.raises(kb.KeepError):
            c.write(*bad)


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_quotients_beside_a_border_between_codes(fmt):
    """x / scale next to every border between two codes, for scales over the whole range: codes as a division gives them"""
    r = np.random.default_rng(17)
    n, dh = 4096, 128
    q = so.TOP[fmt]
    edge = np.arange(127) + 0.5 if fmt == "int8" else np.unique(np.abs(np.concatenate(
        [(a[:-1] + a[1:]) / 2 for a in [np.sort(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy())]])))
    x = np.empty((2, n, 1, dh), np.float32)
    x[..., 0] = np.exp2(r.uniform(-126, 120, (2, n, 1))) * r.uniform(1, 2, (2, n, 1))      # the head's largest
    x[..., 0].flat[:64] = 1e-45 * np.arange(64)
    scale = np.maximum(x[..., :1] * np.float32(1) / np.float32(q), np.float32(2.0 ** -126)).astype(np.float64)
    x[..., 1:] = (r.choice(edge, (2, n, 1, dh - 1)) * scale * (1 + r.integers(-3, 4, (2, n, 1, dh - 1)) * 2.0 ** -24)
                  * r.choice([-1, 1], (2, n, 1, dh - 1)))
    x[..., 1:] = np.clip(x[..., 1:], -np.abs(x[..., :1]), np.abs(x[..., :1]))
    c = make(fmt, n // 16, 16, 1, dh)
    c.write(torch.from_numpy(x[0]).cuda(), torch.from_numpy(x[1]).cuda(), torch.arange(n, dtype=torch.int32).cuda())
    for got, scales, rows in ((c.k, c.k_scale, x[0]), (c.v, c.v_scale, x[1])):
        want, s = so.quantise(rows, fmt)
        assert np.array_equal(scales.cpu().numpy().reshape(n, 1), s)
        assert np.array_equal(as_numbers(got).reshape(n, 1, dh), want)
