"""Pins of the serving operators' oracle: against independent expressions, closed forms and brute force, on the CPU."""
import math

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import serve_oracle as so


def test_half_layout_is_complex_multiplication_and_composes():
    r = np.random.default_rng(0)
    x = r.standard_normal((5, 3, 16))
    f, m = so.rope_frequencies(12, 1e4)
    pos = np.array([0, 1, 7, 1000, -3])
    y = so.rope(x, pos, f)
    z = (x[..., :6] + 1j * x[..., 6:12]) * np.exp(1j * pos[:, None, None] * f)
    assert m == 1.0 and np.allclose(y[..., :6], z.real) and np.allclose(y[..., 6:12], z.imag)
    assert np.array_equal(y[..., 12:], x[..., 12:])
    assert np.allclose(so.rope(y, -pos, f), x) and np.allclose(so.rope(so.rope(x, pos, f), pos, f), so.rope(x, 2 * pos, f))


def test_interleaved_is_half_with_the_values_reordered():
    r = np.random.default_rng(1)
    x = r.standard_normal((3, 2, 8))
    f, _ = so.rope_frequencies(8, 1e4)
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    assert np.allclose(so.rope(x, [3, 9, 27], f, interleaved=True)[..., order], so.rope(x[..., order], [3, 9, 27], f))


def test_scalings():
    plain, _ = so.rope_frequencies(128, 1e6)
    assert plain[0] == 1 and np.allclose(plain[1:] / plain[:-1], 1e6 ** (-2 / 128))
    assert np.allclose(so.rope_frequencies(128, 1e6, "linear", 2.0)[0], plain / 2)
    base, _ = so.rope_frequencies(128, 1e6, "base", 4.0)
    assert base[0] == 1 and math.isclose(base[-1], plain[-1] / 4)
    parts, m = so.rope_frequencies(128, 1e6, "parts", 4.0, 32768)
    turns = 32768 * plain / (2 * math.pi)
    assert np.allclose(parts[turns > 32], plain[turns > 32]) and np.allclose(parts[turns < 1], plain[turns < 1] / 4)
    assert math.isclose(m, 1 + 0.1 * math.log(4)) and (np.diff(parts) < 0).all()


def test_quantise_against_torch():
    r = np.random.default_rng(2)
    x = (r.standard_normal((200, 32)) * 2.0 ** r.integers(-30, 30, (200, 1))).astype(np.float32)
    x[0], x[1], x[2, 3], x[3, 4], x[4] = 0, 1e-41, np.nan, np.inf, x[4] * np.float32(1e-38)
    for fmt, dt in (("fp8", torch.float8_e4m3fn), ("int8", torch.int8)):
        c, s = so.quantise(x, fmt)
        assert np.isnan(s[2:4]).all() and (c[2:4] == 0).all() and s[0] == np.float32(2.0 ** -126) and (c[0] == 0).all()
        ok = np.r_[0:2, 4:200]
        u = torch.from_numpy(x[ok] / s[ok, None]).clamp(-float(so.TOP[fmt]), float(so.TOP[fmt]))
        want = (u.round() if fmt == "int8" else u).to(dt).float().numpy()
        assert np.array_equal(c[ok], want)
        err = np.abs(so.dequantise(c, s)[5:].astype(np.float64) - x[5:])
        top = np.abs(x[5:]).max(-1, keepdims=True)
        # half a step of the grid: 1/254 of the largest, or 2^-4 of the value (2^-10 codes below the smallest normal)
        bound = top / 254 if fmt == "int8" else np.maximum(np.abs(x[5:]) * 2.0 ** -4, top / 448 * 2.0 ** -10)
        assert (err <= bound * (1 + 1e-6)).all()


def test_fp8_grid():
    assert len(so.FP8) == 127 and so.FP8[-1] == 448 and so.FP8[1] == 2.0 ** -9 and (np.diff(so.FP8) > 0).all()
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, so.FP8)


@pytest.mark.parametrize("window", [0, 5])
def test_attention_against_torch(window):
    r = np.random.default_rng(3)
    size, pages, hkv, rep, dh = 4, 9, 2, 3, 16
    kp, vp = r.standard_normal((2, pages, hkv, size, dh))
    lens, new = [13, 1, 0, 7], [4, 1, 2, 0]
    table = np.array([[3, 0, 8, 5], [1, 99, -1, 7], [0, 0, 0, 0], [2, 6, 0, 0]])
    start = np.concatenate([[0], np.cumsum(new)])
    q = r.standard_normal((start[-1] + 1, hkv * rep, dh))
    out, lse, absum = so.paged_attention(q, kp, vp, start, lens, table, window)
    assert np.isnan(out[-1]).all() and (out[start[2]:start[3]] == 0).all() and (lse[start[2]:start[3]] == -np.inf).all()
    for s in (0, 1):
        n, t = new[s], lens[s]
        flat = [table[s][i // size] * size + i % size for i in range(t)]
        k = kp.transpose(0, 2, 1, 3).reshape(-1, hkv, dh)[flat]
        v = vp.transpose(0, 2, 1, 3).reshape(-1, hkv, dh)[flat]
        pos, key = np.arange(t - n, t)[:, None], np.arange(t)[None]
        mask = (key <= pos) & (key > pos - (window or 1000))
        want = F.scaled_dot_product_attention(torch.from_numpy(q[start[s]:start[s + 1]]).transpose(0, 1),
                                              torch.from_numpy(k).transpose(0, 1), torch.from_numpy(v).transpose(0, 1),
                                              attn_mask=torch.from_numpy(mask), enable_gqa=True)
        assert np.allclose(out[start[s]:start[s + 1]], want.transpose(0, 1).numpy())
    assert (absum[:5] >= np.abs(out[:5]) - 1e-12).all()


def test_sampling_follows_the_distribution():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    for temp, share in ((1.0, np.array([0.1, 0.4, 0.2, 0.3])), (0.5, np.array([0.01, 0.16, 0.04, 0.09]) / 0.3)):
        got = [so.sample(x, (i + 0.5) / 1000, temp) for i in range(1000)]
        for t in range(4):
            assert abs(sum(g[0] == t for g in got) / 1000 - share[t]) < 2e-3
            assert all(abs(g[1] - share[t]) < 1e-11 for g in got if g[0] == t)
    assert [so.sample(x, u)[0] for u in (0.0, 0.39, 0.41, 0.69, 0.71, 0.89, 0.91)] == [1, 1, 3, 3, 2, 2, 0]   # by rank


def test_sampling_limits():
    x = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    us = (np.arange(200) + 0.5) / 200
    def tokens(**kw):
        return {so.sample(x, u, **kw)[0] for u in us}
    assert tokens() == {0, 1, 2, 3} and tokens(top_k=2) == {1, 3} and tokens(top_k=9) == {0, 1, 2, 3}
    assert tokens(top_p=0.69) == {1, 3} and tokens(top_p=0.71) == {1, 2, 3} and tokens(top_p=0.0) == {1}
    assert tokens(min_p=0.49) == {1, 2, 3} and tokens(min_p=0.6) == {1, 3} and tokens(min_p=2.0) == {1}
    assert tokens(top_k=2, top_p=0.5) == {1} and tokens(top_k=2, top_p=0.6) == {1, 3}     # a share of the two kept
    assert tokens(temperature=0.0) == {1} and tokens(temperature=-1.0) == {1} and tokens(temperature=float("nan")) == {1}


def test_sampling_ties_and_odd_rows():
    inf, nan = np.inf, np.nan
    assert [so.sample([2.0, 1.0, 2.0, 2.0], u, top_k=2)[0] for u in (0.1, 0.9)] == [0, 2]
    assert so.sample([nan, -inf], 0.5) == (-1, 0.0)
    assert so.sample([nan, -inf, 3.0], 0.99) == (2, 1.0)
    assert {so.sample([1.0, inf, 5.0, inf], u)[0] for u in (0.1, 0.6)} == {1, 3}
    assert so.sample([0.0, -28.0], 1.0)[0] in (0, 1) and so.sample([0.0, -29.0], 1.0) == (0, 1.0)
