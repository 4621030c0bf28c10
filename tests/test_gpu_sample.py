"""keep_sample and keep_decode_sampled against the oracle's whole-number arithmetic: every limit, ties, flat rows, odd values."""
import math

import numpy as np
import pytest
import torch

import keep_synth as ks
from gpu_util import Problem
from oracle import serve_oracle as so
from paper_2602_23592_amd import KeepError
from paper_2602_23592_amd import binding as kb
from test_gpu_decode import head_weights

pytestmark = pytest.mark.gpu


def fast(x, u, t, k, p, mp):
    """so.sample's rule with numpy arrays, for rows of real size"""
    x = np.asarray(x, dtype=np.float64)
    if not np.any(x > -np.inf):
        return -1, 0.0
    best = int(np.nanargmax(x))
    if not t > 0:
        return best, 1.0
    with np.errstate(all="ignore"):
        y = np.where(x == x[best], 0.0, x[best] - x) / t
        w = np.rint(np.exp(-y) * so.ONE)
    w = np.where(np.isnan(w), 0, w).astype(np.int64)
    ids = np.flatnonzero(w >= (max(1, math.ceil(min(mp, 1.0) * so.ONE)) if mp > 0 else 1))
    ids = ids[np.lexsort((ids, -x[ids]))]
    ids = ids[:k] if k >= 1 else ids
    ends = np.cumsum(w[ids])
    if p < 1:
        ids = ids[:np.searchsorted(ends, max(1, math.ceil(p * float(int(ends[-1])))), side="left") + 1]
    ends = ends[:len(ids)]
    total = int(ends[-1])
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    at = int(np.searchsorted(ends, min(math.floor(u * float(total)), total - 1), side="right"))
    return int(ids[at]), int(w[ids[at]]) / total


def check(x, u, t=None, k=None, p=None, mp=None, rule=fast):
    n = len(x)
    dev = lambda a, dt: None if a is None else torch.tensor(a, dtype=dt, device="cuda")
    f32 = torch.float32
    probs = torch.full((n,), 7.0, device="cuda")
    got = kb.sample(x.cuda(), dev(u, f32), dev(t, f32), dev(k, torch.int32), dev(p, f32), dev(mp, f32), probs=probs).cpu().numpy()
    f = lambda a, i, d: d if a is None else float(np.float32(a[i]))
    rows = x.double().numpy()
    for i in range(n):
        want, prob = rule(rows[i], f(u, i, 0), f(t, i, 1.0), 0 if k is None else k[i], f(p, i, 1.0), f(mp, i, 0.0))
        assert got[i] == want, (i, got[i], want)
        assert abs(float(probs[i]) - prob) <= 2.0 ** -23 * prob


def mixture(n, seed):
    r = np.random.default_rng(seed)
    return dict(u=r.random(n).astype(np.float32), t=r.choice([0.0, 0.3, 0.7, 1.0, 1.5, 4.0], n), k=r.choice([0, 1, 5, 50, 400], n),
                p=r.choice([1.0, 0.99, 0.9, 0.5, 0.1], n), mp=r.choice([0.0, 0.0, 0.01, 0.2], n))


def test_the_fast_rule_is_the_oracles():
    r = np.random.default_rng(1)
    for i in range(300):
        x = np.round(r.standard_normal(r.integers(1, 40)) * r.choice([0.5, 3.0, 20.0]), int(r.integers(0, 4)))
        m = {n: v[0] for n, v in mixture(1, 100 + i).items()}
        a = (x, float(m["u"]), float(m["t"]), int(m["k"]), float(np.float32(m["p"])), float(np.float32(m["mp"])))
        assert fast(*a)[0] == so.sample(*a)[0] and abs(fast(*a)[1] - so.sample(*a)[1]) < 1e-12


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1024, 1025, 4099, 32000, 152064, 300007])
def test_mixed_requests(dtype, vocab):
    n = 24
    x = 3.0 * torch.randn(n, vocab, generator=torch.Generator().manual_seed(vocab))
    check(x.to(dtype), **mixture(n, vocab))


@pytest.mark.parametrize("rows", [1, 2, 17, 130, 300])
def test_row_counts(rows):
    x = 2.5 * torch.randn(rows, 5003, generator=torch.Generator().manual_seed(rows))
    check(x, **mixture(rows, rows))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_many_rows_of_a_large_vocabulary(dtype):
    """more rows than are divided among workgroups; some of them flat"""
    x = 3.0 * torch.randn(70, 60001, generator=torch.Generator().manual_seed(7))
    x[::9] = 1.25
    check(x.to(dtype), **mixture(70, 70))


@pytest.mark.parametrize("vocab", [5000, 152064])
def test_flat_and_nearly_flat_rows(vocab):
    """thousands of tokens in one bin: equal logits, two values, steps of one unit in the last place, zeros of both signs"""
    g = torch.Generator().manual_seed(3)
    one = torch.ones(vocab)
    rows = [one * 2.5, one.clone(), torch.where(torch.rand(vocab, generator=g) < 0.5, 1.0, 1.0 + 2.0 ** -20),
            (torch.randint(0, 1 << 16, (vocab,), generator=g).float() * 2.0 ** -23 + 1.0), one * 0.0, one * -1e30]
    rows[1][17] = 1.0 + 2.0 ** -23
    rows[4][1::2] = -0.0
    x = torch.stack(rows * 4)
    n = len(x)
    m = mixture(n, vocab)
    m["t"] = np.where(m["t"] == 0, 1.0, m["t"])
    m["k"] = np.r_[[0] * 6, [vocab - 1] * 6, [4100] * 6, [3] * 6]
    m["mp"] = np.zeros(n)
    check(x, **m)


def test_ends_of_the_unit_interval_and_parameters_out_of_range():
    x = 2.0 * torch.randn(14, 777, generator=torch.Generator().manual_seed(5))
    nan, inf = math.nan, math.inf
    check(x, [0.0, 1 - 2.0 ** -24, 1.0, 5.0, -1.0, nan, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5],
          t=[1, 1, 1, 1, 1, 1, -2.0, nan, 1e-30, 1e30, 1, 1, 1, 1], k=[0, 0, 0, 0, 0, 0, 0, 0, 0, 0, -5, 778, 2 ** 31 - 1, -2 ** 31],
          p=[1, 1, 1, 1, 1, 1, 1, 1, 1, 1, nan, 7.0, -1.0, 0.0], mp=[0, 0, 0, 0, 0, 0, 0, 0, 0, 0, nan, -1.0, 0.0, 3.0])
    check(x[:2], [0.999, 0.3], t=[inf, inf])              # flat over everything finite
    check(x, [0.25] * 14)                                  # no parameters


def test_odd_logits():
    nan, inf = math.nan, math.inf
    x = torch.randn(10, 3000, generator=torch.Generator().manual_seed(6))
    x[0] = nan
    x[1] = -inf
    x[2, ::2] = nan
    x[3, 100:] = -inf
    x[4, 5] = x[4, 2999] = inf
    x[5] = -inf
    x[5, 1234] = -3e38
    x[6] = torch.finfo(torch.float32).min
    x[7, :] = nan
    x[7, 7] = inf
    x[8] = torch.linspace(-3e38, 3e38, 3000)
    for u in (0.0, 0.4, 0.9999):
        check(x, [u] * 10, t=[0.8] * 10, k=[0] * 10, p=[0.95] * 10, rule=so.sample)
        check(x, [u] * 10, t=[0.0] * 10, rule=so.sample)


def test_strided_and_unaligned_rows():
    buf = torch.randn(6 * 1501 + 3, generator=torch.Generator().manual_seed(7)).cuda()
    x = buf[3:].view(6, 1501)[:, 1:1400]
    m = mixture(6, 7)
    got = kb.sample(x, torch.tensor(m["u"], device="cuda"))
    assert got.tolist() == [fast(r, float(u), 1.0, 0, 1.0, 0.0)[0] for r, u in zip(x.double().cpu().numpy(), m["u"])]


def test_binding_refuses():
    x, u = torch.zeros(3, 10, device="cuda"), torch.zeros(3, device="cuda")
    for args, kw in (((x.double(), u), {}), ((x[0], u), {}), ((x, u[:2]), {}), ((x, u.double()), {}), ((x.t(), torch.zeros(10, device="cuda")), {}),
                     ((x, u, u[:1]), {}), ((x, u), {"tokens": u}), ((x, u), {"workspace": u}), ((x[:1].expand(3, 10), u), {}),
                     ((x, u.cpu()), {})):
        with pytest.raises(KeepError):
            kb.sample(*args, **kw)


@pytest.mark.parametrize("shape", [ks.ModelShape(2, 128, 6, 2, 64, 200, 2011, 1.0e6, 1e-6, "f32"),
                                   ks.ModelShape(2, 512, 8, 2, 128, 1024, 1031, 1.0e6, 1e-6, "bf16")], ids=["f32", "bf16"])
def test_decode_sampled(shape):
    pb = Problem(shape, [12, 9], 3, seed=8, std=0.1)
    n, new = pb.n_tokens, 6
    ctx = pb.context(max_tokens=n + new)
    fn, lm = (t.cuda() for t in head_weights(shape))
    dt = ks.torch_dtype(shape.storage)
    kc = torch.zeros((2, n + new, shape.n_kv_heads, shape.head_dim), dtype=dt, device="cuda")
    vc = torch.zeros_like(kc)
    xf = torch.empty((3, shape.hidden), dtype=dt, device="cuda")
    ctx.prefill(pb.prompt(), [1.0, 1.0], 1, kc, vc, xf, cache_rows=n + new)
    lg = torch.empty((new, shape.vocab), device="cuda")
    greedy = ctx.decode(fn, lm, xf[-1], kc, vc, n, new, logits_out=lg)
    greedy_lg = lg.clone()
    toks, probs = ctx.decode_sampled(fn, lm, xf[-1], kc, vc, n, [0.5] * new, temperature=0.0, logits_out=lg)
    assert toks == greedy and probs == [1.0] * new and torch.equal(lg, greedy_lg)
    u = [0.9, 0.1, 0.0, 0.999, 0.5, 0.7]
    toks, probs = ctx.decode_sampled(fn, lm, xf[-1], kc, vc, n, u, 1.3, 40, 0.97, 0.001, logits_out=lg)
    f = lambda v: float(np.float32(v))
    for t, row in enumerate(lg.double().cpu().numpy()):
        want, prob = fast(row, f(u[t]), f(1.3), 40, f(0.97), f(0.001))
        assert toks[t] == want and abs(probs[t] - prob) <= 2.0 ** -23 * prob
    # each token was fed to the next step: forcing the same ones gives the same logits
    again = torch.empty_like(lg)
    ctx.decode(fn, lm, xf[-1], kc, vc, n, new, logits_out=again, forced_tokens=toks[:-1])
    assert torch.equal(again, lg)
    for kw in (dict(uniform=[1.0] * 2), dict(uniform=[math.nan] * 2), dict(uniform=[-0.1, 0.5]), dict(uniform=[]),
               dict(temperature=math.inf), dict(top_p=math.nan), dict(min_p=math.inf), dict(uniform=[0.5] * 65)):
        with pytest.raises(KeepError):
            ctx.decode_sampled(fn, lm, xf[-1], kc, vc, n, **{"uniform": [0.5] * 2, **kw})
    assert ctx.decode(fn, lm, xf[-1], kc, vc, n, new) == greedy
