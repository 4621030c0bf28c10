"""A chunk of new tokens after a joined prompt, each step held to its own bound: the rotated rows, the rows stored, and attention
over what is stored.  Looser joint bounds would let a rotation one position off, or a missing key, through."""
import numpy as np
import pytest
import torch

import keep_synth as ks
from gpu_util import Problem
from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb
from test_gpu_paged_cache import as_numbers
from test_gpu_rope_rows import bound

pytestmark = pytest.mark.gpu

SHAPE = ks.ModelShape(2, 512, 8, 2, 128, 1024, 1031, 1.0e6, 1e-6, "bf16")


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "int8"])
def test_every_step_of_a_chunk_after_the_prefill(fmt):
    glen, lq, size, new, layer = [40, 7, 65], 9, 11, 5, 1
    pb = Problem(SHAPE, glen, lq, seed=6, std=0.05)
    n = pb.n_tokens
    pages = -(-(n + new) // size)
    kc = torch.zeros((2, pages * size, 2, 128), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    xf = torch.empty((lq, SHAPE.hidden), dtype=torch.bfloat16, device="cuda")
    pb.context(max_tokens=pages * size).prefill(pb.prompt(), [1.0, 0.5], 2, kc, vc, xf, cache_rows=pages * size)
    paged = lambda t: t[layer].view(pages, size, 2, 128).transpose(1, 2)
    if fmt == "bf16":
        cache = kb.PagedCache(paged(kc), paged(vc))
    else:
        cache = kb.PagedCache.empty({"fp8": torch.float8_e4m3fn, "int8": torch.int8}[fmt], pages, size, 2, 128)
        for t in (cache.k, cache.v):
            t.view(torch.uint8).zero_()
        cache.k_scale.zero_(), cache.v_scale.zero_()
        cache.write(kc[layer, :n], vc[layer, :n], torch.arange(n, dtype=torch.int32, device="cuda"))
    qkv = torch.randn(new, 12, 128, generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    raw = qkv.double().cpu().numpy()
    freq, _ = kb.rope_frequencies(128, SHAPE.rope_theta)
    pos = torch.arange(n, n + new, dtype=torch.int32, device="cuda")
    kb.rope_rows(q, k, pos, torch.from_numpy(freq).cuda())
    cache.write(k, v, pos)
    lse = torch.empty((new, 8), device="cuda")
    out = kb.paged_attention(q, cache, torch.tensor([0, new], dtype=torch.int32, device="cuda"),
                             torch.tensor([n + new], dtype=torch.int32, device="cuda"),
                             torch.arange(pages, device="cuda", dtype=torch.int32)[None], lse=lse)
    rows = qkv.double().cpu().numpy()
    # 1. rotation: queries and keys; the values as they were
    turned = so.rope(raw[:, :10], pos.tolist(), freq)
    within = lambda want: np.abs(rows[:, :10] - want) <= bound(raw[:, :10], want, 128, torch.bfloat16, False)
    assert within(turned).all() and np.array_equal(rows[:, 10:], raw[:, 10:])
    assert not within(so.rope(raw[:, :10], (pos + 1).tolist(), freq))[:, 8:].all()
    # 2. the rows stored are these
    stored = []
    for t, s, part in ((cache.k, cache.k_scale, rows[:, 8:10]), (cache.v, cache.v_scale, rows[:, 10:])):
        x = as_numbers(t).astype(np.float64)
        x = (x if s is None else x * s.double().cpu().numpy()[..., None]).transpose(0, 2, 1, 3).reshape(-1, 2, 128)
        want = part if fmt == "bf16" else np.float64(so.quantise(part, fmt)[0]) * np.float64(so.quantise(part, fmt)[1])[..., None]
        assert np.array_equal(x[n:n + new], want)
        stored.append(x[:n + new])
    # 3. attention of these rows over what is stored
    total = n + new
    # a score: dh products and sums of binary32 and a few operations more; a probability twice that, its exponential, the sum of
    # them; each rounded to bf16, and the result
    qk = np.linalg.norm(rows[:, :8], axis=-1).max() * np.linalg.norm(stored[0], axis=-1).max() * 128 ** -0.5
    ds = (128 + 8) * 2.0 ** -24 * qk
    rel = 2 * ds + 2.0 ** -22 + (total + 64) * 2.0 ** -24 + 2.0 ** -8

    def holds(ks_, vs_, length):
        one = lambda t: t[:, :, None]                 # pages of one token
        want, wl, absum = so.paged_attention(rows[:, :8], one(ks_), one(vs_), [0, new], [length], np.arange(length)[None])
        return (np.abs(out.double().cpu().numpy() - want) <= rel * absum + 2.0 ** -8 * np.abs(want)).all(), \
            (np.abs(lse.double().cpu().numpy() - wl) <= ds + 2.0 ** -22 + (total + 64) * 2.0 ** -24 + 2.0 ** -23 * np.abs(wl)).all()

    assert holds(*stored, total) == (True, True)
    # (what the bounds tell apart: the oracle without the newest key, and with the new keys one position off)
    assert holds(stored[0], stored[1], total - 1) == (False, False)
    off = stored[0].copy()
    off[n:] = so.rope(raw[:, 8:10], (pos + 1).tolist(), freq)
    assert holds(off, stored[1], total) == (False, False)
