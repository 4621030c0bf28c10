"""The serving operators as they are used together: memories kept in 8-bit pages and joined by a prefill, a joined cache
continued with new tokens, and a decoding step captured once and replayed as the sequences grow."""
import numpy as np
import pytest
import torch

import keep_synth as ks
from gpu_util import Problem
from oracle import serve_oracle as so
from paper_2602_23592_amd import KeepPrompt
from paper_2602_23592_amd import binding as kb

pytestmark = pytest.mark.gpu

SHAPE = ks.ModelShape(2, 512, 8, 2, 128, 1024, 1031, 1.0e6, 1e-6, "bf16")


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("fmt", ["fp8", "int8"])
def test_memories_from_8_bit_pages_join_like_their_values(fmt):
    """Group blocks written to pages and read back are the blocks a prefill takes; it gives what the stored values give."""
    glen, lq = [40, 7, 65], 9
    pb = Problem(SHAPE, glen, lq, seed=6, std=0.05)
    cache = kb.PagedCache.empty({"fp8": torch.float8_e4m3fn, "int8": torch.int8}[fmt], 60, 16, 2, 128)
    free = torch.randperm(60 * 16, generator=torch.Generator().manual_seed(1)).to(torch.int32).cuda()
    at, read, stored = 0, ([], []), ([], [])
    for l in range(2):
        rows = ([], [], [], [])
        for g, n in enumerate(glen):
            slots = free[at:at + n]
            at += n
            k, v = pb.kb_d[l][g], pb.vb_d[l][g]
            cache.write(k, v, slots)
            back = torch.empty_like(k), torch.empty_like(v)
            cache.read(slots, *back)
            for i, t in enumerate((k, v)):
                rows[i].append(back[i])
                rows[2 + i].append(torch.from_numpy(so.dequantise(*so.quantise(t.float().cpu().numpy(), fmt))).bfloat16().cuda())
        for i in range(2):
            read[i].append(rows[i])
            stored[i].append(rows[2 + i])
    res = []
    for kblocks, vblocks in (read, stored):
        kc, vc = pb.empty_cache()
        xf = torch.empty((lq, SHAPE.hidden), dtype=torch.bfloat16, device="cuda")
        pr = KeepPrompt(glen, lq, pb.ids, kblocks, vblocks, 2)
        sets, _ = pb.context().prefill(pr, [0.0, 0.0], 1, kc, vc, xf)
        torch.cuda.synchronize()
        res.append((sets, kc, vc, xf))
    assert res[0][0] == res[1][0] and all(torch.equal(a, b) for a, b in zip(res[0][1:], res[1][1:]))


@pytest.mark.parametrize("fmt", ["bf16", "int8"])
def test_a_chunk_after_the_prefill(fmt):
    """New tokens after a joined prompt: rotated to their positions, stored, attending to the prompt and to each other.  In
    bf16 the prefill's own cache serves as the pages; in 8 bits it is copied into pages first."""
    glen, lq, size, new = [40, 7, 65], 9, 11, 5
    pb = Problem(SHAPE, glen, lq, seed=6, std=0.05)
    n = pb.n_tokens                                   # 121 = 11 pages of 11
    pages = -(-(n + new) // size)
    kc = torch.zeros((2, pages * size, 2, 128), dtype=torch.bfloat16, device="cuda")
    vc = torch.zeros_like(kc)
    xf = torch.empty((lq, SHAPE.hidden), dtype=torch.bfloat16, device="cuda")
    pb.context(max_tokens=pages * size).prefill(pb.prompt(), [1.0, 0.5], 2, kc, vc, xf, cache_rows=pages * size)
    layer = 1
    joined = kb.PagedCache(kc[layer].view(pages, size, 2, 128).transpose(1, 2), vc[layer].view(pages, size, 2, 128).transpose(1, 2))
    every = torch.arange(n, dtype=torch.int32, device="cuda")
    cache = joined
    if fmt == "int8":
        cache = kb.PagedCache.empty(torch.int8, pages, size, 2, 128)
        k, v = (torch.empty((n, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        joined.read(every, k, v)
        assert torch.equal(k, kc[layer, :n]) and torch.equal(v, vc[layer, :n])
        cache.write(k, v, every)
    g = torch.Generator().manual_seed(2)
    qkv = torch.randn(new, 12, 128, generator=g).bfloat16().cuda()
    q, k, v = qkv[:, :8], qkv[:, 8:10], qkv[:, 10:]
    raw = qkv.double().cpu().numpy()
    freq, _ = kb.rope_frequencies(128, SHAPE.rope_theta)
    pos = torch.arange(n, n + new, dtype=torch.int32, device="cuda")
    kb.rope_rows(q, k, pos, torch.from_numpy(freq).cuda())
    cache.write(k, v, pos)
    lse = torch.empty((new, 8), device="cuda")
    out = kb.paged_attention(q, cache, i32([0, new]), i32([n + new]), torch.arange(pages, device="cuda", dtype=torch.int32)[None],
                             lse=lse)
    # the oracle, from the prefill's cache and the unrotated rows
    bf = lambda t: torch.from_numpy(t).bfloat16().double().numpy()
    qr, kr = (bf(so.rope(raw[:, a:b], pos.tolist(), freq)) for a, b in ((0, 8), (8, 10)))
    ks_, vs_ = np.concatenate([kc[layer, :n].double().cpu().numpy(), kr]), np.concatenate([vc[layer, :n].double().cpu().numpy(), raw[:, 10:]])
    if fmt == "int8":
        ks_, vs_ = (so.dequantise(*so.quantise(t, "int8")).astype(np.float64) for t in (ks_, vs_))
    one = lambda t: t[:, :, None]                     # pages of one token
    want, wl, absum = so.paged_attention(qr, one(ks_), one(vs_), [0, new], [n + new], np.arange(n + new)[None])
    # a rotated value next to a border may round the other way: a step of bf16 (2^-7) in some of 128 products of a score
    ds = 2.0 ** -7 * np.abs(qr).max() * np.abs(ks_).max() * 128 ** 0.5 * 2
    assert (np.abs(out.double().cpu().numpy() - want) <= (2.0 ** -7 + 2.0 ** -6 * ds) * absum + 2.0 ** -8 * np.abs(want) + 1e-3).all()
    assert (np.abs(lse.double().cpu().numpy() - wl) <= 2.0 ** -6 * ds + 1e-3).all()


@pytest.mark.parametrize("fmt", ["bf16", "fp8"])
def test_a_captured_step_follows_the_sequences(fmt):
    """Rotation, write, attention and choice in one graph; lengths, positions, slots and uniforms change between replays."""
    hq, hkv, dh, size, seqs, steps, vocab = 8, 2, 128, 16, 5, 6, 5003
    g = torch.Generator().manual_seed(4)
    start_len = [0, 1, 15, 100, 333]
    width = (max(start_len) + steps) // size + 1
    table = torch.randperm(seqs * width, generator=g).to(torch.int32).view(seqs, width)
    cache = kb.PagedCache.empty({"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}[fmt], seqs * width, size, hkv, dh)
    for s, n in enumerate(start_len):
        pos = torch.arange(n)
        slots = (table[s, pos // size] * size + (pos % size).int()).cuda()
        if n:
            cache.write(torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(), torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(), slots)
    table_d, q_start = table.cuda(), i32(list(range(seqs + 1)))
    freq = torch.from_numpy(kb.rope_frequencies(dh)[0]).cuda()
    head = torch.randn(hq * dh, vocab, generator=g).cuda() * 0.05
    feeds = [torch.randn(seqs, hq + 2 * hkv, dh, generator=g).bfloat16().cuda() for _ in range(steps)]
    uniforms = [torch.rand(seqs, generator=g).cuda() for _ in range(steps)]
    top_k, temp = i32([0, 5, 1, 300, 0]), torch.tensor([1.0, 0.7, 1.0, 2.0, 0.0], device="cuda")
    logits_of = lambda out: out.flatten(1).float() @ head

    class Step:
        def __init__(self):
            self.qkv, self.u = feeds[0].clone(), uniforms[0].clone()
            self.pos, self.slots, self.lens = i32([0] * seqs), i32([-1] * seqs), i32([1] * seqs)
            self.out = torch.empty(seqs, hq, dh, dtype=torch.bfloat16, device="cuda")
            self.tokens, self.probs = i32([0] * seqs), torch.zeros(seqs, device="cuda")
            self.logits = torch.zeros(seqs, vocab, device="cuda")
            self.ws_a = torch.empty(kb.paged_attention_workspace_bytes(hq, cache, seqs), dtype=torch.uint8, device="cuda")
            self.ws_s = torch.empty(kb.sample_workspace_bytes(seqs, vocab), dtype=torch.uint8, device="cuda")

        def feed(self, t):
            lens = [n + t for n in start_len]
            self.qkv.copy_(feeds[t])
            self.u.copy_(uniforms[t])
            self.pos.copy_(torch.tensor(lens))
            self.slots.copy_(torch.tensor([int(table[s, n // size]) * size + n % size for s, n in enumerate(lens)]))
            self.lens.copy_(torch.tensor(lens) + 1)

        def attend(self):
            q, k, v = self.qkv[:, :hq], self.qkv[:, hq:hq + hkv], self.qkv[:, hq + hkv:]
            kb.rope_rows(q, k, self.pos, freq)
            cache.write(k, v, self.slots)
            kb.paged_attention(q, cache, q_start, self.lens, table_d, out=self.out, workspace=self.ws_a)

        def choose(self):
            kb.sample(self.logits, self.u, temp, top_k, tokens=self.tokens, probs=self.probs, workspace=self.ws_s)

    eager, want = Step(), []
    for t in range(steps):
        eager.feed(t)
        eager.attend()
        eager.logits.copy_(logits_of(eager.out))
        eager.choose()
        want.append([x.clone() for x in (eager.out, eager.logits, eager.tokens, eager.probs)])
    step = Step()
    side = torch.cuda.Stream()
    step.feed(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):                       # (kernels are loaded before the capture)
        step.attend()
        step.choose()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        step.attend()
    with torch.cuda.graph(graphs[1]):
        step.choose()
    for t in range(steps):
        step.feed(t)
        graphs[0].replay()
        step.logits.copy_(logits_of(step.out))
        graphs[1].replay()
        torch.cuda.synchronize()
        for a, b in zip((step.out, step.logits, step.tokens, step.probs), want[t]):
            assert torch.equal(a, b), t


def test_calls_on_other_streams_and_at_the_same_time():
    """Two streams, a workspace each; the tensors were made on a third."""
    hq, hkv, dh, n = 4, 2, 64, 2000
    g = torch.Generator().manual_seed(5)
    cache = kb.PagedCache.empty(torch.bfloat16, 130, 16, hkv, dh)
    slots = torch.arange(n, dtype=torch.int32, device="cuda")
    cache.write(torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(), torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(), slots)
    table = torch.arange(130, dtype=torch.int32, device="cuda")[None]
    qs = [torch.randn(m, hq, dh, generator=g).bfloat16().cuda() for m in (1, 300)]
    logits, u = torch.randn(3, 40000, generator=g).cuda(), torch.rand(3, generator=g).cuda()
    args = [(q, cache, i32([0, len(q)]), i32([n]), table) for q in qs]
    want = [kb.paged_attention(*a) for a in args] + [kb.sample(logits, u)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(3):
        outs = [torch.empty_like(w) for w in want]
        ws = [torch.empty(kb.paged_attention_workspace_bytes(hq, cache, 1), dtype=torch.uint8, device="cuda") for _ in qs]
        ws.append(torch.empty(kb.sample_workspace_bytes(3, 40000), dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        for i in range(2):
            kb.paged_attention(*args[i], out=outs[i], workspace=ws[i], stream=streams[i])
        kb.sample(logits, u, tokens=outs[2], workspace=ws[2], stream=streams[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("as_handle", [False, True])
def test_what_a_call_allocates_belongs_to_its_stream(as_handle):
    """Results and workspaces of calls that wait on a busy stream, while the current one takes and fills memory of their sizes"""
    hq, hkv, dh, n = 4, 2, 64, 3000
    g = torch.Generator().manual_seed(6)
    cache = kb.PagedCache.empty(torch.bfloat16, 190, 16, hkv, dh)
    cache.write(torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(), torch.randn(n, hkv, dh, generator=g).bfloat16().cuda(),
                torch.arange(n, dtype=torch.int32, device="cuda"))
    table = torch.arange(190, dtype=torch.int32, device="cuda")[None]
    q = torch.randn(40, hq, dh, generator=g).bfloat16().cuda()
    logits, u = torch.randn(3, 60000, generator=g).cuda(), torch.rand(3, generator=g).cuda()
    args = (q, cache, i32([0, 40]), i32([n]), table)
    want = [kb.paged_attention(*args), kb.sample(logits, u)]
    sizes = [kb.paged_attention_workspace_bytes(hq, cache, 1), kb.sample_workspace_bytes(3, 60000), q.numel() * 2, 12]
    a = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            busy = a
            for _ in range(20):
                busy = a @ a
        s = side.cuda_stream if as_handle else side
        got = [kb.paged_attention(*args, stream=s), kb.sample(logits, u, stream=s)]
        filled = [torch.full((size,), 255, dtype=torch.uint8, device="cuda") for size in sizes]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and all((f == 255).all() for f in filled)
