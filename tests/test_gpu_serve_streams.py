"""Tensors that are dropped behind a serving call on a stream of its own, while the current stream takes and fills their memory."""
import pytest
import torch

from paper_2602_23592_amd import binding as kb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("as_handle", [False, True])
def test_inputs_may_be_dropped_behind_the_call(as_handle):
    hq, hkv, dh, n, rows, vocab = 4, 2, 64, 3000, 40, 60000
    g = torch.Generator().manual_seed(6)
    randn = lambda *shape: torch.randn(*shape, generator=g)
    host = dict(k=randn(n, hkv, dh).bfloat16(), v=randn(n, hkv, dh).bfloat16(), q=randn(rows, hq, dh).bfloat16(), x=randn(3, vocab),
                u=torch.rand(3, generator=g), slots=torch.arange(n, dtype=torch.int32), pos=torch.arange(rows, dtype=torch.int32),
                freq=torch.from_numpy(kb.rope_frequencies(dh)[0]), start=torch.tensor([0, rows], dtype=torch.int32),
                lens=torch.tensor([n], dtype=torch.int32), table=torch.arange(190, dtype=torch.int32)[None],
                k_top=torch.tensor([5, 0, 40], dtype=torch.int32), temp=torch.tensor([0.5, 1.0, 2.0]))

    def step(stream):
        dev = lambda name: host[name].cuda()
        cache = kb.PagedCache.empty(torch.int8, 190, 16, hkv, dh)
        cache.write(dev("k"), dev("v"), dev("slots"), stream=stream)
        q, _ = kb.rope_rows(dev("q"), None, dev("pos"), dev("freq"), stream=stream)
        out = kb.paged_attention(q, cache, dev("start"), dev("lens"), dev("table"), stream=stream)
        return out, kb.sample(dev("x"), dev("u"), dev("temp"), dev("k_top"), stream=stream)

    want = step(None)
    torch.cuda.synchronize()
    a = torch.randn(4096, 4096, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            busy = a
            for _ in range(20):
                busy = a @ a
        got = step(side.cuda_stream if as_handle else side)
        # (zeros: whatever a call still read of them would be lengths, pages, slots and numbers of its range)
        filled = [torch.zeros_like(t, device="cuda") for t in host.values() for _ in range(2)]
        filled += [torch.zeros(190, hkv, 16, dh, dtype=torch.int8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and all((f == 0).all() for f in filled)
