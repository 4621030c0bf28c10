"""keep_sample at the ends of its arguments' ranges."""
import pytest
import torch

from paper_2602_23592_amd import binding as kb
from test_gpu_sample import check, mixture

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_the_largest_vocabulary(dtype):
    n, vocab = 4, kb.KEEP_SAMPLE_MAX_VOCAB
    x = 3.0 * torch.randn(n, vocab, generator=torch.Generator().manual_seed(1))
    x[3] = 0.5                                            # (every token weighs 2^40: the sum is 2^60)
    check(x.to(dtype), **mixture(n, 1))
    check(x.to(dtype), [0.3, 0.999999, 0.0, 0.7])


def test_the_most_rows_of_a_call():
    x = torch.randn(65535, 5, generator=torch.Generator().manual_seed(2)).bfloat16()
    u = torch.rand(65535, generator=torch.Generator().manual_seed(3))
    probs = torch.empty(65535, device="cuda")
    got = kb.sample(x.cuda(), u.cuda(), probs=probs).cpu().long()
    # by the distribution itself: the weights that rank before the token, and with it, enclose u (double arithmetic, 2^-40 each)
    p = torch.softmax(x.double(), -1)
    ids = torch.arange(5)
    before = lambda v, i: (v[:, :, None] < v[:, None, :]) | ((v[:, :, None] == v[:, None, :]) & (i[:, None] > i[None]))
    first = (before(x.float(), ids).double() * p[:, None, :]).sum(-1).gather(1, got[:, None])[:, 0]
    mine = p.gather(1, got[:, None])[:, 0]
    assert (first <= u.double() + 1e-11).all() and (u.double() <= first + mine + 1e-11).all()
    assert ((probs.cpu().double() - mine).abs() <= 2.0 ** -23 * mine).all()
