"""Attention of the recompute path with scores far beyond what a binary32 exponent resolves: still a softmax."""
import numpy as np
import pytest
import torch

import keep_synth as ks
from gpu_util import Problem, to_np
from paper_2602_23592_amd import binding as kb

pytestmark = pytest.mark.gpu

SHAPE = ks.ModelShape(1, 512, 4, 2, 128, 512, 64, 1.0e6, 1e-6, "bf16")


@pytest.mark.parametrize("path", [kb.KEEP_KERNELS_AUTO, kb.KEEP_KERNELS_GENERIC], ids=["mfma", "generic"])
@pytest.mark.parametrize("power", [5, 10, 11, 12, 14, 16, 30, 55])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_scores_of_any_finite_size(path, power, sign):
    """Queries and keys are their biases, 2^power everywhere, turned to their positions.  A row's own key is then its nearest by
    some 2 % of the score (the sum of 1 - cos over the pairs, one position apart), so it takes the whole softmax; with the
    opposite sign the first row sees only itself and every row stays finite."""
    pb = Problem(SHAPE, [300, 60], 40, random_cache=True)
    w = pb.layers_d[0]
    w["wq"].zero_(), w["wk"].zero_()
    w["bq"].fill_(2.0 ** power), w["bk"].fill_(sign * 2.0 ** power)
    ctx = pb.context(path)
    assert ctx.uses_mfma == (path == kb.KEEP_KERNELS_AUTO)
    kc, vc = pb.empty_cache()
    n = pb.n_tokens
    x_out = torch.empty((n, SHAPE.hidden), dtype=torch.bfloat16, device="cuda")
    ctx.recompute_layer(pb.prompt(), 0, [0, 1], None, x_out, kc[0], vc[0])
    o = ctx.read_layer_state(kb.KEEP_STATE_ATTN_OUT, n).astype(np.float64).reshape(n, 4, 128)
    lse = ctx.read_layer_state(kb.KEEP_STATE_LSE, n).astype(np.float64)
    k, v = to_np(kc[0]), to_np(vc[0])
    assert np.isfinite(o).all() and np.isfinite(lse).all()
    own = sign * (k * k).sum(-1).repeat(2, -1) * 128 ** -0.5
    rows = slice(0, n if sign > 0 else 1)
    # the probability and the result are rounded to bf16; queries and keys are the same rounded numbers
    assert (np.abs(o - v.repeat(2, 1))[rows] <= (2.0 ** -8 + 2.0 ** -8 + 2.0 ** -16) * np.abs(v.repeat(2, 1))[rows]).all()
    assert (np.abs(lse - own)[rows] <= 2.0 ** -16 * np.abs(own)[rows]).all()
