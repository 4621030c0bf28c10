"""keep_rope_rows against the 64-bit oracle: layouts, parts of a head, types, strides, positions near and far."""
import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb

pytestmark = pytest.mark.gpu


def bound(x, y, n_rot, dtype, interleaved):
    """Cosine, sine and both products are rounded to binary32 (twice each, half a step 2^-24), then the sum, then the result
    to its type; angles are good to 2^-53 of their size."""
    x1, x2 = (x[..., 0:n_rot:2], x[..., 1:n_rot:2]) if interleaved else (x[..., :n_rot // 2], x[..., n_rot // 2:n_rot])
    pair = np.abs(x1) + np.abs(x2)
    b = np.zeros_like(y)
    if interleaved:
        b[..., 0:n_rot:2] = b[..., 1:n_rot:2] = pair
    else:
        b[..., :n_rot // 2] = b[..., n_rot // 2:n_rot] = pair
    return 1.3 * 4 * 2.0 ** -24 * b + torch.finfo(dtype).eps / 2 * np.abs(y) * (dtype != torch.float32) + 1e-30


def run(rows, hq, hkv, dh, rot, dtype, inter, positions, in_place=False, pad=0, shift=0, scaling="plain"):
    """q and k lie in one buffer of fused rows, `pad` values apart and `shift` from an aligned address"""
    g = torch.Generator().manual_seed(rows * 7 + dh)
    width = (hq + hkv) * dh + pad
    buf = torch.randn(rows * width + shift, generator=g).to(dtype).cuda()[shift:].view(rows, width)
    q, k = buf[:, :hq * dh].unflatten(1, (hq, dh)), buf[:, hq * dh:(hq + hkv) * dh].unflatten(1, (hkv, dh))
    before = buf.clone()
    freq, mag = kb.rope_frequencies(rot, 1e6, ["plain", "linear", "base", "parts"].index(scaling), 4.0, 32768)
    pos = torch.tensor(positions, dtype=torch.int32)
    out = torch.full((rows, hq + hkv, dh), 7.0, dtype=dtype, device="cuda")
    kw = {} if in_place else {"q_out": out[:, :hq], "k_out": out[:, hq:]}
    qo, ko = kb.rope_rows(q if hq else None, k if hkv else None, pos.cuda(), torch.from_numpy(freq).cuda(),
                          layout=int(inter), magnitude=mag, **{n: t for n, t in kw.items() if (hq if n[0] == "q" else hkv)})
    torch.cuda.synchronize()
    x = before[:, :(hq + hkv) * dh].unflatten(1, (hq + hkv, dh)).double().cpu().numpy()
    want = so.rope(x, positions, freq, inter, np.float64(np.float32(mag)))
    got = torch.cat([t for t in (qo, ko) if t is not None], 1).double().cpu().numpy()
    assert (np.abs(got - want) <= bound(x, want, rot, dtype, inter)).all(), np.abs(got - want).max()
    assert np.array_equal(got[..., rot:], x[..., rot:])
    if in_place:
        assert torch.equal(buf[:, (hq + hkv) * dh:], before[:, (hq + hkv) * dh:])
    else:
        assert torch.equal(buf, before)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("inter", [False, True], ids=["half", "interleaved"])
@pytest.mark.parametrize("dh,rot", [(128, 128), (128, 64), (64, 64), (80, 32), (256, 256), (16, 2), (9, 6), (128, 100)])
def test_layouts(dtype, inter, dh, rot):
    run(5, 4, 2, dh, rot, dtype, inter, [0, 1, 77, 4096, 131071])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("in_place,pad,shift", [(True, 0, 0), (True, 128, 0), (False, 64, 0), (True, 3, 0), (False, 0, 1), (True, 0, 5)])
def test_strides_addresses_and_in_place(dtype, in_place, pad, shift):
    run(7, 6, 2, 64, 32, dtype, False, [5, 4, 3, 2, 1, 0, 9], in_place, pad, shift)
    run(3, 6, 2, 64, 32, dtype, True, [5, 4, 3], in_place, pad, shift)


@pytest.mark.parametrize("scaling", ["plain", "linear", "base", "parts"])
def test_far_and_negative_positions(scaling):
    # at position 2^31 - 1 a double angle of pair 0 is good to 2^-22
    run(6, 2, 1, 64, 64, torch.bfloat16, False, [-1, -40000, 1 << 20, 16777217, (1 << 31) - 1, -(1 << 31)], scaling=scaling)
    run(4, 2, 1, 64, 64, torch.float32, False, [-1, -40000, 1 << 20, 16777217], scaling=scaling)


def test_queries_or_keys_alone_and_many_rows():
    run(3, 0, 2, 64, 64, torch.float32, False, [1, 2, 3])
    run(3, 2, 0, 64, 64, torch.float32, False, [1, 2, 3])
    # the launch of four rows per workgroup, with rows left over
    n, dh = 8193, 32
    x = torch.randn(n, 2, dh, generator=torch.Generator().manual_seed(1))
    f, _ = kb.rope_frequencies(dh, 1e4)
    pos = torch.arange(n, dtype=torch.int32).flip(0).contiguous()
    y, _ = kb.rope_rows(x.cuda(), None, pos.cuda(), torch.from_numpy(f).cuda(), q_out=torch.empty_like(x, device="cuda"))
    z = torch.view_as_complex(torch.stack([x[..., :16], x[..., 16:]], -1).double()) * torch.polar(
        torch.ones(n, 1, 16, dtype=torch.float64), pos.double()[:, None, None] * torch.from_numpy(f))
    want = torch.cat([z.real, z.imag], -1).numpy()
    assert (np.abs(y.double().cpu().numpy() - want) <= bound(x.double().numpy(), want, dh, torch.float32, False)).all()


def test_turning_back_restores_the_keys():
    """A group's keys at its place in a prompt, taken back to group-local positions."""
    f, _ = kb.rope_frequencies(128)
    f = torch.from_numpy(f).cuda()
    k = torch.randn(300, 8, 128, generator=torch.Generator().manual_seed(2)).cuda()
    pos = torch.full((300,), 31000, dtype=torch.int32, device="cuda")
    _, a = kb.rope_rows(None, k, pos, f, k_out=torch.empty_like(k))
    _, b = kb.rope_rows(None, a, -pos, f, k_out=torch.empty_like(k))
    # two turns, each off by at most 4 * 2^-24 of the pair's two values (see bound); a turn keeps their length
    pair = (k[..., :64].abs() + k[..., 64:].abs()).repeat(1, 1, 2)
    assert ((b - k).abs() <= 1.3 * 4 * 2.0 ** -24 * pair * 2.5).all()


def test_binding_refuses():
    q = torch.zeros(4, 2, 64, device="cuda")
    pos, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.ones(32, dtype=torch.float64, device="cuda")
    for args, kw in (((q, q.bfloat16(), pos, f), {}), ((q, None, pos[:3], f), {}), ((q, None, pos.long(), f), {}),
                     ((q, None, pos, f.float()), {}), ((q, None, pos.cpu(), f), {}), ((None, None, pos, f), {}),
                     ((q.transpose(1, 2), None, pos, f), {}), ((q, None, pos, f), {"q_out": q[:, :1]}),
                     ((q[:1].expand(4, 2, 64), None, pos, f), {}), ((q, None, pos, f), {"layout": 9})):
        with pytest.raises(kb.KeepError) as e:
            kb.rope_rows(*args, **kw)
        assert e.value.status == kb.KEEP_ERR_INVALID_ARG
