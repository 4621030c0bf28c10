"""What the serving entry points refuse, before anything touches a device (no GPU needed; pointers are never followed)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import serve_oracle as so
from paper_2602_23592_amd import binding as kb

ARG, SHAPE, WORKSPACE = kb.KEEP_ERR_INVALID_ARG, kb.KEEP_ERR_SHAPE, kb.KEEP_ERR_WORKSPACE
P = 0x100000          # an address, aligned to everything


def text():
    return kb.load_library().keep_last_error(None).decode()


@pytest.mark.parametrize("scaling,name", [(0, "plain"), (1, "linear"), (2, "base"), (3, "parts")])
@pytest.mark.parametrize("rot", [2, 10, 64, 128])
def test_frequencies_match_oracle(scaling, name, rot):
    f, m = kb.rope_frequencies(rot, 1e6, scaling, 4.0, 32768, 32.0, 1.0)
    ref, rm = so.rope_frequencies(rot, 1e6, name, 4.0, 32768, 32.0, 1.0)
    assert np.allclose(f, ref, rtol=1e-13, atol=0) and m == np.float32(rm)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=-2), dict(theta=0.0), dict(theta=math.inf),
                                dict(theta=math.nan), dict(scaling=4), dict(scaling=-1), dict(scaling=1, factor=0.5),
                                dict(scaling=2, factor=math.nan), dict(scaling=3, trained_len=0),
                                dict(scaling=3, fast=1.0, slow=1.0), dict(scaling=3, slow=-1.0)])
def test_frequencies_refuse(kw):
    with pytest.raises(kb.KeepError) as e:
        kb.rope_frequencies(**{"rot_dim": 8, "factor": 2.0, **kw})
    assert e.value.status == ARG and "keep_rope_frequencies" in str(e.value)


def _rope(q=P, q_out=P, k=P + 4096 * 4, k_out=P + 4096 * 4, pos=P, freq=P, **kw):
    d = dict(dtype=0, n_rows=4, n_q_heads=4, n_kv_heads=2, head_dim=64, rot_dim=64, layout=0, magnitude=1.0, q_in_stride=256,
             q_out_stride=256, k_in_stride=128, k_out_stride=128)
    d.update(kw)
    return kb.load_library().keep_rope_rows(C.byref(kb.RopeRowsDesc(**d)), q, q_out, k, k_out, pos, freq, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), ARG), (dict(layout=2), ARG), (dict(n_rows=-1), ARG), (dict(n_q_heads=0, n_kv_heads=0), ARG),
    (dict(n_kv_heads=-1), ARG), (dict(head_dim=0), SHAPE), (dict(head_dim=1025), SHAPE), (dict(rot_dim=0), ARG),
    (dict(rot_dim=5), ARG), (dict(rot_dim=66), ARG), (dict(q_in_stride=255), ARG), (dict(k_out_stride=0), ARG),
    (dict(q=None), ARG), (dict(k_out=None), ARG), (dict(pos=None), ARG), (dict(freq=None), ARG), (dict(q=P + 2), ARG),
    (dict(q_out=P + 1024), ARG),                            # overlaps its input
    (dict(q_out_stride=300), ARG),                          # in place, other stride
    (dict(n_q_heads=1 << 20, head_dim=1024, q_in_stride=1 << 30, q_out_stride=1 << 30), SHAPE)])
def test_rope_refuses(kw, status):
    assert _rope(**kw) == status and text().startswith("keep_rope_rows")


def test_calls_without_rows_do_nothing():
    lib = kb.load_library()
    assert _rope(n_rows=0, q=None, k=None, q_out=None, k_out=None, pos=None, freq=None) == kb.KEEP_OK
    for call in (lib.keep_cache_write, lib.keep_cache_read):
        assert call(C.byref(_cache()), 0, None, None, 0, 128, None, None) == kb.KEEP_OK
    assert _attend(n_rows=0, q=None) == kb.KEEP_OK and _attend(n_seqs=0, table=None) == kb.KEEP_OK
    assert _sample(n_rows=0, logits=None) == kb.KEEP_OK
    assert lib.keep_rope_rows(None, P, P, P, P, P, P, None) == ARG
    assert lib.keep_cache_write(None, 0, P, P, 1, 128, P, None) == ARG
    assert lib.keep_paged_attention(None, C.byref(_cache()), P, P, P, P, P, None, P, 1 << 40, None) == ARG
    assert lib.keep_sample(None, P, P, None, None, None, None, P, None, P, 1 << 40, None) == ARG


def _cache(**kw):
    d = dict(format=kb.KEEP_CACHE_INT8, n_pages=10, page_size=16, n_kv_heads=2, head_dim=64, page_stride=2048, head_stride=1024,
             token_stride=64, k=P, v=P, k_scale=P, v_scale=P)
    d.update(kw)
    return kb.PagedCacheDesc(**d)


BAD_CACHES = [
    (dict(format=4), ARG), (dict(format=-1), ARG), (dict(n_pages=0), ARG), (dict(page_size=0), ARG), (dict(n_kv_heads=0), ARG),
    (dict(head_dim=72), SHAPE), (dict(head_dim=272, token_stride=272), SHAPE), (dict(head_dim=0), SHAPE),
    (dict(n_pages=1 << 30, page_size=2), SHAPE), (dict(n_kv_heads=5000), SHAPE),
    (dict(token_stride=72), ARG), (dict(token_stride=48), ARG), (dict(head_stride=512), ARG), (dict(page_stride=1024), ARG),
    (dict(head_stride=-1024), ARG), (dict(k=None), ARG), (dict(v=None), ARG), (dict(k=P + 8), ARG), (dict(k_scale=None), ARG),
    (dict(v_scale=P + 2), ARG), (dict(format=kb.KEEP_CACHE_F32, token_stride=66), ARG)]


@pytest.mark.parametrize("kw,status", BAD_CACHES)
def test_bad_caches_are_refused_by_every_call(kw, status):
    lib, c = kb.load_library(), _cache(**kw)
    for call in (lib.keep_cache_write, lib.keep_cache_read):
        assert call(C.byref(c), 0, P, P, 1, 1 << 20, P, None) == status and text().startswith("keep_cache_")
    assert _attend(cache=c) == status and text().startswith("keep_paged_attention")
    assert lib.keep_paged_attention_workspace_bytes(C.byref(c), 4 * max(1, c.n_kv_heads), 1) == 0


@pytest.mark.parametrize("kw", [dict(), dict(token_stride=128, head_stride=64), dict(n_kv_heads=1, head_stride=0),
                                dict(page_size=1, token_stride=0, head_stride=64, page_stride=128),
                                dict(n_pages=1, page_stride=0), dict(format=kb.KEEP_CACHE_BF16, k_scale=None, v_scale=None)])
def test_layouts_that_a_cache_may_have(kw):
    assert kb.load_library().keep_paged_attention_workspace_bytes(C.byref(_cache(**kw)), 4, 1) > 0


@pytest.mark.parametrize("args,status", [
    ((2, P, P, 1, 128, P), ARG), ((0, None, P, 1, 128, P), ARG), ((0, P, None, 1, 128, P), ARG), ((0, P, P, 1, 128, None), ARG),
    ((0, P, P, -1, 128, P), ARG), ((0, P, P, 1, 124, P), ARG), ((0, P, P, 1, 130, P), ARG), ((1, P, P, 1, 132, P), ARG),
    ((0, P + 8, P, 1, 128, P), ARG)])
def test_write_and_read_refuse(args, status):
    lib = kb.load_library()
    for call in (lib.keep_cache_write, lib.keep_cache_read):
        assert call(C.byref(_cache()), *args, None) == status


def _attend(cache=None, q=P, out=P + (1 << 20), start=P, lens=P, table=P, lse=None, ws=P, ws_bytes=1 << 40, **kw):
    d = dict(dtype=0, n_seqs=3, n_rows=5, n_q_heads=4, max_pages=4, window=0, scale=0.0, q_stride=256, out_stride=256)
    d.update(kw)
    return kb.load_library().keep_paged_attention(C.byref(kb.PagedAttentionDesc(**d)), C.byref(cache or _cache()), q, start, lens,
                                                  table, out, lse, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=3), ARG), (dict(n_seqs=-1), ARG), (dict(n_seqs=4097), SHAPE), (dict(n_rows=-1), ARG), (dict(window=-1), ARG),
    (dict(n_q_heads=3), ARG), (dict(n_q_heads=0), ARG), (dict(max_pages=0), ARG), (dict(max_pages=1 << 28), ARG),
    (dict(scale=math.nan), ARG), (dict(scale=math.inf), ARG), (dict(q_stride=252), ARG), (dict(out_stride=258), ARG),
    (dict(n_rows=1 << 30), SHAPE), (dict(q=None), ARG), (dict(out=None), ARG), (dict(start=None), ARG), (dict(lens=None), ARG),
    (dict(table=None), ARG), (dict(ws=None), ARG), (dict(ws=P + 64), ARG), (dict(q=P + 4), ARG), (dict(out=P + 1024), ARG),
    (dict(ws_bytes=4096), WORKSPACE)])
def test_attention_refuses(kw, status):
    assert _attend(**kw) == status and text().startswith("keep_paged_attention")


def test_workspace_bytes_refuse():
    lib = kb.load_library()
    for hq, n in ((3, 1), (0, 1), (4, -1), (4, 4097)):
        assert lib.keep_paged_attention_workspace_bytes(C.byref(_cache()), hq, n) == 0
    for n, v in ((-1, 5), (65536, 5), (1, 0), (1, (1 << 20) + 1)):
        assert lib.keep_sample_workspace_bytes(n, v) == 0
    assert lib.keep_sample_workspace_bytes(65535, 1 << 20) > 0


def _sample(logits=P, uniform=P, tokens=P, ws=P, ws_bytes=1 << 40, **kw):
    d = dict(dtype=0, n_rows=2, vocab=100, row_stride=100)
    d.update(kw)
    return kb.load_library().keep_sample(C.byref(kb.SampleDesc(**d)), logits, uniform, None, None, None, None, tokens, None, ws,
                                         ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=5), ARG), (dict(n_rows=-1), ARG), (dict(n_rows=65536), ARG), (dict(vocab=0), ARG), (dict(row_stride=99), ARG),
    (dict(vocab=(1 << 20) + 1, row_stride=1 << 21), SHAPE), (dict(logits=None), ARG), (dict(uniform=None), ARG),
    (dict(tokens=None), ARG), (dict(ws=None), ARG), (dict(ws=P + 4), ARG), (dict(logits=P + 2), ARG),
    (dict(ws_bytes=16), WORKSPACE)])
def test_sample_refuses(kw, status):
    assert _sample(**kw) == status and text().startswith("keep_sample")


def test_decode_sampled_needs_a_context():
    assert kb.load_library().keep_decode_sampled(None, P, P, P, P, P, 1, 1, 1, None, None, None, None, None) == ARG


@pytest.mark.parametrize("off", [0, 4, 252, -4, -252, 512 * 3 + 200, 260, 512 * 2 - 100])
def test_slices_of_the_same_rows_that_share_an_element(off):
    """rows of 256 values, 512 apart, each 4 bytes: an output that begins `off` values behind the input"""
    far = P + (1 << 22)
    if off:
        assert _rope(q_in_stride=512, q_out_stride=512, q=far, q_out=far + 4 * off) == ARG and "overlap" in text()
    assert _attend(q_stride=512, out_stride=512, q=far, out=far + 4 * off) == ARG and "overlap" in text()


@pytest.mark.parametrize("kw", [
    dict(k=P), dict(k_out=P), dict(k=P, k_out=P), dict(q_out=P + 4096 * 4), dict(k_out=P + 512),                # separate rows
    dict(q_in_stride=512, q_out_stride=512, k_in_stride=512, k_out_stride=512, k=P + 1020, k_out=P + 1020),   # slices of fused rows
    dict(q_in_stride=512, q_out_stride=512, k_in_stride=512, k_out_stride=512, k=P + 1024, k_out=P + 2040),
    dict(n_rows=1, k=P + 1020, k_out=P + 1020)])
def test_rope_refuses_queries_and_keys_that_share_an_element(kw):
    assert _rope(**kw) == ARG and "overlap" in text()


class _NoCall:
    """A library that answers every call, and counts them"""
    calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return kb.KEEP_OK
        return call


@pytest.mark.parametrize("n_new,forced,ok", [(3, [], False), (3, [5], False), (64, [1] * 62, False), (1, [], True), (3, [5, 6], True),
                                             (3, [5, 6, 7], True), (3, None, True)])
def test_forced_tokens_shorter_than_what_the_library_reads_are_refused(n_new, forced, ok):
    t = torch.zeros(2, 4)
    for sampled in (False, True):
        ctx = object.__new__(kb.KeepContext)
        ctx.lib, ctx.handle = _NoCall(), None
        call = (lambda: ctx.decode_sampled(t, t, t, t, t, 1, [0.5] * n_new, forced_tokens=forced)) if sampled else \
            (lambda: ctx.decode(t, t, t, t, t, 1, n_new, forced_tokens=forced))
        if ok:
            call()
            assert ctx.lib.calls == 1
        else:
            with pytest.raises(kb.KeepError, match="forced_tokens"):
                call()
            assert ctx.lib.calls == 0


@pytest.mark.parametrize("stream", [None, 0, 64])
def test_tensors_on_the_host_are_refused(stream):
    """like any other wrong tensor, whatever the stream"""
    x, pos, freq = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    for call in (lambda: kb.rope_rows(x, None, pos, freq, stream=stream), lambda: kb.sample(x[:, 0], x[:, 0, 0].clone(), stream=stream),
                 lambda: kb.PagedCache(x[None], x[None].clone())):
        with pytest.raises(kb.KeepError):
            call()
