"""Refusals of the paged cache's and the sampler's entry points (no GPU needed):
each is reported before any launch, with a message."""
import ctypes

import pytest

from paper_2607_21291_gb300 import build as B
from paper_2607_21291_gb300 import synth as S


@pytest.fixture(scope="module")
def A():
    B.build()
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


P = 4096   # an aligned address; nothing reads it


def cache(A, **kw):
    c = dict(k=P, v=P, k_scale=None, v_scale=None, n_pages=10, page_size=16, store=A.KV_SAME)
    c.update(kw)
    return A._PagedCache(**c)


def batch(A, **kw):
    b = dict(starts=P, lens=P, table=P, n_rows=4, B=2, max_new=2, max_pages=8)
    b.update(kw)
    return A._PagedBatch(**b)


WS = 1 << 40   # bytes the calls are told they have


def attention(A, c, b, shape=S.QWEN25_1_5B, q=P, ld=None, out=P, ws=P, ws_bytes=WS):
    cfg = A.make_cfg(shape)
    return A.lib().adadsf_paged_attention(ctypes.byref(cfg), ctypes.byref(c), ctypes.byref(b), q,
                                          shape.q_dim if ld is None else ld, out, ws, ws_bytes, None)


def append(A, c, b, shape=S.QWEN25_1_5B, qkv=P, tab=P, n_pos=100, pos=None, q_out=None, ws=P, ws_bytes=WS):
    cfg = A.make_cfg(shape)
    return A.lib().adadsf_paged_append(ctypes.byref(cfg), ctypes.byref(c), ctypes.byref(b), qkv, tab, n_pos, pos, q_out,
                                       ws, ws_bytes, None)


def read(A, c, b, shape=S.QWEN25_1_5B, k=P, v=P, ws=P, ws_bytes=WS):
    cfg = A.make_cfg(shape)
    return A.lib().adadsf_paged_read(ctypes.byref(cfg), ctypes.byref(c), ctypes.byref(b), k, v, ws, ws_bytes, None)


def test_cache_and_batch(A):
    bad, not_here = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED
    wrong = [(dict(page_size=24), {}, not_here), (dict(page_size=256), {}, not_here), (dict(n_pages=0), {}, bad),
             (dict(store=2), {}, bad), (dict(k=None), {}, bad), (dict(v=P + 8), {}, bad),
             (dict(store=A.KV_I8), {}, bad), (dict(store=A.KV_I8, k_scale=P, v_scale=P + 4), {}, bad),
             (dict(n_pages=2 ** 31 - 1), {}, not_here),
             ({}, dict(B=-1), bad), ({}, dict(B=0), bad), ({}, dict(n_rows=-1), bad), ({}, dict(n_rows=2 ** 31), not_here),
             ({}, dict(max_new=-1), bad), ({}, dict(max_pages=0), bad), ({}, dict(max_pages=2 ** 30), not_here),
             ({}, dict(starts=None), bad), ({}, dict(lens=P + 2), bad), ({}, dict(table=None), bad)]
    for call in (attention, append, read):
        for c, b, status in wrong:
            assert call(A, cache(A, **c), batch(A, **b)) == status, (call, c, b)
            assert A.adadsf_last_error()
        assert call(A, cache(A), batch(A), shape=S.QWEN25_1_5B.replace(head_dim=96)) == not_here
        assert call(A, cache(A), batch(A), ws=None) == bad
        assert call(A, cache(A), batch(A), ws=P + 16) == bad
        assert call(A, cache(A), batch(A), ws_bytes=128) == A.ERR_WORKSPACE_TOO_SMALL
        assert call(A, cache(A), batch(A, n_rows=0, B=0)) == A.OK        # nothing to do
        cfg = A.make_cfg(S.QWEN25_1_5B)
        name = {attention: "adadsf_paged_attention", append: "adadsf_paged_append", read: "adadsf_paged_read"}[call]
        args = {attention: (P, 1536, P), append: (P, P, 100, None, None), read: (P, P)}[call]
        assert getattr(A.lib(), name)(ctypes.byref(cfg), None, None, *args, P, WS, None) == bad


def test_operands(A):
    c, b = cache(A), batch(A)
    bad = A.ERR_INVALID_ARG
    assert attention(A, c, b, q=None) == attention(A, c, b, q=P + 8) == attention(A, c, b, out=None) == bad
    assert attention(A, c, b, ld=1528) == attention(A, c, b, ld=1540) == bad
    assert append(A, c, b, qkv=None) == append(A, c, b, tab=None) == append(A, c, b, n_pos=0) == bad
    assert append(A, c, b, pos=P + 1) == append(A, c, b, q_out=P + 8) == bad
    assert read(A, c, b, k=None) == read(A, c, b, v=P + 4) == bad


def test_workspace_size(A):
    cfg = A.make_cfg(S.QWEN25_7B)
    f = A.lib().adadsf_paged_attention_workspace_size
    n = f(ctypes.byref(cfg), ctypes.byref(cache(A)), ctypes.byref(batch(A)))
    assert n >= 256 and n % 256 == 0
    assert f(ctypes.byref(cfg), ctypes.byref(cache(A, page_size=20)), ctypes.byref(batch(A))) == 0
    assert "page_size" in A.adadsf_last_error()


def test_sample(A):
    def call(x=P, ld=100, B=2, V=100, dtype=A.F32, t=None, k=None, p=None, m=None, u=P, token=P, lp=None):
        return A.lib().adadsf_sample(x, ld, B, V, dtype, t, k, p, m, u, token, lp, None)
    bad = A.ERR_INVALID_ARG
    for kw in (dict(x=None), dict(x=P + 2), dict(ld=99), dict(B=-1), dict(V=0), dict(dtype=7), dict(u=None),
               dict(token=None), dict(t=P + 2), dict(k=P + 1), dict(lp=P + 3)):
        assert call(**kw) == bad, kw
        assert A.adadsf_last_error()
    assert call(V=397313, ld=397313) == A.ERR_UNSUPPORTED
    assert call(B=0) == A.OK


def test_rope_table(A):
    cfg = A.make_cfg(S.QWEN25_1_5B)
    f = A.lib().adadsf_rope_table
    assert f(ctypes.byref(cfg), -1, P, None) == f(ctypes.byref(cfg), 4, None, None) == A.ERR_INVALID_ARG
    assert f(ctypes.byref(cfg), 0, None, None) == A.OK


def test_a_cache_of_another_shape_is_refused(A, monkeypatch):
    """A cache that was made for other key/value heads, another head size or type than the call's configuration is refused
    by the binding before anything else is looked at: its pages would be read and written out of bounds."""
    import torch
    monkeypatch.setattr(A, "_dev", lambda t, name: None)   # host tensors will do: nothing is launched
    shape = S.QWEN25_1_5B
    cfg = A.make_cfg(shape)
    i32 = dict(dtype=torch.int32)
    b = A.PagedBatch(torch.zeros(2, **i32), torch.zeros(1, **i32), torch.zeros(1, 4, **i32), 1, 1)
    x = torch.zeros(1, shape.qkv_dim, dtype=torch.bfloat16)
    q, kv = x[:, :shape.q_dim], x[:, :shape.kv_dim]
    for store in (A.KV_SAME, A.KV_I8):
        c = A.paged_cache(cfg, 3, 16, store, device="cpu")
        others = [shape.replace(n_kv_heads=4), shape.replace(n_kv_heads=1), shape.replace(head_dim=64)]
        if store == A.KV_SAME:
            others.append(shape.replace(dtype="f32"))
        for other in others:
            wrong = A.make_cfg(other)
            for call in (lambda: A.adadsf_paged_append(wrong, c, b, x, None, None, q, ws=x),
                         lambda: A.adadsf_paged_read(wrong, c, b, kv, kv, ws=x),
                         lambda: A.adadsf_paged_attention(wrong, c, b, q, q, ws=x),
                         lambda: A.adadsf_paged_attention(wrong, c, b, q, q)):
                with pytest.raises(ValueError, match="cache"):
                    call()
    with pytest.raises(ValueError, match="k_out"):           # an 8-bit cache serves either type: only the operand is wrong
        A.adadsf_paged_read(A.make_cfg(shape.replace(dtype="f32")), A.paged_cache(cfg, 3, 16, A.KV_I8, device="cpu"), b, kv, kv, ws=x)
