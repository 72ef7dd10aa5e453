"""Refusals of the losses at the head, the norms and the embedding (no GPU
needed): each is reported before any launch, with a message; and what the
binding checks of tensors."""
import ctypes

import pytest
import torch

from paper_2607_21291_gb300 import build as B


@pytest.fixture(scope="module")
def A():
    B.build()
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


P = 4096        # an aligned address; nothing reads it
WS = 1 << 44    # bytes the calls are told they have
BF, F = 1, 0


def head(A, backward=False, **kw):
    a = dict(h=P, w=2 * P, target=P, n=10, d=64, V=100, dtype=BF, loss=P, lse=P, acc=None, g=None, dh=4 * P, dw=3 * P, add=0, ws=P,
             ws_bytes=WS)
    a.update(kw)
    base = (a["h"], a["w"], a["target"], a["n"], a["d"], a["V"], a["dtype"])
    if backward:
        return A.lib().adadsf_head_loss_backward(*base, a["lse"], a["g"], a["dh"], a["dw"], a["add"], a["ws"], a["ws_bytes"], None)
    return A.lib().adadsf_head_loss(*base, a["loss"], a["lse"], a["acc"], a["ws"], a["ws_bytes"], None)


def distill(A, backward=False, **kw):
    a = dict(h=P, w=2 * P, idx=P, logit=P, k=4, temp=1.0, n=10, d=64, V=100, dtype=BF, loss=P, lse=P, acc=None, g=None, dh=4 * P,
             dw=3 * P, add=0, ws=P, ws_bytes=WS)
    a.update(kw)
    base = (a["h"], a["w"], a["idx"], a["logit"], a["k"], a["temp"], a["n"], a["d"], a["V"], a["dtype"])
    if backward:
        return A.lib().adadsf_distill_loss_backward(*base, a["lse"], a["g"], a["dh"], a["dw"], a["add"], a["ws"], a["ws_bytes"], None)
    return A.lib().adadsf_distill_loss(*base, a["loss"], a["lse"], a["acc"], a["ws"], a["ws_bytes"], None)


def test_head_refusals(A):
    bad, not_here, small = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED, A.ERR_WORKSPACE_TOO_SMALL
    both = [(dict(dtype=2), bad), (dict(n=-1), bad), (dict(d=0), bad), (dict(V=0), bad), (dict(d=60), not_here),
            (dict(d=65544), not_here), (dict(dtype=F, d=62), not_here), (dict(n=2 ** 22 + 1), not_here),
            (dict(V=2 ** 24 + 1), not_here), (dict(h=None), bad), (dict(h=P + 8), bad), (dict(w=None), bad), (dict(w=P + 2), bad),
            (dict(lse=None), bad), (dict(lse=P + 2), bad), (dict(ws=None), bad), (dict(ws=P + 16), bad),
            (dict(ws_bytes=1000), small)]
    for call in (head, distill):
        for backward in (False, True):
            for kw, status in both:
                assert call(A, backward, **kw) == status, (call, backward, kw)
                assert A.adadsf_last_error()
        for kw, status in [(dict(loss=P + 2), bad), (dict(acc=P + 4), bad), (dict(loss=None, acc=P), bad)]:
            assert call(A, False, **kw) == status, kw
        for kw, status in [(dict(dh=None, dw=None), bad), (dict(dh=P + 8), bad), (dict(dw=P + 2), bad), (dict(add=2), bad),
                           (dict(g=P + 1), bad), (dict(dw=2 * P), bad), (dict(dw=P), bad), (dict(dh=P), bad),
                           (dict(dh=2 * P), bad)]:
            assert call(A, True, **kw) == status, kw
        assert call(A, False, n=0) == A.OK
    for backward in (False, True):
        assert head(A, backward, target=None) == bad and head(A, backward, target=P + 1) == bad
        for kw, status in [(dict(idx=None), bad), (dict(logit=None), bad), (dict(idx=P + 2), bad), (dict(k=0), bad),
                           (dict(k=1025), not_here), (dict(temp=0.0), bad), (dict(temp=-1.0), bad), (dict(temp=float("nan")), bad),
                           (dict(temp=float("inf")), bad), (dict(temp=1e-45), bad)]:
            assert distill(A, backward, **kw) == status, kw


def test_head_workspace(A):
    size = A.adadsf_head_workspace_size
    bf, f32 = torch.bfloat16, torch.float32
    assert size(0, 64, 100, bf) > 0
    for n, d, V in ((1, 64, 100), (24, 768, 50304), (4096, 3584, 152064), (65536, 512, 50304)):
        assert size(n, d, V, bf) >= n * d * 2 and size(n, d, V, f32) >= (n + V) * d * 6
        # all of the logits in fp32 do not fit in it
        if n * V > 2 ** 28:
            assert size(n, d, V, bf) < 4 * n * V
    assert size(100, 64, 1000, bf, 64) > size(100, 64, 1000, bf, 1)
    for wrong in ((-1, 64, 100, bf, 1), (1, 4, 100, bf, 1), (1, 64, 0, bf, 1), (1, 64, 100, bf, 0), (1, 64, 100, bf, 2000)):
        with pytest.raises(A.AdadsfError):
            size(*wrong)


def norm_fw(A, **kw):
    a = dict(x=P, w=P, b=P, n=10, d=64, dtype=BF, eps=1e-5, rms=0, y=P, mean=P, rstd=P)
    a.update(kw)
    return A.lib().adadsf_norm_forward(*a.values(), None)


def norm_bw(A, **kw):
    a = dict(dy=P, x=P, w=P, mean=P, rstd=P, add=None, n=10, d=64, dtype=BF, rms=0, dx=P, dw=P, db=P, acc=0, ws=P, ws_bytes=WS)
    a.update(kw)
    return A.lib().adadsf_norm_backward(*a.values(), None)


def test_norm_refusals(A):
    bad, not_here = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED
    for call in (norm_fw, norm_bw):
        for kw, status in [(dict(dtype=3), bad), (dict(n=-1), bad), (dict(d=0), bad), (dict(d=60), not_here), (dict(d=8200), not_here),
                           (dict(dtype=F, d=62), not_here), (dict(n=2 ** 31), not_here), (dict(x=None), bad), (dict(x=P + 4), bad),
                           (dict(w=None), bad), (dict(rstd=None), bad), (dict(rstd=P + 2), bad), (dict(mean=None), bad),
                           (dict(rms=1), bad)]:
            assert call(A, **kw) == status, (call, kw)
            assert A.adadsf_last_error()
    for kw in (dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(b=None), dict(b=P + 2),
               dict(y=None), dict(rms=1, mean=None), dict(rms=1, b=None)):
        assert norm_fw(A, **kw) == bad, kw
    for kw in (dict(dy=None), dict(dx=None), dict(dx=P + 8), dict(add=P + 8), dict(dw=P + 1), dict(db=P + 2), dict(acc=2),
               dict(ws=None), dict(ws=P + 8), dict(rms=1, mean=None), dict(rms=1, db=None)):
        assert norm_bw(A, **kw) == bad, kw
    assert norm_bw(A, ws_bytes=256) == A.ERR_WORKSPACE_TOO_SMALL
    assert norm_fw(A, n=0) == A.OK and norm_bw(A, n=0, acc=1) == A.OK
    with pytest.raises(A.AdadsfError):
        A.adadsf_norm_backward_workspace_size(10, 8200)


def embed_fw(A, **kw):
    a = dict(ids=P, n=10, table=P, V=100, d=64, dtype=BF, scale=1.0, out=P, ws=P, ws_bytes=WS)
    a.update(kw)
    return A.lib().adadsf_embed_forward(*a.values(), None)


def embed_bw(A, **kw):
    a = dict(ids=P, dy=P, n=10, V=100, d=64, dtype=BF, scale=1.0, table=2 * P, acc=0, ws=P, ws_bytes=WS)
    a.update(kw)
    return A.lib().adadsf_embed_backward(*a.values(), None)


def test_embed_refusals(A):
    bad, not_here = A.ERR_INVALID_ARG, A.ERR_UNSUPPORTED
    for call in (embed_fw, embed_bw):
        for kw, status in [(dict(dtype=2), bad), (dict(n=-1), bad), (dict(V=0), bad), (dict(d=0), bad), (dict(d=60), not_here),
                           (dict(dtype=F, d=62), not_here), (dict(d=65544), not_here), (dict(n=2 ** 30 + 1), not_here),
                           (dict(V=2 ** 27 + 1), not_here), (dict(scale=float("nan")), bad), (dict(scale=float("inf")), bad),
                           (dict(ids=None), bad), (dict(ids=P + 2), bad), (dict(table=None), bad), (dict(table=P + 8), bad),
                           (dict(ws=None), bad), (dict(ws=P + 16), bad), (dict(ws_bytes=128), A.ERR_WORKSPACE_TOO_SMALL)]:
            assert call(A, **kw) == status, (call, kw)
            assert A.adadsf_last_error()
    assert embed_fw(A, out=None) == bad and embed_fw(A, out=P + 4) == bad
    for kw in (dict(dy=None), dict(dy=P + 8), dict(acc=2), dict(table=P)):
        assert embed_bw(A, **kw) == bad, kw
    assert embed_fw(A, n=0) == A.OK and embed_bw(A, n=0, acc=1) == A.OK
    with pytest.raises(A.AdadsfError):
        A.adadsf_embed_backward_workspace_size(2 ** 31, 100, 64)


def test_binding_refuses_tensors(A):
    """Tensors of the host, of another type or shape: a ValueError before the library is called."""
    h, w = torch.zeros(4, 64), torch.zeros(10, 64)
    v, t = torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        A.adadsf_head_loss(h, w, t, v, v)
    with pytest.raises(ValueError):
        A.adadsf_distill_loss(h, w, torch.zeros(3, 2, dtype=torch.int32), torch.zeros(4, 2), 1.0, v, v)
    with pytest.raises(ValueError):
        A.adadsf_norm_forward(h, torch.zeros(64), None, h, 1e-5, None, v)
    with pytest.raises(ValueError):
        A.adadsf_norm_backward(h, h, torch.zeros(64), v, h)
    with pytest.raises(ValueError):
        A.adadsf_embed_forward(t, w, h)
    with pytest.raises(ValueError):
        A.adadsf_embed_backward(t, h, w)


@pytest.mark.parametrize("d,V,dtype", [(3584, 152064, "bf16"), (2048, 50304, "bf16"), (512, 50304, "f32"), (64, 300, "bf16"),
                                       (8, 2 ** 20, "bf16"), (1536, 151936, "f32")])
def test_head_workspace_serves_fewer_rows(A, d, V, dtype):
    """A workspace for the longest batch is large enough for every shorter one."""
    size = A.adadsf_head_workspace_size
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    last = 0
    for n in sorted({0, 1, 80, 81, 128, 129, *range(255, 20000, 256), *range(256, 20000, 256), *range(257, 20000, 256),
                     *(r + o for r in (2 ** 15, 2 ** 16, 65537 + 256, 2 ** 18, 2 ** 20, 2 ** 22 - 256) for o in (-1, 0, 1, 256))}):
        now = size(n, d, V, dt)
        assert now >= last, (n, now, last)
        last = now
    assert size(1000, d, V, dt, 64) <= size(2000, d, V, dt, 64)


@pytest.mark.parametrize("V,d", [(152064, 3584), (50304, 768), (300, 64), (40000, 4), (2 ** 27, 8), (1000, 8200)])
def test_embed_workspace_serves_fewer_tokens(A, V, d):
    """A workspace for the longest batch is large enough for every shorter one."""
    size = A.adadsf_embed_backward_workspace_size
    last = 0
    steps = sorted({0, 1, *range(7, 9000, 13), *range(9000, 200000, 511), *(k * 2 ** 20 + o for k in (1, 2, 3, 8, 64) for o in (-1, 0, 1, 2048)),
                    *(per + o for per in (9, 19, 32, 38, 2432, 4864, 77824, 77824 // 3, 311296, 311296 // 14, 77824 // 14, 9962, 311296 // 33)
                      for o in (-1, 0, 1, 2))})
    for n in steps:
        now = size(n, V, d)
        assert now >= last, (n, now, last)
        last = now


def test_head_gradients_of_no_rows(A):
    """An empty batch with a frozen head: the hidden gradient is an empty tensor, whose address is NULL."""
    for call in (head, distill):
        assert call(A, True, n=0, dh=None, dw=None) == A.OK
        assert call(A, True, n=0, dh=None, dw=None, h=None, lse=None) == A.OK
        assert call(A, True, n=1, dh=None, dw=None) == A.ERR_INVALID_ARG


def apart(sizes):
    """Addresses of tensors that lie one behind the other, 4096 bytes or more between them."""
    at, out = 1 << 20, {}
    for name, size in sizes.items():
        out[name] = at
        at += (size // 4096 + 2) * 4096
    return out


def meetings(sizes, outs, allowed=()):
    """One output moved onto another tensor's first byte, its last 16, and so that its own last 16 meet it."""
    base = apart(sizes)
    for o in outs:
        for other in sizes:
            if other == o:
                continue
            for at in (base[other], base[other] + (sizes[other] - 16) // 16 * 16, base[other] - (sizes[o] - 16) // 16 * 16):
                if at == base[other] and (o, other) in allowed:
                    continue
                yield {**base, o: at}, o, other


@pytest.mark.parametrize("dtype", [BF, F])
def test_overlaps_are_refused(A, dtype):
    n, d, V, k = 10, 64, 100, 4
    row = d * (2 if dtype == BF else 4)
    refused = lambda status, o, other: (status == A.ERR_INVALID_ARG and "overlaps" in A.adadsf_last_error(), o, other, A.adadsf_last_error())
    ws = A.adadsf_head_workspace_size(n, d, V, torch.bfloat16 if dtype == BF else torch.float32, k)
    kinds = [(head, dict(h=n * row, w=V * row, target=n * 4)), (distill, dict(h=n * row, w=V * row, idx=n * k * 4, logit=n * k * 4))]
    for call, reads in kinds:
        for backward, more, outs in ((False, dict(loss=n * 4, lse=n * 4, acc=16), ("loss", "lse", "acc")),
                                     (True, dict(lse=n * 4, g=n * 4, dh=n * row, dw=V * row), ("dh", "dw"))):
            for kw, o, other in meetings({**reads, **more, "ws": 4096}, outs):
                got = refused(call(A, backward, dtype=dtype, ws_bytes=ws, **kw), o, other)
                assert got[0], got
    rows = dict(x=n * row, w=row, mean=n * 4, rstd=n * 4)
    for kw, o, other in meetings({**rows, "b": row, "y": n * row}, ("y", "mean", "rstd"), allowed=[("y", "x")]):
        got = refused(norm_fw(A, dtype=dtype, **kw), o, other)
        assert got[0], got
    sizes = {**rows, "dy": n * row, "add": n * row, "dx": n * row, "dw": d * 4, "db": d * 4, "ws": 4096}
    for kw, o, other in meetings(sizes, ("dx", "dw", "db"), allowed=[("dx", "dy"), ("dx", "add"), ("dx", "x")]):
        got = refused(norm_bw(A, dtype=dtype, **kw), o, other)
        assert got[0], got
    for kw, o, other in meetings(dict(ids=n * 4, table=V * row, out=n * row, ws=256), ("out",)):
        got = refused(embed_fw(A, dtype=dtype, **kw), o, other)
        assert got[0], got
    for kw, o, other in meetings(dict(ids=n * 4, dy=n * row, table=V * row, ws=4096), ("table",)):
        got = refused(embed_bw(A, dtype=dtype, **kw), o, other)
        assert got[0], got
