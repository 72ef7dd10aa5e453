"""Steps of torch work and library calls on a stream of the caller's, while the
current one is busy: the same numbers as on the current stream."""
import pytest
import torch

from paper_2607_21291_gb300 import synth as S
from tests import helpers as H

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


def used_side():
    """A side stream whose pool holds memory of ones."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        held = [torch.full((m,), 255, dtype=torch.uint8, device="cuda") for m in (1 << 28, *[1 << 20] * 8, *[1024] * 8)]
        del held
    torch.cuda.synchronize()
    return side


def test_router_step(A):
    from paper_2607_21291_gb300 import align
    shape, B, T, K = S.PYTHIA_70M.replace(n_layers=1), 2, 96, 48
    td = H.tdtype(shape)
    start = A.to_device(H.host_layer(shape, 51), td)
    real = H.to_dev(S.round_to(S.hidden(51, B, T, shape.d), shape.dtype), td)
    cfg = A.make_cfg(shape)
    h_dense = real.clone()
    A.adadsf_sparse_layer_forward(cfg, start, h_dense, T)

    def step(x, stream):
        w = {k: v.clone() for k, v in start.items()}
        return align.router_alignment_step(cfg, w, x, h_dense, K, 3000.0, stream=stream), w

    want_loss, want = step(real, None)
    side, x = used_side(), torch.empty_like(real)
    for _ in range(3):
        x.fill_(1.0)
        torch.cuda._sleep(50_000_000)
        x.copy_(real)
        loss, w = step(x, side)
        assert loss == want_loss
        for k in want:
            assert torch.equal(w[k], want[k]), k


def test_calibration(A):
    from paper_2607_21291_gb300.calibrate import calibrate
    shape, B, T = S.PYTHIA_70M.replace(n_layers=3), 2, 64
    td = H.tdtype(shape)
    layers = [A.to_device(H.host_layer(shape, 7, l), td) for l in range(shape.n_layers)]
    model = A.DeviceModel(A.make_cfg(shape), layers, A.to_device(H.host_extra(shape, 7), td))
    real = torch.from_numpy(S.token_ids(3, B, T, shape.vocab)).cuda()
    want = calibrate(model, real, 0.5)
    side, ids = used_side(), torch.empty_like(real)
    for _ in range(3):
        ids.fill_(0)
        torch.cuda._sleep(50_000_000)
        ids.copy_(real)
        for got, ref in zip(calibrate(model, ids, 0.5, stream=side), want):
            assert (got == ref).all()


@pytest.mark.parametrize("inside", [False, True])
def test_ends_captured(A, inside):
    """A step in a graph, on the captured stream or (inside) on another one that joins the capture for it; replayed on other
    ids, beside eager steps on the side stream."""
    from paper_2607_21291_gb300 import align
    d, V, n = 128, 700, 90
    cfg = A.make_cfg(S.PYTHIA_70M.replace(d=d, vocab=V, dtype="bf16"))
    g = torch.Generator(device="cuda").manual_seed(5)
    w = {"embed": torch.randn(V, d, generator=g, device="cuda").bfloat16(), "final_w": torch.ones(d, device="cuda").bfloat16(),
         "final_b": torch.zeros(d, device="cuda").bfloat16()}
    draws = [torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32) for _ in range(3)]
    target = torch.roll(draws[0], 3).contiguous()
    target[:9] = -1
    want = [align.ends_gradients(cfg, w, ids, target) for ids in draws]
    side, ids = torch.cuda.Stream(), draws[0].clone()
    align.ends_gradients(cfg, w, ids, target, stream=side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, grads = align.ends_gradients(cfg, w, ids, target, stream=side if inside else None)
    for new, (ref_loss, ref) in zip(draws, want):
        ids.copy_(new)
        graph.replay()
        eager_loss, eager = align.ends_gradients(cfg, w, ids, target, stream=side)
        assert torch.equal(loss, ref_loss) and torch.equal(eager_loss, ref_loss)
        for k in ref:
            assert torch.equal(grads[k], ref[k]) and torch.equal(eager[k], ref[k]), k


def test_stream_by_handle(A):
    """A call and a step on an object that has a stream's handle alone."""
    from paper_2607_21291_gb300 import align
    side = used_side()

    class Handle:
        cuda_stream = side.cuda_stream

    d, V, n = 64, 300, 40
    cfg = A.make_cfg(S.PYTHIA_70M.replace(d=d, vocab=V, dtype="f32"))
    g = torch.Generator(device="cuda").manual_seed(6)
    w = {"embed": torch.randn(V, d, generator=g, device="cuda"), "final_w": torch.ones(d, device="cuda"),
         "final_b": torch.zeros(d, device="cuda")}
    ids = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    want_loss, want = align.ends_gradients(cfg, w, ids, ids)
    out = torch.empty(n, d, device="cuda")
    torch.cuda.synchronize()
    A.adadsf_embed_forward(ids, w["embed"], out, stream=Handle())
    loss, grads = align.ends_gradients(cfg, w, ids, ids, stream=Handle())
    assert torch.equal(out, w["embed"][ids.long()]) and torch.equal(loss, want_loss)
    for k in want:
        assert torch.equal(grads[k], want[k]), k
