"""GPU parity of training's two ends against 64-bit forms: cross entropy and
distillation at the LM head, norms and embedding, each with its gradients, and
a run of them together.

Bounds. u = 2^-24 is half a step of fp32 (one rounding), b = 2^-8 of bf16; a sum
of m terms in fp32, in any order, is off by at most m 2u of the sum of their
absolute values (2u a step: the tensor cores do not round their sums to nearest)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U, B16 = 2.0 ** -24, 2.0 ** -8
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def A():
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def randn(g, *shape, std=1.0):
    return torch.randn(*shape, generator=g, device="cuda") * std


def within(got, ref, bound, what):
    """Element by element; bound a tensor or a number."""
    got, ref = got.double(), ref.double()
    assert torch.isfinite(got).all(), what
    over = (got - ref).abs() - bound
    assert float(over.max()) <= 0, (what, float(over.max()), float((got - ref).abs().max()), int((over > 0).sum()))


# ------------------------------------------------------------------ losses at the head
def head_inputs(n, d, V, dtype, seed=0, std=1.0):
    g = gen(seed * 1000 + n + d + V)
    h = randn(g, n, d, std=std).to(DT[dtype])
    w = randn(g, V, d, std=0.3 / math.sqrt(d) * 4).to(DT[dtype])
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    if n > 2:
        target[torch.rand(n, generator=g, device="cuda") < 0.3] = -1
        target[n // 2] = V - 1
    gl = torch.rand(n, generator=g, device="cuda") + 0.1
    return h, w, target, gl


def want_of(target, V):
    """Targets as rows of weights over the classes, and whether a row has one."""
    used = (target >= 0) & (target < V)
    want = torch.zeros(target.numel(), V, dtype=torch.float64, device="cuda")
    want[used, target[used].long()] = 1.0
    return want, used


def teacher_want(idx, logit, V, temp):
    there = (idx >= 0) & (idx < V) & (logit > -math.inf)
    used = there.any(-1)
    t = (logit.double() / temp).masked_fill(~there, -math.inf)
    p = torch.where(used[:, None], torch.softmax(torch.where(used[:, None], t, 0.0), -1), 0.0)
    want = torch.zeros(idx.shape[0], V, dtype=torch.float64, device="cuda")
    want.scatter_add_(1, idx.clamp(0, V - 1).long(), torch.where(there, p, 0.0))
    return want, used, torch.special.xlogy(p, p).sum(-1)


def terms(m, f32, grad):
    """Additions that lose up to 2u each in a sum of m products. A step of the tensor cores adds 16 products and the sum so
    far, 17 terms; where fp32 comes of it, a sum is of chunks of at most 32 steps (bf16 logits 64), added in fp32; bf16
    gradients are one chain."""
    if grad and not f32:
        return m + 64
    steps = 32 if f32 else 64
    return min(m, 17 * steps) + m / (16 * steps) + 64


class Ref:
    """The losses and gradients in 64 bits, and how far the kernels may be from them."""

    def __init__(self, h, w, want, used, ent, gl, temp, k):
        bf = h.dtype == torch.bfloat16
        products = 6 if not bf else 1   # of parts, with what is left out of them: 2^-22 of a product
        h, w, gl = h.double(), w.double(), (torch.ones(h.shape[0], device="cuda") if gl is None else gl).double()
        h = torch.where(used[:, None], h, 0.0)
        d, V = w.shape[1], w.shape[0]
        z = h @ w.T / temp
        size = (h.abs() @ w.abs().T).amax(-1) / temp
        self.lse = torch.where(used, torch.logsumexp(z, -1), 0.0)
        mass = want.sum(-1)
        self.loss = torch.where(used, temp ** 2 * (ent + mass * self.lse - (want * z).sum(-1)), 0.0)
        # a logit: a sum of d products, and its scale; an exponential: 2^-22 and its argument's two roundings; the sum of
        # them: 16 terms a chain, 4 chunks, and the records (V / 128 over 32 threads, then 32)
        far = z.abs().amax(-1) + self.lse.abs()
        e_z = (2 * terms(products * d, not bf, False) + 4) * U * size
        e_lse = e_z + 4 * U + 4 * U * far + 2 * U * (64 + V / 4096 + 32) + 2 * U * self.lse.abs()
        self.e_lse = torch.where(used, e_lse, 0.0)
        # targets: a sum of k weights times logits, the entropy's like it
        self.e_loss = torch.where(used, temp ** 2 * (e_lse + e_z + (2 * k + 16) * U * (far + 2 * ent.abs() + 1)), 0.0)
        q = torch.exp(z - self.lse[:, None])
        s = torch.where(used, gl * temp, 0.0)[:, None]
        G = (q - want) * s
        e_z = (2 * terms(products * d, not bf, True) + 4) * U * size   # of the backward pass's logits
        e_q = (e_z + e_lse + 4 * U + 4 * U * far)[:, None] * q * s.abs() + 4 * U * (q + want) * s.abs()
        e_g = e_q + (B16 * (G.abs() + e_q) if bf else 2 * U * G.abs())
        self.dh, self.dw = G @ w, G.T @ h
        out = B16 if bf else U
        n = h.shape[0]
        t_v, t_n = terms(products * V, not bf, True), terms(products * n, not bf, True)
        self.e_dh = (e_g + 2 * U * t_v * G.abs()) @ w.abs()
        self.e_dh += out * (self.dh.abs() + self.e_dh)
        self.e_dw = (e_g + 2 * U * t_n * G.abs()).T @ h.abs()
        self.e_dw += out * (self.dw.abs() + self.e_dw)
        # roundings of G are independent: their part of a gradient has a 2-norm of about b / sqrt(3) (sum G^2 W^2)^(1/2);
        # twice that, and the outputs' own roundings
        g2 = G * G
        self.n_dh = out * self.dh.norm() + 2 * out / 3 ** 0.5 * (g2 @ (w * w)).sum().sqrt() + (e_q @ w.abs()).norm() * 0.5
        self.n_dw = out * self.dw.norm() + 2 * out / 3 ** 0.5 * (g2.T @ (h * h)).sum().sqrt() + (e_q.T @ h.abs()).norm() * 0.5
        if not bf:   # rounding of long fp32 sums, for which the bound of a chain is all there is
            self.n_dh += self.e_dh.norm()
            self.n_dw += self.e_dw.norm()
        else:
            self.n_dh += 2 * U * (t_v * (G.abs() @ w.abs())).norm()
            self.n_dw += 2 * U * (t_n * (G.abs().T @ h.abs())).norm()

    def check(self, loss, lse, dh, dw, base=None):
        if lse is not None:
            within(lse, self.lse, self.e_lse, "lse")
        if loss is not None:
            within(loss, self.loss, self.e_loss, "loss")
        if dh is not None:
            within(dh, self.dh, self.e_dh, "dh")
            assert float((dh.double() - self.dh).norm()) <= float(self.n_dh), "dh's norm"
        if dw is not None:
            b = 0.0 if base is None else base.double()
            out = B16 if dw.dtype == torch.bfloat16 else U
            more = 0.0 if base is None else 2 * out * b.abs()
            within(dw, self.dw + b, self.e_dw + more, "dw")
            if base is None:
                assert float((dw.double() - self.dw).norm()) <= float(self.n_dw), "dw's norm"


def ce(A, h, w, target, gl=None, grads=True, ws=None, stream=None):
    n = h.shape[0]
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    acc = torch.zeros(2, dtype=torch.float64, device="cuda")
    A.adadsf_head_loss(h, w, target, loss, lse, acc=acc, ws=ws, stream=stream)
    dh = dw = None
    if grads:
        dh, dw = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
        A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_h=dh, grad_w=dw, ws=ws, stream=stream)
    return loss, lse, acc, dh, dw


HEADS = [(1, 64, 100, "bf16"), (3, 8, 1, "bf16"), (24, 768, 5003, "bf16"), (130, 200, 257, "bf16"), (257, 520, 1000, "bf16"),
         (300, 768, 1280, "bf16"), (700, 264, 255, "bf16"), (9000, 64, 12001, "bf16"),
         (65, 64, 31, "bf16"), (97, 136, 33, "bf16"), (128, 136, 20011, "bf16"), (129, 72, 300, "bf16"),
         (33, 4, 5000, "f32"), (80, 100, 20011, "f32"), (81, 68, 300, "f32"), (40, 5124, 700, "f32"),
         (200, 5124, 700, "f32"), (40, 5128, 700, "bf16"), (200, 5128, 700, "bf16"),
         (1, 4, 1, "f32"), (5, 132, 130, "f32"), (77, 512, 3001, "f32"), (515, 100, 777, "f32"), (9000, 32, 6002, "f32")]


@pytest.mark.parametrize("n,d,V,dtype", HEADS)
def test_head_loss(A, n, d, V, dtype):
    """Sizes on both sides of tiles, boxes and k blocks; many row tiles and several pieces of the classes in the last of
    either type. Twice the same bits."""
    h, w, target, gl = head_inputs(n, d, V, dtype)
    want, used = want_of(target, V)
    ref = Ref(h, w, want, used, torch.zeros(n, dtype=torch.float64, device="cuda"), gl, 1.0, 1)
    loss, lse, acc, dh, dw = ce(A, h, w, target, gl)
    ref.check(loss, lse, dh, dw)
    assert float(acc[1]) == int(used.sum())
    assert float(acc[0]) == pytest.approx(float(loss.double().sum()), rel=1e-12, abs=1e-12)
    assert (loss[~used] == 0).all() and (lse[~used] == 0).all() and (dh[~used] == 0).all()
    again = ce(A, h, w, target, gl)
    for x, y in zip((loss, lse, dh, dw), (again[0], again[1], again[3], again[4])):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n,d,V,dtype", [(5, 136, 3000, "bf16"), (128, 64, 700, "bf16"), (130, 200, 900, "bf16"), (513, 72, 5000, "bf16"),
                                         (3000, 64, 500, "bf16"), (9000, 64, 12001, "bf16"), (81, 64, 700, "f32")])
def test_every_row_has_a_target(A, n, d, V, dtype):
    """bf16 rows are then read where they are; they may be the last of their memory."""
    h, w, target, gl = head_inputs(n, d, V, dtype)
    target = torch.randint(0, V, (n,), generator=gen(n), device="cuda", dtype=torch.int32)
    want, used = want_of(target, V)
    ref = Ref(h, w, want, used, torch.zeros(n, dtype=torch.float64, device="cuda"), gl, 1.0, 1)
    loss, lse, acc, dh, dw = ce(A, h, w, target, gl)
    ref.check(loss, lse, dh, dw)
    assert float(acc[1]) == n


def distill_inputs(n, d, V, k, dtype, seed=1):
    h, w, target, gl = head_inputs(n, d, V, dtype, seed)
    g = gen(n * k + V)
    idx = torch.randint(0, V, (n, k), generator=g, device="cuda", dtype=torch.int32)   # the same class twice now and then
    logit = randn(g, n, k, std=3.0)
    gone = torch.rand(n, k, generator=g, device="cuda") < 0.2
    idx[gone] = -1
    logit[torch.rand(n, k, generator=g, device="cuda") < 0.05] = -math.inf
    idx[target < 0] = -1
    logit[gone] = math.nan                                                             # of slots not in use
    return h, w, idx, logit, gl


def distill(A, h, w, idx, logit, temp, gl, ws=None):
    n = h.shape[0]
    loss, lse = torch.full((n,), 7.0, device="cuda"), torch.full((n,), 7.0, device="cuda")
    A.adadsf_distill_loss(h, w, idx, logit, temp, loss, lse, ws=ws)
    dh, dw = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
    A.adadsf_distill_loss_backward(h, w, idx, logit, lse, temp, grad_loss=gl, grad_h=dh, grad_w=dw, ws=ws)
    return loss, lse, dh, dw


@pytest.mark.parametrize("n,d,V,k,temp,dtype", [(1, 64, 100, 1, 1.0, "bf16"), (40, 128, 300, 7, 2.0, "bf16"),
                                                (300, 520, 1000, 64, 0.7, "bf16"), (33, 64, 70, 1024, 1.0, "bf16"),
                                                (9000, 64, 11000, 20, 4.0, "bf16"), (128, 64, 9000, 33, 1.5, "bf16"),
                                                (100, 68, 9000, 9, 1.0, "f32"), (5, 132, 130, 3, 1.0, "f32"),
                                                (200, 256, 3001, 129, 2.0, "f32"), (9000, 32, 6002, 5, 1.0, "f32")])
def test_distill_loss(A, n, d, V, k, temp, dtype):
    h, w, idx, logit, gl = distill_inputs(n, d, V, k, dtype)
    want, used, ent = teacher_want(idx, logit, V, temp)
    ref = Ref(h, w, want, used, ent, gl, temp, k)
    got = distill(A, h, w, idx, logit, temp, gl)
    ref.check(*got)
    again = distill(A, h, w, idx, logit, temp, gl)
    for x, y in zip(got, again):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_distill_of_one_class_is_cross_entropy(A, dtype):
    """One slot at temperature 1: weight 1, entropy 0; the same products and sums."""
    h, w, target, gl = head_inputs(70, 128, 500, dtype)
    loss, lse, _, dh, dw = ce(A, h, w, target, gl)
    logit = randn(gen(3), 70, 1)
    got = distill(A, h, w, target[:, None].contiguous(), logit, 1.0, gl)
    for x, y in zip(got, (loss, lse, dh, dw)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_target_reach_nothing(A, dtype):
    """Infinities and NaN in rows without a target; the others as without them, bit for bit."""
    h, w, target, gl = head_inputs(140, 128, 700, dtype)
    clean = ce(A, h, w, target, gl)
    dirty = h.clone()
    dirty[target < 0] = torch.tensor([math.nan, math.inf, -math.inf, 1e30], device="cuda", dtype=h.dtype).repeat(32)
    gl2 = torch.where(target < 0, math.nan, gl)
    got = ce(A, dirty, w, target, gl2)
    for x, y in zip(got, clean):
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_row_has_a_target(A, dtype):
    h, w, target, gl = head_inputs(300, 64, 400, dtype)
    loss, lse, acc, dh, dw = ce(A, h, w, torch.full_like(target, -100), gl)
    for x in (loss, lse, acc, dh, dw):
        assert (x == 0).all()
    none = ce(A, h[:0], w, target[:0], gl[:0])
    assert (none[4] == 0).all() and (none[2] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_rows(A, dtype):
    """An empty batch, each gradient by itself: the head's is cleared, or left where it is added to."""
    h, w, target, gl = head_inputs(3, 64, 400, dtype)
    v, idx, logit = gl[:0], target[:0, None].contiguous(), gl[:0, None].contiguous()
    calls = [lambda **kw: A.adadsf_head_loss_backward(h[:0], w, target[:0], v, grad_loss=v, **kw),
             lambda **kw: A.adadsf_distill_loss_backward(h[:0], w, idx, logit, v, 2.0, grad_loss=v, **kw)]
    for call in calls:
        call(grad_h=torch.empty_like(h[:0]))
        dw = torch.full_like(w, 7.0)
        call(grad_w=dw, accumulate_w=True)
        assert (dw == 7).all()
        call(grad_w=dw)
        assert (dw == 0).all()


def test_classes_out_of_range(A):
    h, w, target, gl = head_inputs(50, 64, 400, "bf16")
    ws = A.workspace(A.adadsf_head_workspace_size(50, 64, 400, h.dtype, 4))
    bad = target.clone()
    bad[7] = 400
    got = ce(A, h, w, bad, gl, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    bad[7] = -1
    for x, y in zip(got, ce(A, h, w, bad, gl, ws=ws)):
        assert torch.equal(x, y)
    assert A.adadsf_sync_check(ws) == A.OK
    _, _, idx, logit, _ = distill_inputs(50, 64, 400, 4, "bf16")
    idx[9] = torch.tensor([400, 2 ** 31 - 1, 3, -5], device="cuda", dtype=torch.int32)
    logit[9] = 1.0
    got = distill(A, h, w, idx, logit, 1.0, gl, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    idx[9, :2] = -1
    for x, y in zip(got, distill(A, h, w, idx, logit, 1.0, gl, ws=ws)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("n,d,V,dtype", [(300, 128, 700, "bf16"), (9000, 64, 12001, "bf16"), (200, 64, 300, "f32")])
def test_head_gradients_apart_and_added(A, n, d, V, dtype):
    """Each gradient by itself is the pair's; the head's added to what is there; no weights are weights of one."""
    h, w, target, gl = head_inputs(n, d, V, dtype)
    loss, lse, _, dh, dw = ce(A, h, w, target, gl)
    one = torch.full_like(h, 7.0)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_h=one)
    assert torch.equal(one, dh)
    two = torch.full_like(w, 7.0)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_w=two)
    assert torch.equal(two, dw)
    want, used = want_of(target, V)
    zero = torch.zeros(n, dtype=torch.float64, device="cuda")
    ref = Ref(h, w, want, used, zero, gl, 1.0, 1)
    base = randn(gen(5), V, d, std=0.2).to(h.dtype)
    two.copy_(base)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_w=two, accumulate_w=True)
    ref.check(None, None, None, two, base=base)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_h=one, grad_w=two)
    Ref(h, w, want, used, zero, None, 1.0, 1).check(None, None, one, two)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_wide_logits(A, dtype):
    """Logits of some thousands: no overflow, a loss of their size, gradients of single classes."""
    h, w, target, gl = head_inputs(60, 128, 900, dtype, std=1500.0)
    want, used = want_of(target, 900)
    ref = Ref(h, w, want, used, torch.zeros(60, dtype=torch.float64, device="cuda"), gl, 1.0, 1)
    loss, lse, _, dh, dw = ce(A, h, w, target, gl)
    assert float(ref.lse.max()) > 1000
    within(lse, ref.lse, ref.e_lse, "lse")
    within(loss, ref.loss, ref.e_loss, "loss")
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()


def test_head_gradient_is_the_losses_difference(A):
    """Against differences of the 64-bit loss, and the kernel against the same formula (fp32)."""
    n, d, V = 6, 16, 40
    h, w, target, gl = head_inputs(n, d, V, "f32")
    idx = torch.randint(0, V, (n, 5), generator=gen(1), device="cuda", dtype=torch.int32)
    logit, temp = randn(gen(2), n, 5), 1.7
    for form in ("ce", "distill"):
        if form == "ce":
            want, used = want_of(target, V)
            ent, t = torch.zeros(n, dtype=torch.float64, device="cuda"), 1.0
            _, _, _, dh, dw = ce(A, h, w, target, gl)
        else:
            want, used, ent = teacher_want(idx, logit, V, temp)
            t = temp
            _, _, dh, dw = distill(A, h, w, idx, logit, temp, gl)

        def total(hh, ww):
            z = hh @ ww.T / t
            row = t * t * (ent + want.sum(-1) * torch.logsumexp(z, -1) - (want * z).sum(-1))
            return float((torch.where(used, row, 0.0) * gl.double()).sum())

        for x, grad, other in ((h, dh, w), (w, dw, h)):
            for i, j in ((0, 0), (3, 7), (5, 15)):
                step = torch.zeros_like(x, dtype=torch.float64)
                step[i, j] = 1e-4
                xd, od = x.double(), other.double()
                hi = total(xd + step, od) if x is h else total(od, xd + step)
                lo = total(xd - step, od) if x is h else total(od, xd - step)
                # differences: 1e-8 of the third derivative, and 1e-15 of a loss of tens over 1e-4
                assert (hi - lo) / 2e-4 == pytest.approx(float(grad[i, j]), rel=2e-5, abs=2e-6)


def test_head_captured(A):
    """A forward and backward call in a graph, replayed on other inputs in the same places; a second graph on the same
    workspace behind it; calls on another stream."""
    n, d, V = 200, 128, 3000
    ws = A.workspace(A.adadsf_head_workspace_size(9000, 64, 12001, torch.bfloat16, 4))
    h, w, target, gl = head_inputs(n, d, V, "bf16")
    loss, lse = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    dh, dw = torch.empty_like(h), torch.empty_like(w)

    def step():
        A.adadsf_head_loss(h, w, target, loss, lse, ws=ws)
        A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_h=dh, grad_w=dw, ws=ws)

    big = head_inputs(1000, 64, 5000, "bf16", seed=8)
    big_out = [torch.empty(1000, device="cuda"), torch.empty(1000, device="cuda")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        A.adadsf_head_loss(big[0], big[1], big[2], *big_out, ws=ws)
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()]
    with torch.cuda.graph(graphs[0]):
        step()
    with torch.cuda.graph(graphs[1]):
        A.adadsf_head_loss(big[0], big[1], big[2], *big_out, ws=ws)
    for seed in (3, 4):
        for dst, src in zip((h, w, target, gl), head_inputs(n, d, V, "bf16", seed=seed)):
            dst.copy_(src)
        graphs[0].replay()
        graphs[1].replay()
        graphs[0].replay()
        got = [x.clone() for x in (loss, lse, dh, dw)]
        want = ce(A, h, w, target, gl)
        for x, y in zip(got, (want[0], want[1], want[3], want[4])):
            assert torch.equal(x, y)
        assert torch.equal(big_out[0], ce(A, *big[:3], grads=False)[0])


@pytest.mark.parametrize("n,dtype", [(6, "bf16"), (130, "bf16"), (6, "f32"), (130, "f32")])
def test_head_of_more_than_2_31_numbers(A, n, dtype):
    """The head and its gradient pass 2^31 elements; the classes at its end, and around the border, as the first ones."""
    d, V = 2048, 1_100_000
    g = gen(n)
    h = randn(g, n, d).to(DT[dtype])
    w = torch.empty(V, d, dtype=DT[dtype], device="cuda").normal_(0.0, 0.05, generator=g)
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    border = 2 ** 31 // d
    target[:4] = torch.tensor([0, border - 1, border, V - 1], device="cuda", dtype=torch.int32)
    loss, lse, _, dh, dw = ce(A, h, w, target)
    hd, step = h.double(), 100_000
    z = torch.cat([hd @ w[c:c + step].double().T for c in range(0, V, step)], 1)
    size = torch.stack([(hd.abs() @ w[c:c + step].double().abs().T).amax(-1) for c in range(0, V, step)]).amax(0)
    ref = torch.logsumexp(z, -1)
    products = 1 if dtype == "bf16" else 6
    # as Ref's bounds
    far = z.abs().amax(-1) + ref.abs()
    e_z = (2 * terms(products * d, dtype == "f32", False) + 4) * U * size
    e_lse = e_z + 4 * U + 4 * U * far + 2 * U * (64 + V / 4096 + 32) + 2 * U * ref.abs()
    within(lse, ref, e_lse, "lse")
    within(loss, ref - z.gather(1, target[:, None].long())[:, 0], e_lse + e_z + 18 * U * (far + 1), "loss")
    G = torch.exp(z - ref[:, None])
    e_z = (2 * terms(products * d, dtype == "f32", True) + 4) * U * size
    e_g = G * (e_z + e_lse + 8 * U + 4 * U * far)[:, None]
    G[torch.arange(n), target.long()] -= 1
    out = B16 if dtype == "bf16" else U
    e_g += 4 * U * (G.abs() + 2 * (G < 0)) + (B16 if dtype == "bf16" else 2 * U) * (G.abs() + e_g)
    t_v, t_n = terms(products * V, dtype == "f32", True), terms(products * n, dtype == "f32", True)
    ref_h, e_h = torch.zeros_like(hd), torch.zeros_like(hd)
    for c in range(0, V, step):
        wd = w[c:c + step].double()
        ref_h += G[:, c:c + step] @ wd
        e_h += (e_g[:, c:c + step] + 2 * U * t_v * G[:, c:c + step].abs()) @ wd.abs()
    within(dh, ref_h, e_h + out * (ref_h.abs() + e_h), "dh")
    for c in (0, border - 256, V - 512):
        at = slice(c, c + 512)
        ref_w, e_w = G[:, at].T @ hd, (e_g[:, at] + 2 * U * t_n * G[:, at].abs()).T @ hd.abs()
        within(dw[at], ref_w, e_w + out * (ref_w.abs() + e_w), "dw")


def test_head_of_a_million_rows(A):
    """Rows times classes of a piece pass 2^31; rows without a target among them."""
    n, d, V = 1_100_000, 64, 2100
    g = gen(11)
    h, w = randn(g, n, d).to(torch.bfloat16), randn(g, V, d, std=0.1).to(torch.bfloat16)
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    target[torch.rand(n, generator=g, device="cuda") < 0.01] = -1
    loss, lse, acc, dh, dw = ce(A, h, w, target)
    assert float(acc[1]) == int((target >= 0).sum())
    for rows in (slice(0, 300), slice(n // 2, n // 2 + 300), slice(n - 300, n)):
        want, used = want_of(target[rows], V)
        ref = Ref(h[rows], w, want, used, torch.zeros(300, dtype=torch.float64, device="cuda"), None, 1.0, 1)
        ref.check(loss[rows], lse[rows], dh[rows], None)
    total = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    for c in range(0, n, 50_000):
        at = slice(c, c + 50_000)
        z, (want, used) = h[at].double() @ w.double().T, want_of(target[at], V)
        total += ((torch.softmax(z, -1) - want) * used[:, None]).T @ h[at].double()
    # a chain of 65536 rows is 4096 steps, each of which cuts at most 2u of the sum so far; entries of either sign make the
    # sum a walk, of which the final sum holds half at a step's mean: 4096 u of it, twice that with the 17 chains' sums and
    # 2e-3 of independent roundings over 134400 entries
    short = float(((dw.double() - total) * total).sum() / total.square().sum())
    assert abs(short) <= 4096 * 2 * U, short


@pytest.mark.parametrize("n,dtype", [(20, "bf16"), (300, "bf16"), (20, "f32"), (300, "f32")])
def test_head_row_of_nan_stays_in_its_row(A, n, dtype):
    """A NaN or infinity in a row with a target: its own loss and hidden gradient, the others' bits as before."""
    h, w, target, gl = head_inputs(n, 128, 700, dtype)
    target[3], target[9] = 5, 6
    clean = ce(A, h, w, target, gl)
    h[3, 7], h[9, 11] = math.nan, math.inf
    got = ce(A, h, w, target, gl)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[3] = keep[9] = False
    for i in (0, 1, 3):
        assert torch.equal(got[i][keep], clean[i][keep])
    assert not torch.isfinite(got[0][~keep]).any() and torch.isnan(got[3][3]).all()


@pytest.mark.parametrize("n,d", [(1, 256), (20, 256), (80, 256), (81, 256), (300, 512)])
def test_head_gradients_of_sure_rows(A, n, d):
    """fp32 rows that are nearly sure of their target, at logits of a hundred: q - 1 there is a difference of numbers near 1,
    so both passes have to see the same logits. A column of ones in the head sums a row's G, which is 0 but for rounding."""
    V = 300
    g = gen(n + d)
    w = randn(g, V, d).abs() * 0.5
    h = randn(g, n, d).abs()
    target = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    w[:, 7] = 1.0
    h[:, 7] = 0.0
    z = h.double() @ w.double().T
    lift = (z.amax(-1) - z[torch.arange(n), target.long()] + 6.0) / (w[target.long()].double() ** 2).sum(-1)
    h += (lift[:, None] * w[target.long()]).float()
    h[:, 7] = 0.0
    loss, lse, _, dh, _ = ce(A, h, w, target)
    z = h.double() @ w.double().T
    ref = torch.logsumexp(z, -1)
    q = torch.exp(z - ref[:, None])
    spread = (q * (z.amax(-1, keepdim=True) - z)).sum(-1) + (q * (z - ref[:, None]).abs()).sum(-1)
    size = 2 * (1 - q[torch.arange(n), target.long()])   # the sum of |G|
    # for logits that are the same in both passes: the logarithm's rounding; arguments of the exponentials (3 roundings of either
    # pass), the exponentials (2^-22), their sums (V / 128 records of 128), logf and G's own; the sum of G in a chain
    bound = U * ref.abs() + 3 * U * spread + (4 + 4 + 8 + 8) * U + 2 * U * (64 + 32) * size + 2 * U * terms(6 * V, True, True) * size
    within(dh[:, 7], torch.zeros(n, device="cuda"), bound, "sum of G")


@pytest.mark.parametrize("n", [1, 20, 33, 64, 65, 80, 81, 200])
@pytest.mark.parametrize("d", [64, 132, 1028])
def test_head_of_one_class_has_no_gradient(A, n, d):
    """fp32: the logarithm of one class is its logit, so that q - 1 is 0 where both passes have the same logits, however these
    are added up, and nothing else where they differ by a rounding."""
    h, w, _, _ = head_inputs(n, d, 1, "f32")
    loss, lse, _, dh, dw = ce(A, h, w, torch.zeros(n, dtype=torch.int32, device="cuda"))
    for x in (loss, dh, dw):
        assert (x == 0).all()


@pytest.mark.parametrize("n", [1, 20, 127, 128, 129, 300])
@pytest.mark.parametrize("d", [64, 520, 1000, 5128])
def test_bf16_head_of_one_class_has_no_gradient(A, n, d):
    """As for fp32 above: both passes have the same bf16 logits, also where few rows' losses come from another kernel."""
    h, w, target, _ = head_inputs(n, d, 1, "bf16")
    for t in (torch.zeros_like(target), target):
        loss, lse, _, dh, dw = ce(A, h, w, t)
        for x in (loss, dh, dw):
            assert (x == 0).all()


@pytest.mark.parametrize("n", [1, 20, 128, 129, 300])
@pytest.mark.parametrize("d", [520, 2048, 5128])
def test_bf16_head_gradients_of_sure_rows(A, n, d):
    """bf16 rows that are all but sure of class 5, by products of one sign that add up to logits of some 60: q - 1 there, of
    some 1e-4, is a difference of numbers near 1. A column of ones in the head sums a row's G, which is 0 but for
    roundings; a column that only class 5 has picks its entry."""
    V = 300
    g = gen(n * 3 + d)
    w = (randn(g, V, d).abs() * (60 / (0.64 * d))).to(torch.bfloat16)
    h = randn(g, n, d).abs()
    w[:, 7], w[:, 8] = 1.0, 0.0
    w[5, 8] = 1.0
    h[:, 7:9] = 0.0
    z = h.double() @ w.double().T
    along = w[5].double().clone()
    along[7:9] = 0.0
    gap = along @ (along - w.double()).T      # by how much a step along class 5's row raises its logit over another's
    gap[5] = math.inf
    assert float(gap.min()) > 0
    lift = ((z - z[:, 5:6] + 12.0) / gap).amax(-1).clamp(min=0.0)
    h = (h + (lift[:, None] * along).float()).to(torch.bfloat16)
    h[:, 7:9] = 0.0
    loss, lse, _, dh, _ = ce(A, h, w, torch.full((n,), 5, dtype=torch.int32, device="cuda"))
    z = h.double() @ w.double().T
    ref = torch.logsumexp(z, -1)
    q = torch.exp(z - ref[:, None])
    rest = q.clone()
    rest[:, 5] = 0.0
    rest = rest.sum(-1)                       # 1 - q of class 5; the sum of |G| is twice that
    assert float(rest.max()) < 2e-3
    spread = (q * (z.amax(-1, keepdim=True) - z)).sum(-1) + (q * (z - ref[:, None]).abs()).sum(-1)
    # the same logits in both passes: as in test_head_gradients_of_sure_rows, and G's rounding to bf16
    one = U * ref.abs() + 3 * U * spread + (4 + 4 + 8 + 8) * U + 2 * U * (64 + 32) * 2 * rest
    bound = one + B16 * 2 * rest + 2 * U * terms(V, False, True) * 2 * rest
    within(dh[:, 7], torch.zeros(n, device="cuda"), (1 + B16) * bound, "sum of G")
    # the others' shares go by the logits' differences
    e_z = 2 * (2 * terms(d, False, False) + 4) * U * (h.double().abs() @ w.double().abs().T).amax(-1)
    bound = one + e_z * rest
    within(dh[:, 8], -rest, bound + 2 * B16 * (rest + bound), "G of the target")


@pytest.mark.parametrize("n", [60, 200])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (5128, "bf16"), (128, "f32"), (1028, "f32")])
def test_wide_logits_gradients(A, n, d, dtype):
    """Logits of thousands: the gradients too are as near as their sums' bounds."""
    h, w, target, gl = head_inputs(n, d, 900, dtype, std=1500.0)
    want, used = want_of(target, 900)
    ref = Ref(h, w, want, used, torch.zeros(n, dtype=torch.float64, device="cuda"), gl, 1.0, 1)
    # most entries of G lie below fp32's normal numbers, where exponentials, their shares and products are zeros: each by
    # less than 2^-126, which meets the other operand
    hd = torch.where(used[:, None], h.double().abs(), 0.0)
    ref.e_dh += 3 * 2.0 ** -126 * w.double().abs().sum(0)
    ref.e_dw += 3 * 2.0 ** -126 * hd.sum(0)
    loss, lse, _, dh, dw = ce(A, h, w, target, gl)
    assert float(ref.lse.max()) > 1000
    ref.check(loss, lse, dh, dw)


def cut_of(steps):
    """How far a long sum of like numbers falls short on average where chunks of `steps` steps of the tensor cores are added
    up in fp32: at step i a chunk holds i / steps of its sum, of which an addition cuts off less than 2^-23, half of that on
    average: 2^-24 (steps + 1) / 2 in all. The sums of the chunks are rounded to nearest, which has no mean; one rounding's
    room for them and the result. (Chunks of twice the length lose 0.7 of their own bound, as sums lie anywhere between two
    powers of two: more than this.)"""
    return U * ((steps + 1) / 2 + 1)


@pytest.mark.parametrize("n,d,dtype,steps", [(100, 5120, "bf16", 32), (400, 5120, "bf16", 32), (64, 8192, "f32", 16), (200, 8192, "f32", 16)])
def test_chunks_of_the_logits(A, n, d, dtype, steps):
    """Logits of products of one sign, which the logarithm of one class is: short by what chunks of this length lose."""
    g = gen(n + d)
    h, w = randn(g, n, d).abs().to(DT[dtype]), (randn(g, 1, d).abs() / d).to(DT[dtype])
    _, lse, _, _, _ = ce(A, h, w, torch.zeros(n, dtype=torch.int32, device="cuda"), grads=False)
    ref = (h.double() @ w.double().T)[:, 0]
    short = float(((ref - lse.double()) / ref).mean())
    more = U if dtype == "f32" else 0.0   # the three products of parts that are left out: 2^-24 of a product at most on average
    assert -U <= short <= cut_of(steps) + more, short / U


@pytest.mark.parametrize("what", ["rows", "classes"])
def test_chunks_of_the_gradients(A, what):
    """fp32 gradients as sums of one sign over many rows, and over many classes: every logit is 0, so that G is the same
    number everywhere but at the target, which meets zeros; a column with a single 1 has that number itself."""
    d = 64
    g = gen(3)
    if what == "rows":
        n, V = 8192, 2
        h, w = randn(g, n, d).abs(), torch.zeros(V, d, device="cuda")
        x = h
    else:
        n, V = 100, 8192
        h, w = torch.zeros(n, d, device="cuda"), randn(g, V, d).abs()
        w[0] = 0.0
        x = w
    x[:, 0] = 0.0
    x[5, 0] = 1.0
    _, _, _, dh, dw = ce(A, h, w, torch.zeros(n, dtype=torch.int32, device="cuda"))
    got = (dw[1:2] if what == "rows" else dh).double()
    ref = x.double().sum(0) * got[:, :1]
    assert (got[:, :1] > 0).all()
    short = float(((ref - got) / ref)[:, 1:].mean())
    assert -U <= short <= cut_of(16) + 2 * U, short / U   # the products left out, and the single one's rounding


@pytest.mark.parametrize("n,V", [(1, 31), (32, 33), (33, 64), (64, 65), (65, 4900), (80, 5000), (50, 180000)])
def test_head_gradients_of_few_rows(A, n, V):
    """fp32 rows on both sides of the zeros that products over rows need, classes on both sides of their blocks and more than a
    piece has, some rows without a target; distillation as well; each gradient by itself."""
    d = 100
    h, w, target, gl = head_inputs(n, d, V, "f32")
    want, used = want_of(target, V)
    zero = torch.zeros(n, dtype=torch.float64, device="cuda")
    ref = Ref(h, w, want, used, zero, gl, 1.0, 1)
    loss, lse, _, dh, dw = ce(A, h, w, target, gl)
    ref.check(loss, lse, dh, dw)
    one, two = torch.full_like(h, 7.0), torch.full_like(w, 7.0)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_h=one)
    A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_w=two)
    assert torch.equal(one, dh) and torch.equal(two, dw)
    h, w, idx, logit, gl = distill_inputs(n, d, V, 9, "f32")
    want, used, ent = teacher_want(idx, logit, V, 2.0)
    Ref(h, w, want, used, ent, gl, 2.0, 9).check(*distill(A, h, w, idx, logit, 2.0, gl))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_weights_of_rows(A, dtype):
    """Weights below zero and of zero; what they hold in rows without a target; all of them zero."""
    n, V = 200, 700
    h, w, target, gl = head_inputs(n, 128, V, dtype)
    gl = gl - 0.6
    gl[5], target[5] = 0.0, 3
    want, used = want_of(target, V)
    ref = Ref(h, w, want, used, torch.zeros(n, dtype=torch.float64, device="cuda"), gl, 1.0, 1)
    clean = ce(A, h, w, target, gl)
    ref.check(clean[0], clean[1], clean[3], clean[4])
    odd = gl.clone()
    odd[~used] = math.inf
    odd[(~used).nonzero()[0]] = math.nan
    got = ce(A, h, w, target, odd)
    assert torch.equal(got[3], clean[3]) and torch.equal(got[4], clean[4])
    got = ce(A, h, w, target, torch.zeros_like(gl))
    assert (got[3] == 0).all() and (got[4] == 0).all()


def test_head_workspace_of_more_rows(A):
    """One workspace for the longest batch: a shorter one in it, which takes the classes in fewer and larger pieces."""
    d, V = 64, 152064
    ws = A.workspace(A.adadsf_head_workspace_size(800, d, V, torch.bfloat16))
    for n in (800, 768):
        h, w, target, gl = head_inputs(n, d, V, "bf16")
        got, want = ce(A, h, w, target, gl, ws=ws), ce(A, h, w, target, gl)
        for x, y in zip(got, want):
            assert torch.equal(x, y)


def test_tensors_side_by_side(A):
    """All of a call's tensors and its workspace in one buffer, one ending where the next begins; the norm's gradient in
    place of its input."""
    n, d, V = 32, 64, 96
    h, w, target, gl = head_inputs(n, d, V, "bf16")
    want = ce(A, h, w, target, gl)
    size = (A.adadsf_head_workspace_size(n, d, V, torch.bfloat16) + 255) // 256 * 256
    buf, at = torch.zeros(size + (1 << 16), dtype=torch.uint8, device="cuda"), [0]

    def place(t):
        out = buf[at[0]:at[0] + t.numel() * t.element_size()].view(t.dtype).view(t.shape)
        at[0] += t.numel() * t.element_size()
        return out.copy_(t)

    h2, dh, w2, dw, t2, loss, g2, lse = (place(t) for t in (h, h, w, w, target, gl, gl, gl))
    assert at[0] % 256 == 0
    ws = buf[at[0]:at[0] + size]
    at[0] += size
    acc = place(torch.zeros(2, dtype=torch.float64, device="cuda"))
    A.adadsf_head_loss(h2, w2, t2, loss, lse, acc=acc, ws=ws)
    A.adadsf_head_loss_backward(h2, w2, t2, lse, grad_loss=g2, grad_h=dh, grad_w=dw, ws=ws)
    for x, y in zip((loss, lse, acc, dh, dw), want):
        assert torch.equal(x, y)
    for dtype, rms in (("bf16", False), ("f32", True)):
        x, wn, b, dy, add = norm_inputs(500, 768, dtype, rms, True)
        _, mean, rstd, dx, _, _ = norm(A, x, wn, b, dy, add)
        A.adadsf_norm_backward(dy, x, wn, rstd, x, mean=mean, add=add)
        assert torch.equal(x, dx)


def test_calls_at_once(A):
    """Two streams, a workspace each, calls of different kernels of every operator in flight together."""
    def work(n, d, V, dtype):
        h, w, target, gl = head_inputs(n, d, V, dtype)
        x, wn, b, dy, _ = norm_inputs(n, d, dtype, False, False)
        size = max(A.adadsf_head_workspace_size(n, d, V, h.dtype), A.adadsf_norm_backward_workspace_size(n, d),
                   A.adadsf_embed_backward_workspace_size(n, V, d))
        ws, ids = A.workspace(size), torch.randint(0, V, (n,), device="cuda", dtype=torch.int32)

        def run():
            table = torch.full_like(w, 7.0)
            A.adadsf_embed_backward(ids, h, table, ws=ws)
            return [*ce(A, h, w, target, gl, ws=ws), *norm(A, x, wn, b, dy, None, ws=ws), table]
        return run

    calls = [work(100, 256, 30000, "bf16"), work(700, 512, 9000, "f32")]
    want = [c() for c in calls]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(calls[i]())
    torch.cuda.synchronize()
    for i in range(2):
        for outs in got[i]:
            for x, y in zip(outs, want[i]):
                assert torch.equal(x, y)


def test_scratch_of_calls_on_another_stream(A):
    """Calls on a side stream without a workspace, while the current stream is busy: what they make by themselves comes from
    memory that held ones, cleared in order with their kernels."""
    n, d, V = 24, 256, 3000
    h, w, target, gl = head_inputs(n, d, V, "bf16")
    x, wn, b, dy, _ = norm_inputs(n, d, "bf16", False, False)
    ids = torch.randint(0, V, (n,), generator=gen(4), device="cuda", dtype=torch.int32)
    vectors, rows = [torch.empty(n, device="cuda") for _ in range(4)], [torch.empty_like(x) for _ in range(4)]
    dw, db, head, table = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.empty_like(w), torch.empty_like(w)
    outs = [*vectors, *rows, dw, db, head, table]

    def run(stream):
        loss, lse, mean, rstd = vectors
        y, dx, out, dh = rows
        A.adadsf_embed_forward(ids, w, out, stream=stream)
        A.adadsf_norm_forward(x, wn, b, y, 1e-5, mean, rstd, stream=stream)
        A.adadsf_head_loss(h, w, target, loss, lse, stream=stream)
        A.adadsf_head_loss_backward(h, w, target, lse, grad_loss=gl, grad_h=dh, grad_w=head, stream=stream)
        A.adadsf_norm_backward(dy, x, wn, rstd, dx, mean=mean, grad_w=dw, grad_b=db, stream=stream)
        A.adadsf_embed_backward(ids, dy, table, stream=stream)

    run(None)
    want = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        held = [torch.full((m,), 255, dtype=torch.uint8, device="cuda") for m in (1 << 28, 1 << 20, 1 << 20, 256, 256)]
        del held
    for t in outs:
        t.fill_(7)
    torch.cuda.synchronize()
    for _ in range(3):
        torch.cuda._sleep(100_000_000)
        run(side)
    torch.cuda.synchronize()
    for got, ref in zip(outs, want):
        assert torch.equal(got, ref)


# ------------------------------------------------------------------ norms
def norm_inputs(n, d, dtype, rms, res):
    g = gen(n * 7 + d)
    x = randn(g, n, d) * torch.exp(randn(g, n, 1, std=0.5)) + randn(g, 1, d, std=0.5)
    x = x.to(DT[dtype])
    w = (1 + randn(g, d, std=0.2)).to(x.dtype)
    b = None if rms else randn(g, d, std=0.2).to(x.dtype)
    dy = randn(g, n, d).to(x.dtype)
    add = randn(g, n, d).to(x.dtype) if res else None
    return x, w, b, dy, add


def norm(A, x, w, b, dy, add, eps=1e-5, ws=None, dw=None, db=None, accumulate=False):
    n, d = x.shape
    y, dx = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
    mean = None if b is None else torch.full((n,), 7.0, device="cuda")
    rstd = torch.full((n,), 7.0, device="cuda")
    dw = torch.full((d,), 7.0, device="cuda") if dw is None else dw
    db = None if b is None else torch.full((d,), 7.0, device="cuda") if db is None else db
    A.adadsf_norm_forward(x, w, b, y, eps, mean, rstd)
    A.adadsf_norm_backward(dy, x, w, rstd, dx, mean=mean, add=add, grad_w=dw, grad_b=db, accumulate=accumulate, ws=ws)
    return y, mean, rstd, dx, dw, db


def norm_check(x, w, b, dy, add, got, eps=1e-5, base=(0.0, 0.0)):
    y, mean, rstd, dx, dw, db = got
    out = B16 if x.dtype == torch.bfloat16 else U
    xr = x.double().requires_grad_(True)
    n, d = x.shape
    m = xr.mean(-1, keepdim=True) if b is not None else torch.zeros(n, 1, dtype=torch.float64, device="cuda")
    c = xr - m
    r = (c.square().mean(-1, keepdim=True) + eps) ** -0.5
    xh = c * r
    (ref_dx,) = torch.autograd.grad(xh, xr, dy.double() * w.double())
    m, c, r, xh = (t.detach() for t in (m, c, r, xh))
    # a thread adds at most 32 values, then 5 steps of a warp and 16 warps: 64 terms' roundings
    s = 64 * 2 * U
    e_m = s * x.double().abs().mean(-1, keepdim=True) if b is not None else torch.zeros_like(m)
    e_r = (s + 4 * U) * r + e_m * r * r          # of rstd: its sum's, and what the mean's error adds
    e_xh = e_m * r + c.abs() * e_r + 2 * U * (xh.abs() + x.double().abs() * r)
    if mean is not None:
        within(mean, m[:, 0], e_m[:, 0] + U * m[:, 0].abs(), "mean")
    within(rstd, r[:, 0], e_r[:, 0], "rstd")
    ref = xh * w.double() + (0.0 if b is None else b.double())
    within(y, ref, out * ref.abs() + (1 + out) * (w.double().abs() * e_xh + 2 * U * (ref.abs() + (xh * w.double()).abs())), "y")
    a = dy.double() * w.double()
    c2 = (a * xh).mean(-1, keepdim=True)
    e_c1 = s * a.abs().mean(-1, keepdim=True)
    e_c2 = s * (a * xh).abs().mean(-1, keepdim=True) + (a.abs() * e_xh).mean(-1, keepdim=True)
    e = r * (e_c1 + xh.abs() * e_c2 + e_xh * c2.abs() + 6 * U * (a.abs() + a.mean(-1, keepdim=True).abs() + (xh * c2).abs())) \
        + e_r / r * ref_dx.abs()
    if add is not None:
        ref_dx = ref_dx + add.double()
        e = e + 2 * U * (ref_dx.abs() + add.double().abs())
    within(dx, ref_dx, (1 + out) * e + out * ref_dx.abs(), "dx")
    # sums over the rows: at most as many steps as rows
    ref_w = (dy.double() * xh).sum(0)
    within(dw, ref_w + base[0], 2 * U * (n + 32) * (dy.double() * xh).abs().sum(0) + (dy.double().abs() * e_xh).sum(0)
           + 2 * U * (ref_w + base[0]).abs() + 1e-30, "dw")
    if db is not None:
        ref_b = dy.double().sum(0)
        within(db, ref_b + base[1], 2 * U * (n + 32) * dy.double().abs().sum(0) + 2 * U * (ref_b + base[1]).abs() + 1e-30, "db")


@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("n,d,dtype", [(1, 8, "bf16"), (24, 768, "bf16"), (3, 256, "bf16"), (400, 264, "bf16"), (2000, 64, "bf16"),
                                       (5000, 128, "bf16"), (700, 3584, "bf16"), (9, 4096, "bf16"), (310, 4104, "bf16"),
                                       (5, 8192, "bf16"), (1, 4, "f32"), (2044, 512, "f32"), (33, 132, "f32"), (3000, 100, "f32"),
                                       (10, 2048, "f32"), (311, 2052, "f32"), (7, 4100, "f32"), (309, 8192, "f32")])
def test_norm(A, n, d, dtype, rms):
    """Widths on both sides of every split over threads, few and many rows."""
    for res in (False, True):
        args = norm_inputs(n, d, dtype, rms, res)
        got = norm(A, *args)
        norm_check(*args, got)
        for x, y in zip(got, norm(A, *args)):
            assert x is None or torch.equal(x, y)


def test_norm_in_place_and_added(A):
    x, w, b, dy, add = norm_inputs(500, 768, "bf16", False, True)
    y, mean, rstd, dx, dw, db = norm(A, x, w, b, dy, add)
    x2, m2, r2 = x.clone(), torch.empty_like(mean), torch.empty_like(rstd)
    A.adadsf_norm_forward(x2, w, b, x2, 1e-5, m2, r2)
    assert torch.equal(x2, y) and torch.equal(m2, mean)
    for which in (0, 1):
        g, a = dy.clone(), add.clone()
        A.adadsf_norm_backward(g, x, w, rstd, (g, a)[which], mean=mean, add=a)
        assert torch.equal((g, a)[which], dx)
    base_w, base_b = randn(gen(1), 768, std=30.0), randn(gen(2), 768, std=30.0)
    got = norm(A, x, w, b, dy, add, dw=base_w.clone(), db=base_b.clone(), accumulate=True)
    norm_check(x, w, b, dy, add, got, base=(base_w.double(), base_b.double()))
    dw0, db0 = torch.full((768,), 7.0, device="cuda"), torch.full((768,), 7.0, device="cuda")
    A.adadsf_norm_backward(dy[:0], x[:0], w, rstd[:0], dx[:0], mean=mean[:0], grad_w=dw0, grad_b=db0)
    assert (dw0 == 0).all() and (db0 == 0).all()


def test_norm_row_of_one_value(A):
    """A constant row has no spread: rstd = eps^-1/2, xhat 0, and no gradient but what the formula gives."""
    x, w, b, dy, _ = norm_inputs(40, 512, "f32", False, False)
    x[7] = 2.0
    x[8] = 0.0
    got = norm(A, x, w, b, dy, None)
    norm_check(x, w, b, dy, None, got)
    assert torch.equal(got[0][7], b) and torch.equal(got[0][8], b)


@pytest.mark.parametrize("n,d,dtype", [(1, 512, "f32"), (1, 2048, "f32"), (1, 4096, "f32"), (40, 512, "f32"),
                                       (700, 512, "f32"), (1, 1024, "bf16"), (1, 8192, "bf16"), (700, 2048, "bf16")])
def test_norm_of_rows_far_from_zero(A, n, d, dtype):
    """Rows whose mean is hundreds of times their spread (bf16: its last places): whole numbers, so that sums, mean and the
    differences to it are exact and xhat is off by roundings of its own size only, in fp32 in either pass. The bf16
    gradient's is x rstd - mean rstd: roundings of the mean's size, 2 of them, far below those of bf16."""
    g = gen(n + d)
    mean = 1000.0 if dtype == "f32" else 192.0
    half = torch.randint(1, 4, (n, d // 2), generator=g, device="cuda").float()
    if dtype == "bf16":
        half = half.clamp(max=2)
    off = torch.stack([half, -half], -1).reshape(n, d)[:, torch.randperm(d, generator=g, device="cuda")]
    x = (mean + off).to(DT[dtype])
    assert torch.equal(x.float(), mean + off)
    _, w, b, dy, _ = norm_inputs(n, d, dtype, False, False)
    y, got_mean, rstd, dx, dw, db = norm(A, x, w, b, dy, None)
    assert (got_mean == mean).all()
    out = B16 if dtype == "bf16" else U
    xd, wd, dyd = off.double(), w.double(), dy.double()
    r = (xd.square().mean(-1, keepdim=True) + 1e-5) ** -0.5
    xh = xd * r
    # the squares' sum is exact; its scale, eps, root and quotient: 4 roundings (2 ulp each at most)
    within(rstd, r[:, 0], 8 * U * r[:, 0], "rstd")
    e_xh = 12 * U * xh.abs()
    ref = xh * wd + b.double()
    within(y, ref, out * ref.abs() + (1 + out) * (wd.abs() * e_xh + 3 * U * (ref.abs() + (xh * wd).abs())), "y")
    far = 2 * U * mean * r if dtype == "bf16" else torch.zeros_like(r)
    a = dyd * wd
    s = 64 * 2 * U   # as in norm_check
    m1, m2 = a.mean(-1, keepdim=True), (a * xh).mean(-1, keepdim=True)
    ref = r * (a - m1 - xh * m2)
    e = r * (s * a.abs().mean(-1, keepdim=True) + xh.abs() * (s + 12 * U) * (a * xh).abs().mean(-1, keepdim=True)
             + 6 * U * (a.abs() + m1.abs() + (xh * m2).abs())) + 12 * U * r * (a.abs() + m1.abs() + (xh * m2).abs()) \
        + r * far * (xh.abs() * a.abs().mean(-1, keepdim=True) + 2 * m2.abs())
    within(dx, ref, (1 + out) * e + out * ref.abs(), "dx")
    size = (dyd * xh).abs().sum(0)
    # a sum of n numbers beside zeros
    within(dw, (dyd * xh).sum(0), 2 * U * n * size + 14 * U * size + (1 + 2 * U * n) * (dyd.abs() * far).sum(0), "dw")


@pytest.mark.parametrize("rms", [False, True])
def test_norm_of_more_than_2_31_numbers(A, rms):
    n, d = 1_060_000, 2048
    g = gen(5)
    x = torch.empty(n, d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
    dy = torch.empty_like(x).normal_(0.0, 1.0, generator=g)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    b = None if rms else torch.zeros_like(w)
    y, mean, rstd, dx, dw, db = norm(A, x, w, b, dy, None)
    rows = slice(n - 400, n)   # their part of the sums: the same rows by themselves
    part = norm(A, x[rows], w, b, dy[rows], None)
    norm_check(x[rows], w, b, dy[rows], None, (y[rows], None if rms else mean[rows], rstd[rows], dx[rows], part[4], part[5]))
    ref_w, ref_b, size, size_b = (torch.zeros(d, dtype=torch.float64, device="cuda") for _ in range(4))
    for c in range(0, n, 100_000):
        at = slice(c, c + 100_000)
        xh = x[at].double() * rstd[at, None].double()
        if not rms:
            xh = xh - (mean[at].double() * rstd[at].double())[:, None]
        ref_w += (dy[at].double() * xh).sum(0)
        ref_b += dy[at].double().sum(0)
        size += (dy[at].double() * xh).abs().sum(0)
        size_b += dy[at].double().abs().sum(0)
    # a chain has at most the rows of a block (304 blocks of this width), their sums 16 and 32 more; xhat is off by at most
    # 3 roundings of |x| rstd + |mean| rstd < 8
    within(dw, ref_w, 2 * U * (n / 304 + 64) * size + 3 * U * 8 * size_b, "dw")
    if not rms:
        within(db, ref_b, 2 * U * (n / 304 + 64) * size_b, "db")


# ------------------------------------------------------------------ embedding
def embed_check(A, ids, table, dy, scale, base=None, ws=None):
    V, d = table.shape
    out = B16 if table.dtype == torch.bfloat16 else U
    used = (ids >= 0) & (ids < V)
    y = torch.full_like(dy, 7.0)
    A.adadsf_embed_forward(ids, table, y, scale=scale, ws=ws)
    ref = torch.where(used[:, None], table.double()[ids.clamp(0, V - 1).long()] * scale, 0.0)
    within(y, ref, (out + 4 * U) * ref.abs(), "y")
    got = torch.full_like(table, 7.0) if base is None else base.clone()
    A.adadsf_embed_backward(ids, dy, got, scale=scale, accumulate=base is not None, ws=ws)
    at, rows = ids[used].long(), dy[used].double()
    ref = torch.zeros(V, d, dtype=torch.float64, device="cuda").index_add_(0, at, rows)
    size = torch.zeros_like(ref).index_add_(0, at, rows.abs())
    count = torch.zeros(V, dtype=torch.float64, device="cuda").index_add_(0, at, torch.ones_like(at, dtype=torch.float64))
    ref, b = ref * scale, 0.0 if base is None else base.double()
    err = abs(scale) * 2 * U * (count[:, None] + 2) * size + 4 * U * (ref.abs() + (b if base is None else b.abs()))
    within(got, ref + b, (1 + out) * err + out * (ref + b).abs(), "dtable")
    untouched = count == 0
    if base is None:
        assert (got[untouched] == 0).all()
    else:
        assert torch.equal(got[untouched], base[untouched])
    again = torch.full_like(table, 3.0) if base is None else base.clone()
    A.adadsf_embed_backward(ids, dy, again, scale=scale, accumulate=base is not None, ws=ws)
    assert torch.equal(got, again)


@pytest.mark.parametrize("n,V,d,dtype", [(1, 1, 8, "bf16"), (31, 50, 64, "bf16"), (33, 5, 264, "bf16"), (100, 50304, 768, "bf16"),
                                         (4096, 1000, 64, "bf16"), (4097, 1000, 72, "bf16"), (20000, 300, 40, "bf16"),
                                         (6000, 300000, 8, "bf16"), (700, 100, 8200, "bf16"), (2044, 3000, 512, "f32"),
                                         (65, 2, 4, "f32"), (70000, 7, 4, "f32"), (5000, 513, 260, "f32")])
def test_embed(A, n, V, d, dtype):
    """Both sorts, one to three digits, ids that fill many runs, fewer ids than threads."""
    g = gen(n + V)
    table = randn(g, V, d).to(DT[dtype])
    dy = randn(g, n, d).to(DT[dtype])
    ids = (torch.rand(n, generator=g, device="cuda") ** 3 * V).to(torch.int32)
    ids[torch.rand(n, generator=g, device="cuda") < 0.1] = -1
    embed_check(A, ids, table, dy, 1.0)
    embed_check(A, ids, table, dy, -2.5, base=randn(g, V, d).to(DT[dtype]))


def test_embed_workspace_of_more_tokens(A):
    """One workspace for the longest batch: a shorter one in it, of more and shorter runs."""
    V, d = 3000, 3584
    ws = A.workspace(A.adadsf_embed_backward_workspace_size(6000, V, d))
    g = gen(12)
    table, dy = randn(g, V, d).to(torch.bfloat16), randn(g, 6000, d).to(torch.bfloat16)
    ids = torch.randint(0, V, (6000,), generator=g, device="cuda", dtype=torch.int32)
    for n in (6000, 5558, 4096):
        embed_check(A, ids[:n], table, dy[:n], 1.0, ws=ws)


@pytest.mark.parametrize("n", [200, 6000])
def test_embed_of_more_than_2_31_numbers(A, n):
    """Rows of a table past 2^31 elements: the last one, the ones at the border, the others left or cleared."""
    V, d = 1_100_000, 2048
    g = gen(n)
    table = torch.empty(V, d, dtype=torch.bfloat16, device="cuda").normal_(0.0, 1.0, generator=g)
    dy = randn(g, n, d).to(torch.bfloat16)
    border = 2 ** 31 // d
    ids = torch.randint(border - 3, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[:5] = torch.tensor([V - 1, 0, border, border - 1, V - 1], device="cuda", dtype=torch.int32)
    y = torch.full_like(dy, 7.0)
    A.adadsf_embed_forward(ids, table, y)
    assert torch.equal(y, table[ids.long()])
    before = table[5:9].clone()
    A.adadsf_embed_backward(ids, dy, table)
    there, slot = ids.long().unique(return_inverse=True)
    ref = torch.zeros(there.numel(), d, dtype=torch.float64, device="cuda").index_add_(0, slot, dy.double())
    size = torch.zeros_like(ref).index_add_(0, slot, dy.double().abs())
    # an id comes n times at most; a sum of its rows, rounded once
    within(table[there], ref, 2 * U * n * size * (1 + B16) + B16 * ref.abs(), "dtable")
    left = torch.ones(V, dtype=torch.bool, device="cuda")
    left[there] = False
    for c in range(0, V, 100_000):
        assert (table[c:c + 100_000][left[c:c + 100_000]] == 0).all()
    table[5:9] = before
    A.adadsf_embed_backward(ids, dy, table, accumulate=True)
    assert torch.equal(table[5:9], before)


@pytest.mark.parametrize("n", [32, 64, 65, 3000, 9000])
def test_embed_one_id_and_none(A, n):
    g = gen(n)
    table, dy = randn(g, 40, 64).to(torch.bfloat16), randn(g, n, 64).to(torch.bfloat16)
    dy[1::2] = math.nan
    ids = torch.full((n,), -1, device="cuda", dtype=torch.int32)
    got = torch.full_like(table, 7.0)
    A.adadsf_embed_backward(ids, dy, got)
    assert (got == 0).all()                                # what padding's rows hold reaches nothing
    ids[::2] = 39
    embed_check(A, ids, table, torch.nan_to_num(dy), 1.0)
    A.adadsf_embed_backward(ids, dy, got)
    assert torch.isfinite(got).all()


def test_embed_out_of_range(A):
    g = gen(5)
    table, dy = randn(g, 100, 64), randn(g, 5000, 64)
    ws = A.workspace(A.adadsf_embed_backward_workspace_size(5000, 100, 64))
    for n in (50, 5000):
        ids = torch.randint(0, 100, (n,), generator=g, device="cuda", dtype=torch.int32)
        ids[3], ids[4] = 100, 2 ** 31 - 1
        got, y = torch.empty_like(table), torch.empty(n, 64, device="cuda")
        A.adadsf_embed_backward(ids, dy[:n], got, ws=ws)
        assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
        A.adadsf_embed_forward(ids, table, y, ws=ws)
        assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
        assert (y[3:5] == 0).all()
        ids[3:5] = -1
        want = torch.empty_like(table)
        A.adadsf_embed_backward(ids, dy[:n], want, ws=ws)
        assert A.adadsf_sync_check(ws) == A.OK
        assert torch.equal(got, want)


def test_embed_backward_captured(A):
    g = gen(6)
    for n in (300, 6000):
        table, dy = torch.empty(500, 64, device="cuda"), randn(g, n, 64)
        ids = torch.randint(0, 500, (n,), generator=g, device="cuda", dtype=torch.int32)
        ws = A.workspace(A.adadsf_embed_backward_workspace_size(n, 500, 64))
        A.adadsf_embed_backward(ids, dy, table, ws=ws)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            A.adadsf_embed_backward(ids, dy, table, ws=ws)
        ids.copy_(torch.randint(0, 500, (n,), generator=g, device="cuda", dtype=torch.int32))
        graph.replay()
        got = table.clone()
        A.adadsf_embed_backward(ids, dy, table, ws=ws)
        assert torch.equal(got, table)


# ------------------------------------------------------------------ a run of them together
@pytest.mark.parametrize("arch,dtype,tied,teacher", [("neox", "bf16", True, False), ("qwen", "bf16", False, True),
                                                     ("neox", "f32", True, True), ("qwen", "f32", True, False)])
def test_ends_together(A, arch, dtype, tied, teacher):
    """Embedding, a stand-in for the layers, final norm, head, loss and back, as a training step calls them (align.py),
    against 64-bit autograd of the same composition. bf16 rounds five tensors on the way (rows, normed rows, the logits'
    gradients, the norm's and the outputs): each is off by 2^-8 / sqrt(3) of its size at most on average, through a norm
    and products that carry it on at about its relative size: 2-norms within 5 x 2^-8. fp32: chains as in test_head_loss,
    of sizes that random signs leave far below their bound: 1e-5."""
    from paper_2607_21291_gb300 import align
    from paper_2607_21291_gb300 import synth as S
    d, V, B, T = 128, 700, 3, 50
    shape = (S.PYTHIA_70M if arch == "neox" else S.QWEN25_1_5B).replace(d=d, vocab=V, dtype=dtype)
    cfg = A.make_cfg(shape)
    g = gen(17)
    td = DT[dtype]
    w = {"embed": randn(g, V, d, std=0.3).to(td), "final_w": (1 + randn(g, d, std=0.1)).to(td)}
    if arch == "neox":
        w["final_b"] = randn(g, d, std=0.1).to(td)
    if not tied:
        w["head"] = randn(g, V, d, std=0.1).to(td)
    ids = torch.randint(0, V, (B, T), generator=g, device="cuda", dtype=torch.int32)
    target = torch.roll(ids, -1, 1).contiguous()
    ids[2, 30:] = -1
    target[:, -1] = -1
    target[2, 29:] = -1
    target[0, :7] = -1
    top = None
    if teacher:
        idx = torch.randint(0, V, (B * T, 6), generator=g, device="cuda", dtype=torch.int32)
        idx[target.reshape(-1) < 0] = -1
        top = (idx, randn(g, B * T, 6, std=2.0), 1.5)
    turn = randn(g, d, d, std=d ** -0.5).to(td)

    def body(x):
        return (x.float() @ turn.float()).to(td), lambda gy: (gy.float() @ turn.float().T).to(td)

    loss, grads = align.ends_gradients(cfg, w, ids, target, body=body, top=top, scale=2.0)
    leaf = {k: v.double().requires_grad_(True) for k, v in w.items()}
    used = ids.reshape(-1) >= 0
    x = torch.where(used[:, None], leaf["embed"][ids.reshape(-1).clamp(min=0).long()] * 2.0, 0.0)
    y = x @ turn.double()
    c = y if arch == "qwen" else y - y.mean(-1, keepdim=True)
    hid = c * (c.square().mean(-1, keepdim=True) + shape.norm_eps) ** -0.5 * leaf["final_w"]
    if arch == "neox":
        hid = hid + leaf["final_b"]
    z = hid @ leaf["embed" if tied else "head"].T
    if teacher:
        temp = top[2]
        want, valid, ent = teacher_want(top[0], top[1], V, temp)
    else:
        temp, (want, valid) = 1.0, want_of(target.reshape(-1), V)
        ent = torch.zeros(B * T, dtype=torch.float64, device="cuda")
    row = temp ** 2 * (ent - (want * torch.log_softmax(z / temp, -1)).sum(-1))
    mean = torch.where(valid, row, 0.0).sum() / valid.sum()
    ref = dict(zip(leaf, torch.autograd.grad(mean, list(leaf.values()))))
    tol = 5 * B16 if dtype == "bf16" else 1e-5
    assert float(loss) == pytest.approx(float(mean.detach()), rel=tol)
    assert set(grads) == set(ref)
    for k in ref:
        assert float((grads[k].double() - ref[k]).norm()) <= tol * float(ref[k].norm()), k
    before = {k: v.clone() for k, v in w.items()}
    assert float(align.ends_step(cfg, w, ids, target, 0.5, body=body, top=top, scale=2.0)) == float(loss)
    for k in w:   # one rounding of the update
        step = before[k].double() - 0.5 * grads[k].double()
        within(w[k], step, (B16 if dtype == "bf16" else U) * 2 * step.abs() + 1e-7, k)


@pytest.mark.parametrize("dtype,tied", [("bf16", True), ("f32", False)])
def test_ends_on_another_stream(A, dtype, tied):
    """A step on a stream of the caller's while the current one is busy and writes the ids behind that: the same bits as on
    the current stream, results read on the current one without more ado, and freed there."""
    from paper_2607_21291_gb300 import align
    from paper_2607_21291_gb300 import synth as S
    d, V, n = 128, 700, 150
    cfg = A.make_cfg(S.PYTHIA_70M.replace(d=d, vocab=V, dtype=dtype))
    g = gen(19)
    w = {"embed": randn(g, V, d, std=0.3).to(DT[dtype]), "final_w": (1 + randn(g, d, std=0.1)).to(DT[dtype]),
         "final_b": randn(g, d, std=0.1).to(DT[dtype])}
    if not tied:
        w["head"] = randn(g, V, d, std=0.1).to(DT[dtype])
    real = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    target = torch.roll(real, -1).contiguous()
    target[:40] = -1
    turn = randn(g, d)
    on = []

    def body(x):
        on.append(torch.cuda.current_stream())
        return (x.float() * turn).to(x.dtype), lambda gy: (gy.float() * turn).to(gy.dtype)

    want_loss, want = align.ends_gradients(cfg, w, real, target, body=body)
    want_w = {k: v.clone() for k, v in w.items()}
    align.ends_step(cfg, want_w, real, target, 0.5, body=body)
    side, ids = torch.cuda.Stream(), torch.empty_like(real)
    with torch.cuda.stream(side):
        held = [torch.full((m,), 255, dtype=torch.uint8, device="cuda") for m in (1 << 28, *[1 << 20] * 8, *[1024] * 8)]
        del held
    torch.cuda.synchronize()
    for _ in range(3):
        ids.fill_(-1)
        torch.cuda._sleep(50_000_000)
        ids.copy_(real)
        loss, grads = align.ends_gradients(cfg, w, ids, target, body=body, stream=side)
        mine = {k: v.clone() for k, v in w.items()}
        step_loss = align.ends_step(cfg, mine, ids, target, 0.5, body=body, stream=side)
        assert on[-1] == side and torch.cuda.current_stream() != side
        got = {k: v + 0 for k, v in grads.items()}
        assert torch.equal(loss, want_loss) and torch.equal(step_loss, want_loss)
        del grads, loss, step_loss
        with torch.cuda.stream(side):
            torch.full((1 << 22,), 7.0, device="cuda")
        for k in want:
            assert torch.equal(got[k], want[k]) and torch.equal(mine[k], want_w[k]), k
