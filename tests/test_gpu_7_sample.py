"""Sampling on the GPU (adadsf_sample) against a plain 64-bit form, through the C
ABI.

A 32-bit exponential of a 32-bit product is off by at most about 2^-22 + |z| 2^-23
relatively (|z| < 28 for a weight above 2^-40), and a weight by half a unit of 2^-40
more: running sums agree within 1e-5 of their total. So the drawn token has
to lie where u points in the 64-bit running sum within 2e-5 of the total, in a set cut
at top_p within 1e-5, and its log-probability agrees within 1e-4 absolutely (4e-6 from z, as
much from the total; cuts that a rounding moves are excluded by the first check).
Where weights are equal whole numbers the result is exact."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


def draw(A, logits, u, temperature=None, top_k=None, top_p=None, min_p=None):
    B = logits.shape[0]
    f = lambda v, dt=torch.float32: None if v is None else torch.tensor(v, dtype=dt, device="cuda")   # noqa: E731
    token = torch.full((B,), -7, dtype=torch.int32, device="cuda")
    logprob = torch.full((B,), math.nan, device="cuda")
    A.adadsf_sample(logits, f(u), token, f(temperature), f(top_k, torch.int32), f(top_p), f(min_p), logprob)
    again = torch.full_like(token, -7)
    A.adadsf_sample(logits, f(u), again, f(temperature), f(top_k, torch.int32), f(top_p), f(min_p))
    torch.cuda.synchronize()
    assert torch.equal(token, again)
    return token.cpu().numpy(), logprob.cpu().numpy()


def kept64(x, t, k, p, floor):
    """(weights, kept mask with top_p = p) of one row in 64 bits."""
    x = np.where(np.isnan(x), -np.inf, x)
    top = x.max()
    with np.errstate(invalid="ignore"):
        z = np.where(x == top, 0.0, (x - top) / t)
    w = np.rint(np.exp(z) * 2.0 ** 40) / 2.0 ** 40
    order = np.argsort(-x, kind="stable")
    ws = w[order]
    keep = np.ones(x.size, dtype=bool)
    if 0 < k < x.size:
        keep[k:] = False
    ws = np.where(keep, ws, 0.0)
    if p < 1:
        keep &= np.cumsum(ws) - ws < p * ws.sum()
    if floor > 0:
        keep &= np.exp(z)[order] >= min(floor, 1.0) * (1 + 1e-5)
    keep[0] = True
    out = np.zeros(x.size, dtype=bool)
    out[order[keep]] = True
    return w, z, out


def check_row(x, token, logprob, t, k, p, floor, u):
    if not t > 0:
        best = np.where(np.isnan(x), -np.inf, x)
        assert token == int(np.argmax(best)) and logprob == 0
        return
    ok = False
    for dp in ((0.0, -1e-5, 1e-5) if p < 1 else (0.0,)):
        for df in ((1.0, 1 - 2e-5) if floor > 0 else (1.0,)):
            w, z, keep = kept64(x, t, k, p + dp if p + dp > 0 else p, floor * df)
            kw = np.where(keep, w, 0.0)
            c = np.cumsum(kw)
            lo, hi = c[token] - kw[token], c[token]
            if keep[token] and lo - 2e-5 * c[-1] <= u * c[-1] <= hi + 2e-5 * c[-1] and \
                    abs(logprob - (z[token] - math.log(c[-1]))) <= 1e-4:
                ok = True
    assert ok, (token, logprob, t, k, p, floor, u)


SETTINGS = [   # temperature, top_k, top_p, min_p
    (1.0, 0, 1.0, 0.0), (0.7, 50, 1.0, 0.0), (1.3, 0, 0.9, 0.0), (0.8, 40, 0.95, 0.0), (1.0, 0, 1.0, 0.05),
    (1.1, 200, 0.5, 0.01), (0.0, 5, 0.5, 0.0), (2.5, 1, 1.0, 0.0), (1.0, 0, 1e-6, 0.0), (0.05, 0, 0.99, 0.0),
    (30.0, 1000, 0.999, 0.0), (1.0, 3, 0.8, 1.0),
]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 33, 511, 512, 4096, 4097, 50257, 151936, 152064])
def test_settings(A, V, dtype):
    g = torch.Generator().manual_seed(V)
    B = 3 * len(SETTINGS)
    logits = 2.5 * torch.randn(B, V, generator=g)
    logits[:, :: max(1, V // 7)] += 6
    logits = logits.to(dtype).cuda()
    u = torch.rand(B, generator=g).tolist()
    u[0], u[1] = 0.0, 1 - 2.0 ** -24
    per = [SETTINGS[b % len(SETTINGS)] for b in range(B)]
    token, logprob = draw(A, logits, u, *[[s[i] for s in per] for i in range(4)])
    x = logits.double().cpu().numpy()
    for b in range(B):
        assert 0 <= token[b] < V
        check_row(x[b], int(token[b]), float(logprob[b]), *per[b], u[b])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [4097, 20000, 152064])
def test_few_and_many_survivors(A, V, dtype):
    """Cuts that leave a handful to thousands of tokens, around the sizes where a row's search changes
    its way: ties by the hundred, rows sorted either way (all likely tokens in one part of
    the row), rows of which a hundred tokens are not masked, alone or in every part."""
    g = torch.Generator().manual_seed(V + 1)
    kinds = [torch.randn(V, generator=g) * 2, torch.round(torch.randn(V, generator=g) * 8) / 4]
    kinds += [kinds[0].sort().values, kinds[1].sort(descending=True).values]
    few = torch.full((V,), -math.inf)
    few[torch.randperm(V, generator=g)[:100]] = torch.randn(100, generator=g)
    here = torch.full((V,), -math.inf)
    here[V // 2:V // 2 + 100] = torch.randn(100, generator=g)
    kinds += [few, here]
    per = [(t, k, p, f) for k in (1, 2, 127, 128, 129, 700, 0) for t, p, f in ((1.0, 1.0, 0.0), (0.6, 0.9, 0.0), (1.5, 0.97, 0.02))]
    rows = [(x, s) for x in kinds for s in per]
    logits = torch.stack([x for x, _ in rows]).to(dtype).cuda()
    u = torch.rand(len(rows), generator=g).tolist()
    token, logprob = draw(A, logits, u, *[[s[i] for _, s in rows] for i in range(4)])
    x = logits.double().cpu().numpy()
    for b, (_, s) in enumerate(rows):
        check_row(x[b], int(token[b]), float(logprob[b]), *s, u[b])


def test_defaults_and_many_rows(A):
    """No settings at all, more rows than fit the machine at once, rows of a wider
    matrix that start at odd places."""
    g = torch.Generator().manual_seed(1)
    B, V = 700, 1003
    wide = torch.randn(B, V + 14, generator=g).cuda()
    logits = wide[:, 3:3 + V]
    u = torch.rand(B, generator=g).tolist()
    token, logprob = draw(A, logits, u)
    x = logits.double().cpu().numpy()
    for b in range(B):
        check_row(x[b], int(token[b]), float(logprob[b]), 1.0, 0, 1.0, 0.0, u[b])
    counts = np.bincount(draw(A, logits[:1].expand(600, V).contiguous(), [(i + 0.5) / 600 for i in range(600)])[0], minlength=V)
    w = np.exp(x[0] - x[0].max())
    assert np.abs(counts / 600 - w / w.sum()).max() <= 2 / 600      # an even ladder of u counts every token's share


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [9, 777, 40001])
def test_equal_logits_go_by_index(A, V, dtype):
    """Equal logits: top-k keeps the first k, top-p the first ones whose number
    reaches p of them; the draw is floor(u kept) exactly."""
    k = max(1, V // 3)
    u = [0.0, 0.2501, 0.7501, 1 - 2.0 ** -24]
    logits = torch.full((4, V), -1.25, dtype=dtype, device="cuda")
    token, logprob = draw(A, logits, u, None, [k] * 4)
    assert token.tolist() == [min(int(x * k), k - 1) for x in u]
    assert np.allclose(logprob, -math.log(k), atol=1e-5)
    p = float(np.float32(0.3))
    n = math.ceil(p * V)
    token, _ = draw(A, logits, u, None, None, [p] * 4)
    assert token.tolist() == [min(int(x * n), n - 1) for x in u]
    n = math.ceil(p * k)
    token, _ = draw(A, logits, u, None, [k] * 4, [p] * 4)
    assert token.tolist() == [min(int(x * n), n - 1) for x in u]
    # two levels: the higher ones all kept, ties cut among the lower
    logits[:, 1::2] = 2.0
    high = V // 2
    k = high + 2
    token, _ = draw(A, logits, [1 - 2.0 ** -24] * 4, [1e9] * 4, [k] * 4)
    assert token.tolist() == [1 + 2 * (high - 1) if 1 + 2 * (high - 1) > 2 else 2] * 4
    token, _ = draw(A, logits, u, [0.0] * 4)
    assert token.tolist() == [1] * 4


def test_signed_zeros_are_equal(A):
    logits = torch.tensor([[-0.0, 0.0, -0.0, 0.0]], device="cuda")
    assert draw(A, logits, [0.9], None, [2])[0].tolist() == [1]
    assert draw(A, logits, [0.9], [0.0])[0].tolist() == [0]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [64, 20000])
def test_masked_logits(A, V, dtype):
    """Tokens masked with -infinity, NaN or the type's lowest value are not drawn; a row of nothing
    else gives -1; a row masked but for one token gives it; +infinity takes all."""
    g = torch.Generator().manual_seed(3)
    low = torch.finfo(dtype).min
    rows = []
    for mask in (-math.inf, math.nan, low):
        x = torch.randn(V, generator=g)
        x[torch.rand(V, generator=g) < 0.9] = mask
        x[5] = 1.0
        rows.append(x)
    only = torch.full((V,), -math.inf)
    only[V - 1] = low
    rows += [only, torch.full((V,), -math.inf), torch.full((V,), math.nan)]
    inf = torch.randn(V, generator=g)
    inf[7] = inf[20] = math.inf
    rows.append(inf)
    logits = torch.stack(rows).to(dtype).cuda()
    x = logits.double().cpu().numpy()
    for u in (0.0, 0.4, 0.49, 0.51, 1 - 2.0 ** -24):
        for s in ((None, None, None, None), ([0.7] * 7, [30] * 7, [0.9] * 7, [0.01] * 7), ([0.0] * 7, None, None, None),
                  ([1e30] * 7, None, None, None), ([math.inf] * 7, None, None, None)):
            token, logprob = draw(A, logits, [u] * 7, *s)
            assert token[4] == token[5] == -1 and logprob[4] == logprob[5] == -math.inf
            assert token[3] == V - 1 and logprob[3] == 0
            assert token[6] == 7 if u < 0.5 or (s[0] and s[0][0] == 0) else token[6] == 20
            for b in range(2):
                assert np.isfinite(x[b, token[b]])
            if s[0] is None or s[0][0] < 1:
                assert x[2, token[2]] > -100


def test_settings_that_keep_everything_or_one(A):
    g = torch.Generator().manual_seed(4)
    logits = torch.randn(6, 5000, generator=g).cuda()
    u = [0.3] * 6
    plain = draw(A, logits, u)[0].tolist()
    nan = math.nan
    assert draw(A, logits, u, [1.0] * 6, [0, -1, 5000, 6000, 2 ** 31 - 1, -2 ** 31], [1.0, 1.5, nan, 1.0, 2.0, 1.0],
                [0.0, -1.0, nan, 0.0, 0.0, 0.0])[0].tolist() == plain
    best = logits.argmax(-1).tolist()
    assert draw(A, logits, u, [nan, -1.0, 0.0, 1e-30, 1e-45, 1.0], None, [1.0] * 5 + [0.0])[0].tolist() == best
    assert draw(A, logits, u, None, [1] * 6)[0].tolist() == best
    assert draw(A, logits, u, None, None, [-1.0] * 6)[0].tolist() == best
    assert draw(A, logits, u, None, None, None, [5.0] * 6)[0].tolist() == best
    assert draw(A, logits, [nan] * 6)[0].tolist() == draw(A, logits, [0.0] * 6)[0].tolist() == draw(A, logits, [-3.0] * 6)[0].tolist()
    assert draw(A, logits, [1.0] * 6)[0].tolist() == draw(A, logits, [1 - 2.0 ** -24] * 6)[0].tolist() == draw(A, logits, [math.inf] * 6)[0].tolist()


def test_largest_vocabulary_and_graph(A):
    V = 397312
    g = torch.Generator().manual_seed(5)
    logits = (3 * torch.randn(2, V, generator=g)).cuda()
    u = torch.tensor([0.25, 0.75], device="cuda")
    token, logprob = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, device="cuda")
    p = torch.tensor([0.9, 1.0], device="cuda")
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        A.adadsf_sample(logits, u, token, top_p=p, logprob=logprob)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        A.adadsf_sample(logits, u, token, top_p=p, logprob=logprob)
    for v in (0.1, 0.6):
        u.fill_(v)
        graph.replay()
        torch.cuda.synchronize()
        x = logits.double().cpu().numpy()
        for b in range(2):
            check_row(x[b], int(token[b]), float(logprob[b]), 1.0, 0, float(p[b]), 0.0, float(u[b]))


def test_refusals(A):
    x = torch.zeros(2, 8, device="cuda")
    u, t = torch.zeros(2, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        A.adadsf_sample(x.half(), u, t)
    with pytest.raises(ValueError):
        A.adadsf_sample(x.t(), u, t)
    with pytest.raises(ValueError):
        A.adadsf_sample(x, u[:1], t)
    with pytest.raises(ValueError):
        A.adadsf_sample(x, u, t.long())
    with pytest.raises(ValueError):
        A.adadsf_sample(x, u, t, top_k=u)


# Weights in units of 2^-40 that round up by up to the factor of two that rounding has, and top_p so close to 1 that the
# cut falls among them.
NEAR_ONE = [1 - 2.0 ** -24, 1 - 2.0 ** -23, 1 - 2.0 ** -22, 1 - 3.5e-7, 1 - 2.0 ** -21, 1 - 2.0 ** -20, 0.999998, 0.999994, 0.9999]


@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("dtype,V,low,high", [
    (torch.float32, 50304, math.log(2.56) - 40 * math.log(2), 0.0), (torch.float32, 152064, math.log(2.53) - 40 * math.log(2), 0.0),
    (torch.float32, 152064, math.log(0.55) - 40 * math.log(2), 0.0), (torch.float32, 397312, math.log(0.52) - 40 * math.log(2), 0.0),
    (torch.float32, 4096, math.log(0.7) - 40 * math.log(2), 0.0), (torch.float32, 152064, -0.5, 27.5), (torch.float32, 152064, 0.0, 28.0),
    (torch.bfloat16, 152064, 0.0, 28.0), (torch.bfloat16, 151936, 0.0, 27.5), (torch.bfloat16, 397312, 0.0, 28.0),
    (torch.bfloat16, 50304, 0.0, 26.75)], ids=str)
def test_cut_in_a_flat_tail(A, dtype, V, low, high, at):
    """One large logit above equal ones that weigh a unit or a few: kept are the large one and the first of
    the others, as many as top_p asks for in whole units, and the draw goes by exact sums. With a temperature
    of 1/2 and half the distances too. What is drawn is written in any case."""
    u = [0.0, 0.25, 0.75, 1 - 2.0 ** -24]
    rows = [(p, x, t) for p in NEAR_ONE for x in u for t in (1.0, 0.5)]
    x = torch.full((len(rows), V), low, dtype=torch.float32)
    top = {"first": 0, "middle": V // 3, "last": V - 1}[at]
    x[:, top] = high
    x = (x * torch.tensor([[t] for _, _, t in rows])).to(dtype)
    other = (top + 1) % V
    z = (x[:, other].double() - x[:, top].double()).numpy() / np.array([t for _, _, t in rows])
    token, logprob = draw(A, x.cuda(), [r[1] for r in rows], [r[2] for r in rows], None, [r[0] for r in rows])
    for b, (p, v, _) in enumerate(rows):
        units = math.exp(z[b]) * 2.0 ** 40
        w = round(units)
        assert abs(units - w) < 0.49                                  # clear of a tie
        p, v, one = float(np.float32(p)), float(np.float32(v)), 2 ** 40
        total = one + w * (V - 1)
        n = 0 if w == 0 else min(V - 1, max(0, math.ceil((p * total - one) / w)))   # others kept
        kept = one + n * w
        mark = int(v * kept)
        before = min(n, top)                                          # kept others ahead of the large one
        if w and mark < before * w:
            want = mark // w
        elif mark < before * w + one:
            want = top
        else:
            want = top + 1 + (mark - before * w - one) // w
        assert token[b] == want, (p, v, w, n, token[b], want)
        assert abs(logprob[b] - ((0.0 if want == top else z[b]) - math.log(kept / one))) <= 1e-4
