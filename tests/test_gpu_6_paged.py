"""Paged cache on the GPU (adadsf_paged_append, adadsf_paged_read,
adadsf_paged_attention) against plain 64-bit formulas, through the C ABI.

Every slot that no token owns (unused pages, the rest of a last page) holds
NaN, and table entries past a sequence's pages hold -1 or an enormous number:
neither may show in a result.

Attention bounds, per output element, as multiples of a = softmax(S) |V|:
  scores      a fp32 sum of hd products is off by at most (hd + 4) 2^-24 times the sum of
              their absolute values; an exponential of it by twice that, relatively
              (its own and the row sum's)
  weights     2^-21 for the exponential, (keys + 8) 2^-24 for the sums
  bf16        2^-9 for each weight's rounding (a bit more where it is scaled first),
              2^-9 for the output's, 2^-17 in all for products of the two
Cached values are exact in the reference, whole numbers times their scale."""
import math

import numpy as np
import pytest
import torch

from paper_2607_21291_gb300 import synth as S

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    from paper_2607_21291_gb300 import adadsf
    adadsf.lib()
    return adadsf


def shape_of(H, Hkv, hd, dtype, rotary=None):
    base = S.PYTHIA_70M if dtype == "f32" else S.PYTHIA_160M
    return base.replace(n_heads=H, n_kv_heads=Hkv, head_dim=hd, dtype=dtype, rotary_dim=hd if rotary is None else rotary)


def tdt(shape):
    return torch.float32 if shape.dtype == "f32" else torch.bfloat16


class World:
    """A pool with every sequence's tokens in shuffled pages, NaN everywhere else."""

    def __init__(self, A, shape, store, page, seqs, seed=0, spare=3, first_page=0):
        g = torch.Generator().manual_seed(seed)
        self.shape, self.cfg, self.page = shape, A.make_cfg(shape), page
        lens = [l for _, l in seqs]
        need = [-(-l // page) for l in lens]
        used = sum(need) + spare
        n_pages = first_page + used
        order = (torch.randperm(used, generator=g) + first_page).tolist()
        width = max(need + [1]) + 1
        table, at = [], 0
        for b, n in enumerate(need):
            table.append(order[at:at + n] + [(-1, 2 ** 30)[b % 2]] * (width - n))
            at += n
        kv_shape = (n_pages, shape.n_kv_heads, page, shape.head_dim)
        i8 = store == "i8"
        dt = torch.int8 if i8 else tdt(shape)
        self.k, self.v = (torch.empty(kv_shape, dtype=dt, device="cuda") for _ in range(2))
        self.ks = self.vs = None
        live = slice(first_page, n_pages)
        if i8:
            self.ks, self.vs = (torch.empty(kv_shape[:3], device="cuda") for _ in range(2))
            for t in (self.k, self.v):
                t[live] = 85
            for t in (self.ks, self.vs):
                t[live] = math.nan
        else:
            for t in (self.k, self.v):
                t[live] = math.nan
        self.K, self.V = [], []      # per sequence [len, Hkv, hd] float64, what the cache stands for
        for b, l in enumerate(lens):
            for name, out in (("k", self.K), ("v", self.V)):
                x = torch.randn(l, shape.n_kv_heads, shape.head_dim, generator=g).cuda()
                if l:
                    x *= torch.exp(0.4 * torch.randn(l, 1, 1, generator=g)).cuda()
                pages = torch.tensor([table[b][p // page] for p in range(l)], dtype=torch.long, device="cuda")
                slots = torch.arange(l, device="cuda") % page
                if i8:
                    q = torch.randint(-127, 128, x.shape, generator=g).to(torch.int8).cuda()
                    s = (x.abs().amax(-1) / 127).float()
                    if l:
                        getattr(self, name)[pages, :, slots] = q
                        getattr(self, name + "s")[pages, :, slots] = s
                    out.append(q.double() * s.double()[..., None])
                else:
                    y = x.to(dt)
                    if l:
                        getattr(self, name)[pages, :, slots] = y
                    out.append(y.double())
        starts = np.concatenate([[0], np.cumsum([n for n, _ in seqs])])
        self.seqs, self.n_rows = seqs, int(starts[-1])
        self.starts = torch.tensor(starts, dtype=torch.int32, device="cuda")
        self.lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.table = torch.tensor(table, dtype=torch.int32, device="cuda")
        self.cache = A.PagedCache(self.cfg, self.k, self.v, self.ks, self.vs)
        self.batch = A.PagedBatch(self.starts, self.lens, self.table, self.n_rows, max(n for n, _ in seqs))


def attend64(w, q):
    """(output, bound on its error) of every row in 64 bits."""
    s = w.shape
    H, hd, G = s.n_heads, s.head_dim, s.n_heads // s.n_kv_heads
    out = torch.zeros(w.n_rows, H, hd, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(out)
    r = 0
    for b, (n, l) in enumerate(w.seqs):
        if n and l:
            x = q[r:r + n].double().reshape(n, H, hd)
            k, v = (t[b].repeat_interleave(G, 1) for t in (w.K, w.V))       # [l, H, hd]
            sc = torch.einsum("nhd,lhd->hnl", x, k) / math.sqrt(hd)
            size = torch.einsum("nhd,lhd->hnl", x.abs(), k.abs()) / math.sqrt(hd)
            vis = torch.arange(l, device="cuda")[None] <= l - n + torch.arange(n, device="cuda")[:, None]
            some = vis.any(-1)
            p = torch.where(vis, sc, -math.inf)
            p = torch.where(some[:, None], torch.softmax(p, -1), 0.0)
            a = torch.einsum("hnl,lhd->nhd", p, v.abs())
            out[r:r + n] = torch.einsum("hnl,lhd->nhd", p, v)
            e = 2 * (hd + 4) * 2.0 ** -24 * torch.where(vis, size, 0.0).amax(-1).T[..., None]   # [n, H, 1]
            e = e + 2.0 ** -21 + (l + 8) * 2.0 ** -24
            if s.dtype == "bf16":
                e = e + 2.0 ** -9 + 2.0 ** -9 + 2.0 ** -17
            bound[r:r + n] = e * a
        r += n
    return out.reshape(w.n_rows, -1), bound.reshape(w.n_rows, -1)


def check_attention(A, w, q, out):
    ref, bound = attend64(w, q)
    got = out.double()
    assert torch.isfinite(got).all()
    bad = (got - ref).abs() > bound
    assert not bad.any(), (int(bad.sum()), float(((got - ref).abs() / bound.clamp(min=1e-30)).max()))
    # rows that see nothing are zeros, exactly
    assert (got[(bound == 0).all(-1)] == 0).all()


def queries(w, seed=1, scale=1.3):
    g = torch.Generator().manual_seed(seed)
    return (scale * torch.randn(w.n_rows, w.shape.q_dim, generator=g)).to(tdt(w.shape)).cuda()


def attend(A, w, q, ws=None):
    out = torch.full((w.n_rows, w.shape.q_dim), math.nan, dtype=tdt(w.shape), device="cuda")
    if ws is None:
        ws = A.workspace(A.adadsf_paged_attention_workspace_size(w.cfg, w.cache, w.batch))
    A.adadsf_paged_attention(w.cfg, w.cache, w.batch, q, out, ws=ws)
    assert A.adadsf_sync_check(ws) == A.OK
    return out


HEADS = [(8, 8, 64, "f32"), (4, 2, 128, "f32"), (12, 12, 64, "bf16"), (16, 16, 128, "bf16"), (12, 2, 128, "bf16"),
         (28, 4, 128, "bf16"), (16, 1, 64, "bf16"), (7, 1, 64, "bf16"), (34, 2, 128, "bf16"), (20, 1, 64, "f32")]
SEQS = {
    "one key": [(1, 1)],
    "decode": [(1, 100), (1, 1), (1, 16), (1, 129), (1, 700), (1, 64), (1, 65)],
    "idle": [(0, 0), (1, 40), (0, 333), (0, 0), (1, 2), (0, 1)],
    "prompt": [(5, 5), (130, 130), (64, 64)],
    "chunk": [(33, 400), (1, 257), (0, 90), (17, 17), (200, 1000), (2, 128)],
    "no place": [(4, 2), (3, 0), (1, 0), (20, 19), (1, 5)],
    "many": [(1 + b % 3, 3 + 7 * b) for b in range(70)],
    "long": [(1, 5003), (3, 2048), (1, 9)],
}


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("case", sorted(SEQS))
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_attention(A, heads, case, store):
    page = (16, 32, 64, 128)[(len(case) + HEADS.index(heads)) % 4]
    w = World(A, shape_of(*heads), store, page, SEQS[case], seed=len(case))
    q = queries(w)
    check_attention(A, w, q, attend(A, w, q))


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_attention_page_sizes(A, page, store):
    """Lengths around the ends of pages and tiles, in chunks and single tokens."""
    seqs = [(n, l) for l in (page - 1, page, page + 1, 127, 128, 129, 256) for n in (1, 9)]
    for heads in ((12, 2, 128, "bf16"), (12, 12, 64, "bf16"), (8, 8, 64, "f32")):
        w = World(A, shape_of(*heads), store, page, seqs, seed=page)
        q = queries(w)
        check_attention(A, w, q, attend(A, w, q))
        single = World(A, shape_of(*heads), store, page, [(1, l) for _, l in seqs], seed=page)
        q = queries(single)
        check_attention(A, single, q, attend(A, single, q))


@pytest.mark.parametrize("n", [2, 3, 8, 16, 17, 18, 19, 36, 37, 127, 128, 129, 300])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (12, 12, 64, "bf16"), (8, 8, 64, "f32")], ids=str)
def test_attention_chunk_lengths(A, heads, n):
    w = World(A, shape_of(*heads), "i8" if n % 2 else "same", 32, [(n, 3 * n + 50), (1, 77), (n, n)], seed=n)
    q = queries(w)
    check_attention(A, w, q, attend(A, w, q))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (8, 8, 64, "f32")], ids=str)
def test_attention_extreme_scores(A, heads, new):
    """Scores of hundreds, of both signs and in any order along the keys: one
    weight of nearly 1, the others down to 0."""
    w = World(A, shape_of(*heads), "same", 64, [(new, 900), (new, 131)], seed=3)
    q = queries(w, scale=60.0)
    check_attention(A, w, q, attend(A, w, q))


@pytest.mark.parametrize("new", [1, 30])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_strided_queries(A, dtype, new):
    """Queries read in place from rows of query, key and value features, and
    outputs of two runs the same to the bit."""
    w = World(A, shape_of(12, 2, 128, dtype), "i8", 64, [(new, 500), (new, 1200)], seed=4)
    q = queries(w)
    wide = torch.full((w.n_rows, w.shape.qkv_dim), math.nan, dtype=tdt(w.shape), device="cuda")
    wide[:, :w.shape.q_dim] = q
    a, b = attend(A, w, q), attend(A, w, wide[:, :w.shape.q_dim])
    assert torch.equal(a, b)
    check_attention(A, w, q, a)


def test_attention_far_pages(A):
    """Pages whose features lie past 2^32 bytes and 2^31 elements of the pool."""
    shape = shape_of(8, 4, 128, "bf16")
    first = 2 ** 31 // (4 * 128 * 128) + 100
    for new in (1, 70):
        w = World(A, shape, "same", 128, [(new, 700), (new, 200)], seed=5, first_page=first)
        q = queries(w)
        check_attention(A, w, q, attend(A, w, q))
        del w
        torch.cuda.empty_cache()


@pytest.mark.parametrize("new", [1, 20])
def test_attention_counts_on_the_device(A, new):
    """One graph, captured on another stream, over sequences that grow: lengths, rows and
    tables are read when it runs. One workspace serves calls of other shapes in between."""
    shape = shape_of(28, 4, 128, "bf16")
    full = World(A, shape, "same", 32, [(new, 900), (new, 640)], seed=6)
    ws = A.workspace(A.adadsf_paged_attention_workspace_size(full.cfg, full.cache, full.batch))
    q = queries(full)
    out = torch.empty_like(q)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        A.adadsf_paged_attention(full.cfg, full.cache, full.batch, q, out, ws=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        A.adadsf_paged_attention(full.cfg, full.cache, full.batch, q, out, ws=ws)
    other = World(A, shape, "same", 32, [(1, 33)], seed=7)
    K, V = full.K, full.V
    for l0, l1 in ((900, 640), (21, 640), (300, 20), (899, 1)):
        full.lens.copy_(torch.tensor([l0, l1], dtype=torch.int32))
        full.seqs = [(new, l0), (new, l1)]
        full.K, full.V = [K[0][:l0], K[1][:l1]], [V[0][:l0], V[1][:l1]]
        qo = queries(other)
        oo = torch.empty_like(qo)
        A.adadsf_paged_attention(other.cfg, other.cache, other.batch, qo, oo, ws=ws)
        torch.cuda.synchronize()
        out.fill_(math.nan)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(A, full, q, out)
        check_attention(A, other, qo, oo)
    assert A.adadsf_sync_check(ws) == A.OK


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (8, 8, 64, "f32")], ids=str)
@pytest.mark.parametrize("store", ["same", "i8"])
def test_attention_reports_bad_counts(A, heads, store, new):
    """A page number outside the pool is reported and its tokens count as zeros;
    lengths past the table are reported. The next call is well again."""
    w = World(A, shape_of(*heads), store, 16, [(new, 100), (new, 90)], seed=8)
    q = queries(w)
    ws = A.workspace(A.adadsf_paged_attention_workspace_size(w.cfg, w.cache, w.batch))
    good = w.table.clone()
    for wrong in (-1, w.cache.n_pages, 2 ** 31 - 1):
        w.table[0, 2] = wrong
        out = torch.empty_like(q)
        A.adadsf_paged_attention(w.cfg, w.cache, w.batch, q, out, ws=ws)
        assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
        keep = [t[0][32:48].clone() for t in (w.K, w.V)]
        for t in (w.K, w.V):
            t[0][32:48] = 0
        check_attention(A, w, q, out)
        for t, k in zip((w.K, w.V), keep):
            t[0][32:48] = k
        w.table.copy_(good)
    lens = w.lens.clone()
    w.lens[1] = w.table.shape[1] * 16 + 1
    out = torch.empty_like(q)
    A.adadsf_paged_attention(w.cfg, w.cache, w.batch, q, out, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    w.lens.copy_(lens)
    check_attention(A, w, q, attend(A, w, q, ws))


# ------------------------------------------------------------------ write and read back
def quantised64(x):
    """(whole numbers, scale) by the header's rule: a 32-bit reciprocal and products, then
    the nearest whole number, ties to even."""
    m = np.abs(x).max(-1)
    live = m >= np.float32(2.0 ** -100)
    with np.errstate(divide="ignore", invalid="ignore"):
        inv = np.where(live, np.float32(1) / m * np.float32(127), np.float32(0)).astype(np.float32)
    s = np.where(live, m / np.float32(127), np.float32(0)).astype(np.float32)
    return np.rint(x * inv[..., None]).astype(np.int64), s


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads", [(8, 8, 64, "f32", 16), (4, 2, 128, "f32", 128), (12, 12, 64, "bf16", 16),
                                   (16, 16, 128, "bf16", 32), (28, 4, 128, "bf16", 128), (6, 3, 64, "bf16", 12),
                                   (4, 4, 64, "f32", 0), (2, 1, 128, "bf16", 0)], ids=str)
def test_append_and_read(A, heads, store):
    """Keys and values of new tokens in their slots, bit for bit what the rule gives
    for the turned 32-bit values, every other slot untouched; the queries; and
    the whole cache read back."""
    shape = shape_of(*heads[:4], rotary=heads[4])
    seqs = [(3, 40), (1, 1), (0, 17), (16, 16), (5, 133), (4, 2), (0, 0), (1, 64), (1, 65)]
    page = 32
    w = World(A, shape, store, page, seqs, seed=9)
    g = torch.Generator().manual_seed(10)
    n, H, hkv, hd = w.n_rows, shape.n_heads, shape.n_kv_heads, shape.head_dim
    qkv = torch.randn(n, H + 2 * hkv, hd, generator=g)
    qkv[1, H] = 0                                            # a key of zeros
    qkv[2, H + hkv] = 2.0 ** -120                            # a value too small for a scale
    qkv[4, H + 2 * hkv - 1] *= 2.0 ** 60
    qkv = qkv.to(tdt(shape)).cuda()
    pos = torch.randint(0, 5000, (n,), generator=g).to(torch.int32).cuda()
    tab = A.adadsf_rope_table(w.cfg, 5000) if shape.rotary_dim else None
    before = [t.clone() for t in (w.k, w.v)]
    q_out = torch.empty(n, H * hd, dtype=tdt(shape), device="cuda")
    ws = A.workspace(256)
    A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv.reshape(n, -1), tab, pos, q_out, ws=ws)
    assert A.adadsf_sync_check(ws) == A.OK

    x = qkv.float().cpu().numpy()
    half = shape.rotary_dim // 2
    if half:
        t = tab.cpu().numpy()[pos.cpu().numpy()][:, None]
        a, b = x[:, :H + hkv, :half].copy(), x[:, :H + hkv, half:2 * half].copy()
        x[:, :H + hkv, :half] = a * t[..., 0] - b * t[..., 1]
        x[:, :H + hkv, half:2 * half] = b * t[..., 0] + a * t[..., 1]
        ang = pos.cpu().numpy()[:, None].astype(np.float64) * shape.rope_theta ** (-2.0 * np.arange(half) / (2 * half))
        assert np.abs(t[:, 0, :, 0] - np.cos(ang)).max() < 3e-7 and np.abs(t[:, 0, :, 1] - np.sin(ang)).max() < 3e-7
    cast = lambda y: torch.from_numpy(np.ascontiguousarray(y)).to(tdt(shape))   # noqa: E731
    assert torch.equal(q_out.cpu().reshape(n, H, hd), cast(x[:, :H]))
    r = 0
    touched = torch.zeros(w.k.shape[0], page, dtype=torch.bool)
    table = w.table.cpu()
    for b, (k, l) in enumerate(seqs):
        for i in range(k):
            p = l - k + i
            if p >= 0:
                at = (int(table[b, p // page]), p % page)
                touched[at] = True
                for pool, scale, vec in ((w.k, w.ks, x[r, H:H + hkv]), (w.v, w.vs, x[r, H + hkv:])):
                    if store == "i8":
                        whole, s = quantised64(vec)
                        assert (pool[at[0], :, at[1]].cpu().numpy() == whole).all()
                        assert (scale[at[0], :, at[1]].cpu().numpy() == s).all()
                        new = whole.astype(np.float64) * s[:, None].astype(np.float64)
                    else:
                        assert torch.equal(pool[at[0], :, at[1]].cpu(), cast(vec))
                        new = cast(vec).double().numpy()
                    (w.K if pool is w.k else w.V)[b][p] = torch.from_numpy(new).cuda()
            r += 1
    for pool, old in zip((w.k, w.v), before):
        same = (pool == old) | (pool != pool) & (old != old)
        assert same.all(-1).all(1).cpu()[~touched].all()

    # everything back: as many rows as cached tokens, one of them with a row before its first token
    rows = [l + (b == 1) for b, (_, l) in enumerate(seqs)]
    starts = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda")
    batch = A.PagedBatch(starts, w.lens, w.table, sum(rows), max(rows))
    out = [torch.full((sum(rows), hkv * hd), math.nan, dtype=tdt(shape), device="cuda") for _ in range(2)]
    A.adadsf_paged_read(w.cfg, w.cache, batch, *out, ws=ws)
    assert A.adadsf_sync_check(ws) == A.OK
    for got, want in zip(out, (w.K, w.V)):
        at = 0
        for b, (_, l) in enumerate(seqs):
            for _ in range(rows[b] - l):
                assert (got[at] == 0).all()
                at += 1
            # one rounding of the product to 32 bits, one to the type
            assert torch.equal(got[at:at + l].reshape(l, hkv, hd), want[b].float().to(tdt(shape)))
            at += l


def test_append_then_attention(A):
    """A prompt in chunks of 48, then single tokens, into an 8-bit cache: every row
    as attention over what the cache then holds."""
    shape = shape_of(12, 2, 128, "bf16")
    total, page = 130, 32
    w = World(A, shape, "i8", page, [(1, total), (1, total)], seed=11)
    tab = A.adadsf_rope_table(w.cfg, 4 * total)
    g = torch.Generator().manual_seed(12)
    at = 0
    K, V = ([torch.zeros(total, 2, 128, dtype=torch.float64, device="cuda") for _ in range(2)] for _ in range(2))
    while at < total:
        n = 48 if at < 96 else 1
        n = min(n, total - at)
        at += n
        w.seqs, w.n_rows = [(n, at), (n, at)], 2 * n
        w.starts.copy_(torch.tensor([0, n, 2 * n], dtype=torch.int32))
        w.lens.fill_(at)
        w.batch = A.PagedBatch(w.starts, w.lens, w.table, 2 * n, n)
        qkv = torch.randn(2 * n, shape.qkv_dim, generator=g).to(torch.bfloat16).cuda()
        q = torch.empty(2 * n, shape.q_dim, dtype=torch.bfloat16, device="cuda")
        A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv, tab, None, q)
        out = attend(A, w, q)
        pages = w.table.cpu()
        for b in range(2):
            for i in range(at - n, at):
                p, s = int(pages[b, i // page]), i % page
                K[b][i] = w.k[p, :, s].double() * w.ks[p, :, s].double()[:, None]
                V[b][i] = w.v[p, :, s].double() * w.vs[p, :, s].double()[:, None]
        w.K, w.V = [x[:at] for x in K], [x[:at] for x in V]
        check_attention(A, w, q, out)


@pytest.mark.parametrize("store", ["same", "i8"])
def test_append_of_infinities_and_nan(A, store):
    """A head's vector with an infinity or a NaN reads back as NaN from an 8-bit
    cache and as itself otherwise; its neighbours are untouched by it."""
    shape = shape_of(4, 2, 64, "bf16", rotary=0)
    w = World(A, shape, store, 16, [(4, 4)], seed=13)
    qkv = torch.randn(4, 8, 64).to(torch.bfloat16).cuda()
    qkv[1, 4, 7], qkv[2, 7, 0], qkv[3, 5, 63] = math.inf, math.nan, -math.inf
    ws = A.workspace(256)
    A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv.reshape(4, -1), None, None, None, ws=ws)
    k, v = (torch.empty(4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    A.adadsf_paged_read(w.cfg, w.cache, w.batch, k, v, ws=ws)
    assert A.adadsf_sync_check(ws) == A.OK
    got = torch.cat([k.reshape(4, 2, 64), v.reshape(4, 2, 64)], 1)
    want = qkv[:, 4:]
    if store == "same":
        assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.5), want.nan_to_num(0.5))
        return
    bad = ~torch.isfinite(want).all(-1)
    assert int(bad.sum()) == 3 and got[bad].isnan().all() and torch.isfinite(got[~bad]).all()


def test_append_reports_bad_places(A):
    shape = shape_of(4, 2, 64, "bf16", rotary=16)
    w = World(A, shape, "same", 16, [(2, 30), (2, 30)], seed=14)
    tab = A.adadsf_rope_table(w.cfg, 64)
    qkv = torch.randn(4, shape.qkv_dim).to(torch.bfloat16).cuda()
    ws = A.workspace(256)
    k = w.k.clone()
    page = int(w.table[1, 1])
    w.table[1, 1] = w.cache.n_pages
    A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv, tab, None, None, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    assert torch.equal(w.k[page].nan_to_num(), k[page].nan_to_num())       # that sequence's slots are not written
    out = [torch.empty(4, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    A.adadsf_paged_read(w.cfg, w.cache, w.batch, *out, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    assert (out[0][2:] == 0).all() and (out[0][:2] != 0).any()
    w.table[1, 1] = page
    pos = torch.tensor([0, 64, 63, -1], dtype=torch.int32, device="cuda")
    A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv, tab, pos, None, ws=ws)
    assert A.adadsf_sync_check(ws) == A.ERR_INVALID_ARG
    pos.clamp_(0, 63)
    A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv, tab, pos, None, ws=ws)
    assert A.adadsf_sync_check(ws) == A.OK


def test_binding_refuses(A):
    shape = shape_of(4, 2, 64, "bf16")
    cfg = A.make_cfg(shape)
    z = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt, device="cuda")   # noqa: E731
    with pytest.raises(ValueError):
        A.PagedCache(cfg, z(3, 4, 16, 64), z(3, 4, 16, 64))                       # heads
    with pytest.raises(ValueError):
        A.PagedCache(cfg, z(3, 2, 16, 64), z(3, 2, 16, 64, dt=torch.float32))
    with pytest.raises(ValueError):
        A.PagedCache(cfg, z(3, 2, 16, 64, dt=torch.int8), z(3, 2, 16, 64, dt=torch.int8))   # no scales
    cache = A.paged_cache(cfg, 3, 16, A.KV_I8)
    i32 = dict(dtype=torch.int32, device="cuda")
    starts, lens, table = (torch.zeros(n, **i32) for n in (3, 2, 8))
    with pytest.raises(ValueError):
        A.PagedBatch(starts[:2], lens, table.reshape(2, 4), 2, 1)
    with pytest.raises(ValueError):
        A.PagedBatch(starts, lens.long(), table.reshape(2, 4), 2, 1)
    batch = A.PagedBatch(starts, lens, table.reshape(2, 4), 2, 1)
    with pytest.raises(ValueError):
        A.adadsf_paged_attention(cfg, cache, batch, z(2, 128), z(2, 256))
    with pytest.raises(ValueError):
        A.adadsf_paged_attention(cfg, cache, batch, z(2, 512)[:, ::2], z(2, 256))
    with pytest.raises(A.AdadsfError) as e:
        A.adadsf_paged_attention(cfg, cache, batch, z(2, 256), z(2, 256), ws=A.workspace(256))
    assert e.value.status == A.ERR_WORKSPACE_TOO_SMALL
    with pytest.raises(ValueError):
        A.adadsf_paged_append(cfg, cache, batch, z(2, 500), None)
    with pytest.raises(A.AdadsfError):
        A.adadsf_paged_append(cfg, cache, batch, z(2, 512), None)                 # a rotary model needs its table


# ------------------------------------------------------------------ long contexts of chunks, masked infinities
@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (12, 12, 64, "bf16")], ids=str)
def test_attention_long_chunks(A, heads, store):
    """Chunks over more keys than those whose weights enter the products in two parts: a
    weight then is one bf16 (off by 2^-8 of itself at most, as the output's rounding is),
    which the bound of this test adds to the others."""
    w = World(A, shape_of(*heads), store, 64, [(40, 5000), (150, 2300), (1, 4097), (300, 700)], seed=15)
    q = queries(w)
    ref, bound = attend64(w, q)
    got = attend(A, w, q).double()
    a = bound / (2.0 ** -8 + 2.0 ** -17)      # at least softmax |V|
    assert ((got - ref).abs() <= bound + (2.0 ** -8 + 2.0 ** -16) * a).all()


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (12, 2, 128, "bf16"), (16, 1, 64, "bf16"), (12, 12, 64, "bf16")], ids=str)
def test_attention_many_odd_chunks(A, heads, store):
    """Chunks around whole row tiles (128 rows: R tokens of a group's heads) and pairs of them, over
    lengths around whole blocks of keys, enough of them to be taken as chunks."""
    R = 128 // (heads[0] // heads[1])
    new = [R - 1, R, R + 1, 2 * R - 1, 2 * R, 2 * R + 1, 4 * R + 1, 1, 0]
    seqs = [(n, n + more) for k, n in enumerate(new) for more in (0, (127, 128, 129, 1, 256)[k % 5] + k)]
    w = World(A, shape_of(*heads), store, 32, seqs + [(R, R - 3)] * 4, seed=17)
    q = queries(w)
    check_attention(A, w, q, attend(A, w, q))


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads,seqs", [((28, 4, 128, "bf16"), [(20, 20000)]), ((16, 1, 64, "bf16"), [(8, 30011)]),
                                        ((7, 1, 128, "bf16"), [(30, 9001), (1, 300), (25, 9500)])], ids=str)
def test_attention_many_pieces(A, heads, seqs, store):
    """Few rows over many keys: tens of CTAs share an item, and their pieces are joined in
    two steps. The bound is that of long chunks; a second call with the same workspace gives the same bits."""
    w = World(A, shape_of(*heads), store, 128, seqs, seed=16)
    q = queries(w)
    ref, bound = attend64(w, q)
    a = bound / (2.0 ** -8 + 2.0 ** -17)
    ws = A.workspace(A.adadsf_paged_attention_workspace_size(w.cfg, w.cache, w.batch))
    got = attend(A, w, q, ws)
    assert ((got.double() - ref).abs() <= bound + (2.0 ** -8 + 2.0 ** -16) * a).all()
    assert torch.equal(attend(A, w, q, ws), got)


def _spoil(w, what, b, place, feature):
    """Makes a cached key or value of sequence b hold an infinity or a NaN, in the pool and in the
    reference; an 8-bit vector becomes NaN as a whole (a NaN scale, numbers zero)."""
    page, slot = int(w.table[b, place // w.page]), place % w.page
    pool, scale, ref = (w.k, w.ks, w.K) if what[0] == "k" else (w.v, w.vs, w.V)
    bad = {"inf": math.inf, "-inf": -math.inf, "nan": math.nan}[what[1]]
    if scale is not None:
        pool[page, 1, slot] = 0
        scale[page, 1, slot] = math.nan
        ref[b][place, 1] = math.nan
    else:
        pool[page, 1, slot, feature] = bad
        ref[b][place, 1, feature] = bad


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("new", [1, 3, 60, 200])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (8, 8, 64, "bf16"), (8, 2, 128, "bf16"), (8, 8, 64, "f32")], ids=str)
def test_attention_infinities_of_later_tokens(A, heads, new, store):
    """Infinities and NaN in keys and values of new tokens and of old ones: rows that do not
    see them are as if they were not there, rows that see them are infinite or NaN
    where the formula is."""
    w = World(A, shape_of(*heads), store, 32, [(new, 300), (new, new), (new, 150)], seed=new)
    clean = [[x.clone() for x in t] for t in (w.K, w.V)]
    _spoil(w, ("v", "inf"), 0, 299, 5)
    _spoil(w, ("v", "nan"), 1, new - 1, 63)
    if new > 2:
        _spoil(w, ("v", "-inf"), 0, 298, 17)
        _spoil(w, ("v", "inf"), 1, new // 2, 0)
        _spoil(w, ("k", "nan"), 2, 150 - new // 3, 9)
    q = queries(w, scale=0.5)
    out = attend(A, w, q).double().reshape(w.n_rows, w.shape.n_heads, w.shape.head_dim)
    bad = [w.K, w.V]
    w.K, w.V = clean
    ref, bound = (t.reshape(out.shape) for t in attend64(w, q))
    G, r = w.shape.n_heads // w.shape.n_kv_heads, 0
    for b, (n, l) in enumerate(w.seqs):
        for i in range(n):
            seen = max(0, l - n + i + 1)
            mine = slice(G, 2 * G)                                         # the query heads of key/value head 1
            want = torch.ones(w.shape.n_heads, w.shape.head_dim, dtype=torch.bool, device="cuda")
            if not torch.isfinite(bad[0][b][:seen, 1]).all():
                want[mine] = False
            else:
                want[mine] = torch.isfinite(bad[1][b][:seen, 1]).all(0)
            got = torch.isfinite(out[r])
            assert torch.equal(got, want), (b, i)
            assert ((out[r] - ref[r]).abs()[want] <= bound[r][want]).all(), (b, i)
            r += 1


@pytest.mark.parametrize("new", [1, 3, 200])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (12, 12, 64, "bf16"), (8, 8, 64, "f32")], ids=str)
def test_attention_nan_scale_of_no_weight(A, heads, new):
    """8 bits: a visible token whose value has a NaN scale makes the row NaN however small its weight is, also where
    that is 0 in 32 bits; rows that do not see it are as without it."""
    w = World(A, shape_of(*heads), "i8", 32, [(new, 300), (new, 150 + new), (new, 200 + new)], seed=18)
    q = queries(w).abs()
    G, hd = w.shape.n_heads // w.shape.n_kv_heads, w.shape.head_dim
    clean = [[x.clone() for x in t] for t in (w.K, w.V)]
    at = [(0, 17), (1, 150 + new // 2), (2, 200 + new - 1)]          # seen by all rows, by half of them, by the last
    for b, place in at:
        _spoil(w, ("v", "nan"), b, place, 0)
        page, slot = int(w.table[b, place // w.page]), place % w.page
        w.k[page, 1, slot], w.ks[page, 1, slot] = -127, 1.0
        clean[0][b][place, 1] = -127.0
    out = attend(A, w, q).double().reshape(w.n_rows, w.shape.n_heads, hd)
    w.K, w.V = clean
    ref, bound = (t.reshape(out.shape) for t in attend64(w, q))
    r = 0
    for b, (n, l) in enumerate(w.seqs):
        for i in range(n):
            hit = l - n + i >= at[b][1]
            want = torch.ones(w.shape.n_heads, hd, dtype=torch.bool, device="cuda")
            if hit:
                want[G:2 * G] = False
            assert torch.equal(torch.isfinite(out[r]), want), (b, i)
            assert ((out[r] - ref[r]).abs()[want] <= bound[r][want]).all(), (b, i)
            r += 1


@pytest.mark.parametrize("heads,store,seqs", [((28, 4, 128, "bf16"), "same", [(300, 2000), (90, 700)]), ((12, 2, 128, "bf16"), "i8", [(250, 1500)]),
                                              ((12, 12, 64, "bf16"), "same", [(200, 900)]), ((8, 8, 64, "f32"), "same", [(70, 300)]),
                                              ((28, 4, 128, "bf16"), "same", [(1, 900), (2, 70)])], ids=str)
def test_attention_loose_bound_of_new_tokens(A, heads, store, seqs):
    """max_new is a bound of the host's: one far above the rows that there are, up to the largest int32, gives the bits
    that the closest one gives (as many CTAs share the work)."""
    w = World(A, shape_of(*heads), store, 64, seqs, seed=19)
    q = queries(w)
    want = None
    for bound in (w.n_rows, 2 ** 20, 2 ** 31 - 1):
        w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, bound)
        out = attend(A, w, q)
        check_attention(A, w, q, out)
        want = out if want is None else want
        assert torch.equal(out, want), bound


@pytest.mark.parametrize("idle", [0, 400])
@pytest.mark.parametrize("call", ["append", "read", "attention"])
def test_bad_counts_of_any_sequence_are_reported(A, call, idle):
    """Each count that breaks the header's rules is reported, also one of a sequence without rows, and the rows of
    the others are answered."""
    shape = shape_of(4, 2, 64, "bf16", rotary=0)
    w = World(A, shape, "same", 16, [(2, 30), (0, 20), (2, 40)] + [(0, 7)] * idle + [(1, 3)], seed=20)
    qkv = torch.randn(w.n_rows, shape.qkv_dim).to(torch.bfloat16).cuda()
    q = queries(w)
    ws = A.workspace(A.adadsf_paged_attention_workspace_size(w.cfg, w.cache, w.batch))

    def run():
        out = [torch.full((w.n_rows, n), 9.0, dtype=torch.bfloat16, device="cuda") for n in (128, 128, 256)]
        if call == "append":
            A.adadsf_paged_append(w.cfg, w.cache, w.batch, qkv, None, None, None, ws=ws)
        elif call == "read":
            A.adadsf_paged_read(w.cfg, w.cache, w.batch, *out[:2], ws=ws)
        else:
            A.adadsf_paged_attention(w.cfg, w.cache, w.batch, q, out[2], ws=ws)
        return A.adadsf_sync_check(ws), out

    status, good = run()
    assert status == A.OK
    room = w.table.shape[1] * 16
    last = len(w.seqs) - 1
    for name, at, wrong in (("lens", 1, -1), ("lens", 1, room + 1), ("lens", 1, 2 ** 31 - 1), ("lens", last - (idle > 0), -5),
                            ("starts", 0, -1), ("starts", last + 1, w.n_rows + 1), ("starts", 1, 2 ** 31 - 1), ("starts", 2, -2 ** 31)):
        t = getattr(w, name)
        keep = t.clone()
        t[at] = wrong
        status, out = run()
        assert status == A.ERR_INVALID_ARG, (name, at, wrong)
        t.copy_(keep)
        if name == "lens" and (at == 1 or idle):                      # an idle sequence's: the rows are as they were
            for a, b in zip(out, good):
                assert torch.equal(a, b), (name, at, wrong)
    w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, 1)     # more rows of a sequence than the host said
    assert run()[0] == A.ERR_INVALID_ARG
    w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, 2)
    status, out = run()
    assert status == A.OK
    for a, b in zip(out, good):
        assert torch.equal(a, b)


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("new", [20, 60, 130])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (8, 8, 64, "bf16"), (8, 2, 128, "bf16")], ids=str)
def test_attention_infinities_under_a_wide_table(A, heads, new, store):
    """As the test of infinities in later tokens, with tables of 2^20 tokens a sequence: few rows over what could be
    that many keys are taken as chunks, so the chunk kernel's own way with such values is what runs at these heads."""
    w = World(A, shape_of(*heads), store, 32, [(new, 300), (new, new), (new, 150), (0, 40)], seed=new)
    wide = torch.full((4, 2 ** 20 // 32), -1, dtype=torch.int32, device="cuda")
    wide[:, :w.table.shape[1]] = w.table
    w.table = wide
    w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, new)
    clean = [[x.clone() for x in t] for t in (w.K, w.V)]
    _spoil(w, ("v", "inf"), 0, 299, 5)
    _spoil(w, ("v", "nan"), 1, new - 1, 63)
    _spoil(w, ("v", "-inf"), 0, 298, 17)
    _spoil(w, ("v", "inf"), 1, new // 2, 0)
    _spoil(w, ("k", "nan"), 2, 150 - new // 3, 9)
    q = queries(w, scale=0.5)
    out = attend(A, w, q).double().reshape(w.n_rows, w.shape.n_heads, w.shape.head_dim)
    bad = [w.K, w.V]
    w.K, w.V = clean
    ref, bound = (t.reshape(out.shape) for t in attend64(w, q))
    G, r = w.shape.n_heads // w.shape.n_kv_heads, 0
    for b, (n, l) in enumerate(w.seqs):
        for i in range(n):
            seen = l - n + i + 1
            mine = slice(G, 2 * G)
            want = torch.ones(w.shape.n_heads, w.shape.head_dim, dtype=torch.bool, device="cuda")
            if not torch.isfinite(bad[0][b][:seen, 1]).all():
                want[mine] = False
            else:
                want[mine] = torch.isfinite(bad[1][b][:seen, 1]).all(0)
            assert torch.equal(torch.isfinite(out[r]), want), (b, i)
            assert ((out[r] - ref[r]).abs()[want] <= bound[r][want]).all(), (b, i)
            r += 1


@pytest.mark.parametrize("store", ["same", "i8"])
@pytest.mark.parametrize("heads", [(28, 4, 128, "bf16"), (12, 12, 64, "bf16"), (12, 2, 128, "bf16"), (16, 1, 64, "bf16")], ids=str)
def test_attention_under_a_wide_table(A, heads, store):
    """Few new tokens, some of them on nothing, under a table far wider than the longest sequence."""
    w = World(A, shape_of(*heads), store, 16, [(17, 300), (33, 33), (5, 1000), (0, 9), (1, 1), (20, 19), (19, 129), (3, 0)], seed=21)
    wide = torch.full((8, 2 ** 20 // 16), 2 ** 30, dtype=torch.int32, device="cuda")
    wide[:, :w.table.shape[1]] = w.table
    w.table = wide
    w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, 33)
    q = queries(w)
    check_attention(A, w, q, attend(A, w, q))


@pytest.mark.parametrize("heads,seqs", [((28, 4, 128, "bf16"), [(4, 9000 + 40 * b) for b in range(8)]),
                                        ((12, 2, 128, "bf16"), [(5, 20000), (1, 3), (0, 50), (3, 2), (5, 30000)]),
                                        ((12, 12, 64, "bf16"), [(32, 12000 + b) for b in range(4)]),
                                        ((16, 1, 64, "bf16"), [(2, 40000), (1, 1), (2, 2)])], ids=str)
def test_attention_two_row_groups_of_8_bits(A, heads, seqs):
    """17 to 32 packed rows a sequence over long 8-bit caches: two groups of rows a head, cut in pieces; the same under a
    table far wider than the sequences."""
    w = World(A, shape_of(*heads), "i8", 64, seqs, seed=22)
    q = queries(w)
    got = attend(A, w, q)
    check_attention(A, w, q, got)
    wide = torch.full((len(seqs), 2 ** 17), -1, dtype=torch.int32, device="cuda")
    wide[:, :w.table.shape[1]] = w.table
    w.table = wide
    w.batch = A.PagedBatch(w.starts, w.lens, w.table, w.n_rows, max(n for n, _ in seqs))
    assert torch.equal(attend(A, w, q), got)
