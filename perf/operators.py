"""Performance cases of generation from a paged cache: the operators a serving
program calls beside the depth-sparse forward, through the entry points of
paper_2607_21291_gb300.adadsf.

A layer that keeps r_l T tokens caches r_l T keys and values, another number in
every layer and sequence, so the cache is cut into pages that all layers and
sequences share. With n_b new tokens of sequence b at the end of its len_b cached
ones, one packed row a new token:

  attend   causal attention of the new tokens (one of a sequence, or a chunk)
           over the pages (adadsf_paged_attention)
  cache    rotary, quantisation and write of the new keys and values, rotary of
           the queries, then the whole cache read back as a contiguous one
           (adadsf_paged_append, adadsf_paged_read)
  sample   the next token from logits by temperature, top-k, top-p and min-p with
           a given random number a row (adadsf_sample)

store: "same" keeps keys and values in the model's type, "i8" as 8-bit whole
numbers with one fp32 scale a token and key/value head.

run() takes the library's entry points where `own` is true and elementary torch
operations in 32 bits otherwise.
"""
from __future__ import annotations

import math
import random

import torch

own = False

# backbone: heads, key/value heads, head size, rotary features, rotary base, vocabulary, type, and the rest of the
# shape that a configuration names
SHAPES = {
    "pythia-70m": dict(n_heads=8, n_kv_heads=8, head_dim=64, rotary_dim=16, theta=1e4, dtype=torch.float32),
    "pythia-160m": dict(n_heads=12, n_kv_heads=12, head_dim=64, rotary_dim=16, theta=1e4, dtype=torch.bfloat16),
    "pythia-1.4b": dict(n_heads=16, n_kv_heads=16, head_dim=128, rotary_dim=32, theta=1e4, dtype=torch.bfloat16),
    "qwen2.5-1.5b": dict(n_heads=12, n_kv_heads=2, head_dim=128, rotary_dim=128, theta=1e6, dtype=torch.bfloat16),
    "qwen2.5-7b": dict(n_heads=28, n_kv_heads=4, head_dim=128, rotary_dim=128, theta=1e6, dtype=torch.bfloat16),
}
PAGES = (16, 32, 64, 128)
VOCABS = (50304, 151936, 152064)
UNIT = 2.0 ** 40          # sampling weights are whole multiples of 1 / UNIT of the largest
MOST_SCORES = 28 * 2048 * 16384   # scores of the largest listed chunk
MOST_CACHE = 8 * 32768 * 2 * 512 * 2   # bytes of the largest listed cache
MOST_ROWS = 16 * 2048     # cached tokens of the largest listed read
MOST_LOGITS = 256 * 151936


def listed():
    return [
        # one user's next token on a small model: latency
        {"name": "decode_small", "kind": "attend", "shape": "pythia-160m", "store": "same", "page": 16, "B": 1,
         "ctx": 100, "new": 1, "ragged": False},
        # a serving batch of unequal lengths, 8-bit cache, one token each
        {"name": "decode_7b_i8", "kind": "attend", "shape": "qwen2.5-7b", "store": "i8", "page": 64, "B": 16,
         "ctx": 4096, "new": 1, "ragged": True},
        # long documents, one token each: the cache's bandwidth
        {"name": "decode_long", "kind": "attend", "shape": "qwen2.5-7b", "store": "same", "page": 128, "B": 8,
         "ctx": 32767, "new": 1, "ragged": False},
        # a chunk of a long prompt after what is cached of it: the largest
        {"name": "chunk_7b", "kind": "attend", "shape": "qwen2.5-7b", "store": "same", "page": 64, "B": 1,
         "ctx": 14336, "new": 2048, "ragged": False},
        # prompts and generated tokens in one batch, some sequences idle, 8-bit cache, odd sizes
        {"name": "chunk_ragged_i8", "kind": "attend", "shape": "qwen2.5-1.5b", "store": "i8", "page": 32, "B": 7,
         "ctx": 3001, "new": 777, "ragged": True},
        # evaluation of a small fp32 checkpoint
        {"name": "chunk_f32", "kind": "attend", "shape": "pythia-70m", "store": "same", "page": 16, "B": 3,
         "ctx": 511, "new": 129, "ragged": False},
        # one user's next token, written and read back: latency
        {"name": "cache_small", "kind": "cache", "shape": "pythia-160m", "store": "same", "page": 16, "B": 1,
         "ctx": 100, "new": 1, "ragged": False},
        # chunks of a batch of prompts into an 8-bit cache
        {"name": "cache_7b_i8", "kind": "cache", "shape": "qwen2.5-7b", "store": "i8", "page": 64, "B": 16,
         "ctx": 1536, "new": 512, "ragged": False},
        # a ragged fp32 batch into an 8-bit cache
        {"name": "cache_f32_i8", "kind": "cache", "shape": "pythia-70m", "store": "i8", "page": 32, "B": 5,
         "ctx": 300, "new": 383, "ragged": True},
        # one user's next token: latency
        {"name": "sample_one", "kind": "sample", "B": 1, "V": 50304, "dtype": "bf16"},
        # a serving batch, fp32 logits
        {"name": "sample_7b", "kind": "sample", "B": 16, "V": 152064, "dtype": "f32"},
        # several answers to every prompt of a batch
        {"name": "sample_many", "kind": "sample", "B": 256, "V": 151936, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attend", "attend", "attend", "cache", "sample", "sample"))
    if kind == "sample":
        V = rng.choice(VOCABS) if rng.random() < 0.6 else _log_int(rng, 200, 152064)
        B = _log_int(rng, 1, 256)
        dtype = rng.choice(("bf16", "f32"))
        return {"kind": "sample", "B": max(1, min(B, MOST_LOGITS // (V * (2 if dtype == "f32" else 1)))), "V": V,
                "dtype": dtype}
    shape = rng.choice(tuple(SHAPES))
    s = SHAPES[shape]
    store = rng.choice(("same", "i8"))
    token = 2 * s["n_kv_heads"] * s["head_dim"] * (4 if s["dtype"] == torch.float32 else 2)
    B, page, ragged = _log_int(rng, 1, 32), rng.choice(PAGES), rng.random() < 0.5
    if kind == "cache":
        new = 1 if rng.random() < 0.3 else _log_int(rng, 2, 700)
        B = max(1, min(B, MOST_ROWS // (2 * new)))
        ctx = _log_int(rng, 1, 4096)
        return {"kind": "cache", "shape": shape, "store": store, "page": page, "B": B,
                "ctx": max(0, min(ctx, MOST_ROWS // (4 * B) - new)), "new": new, "ragged": ragged}
    new = 1 if rng.random() < 0.45 else _log_int(rng, 2, 2048)
    ctx = _log_int(rng, 1, 32767)
    ctx = min(ctx, MOST_CACHE // token - new)
    if s["dtype"] == torch.float32:   # fp32 is for evaluating small checkpoints
        new, ctx = min(new, 700), min(ctx, 4000)
    ctx = max(0, min(ctx, MOST_SCORES // (s["n_heads"] * new) - new))
    most = min(MOST_CACHE // (token * (ctx + new)), MOST_SCORES // (s["n_heads"] * new * (ctx + new)))
    return {"kind": "attend", "shape": shape, "store": store, "page": page, "B": max(1, min(B, most)), "ctx": ctx,
            "new": new, "ragged": ragged}


# ------------------------------------------------------------------ inputs
def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + tag) & 0x7FFFFFFFFFFF)


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)


def _counts(case):
    """(new tokens, cached tokens with the new ones) of every sequence. Ragged: any number up to the case's, a sequence
    in six with none, chunks and single tokens mixed."""
    B, ctx, new = case["B"], case["ctx"], case["new"]
    if not case["ragged"]:
        return [new] * B, [ctx + new] * B
    rng = random.Random("%d %d %d %d" % (B, ctx, new, case["page"]))
    n, total = [], []
    for b in range(B):
        kind = rng.random()
        n.append(new if b == 0 else 0 if kind < 1 / 6 else 1 if kind < 1 / 3 else rng.randint(1, new))
        total.append((ctx if b == B - 1 else rng.randint(0, ctx)) + n[-1])
    return n, total


def _starts(counts):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    return at


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _quantised(x):
    """8-bit whole numbers and scales of the last axis: scale = largest / 127, x -> round(x * (127 / largest)), ties
    to even; all zeros below 2^-100."""
    most = x.abs().amax(-1)
    live = most >= 2.0 ** -100
    scale = torch.where(live, most / 127.0, 0.0)
    inv = torch.where(live, 127.0 / most, 0.0)
    return torch.round(x * inv[..., None]).to(torch.int8), scale


def _kv(seed, tag, shape):
    """Keys or values: rows that differ in size, a few strong features."""
    x = _normal(_gen(seed, tag), shape)
    x *= torch.exp(_normal(_gen(seed, tag + 1), shape[:-1] + (1,), 0.3))
    x *= torch.exp(_normal(_gen(seed, tag + 2), shape[-1:], 0.4))
    return x


def _pages(case, s, seed, lens):
    """Pool of pages in an arbitrary order, as pages come and go, and each sequence's pages (-1 past its end)."""
    page, width = case["page"], max(1, -(-max(lens) // case["page"]))
    need = [-(-n // page) for n in lens]
    n_pages = sum(need) + max(2, sum(need) // 8)
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device="cuda").tolist()
    table, at = [], 0
    for n in need:
        table += order[at:at + n] + [-1] * (width - n)
        at += n
    st = {"table": _int32(table).reshape(len(lens), width)}
    shape = (n_pages, s["n_kv_heads"], page, s["head_dim"])
    for i, name in enumerate("kv"):
        x = _kv(seed, 10 + 10 * i, shape)
        st[name + "_scale"] = None
        if case["store"] == "i8":
            st[name], st[name + "_scale"] = _quantised(x)
        else:
            st[name] = x.to(s["dtype"])
        del x
    return st


def prepare(case, seed):
    st = {"case": case}
    if case["kind"] == "sample":
        B, V = case["B"], case["V"]
        g = _gen(seed, 2)
        # logits of a language model: a wide bulk and a tail of likely tokens, sharper in some rows
        x = _normal(g, (B, V), 2.0) * torch.exp(_normal(_gen(seed, 3), (B, 1), 0.2))
        likely = torch.randint(0, V, (B, 24), generator=g, device="cuda")
        x.scatter_add_(1, likely, torch.rand(B, 24, generator=g, device="cuda") * 12.0)
        st["logits"] = (x + 0.0).to(torch.bfloat16 if case["dtype"] == "bf16" else torch.float32) + 0.0
        r = torch.rand(6, B, generator=_gen(seed, 4), device="cuda")
        # every user's own settings: one in eight greedy, half with top-k, three in four with top-p, one in four with min-p
        st["temperature"] = torch.where(r[0] < 0.125, 0.0, 0.5 + r[0])
        st["top_k"] = torch.where(r[1] < 0.5, 0.0, torch.exp(r[1] * 12.0 - 5.0)).to(torch.int32).clamp_(max=V)
        st["top_p"] = torch.where(r[2] < 0.25, 1.0, 0.4 + 0.599 * r[2])
        st["min_p"] = torch.where(r[3] < 0.75, 0.0, 0.2 * (r[3] - 0.75))
        st["u"] = r[4]
        st["token"] = torch.empty(B, dtype=torch.int32, device="cuda")
        st["logprob"] = torch.empty(B, dtype=torch.float32, device="cuda")
        return st
    s = SHAPES[case["shape"]]
    n, lens = _counts(case)
    rows, kv_rows = sum(n), sum(lens)
    st.update(_pages(case, s, seed, lens))
    st["lens"], st["starts"] = _int32(lens), _int32(_starts(n))
    st["longest"], st["most_new"], st["rows"] = max(lens), max(n), rows
    H, hd, hkv = s["n_heads"], s["head_dim"], s["n_kv_heads"]
    if case["kind"] == "attend":
        st["q"] = _normal(_gen(seed, 5), (rows, H * hd), 1.2).to(s["dtype"])
        st["out"] = torch.empty_like(st["q"])
    else:
        st["qkv"] = _kv(seed, 5, (rows, H + 2 * hkv, hd)).reshape(rows, -1).to(s["dtype"])
        # original positions of the kept tokens: ascending, with gaps
        st["n_pos"] = 3 * (case["ctx"] + case["new"]) + 8
        first = torch.tensor([2 * (l - k) for l, k in zip(lens, n)], device="cuda")
        gaps = torch.randint(0, 2, (rows,), generator=_gen(seed, 8), device="cuda")
        seq, i = _row_places(st)
        st["pos"] = (first[seq] + 2 * i + gaps).to(torch.int32)
        half = s["rotary_dim"] // 2
        turn = s["theta"] ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
        ang = torch.arange(st["n_pos"], device="cuda", dtype=torch.float64)[:, None] * turn
        st["tab"] = torch.stack([torch.cos(ang), torch.sin(ang)], -1).float()
        st["q_out"] = torch.empty(rows, H * hd, device="cuda", dtype=s["dtype"])
        st["read_starts"], st["read_rows"] = _int32(_starts(lens)), kv_rows
        st["k_out"] = torch.empty(kv_rows, hkv * hd, device="cuda", dtype=s["dtype"])
        st["v_out"] = torch.empty_like(st["k_out"])
    if own:   # the handles that a program keeps: configuration, cache, batch and workspace
        from paper_2607_21291_gb300 import adadsf as A
        from paper_2607_21291_gb300 import synth as S
        shapes = {x.name: x for x in (S.PYTHIA_70M, S.PYTHIA_160M, S.PYTHIA_1_4B, S.QWEN25_1_5B, S.QWEN25_7B)}
        st["cfg"] = A.make_cfg(shapes[case["shape"]])
        st["cache"] = A.PagedCache(st["cfg"], st["k"], st["v"], st["k_scale"], st["v_scale"])
        st["batch"] = A.PagedBatch(st["starts"], st["lens"], st["table"], rows, st["most_new"])
        if case["kind"] == "attend":
            st["ws"] = A.workspace(A.adadsf_paged_attention_workspace_size(st["cfg"], st["cache"], st["batch"]))
        else:
            st["read_batch"] = A.PagedBatch(st["read_starts"], st["lens"], st["table"], kv_rows, st["longest"])
            st["ws"] = A.workspace(256)
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    kind = st["case"]["kind"]
    if not own:
        return {"attend": _plain_attend, "cache": _plain_cache, "sample": _plain_sample}[kind](st)
    from paper_2607_21291_gb300 import adadsf as A
    if kind == "sample":
        A.adadsf_sample(st["logits"], st["u"], st["token"], temperature=st["temperature"], top_k=st["top_k"],
                        top_p=st["top_p"], min_p=st["min_p"], logprob=st["logprob"])
        return {"token": st["token"], "logprob": st["logprob"]}
    if kind == "attend":
        A.adadsf_paged_attention(st["cfg"], st["cache"], st["batch"], st["q"], st["out"], ws=st["ws"])
        return st["out"]
    A.adadsf_paged_append(st["cfg"], st["cache"], st["batch"], st["qkv"], st["tab"], st["pos"], st["q_out"], ws=st["ws"])
    A.adadsf_paged_read(st["cfg"], st["cache"], st["read_batch"], st["k_out"], st["v_out"], ws=st["ws"])
    return {"q": st["q_out"], "k": st["k_out"], "v": st["v_out"]}


# ------------------------------------------------------------------ plain forms (torch, 32 bits)
def _row_places(st, starts="starts", rows="rows"):
    """Sequence of every packed row, and its place among the sequence's rows."""
    r = torch.arange(st[rows], device="cuda")
    at = st[starts].long()
    seq = torch.searchsorted(at, r, right=True) - 1
    return seq, r - at[seq]


def _plain_attend(st):
    case = st["case"]
    s = SHAPES[case["shape"]]
    H, hkv, hd, page = s["n_heads"], s["n_kv_heads"], s["head_dim"], case["page"]
    B, L, n, G = case["B"], st["longest"], st["most_new"], s["n_heads"] // s["n_kv_heads"]
    if st["rows"] == 0:
        return torch.zeros_like(st["q"])
    table = st["table"].long().clamp(min=0)
    span = table.shape[1] * page
    kv = []
    for name in ("k", "v"):
        x = st[name][table].float()                           # [B, pages, hkv, page, hd]
        if st[name + "_scale"] is not None:
            x = x * st[name + "_scale"][table][..., None]
        kv.append(x.permute(0, 2, 1, 3, 4).reshape(B, hkv, span, hd)[:, :, :L])
    starts, lens = st["starts"].long(), st["lens"].long()
    count = starts[1:] - starts[:-1]
    i = torch.arange(n, device="cuda")
    at = (starts[:-1, None] + i).clamp(max=st["rows"] - 1)      # [B, n]
    q = st["q"].float()[at].reshape(B, n, hkv, G, hd).permute(0, 2, 3, 1, 4).reshape(B, hkv, G * n, hd)
    score = (q @ kv[0].transpose(-1, -2)).div_(math.sqrt(hd)).reshape(B, hkv, G, n, L)
    last = lens[:, None] - count[:, None] + i                   # a new token's own place in the cache
    hidden = torch.arange(L, device="cuda") > last[..., None]   # [B, n, L]
    score.masked_fill_(hidden[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True).clamp_(min=-3e38)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.reshape(B, hkv, G * n, L) @ kv[1]).reshape(B, hkv, G, n, hd) / total.clamp(min=1e-30)
    seq, place = _row_places(st)
    return o.permute(0, 3, 1, 2, 4)[seq, place].reshape(st["rows"], H * hd).to(s["dtype"])


def _turned(x, cos, sin):
    half = cos.shape[-1]
    a, b = x[..., :half], x[..., half:2 * half]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1)


def _plain_cache(st):
    case = st["case"]
    s = SHAPES[case["shape"]]
    H, hkv, hd, page, rows = s["n_heads"], s["n_kv_heads"], s["head_dim"], case["page"], st["rows"]
    lens, starts, table = st["lens"].long(), st["starts"].long(), st["table"].long()
    x = st["qkv"].float().reshape(rows, H + 2 * hkv, hd)
    turn = st["tab"][st["pos"].long()]
    qk = _turned(x[:, :H + hkv], turn[:, None, :, 0], turn[:, None, :, 1])
    seq, i = _row_places(st)
    at = lens[seq] - (starts[seq + 1] - starts[seq]) + i
    where = (table[seq, at // page], slice(None), at % page)
    for name, new in (("k", qk[:, H:]), ("v", x[:, H + hkv:])):
        if st[name + "_scale"] is not None:
            st[name][where], st[name + "_scale"][where] = _quantised(new)
        else:
            st[name][where] = new.to(s["dtype"])
    seq, at = _row_places(st, "read_starts", "read_rows")
    where = (table[seq, at // page], slice(None), at % page)
    back = []
    for name in ("k", "v"):
        y = st[name][where].float()
        if st[name + "_scale"] is not None:
            y = y * st[name + "_scale"][where][..., None]
        back.append(y.reshape(-1, hkv * hd).to(s["dtype"]))
    return {"q": qk[:, :H].reshape(rows, H * hd).to(s["dtype"]), "k": back[0], "v": back[1]}


def _plain_sample(st):
    """Tokens in descending order of logit (equal ones by index) are kept while they are among the first top_k, while
    the weight before them is under top_p of the first top_k's, and while their weight is min_p of the largest or
    more. The token is the first, in the order of the vocabulary, whose running weight is over u times the kept."""
    x = st["logits"].float()
    B, V = x.shape
    t, k = st["temperature"][:, None], st["top_k"].long()[:, None]
    top = x.amax(-1, keepdim=True)
    z = torch.where(x == top, 0.0, (x - top) * (1.0 / t))
    w = torch.exp(z)
    whole = (w.double() * UNIT).round().long()
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    rank = torch.arange(V, device="cuda")
    ws = whole.gather(1, order)
    keep = (rank < torch.where(k > 0, k, V)).expand(B, V)
    ws = torch.where(keep, ws, 0)
    running = ws.cumsum(-1)
    total = running[:, -1:]
    top_p = st["top_p"].double()[:, None]
    keep = keep & ((top_p >= 1.0) | ((running - ws).double() < top_p * total.double())) & (w.gather(1, order) >= st["min_p"][:, None])
    keep = keep | (rank == 0)
    kept = torch.zeros(B, V, dtype=torch.bool, device="cuda").scatter_(1, order, keep)
    running = torch.where(kept, whole, 0).cumsum(-1)
    total = running[:, -1:]
    mark = torch.minimum((st["u"].double()[:, None] * total.double()).long(), total - 1)
    drawn = torch.searchsorted(running, mark, right=True)
    greedy = t <= 0.0
    token = torch.where(greedy, order[:, :1], drawn)
    rest = ((total - int(UNIT)).double() / UNIT).float()
    logprob = torch.where(greedy, 0.0, z.gather(1, token) - torch.log1p(rest))
    return {"token": token[:, 0].to(torch.int32), "logprob": logprob[:, 0]}


# ------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "sample":
        size = case["B"] * case["V"]
        return {"bytes": float(size * (2 if case["dtype"] == "bf16" else 4)), "flops": 4.0 * size}
    s = SHAPES[case["shape"]]
    es = 4 if s["dtype"] == torch.float32 else 2
    hkv, hd = s["n_kv_heads"], s["head_dim"]
    q = s["n_heads"] * hd
    n, lens = _counts(case)
    cached = 2 * hkv * (hd + 4 if case["store"] == "i8" else hd * es)      # bytes of one cached token
    if case["kind"] == "attend":
        return {"bytes": float(sum(l for k, l in zip(n, lens) if k) * cached + 2 * sum(n) * q * es),
                "flops": sum(4.0 * q * (k * (l - k) + k * (k + 1) / 2) for k, l in zip(n, lens))}
    # the new rows in, turned queries and cached tokens out; every cached token in (the new ones are at hand), and out
    return {"bytes": float(sum(n) * ((2 * q + 2 * hkv * hd) * es + cached) + (sum(lens) - sum(n)) * cached +
                           sum(lens) * 2 * hkv * hd * es),
            "flops": float(sum(n) * (q + hkv * hd) * 3 + (sum(n) + sum(lens)) * 2 * hkv * hd)}


# ------------------------------------------------------------------ 64-bit references
def exact(case, seed):
    st = prepare(case, seed)
    return {"attend": _exact_attend, "cache": _exact_cache, "sample": _exact_sample}[case["kind"]](st)


def _exact_attend(st):
    case = st["case"]
    s = SHAPES[case["shape"]]
    H, hkv, hd, G = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["n_heads"] // s["n_kv_heads"]
    n, lens = _counts(case)
    starts = _starts(n)
    out = torch.zeros(sum(n), H, hd, dtype=torch.float64, device="cuda")
    for b, (k, l) in enumerate(zip(n, lens)):
        if k == 0:
            continue
        pages = st["table"][b, :-(-l // case["page"])].tolist()
        q = st["q"][starts[b]:starts[b + 1]].double().reshape(k, H, hd)
        allowed = torch.ones(k, l, dtype=torch.bool, device="cuda").tril(l - k)
        for g in range(hkv):
            key, val = (torch.cat([_as64(st, name, p, g) for p in pages])[:l] for name in ("k", "v"))
            for h in range(g * G, g * G + G):
                a = torch.softmax((q[:, h] @ key.T * hd ** -0.5).masked_fill(~allowed, -math.inf), -1)
                out[starts[b]:starts[b + 1], h] = a @ val
    return out.reshape(sum(n), H * hd)


def _as64(st, name, page, head):
    x = st[name][page, head].double()
    scale = st[name + "_scale"]
    return x if scale is None else x * scale[page, head].double()[:, None]


def _exact_cache(st):
    """The queries turned and the cached values as they are before any rounding: those of new tokens from the formula."""
    case = st["case"]
    s = SHAPES[case["shape"]]
    H, hkv, hd, half = s["n_heads"], s["n_kv_heads"], s["head_dim"], s["rotary_dim"] // 2
    n, lens = _counts(case)
    x = st["qkv"].double().reshape(sum(n), H + 2 * hkv, hd)
    turn = torch.view_as_complex(st["tab"].double().contiguous())[st["pos"].long()][:, None]
    y = torch.complex(x[:, :H + hkv, :half], x[:, :H + hkv, half:2 * half]) * turn
    x[:, :H + hkv, :half], x[:, :H + hkv, half:2 * half] = y.real, y.imag
    k_out = torch.empty(sum(lens), hkv, hd, dtype=torch.float64, device="cuda")
    v_out = torch.empty_like(k_out)
    row = at = 0
    for b, (k, l) in enumerate(zip(n, lens)):
        for name, out, first in (("k", k_out, H), ("v", v_out, H + hkv)):
            pages = st["table"][b, :-(-l // case["page"])].long()
            if pages.numel():
                old = st[name][pages].double()
                if st[name + "_scale"] is not None:
                    old = old * st[name + "_scale"][pages].double()[..., None]
                out[at:at + l] = old.transpose(1, 2).reshape(-1, hkv, hd)[:l]
            new = x[row:row + k, first:first + hkv]
            if case["store"] == "i8":
                step = new.abs().amax(-1, keepdim=True) / 127.0
                new = torch.round(new / step) * step
            out[at + l - k:at + l] = new
        row, at = row + k, at + l
    return {"q": x[:, :H].reshape(-1, H * hd), "k": k_out.reshape(-1, hkv * hd), "v": v_out.reshape(-1, hkv * hd)}


def _exact_sample(st):
    """Log-probabilities of the drawn tokens; the tokens themselves are whole numbers."""
    x = st["logits"].double()
    out = []
    for b in range(x.shape[0]):
        t, k, p, floor, u = (float(st[name][b]) for name in ("temperature", "top_k", "top_p", "min_p", "u"))
        if t <= 0.0:
            out.append(0.0)
            continue
        z = (x[b] - x[b].max()) / t
        w = torch.exp(z)
        ranked, order = torch.sort(x[b], descending=True, stable=True)
        r = w[order]
        if k > 0:
            r = r * (torch.arange(r.numel(), device="cuda") < k)
        keep = r >= max(floor, 2.0 ** -41)
        if p < 1.0:
            keep &= r.cumsum(0) - r < p * r.sum()
        keep[0] = True
        kept = torch.zeros_like(w)
        kept[order[keep]] = w[order[keep]]
        c = kept.cumsum(0)
        i = min(int(torch.searchsorted(c, u * c[-1], right=True)), w.numel() - 1)
        out.append(float(z[i] - torch.log(c[-1])))
    return {"token": None, "logprob": torch.tensor(out, dtype=torch.float64, device="cuda")}
