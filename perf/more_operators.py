"""Performance cases of the two ends of a language model in training: what lies
between token ids and the first layer, and between the last layer and the loss,
through the entry points of paper_2607_21291_gb300.adadsf.

  ce       cross entropy of the next token through the LM head, in pieces of the
           vocabulary, no logit stored (adadsf_head_loss, adadsf_head_loss_backward):
           a row's logits are h W^T, its loss lse - l[target]
  distill  a teacher's top logits as targets (adadsf_distill_loss, ..._backward):
           p the softmax of the teacher's k logits / T, q that of all of the row's
           logits / T, the loss T^2 sum p (log p - log q)
  norm     LayerNorm or RMSNorm and its gradients, the weights' among them
           (adadsf_norm_forward, adadsf_norm_backward)
  embed    scaled rows of the embedding and the table's gradient, summed over
           sorted tokens (adadsf_embed_forward, adadsf_embed_backward)

Rows without a target (prompts, padding; target or ids of -1) have no loss and no
gradient. run() takes the library's entry points where `own` is true and
elementary torch operations in 32 bits otherwise.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

# hidden size and vocabulary of the backbones, and the type they are trained in here
SHAPES = {
    "pythia-70m": (512, 50304, "f32"),
    "pythia-160m": (768, 50304, "bf16"),
    "pythia-1.4b": (2048, 50304, "bf16"),
    "qwen2.5-1.5b": (1536, 151936, "bf16"),
    "qwen2.5-7b": (3584, 152064, "bf16"),
}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZES = {"f32": 4, "bf16": 2}
MOST_PRODUCT = {"bf16": 4096 * 152064 * 3584, "f32": 777 * 50304 * 512}   # rows x vocabulary x features of the largest
MOST_LOGITS = 16384 * 152064              # of a plain form, which keeps them
MOST_ROW_VALUES = 65536 * 3584            # values of the largest norm and embedding
MOST_EXACT = 4e12                         # multiply-adds of a product in 64 bits that take some seconds
EPS = 1e-5


def _head(name, kind, shape, B, T, train, **more):
    d, V, dtype = SHAPES[shape]
    return {"name": name, "kind": kind, "d": d, "V": V, "dtype": dtype, "B": B, "T": T, "train": train, **more}


def listed():
    return [
        # log-probabilities of one short answer: latency
        _head("ce_score_160m", "ce", "pythia-160m", 1, 24, False),
        # fine-tuning batches: prompts and padding carry no loss
        _head("ce_train_1_4b", "ce", "pythia-1.4b", 8, 511, True),
        # the same at the largest head
        _head("ce_train_7b", "ce", "qwen2.5-7b", 2, 2048, True),
        # a small fp32 checkpoint
        _head("ce_train_f32", "ce", "pythia-70m", 3, 259, True),
        # stored logits of a teacher, 64 a token
        _head("distill_1_5b", "distill", "qwen2.5-1.5b", 4, 600, True, k=64, temp=2.0),
        # evaluation against a teacher's few logits
        _head("distill_eval_f32", "distill", "pythia-70m", 1, 77, False, k=8, temp=1.0),
        # one short sequence: latency
        {"name": "norm_small", "kind": "norm", "d": 768, "dtype": "bf16", "rows": 24, "rms": False, "res": False},
        # a training batch of the largest shape, the residual's gradient added
        {"name": "norm_7b", "kind": "norm", "d": 3584, "dtype": "bf16", "rows": 65536, "rms": True, "res": True},
        # a batch of a small fp32 checkpoint
        {"name": "norm_f32", "kind": "norm", "d": 512, "dtype": "f32", "rows": 2044, "rms": False, "res": True},
        # one short sequence: the table's gradient is almost all zeros
        {"name": "embed_small", "kind": "embed", "d": 768, "V": 50304, "dtype": "bf16", "B": 1, "T": 100, "scale": 1.0},
        # a training batch of the largest shape
        {"name": "embed_7b", "kind": "embed", "d": 3584, "V": 152064, "dtype": "bf16", "B": 16, "T": 4096, "scale": 1.0},
        # a padded fp32 batch, rows scaled by sqrt(d)
        {"name": "embed_f32", "kind": "embed", "d": 512, "V": 50304, "dtype": "f32", "B": 4, "T": 511,
         "scale": math.sqrt(512.0)},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, dtype, hi):
    """A hidden size: a whole number of 16-byte vectors."""
    unit = 16 // SIZES[dtype]
    return unit * _log_int(rng, 64 // unit, hi // unit)


def draw(rng):
    kind = rng.choice(("ce", "ce", "distill", "norm", "embed"))
    shape = rng.choice(tuple(SHAPES))
    d, V, dtype = SHAPES[shape]
    if rng.random() < 0.4:
        dtype = rng.choice(("f32", "bf16", "bf16"))
        d, V = _width(rng, dtype, 5120), _log_int(rng, 100, 152064)
    B = _log_int(rng, 1, 16)
    if kind in ("ce", "distill"):
        most = min(MOST_PRODUCT[dtype] // (V * d), MOST_LOGITS // V)
        B = min(B, most)
        T = min(_log_int(rng, 1, 4096), most // B)
        case = {"kind": kind, "d": d, "V": V, "dtype": dtype, "B": B, "T": T, "train": rng.random() < 0.7}
        if kind == "distill":
            case["k"], case["temp"] = min(V, _log_int(rng, 1, 128)), rng.choice((1.0, 2.0, 0.7, 4.0))
        return case
    if kind == "norm":
        rows = min(_log_int(rng, 1, 65536), MOST_ROW_VALUES // (d * (2 if dtype == "f32" else 1)))
        return {"kind": "norm", "d": d, "dtype": dtype, "rows": rows, "rms": rng.random() < 0.5, "res": rng.random() < 0.5}
    T = min(_log_int(rng, 1, 8192), MOST_ROW_VALUES // (B * d * (2 if dtype == "f32" else 1)))
    return {"kind": "embed", "d": d, "V": V, "dtype": dtype, "B": B, "T": T, "scale": rng.choice((1.0, math.sqrt(d)))}


# ------------------------------------------------------------------ inputs
def _gen(seed, tag):
    return torch.Generator(device="cuda").manual_seed((int(seed) * 1000003 + tag) & 0x7FFFFFFFFFFF)


def _normal(g, shape, std=1.0):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).mul_(std)


def _used(case):
    """Which tokens count: sequence b has a prompt before them and padding behind; the last of a sequence has no
    next token. A batch of one has neither."""
    B, T = case["B"], case["T"]
    rng = random.Random("%d %d" % (B, T))
    used = np.zeros((B, T), dtype=bool)
    for b in range(B):
        first = 0 if B == 1 else rng.randint(0, T // 4)
        last = T if B == 1 else T - rng.randint(0, T // 6)
        used[b, first:max(first, last)] = True
    return used.reshape(-1)


def _shares(V):
    """How often the tokens of a vocabulary come, by rank (Zipf's law)."""
    p = 1.0 / (np.arange(V, dtype=np.float64) + 2.7)
    return p / p.sum()


def _tokens(seed, tag, n, V):
    cum = torch.from_numpy(np.cumsum(_shares(V))).to("cuda")
    u = torch.rand(n, generator=_gen(seed, tag), device="cuda", dtype=torch.float64)
    rank = torch.searchsorted(cum, u, right=True).clamp_(max=V - 1)
    return torch.randperm(V, generator=_gen(seed, tag + 1), device="cuda")[rank]


def prepare(case, seed):
    st = {"case": case}
    d, dtype = case["d"], DTYPES[case["dtype"]]
    if case["kind"] == "norm":
        n = case["rows"]
        # residual stream: rows of different size, a few strong features, a mean
        x = _normal(_gen(seed, 1), (n, d)) * torch.exp(_normal(_gen(seed, 2), (n, 1), 0.5))
        x += _normal(_gen(seed, 3), (1, d), 0.5)
        st["x"] = x.to(dtype)
        st["w"] = (1.0 + _normal(_gen(seed, 4), (d,), 0.1)).to(dtype)
        st["b"] = None if case["rms"] else _normal(_gen(seed, 5), (d,), 0.1).to(dtype)
        st["dy"] = _normal(_gen(seed, 6), (n, d), 1e-3).to(dtype)
        st["res"] = _normal(_gen(seed, 7), (n, d), 1e-3).to(dtype) if case["res"] else None
        st["y"], st["dx"] = torch.empty_like(st["x"]), torch.empty_like(st["x"])
        st["mean"] = None if case["rms"] else torch.empty(n, device="cuda")
        st["rstd"] = torch.empty(n, device="cuda")
        st["dw"] = torch.empty(d, device="cuda")
        st["db"] = None if case["rms"] else torch.empty(d, device="cuda")
    else:
        V, n = case["V"], case["B"] * case["T"]
        used = torch.from_numpy(_used(case)).to("cuda")
        token = torch.where(used, _tokens(seed, 1, n, V), -1).to(torch.int32)
        if case["kind"] == "embed":
            st["ids"], st["table"] = token, _normal(_gen(seed, 3), (V, d), 0.02).to(dtype)
            st["dy"] = _normal(_gen(seed, 4), (n, d), 1e-3).to(dtype)
            st["y"], st["dtable"] = torch.empty_like(st["dy"]), torch.empty_like(st["table"])
        else:
            w = _normal(_gen(seed, 3), (V, d), 0.02)
            # final hidden states that point to their target, some more than others
            lift = torch.rand(n, 1, generator=_gen(seed, 4), device="cuda") * (16.0 / (d * 0.0004))
            h = _normal(_gen(seed, 5), (n, d), min(1.0, 96.0 / math.sqrt(d)))
            h += lift * w[token.clamp(min=0).long()]
            st["h"], st["w"], st["target"] = h.to(dtype), w.to(dtype), token
            del w, h
            st["loss"], st["lse"] = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
            # the mean over the tokens that count
            st["g"] = torch.full((n,), 1.0 / max(1, int(_used(case).sum())), device="cuda")
            if case["train"]:
                st["dh"], st["dw"] = torch.empty_like(st["h"]), torch.empty_like(st["w"])
            if case["kind"] == "distill":
                k = case["k"]
                # the teacher's classes differ, the target among them as a rule; fewer are stored for some tokens
                step = V // k
                at = torch.randint(0, step, (n, k), generator=_gen(seed, 6), device="cuda")
                idx = (token[:, None].clamp(min=0) + torch.arange(k, device="cuda") * step) % (step * k)
                idx = torch.where(torch.arange(k, device="cuda") > 0, idx - idx % step + at, idx)
                logit = 10.0 - 3.0 * torch.log1p(torch.arange(k, device="cuda", dtype=torch.float32))
                logit = logit + _normal(_gen(seed, 7), (n, k), 0.5)
                short = torch.rand(n, 1, generator=_gen(seed, 8), device="cuda") < 0.1
                gone = (token[:, None] < 0) | (short & (torch.arange(k, device="cuda") >= max(1, k // 2)))
                st["idx"], st["logit"] = torch.where(gone, -1, idx).to(torch.int32), logit
    if own:   # the workspace that a program keeps
        from paper_2607_21291_gb300 import adadsf as A
        if case["kind"] == "norm":
            st["ws"] = A.workspace(A.adadsf_norm_backward_workspace_size(st["x"].shape[0], d))
        elif case["kind"] == "embed":
            st["ws"] = A.workspace(A.adadsf_embed_backward_workspace_size(n, V, d))
        else:
            st["ws"] = A.workspace(A.adadsf_head_workspace_size(n, d, V, st["h"].dtype, case.get("k", 1)))
    return st


# ------------------------------------------------------------------ one pass
def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        return {"ce": _plain_ce, "distill": _plain_distill, "norm": _plain_norm, "embed": _plain_embed}[kind](st)
    from paper_2607_21291_gb300 import adadsf as A
    if kind == "norm":
        A.adadsf_norm_forward(st["x"], st["w"], st["b"], st["y"], eps=EPS, mean=st["mean"], rstd=st["rstd"])
        A.adadsf_norm_backward(st["dy"], st["x"], st["w"], st["rstd"], st["dx"], mean=st["mean"], add=st["res"],
                               grad_w=st["dw"], grad_b=st["db"], ws=st["ws"])
        return {"y": st["y"], "dx": st["dx"], "dw": st["dw"], "db": st["db"]}
    if kind == "embed":
        A.adadsf_embed_forward(st["ids"], st["table"], st["y"], scale=case["scale"], ws=st["ws"])
        A.adadsf_embed_backward(st["ids"], st["dy"], st["dtable"], scale=case["scale"], ws=st["ws"])
        return {"y": st["y"], "dtable": st["dtable"]}
    if kind == "ce":
        A.adadsf_head_loss(st["h"], st["w"], st["target"], loss=st["loss"], lse=st["lse"], ws=st["ws"])
        if case["train"]:
            A.adadsf_head_loss_backward(st["h"], st["w"], st["target"], st["lse"], grad_loss=st["g"], grad_h=st["dh"],
                                        grad_w=st["dw"], ws=st["ws"])
    else:
        A.adadsf_distill_loss(st["h"], st["w"], st["idx"], st["logit"], temperature=case["temp"], loss=st["loss"],
                              lse=st["lse"], ws=st["ws"])
        if case["train"]:
            A.adadsf_distill_loss_backward(st["h"], st["w"], st["idx"], st["logit"], st["lse"],
                                           temperature=case["temp"], grad_loss=st["g"], grad_h=st["dh"],
                                           grad_w=st["dw"], ws=st["ws"])
    if case["train"]:
        return {"loss": st["loss"], "lse": st["lse"], "dh": st["dh"], "dw": st["dw"]}
    return {"loss": st["loss"], "lse": st["lse"]}


# ------------------------------------------------------------------ plain forms (torch, 32 bits)
def _plain_lse(z):
    top = z.amax(-1, keepdim=True)
    return (top + torch.log(torch.exp(z - top).sum(-1, keepdim=True)))[:, 0]


def _plain_grads(st, g, h, w):
    dtype = st["h"].dtype
    return {"dh": (g @ w).to(dtype), "dw": (g.T @ h).to(dtype)}


def _plain_ce(st):
    h, w = st["h"].float(), st["w"].float()
    used = st["target"] >= 0
    at = st["target"].clamp(min=0).long()[:, None]
    z = h @ w.T
    lse = _plain_lse(z)
    out = {"loss": torch.where(used, lse - z.gather(1, at)[:, 0], 0.0), "lse": torch.where(used, lse, 0.0)}
    if st["case"]["train"]:
        q = z.sub_(lse[:, None]).exp_()
        q.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
        q.mul_(torch.where(used, st["g"], 0.0)[:, None])
        out.update(_plain_grads(st, q, h, w))
    return out


def _plain_distill(st):
    h, w, temp = st["h"].float(), st["w"].float(), st["case"]["temp"]
    there = st["idx"] >= 0
    used = there.any(-1)
    at = st["idx"].clamp(min=0).long()
    t = torch.where(there, st["logit"] / temp, -math.inf)
    top = torch.where(used[:, None], t.amax(-1, keepdim=True), 0.0)
    e = torch.exp(t - top)
    total = torch.where(used[:, None], e.sum(-1, keepdim=True), 1.0)
    p, log_p = e / total, t - top - torch.log(total)
    z = (h @ w.T).div_(temp)
    lse = _plain_lse(z)
    kl = torch.where(there & (p > 0), p * (log_p - (z.gather(1, at) - lse[:, None])), 0.0).sum(-1)
    out = {"loss": torch.where(used, temp * temp * kl, 0.0), "lse": torch.where(used, lse, 0.0)}
    if st["case"]["train"]:
        q = z.sub_(lse[:, None]).exp_()
        q.scatter_add_(1, at, torch.where(there, -p, 0.0))
        q.mul_(torch.where(used, st["g"] * temp, 0.0)[:, None])
        out.update(_plain_grads(st, q, h, w))
    return out


def _plain_norm(st):
    x, w, dy = st["x"].float(), st["w"].float(), st["dy"].float()
    rms = st["case"]["rms"]
    c = x if rms else x - x.mean(-1, keepdim=True)
    rstd = 1.0 / torch.sqrt((c * c).mean(-1, keepdim=True) + EPS)
    xhat = c * rstd
    y = xhat * w if rms else xhat * w + st["b"].float()
    a = dy * w
    dx = a - xhat * (a * xhat).mean(-1, keepdim=True)
    if not rms:
        dx = dx - a.mean(-1, keepdim=True)
    dx = dx * rstd
    if st["res"] is not None:
        dx = dx + st["res"].float()
    dtype = st["x"].dtype
    # sums over many rows: in 64 bits
    return {"y": y.to(dtype), "dx": dx.to(dtype), "dw": (dy * xhat).sum(0, dtype=torch.float64).float(),
            "db": None if rms else dy.sum(0, dtype=torch.float64).float()}


def _plain_embed(st):
    ids, table, scale = st["ids"].long(), st["table"], st["case"]["scale"]
    used = (ids >= 0)[:, None]
    at = ids.clamp(min=0)
    y = torch.where(used, table[at].float() * scale, 0.0).to(table.dtype)
    grad = torch.zeros(table.shape, dtype=torch.float32, device="cuda")
    grad.index_add_(0, at, torch.where(used, st["dy"].float(), 0.0))
    return {"y": y, "dtable": grad.mul_(scale).to(table.dtype)}


# ------------------------------------------------------------------ work
def work(case):
    d, es = case["d"], SIZES[case["dtype"]]
    if case["kind"] == "norm":
        # x read once by each pass, dy (and the residual's gradient) in, y and dx out
        n = case["rows"] * d
        return {"bytes": float(n * es * (5 + case["res"])), "flops": 20.0 * n}
    V, used = case["V"], int(_used(case).sum())
    if case["kind"] == "embed":
        n = case["B"] * case["T"]
        rows = float((1.0 - (1.0 - _shares(V)) ** used).sum())      # of the table, that are read
        return {"bytes": float((rows * d + n * d + used * d + V * d) * es + 8 * n), "flops": 2.0 * n * d}
    # the logits' product, and one for either gradient; the head read and its gradient written
    products = 3 if case["train"] else 1
    return {"bytes": float((V + used) * d * es * (2 if case["train"] else 1) + 8 * used * case.get("k", 1)),
            "flops": 2.0 * products * used * V * d}


# ------------------------------------------------------------------ 64-bit references
def exact(case, seed):
    if case["kind"] in ("ce", "distill") and float(case["B"] * case["T"]) * case["V"] * case["d"] > MOST_EXACT:
        return None
    st = prepare(case, seed)
    return {"ce": _exact_head, "distill": _exact_head, "norm": _exact_norm, "embed": _exact_embed}[case["kind"]](st)


def _exact_head(st):
    """A block of tokens that count at a time."""
    case = st["case"]
    n, d, V = case["B"] * case["T"], case["d"], case["V"]
    w = st["w"].double()
    out = {"loss": torch.zeros(n, dtype=torch.float64, device="cuda"), "lse": torch.zeros(n, dtype=torch.float64, device="cuda")}
    if case["train"]:
        out["dh"] = torch.zeros(n, d, dtype=torch.float64, device="cuda")
        out["dw"] = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    temp = case.get("temp", 1.0)
    for at in np.array_split(np.flatnonzero(_used(case)), max(1, n * V // 2 ** 28)):
        rows = torch.from_numpy(at).to("cuda")
        h = st["h"][rows].double()
        want = torch.zeros(len(at), V, dtype=torch.float64, device="cuda")
        if case["kind"] == "ce":
            want[torch.arange(len(at), device="cuda"), st["target"][rows].long()] = 1.0
        else:
            idx, logit = st["idx"][rows].long(), st["logit"][rows].double() / temp
            p = torch.softmax(logit.masked_fill(idx < 0, -math.inf), -1)
            want.scatter_add_(1, idx.clamp(min=0), p)
        z = (h @ w.T) / temp
        out["lse"][rows] = torch.logsumexp(z, -1)
        log_q = torch.log_softmax(z, -1)
        out["loss"][rows] = temp * temp * (torch.special.xlogy(want, want) - want * log_q).sum(-1)
        if case["train"]:
            g = (torch.exp(log_q) - want) * (temp * st["g"][rows].double()[:, None])
            out["dh"][rows] = g @ w
            out["dw"] += g.T @ h
    return out


def _exact_norm(st):
    """The gradients by differentiating the normalised rows in 64 bits."""
    rms = st["case"]["rms"]
    d = st["case"]["d"]
    w = st["w"].double()
    y = torch.empty(st["x"].shape, dtype=torch.float64, device="cuda")
    dx, dw, db = torch.empty_like(y), torch.zeros_like(w), torch.zeros_like(w)
    step = max(1, 2 ** 26 // d)
    for i in range(0, y.shape[0], step):
        x = st["x"][i:i + step].double().requires_grad_(True)
        dy = st["dy"][i:i + step].double()
        size = x.square().mean(-1, keepdim=True) if rms else x.var(-1, unbiased=False, keepdim=True)
        xhat = (x if rms else x - x.mean(-1, keepdim=True)) * (size + EPS) ** -0.5
        y[i:i + step] = (xhat * w + (0.0 if rms else st["b"].double())).detach()
        (back,) = torch.autograd.grad(xhat, x, dy * w)
        dx[i:i + step] = back if st["res"] is None else back + st["res"][i:i + step].double()
        dw += (dy * xhat.detach()).sum(0)
        db += dy.sum(0)
    return {"y": y, "dx": dx, "dw": dw, "db": None if rms else db}


def _exact_embed(st):
    V, d = st["table"].shape
    scale, used = st["case"]["scale"], st["ids"] >= 0
    ids = st["ids"][used].long()
    y = torch.zeros(st["dy"].shape, dtype=torch.float64, device="cuda")
    y[used] = st["table"][ids].double() * scale
    grad = torch.zeros(V, d, dtype=torch.float64, device="cuda")
    order = torch.argsort(ids)
    grad.index_add_(0, ids[order], st["dy"][used][order].double() * scale)
    return {"y": y, "dtable": grad}
