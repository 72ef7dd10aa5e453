"""Generation for sequences of different lengths from one paged cache.

The depth-sparse model keeps another number of tokens in every layer and sequence, so
each (layer, sequence) has its own pages of one pool, taken as it grows
(adadsf_paged_append / adadsf_paged_attention), in the model's type or as 8-bit numbers
with scales. The rule is that of adadsf_prefill and adadsf_decode_step: a prompt's
Top-K per layer, and a generated token is kept where its score beats the lowest
kept one of its prompt. The next token is drawn by adadsf_sample. Which rows a step
keeps stays on the device: the host learns lengths only when a page may run out.

The library's kernels do the router, Top-K, projections, rotary and cache, attention and
sampling; norms, activations and residuals are plain torch.

    python -m paper_2607_21291_gb300.serve --shape PYTHIA_160M --batch 4 --new 32 --store i8
"""
from __future__ import annotations

from typing import List, Optional, Sequence

import numpy as np
import torch

from . import adadsf as A
from .synth import NEOX


class PagePool:
    """Pages of one pool, handed out to (layer, sequence) pairs."""

    def __init__(self, n_pages: int, page_size: int, n_layers: int, batch: int, max_pages: int):
        self.page_size, self.max_pages = page_size, max_pages
        self.free = list(range(n_pages - 1, -1, -1))
        self.table = np.zeros((n_layers, batch, max_pages), dtype=np.int32)
        self.held = np.zeros((n_layers, batch), dtype=np.int64)   # pages

    def pages(self, tokens: np.ndarray) -> np.ndarray:
        return -(-tokens // self.page_size)

    def reserve(self, tokens: np.ndarray) -> bool:
        """Room for tokens (n_layers, batch); whether the table changed."""
        want = self.pages(tokens)
        if (want > self.max_pages).any():
            raise ValueError(f"{int(tokens.max())} tokens of a sequence exceed {self.max_pages} pages of {self.page_size}")
        need = int(np.maximum(want - self.held, 0).sum())
        if need > len(self.free):
            raise MemoryError(f"{need} pages needed, {len(self.free)} of the pool are free")
        for l, b in zip(*np.nonzero(want > self.held)):
            for i in range(self.held[l, b], want[l, b]):
                self.table[l, b, i] = self.free.pop()
            self.held[l, b] = want[l, b]
        return need > 0

    def release(self, b: int):
        """Gives sequence b's pages back."""
        for l in range(self.table.shape[0]):
            self.free += self.table[l, b, :self.held[l, b]].tolist()
        self.held[:, b] = 0


class Server:
    """B sequences of one model. layers, extra: device tensors as DeviceModel takes
    them (config without flags); head: (vocab, d)."""

    def __init__(self, cfg: A.ModelCfg, layers: Sequence[dict], extra: dict, head: torch.Tensor, batch: int, max_len: int,
                 n_pages: int, page_size: int = 64, store: int = A.KV_SAME):
        if cfg.flags:
            raise ValueError("the paged path takes no flags")
        self.cfg, self.layers, self.extra, self.head, self.B = cfg, list(layers), extra, head, int(batch)
        self.dtype, self.device = A.TORCH_DTYPE[cfg.dtype], head.device
        L = len(self.layers)
        self.cache = A.paged_cache(cfg, n_pages, page_size, store, self.device)
        self.pool = PagePool(n_pages, page_size, L, self.B, -(-int(max_len) // page_size))
        self.tab = A.adadsf_rope_table(cfg, int(max_len), self.device) if cfg.rotary_dim else None
        self.max_len = int(max_len)
        self.ws, self.attn_ws = A.workspace(256, self.device), A.workspace(256, self.device)
        self.table = torch.zeros(self.pool.table.shape, dtype=torch.int32, device=self.device)
        self.lens = torch.zeros(L, self.B, dtype=torch.int32, device=self.device)
        self.thr = torch.full((L, self.B), float("inf"), device=self.device)
        self.pos = torch.zeros(self.B, dtype=torch.int32, device=self.device)
        self.known, self.steps = np.zeros((L, self.B), dtype=np.int64), 0
        self.grows = np.zeros((L, self.B), dtype=bool)            # where a token can be kept at all
        self.length = np.zeros(self.B, dtype=np.int64)            # tokens of a sequence; 0: none, or released
        self.live = torch.zeros(self.B, dtype=torch.int32, device=self.device)

    # ------------------------------------------------------------ one layer's block on packed rows
    def _norm(self, x: torch.Tensor, w: dict, name: str) -> torch.Tensor:
        x, g = x.float(), w[name + "_w"].float()
        if self.cfg.arch == NEOX:
            y = torch.nn.functional.layer_norm(x, x.shape[-1:], g, w[name + "_b"].float(), self.cfg.norm_eps)
        else:
            y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + self.cfg.norm_eps) * g
        return y.to(self.dtype)

    def _linear(self, x, w, bias=None, act=0):
        out = torch.empty(x.shape[0], w.shape[0], dtype=self.dtype, device=self.device)
        A.adadsf_linear(x, w, bias, out, act, ws=self.ws)
        return out

    def _delta(self, x: torch.Tensor, w: dict, batch: A.PagedBatch, pos: torch.Tensor) -> torch.Tensor:
        """fp32 residual delta of rows x, whose keys and values join the cache."""
        n = x.shape[0]
        qkv = self._linear(self._norm(x, w, "ln1"), w["w_qkv"], w["b_qkv"])
        q = torch.empty(n, self.cfg.n_heads * self.cfg.head_dim, dtype=self.dtype, device=self.device)
        out = torch.zeros_like(q)   # rows of no sequence are not written
        A.adadsf_paged_append(self.cfg, self.cache, batch, qkv, self.tab, pos, q, ws=self.ws)
        need = A.adadsf_paged_attention_workspace_size(self.cfg, self.cache, batch)
        if need > self.attn_ws.numel():
            self.attn_ws = A.workspace(need, self.device)
        A.adadsf_paged_attention(self.cfg, self.cache, batch, q, out, ws=self.attn_ws)
        attn = self._linear(out, w["w_o"], w.get("b_o")).float()
        if self.cfg.arch == NEOX:
            up = self._linear(self._norm(x, w, "ln2"), w["w_up"], w["b_up"], act=1)
            return attn + self._linear(up, w["w_down"], w["b_down"]).float()
        m = self._norm(x.float() + attn, w, "ln2")
        act = torch.nn.functional.silu(self._linear(m, w["w_gate"]).float()) * self._linear(m, w["w_up"]).float()
        return attn + self._linear(act.to(self.dtype), w["w_down"]).float()

    def _scores(self, l: int, x: torch.Tensor) -> torch.Tensor:
        scores = torch.empty(x.shape[0], dtype=torch.float32, device=self.device)
        A.adadsf_router_scores(self.cfg, self.layers[l], x, scores, ws=self.ws)
        return scores

    def _reserve(self, tokens: np.ndarray):
        if self.pool.reserve(tokens):
            self.table.copy_(torch.from_numpy(self.pool.table))

    # ------------------------------------------------------------ prompts, single tokens
    def prefill(self, prompts: Sequence[torch.Tensor], ratios: Sequence[float], kept_out: Optional[list] = None) -> torch.Tensor:
        """B prompts of one token or more; layer l keeps floor(ratios[l] T + 1e-9) tokens
        of one of T, at most all. The final hidden states of the prompts' last tokens. kept_out: gets a
        list of the sequences' kept positions a layer."""
        T = np.array([len(p) for p in prompts])
        if len(T) != self.B or T.min() < 1 or T.max() > self.max_len:
            raise ValueError(f"need {self.B} prompts of 1 to {self.max_len} tokens")
        ratios = np.asarray(ratios, dtype=np.float64)
        if ratios.shape != (len(self.layers),) or not np.isfinite(ratios).all():
            raise ValueError(f"need a finite ratio for each of {len(self.layers)} layers")
        at = np.concatenate([[0], np.cumsum(T)])
        ids = torch.cat([torch.as_tensor(p) for p in prompts]).to(self.device)
        pos = torch.cat([torch.arange(n, dtype=torch.int32, device=self.device) for n in T])
        # as the retention allocation counts them (adadsf_alloc_ratios): 0.29 x 100 falls short of 29 by a rounding
        K = np.clip(np.floor(np.multiply.outer(ratios, T) + 1e-9), 0, T).astype(np.int64)
        self._reserve(K)
        self.known, self.steps, self.grows, self.length = K, 0, K > 0, T.astype(np.int64)
        self.live.fill_(1)
        self.lens.copy_(torch.from_numpy(K.astype(np.int32)))
        self.thr.fill_(float("inf"))
        self.pos.copy_(torch.from_numpy(T.astype(np.int32)))
        starts = torch.from_numpy(np.concatenate([np.zeros((len(K), 1)), np.cumsum(K, 1)], 1).astype(np.int32)).to(self.device)
        x = self.extra["embed"][ids.long()]
        for l, w in enumerate(self.layers):
            scores, kept = self._scores(l, x), []
            for b in range(self.B):
                idx = torch.empty(1, K[l, b], dtype=torch.int32, device=self.device)
                kept.append(idx[0])
                if K[l, b]:
                    A.adadsf_topk_select(scores[at[b]:at[b + 1]].clone()[None], K[l, b], idx)   # a copy is aligned
                    self.thr[l, b] = scores[idx[0].long() + at[b]].min()
            if kept_out is not None:
                kept_out.append(kept)
            rows = torch.cat([idx.long() + at[b] for b, idx in enumerate(kept)])
            if len(rows):
                batch = A.PagedBatch(starts[l], self.lens[l], self.table[l], len(rows), int(K[l].max()))
                xr = x[rows]
                x[rows] = (xr.float() + self._delta(xr, w, batch, pos[rows])).to(self.dtype)
        return self._norm(x[torch.from_numpy(at[1:] - 1).to(self.device)], self.extra, "final")

    def step(self, tokens: torch.Tensor, kept_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """One token of every sequence (B,): their final hidden states. kept_out:
        (n_layers, B) bool. A released sequence's token is of no effect."""
        if self.length.max(initial=0) >= self.max_len:
            raise ValueError(f"a sequence is longer than {self.max_len}")
        if (self.pool.pages(np.where(self.grows, self.known + self.steps + 1, 0)) > self.pool.held).any():
            self.known, self.steps = self.lens.cpu().numpy().astype(np.int64), 0   # a page may run out: look
            self._reserve(np.where(self.grows, self.known + 1, 0))
        self.steps += 1
        self.length += self.length > 0
        x = self.extra["embed"][tokens.long()]
        for l, w in enumerate(self.layers):
            keep = self._scores(l, x) > self.thr[l]
            rows = torch.argsort(keep.logical_not().to(torch.int8), stable=True)   # kept ones first, in order
            starts = torch.nn.functional.pad(keep.cumsum(0, dtype=torch.int32), (1, 0))
            self.lens[l] += keep
            batch = A.PagedBatch(starts, self.lens[l], self.table[l], self.B, 1)
            xr = x[rows]
            delta = torch.where(keep[rows][:, None], self._delta(xr, w, batch, self.pos[rows]), 0.0)
            x[rows] = (xr.float() + delta).to(self.dtype)
            if kept_out is not None:
                kept_out[l] = keep
        self.pos += self.live
        return self._norm(x, self.extra, "final")

    def sample(self, hidden: torch.Tensor, u: torch.Tensor, logprob: Optional[torch.Tensor] = None, **settings) -> torch.Tensor:
        """The next token of each row of hidden states; settings as adadsf_sample takes them."""
        token = torch.empty(hidden.shape[0], dtype=torch.int32, device=self.device)
        A.adadsf_sample(self._linear(hidden, self.head), u, token, logprob=logprob, **settings)
        return token

    def generate(self, prompts: Sequence[torch.Tensor], ratios: Sequence[float], n_new: int, u: torch.Tensor, **settings):
        """(tokens, log-probabilities), (n_new, B) each, from random numbers u (n_new, B)."""
        logprob = torch.empty(n_new, self.B, dtype=torch.float32, device=self.device)
        hidden, tokens = self.prefill(prompts, ratios), []
        for i in range(n_new):
            tokens.append(self.sample(hidden, u[i], logprob[i], **settings))
            if i + 1 < n_new:
                hidden = self.step(tokens[-1])
        self.check()
        return torch.stack(tokens), logprob

    # ------------------------------------------------------------ what a sequence holds
    def cached(self, l: int) -> List[tuple]:
        """Layer l's cached keys (turned) and values of every sequence, as rows (n, kv):
        what moving a sequence elsewhere takes along."""
        n = self.lens[l].cpu().numpy()
        kv = self.cfg.n_kv_heads * self.cfg.head_dim
        starts = torch.from_numpy(np.concatenate([[0], np.cumsum(n)]).astype(np.int32)).to(self.device)
        out = [torch.empty(int(n.sum()), kv, dtype=self.dtype, device=self.device) for _ in range(2)]
        A.adadsf_paged_read(self.cfg, self.cache, A.PagedBatch(starts, self.lens[l], self.table[l], int(n.sum()), max(1, int(n.max()))),
                            *out, ws=self.ws)
        return list(zip(*[t.split(n.tolist()) for t in out]))

    def release(self, b: int):
        """Gives sequence b's pages back to the pool; it takes none again before the next prompts."""
        self.pool.release(b)
        self.lens[:, b] = 0
        self.thr[:, b] = float("inf")
        self.pos[b] = 0
        self.live[b] = 0
        self.known[:, b], self.grows[:, b], self.length[b] = 0, False, 0

    def check(self):
        for ws in (self.ws, self.attn_ws):
            A._check(A.adadsf_sync_check(ws))


def main():
    import argparse
    import time

    from . import synth as S
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--shape", default="PYTHIA_160M", help="a backbone shape of synth.py")
    ap.add_argument("--batch", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=512, help="longest prompt; the others are shorter")
    ap.add_argument("--new", type=int, default=64)
    ap.add_argument("--ratio", type=float, default=0.5, help="kept share of every layer")
    ap.add_argument("--page", type=int, default=64)
    ap.add_argument("--store", choices=("same", "i8"), default="i8")
    ap.add_argument("--top-p", type=float, default=0.9)
    a = ap.parse_args()
    shape = getattr(S, a.shape)
    td = torch.bfloat16 if shape.dtype == "bf16" else torch.float32
    put = lambda d: {k: v.to("cuda", td) for k, v in d.items()}   # noqa: E731
    layers = [put(S.bench_layer_weights(shape, 1, l, "cuda")) for l in range(shape.n_layers)]
    extra = A.to_device(S.model_extra_weights(shape, 1), td)
    max_len = a.prompt + a.new
    pages = shape.n_layers * a.batch * (-(-max_len // a.page) + 1)
    srv = Server(A.make_cfg(shape), layers, extra, extra["embed"], a.batch, max_len, pages, a.page,
                 A.KV_I8 if a.store == "i8" else A.KV_SAME)
    rng = np.random.default_rng(2)
    prompts = [torch.from_numpy(rng.integers(0, shape.vocab, max(1, a.prompt - 37 * b))) for b in range(a.batch)]
    u = torch.from_numpy(rng.random((a.new, a.batch), dtype=np.float32)).cuda()
    top_p = torch.full((a.batch,), a.top_p, device="cuda")
    for turn in ("first", "again"):
        t0 = time.perf_counter()
        tokens, logprob = srv.generate(prompts, [a.ratio] * shape.n_layers, a.new, u, top_p=top_p)
        dt = time.perf_counter() - t0
        held = int(srv.pool.held.sum())
        kept = srv.lens.float().mean().item()
        print(f"{turn}: {a.batch} x {a.new} tokens in {dt * 1e3:.1f} ms; a layer holds {kept:.0f} tokens a sequence, "
              f"{held} pages of {a.page} in all")
        for b in range(a.batch):
            srv.release(b)
    print("tokens of sequence 0:", tokens[:12, 0].tolist())


if __name__ == "__main__":
    main()
