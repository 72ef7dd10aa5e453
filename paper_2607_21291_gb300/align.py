"""Feature-preserving alignment of one sparse layer's router (Sec. 3.5), on
synthetic data: the layer-local form of Eq. 9 with the router trained
through the score gate of the gated variant (Sec. 3.4: the router scores
stay on the differentiable path in training). Every step of the method runs in the
library's kernels (the gated and ungated layer forwards, the Eq. 9 value and
gradient, the router's parameter gradient); this module only sequences the
calls and applies the plain SGD update to the router tensors.

The layer input x and the dense layer's output h_dense are held fixed
(teacher forcing from the dense model, as Eq. 9 compares the two models
layer by layer), so the step's gradient is that of the layer's own L_hid.

The two ends of the model train beside it (ends_gradients, ends_step): embedding,
final norm and LM head against the next tokens (the L_causal of Table 4) or a
teacher's top logits, each operator and its gradient a library call.
"""
from __future__ import annotations

from typing import Callable, Optional

import torch

from . import adadsf as A

ROUTER_KEYS = ("router_w1", "router_b1", "router_w2", "router_b2")


def router_alignment_step(shape_cfg: A.ModelCfg, w: dict, x: torch.Tensor, h_dense: torch.Tensor, K: int,
                          lr: float, stream=None, ws: Optional[torch.Tensor] = None):
    """One SGD step on the router of layer weights `w` (device tensors; the
    router tensors are updated in place) against L_hid of Eq. 9 between the
    gated sparse layer's output on x (B, T, d) and h_dense (B, T, d).
    shape_cfg: the layer's config (the gate flag is set here). Returns the
    layer's L_hid before the step (mean over the B T tokens)."""
    with A.in_order(stream):
        return _router_step(shape_cfg, w, x, h_dense, K, lr, stream, ws)


def _router_step(shape_cfg, w, x, h_dense, K, lr, stream, ws):
    B, T, d = x.shape
    cfg_g = A.ModelCfg.from_buffer_copy(shape_cfg)
    cfg_g.flags = int(cfg_g.flags) | A.FLAG_GATE_SIGMOID
    cfg_p = A.ModelCfg.from_buffer_copy(shape_cfg)
    cfg_p.flags = int(cfg_p.flags) & ~A.FLAG_GATE_SIGMOID
    if ws is None:
        ws = A.workspace(A.adadsf_layer_workspace_size(cfg_g, B, T, K), x.device)
    idx = torch.empty((B, K), dtype=torch.int32, device=x.device)
    y_g = x.clone()
    A.adadsf_sparse_layer_forward(cfg_g, w, y_g, K, idx, None, ws, stream)
    y_p = x.clone()
    idx_p = torch.empty_like(idx)
    A.adadsf_sparse_layer_forward(cfg_p, w, y_p, K, idx_p, None, ws, stream)
    acc = torch.zeros(2, dtype=torch.float64, device=x.device)
    grad_y = torch.empty((B * T, d), dtype=torch.float32, device=x.device)
    A.adadsf_align_hidden(y_g, h_dense, acc, grad_y, stream=stream)
    rows = (torch.arange(B, device=x.device, dtype=torch.int32)[:, None] * T + idx).reshape(-1).contiguous()
    g = A.adadsf_router_backward(cfg_g, w, x, y_p, rows, grad_y, stream=stream)
    # the mean over tokens: scale by 1 / (B T); plain SGD on the router tensors
    h = shape_cfg.router_hidden
    scale = lr / float(B * T)
    sizes = {"router_w1": h * d, "router_b1": h, "router_w2": h, "router_b2": 1}
    off = 0
    for k in ROUTER_KEYS:
        n = sizes[k]
        w[k].sub_((g[off:off + n] * scale).view(w[k].shape).to(w[k].dtype))
        off += n
    return float(acc[0] / acc[1])


def ends_gradients(cfg: A.ModelCfg, w: dict, ids: torch.Tensor, target: Optional[torch.Tensor] = None,
                   body: Optional[Callable] = None, top: Optional[tuple] = None, scale: float = 1.0, stream=None):
    """Loss and gradients of the model's two ends: scale * w["embed"][ids]
    (vocab, d; ids below 0 are padding) -> body -> final norm (w["final_w"],
    GPT-NeoX also w["final_b"]) -> LM head w["head"], or w["embed"] where there
    is none -> cross entropy with target (int32 like ids, below 0: none), or the
    distillation loss of top = (indices, logits, temperature) in its place.
    body(x (tokens, d)) returns (y, pull), the layers' output and the function
    from a gradient at y to the one at x; None: no layers. Returns the mean over
    the tokens that have a loss (0-d, on the device) and the gradients by name;
    a shared table's is the sum of both ends' (rounded to its type after either).
    stream: where all of it runs, body and pull as well (torch's current stream
    inside them); the current stream is waited for before, and waits for the
    results."""
    with A.in_order(stream) as read_outside:
        loss, grads = _ends(cfg, w, ids, target, body, top, scale, stream)
        read_outside(loss, *grads.values())
    return loss, grads


def _ends(cfg, w, ids, target, body, top, scale, stream):
    embed = w["embed"]
    head = w.get("head", embed)
    rms = cfg.arch == A.ARCH_QWEN
    n, d = ids.numel(), embed.shape[1]
    dev = embed.device

    def rows():
        return torch.empty(n, dtype=torch.float32, device=dev)

    k = 1 if top is None else top[0].shape[-1]
    ws = A.workspace(max(A.adadsf_head_workspace_size(n, d, head.shape[0], head.dtype, k),
                         A.adadsf_norm_backward_workspace_size(n, d),
                         A.adadsf_embed_backward_workspace_size(n, embed.shape[0], d)), dev)
    x = torch.empty(n, d, dtype=embed.dtype, device=dev)
    A.adadsf_embed_forward(ids, embed, x, scale=scale, ws=ws, stream=stream)
    y, pull = (x, None) if body is None else body(x)
    h, mean, rstd = torch.empty_like(y), None if rms else rows(), rows()
    A.adadsf_norm_forward(y, w["final_w"], w.get("final_b"), h, cfg.norm_eps, mean, rstd, stream=stream)
    loss, lse = rows(), rows()
    acc = torch.zeros(2, dtype=torch.float64, device=dev)
    grads = {"head" if "head" in w else "embed": torch.empty_like(head), "final_w": torch.empty(d, device=dev)}
    if not rms:
        grads["final_b"] = torch.empty(d, device=dev)
    grad_h = torch.empty_like(h)
    if top is None:
        A.adadsf_head_loss(h, head, target, loss, lse, acc=acc, ws=ws, stream=stream)
    else:
        A.adadsf_distill_loss(h, head, top[0], top[1], top[2], loss, lse, acc=acc, ws=ws, stream=stream)
    count = acc[1].clamp(min=1.0)
    share = (1.0 / count).float().expand(n).contiguous()
    grad_head = grads["head" if "head" in w else "embed"]
    if top is None:
        A.adadsf_head_loss_backward(h, head, target, lse, grad_loss=share, grad_h=grad_h, grad_w=grad_head, ws=ws, stream=stream)
    else:
        A.adadsf_distill_loss_backward(h, head, top[0], top[1], lse, top[2], grad_loss=share, grad_h=grad_h,
                                       grad_w=grad_head, ws=ws, stream=stream)
    A.adadsf_norm_backward(grad_h, y, w["final_w"], rstd, grad_h, mean=mean, grad_w=grads["final_w"],
                           grad_b=grads.get("final_b"), ws=ws, stream=stream)
    grad_x = grad_h if pull is None else pull(grad_h)
    tied = "head" not in w
    if not tied:
        grads["embed"] = torch.empty_like(embed)
    A.adadsf_embed_backward(ids, grad_x, grads["embed"], scale=scale, accumulate=tied, ws=ws, stream=stream)
    return acc[0] / count, grads


def ends_step(cfg: A.ModelCfg, w: dict, ids: torch.Tensor, target: Optional[torch.Tensor], lr: float,
              body: Optional[Callable] = None, top: Optional[tuple] = None, scale: float = 1.0, stream=None):
    """One plain SGD step on the tensors of w (in place) by ends_gradients;
    returns the loss before it."""
    with A.in_order(stream) as read_outside:
        loss, grads = _ends(cfg, w, ids, target, body, top, scale, stream)
        for name, g in grads.items():
            w[name].copy_(w[name].float().sub_(g.float(), alpha=lr))
        read_outside(loss)
    return loss
