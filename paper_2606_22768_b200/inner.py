"""Inner steps of the K workers on one GPU: a small Llama-style decoder whose parameters are rows of the flat [K, ld] matrix that
the outer round works on.

The decoder block runs on the library's operators -- packed causal attention, the fused block norm, and activations kept in 8 bits
for the backward pass -- as autograd functions; matrix products are plain library products, batched over the workers.  All K
workers take their step in one pass: activations are [K * rows, width] with worker m's rows at [m * rows, (m + 1) * rows).

What a block keeps for its backward pass: the residual stream and the block outputs (the norms need them), q, k, v, o and lse, and in
8 bits the inputs of its projections and of SwiGLU (whose output, the last projection's input, comes from there again).  The backward passes are not differentiable themselves: create_graph=True is an error
in them.
"""
from __future__ import annotations

import functools
from dataclasses import dataclass
from typing import Dict, Optional, Tuple

import torch

from . import (ACT8_GROUP, AttnPlan, fgd_act_load8, fgd_act_save8, fgd_attn_backward, fgd_attn_forward, fgd_attn_status, fgd_block_norm_backward, fgd_block_norm_forward,
               fgd_swiglu8_backward, fgd_swiglu8_forward)


# ------------------------------------------------------------------------------- operators
def _first_order(backward):
    """A backward pass whose results carry no graph.  Where one is asked for they would count as constants, and a second derivative would
    silently lack their terms: refused here, since a refusal that waits for the second pass is not reached by every way to start it."""
    @functools.wraps(backward)
    def checked(ctx, *grads):
        if torch.is_grad_enabled():      # in a backward pass: create_graph=True
            raise RuntimeError("the inner step's operators are not differentiable twice: their backward passes do not run with create_graph=True")
        return backward(ctx, *grads)
    return checked


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, plan, scale):
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
        fgd_attn_forward(plan, q, k, v, o, lse, scale)
        ctx.save_for_backward(q, k, v, o, lse)
        ctx.plan, ctx.scale = plan, scale
        return o

    @staticmethod
    @_first_order
    def backward(ctx, do):
        q, k, v, o, lse = ctx.saved_tensors
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        fgd_attn_backward(ctx.plan, q, k, v, o, do.contiguous(), lse, torch.empty_like(lse), dq, dk, dv, ctx.scale)
        return dq, dk, dv, None, None


def attention(q, k, v, plan: AttnPlan, scale: Optional[float] = None):
    """Causal attention over the plan's packed sequences: q [T, Hq, d], k and v [T, Hk, d] -> [T, Hq, d]."""
    return _Attention.apply(q, k, v, plan, scale)


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, y, gate, w_post, w_pre, eps, res_scale):
        x_new = x if y is None else torch.empty_like(x)
        n = torch.empty_like(x)
        fgd_block_norm_forward(x, y, gate, w_post, w_pre, x_new, n, eps, res_scale)
        ctx.save_for_backward(x_new, y, gate, w_post, w_pre)
        ctx.eps, ctx.res_scale = eps, res_scale
        return (x.view_as(x) if y is None else x_new), n

    @staticmethod
    @_first_order
    def backward(ctx, dres, dn):
        x_new, y, gate, w_post, w_pre = ctx.saved_tensors
        like = lambda t: None if t is None else torch.empty(t.shape, dtype=t.dtype, device=t.device)  # noqa: E731
        dx, dy, dgate, dw_post, dw_pre = like(x_new), like(y), like(gate), like(w_post), like(w_pre)
        fgd_block_norm_backward(dn.contiguous(), None if dres is None else dres.contiguous(), x_new, y, gate, w_post, w_pre, dx, dy, dgate, dw_post, dw_pre,
                                ctx.eps, ctx.res_scale)
        return dx, dy, dgate, dw_post, dw_pre, None, None


def block_norm(x, y, gate, w_post, w_pre, eps: float = 1e-5, res_scale: float = 1.0):
    """(x_new, n): the block output y normalised, gated, scaled and added to the stream x, and the norm of the result.  Without y: (x, norm of x)."""
    return _BlockNorm.apply(x, y, gate, w_post, w_pre, eps, res_scale)


class _Swiglu8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gu):
        rows, width = gu.shape[0], gu.shape[1] // 2
        h = torch.empty((rows, width), dtype=gu.dtype, device=gu.device)
        q8 = torch.empty((rows, 2 * width), dtype=torch.int8, device=gu.device)
        e8 = torch.empty((rows, 2 * -(-width // ACT8_GROUP)), dtype=torch.uint8, device=gu.device)
        fgd_swiglu8_forward(gu, h, q8, e8)
        ctx.save_for_backward(q8, e8)
        return h

    @staticmethod
    @_first_order
    def backward(ctx, dh):
        q8, e8 = ctx.saved_tensors
        dgu = torch.empty(q8.shape, dtype=dh.dtype, device=dh.device)
        fgd_swiglu8_backward(dh.contiguous(), q8, e8, dgu)
        return dgu


def swiglu8(gu):
    """silu(g) * u of gu = [g | u], keeping g and u in 8 bits."""
    return _Swiglu8.apply(gu)


class _Linear8(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        K = w.shape[0]
        q8 = torch.empty(x.shape, dtype=torch.int8, device=x.device)
        e8 = torch.empty((x.shape[0], -(-x.shape[1] // ACT8_GROUP)), dtype=torch.uint8, device=x.device)
        fgd_act_save8(x, q8, e8)
        ctx.save_for_backward(q8, e8, w)
        return torch.bmm(x.view(K, -1, x.shape[1]), w.transpose(1, 2)).view(x.shape[0], w.shape[1])

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        q8, e8, w = ctx.saved_tensors
        K = w.shape[0]
        x = torch.empty(q8.shape, dtype=dy.dtype, device=dy.device)
        fgd_act_load8(q8, e8, x)
        dy = dy.contiguous().view(K, -1, w.shape[1])
        return torch.bmm(dy, w).view(x.shape), torch.bmm(dy.transpose(1, 2), x.view(K, -1, x.shape[1]))


def linear8(x, w):
    """Per worker x w^T: x [K * rows, in], w [K, out, in]; keeps x in 8 bits for the gradient of w."""
    return _Linear8.apply(x, w)


class _Swiglu8Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gu, w):
        K, rows, width = w.shape[0], gu.shape[0], gu.shape[1] // 2
        h = torch.empty((rows, width), dtype=gu.dtype, device=gu.device)
        q8 = torch.empty((rows, 2 * width), dtype=torch.int8, device=gu.device)
        e8 = torch.empty((rows, 2 * -(-width // ACT8_GROUP)), dtype=torch.uint8, device=gu.device)
        fgd_swiglu8_forward(gu, h, q8, e8)
        ctx.save_for_backward(q8, e8, w)
        return torch.bmm(h.view(K, -1, width), w.transpose(1, 2)).view(rows, w.shape[1])

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        q8, e8, w = ctx.saved_tensors
        K, rows, width = w.shape[0], q8.shape[0], w.shape[2]
        dy = dy.contiguous().view(K, -1, w.shape[1])
        dgu, h = torch.empty(q8.shape, dtype=dy.dtype, device=dy.device), torch.empty((rows, width), dtype=dy.dtype, device=dy.device)
        fgd_swiglu8_backward(torch.bmm(dy, w).view(rows, width), q8, e8, dgu, h)
        return dgu, torch.bmm(dy.transpose(1, 2), h.view(K, -1, width))


def swiglu8_linear(gu, w):
    """Per worker (silu(g) * u) w^T of gu = [g | u]: gu [K * rows, 2 in], w [K, out, in]; keeps g and u in 8 bits and nothing else: the gradient
    of w takes the product that the backward pass forms again from them."""
    return _Swiglu8Linear.apply(gu, w)


# ------------------------------------------------------------------------------- decoder
@dataclass(frozen=True)
class DecoderConfig:
    vocab: int = 256
    width: int = 256
    layers: int = 2
    n_q_heads: int = 4
    n_kv_heads: int = 2
    head_dim: int = 64
    ffn: int = 512
    eps: float = 1e-5
    rope_base: float = 10000.0

    @property
    def res_scale(self) -> float:
        """Scale of every block's addition to the stream: 1 / sqrt(2 layers)."""
        return (2 * self.layers) ** -0.5


def param_layout(cfg: DecoderConfig) -> Tuple[Dict[str, Tuple[int, Tuple[int, ...]]], int]:
    """{name: (first column, shape)} of one worker's row, and the number of columns.  Every tensor starts on a multiple of 32 columns."""
    layout, at = {}, 0

    def add(name, *shape):
        nonlocal at
        layout[name] = (at, shape)
        n = 1
        for s in shape:
            n *= s
        at += -(-n // 32) * 32

    qkv = (cfg.n_q_heads + 2 * cfg.n_kv_heads) * cfg.head_dim
    add("embed", cfg.vocab, cfg.width)
    for i in range(cfg.layers):
        for block in ("attn", "mlp"):
            for name in ("pre", "post", "gate"):
                add(f"{i}.{block}.{name}", cfg.width)
        add(f"{i}.qkv", qkv, cfg.width)
        add(f"{i}.out", cfg.width, cfg.n_q_heads * cfg.head_dim)
        add(f"{i}.up", 2 * cfg.ffn, cfg.width)
        add(f"{i}.down", cfg.width, cfg.ffn)
    add("final", cfg.width)
    add("head", cfg.vocab, cfg.width)
    return layout, at


def init_params(theta: torch.Tensor, cfg: DecoderConfig, seed: int = 0) -> None:
    """Fills theta [K, ld] with one draw shared by all rows (workers start identical)."""
    layout, P = param_layout(cfg)
    gen = torch.Generator().manual_seed(seed)
    row = torch.zeros(theta.shape[1])
    for name, (at, shape) in layout.items():
        n = 1
        for s in shape:
            n *= s
        if len(shape) == 1:
            row[at:at + n] = 1.0
        else:
            row[at:at + n] = torch.randn(n, generator=gen) * (0.02 if name in ("embed", "head") else shape[1] ** -0.5)
    theta.copy_(row.to(theta.device).expand_as(theta))


def _rope(cfg: DecoderConfig, positions):
    freq = cfg.rope_base ** (-torch.arange(0, cfg.head_dim, 2, device=positions.device, dtype=torch.float32) / cfg.head_dim)
    angle = positions[:, None].float() * freq
    return angle.cos()[:, None], angle.sin()[:, None]


def _rotate(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat((a * cos - b * sin, b * cos + a * sin), -1).to(x.dtype)


def decoder_logits(theta: torch.Tensor, tokens: torch.Tensor, plan: AttnPlan, positions: torch.Tensor, cfg: DecoderConfig,
                   dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """Logits [K, rows, vocab] of the K workers.  theta [K, ld] fp32 (may require gradients), tokens [K, rows], positions [K * rows] of
    every token in its sequence; the plan covers all K * rows tokens, worker after worker."""
    layout, _ = param_layout(cfg)
    K, rows = tokens.shape
    T, hq, hk, d = K * rows, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim

    def vec(name):      # per-channel values, read where they lie in the matrix
        at, (n,) = layout[name]
        return theta[:, at:at + n]

    def mat(name):
        at, (o, i) = layout[name]
        return theta[:, at:at + o * i].to(dtype).view(K, o, i)

    cos, sin = _rope(cfg, positions)
    embed = mat("embed")
    x = torch.gather(embed, 1, tokens[:, :, None].expand(-1, -1, cfg.width)).reshape(T, cfg.width)
    x, n = block_norm(x, None, None, None, vec("0.attn.pre"), cfg.eps)
    for i in range(cfg.layers):
        qkv = linear8(n, mat(f"{i}.qkv")).view(T, hq + 2 * hk, d)
        q, k = _rotate(qkv[:, :hq], cos, sin), _rotate(qkv[:, hq:hq + hk], cos, sin)
        o = attention(q, k, qkv[:, hq + hk:], plan)
        y = linear8(o.view(T, hq * d), mat(f"{i}.out"))
        x, n = block_norm(x, y, vec(f"{i}.attn.gate"), vec(f"{i}.attn.post"), vec(f"{i}.mlp.pre"), cfg.eps, cfg.res_scale)
        y = swiglu8_linear(linear8(n, mat(f"{i}.up")), mat(f"{i}.down"))
        after = vec(f"{i + 1}.attn.pre") if i + 1 < cfg.layers else vec("final")
        x, n = block_norm(x, y, vec(f"{i}.mlp.gate"), vec(f"{i}.mlp.post"), after, cfg.eps, cfg.res_scale)
    return linear8(n, mat("head")).view(K, rows, cfg.vocab)


def worker_losses(logits: torch.Tensor, targets: torch.Tensor) -> torch.Tensor:
    """Mean cross entropy of every worker, [K]; targets [K, rows], negative = not counted."""
    lp = torch.log_softmax(logits.float(), -1)
    counted = targets >= 0
    picked = torch.gather(lp, 2, targets.clamp_min(0)[:, :, None])[:, :, 0]
    return -(picked * counted).sum(1) / counted.sum(1).clamp_min(1)


class InnerSteps:
    """H local AdamW steps of all K workers on theta [K, ld] (each worker's own gradient, its own moments)."""

    def __init__(self, theta: torch.Tensor, cfg: DecoderConfig, lr: float = 1e-3, betas=(0.9, 0.95), eps: float = 1e-8, weight_decay: float = 0.0):
        self.theta, self.cfg, self.lr, self.betas, self.eps, self.weight_decay = theta, cfg, lr, betas, eps, weight_decay
        self.m, self.v, self.t = torch.zeros_like(theta), torch.zeros_like(theta), 0

    def step(self, tokens, targets, plan: AttnPlan, positions) -> torch.Tensor:
        """One step on a batch; returns the workers' losses before it.  Raises FgdError, with parameters and moments as they were, if a
        device-side wait of the attention kernels gave up (it waits for the gradients to know)."""
        leaf = self.theta.detach().requires_grad_(True)
        losses = worker_losses(decoder_logits(leaf, tokens, plan, positions, self.cfg), targets)
        losses.sum().backward()      # (the workers share no parameter: every row gets its own worker's gradient)
        fgd_attn_status(plan)
        with torch.no_grad():
            self.t += 1
            b1, b2 = self.betas
            self.m.lerp_(leaf.grad, 1 - b1)
            self.v.mul_(b2).addcmul_(leaf.grad, leaf.grad, value=1 - b2)
            update = (self.m / (1 - b1 ** self.t)) / ((self.v / (1 - b2 ** self.t)).sqrt() + self.eps)
            self.theta.mul_(1 - self.lr * self.weight_decay).sub_(update, alpha=self.lr)
        return losses.detach()
