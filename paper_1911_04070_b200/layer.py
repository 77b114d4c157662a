"""BP-Transformer layers on top of the graph self-attention library (arXiv 1911.04070, Sec. 3.3,
Algorithm 2): PyTorch modules whose attention runs in libbpt.so.

The graph self-attention, the gated feed-forward block and the seam between two blocks (norms, gate, residual) are this
package's own operators; the projections, and in the paper's form of the layer the feed-forward block and the norms, are plain
PyTorch operators around them, so that each can be dropped into a model and trained.  Nothing here falls back to another
implementation of an operator: a gated block in float32 is written out in PyTorch operators.
"""
from __future__ import annotations

import math

import torch
from torch import nn
from torch.autograd import forward_ad
from torch.autograd.function import once_differentiable

from . import binding


# Inference (no gradient, bfloat16, model width 128 / 256 / 512): the output projection, the residual and the first
# layer normalisation of a layer run in the library's fused kernel (bpt_out_proj_norm) instead of three operators.
FUSE_OUT_PROJ_NORM = True


class _GraphSelfAttention(torch.autograd.Function):
    """out = GSA(q, k, v, rel_emb) over the BPT graph; backward through bpt_attn_bwd."""

    @staticmethod
    def forward(ctx, q, k, v, rel_emb, g, scale, lengths, dropout_p, dropout_seed):
        q, k, v, rel_emb = q.contiguous(), k.contiguous(), v.contiguous(), rel_emb.contiguous()
        out, lse = binding.bpt_attn_fwd(g, q, k, v, rel_emb, scale, lengths=lengths, dropout_p=dropout_p,
                                        dropout_seed=dropout_seed)
        if binding.CHECK_DEVICE_STATUS and binding.bpt_check(getattr(out, "_bpt_workspace", None)):
            raise RuntimeError("graph self-attention forward: a device-side wait timed out, results are invalid")
        ctx.save_for_backward(q, k, v, rel_emb, out, lse)
        ctx.g, ctx.scale, ctx.lengths, ctx.drop = g, scale, lengths, (dropout_p, dropout_seed)
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, rel_emb, out, lse = ctx.saved_tensors
        dq, dk, dv, d_rel = binding.bpt_attn_bwd(ctx.g, q, k, v, rel_emb, ctx.scale, out, lse, d_out.contiguous(),
                                                 lengths=ctx.lengths, dropout_p=ctx.drop[0], dropout_seed=ctx.drop[1])
        if binding.CHECK_DEVICE_STATUS and binding.bpt_check(getattr(dq, "_bpt_workspace", None)):
            raise RuntimeError("graph self-attention backward: a device-side wait timed out, results are invalid")
        return dq, dk, dv, d_rel.to(rel_emb.dtype), None, None, None, None, None


def graph_self_attention(g: binding.Graph, q, k, v, rel_emb, scale=None, lengths=None, dropout_p=0.0, dropout_seed=0):
    """Differentiable graph self-attention with tree relative positions (Sec. 3.1, 3.4).

    q, k, v: [B, 2n-1, H, d] (float32 or bfloat16, on the graph's device); rel_emb: [n_rel, d], shared
    by the heads; lengths: optional int32 [B]; dropout_p / dropout_seed: attention dropout (the mask is a
    function of the seed, so the backward pass rebuilds it).  Returns [B, 2n-1, H, d]."""
    scale = 1.0 / math.sqrt(q.shape[-1]) if scale is None else float(scale)
    return _GraphSelfAttention.apply(q, k, v, rel_emb, g, scale, lengths, float(dropout_p), int(dropout_seed))


def _check_constant(name, v):
    """alpha and eps are numbers; a tensor would be read as one, and its gradient or tangent lost."""
    if isinstance(v, torch.Tensor) and ((v.requires_grad and torch.is_grad_enabled()) or forward_ad.unpack_dual(v).tangent is not None):
        raise NotImplementedError("residual_norm has no derivative with respect to %s; a learned factor goes into gate or h" % name)


def residual_norm(h, b=None, weight=None, bias=None, norm="layer", post_norm=None, post_weight=None, post_bias=None, gate=None,
                  alpha=1.0, eps=1e-5, return_sum=False):
    """The seam between two blocks, differentiable:  r = alpha * h + gate * post_norm(b),  y = norm(r)  over the last axis.

    h: the residual stream [..., D], b: the output of the block before (None: r = alpha * h), both float32 or bfloat16.
    norm / post_norm: "layer", "rms" or None, with their weights and biases [D] (None: 1 and 0).  gate: [D], or h's shape
    with the trailing row axes of length one ([B, 1, D]: a gate per sequence), or None (1).  alpha, eps: numbers.  With norm="layer" and nothing
    else this is the norm(H + A) of Algorithm 2; with post_norm it is the norm after the block before and the norm
    before the block that follows.  Returns y; (r, y) with return_sum; r with norm=None.  Can be captured in a CUDA graph with
    its backward pass, which is refused there while a graph of the same leaves made on the default stream is alive.  Reverse mode,
    first order; forward-mode tangents and torch.jit.trace are refused."""
    if type(alpha) is not float or type(eps) is not float:
        _check_constant("alpha", alpha)
        _check_constant("eps", eps)
    kind, post = binding.NORM_KINDS.get(norm), binding.NORM_KINDS.get(post_norm)
    if kind is not None and post is not None:
        out = binding.load_native().residual_norm(h, b, weight, bias, post_weight, post_bias, gate, kind, post, alpha, eps, return_sum)
        if out is not None:
            return out
    cont = lambda t: t if t is None else t.contiguous()
    binding.bpt_res_norm_fwd(*map(cont, (h, b, weight, bias)), norm, post_norm, *map(cont, (post_weight, post_bias, gate)), alpha, eps,
                             return_sum)                                                            # says what is wrong
    raise RuntimeError("residual_norm: refused")


def _aligned(t):
    """Contiguous and on the 16-byte boundary that the feed-forward kernels need; a contiguous view may start anywhere."""
    t = t.contiguous()
    return t.clone() if t.data_ptr() % 16 else t


class _GatedFeedForward(torch.autograd.Function):
    """The same function as the native one, which looks at the device status after every call (binding.CHECK_DEVICE_STATUS)."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act):
        y = binding.bpt_gated_ff_fwd(x, w_gate, w_up, w_down, act)
        if binding.CHECK_DEVICE_STATUS and binding.bpt_check(y._bpt_workspace):
            raise RuntimeError("gated feed-forward: a device-side wait timed out, results are invalid")
        ctx.save_for_backward(x, w_gate, w_up, w_down)
        ctx.act = act
        return y

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        if forward_ad.unpack_dual(dy).tangent is not None:
            raise NotImplementedError("gated_feed_forward backward has no forward-mode derivative")
        x, w_gate, w_up, w_down = map(_aligned, ctx.saved_tensors)
        need = ctx.needs_input_grad
        grads = binding.bpt_gated_ff_bwd(x, w_gate, w_up, w_down, _aligned(dy), ctx.act, need_dx=need[0], need_dw=any(need[1:4]))
        first = grads[0] if need[0] else grads[1]
        if binding.CHECK_DEVICE_STATUS and binding.bpt_check(first._bpt_workspace):
            raise RuntimeError("gated feed-forward backward: a device-side wait timed out, results are invalid")
        return tuple(g if n else None for g, n in zip(grads, need)) + (None,)


def gated_feed_forward(x, w_gate, w_up, w_down, act="silu"):
    """Differentiable gated feed-forward block over the last axis:  (act(x w_gate^T) * (x w_up^T)) w_down^T.

    x: [..., D] bfloat16; w_gate, w_up: [F, D], w_down: [D, F] (the layout of a linear layer's weight), D and F multiples
    of 8; act: "silu", "gelu" (with erf) or "relu".  Any strides and offsets: what is not contiguous or does not start on a
    16-byte boundary is copied first.  Nothing but x and the weights is kept for the backward pass.  A device-side wait that
    expired, in either pass, shows in binding.bpt_check_device.  Capture, modes of
    differentiation and tracing as in residual_norm."""
    if binding.CHECK_DEVICE_STATUS:
        if torch.jit.is_tracing():
            raise NotImplementedError("gated_feed_forward cannot be traced by torch.jit")
        return _GatedFeedForward.apply(*map(_aligned, (x, w_gate, w_up, w_down)), act)
    code = binding.ACTIVATIONS.get(act)
    out = None if code is None else binding.load_native().gated_feed_forward(x, w_gate, w_up, w_down, code)
    if out is None:
        binding.bpt_gated_ff_fwd(*map(_aligned, (x, w_gate, w_up, w_down)), act)      # says what is wrong
        raise RuntimeError("gated_feed_forward: refused")
    y, y._bpt_workspace = out
    return y


class BPTLayer(nn.Module):
    """One layer of Algorithm 2:  Z = norm(H + GSA(H)),  H' = norm(Z + FFN(Z)).

    H holds the states of all 2n-1 nodes.  The relation embeddings are a parameter of the layer
    (Sec. 3.4: not shared between layers, shared between the heads).

    Two forms beyond the paper's, for deeper stacks and language models:
    gated: "silu", "gelu" or "relu" makes the FFN the gated block (act(Z Wg^T) * (Z Wu^T)) Wd^T (d_model and d_ff multiples of
    8; in bfloat16 it runs in gated_feed_forward).
    sandwich: norms before and after each block, with a learned gate per channel and the residual scaled by alpha:
    R = alpha H + gate1 * norm1(GSA(pre1(H))),  H' = alpha R + gate2 * norm2(FFN(pre2(R))); everything between two blocks
    is one residual_norm call."""

    def __init__(self, g: binding.Graph, d_model: int, n_heads: int, d_ff: int, rel_std: float = 0.02,
                 attn_dropout: float = 0.0, gated=None, sandwich: bool = False, alpha: float = 1.0):
        super().__init__()
        self.attn_dropout = attn_dropout
        if d_model % n_heads:
            raise ValueError("d_model must be a multiple of n_heads")
        if gated is not None and gated not in binding.ACTIVATIONS:
            raise ValueError("gated must be None or one of %s" % ", ".join(map(repr, binding.ACTIVATIONS)))
        if gated is not None and (d_model % 8 or d_ff % 8):
            raise ValueError("a gated layer needs d_model and d_ff that are multiples of 8")
        if alpha != 1.0 and not sandwich:
            raise ValueError("alpha scales the residual of the sandwich form")
        self.g, self.h, self.dh = g, n_heads, d_model // n_heads
        self.gated, self.sandwich, self.alpha = gated, sandwich, float(alpha)
        self.wq, self.wk, self.wv, self.wo = (nn.Linear(d_model, d_model, bias=False) for _ in range(4))
        self.rel_emb = nn.Parameter(torch.randn(g.n_rel, self.dh) * rel_std)
        self.norm1, self.norm2 = nn.LayerNorm(d_model), nn.LayerNorm(d_model)
        if gated is None:
            self.ff1, self.ff2 = nn.Linear(d_model, d_ff), nn.Linear(d_ff, d_model)
        else:
            self.ff_gate, self.ff_up = nn.Linear(d_model, d_ff, bias=False), nn.Linear(d_model, d_ff, bias=False)
            self.ff_down = nn.Linear(d_ff, d_model, bias=False)
        if sandwich:
            self.pre1, self.pre2 = nn.LayerNorm(d_model), nn.LayerNorm(d_model)
            self.gate1, self.gate2 = nn.Parameter(torch.ones(d_model)), nn.Parameter(torch.ones(d_model))

    def feed_forward(self, z):
        if self.gated is None:
            return self.ff2(torch.relu(self.ff1(z)))
        if z.dtype == torch.bfloat16 and self.ff_gate.weight.dtype == torch.bfloat16:
            return gated_feed_forward(z, self.ff_gate.weight, self.ff_up.weight, self.ff_down.weight, self.gated)
        return self.ff_down(getattr(torch.nn.functional, self.gated)(self.ff_gate(z)) * self.ff_up(z))

    def attention_input(self, h):
        """What the attention's projections take: H, or pre1(H) in the sandwich form."""
        return residual_norm(h, None, self.pre1.weight, self.pre1.bias, eps=self.pre1.eps) if self.sandwich else h

    def after_attention(self, h, a, next_norm=None, fuse: bool = True):
        """H' from the layer's input H and the attention's output a, both [..., d_model]; with next_norm (a LayerNorm, sandwich
        form) the pair (H', next_norm(H')).  fuse: the output projection may run in bpt_out_proj_norm."""
        if self.sandwich:
            n1, n2, p2 = self.norm1, self.norm2, self.pre2
            r, y = residual_norm(h, self.wo(a), p2.weight, p2.bias, "layer", "layer", n1.weight, n1.bias, self.gate1, self.alpha, n1.eps, True)
            f = self.feed_forward(y)
            if next_norm is None:
                return residual_norm(r, f, norm=None, post_norm="layer", post_weight=n2.weight, post_bias=n2.bias, gate=self.gate2,
                                     alpha=self.alpha, eps=n2.eps)
            return residual_norm(r, f, next_norm.weight, next_norm.bias, "layer", "layer", n2.weight, n2.bias, self.gate2, self.alpha, n2.eps, True)
        D = h.shape[-1]
        if (fuse and FUSE_OUT_PROJ_NORM and not torch.is_grad_enabled() and h.dtype == torch.bfloat16 and D in (128, 256, 512)
                and self.wo.weight.dtype == torch.bfloat16):
            z = binding.bpt_out_proj_norm(a, self.wo.weight.contiguous(), h.contiguous(), self.norm1.weight.float(),
                                          self.norm1.bias.float(), self.norm1.eps)
        elif self.gated is None:
            z = self.norm1(h + self.wo(a))
        else:
            z = residual_norm(h, self.wo(a), self.norm1.weight, self.norm1.bias, eps=self.norm1.eps)
        if self.gated is None:
            return self.norm2(z + self.feed_forward(z))
        return residual_norm(z, self.feed_forward(z), self.norm2.weight, self.norm2.bias, eps=self.norm2.eps)

    def forward(self, h, lengths=None, y=None, next_norm=None):
        """y: pre1(H) where the caller has it already (sandwich form); next_norm: see after_attention."""
        B, N, D = h.shape
        split = lambda x: x.view(B, N, self.h, self.dh)
        p_drop = self.attn_dropout if self.training else 0.0
        seed = int(torch.randint(0, 2 ** 62, (1,)).item()) if p_drop else 0   # a fresh mask per call, from torch's CPU generator
        x = self.attention_input(h) if y is None else y
        a = graph_self_attention(self.g, split(self.wq(x)), split(self.wk(x)), split(self.wv(x)),
                                 self.rel_emb.to(x.dtype), lengths=lengths, dropout_p=p_drop, dropout_seed=seed)
        return self.after_attention(h, a.reshape(B, N, D), next_norm)


class BPTEncoder(nn.Module):
    """A stack of BPT layers over one sequence length n (a power of two).

    Token nodes start from the given token states, span nodes from zero, and all nodes are updated
    together in every layer (Sec. 3.3).  `readout`: "tokens" returns the token states [B, n, D]
    (language modelling, translation), "root" the root node's state [B, D] (classification).
    gated, sandwich, alpha: the layers' forms (see BPTLayer); a sandwich stack ends with one more norm, norm_out."""

    def __init__(self, n: int, k: int, d_model: int, n_heads: int, d_ff: int, n_layers: int, left_only: bool = False,
                 device="cuda", attn_dropout: float = 0.0, gated=None, sandwich: bool = False, alpha: float = 1.0):
        super().__init__()
        self.n, self.sandwich = n, sandwich
        self.g = binding.bpt_build_graph(n, k, binding.BPT_LEFT_ONLY if left_only else 0, device=device)
        self.layers = nn.ModuleList(BPTLayer(self.g, d_model, n_heads, d_ff, attn_dropout=attn_dropout, gated=gated, sandwich=sandwich,
                                             alpha=alpha) for _ in range(n_layers))
        if sandwich:
            self.norm_out = nn.LayerNorm(d_model)

    def forward(self, tokens, lengths=None, readout: str = "tokens"):
        B, n, D = tokens.shape
        if n != self.n:
            raise ValueError("expected %d token states per sequence, got %d" % (self.n, n))
        h = torch.cat([tokens, tokens.new_zeros(B, n - 1, D)], dim=1)
        if self.sandwich:
            y = None
            for layer, norm in zip(self.layers, [l.pre1 for l in self.layers[1:]] + [self.norm_out]):
                h, y = layer(h, lengths, y, norm)
            h = y if len(self.layers) else residual_norm(h, None, self.norm_out.weight, self.norm_out.bias, eps=self.norm_out.eps)
        else:
            for layer in self.layers:
                h = layer(h, lengths)
        if readout == "tokens":
            return h[:, :n]
        if readout == "root":
            return h[:, -1]
        raise ValueError("readout must be 'tokens' or 'root'")


class BPTDecoder:
    """Step-by-step evaluation of a left-only BPTEncoder with cached per-layer state, for autoregressive use
    (Sec. 4.2 trains BPT as a language model; generation feeds it one token at a time).

    When token i arrives, the only nodes whose state changes in any layer are token i and its log2(n)
    ancestors: every other token lies to its left and attends only nodes that lie wholly to its own left.
    The decoder therefore keeps, per layer, the input states of all 2n-1 nodes and their key / value
    rows, recomputes those log2(n) + 1 rows per layer with `bpt_attn_fwd_rows` and lengths = i + 1 (the
    ancestors then attend exactly the tokens seen so far), and returns the last layer's state of token i.
    A span is complete once its last token has arrived; from then on its cached state is the one a full
    forward pass over the finished sequence computes, so the token outputs of the steps equal the token
    rows of `BPTEncoder.forward` on the whole sequence."""

    def __init__(self, enc: BPTEncoder, batch: int, dtype=torch.float32):
        g = enc.g
        if not (g.dims.flags & binding.BPT_LEFT_ONLY):
            raise ValueError("step-by-step decoding needs the left-only graph")
        self.enc, self.g, self.n, self.batch = enc, g, enc.n, batch
        first = enc.layers[0]
        dev = first.rel_emb.device
        D, H, dh, N = first.h * first.dh, first.h, first.dh, g.n_nodes
        self.L = g.dims.n_levels
        self.h = [torch.zeros(batch, N, D, device=dev, dtype=dtype) for _ in range(len(enc.layers) + 1)]
        heads = lambda: torch.zeros(batch, N, H, dh, device=dev, dtype=dtype)
        self.q, self.k, self.v, self.a = ([heads() for _ in enc.layers] for _ in range(4))
        self.lse = torch.zeros(batch, N, H, device=dev, dtype=torch.float32)
        self.pos = 0

    def rows_of_step(self, i: int):
        """Token i and its ancestors, finest first."""
        n = self.n
        return [i] + [2 * n - ((2 * n) >> j) + (i >> j) for j in range(1, self.L + 1)]

    @torch.no_grad()
    def step(self, token_state):
        """token_state: [batch, D], the input state of the next token.  Returns its output state [batch, D]."""
        i = self.pos
        if i >= self.n:
            raise ValueError("the sequence is full (n = %d)" % self.n)
        rows = self.rows_of_step(i)
        B, R = self.batch, len(rows)
        dev = self.h[0].device
        idx = torch.tensor(rows, device=dev)
        rows_t = torch.tensor([rows] * B, dtype=torch.int32, device=dev)
        lens = torch.full((B,), i + 1, dtype=torch.int32, device=dev)
        self.h[0][:, i] = token_state.to(self.h[0].dtype)
        for li, layer in enumerate(self.enc.layers):
            hr = self.h[li][:, idx]                                     # [B, R, D]; span rows of layer 0 are zero
            x = layer.attention_input(hr)
            split = lambda t: t.view(B, R, layer.h, layer.dh)
            self.q[li][:, idx] = split(layer.wq(x))
            self.k[li][:, idx] = split(layer.wk(x))
            self.v[li][:, idx] = split(layer.wv(x))
            binding.bpt_attn_fwd_rows(self.g, self.q[li], self.k[li], self.v[li], layer.rel_emb.to(hr.dtype).contiguous(),
                                      1.0 / math.sqrt(layer.dh), rows_t, self.a[li], self.lse, lengths=lens)
            self.h[li + 1][:, idx] = layer.after_attention(hr, self.a[li][:, idx].reshape(B, R, -1), fuse=False)
        self.pos += 1
        out = self.h[-1][:, i]
        if self.enc.sandwich:
            norm = self.enc.norm_out
            out = residual_norm(out, None, norm.weight, norm.bias, eps=norm.eps)
        return out
