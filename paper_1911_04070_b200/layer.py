"""BP-Transformer layers on top of the graph self-attention library (arXiv 1911.04070, Sec. 3.3,
Algorithm 2): PyTorch modules whose attention runs in libbpt.so.

The graph self-attention, the gated feed-forward block, the seam between two blocks (norms, gate, residual), and at the ends of a
language model the way from ids to node states, the clipping of gradients and the adjustment of logits are this
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


def _check_constant(name, v, of="residual_norm", instead="gate or h"):
    """alpha, eps and scale are numbers; a tensor would be read as one, and its gradient or tangent lost."""
    if isinstance(v, torch.Tensor) and ((v.requires_grad and torch.is_grad_enabled()) or forward_ad.unpack_dual(v).tangent is not None):
        raise NotImplementedError("%s has no derivative with respect to %s; a learned factor goes into %s" % (of, name, instead))


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


def token_states(ids, weight, scale=1.0, span_rows=0, lengths=None, padding_idx=None, dtype=None):
    """Token ids to node states, differentiable in the table:  out[..., t, :] = scale * weight[ids[..., t]]  for t < lengths[...], zeros behind
    the length and in the span_rows rows behind the tokens (Sec. 3.3: span nodes start from zero; n - 1 of them in a tree over n tokens).

    ids: [..., n] int32 or int64; weight: [V, D] float32 or bfloat16; lengths: int32 of the shape ids.shape[:-1], or None; ids behind it are
    not looked at; scale: a number; dtype: of the result (default: weight's).  Returns [..., n + span_rows, D].  The gradient
    is the whole [V, D], in weight's type, summed in float32 in the order of the tokens (bit-reproducible); it is zero at padding_idx.  An
    id outside the table reads nothing: its row is zeros, it adds nothing to the gradient, and binding.bpt_check_device says so.
    Capture, modes of differentiation and tracing as in residual_norm."""
    if type(scale) is not float:
        _check_constant("scale", scale, "token_states", "weight")
    padding = -1 if padding_idx is None else padding_idx if padding_idx >= 0 else -2       # -1 is none, below that is refused
    out = binding.load_native().token_states(ids, weight, lengths, scale, span_rows, padding, dtype)
    if out is None:
        if weight.dim() == 2 and padding_idx is not None and not 0 <= padding_idx < weight.shape[0]:
            raise ValueError("padding_idx must be None or an id of the table")
        cont = lambda t: t if t is None else t.contiguous()
        binding.bpt_embed_fwd(cont(ids), cont(weight), scale, span_rows, cont(lengths), dtype)                     # says what is wrong
        raise RuntimeError("token_states: refused")
    if binding.CHECK_DEVICE_STATUS:
        status = binding.bpt_check_device(ids.device)
        if status == 8:
            raise IndexError("token_states: an id is outside the table")
        if status:
            raise RuntimeError("a device-side wait timed out before token_states")
    return out


def _clip(grads, out, norm_type, clip, max_norm, eps):
    grads = grads if isinstance(grads, torch.Tensor) else list(grads)
    out = out if out is None or isinstance(out, torch.Tensor) else list(out)
    code = binding.GRAD_NORMS.get(norm_type)
    norm = None if code is None else binding.load_native().clip_gradients(grads, out, code, clip, max_norm, eps)
    if norm is None:        # says what is wrong
        as_list = lambda t: [t] if isinstance(t, torch.Tensor) else t
        if out is not None and len(as_list(out)) != len(as_list(grads)):
            raise ValueError("out must have an entry for every gradient")
        pairs = [(g, o) for g, o in zip(as_list(grads), as_list(grads if out is None else out)) if g is not None]
        if clip and any(t is not None and t.is_leaf and t.requires_grad for t in (as_list(grads) if out is None else as_list(out))):
            raise ValueError("leaves that require a gradient are not written: give the gradients, not the parameters")
        grads, into = [g.contiguous() for g, _ in pairs], None if out is None else [o if o is None else o.new_empty(o.shape) for _, o in pairs]
        if out is not None and any(o is None for o in into):
            raise ValueError("out must have a tensor for every gradient")
        binding._grad_list(grads, into, norm_type)
        if clip and (not max_norm >= 0 or not eps >= 0):
            raise ValueError("max_norm and eps must not be negative")
        raise ValueError("a tensor is given twice, or what is written overlaps another tensor of the call or itself")
    return norm


def gradient_norm(grads, norm_type=2.0):
    """The 2-norm (norm_type=float("inf"): the largest absolute value) over all elements of a list of tensors, float32 or bfloat16 mixed, as
    a float32 tensor [].  None entries count for nothing; nothing at all gives 0.  Squares are summed in 64 bits where 32 would
    lose them: right for gradients of any size (infinite where float32 has no such number).  Two launches whatever the number of tensors up to
    960; bit-reproducible; can be captured."""
    return _clip(grads, None, norm_type, False, 0.0, 0.0)


def clip_gradients(grads, max_norm, norm_type=2.0, eps=1e-6, out=None):
    """Scales all gradients of a model by min(1, max_norm / (norm + eps)) and returns their norm before (see gradient_norm).

    grads: a list of tensors, float32 or bfloat16 mixed, on one device (``[p.grad for p in model.parameters()]``; None entries are passed over).
    They are scaled in place, and not written where the norm is below max_norm; or, with out (a list of as many tensors, float32 or
    bfloat16, say the gradients of an optimizer's 32-bit master weights), left as they are and the scaled values written there.  Any
    strides; no tensor twice and no overlaps between what is written and anything else; no leaf that requires a gradient is written (a parameter
    given for its gradient is refused).  Gradients whose norm is beyond float32 are scaled by it all the same.  A NaN makes the norm and all results NaN (an
    infinite max_norm scales nothing, whatever the norm).  Nothing
    is read back to the host: can be captured in a CUDA graph, which then uses these very tensors."""
    return _clip(grads, out, norm_type, True, max_norm, eps)


def adjust_logits(logits, history=None, lengths=None, prompt_lengths=None, repetition=1.0, presence=0.0, frequency=0.0, bias=None,
                  bias_ids=None, bias_values=None, allowed=None, out=None):
    """What a decoding step does to its logits [B, V] before a token is taken.  For an id that stands in history[b, :lengths[b]]:
    x / repetition where x > 0, else x * repetition; for one that stands n > 0 times behind the prompt, in history[b, prompt_lengths[b]:lengths[b]]:
    x - frequency * n - presence; then x + bias, and -inf for what is not allowed (NaN there, too; a row without an allowed id is all -inf).

    logits: float32 or bfloat16.  history: [B, T] int32 or int64; lengths, prompt_lengths: int32 [B] (None: T and 0); ids outside the
    vocabulary count for nothing.  repetition (above 0), presence, frequency: numbers, or float32 tensors [B], one setting per row.
    bias: [V] or [B, V], float32 or bfloat16.  bias_ids (int32 or int64), bias_values (float32): [B, K], a few biased ids per row (outside the
    vocabulary: no effect; given twice: the last one counts).  allowed: int32 [ceil(V / 32)] or [B, ceil(V / 32)], bit v % 32 of word v // 32 set
    where id v is allowed.  out: a tensor [B, V], float32 or bfloat16, its rows without gaps, the logits themselves for one (default: a new one of the logits'
    type), apart from all other arguments.  Any strides.  Computed in float32, rounded once.  For inference: arguments that require a gradient are refused."""
    got = binding.load_native().adjust_logits(logits, history, lengths, prompt_lengths, repetition, presence, frequency, bias, bias_ids, bias_values,
                                              allowed, out)
    if got is None:
        cont = lambda t: t.contiguous() if isinstance(t, torch.Tensor) else t
        if out is not None and (out.shape != logits.shape or out.device != logits.device or logits.dim() != 2
                                or (out.shape[1] > 1 and out.stride(1) != 1) or (out.shape[0] > 1 and out.stride(0) < out.shape[1])):
            raise ValueError("out must be [B, V] on the device of the logits, its rows without gaps")
        binding.bpt_adjust_logits(*map(cont, (logits, history, lengths, prompt_lengths, repetition, presence, frequency, bias, bias_ids, bias_values,
                                              allowed)), None if out is None else out.new_empty(out.shape))      # says what is wrong
        raise ValueError("out overlaps the logits without being them, or another argument")
    return got


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
        return self.forward_nodes(torch.cat([tokens, tokens.new_zeros(B, n - 1, D)], dim=1), lengths, readout)

    def forward_nodes(self, h, lengths=None, readout: str = "tokens"):
        """The same from the states of all nodes [B, 2n-1, D] (token_states makes them from ids)."""
        n = self.n
        if h.shape[1] != 2 * n - 1:
            raise ValueError("expected the states of %d nodes per sequence, got %d" % (2 * n - 1, h.shape[1]))
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


class BPTLanguageModel(nn.Module):
    """Token ids to logits with a left-only BPTEncoder (Sec. 4.2): node states from a table of embeddings scaled by sqrt(d_model), the stack,
    and a projection to the vocabulary by the same table (tied) or by one of its own.

    vocab: ids 0 .. vocab - 1; padding_idx: an id whose embedding is not trained by its own places; the other arguments are BPTEncoder's."""

    def __init__(self, vocab: int, n: int, k: int, d_model: int, n_heads: int, d_ff: int, n_layers: int, tied: bool = True, padding_idx=None,
                 device="cuda", **form):
        super().__init__()
        if vocab < 1 or (padding_idx is not None and not 0 <= padding_idx < vocab):
            raise ValueError("vocab must be at least 1, and padding_idx None or an id below it")
        self.vocab, self.padding_idx, self.scale = vocab, padding_idx, math.sqrt(d_model)
        self.embedding = nn.Parameter(torch.randn(vocab, d_model) * d_model ** -0.5)
        self.encoder = BPTEncoder(n, k, d_model, n_heads, d_ff, n_layers, left_only=True, device=device, **form)
        self.head = None if tied else nn.Linear(d_model, vocab, bias=False)

    def logits(self, h):
        """[..., d_model] states of tokens to [..., vocab] logits of what follows them."""
        return torch.nn.functional.linear(h, self.embedding if self.head is None else self.head.weight)

    def forward(self, ids, lengths=None):
        """ids: [B, n] int32 or int64, n the encoder's; lengths: int32 [B], or None (all n; what stands behind a length is not looked at).
        Returns the logits [B, n, vocab]; those behind a length mean nothing."""
        n = self.encoder.n
        if ids.dim() != 2 or ids.shape[1] != n:
            raise ValueError("expected %d ids per sequence (pad shorter ones and give lengths)" % n)
        h = token_states(ids, self.embedding, self.scale, n - 1, lengths, self.padding_idx)
        return self.logits(self.encoder.forward_nodes(h, lengths))

    def loss(self, ids, lengths=None):
        """The mean cross entropy, in float32, of each token given those before it.  An id outside the vocabulary is no target; token_states
        reports it."""
        x = self(ids, lengths)[:, :-1].float()
        want = ids[:, 1:].long()
        want = want.masked_fill((want < 0) | (want >= self.vocab), -100)        # cross_entropy would end the process's use of the device
        if lengths is not None:
            want = want.masked_fill(torch.arange(1, ids.shape[1], device=ids.device) >= lengths[:, None], -100)
        return torch.nn.functional.cross_entropy(x.reshape(-1, self.vocab), want.reshape(-1), ignore_index=-100)

    @torch.no_grad()
    def generate(self, prompt, steps: int, temperature: float = 0.0, generator=None, allowed=None, end_id=None, **settings):
        """Continues the prompts [B, P] (P >= 1 ids each, int32 or int64) by `steps` ids, token by token with cached states (BPTDecoder).

        allowed: the ids that may follow, as adjust_logits takes them, or a function of the ids so far [B, t] that returns them (a grammar).
        settings: repetition, presence, frequency, bias, bias_ids, bias_values, see adjust_logits; the prompt counts for repetition only.
        temperature 0 takes the largest logit (the lowest id of equal ones), another one draws from softmax(logits / temperature) with
        torch's `generator`.  A sequence has ended at the first step at which its mask or bias leaves it no id (logits of -inf only): it takes
        end_id there and at all steps behind; without an end_id it raises ValueError when the steps are through.  So does a draw from logits that are
        not finite, or not after the division.  Returns [B, P + steps] ids."""
        B, P = prompt.shape
        if P < 1 or steps < 0 or P + steps > self.encoder.n:
            raise ValueError("a prompt of at least one id and room for it and the steps in %d ids are needed" % self.encoder.n)
        if temperature < 0:
            raise ValueError("temperature must not be negative")
        if end_id is not None and not 0 <= end_id < self.vocab:
            raise ValueError("end_id must be None or an id of the vocabulary")
        ids = torch.cat([prompt, prompt.new_zeros(B, steps)], dim=1)
        lengths, prompts = (torch.full((B,), P, dtype=torch.int32, device=ids.device) for _ in range(2))
        dec = BPTDecoder(self.encoder, B, dtype=self.embedding.dtype)
        # a step's largest logits say whether there was anything to take; they are looked at when all steps are through
        forbids = allowed is not None or settings.get("bias") is not None or settings.get("bias_values") is not None
        tops, ended = [], torch.zeros(B, dtype=torch.bool, device=ids.device)
        for t in range(P + steps - 1):
            state = dec.step(token_states(ids[:, t], self.embedding, self.scale))
            if t < P - 1:
                continue
            # in float32 from here on, in place
            x = self.logits(state).float()
            adjust_logits(x, ids, lengths, prompts, allowed=allowed(ids[:, :t + 1]) if callable(allowed) else allowed, out=x, **settings)
            lengths += 1
            if temperature > 0:
                tops.append(x.amax(-1))
                p = torch.softmax(x / temperature, -1).nan_to_num_(nan=1.0)         # a row of NaN is no row to draw from; what is drawn there is dropped
                new = torch.multinomial(p, 1, generator=generator)[:, 0]
            elif forbids:
                top, new = x.max(-1)
                tops.append(top)
            else:
                new = x.argmax(-1)
            if callable(allowed):           # which is shown the ids
                ended |= tops[-1] == -math.inf
                new = new.masked_fill(ended, end_id or 0)
            ids[:, t + 1] = new
        if tops:
            top = torch.stack(tops, 1)
            divided = top / temperature if temperature > 0 else None
            if divided is not None and bool((~(divided < math.inf) | (divided == -math.inf) & (top > -math.inf)).any()):
                raise ValueError("logits were not finite, or not after the division by the temperature")
            over = (top == -math.inf).cumsum(1) > 0
            if end_id is not None:
                ids[:, P:].masked_fill_(over, end_id)
            elif bool(over.any()):
                raise ValueError("a sequence was left without an allowed id; an end_id is what such a sequence takes from there on")
        return ids


def training_step(model, optimizer, ids, lengths=None, max_norm: float = 1.0):
    """One step of a BPTLanguageModel: loss, backward pass, clipping of all gradients by their norm, the optimizer's step.  Returns (loss, norm
    before clipping) as tensors on the device; nothing is read back."""
    optimizer.zero_grad(set_to_none=True)
    loss = model.loss(ids, lengths)
    loss.backward()
    norm = clip_gradients([p.grad for p in model.parameters()], max_norm)
    optimizer.step()
    return loss.detach(), norm
