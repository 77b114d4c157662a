"""BPTLayer / BPTEncoder / BPTDecoder in their gated and sandwich forms: the run of the position-wise operators together, as a
model uses them, against the float64 layer oracle -- outputs, every gradient, and step-by-step decoding.

Bounds, as for the plain layer: float32 2e-4 of the largest value (the general attention kernels' own rounding dominates);
bfloat16 10 % in the 2-norm, since single relu gates and softmax weights turn on the rounding of PyTorch's bf16 products."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

NAMES = {"wq": "wq.weight", "wk": "wk.weight", "wv": "wv.weight", "wo": "wo.weight", "rel_emb": "rel_emb",
         "ln1_w": "norm1.weight", "ln1_b": "norm1.bias", "ln2_w": "norm2.weight", "ln2_b": "norm2.bias"}
PLAIN = {"ff1_w": "ff1.weight", "ff1_b": "ff1.bias", "ff2_w": "ff2.weight", "ff2_b": "ff2.bias"}
GATED = {"ff_gate": "ff_gate.weight", "ff_up": "ff_up.weight", "ff_down": "ff_down.weight"}
SANDWICH = {"pre1_w": "pre1.weight", "pre1_b": "pre1.bias", "pre2_w": "pre2.weight", "pre2_b": "pre2.bias", "gate1": "gate1", "gate2": "gate2"}
FORMS = [("silu", True, 0.8), ("gelu", False, 1.0), ("relu", True, 1.0), (None, True, 0.5)]


def _encoder(n, k, D, H, F, n_layers, left_only, dtype, form):
    import torch
    from paper_1911_04070_b200 import layer
    gated, sandwich, alpha = form
    enc = layer.BPTEncoder(n, k, D, H, F, n_layers, left_only=left_only, device="cuda:0", gated=gated, sandwich=sandwich, alpha=alpha).to("cuda:0")
    g = torch.Generator(device="cuda:0").manual_seed(5)
    with torch.no_grad():
        for name, p in enc.named_parameters():
            if "rel_emb" in name:
                p.mul_(10.0)                # relation embeddings large enough to matter
            elif p.dim() == 1:              # norms and gates away from ones and zeros
                p.add_(0.2 * torch.randn(p.shape, generator=g, device="cuda:0"))
            p.copy_(p.to(dtype).float())
    return enc.to(dtype)


def _oracle(enc, tokens, n, k, left_only, H, form, lengths):
    from oracle import bpt_layer, bpt_oracle as orc
    import torch
    gated, sandwich, alpha = form
    names = {**NAMES, **(PLAIN if gated is None else GATED), **(SANDWICH if sandwich else {})}
    g = orc.enumerate_graph(n, k, 1 if left_only else 0)
    ws = [{a: dict(l.named_parameters())[b].detach().double().cpu().requires_grad_(True) for a, b in names.items()} for l in enc.layers]
    x = tokens.detach().double().cpu().requires_grad_(True)
    B, _, D = x.shape
    mask, rel = bpt_layer.dense_tables(g, lengths, B)
    h = torch.cat([x, torch.zeros(B, n - 1, D, dtype=x.dtype)], dim=1)
    for w in ws:
        h = bpt_layer.layer_forward_form(h, w, mask, rel, H, gated, sandwich, alpha)
    out = None
    if sandwich:
        out = {a: p.detach().double().cpu().requires_grad_(True) for a, p in enc.norm_out.named_parameters()}
        h, _ = bpt_layer.res_norm(h, None, out["weight"], out["bias"])
    return x, ws, out, h[:, :n], names


@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("dtype,D,H,F,tol", [("float32", 64, 2, 96, 2e-4), ("bfloat16", 128, 2, 264, 1e-1)])
def test_outputs_and_gradients(form, dtype, D, H, F, tol):
    import torch
    torch.manual_seed(0)
    dt = getattr(torch, dtype)
    n, k, B, lengths = (32, 2, 2, [32, 19]) if dtype == "float32" else (128, 4, 2, [128, 77])
    enc = _encoder(n, k, D, H, F, 2, False, dt, form)
    tokens = torch.randn(B, n, D).to(dt).to("cuda:0").requires_grad_(True)
    up = torch.randn(B, n, D, device="cuda:0")
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda:0")
    y = enc(tokens, lens)
    (y.float() * up).sum().backward()
    x64, ws, out64, y64, names = _oracle(enc, tokens, n, k, False, H, form, lengths)
    (y64 * up.double().cpu()).sum().backward()

    def close(name, got, want):
        got, want = got.detach().double().cpu().numpy(), want.detach().numpy()
        assert np.isfinite(got).all(), name
        if dt == torch.float32:
            err, scale = np.abs(got - want).max(), np.abs(want).max()
        else:
            err, scale = np.linalg.norm(got - want), np.linalg.norm(want)
        assert err <= tol * max(scale, 1e-30), "%s: %.3e vs scale %.3e" % (name, err, scale)

    close("output", y, y64)
    close("d tokens", tokens.grad, x64.grad)
    for li, l in enumerate(enc.layers):
        ps = dict(l.named_parameters())
        assert len(ps) == len(names)
        for a, b in names.items():
            close("layer %d d %s" % (li, a), ps[b].grad, ws[li][a].grad)
    if out64:
        for a, p in enc.norm_out.named_parameters():
            close("d norm_out " + a, p.grad, out64[a].grad)


def test_a_bf16_sandwich_layer_runs_on_the_operators():
    """Two layers: one norm at the start, one seam after each block; no other norm, no separate activation."""
    import torch
    from paper_1911_04070_b200 import binding
    enc = _encoder(128, 4, 128, 2, 264, 2, False, torch.bfloat16, ("silu", True, 0.8))
    x = torch.randn(2, 128, 128, device="cuda:0").bfloat16().requires_grad_(True)
    binding.bpt_trace_begin(128)
    y = enc(x)
    names = [a for a, _ in binding.bpt_trace_end(128)]
    assert names.count("res_norm_fwd") == 5 and names.count("gated_ff_in") == 2 and names.count("gated_ff_out") == 2, names
    binding.bpt_trace_begin(128)
    y.float().sum().backward()
    names = [a for a, _ in binding.bpt_trace_end(128)]
    assert names.count("res_norm_bwd") == 5 and names.count("gated_ff_bwd_in") == 2 and names.count("gated_ff_dw") == 2, names
    assert binding.bpt_check(None) == 0


@pytest.mark.parametrize("form", [("silu", True, 0.8), ("gelu", False, 1.0)])
@pytest.mark.parametrize("dtype,tol", [("float32", 5e-5), ("bfloat16", 6e-2)])
def test_step_by_step_decoding_reproduces_the_full_forward(form, dtype, tol):
    """float32: the same kernels on fewer rows, dense products in another order.  bfloat16: besides that the few-rows kernels keep
    the inner row unrounded, and PyTorch's products round at other shapes: two bf16 pipelines, 2-norm."""
    import torch
    from paper_1911_04070_b200 import layer
    torch.manual_seed(1)
    n, k, B, D, H, F = 64, 3, 2, 64, 2, 136
    enc = _encoder(n, k, D, H, F, 2, True, getattr(torch, dtype), form).eval()
    tokens = torch.randn(B, n, D, device="cuda:0").to(getattr(torch, dtype))
    with torch.no_grad():
        full = enc(tokens).float()
    dec = layer.BPTDecoder(enc, B, dtype=tokens.dtype)
    steps = torch.stack([dec.step(tokens[:, i]) for i in range(n)], dim=1).float()
    if dtype == "float32":
        err, scale = (steps - full).abs().max().item(), full.abs().max().item()
    else:
        err, scale = (steps - full).norm().item(), full.norm().item()
    assert err <= tol * scale, (err, scale)


def test_refusals():
    from paper_1911_04070_b200 import layer
    mk = lambda **kw: layer.BPTEncoder(32, 2, kw.pop("D", 64), 2, kw.pop("F", 64), 1, device="cuda:0", **kw)
    for kw in (dict(gated="tanh"), dict(gated="silu", F=60), dict(gated="silu", D=36), dict(alpha=0.5)):
        with pytest.raises(ValueError):
            mk(**kw)


_CAPTURE = r"""
import torch
from paper_1911_04070_b200 import layer
t = lambda *s: torch.randn(*s, device="cuda:0").bfloat16().mul_(0.1).requires_grad_(True)
x, wg, wu, wd, w = t(40, 64), t(128, 64), t(128, 64), t(64, 128), t(64)
which = {"ff": (lambda: layer.gated_feed_forward(x, wg, wu, wd), (x, wg, wu, wd)), "norm": (lambda: layer.residual_norm(x, None, w), (x, w))}
for name, (call, leaves) in which.items():
    def backward():
        for v in leaves:
            v.grad = None
        call().float().square().sum().backward()
        return [v.grad for v in leaves]
    want = [g.clone() for g in backward()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        backward()
    torch.cuda.synchronize()
    alive = call()                       # on the default stream: the leaves' accumulation nodes are this graph's
    graph = torch.cuda.CUDAGraph()
    try:
        with torch.cuda.graph(graph):
            backward()
    except RuntimeError as e:
        assert "still alive" in str(e), e
    else:
        raise AssertionError(name + ": not refused")
    assert all(torch.equal(a, b) for a, b in zip(want, backward()))      # nothing is left of the attempt
    del alive, graph
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = backward()
    for g in got:
        g.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got)), name
print("captured")
"""


def test_captured_backward_beside_a_living_eager_graph():
    """Refused while the capture is whole; with the eager graph deleted the same pass is captured and replays the same bits."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _CAPTURE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
