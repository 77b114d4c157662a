"""bpt_res_norm (norm after a block, gate, scaled residual, norm before the next block) and its backward against the
float64 oracle, over types, widths, row counts, gates and absent parts.

Tolerances, fixed before the first run.  A stored value is rounded once: at most eps / 2 of its type, relative (bf16
2^-8, fp32 2^-24).  The fp32 arithmetic before it is a chain of at most ~40 roundings of terms no larger than the sum
of the absolute terms of the formula, S (taken from the oracle's own tensors below), times the amplification of the
subtraction of the mean, A = 1 + max|x| / sigma per normalised row (an error of u |x| in x is an error of
u |x| / sigma in the normalised value).  64 u S A with u = 2^-24 covers it.  A column sum of R rows adds at most
R / 148 + 64 roundings in sequence to that; 512 u S A holds for every row count here."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def _case(rows_shape, D, dtype, norm, post, gate_shape, alpha, param, seed, offset=0.0, device="cuda:0"):
    import torch
    g = torch.Generator().manual_seed(seed)
    t = {"bf16": torch.bfloat16, "f32": torch.float32}
    rnd = lambda *shape, s=1.0, m=0.0, d=dtype: (torch.randn(*shape, generator=g) * s + m).to(t[d])
    x = dict(h=rnd(*rows_shape, D, m=offset), b=rnd(*rows_shape, D, s=0.5, m=-offset))
    for name, kind in (("", norm), ("post_", post)):
        x[name + "weight"] = rnd(D, s=0.3, m=1.0, d=param) if kind else None
        x[name + "bias"] = rnd(D, s=0.3, d=param) if kind == "layer" else None
    x["gate"] = None if gate_shape is None else rnd(*gate_shape, s=0.3, m=0.8, d=param)
    up = dict(dr=rnd(*rows_shape, D), dy=rnd(*rows_shape, D))
    dev = lambda d: {a: None if b is None else b.to(device) for a, b in d.items()}
    return dev(x), dev(up), dict(norm=norm, post_norm=post, alpha=alpha, eps=1e-5)


def _amp(x):
    """1 + max|x| / sigma per row."""
    sig = (((x - x.mean(-1, keepdims=True)) ** 2).mean(-1, keepdims=True) + 1e-5) ** 0.5
    return 1 + np.abs(x).max(-1, keepdims=True) / sig


def _close(name, got, want, scale, half, c=64):
    got = got.detach().double().cpu().numpy()
    assert got.shape == want.shape and np.isfinite(got).all(), name
    bad = np.abs(got - want) > half * np.abs(want) * (1 + 2 * half) + c * U * scale
    assert not bad.any(), "%s: %d of %d outside, worst %.3g at scale %.3g" % (
        name, bad.sum(), bad.size, np.abs(got - want)[bad].max(), np.broadcast_to(scale, want.shape)[bad].max())


def _oracle(x, up, cfg):
    import torch
    from oracle import bpt_layer
    leaf = {a: None if v is None else v.detach().double().cpu().requires_grad_(True) for a, v in x.items()}
    y, r = bpt_layer.res_norm(**leaf, **cfg)
    names = [a for a in leaf if leaf[a] is not None]
    loss = (r * up["dr"].double().cpu()).sum() if up["dr"] is not None else 0.0
    loss = loss + ((y * up["dy"].double().cpu()).sum() if cfg["norm"] and up["dy"] is not None else 0.0)
    grads = dict(zip(names, torch.autograd.grad(loss, [leaf[a] for a in names], allow_unused=True)))
    return y.detach().numpy(), r.detach().numpy(), {a: np.zeros(tuple(leaf[a].shape)) if g is None else g.numpy() for a, g in grads.items()}


def _check(x, up, cfg, dtype, param):
    import torch
    from paper_1911_04070_b200 import layer
    leaf = {a: None if v is None else v.clone().requires_grad_(True) for a, v in x.items()}
    norm = cfg["norm"]
    out = layer.residual_norm(**leaf, **cfg, return_sum=True)
    r, y = out if norm else (out, None)
    y64, r64, g64 = _oracle(x, up, cfg)
    f = lambda a: None if x[a] is None else x[a].double().cpu().numpy()
    h, b, w, pw = f("h"), f("b"), f("weight"), f("post_weight")
    gate = 1.0 if x["gate"] is None else f("gate")
    amp_b = _amp(b) if cfg["post_norm"] else 1.0
    big = lambda v: np.abs(v).max(-1, keepdims=True)
    wmax, pwmax = (1.0 if v is None else np.abs(v).max() for v in (w, pw))
    biasmax = [0.0 if x[a] is None else float(x[a].float().abs().max()) for a in ("bias", "post_bias")]
    n_s = big(np.abs(r64) + np.abs(cfg["alpha"] * h)) if cfg["post_norm"] else big(b)      # |gate n| <= |r| + |alpha h|
    r_s = (np.abs(cfg["alpha"]) * big(h) + n_s + biasmax[1]) * amp_b
    _close("r", r, r64, r_s, HALF[dtype])
    amp_r = 1.0
    if norm:
        sig = (((r64 - (r64.mean(-1, keepdims=True) if norm == "layer" else 0)) ** 2).mean(-1, keepdims=True) + 1e-5) ** 0.5
        amp_r = 1 + r_s / sig
        _close("y", y, y64, (big(y64) + wmax + biasmax[0]) * amp_r, HALF[dtype])
    tops = [(r, up["dr"])] + ([(y, up["dy"])] if norm else [])
    tops = [(a, u) for a, u in tops if u is not None]
    names = [a for a in leaf if leaf[a] is not None]
    grads = dict(zip(names, torch.autograd.grad([a for a, _ in tops], [leaf[a] for a in names], [u for _, u in tops])))
    # sums of absolute terms of the gradient formulas
    z = lambda k: 0.0 if up[k] is None else np.abs(up[k].double().cpu().numpy())
    d_s = big(z("dr") + np.zeros_like(h))
    if norm:
        xh = np.abs(y64 - (0 if x["bias"] is None else f("bias"))) / (1.0 if w is None else np.maximum(np.abs(w), 1e-2))
        d_s = d_s + big(z("dy")) * wmax * (1 + big(xh) ** 2) / sig * amp_r
    _close("dh", grads["h"], g64["h"], np.abs(cfg["alpha"]) * d_s, HALF[dtype])
    gmax = np.abs(gate).max()
    db_s = gmax * d_s
    if cfg["post_norm"]:
        sb = (((b - (b.mean(-1, keepdims=True) if cfg["post_norm"] == "layer" else 0)) ** 2).mean(-1, keepdims=True) + 1e-5) ** 0.5
        bh = big(np.abs(b - (b.mean(-1, keepdims=True) if cfg["post_norm"] == "layer" else 0)) / sb)
        db_s = db_s * pwmax * (1 + bh ** 2) / sb * amp_b
    _close("db", grads["b"], g64["b"], db_s, HALF[dtype])
    flat = lambda v: np.broadcast_to(v, h.shape).reshape(-1, h.shape[-1])
    cols = lambda v: flat(v).sum(0)
    if norm and w is not None:
        _close("d_weight", grads["weight"], g64["weight"], cols((z("dy") + np.zeros_like(h)) * big(xh) * amp_r), HALF[param], 512)
        if x["bias"] is not None:
            _close("d_bias", grads["bias"], g64["bias"], cols(z("dy") + np.zeros_like(h)), HALF[param], 512)
    if x["gate"] is not None:
        s = flat(d_s * (r_s + n_s))
        gs = grads["gate"].shape
        G = int(np.prod(gs[:-1]))
        _close("d_gate", grads["gate"], g64["gate"], s.reshape(G, -1, h.shape[-1]).sum(1).reshape(gs), HALF[param], 512)
    if cfg["post_norm"]:
        _close("d_post_weight", grads["post_weight"], g64["post_weight"], cols(gmax * d_s * bh * amp_b), HALF[param], 512)
        if x["post_bias"] is not None:
            _close("d_post_bias", grads["post_bias"], g64["post_bias"], cols(gmax * d_s), HALF[param], 512)


KINDS = [("layer", None), ("layer", "layer"), ("rms", "rms"), ("rms", "layer"), (None, "layer"), (None, None), ("rms", None)]


@pytest.mark.parametrize("norm,post", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_kinds(norm, post, dtype):
    _check(*_case((3, 45), 96, dtype, norm, post, (96,), 0.5, "f32", 1), dtype, "f32")


@pytest.mark.parametrize("D", [1, 2, 3, 8, 31, 200, 201, 256, 264, 511, 512, 520, 1000, 1024, 1032, 2047, 2048, 2056, 4095, 4096, 4104, 8191, 8192])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_widths(D, dtype):
    x = _case((37,), D, dtype, "layer" if D > 1 else "rms", "layer" if D > 2 else "rms", (D,), 1.25, dtype, 2 + D)
    if D <= 3:      # a row of one to three channels can have almost no variance: the amplification of its mean is then unbounded
        x = _case((37,), D, dtype, "rms", "rms", (D,), 1.25, dtype, 2 + D)
    _check(*x, dtype, dtype)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 147, 148, 149, 1184, 1185, 5000, 65532])
def test_row_counts(rows):
    _check(*_case((rows,), 64, "bf16", "layer", "rms", (64,), 1.0, "bf16", rows), "bf16", "bf16")
    _check(*_case((rows,), 520, "f32", "rms", None, None, 1.0, "f32", rows), "f32", "f32")


@pytest.mark.parametrize("shape,gate", [((4, 33), (4, 1)), ((4, 33), (4, 33)), ((4, 33), (1, 1)), ((1, 33), (1, 1)), ((4, 1), (4, 1)),
                                        ((300, 3), (300, 1)), ((700, 2), (700, 2)), ((2, 3, 5), (2, 1, 1)), ((2, 3, 5), (2, 3, 1)), ((1, 1), (1, 1)),
                                        ((2, 4000), (2, 1))])
@pytest.mark.parametrize("D", [72, 1100, 77])
@pytest.mark.parametrize("dtype,param", [("bf16", "bf16"), ("f32", "f32"), ("bf16", "f32")])
def test_gates(shape, gate, D, dtype, param):
    _check(*_case(shape, D, dtype, "layer", "rms", (*gate, D), 1.0, param, 3), dtype, param)


@pytest.mark.parametrize("missing", ["dy", "dr"])
def test_one_upstream_gradient_missing(missing):
    x, up, cfg = _case((50,), 128, "bf16", "layer", "layer", (128,), 1.0, "f32", 4)
    up[missing] = None
    _check(x, up, cfg, "bf16", "f32")


def test_rows_far_from_zero():
    """A mean 200 deviations away: the variance is taken about the mean."""
    _check(*_case((65,), 512, "f32", "layer", "layer", None, 1.0, "f32", 5, offset=200.0), "f32", "f32")


def test_without_b_it_is_the_norm_alone():
    import torch
    from oracle import bpt_layer
    from paper_1911_04070_b200 import layer
    h = torch.randn(9, 96, device="cuda:0", requires_grad=True)
    w, c = torch.randn(96, device="cuda:0", requires_grad=True), torch.randn(96, device="cuda:0", requires_grad=True)
    d = torch.randn(9, 96, device="cuda:0")
    y = layer.residual_norm(h, None, w, c)
    grads = torch.autograd.grad(y, (h, w, c), d)
    l64 = [t.detach().double().cpu().requires_grad_(True) for t in (h, w, c)]
    y64, _ = bpt_layer.res_norm(l64[0], None, l64[1], l64[2])
    g64 = torch.autograd.grad(y64, l64, d.double().cpu())
    _close("y", y, y64.detach().numpy(), 10.0, U)
    for a, b in zip(grads, g64):
        _close("grad", a, b.numpy(), 200.0, U)


def test_special_rows():
    """A row of equal values under the layer norm is its bias; NaN and infinity stay in their row; no rows give empty results."""
    import torch
    from paper_1911_04070_b200 import binding, layer
    D = 40
    h = torch.randn(5, D, device="cuda:0")
    h[1] = 3.0
    h[2, 7] = float("nan")
    h[3, 9] = float("inf")
    w, c = torch.full((D,), 2.0, device="cuda:0"), torch.arange(D, device="cuda:0").float()
    b = torch.zeros_like(h)
    y = layer.residual_norm(h, b, w, c)
    assert torch.equal(y[1], c) and torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
    ref = layer.residual_norm(h[[0, 4]], b[:2], w, c)
    assert torch.equal(y[[0, 4]], ref)
    e = torch.zeros(0, D, device="cuda:0", requires_grad=True)
    wl = w.clone().requires_grad_(True)
    gate = torch.ones(D, device="cuda:0", requires_grad=True)
    y = layer.residual_norm(e, e * 1, wl, c, gate=gate)
    assert y.shape == (0, D)
    ge, gw, gg = torch.autograd.grad(y.sum(), (e, wl, gate))
    assert ge.shape == (0, D) and (gw == 0).all() and (gg == 0).all()
    # a zero gate removes the branch, whatever finite value it holds
    y0 = layer.residual_norm(h[:1], 1e30 * torch.randn_like(h[:1]), w, c, gate=torch.zeros(D, device="cuda:0"))
    assert torch.equal(y0, layer.residual_norm(h[:1], b[:1], w, c))


@pytest.mark.parametrize("lead,gate", [((4, 0), (4, 1)), ((0, 5), (1, 1)), ((0, 5), (0, 1)), ((4, 0), (4, 0)), ((0, 0), (1,))])
def test_empty_batches_and_sequences(lead, gate):
    """No rows: empty results, and gradients of zero for whatever is shared by rows."""
    import torch
    from paper_1911_04070_b200 import layer
    D = 72
    t = lambda *s: torch.ones(*s, D, device="cuda:0", requires_grad=True)
    v = dict(h=t(*lead), b=t(*lead), weight=t(), bias=t(), post_weight=t(), gate=t(*gate))
    r, y = layer.residual_norm(**v, norm="layer", post_norm="rms", return_sum=True)
    assert r.shape == y.shape == (*lead, D)
    for a, g in zip(v.values(), torch.autograd.grad((r.sum() + y.sum()), list(v.values()))):
        assert g.shape == a.shape and (g == 0).all()


def test_results_do_not_depend_on_alignment_or_neighbours():
    """Views that are contiguous but not 16-byte aligned, results in place of the inputs, and the memory around the rows."""
    import torch
    from paper_1911_04070_b200 import binding
    D, R = 96, 20
    big = torch.full((3, R * D + 64), 7.0, dtype=torch.bfloat16, device="cuda:0")
    src = torch.randn(2, R, D, device="cuda:0").bfloat16()
    h, b = (big[i, 1:1 + R * D].view(R, D) for i in range(2))
    h.copy_(src[0]); b.copy_(src[1])
    want_y, want_r = binding.bpt_res_norm_fwd(src[0], src[1], norm="rms", post_norm="layer", want_sum=True)
    out = big[2, 1:1 + R * D].view(R, D)
    y, r = binding.bpt_res_norm_fwd(h, b, norm="rms", post_norm="layer", want_sum=True, y=out)
    tol = 2 * 2.0 ** -8 * want_y.float().abs().max()      # two groupings of one fp32 sum may round to neighbouring bf16 values
    assert (y.float() - want_y.float()).abs().max() <= tol and (r.float() - want_r.float()).abs().max() <= 2 * 2.0 ** -8 * want_r.float().abs().max()
    assert (big[2, :1] == 7).all() and (big[2, 1 + R * D:] == 7).all()
    hc, bc = src[0].clone(), src[1].clone()
    y, r = binding.bpt_res_norm_fwd(hc, bc, norm="rms", post_norm="layer", want_sum=True, y=bc, r=hc)
    assert torch.equal(bc, want_y) and torch.equal(hc, want_r)


def test_reproducible_captured_and_on_another_stream():
    import torch
    from paper_1911_04070_b200 import layer
    x, up, cfg = _case((5, 211), 512, "bf16", "layer", "layer", (5, 1, 512), 0.5, "f32", 6)
    leaf = {a: v.requires_grad_(True) for a, v in x.items()}

    def step():
        r, y = layer.residual_norm(**leaf, **cfg, return_sum=True)
        grads = torch.autograd.grad((y, r), list(leaf.values()), (up["dy"], up["dr"]))
        return [y.detach(), r.detach()] + list(grads)      # no graph of the leaves outlives a step, nor reaches the capture

    want = [t.clone() for t in step()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = step()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(2):
        for t in got:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


def test_offsets_past_32_bits():
    """More than 2^31 elements: the last rows are what a small call makes of them."""
    import torch
    from paper_1911_04070_b200 import binding
    rows, D = 270_001, 8192
    g = torch.Generator(device="cuda:0").manual_seed(0)
    h = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda:0").normal_(generator=g)
    b = torch.empty_like(h).normal_(generator=g)
    w = torch.rand(D, device="cuda:0")
    stats = torch.empty(rows, 4, device="cuda:0")
    kw = dict(weight=w, norm="rms", post_norm="layer", gate=w)
    y, r = binding.bpt_res_norm_fwd(h, b, want_sum=True, stats=stats, **kw)
    tail = slice(rows - 5, rows)
    ht, bt, st = h[tail].clone(), b[tail].clone(), torch.empty(5, 4, device="cuda:0")
    yt, rt = binding.bpt_res_norm_fwd(ht, bt, want_sum=True, stats=st, **kw)
    assert torch.equal(y[tail], yt) and torch.equal(r[tail], rt) and torch.equal(stats[tail], st)
    dh, db, *_ = binding.bpt_res_norm_bwd(h, b, y, None, stats, need=(True, True) + (False,) * 5, **kw)
    dht, dbt, *_ = binding.bpt_res_norm_bwd(ht, bt, yt, None, st, need=(True, True) + (False,) * 5, **kw)
    assert torch.equal(dh[tail], dht) and torch.equal(db[tail], dbt)


def test_two_streams_at_once():
    import torch
    from paper_1911_04070_b200 import layer
    sets = [_case((3, 700), 512, "bf16", "layer", "layer", (3, 1, 512), 0.5, "f32", 30 + i) for i in range(2)]
    leaves = [{a: v.requires_grad_(True) for a, v in x.items()} for x, _, _ in sets]

    def step(i):
        r, y = layer.residual_norm(**leaves[i], **sets[i][2], return_sum=True)
        grads = torch.autograd.grad((y, r), list(leaves[i].values()), (sets[i][1]["dy"], sets[i][1]["dr"]))
        return [y.detach(), r.detach()] + list(grads)

    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(8):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(step(i))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for res in got[i] for a, b in zip(res, want[i]))


def test_strided_inputs_and_gradients_reach_the_same_result():
    import torch
    from paper_1911_04070_b200 import layer
    h = torch.randn(64, 30, device="cuda:0").t().requires_grad_(True)           # column-major
    b = torch.randn(30, 128, device="cuda:0")[:, ::2].requires_grad_(True)
    w = torch.randn(64, device="cuda:0", requires_grad=True)
    y = layer.residual_norm(h, b, w)
    g = torch.autograd.grad(y.sum(), (h, b, w))                                 # an expanded upstream gradient
    hc, bc = (t.detach().contiguous().requires_grad_(True) for t in (h, b))
    yc = layer.residual_norm(hc, bc, w)
    gc = torch.autograd.grad(yc, (hc, bc, w), torch.ones_like(yc))
    assert torch.equal(y, yc) and all(torch.equal(a, c) for a, c in zip(g, gc))


def test_double_backward_is_refused():
    import torch
    from paper_1911_04070_b200 import layer
    h = torch.randn(4, 16, device="cuda:0", requires_grad=True)
    g, = torch.autograd.grad(layer.residual_norm(h, h.detach()).sum(), h, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_python_refusals():
    import torch
    from paper_1911_04070_b200 import binding
    f = binding.bpt_res_norm_fwd
    h = torch.zeros(4, 32, device="cuda:0")
    w = torch.zeros(32, device="cuda:0")
    for kw in (dict(b=h[:2]), dict(b=h.bfloat16()), dict(b=h.t()), dict(b=h.cpu()), dict(norm="batch"), dict(weight=w[:16]),
               dict(weight=w, bias=w.bfloat16()), dict(norm=None, weight=w), dict(post_weight=w, b=h), dict(gate=w), dict(b=h, gate=h[:2]),
               dict(b=h, gate=torch.zeros(1, 1, 32, device="cuda:0")), dict(b=h, gate=torch.zeros(4, 1, device="cuda:0")), dict(post_norm="rms"),
               dict(y=h[:2]), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            f(h, **kw)
    with pytest.raises(ValueError):
        f(h.t())
    with pytest.raises(TypeError):
        f(h.half())
    with pytest.raises(binding.BptError) as ei:
        f(torch.zeros(2, 8200, device="cuda:0"))
    assert ei.value.status == 2
    with pytest.raises(binding.BptError) as ei:
        binding.bpt_res_norm_bwd(h, h, h, None, torch.zeros(4, 4, device="cuda:0"), workspace=torch.empty(16, dtype=torch.uint8, device="cuda:0"))
    assert ei.value.status == 3
    with pytest.raises(ValueError):
        binding.bpt_res_norm_bwd(h, h, h, None, torch.zeros(4, 3, device="cuda:0"))
    with pytest.raises(binding.BptError) as ei:
        binding.bpt_res_norm_bwd(h, h, h, None, None)
    assert ei.value.status == 1


def test_layer_function_refuses_like_the_binding():
    import torch
    from paper_1911_04070_b200 import binding, layer
    h = torch.zeros(4, 32, device="cuda:0", requires_grad=True)
    w = torch.zeros(32, device="cuda:0")
    for kw in (dict(b=h[:2]), dict(b=h.bfloat16()), dict(norm="batch"), dict(post_norm="batch", b=h), dict(weight=w[:16]), dict(weight=w, bias=w.bfloat16()),
               dict(norm=None, weight=w), dict(gate=w), dict(b=h, gate=h[:2]), dict(post_norm="rms"), dict(weight=w.cpu())):
        with pytest.raises(ValueError):
            layer.residual_norm(h, **kw)
    with pytest.raises(ValueError):
        layer.residual_norm(h.cpu(), h.cpu())
    with pytest.raises(TypeError):
        layer.residual_norm(h.half())
    with pytest.raises(binding.BptError) as ei:
        layer.residual_norm(torch.zeros(2, 8200, device="cuda:0"))
    assert ei.value.status == 2


def test_gradients_only_where_asked_for():
    import torch
    from paper_1911_04070_b200 import layer
    x, up, cfg = _case((6, 50), 96, "f32", "layer", "layer", (6, 1, 96), 0.5, "f32", 40)
    full = {a: v.clone().requires_grad_(True) for a, v in x.items()}
    r, y = layer.residual_norm(**full, **cfg, return_sum=True)
    want = dict(zip(full, torch.autograd.grad((y, r), list(full.values()), (up["dy"], up["dr"]))))
    for some in (("h",), ("gate",), ("weight", "post_bias"), ("b", "bias")):
        leaf = {a: v.clone().requires_grad_(a in some) for a, v in x.items()}
        r, y = layer.residual_norm(**leaf, **cfg, return_sum=True)
        torch.autograd.backward((y, r), (up["dy"], up["dr"]))
        for a in x:
            assert (leaf[a].grad is None) == (a not in some)
            assert a not in some or torch.equal(leaf[a].grad, want[a])
    # a graph kept for a second pass gives the same gradients again
    r, y = layer.residual_norm(**full, **cfg, return_sum=True)
    for _ in range(2):
        got = torch.autograd.grad((y, r), list(full.values()), (up["dy"], up["dr"]), retain_graph=True)
        assert all(torch.equal(a, b) for a, b in zip(got, want.values()))
