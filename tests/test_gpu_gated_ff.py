"""bpt_gated_ff (gated feed-forward block) and its backward against the float64 oracle, over row counts, ragged widths
and activations.

Tolerances, fixed before the first run.  A result is rounded once to bf16: at most 2^-8 of its value.  Before that, the
inner row h, dG and dU are each rounded once to bf16 as operands of the next product; such a rounding is off by at most
2^-8 of the value and evenly spread, hence a standard deviation of at most 2^-8 / sqrt(3), and the terms of a product's
sum err independently: the sum's deviation is 2^-8 / sqrt(3) * sqrt(sum of squared terms).  Eight deviations, 4.7 * 2^-8 *
sqrt(sum of squared terms), hold for far more elements than are compared.  fp32 accumulation and the approximate
exponential (relative 2^-20) are far below that."""
import pytest

pytestmark = pytest.mark.gpu

H = 2.0 ** -8
SIZES = [(8, 8), (16, 24), (64, 64), (72, 200), (136, 128), (200, 712), (264, 520), (512, 1368), (512, 2048), (1024, 136), (128, 4096)]
ROWS = [1, 2, 5, 8, 9, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 511, 1023, 4099]


def _inputs(rows, D, F, seed, scale=1.0):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    r = lambda *s, std: (torch.randn(*s, generator=g, device="cuda:0") * std).bfloat16()
    return dict(x=r(rows, D, std=scale), w_gate=r(F, D, std=D ** -0.5), w_up=r(F, D, std=D ** -0.5), w_down=r(D, F, std=F ** -0.5)), r(rows, D, std=1.0)


def _close(name, got, want, squares):
    import torch
    assert got.dtype == torch.bfloat16 and got.shape == want.shape, name
    got = got.double()
    assert torch.isfinite(got).all(), name
    err = (got - want).abs()
    bad = err > H * want.abs() * (1 + 2 * H) + 4.7 * H * squares.sqrt() + 1e-30
    assert not bad.any(), "%s: %d of %d outside, worst %.3g at %s" % (name, int(bad.sum()), bad.numel(), float(err[bad].max()), bad.nonzero()[0].tolist())


def _check(v, dy, act, backward=True):
    import torch
    from oracle import bpt_layer
    from paper_1911_04070_b200 import binding, layer
    leaf = {a: t.clone().requires_grad_(backward) for a, t in v.items()}
    y = layer.gated_feed_forward(**leaf, act=act)
    d = {a: t.double().requires_grad_(True) for a, t in v.items()}
    y64 = bpt_layer.gated_ff(**d, act=act)
    g = d["x"] @ d["w_gate"].T
    u = d["x"] @ d["w_up"].T
    one = torch.ones_like(g)
    act64 = {"relu": lambda z: torch.where(z > 0, z, 0 * z), "silu": lambda z: z / (1 + torch.exp(-z)),
             "gelu": lambda z: z * 0.5 * (1 + torch.erf(z / 2 ** 0.5))}[act]
    av = act64(g)
    da, = torch.autograd.grad(av, g, one, retain_graph=True)
    h, da, av, u = ((av * u).detach(), da, av.detach(), u.detach())
    sq = lambda t: t.detach().double() ** 2
    _close("y", y.detach(), y64.detach(), sq(h) @ sq(v["w_down"]).T)
    assert binding.bpt_check(getattr(y, "_bpt_workspace", None)) == 0
    if not backward:
        return y
    grads = torch.autograd.grad(y, list(leaf.values()), dy)
    want = torch.autograd.grad(y64, list(d.values()), dy.double())
    dh = dy.double() @ v["w_down"].double()
    dg, du = dh * u * da, dh * av
    _close("dx", grads[0], want[0], sq(dg) @ sq(v["w_gate"]) + sq(du) @ sq(v["w_up"]))
    _close("dw_gate", grads[1], want[1], sq(dg).T @ sq(v["x"]))
    _close("dw_up", grads[2], want[2], sq(du).T @ sq(v["x"]))
    _close("dw_down", grads[3], want[3], sq(dy).T @ sq(h))
    return (y, *grads)


@pytest.mark.parametrize("D,F", SIZES)
@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
def test_sizes(D, F, act):
    _check(*_inputs(400, D, F, D + F), act)     # enough rows for the tensor-memory kernels at every size


@pytest.mark.parametrize("rows", ROWS)
@pytest.mark.parametrize("D,F", [(64, 136), (512, 2048)])
def test_row_counts(rows, D, F):
    _check(*_inputs(rows, D, F, rows), "silu")


@pytest.mark.parametrize("rows,D,F", [(8, 1024, 4096), (9, 1024, 4096), (32, 1024, 4096), (33, 1024, 4096), (64, 1024, 4096), (65, 64, 136), (384, 64, 136),
                                      (385, 64, 136), (128, 512, 2048), (129, 512, 2048), (300, 256, 1024), (200, 264, 520), (16, 1200, 3000), (17, 2000, 5000)])
def test_on_both_sides_of_the_few_rows_rule(rows, D, F):
    _check(*_inputs(rows, D, F, rows + F), "silu")


def test_many_tiles_per_pair():
    _check(*_inputs(20011, 256, 520, 3), "silu")


def test_a_batch_of_long_sequences():
    _check(*_inputs(65532, 512, 2048, 4), "silu")


def test_large_scores():
    """Inner values of hundreds: the activation saturates on both sides without overflow."""
    _check(*_inputs(130, 128, 256, 5, scale=300.0), "silu")
    _check(*_inputs(130, 128, 256, 6, scale=300.0), "gelu")


@pytest.mark.parametrize("rows", [1, 2, 31, 32, 33, 63, 64])
@pytest.mark.parametrize("D,F", [(8, 8), (72, 136), (512, 1368)])
def test_few_rows_round_once(rows, D, F):
    """Up to 64 rows the operands of the second products keep 16 bits (two bf16 terms, remainder 2^-17): what is left is the
    rounding of the result, 2^-8, and 8 deviations of the remainders' rounding and of fp32 sums."""
    import torch
    from oracle import bpt_layer
    from paper_1911_04070_b200 import binding
    v, dy = _inputs(rows, D, F, rows + D)
    got = (binding.bpt_gated_ff_fwd(**v, act="gelu"),) + binding.bpt_gated_ff_bwd(**v, dy=dy, act="gelu")
    d = {a: t.double().requires_grad_(True) for a, t in v.items()}
    y = bpt_layer.gated_ff(**d, act="gelu")
    want = (y.detach(),) + torch.autograd.grad(y, list(d.values()), dy.double())
    for name, a, b in zip(("y", "dx", "dw_gate", "dw_up", "dw_down"), got, want):
        err = (a.double() - b).abs()
        assert (err <= H * b.abs() * (1 + H) + 2.0 ** -13 * b.abs().max()).all(), (name, float(err.max()))


@pytest.mark.parametrize("act", ["silu", "gelu", "relu"])
@pytest.mark.parametrize("rows", [1, 8, 40000])
def test_activations_on_their_own(act, rows):
    """Weights that pick g and 1 out of x and give the inner row back: y is act(g), dx[:, 0] its derivative.  One rounding of the
    inner row (the second product and its rounding are exact), the derivative rounded once more as an operand; beside that the
    approximations: relative 2^-20, and 2e-7 absolute (1.5e-7 / 2 of the tail, fp32 roundings) for gelu, times |g|."""
    import torch
    from paper_1911_04070_b200 import binding
    g = torch.cat([torch.linspace(-40, 40, 30001), torch.linspace(-1, 1, 9997), torch.tensor([0.0, -88.0])]).double()[-rows:].bfloat16().cuda()
    n = g.numel()
    x = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda:0")
    x[:, 0], x[:, 1] = g, 1
    pick = lambda c: torch.zeros(8, 8, dtype=torch.bfloat16, device="cuda:0").index_fill_(1, torch.tensor([c], device="cuda:0"), 1)
    eye = torch.eye(8, dtype=torch.bfloat16, device="cuda:0")
    y = binding.bpt_gated_ff_fwd(x, pick(0), pick(1), eye, act)
    z = g.double().requires_grad_(True)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[act](z)
    df, = torch.autograd.grad(f.sum(), z)
    slack = 2.0 ** -20 * f.abs() + (3e-7 * z.abs() + 1e-30)
    err = (y.double() - f[:, None]).abs()
    assert (err <= (H * f.abs() + slack)[:, None]).all(), float(err.max())
    one = torch.zeros(n, 8, dtype=torch.bfloat16, device="cuda:0")
    one[:, 3] = 1
    dx, *_ = binding.bpt_gated_ff_bwd(x, pick(0), pick(1), eye, one, act)
    err = (dx[:, 0].double() - df).abs()
    assert (err <= 2 * H * df.abs() * (1 + H) + 3e-7 * (1 + z.abs())).all(), float(err.max())
    err = (dx[:, 1].double() - f).abs()
    assert (err <= 2 * H * f.abs() * (1 + H) + slack).all()


@pytest.mark.parametrize("rows", [3, 500])
def test_nan_and_infinity_stay_in_their_rows(rows):
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(rows, 72, 136, 7)
    y = layer.gated_feed_forward(**v)
    x = v["x"].clone()
    x[1, 5] = float("nan")
    x[0, 3] = float("inf")
    y2 = layer.gated_feed_forward(**{**v, "x": x})
    assert torch.isnan(y2[1]).all() and not torch.isfinite(y2[0]).all()
    assert torch.equal(y2[2:], y[2:])


def test_no_rows():
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(0, 64, 128, 8)
    leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}
    y = layer.gated_feed_forward(**leaf)
    assert y.shape == (0, 64)
    g = torch.autograd.grad(y, list(leaf.values()), dy)
    assert g[0].shape == (0, 64) and all((t == 0).all() for t in g[1:])


@pytest.mark.parametrize("rows", [1, 7, 65, 500])
def test_memory_around_the_results_is_left_alone(rows):
    import torch
    from paper_1911_04070_b200 import binding
    D, F = 72, 200
    v, dy = _inputs(rows, D, F, 9)
    guard = 1024
    bufs = {n: torch.full((t.numel() + 2 * guard,), 7.0, dtype=torch.bfloat16, device="cuda:0")
            for n, t in (("y", v["x"]), ("dx", v["x"]), ("dw_gate", v["w_gate"]), ("dw_up", v["w_up"]), ("dw_down", v["w_down"]))}
    mid = lambda n, t: bufs[n][guard:guard + t.numel()].view(t.shape)
    want = binding.bpt_gated_ff_fwd(**v)
    got = binding.bpt_gated_ff_fwd(**v, y=mid("y", v["x"]))
    assert torch.equal(got, want)
    want = binding.bpt_gated_ff_bwd(**v, dy=dy)
    got = binding.bpt_gated_ff_bwd(**v, dy=dy, dx=mid("dx", v["x"]), **{"d" + n: mid("d" + n, v[n]) for n in ("w_gate", "w_up", "w_down")})
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    for n, b in bufs.items():
        assert (b[:guard] == 7).all() and (b[-guard:] == 7).all(), n


@pytest.mark.parametrize("rows", [5, 700])
def test_reproducible_captured_and_on_another_stream(rows):
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(rows, 128, 264, 10)
    leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}

    def step():
        y = layer.gated_feed_forward(**leaf, act="gelu")
        grads = torch.autograd.grad(y, list(leaf.values()), dy)
        return [y.detach()] + list(grads)       # no graph of the leaves outlives a step, nor reaches the capture

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


def test_results_do_not_depend_on_what_the_workspace_held():
    import torch
    from paper_1911_04070_b200 import binding
    v, dy = _inputs(444, 136, 264, 11)
    want = (binding.bpt_gated_ff_fwd(**v),) + binding.bpt_gated_ff_bwd(**v, dy=dy)
    ws = [torch.full((binding.bpt_gated_ff_workspace_bytes(444, 136, 264, b),), 0xFF, dtype=torch.uint8, device="cuda:0") for b in (False, True)]
    got = (binding.bpt_gated_ff_fwd(**v, workspace=ws[0]),) + binding.bpt_gated_ff_bwd(**v, dy=dy, workspace=ws[1])
    assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("rows", [5, 500])
def test_from_a_fresh_thread(rows):
    """A thread that has made no CUDA call of its own: every buffer is there already."""
    import threading
    import torch
    from paper_1911_04070_b200 import binding
    v, dy = _inputs(rows, 64, 128, 15)
    want = (binding.bpt_gated_ff_fwd(**v),) + binding.bpt_gated_ff_bwd(**v, dy=dy)
    lib, st = binding.load_library(), torch.cuda.current_stream().cuda_stream
    got = [torch.empty_like(t) for t in want]
    ws = [torch.empty(max(256, binding.bpt_gated_ff_workspace_bytes(rows, 64, 128, b)), dtype=torch.uint8, device="cuda:0") for b in (False, True)]
    torch.cuda.synchronize()
    ptr = [t.data_ptr() for t in v.values()]
    for k, call in enumerate((lambda: lib.bpt_gated_ff_fwd(*ptr, got[0].data_ptr(), rows, 64, 128, 1, None, ws[0].data_ptr(), ws[0].numel(), st),
                              lambda: lib.bpt_gated_ff_bwd(*ptr, dy.data_ptr(), *[t.data_ptr() for t in got[1:]], rows, 64, 128, 1, None,
                                                           ws[1].data_ptr(), ws[1].numel(), st))):
        status = []
        t = threading.Thread(target=lambda: status.append(call()))
        t.start()
        t.join()
        assert status == [0]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows", [7, 200, 500, 3000])
def test_two_streams_at_once(rows):
    """Calls whose work overlaps on the GPU, each with its own workspace: the same bits as one after the other."""
    import torch
    from paper_1911_04070_b200 import binding
    sets = [_inputs(rows, 256, 520, 20 + i) for i in range(2)]
    want = [(binding.bpt_gated_ff_fwd(**v),) + binding.bpt_gated_ff_bwd(**v, dy=dy) for v, dy in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(8):
        for i, (v, dy) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                got[i].append((binding.bpt_gated_ff_fwd(**v),) + binding.bpt_gated_ff_bwd(**v, dy=dy))
    torch.cuda.synchronize()
    for i in range(2):
        for res in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(res, want[i]))


def test_offsets_past_32_bits():
    """The inner rows of the last tiles lie more than 2^32 bytes and 2^31 elements into the workspace."""
    import torch
    from paper_1911_04070_b200 import binding
    rows, D, F = 1_100_003, 64, 2048
    v, dy = _inputs(rows, D, F, 16)
    y = binding.bpt_gated_ff_fwd(**v)
    dx, *_ = binding.bpt_gated_ff_bwd(**v, dy=dy, need_dw=False)
    tail = slice(rows - 444, rows)      # more rows than the few-rows kernels take: the same kernels on both sides
    assert not binding.load_library().bpt_gated_ff_few_rows(444, D, F)
    vt, dyt = {**v, "x": v["x"][tail].contiguous()}, dy[tail].contiguous()
    yt, dxt = binding.bpt_gated_ff_fwd(**vt), binding.bpt_gated_ff_bwd(**vt, dy=dyt, need_dw=False)[0]
    # the same rows in a small call: equal but for the order of fp32 sums, i.e. one step of bf16 where a rounding border is crossed
    for a, b in ((y[tail], yt), (dx[tail], dxt)):
        assert torch.isfinite(a).all()
        assert ((a.double() - b.double()).abs() <= 2 * H * b.double().abs() + 1e-4 * float(b.double().abs().max())).all()


def test_device_status_is_looked_at_when_asked(monkeypatch):
    import torch
    from paper_1911_04070_b200 import binding, layer
    for rows in (5, 500):
        v, dy = _inputs(rows, 64, 128, 17)
        leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}
        monkeypatch.setattr(binding, "CHECK_DEVICE_STATUS", True)
        layer.gated_feed_forward(**v)
        y = layer.gated_feed_forward(**leaf)
        y.backward(dy)
        y = layer.gated_feed_forward(**leaf)
        monkeypatch.setattr(binding, "bpt_check", lambda ws: 5)
        with pytest.raises(RuntimeError, match="timed out"):
            layer.gated_feed_forward(**v)
        with pytest.raises(RuntimeError, match="timed out"):
            layer.gated_feed_forward(**leaf)
        with pytest.raises(RuntimeError, match="timed out"):
            y.backward(dy)
        monkeypatch.undo()


def test_only_some_gradients():
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(200, 64, 128, 12)
    full = {a: t.clone().requires_grad_(True) for a, t in v.items()}
    want = dict(zip(v, torch.autograd.grad(layer.gated_feed_forward(**full), list(full.values()), dy)))
    for some in (("x",), ("w_up",), ("w_gate", "w_down"), ("x", "w_down")):
        leaf = {a: t.clone().requires_grad_(a in some) for a, t in v.items()}
        layer.gated_feed_forward(**leaf).backward(dy)
        for a in v:
            assert (leaf[a].grad is None) == (a not in some)
            assert a not in some or torch.equal(leaf[a].grad, want[a])


def test_strided_inputs():
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(60, 64, 128, 13)
    x = torch.empty(60, 2, 64, dtype=torch.bfloat16, device="cuda:0")[:, 0].copy_(v["x"])
    y = layer.gated_feed_forward(x, v["w_gate"].t().contiguous().t(), v["w_up"], v["w_down"])
    assert torch.equal(y, layer.gated_feed_forward(**v))
    y3 = layer.gated_feed_forward(v["x"].view(5, 12, 64), v["w_gate"], v["w_up"], v["w_down"])
    assert torch.equal(y3.view(60, 64), y)


def test_python_refusals():
    import torch
    from paper_1911_04070_b200 import binding
    v, dy = _inputs(8, 64, 128, 14)
    f = binding.bpt_gated_ff_fwd
    for kw in (dict(act="tanh"), dict(w_gate=v["w_gate"][:64]), dict(w_up=v["w_up"].t()), dict(w_down=v["w_gate"]), dict(w_down=v["w_down"].float()),
               dict(x=v["x"].t()), dict(x=v["x"].cpu()), dict(y=dy[:4]), dict(w_gate=v["w_gate"].cpu())):
        with pytest.raises(ValueError):
            f(**{**v, **kw})
    with pytest.raises(TypeError):
        f(**{a: t.float() for a, t in v.items()})
    with pytest.raises(binding.BptError) as ei:     # 12 is no multiple of 8
        f(*(t.contiguous() for t in (v["x"][:, :12], v["w_gate"][:, :12], v["w_up"][:, :12], v["w_down"][:12])))
    assert ei.value.status == 2
    with pytest.raises(ValueError):
        binding.bpt_gated_ff_bwd(**v, dy=dy, need_dx=False, need_dw=False)
    with pytest.raises(binding.BptError) as ei:
        f(**v, workspace=torch.empty(256, dtype=torch.uint8, device="cuda:0"))
    assert ei.value.status == 3


def test_layer_function_refuses_like_the_binding():
    import torch
    from paper_1911_04070_b200 import binding, layer
    v, dy = _inputs(8, 64, 128, 18)
    f = layer.gated_feed_forward
    for kw in (dict(act="tanh"), dict(w_gate=v["w_gate"][:64]), dict(w_down=v["w_gate"]), dict(w_down=v["w_down"].float()), dict(x=v["x"].cpu()),
               dict(w_up=v["w_up"].cpu())):
        with pytest.raises(ValueError):
            f(**{**v, **kw})
    with pytest.raises(TypeError):
        f(**{a: t.float() for a, t in v.items()})
    with pytest.raises(binding.BptError) as ei:
        f(v["x"][:, :12], v["w_gate"][:, :12], v["w_up"][:, :12], v["w_down"][:12])
    assert ei.value.status == 2


def test_double_backward_is_refused():
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(8, 64, 128, 19)
    x = v["x"].requires_grad_(True)
    g, = torch.autograd.grad(layer.gated_feed_forward(**v).float().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.float().sum().backward()
