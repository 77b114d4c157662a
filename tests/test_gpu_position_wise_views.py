"""The gated feed-forward block on tensors that are contiguous but start off a 16-byte boundary, as views into flat buffers do and
as the backward of a concatenation hands gradients down: the same bits as from copies of their own."""
import pytest

pytestmark = pytest.mark.gpu
NAMES = ("x", "w_gate", "w_up", "w_down")


def _inputs(rows, D=64, F=136, seed=0):
    import torch
    g = torch.Generator(device="cuda:0").manual_seed(seed)
    r = lambda *s: (torch.randn(*s, generator=g, device="cuda:0") * 0.3).bfloat16()
    return dict(x=r(rows, D), w_gate=r(F, D), w_up=r(F, D), w_down=r(D, F)), r(rows, D)


def _moved(t, by):
    """A contiguous view of the same values, `by` elements into a buffer of its own."""
    import torch
    flat = torch.full((t.numel() + by + 8,), 7.0, dtype=t.dtype, device=t.device)
    v = flat[by:by + t.numel()].view(t.shape)
    v.copy_(t)
    assert v.is_contiguous() and v.data_ptr() % 16 == by * t.element_size() % 16
    return v


def _step(v, dy):
    import torch
    from paper_1911_04070_b200 import layer
    leaf = {a: t.detach().requires_grad_(True) for a, t in v.items()}
    y = layer.gated_feed_forward(**leaf, act="gelu")
    with torch.no_grad():
        assert torch.equal(layer.gated_feed_forward(**v, act="gelu"), y)
    return (y.detach(), *torch.autograd.grad(y, list(leaf.values()), dy))


@pytest.mark.parametrize("check", [False, True])
@pytest.mark.parametrize("rows", [3, 500])
@pytest.mark.parametrize("which", NAMES + ("dy", "all"))
def test_any_start_address(which, rows, check, monkeypatch):
    import torch
    from paper_1911_04070_b200 import binding
    v, dy = _inputs(rows)
    want = _step(v, dy)
    monkeypatch.setattr(binding, "CHECK_DEVICE_STATUS", check)
    for by in (1, 3, 4):
        moved = {a: _moved(t, by) if which in (a, "all") else t for a, t in v.items()}
        got = _step(moved, _moved(dy, by) if which in ("dy", "all") else dy)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("rows", [2, 300])
def test_gradient_through_a_concatenation(rows):
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(rows, seed=1)
    want = _step(v, dy)
    leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}
    y = layer.gated_feed_forward(**leaf, act="gelu")
    z = torch.cat([torch.ones(3, dtype=y.dtype, device=y.device), y.flatten()])
    z.backward(torch.cat([torch.ones(3, dtype=y.dtype, device=y.device), dy.flatten()]))
    assert all(torch.equal(a, leaf[n].grad) for n, a in zip(NAMES, want[1:]))


def test_saved_tensors_that_come_back_elsewhere():
    """Hooks that keep the saved tensors in buffers of their own and hand back views into them."""
    import torch
    from paper_1911_04070_b200 import layer
    v, dy = _inputs(300, seed=2)
    want = _step(v, dy)
    leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}
    with torch.autograd.graph.saved_tensors_hooks(lambda t: _moved(t, 5), lambda t: t):
        y = layer.gated_feed_forward(**leaf, act="gelu")
    got = torch.autograd.grad(y, list(leaf.values()), dy)
    assert all(torch.equal(a, b) for a, b in zip(want[1:], got))


def test_statistics_that_come_back_elsewhere():
    import torch
    from paper_1911_04070_b200 import layer
    h, b, w = (torch.randn(*s, device="cuda:0").requires_grad_(True) for s in ((50, 96), (50, 96), (96,)))
    up = torch.randn(50, 96, device="cuda:0")
    step = lambda: layer.residual_norm(h, b, w, post_norm="rms")
    want = torch.autograd.grad(step(), (h, b, w), up)
    with torch.autograd.graph.saved_tensors_hooks(lambda t: _moved(t, 5), lambda t: t):
        y = step()
    got = torch.autograd.grad(y, (h, b, w), up)
    for a, c in zip(want, got):        # rows off their boundary go element by element: sums in another order, fp32
        assert torch.allclose(a, c, rtol=1e-5, atol=1e-5 * float(a.abs().max()))


def test_a_gate_without_axes_is_refused_with_its_reason():
    """Also where D is 1 and a single number would fit."""
    import torch
    from paper_1911_04070_b200 import binding, layer
    h, gate = torch.randn(4, 1, device="cuda:0"), torch.ones((), device="cuda:0")
    for f in (layer.residual_norm, binding.bpt_res_norm_fwd):
        with pytest.raises(ValueError, match="gate"):
            f(h, h, gate=gate)
    assert torch.equal(layer.residual_norm(h, h, gate=gate.view(1), norm=None), 2 * h)
