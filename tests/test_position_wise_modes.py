"""The position-wise functions of layer.py under PyTorch's other modes of differentiation: refused before anything is computed,
with or without arguments that require a gradient.  No GPU needed: the refusal comes before the look at the device."""
import pytest
import torch
from torch.autograd import forward_ad

DEVICES = ["cpu", pytest.param("cuda:0", marks=pytest.mark.gpu)]
NORM = ("h", "b", "weight", "bias", "post_weight", "post_bias", "gate")
BLOCK = ("x", "w_gate", "w_up", "w_down")


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import build, layer
    build.build()
    return layer


def _norm(device):
    r = lambda *s: torch.randn(*s, device=device)
    return dict(h=r(5, 16), b=r(5, 16), weight=r(16), bias=r(16), post_weight=r(16), post_bias=r(16), gate=r(16), post_norm="layer")


def _block(device):
    r = lambda *s: torch.randn(*s, device=device).bfloat16()
    return dict(x=r(5, 16), w_gate=r(24, 16), w_up=r(24, 16), w_down=r(16, 24))


@pytest.mark.parametrize("device", DEVICES)
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("name", NORM + BLOCK)
def test_forward_mode_is_refused(layer, name, grad, device):
    v, call = (_norm(device), layer.residual_norm) if name in NORM else (_block(device), layer.gated_feed_forward)
    if grad:
        other = next(a for a in v if a != name)
        v[other].requires_grad_(True)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(v[name], torch.ones_like(v[name]))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            call(**{**v, name: dual})
        with pytest.raises(NotImplementedError, match="forward-mode"), torch.no_grad():
            call(**{**v, name: dual})


@pytest.mark.gpu
@pytest.mark.parametrize("name", BLOCK)
def test_forward_mode_is_refused_while_the_status_is_looked_at(layer, name, monkeypatch):
    from paper_1911_04070_b200 import binding
    v = _block("cuda:0")
    monkeypatch.setattr(binding, "CHECK_DEVICE_STATUS", True)
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(v[name], torch.ones_like(v[name]))
        with pytest.raises(RuntimeError), torch.no_grad():
            layer.gated_feed_forward(**{**v, name: dual})


@pytest.mark.gpu
@pytest.mark.parametrize("check", [False, True])
def test_forward_mode_over_the_backward_pass_is_refused(layer, check, monkeypatch):
    from paper_1911_04070_b200 import binding
    monkeypatch.setattr(binding, "CHECK_DEVICE_STATUS", check)
    for v, call in ((_norm("cuda:0"), layer.residual_norm), (_block("cuda:0"), layer.gated_feed_forward)):
        first = next(iter(v.values())).requires_grad_(True)
        with forward_ad.dual_level():
            y = call(**v)
            up = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
            with pytest.raises(NotImplementedError, match="forward-mode"):
                torch.autograd.grad(y, first, up)


@pytest.mark.parametrize("device", DEVICES)
@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("check", [False, True])
def test_tracing_is_refused(layer, grad, device, check, monkeypatch):
    """A trace would hold the allocation of the result and nothing that writes it."""
    from paper_1911_04070_b200 import binding
    monkeypatch.setattr(binding, "CHECK_DEVICE_STATUS", check)
    for v, call in ((_norm(device), layer.residual_norm), (_block(device), layer.gated_feed_forward)):
        first = next(iter(v))
        example = v.pop(first).requires_grad_(grad)
        with pytest.raises(NotImplementedError, match="traced"):
            torch.jit.trace(lambda t: call(**{first: t}, **v), example, check_trace=False)


@pytest.mark.parametrize("name", ["alpha", "eps"])
def test_a_learned_constant_is_refused(layer, name):
    """alpha and eps are numbers: a tensor's gradient or tangent would be lost."""
    v = _norm("cpu")
    with pytest.raises(NotImplementedError, match=name):
        layer.residual_norm(**v, **{name: torch.tensor(0.5, requires_grad=True)})
    with forward_ad.dual_level(), pytest.raises(NotImplementedError, match=name):
        layer.residual_norm(**v, **{name: forward_ad.make_dual(torch.tensor(0.5), torch.tensor(1.0))})


@pytest.mark.gpu
def test_a_constant_given_as_a_tensor_counts_as_its_value(layer):
    v = _norm("cuda:0")
    want = layer.residual_norm(**v, alpha=0.5, eps=0.25)
    assert torch.equal(want, layer.residual_norm(**v, alpha=torch.tensor(0.5), eps=torch.tensor(0.25, device="cuda:0")))
    with torch.no_grad():
        assert torch.equal(want, layer.residual_norm(**v, alpha=torch.tensor(0.5, requires_grad=True), eps=0.25))
    assert torch.equal(layer.residual_norm(**v, alpha=2), layer.residual_norm(**v, alpha=2.0))
