"""layer.clip_gradients where what is written shares memory with something else of the call, in views that the call computes in copies: refused,
and nothing written.  Views that only interleave are taken."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


def _rnd(*shape, seed=[0]):
    seed[0] += 1
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed[0])).to("cuda")


def _refused(layer, grads, out=None, memory=()):
    keep = [t.clone() for t in memory]
    with pytest.raises(ValueError, match="overlaps"):
        layer.clip_gradients(grads, 0.1, out=out)
    assert all(torch.equal(a, b) for a, b in zip(memory, keep))


def test_shifted_views_as_results(layer):
    big = _rnd(40, 96)
    _refused(layer, [_rnd(40, 32), _rnd(40, 32)], [big[:, :32], big[:, 16:48]], [big])
    _refused(layer, [_rnd(40, 32), _rnd(39, 32)], [big[:, :32], big[1:, 31:63]], [big])


def test_a_strided_result_over_a_dense_one_or_a_gradient(layer):
    big = _rnd(40, 96)
    _refused(layer, [_rnd(40, 96), _rnd(40, 32)], [big, big[:, 5:37]], [big])
    _refused(layer, [big, _rnd(40, 32)], [torch.empty_like(big), big[:, 5:37]], [big])
    _refused(layer, [big[:, :40], _rnd(40, 32)], [torch.empty(40, 40, device="cuda"), big[:, 5:37]], [big])
    # a dense result over a gradient that is read from a copy
    _refused(layer, [big[:, :40], _rnd(5, 96)], [torch.empty(40, 40, device="cuda"), big[7:12]], [big])


def test_in_place_a_tensor_and_a_view_of_it(layer):
    big = _rnd(40, 96)
    for views in ([big, big[:, ::2]], [big[:, ::2], big], [big[:, :50], big[:, 49:]], [big[::3], big[:, ::5]], [big.view(-1).as_strided((50, 60), (59, 1))],
                  [big.view(-1).as_strided((3, 4, 5), (4, 4, 1))]):
        _refused(layer, views, None, [big])
    # read only: counted as often as it is given
    n64 = float(torch.cat([big.double().view(-1), big[:, ::2].double().reshape(-1)]).norm())
    assert abs(float(layer.gradient_norm([big, big[:, ::2]])) - n64) <= 5 * U * n64


@pytest.mark.parametrize("cut", [lambda t: (t[:, ::2], t[:, 1::2]), lambda t: t.view(40, 3, 4, 8).unbind(1), lambda t: (t[:20, :50], t[20:, 40:], t[:20, 50:]),
                                 lambda t: (t[::2].t(), t[1::2].t())])
def test_views_that_interleave(layer, cut):
    big = _rnd(40, 96)
    keep = big.clone()
    views = cut(big)
    n64 = float(torch.cat([v.double().reshape(-1) for v in views]).norm())
    norm = layer.clip_gradients(views, 0.1)
    assert abs(float(norm) - n64) <= 5 * U * n64
    want = keep.double()
    for v in cut(want):
        v.mul_(0.1 / (n64 + 1e-6))
    # as in place on tensors of their own: norm, factor and product 8 roundings
    changed = torch.zeros_like(big, dtype=torch.bool)
    for v in cut(changed):
        v.fill_(True)
    off = (big.double() - want).abs()
    assert bool((off <= 8 * U * (1 + 2.0 ** -6) * want.abs())[changed].all()) and torch.equal(big[~changed], keep[~changed])
    src = [_rnd(*v.shape) for v in views]
    layer.clip_gradients(src, 1e9, out=views)
    assert all(torch.equal(a, b) for a, b in zip(src, views))
