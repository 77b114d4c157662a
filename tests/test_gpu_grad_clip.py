"""layer.gradient_norm and layer.clip_gradients on the GPU against plain float64.

Bounds, u = 2^-24.  Norm: 8 squares are added in fp32 (8 u), the rest in fp64; the root halves that, and one rounding: 5 u.  Results: the
factor from that norm by an addition and a division (7 u), the product (1 u), and the rounding to bf16 where that is the type."""
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
INF = float("inf")
U = 2.0 ** -24


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


def _norm64(tensors, kind):
    flat = torch.cat([t.detach().double().reshape(-1) for t in tensors if t is not None])
    return float(flat.abs().max() if kind == INF else flat.square().sum().sqrt())


def _rnd(*shape, dtype=F32, std=1.0, seed=[0]):
    seed[0] += 1
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed[0])) * std).to("cuda", dtype)


def _check(layer, grads, most, kind=2.0, out=None, eps=1e-6):
    before = [None if g is None else g.clone() for g in grads]
    n64 = _norm64(before, kind)
    c = min(1.0, most / (n64 + eps))
    assert abs(float(layer.gradient_norm(grads, kind)) - n64) <= 5 * U * n64
    norm = layer.clip_gradients(grads, most, norm_type=kind, eps=eps, out=out)
    assert norm.shape == () and norm.dtype == F32 and abs(float(norm) - n64) <= 5 * U * n64
    for i, b in enumerate(before):
        if b is None:
            continue
        got = grads[i] if out is None else out[i]
        want = b.double() * c
        # where c = 1 and nothing is rounded the values are those that were there
        tol = (0 if c == 1 else 8 * U) + (torch.finfo(BF16).eps / 2 if got.dtype == BF16 and (c != 1 or b.dtype == F32) else 0)
        off = (got.double() - want).abs()
        assert bool((off <= tol * (1 + 2.0 ** -6) * want.abs() + 2.0 ** -126).all()), (i, float(off.max()))
        if out is not None:
            assert torch.equal(grads[i], b)
    return norm


SHAPES = [[(1,)], [(7,), (2048,), (2049,)], [(3, 5), (0,), (100, 33), (8,)], [(4096, 300)], [(64, 64)] * 23 + [(513,)], [(17,)] * 130,
          [(5, 7)] * 1000, [(3,)] * 1921 + [(70000,)]]


@pytest.mark.parametrize("shapes", SHAPES, ids=[str(len(s)) + "x" + str(s[-1]) for s in SHAPES])
@pytest.mark.parametrize("kind", [2.0, INF])
@pytest.mark.parametrize("most", [0.5, 1e9])
def test_sizes(layer, shapes, kind, most):
    grads = [_rnd(*s, dtype=BF16 if i % 3 == 1 else F32) for i, s in enumerate(shapes)]
    _check(layer, grads, most, kind)


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("ot", [F32, BF16])
@pytest.mark.parametrize("most", [0.5, 1e9])
def test_into_other_tensors(layer, gt, ot, most):
    grads = [_rnd(33, 65, dtype=gt), None, _rnd(9000, dtype=gt)]
    out = [torch.full(g.shape, 7.0, device="cuda", dtype=ot) if g is not None else None for g in grads]
    _check(layer, grads, most, out=out)
    if gt == ot:
        _check(layer, grads, most / 4, out=None)
        alias = [g for g in grads if g is not None]
        want = [g.clone() for g in alias]
        layer.clip_gradients(alias, 1e9, out=alias)                     # the gradients themselves as results
        assert all(torch.equal(a, b) for a, b in zip(alias, want))


# starts off 16-byte boundaries, in the same place and in another one than the result's; what stands beside the views stays as it was
@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("first", range(0, 9))
@pytest.mark.parametrize("n", [1, 6, 15, 2048, 5003])
def test_any_start(layer, gt, first, n):
    buf = _rnd(first + n + 5, dtype=gt)
    keep = buf.clone()
    _check(layer, [buf[first:first + n]], 1e-3)
    assert torch.equal(buf[:first], keep[:first]) and torch.equal(buf[first + n:], keep[first + n:])
    src = _rnd(first + n, dtype=gt)[first:]
    for other in (0, 3, first):
        into = torch.full((other + n + 3,), 9.0, device="cuda", dtype=BF16 if first % 2 else F32)
        _check(layer, [src], 1e-3, out=[into[other:other + n]])
        assert bool((into[:other] == 9).all()) and bool((into[other + n:] == 9).all())


def test_strides(layer):
    big = _rnd(40, 96, dtype=BF16)
    keep = big.clone()
    views = [big[:, :32], big[:, 32:64], _rnd(7, 9).t(), _rnd(2, 8, 3).permute(2, 0, 1)]
    _check(layer, views, 0.1)
    assert torch.equal(big[:, 64:], keep[:, 64:]) and not torch.equal(big[:, :64], keep[:, :64])
    grads = [_rnd(12, 10).t(), _rnd(6, 4), _rnd(12, 10)[:, ::2], _rnd(5, 6).t()]
    out = [torch.empty(10, 12, device="cuda"), _rnd(4, 6).t(), torch.empty(12, 10, device="cuda")[:, 1::2], torch.empty(5, 6, device="cuda").t()]
    _check(layer, grads, 0.1, out=out)
    row = _rnd(1, 50).expand(4, 50)
    assert abs(float(layer.gradient_norm([row])) - _norm64([row], 2.0)) <= 5 * U * _norm64([row], 2.0)
    for bad in ([row], [big[:, :32], big[:, :32]], [row.contiguous()] * 2, [views[2], views[2].t()]):
        with pytest.raises(ValueError, match="overlaps"):
            layer.clip_gradients(bad, 0.1)
    with pytest.raises(ValueError, match="overlaps"):
        layer.clip_gradients([_rnd(40, 32), _rnd(40, 32)], 0.1, out=[big[:, :32], big[:, :32]])


def test_parameters_are_not_taken_for_gradients(layer):
    p = torch.nn.Parameter(_rnd(5))
    keep = p.detach().clone()
    for call in (lambda: layer.clip_gradients([p], 0.1), lambda: layer.clip_gradients(p, 0.1), lambda: layer.clip_gradients([_rnd(5)], 0.1, out=[p])):
        with pytest.raises(ValueError, match="not the parameters"):
            call()
    assert torch.equal(p, keep) and abs(float(layer.gradient_norm([p])) - _norm64([p], 2.0)) <= 5 * U * _norm64([p], 2.0)
    g, = torch.autograd.grad((p ** 3).sum(), [p], create_graph=True)        # not a leaf
    layer.clip_gradients([g], 0.1)
    assert abs(_norm64([g], 2.0) - 0.1) < 1e-6


@pytest.mark.parametrize("std", [1e-42, 1e-30, 1e-22, 1e-12, 1e12, 1e19, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_any_size_of_values(layer, std, dtype):
    g = (torch.randn(20000, generator=torch.Generator().manual_seed(1)).double() * std).to(dtype).to("cuda")
    n64 = _norm64([g], 2.0)
    # a norm below 2^-126 is rounded to a step of 2^-149
    assert abs(float(layer.gradient_norm([g])) - n64) <= 5 * U * n64 + 2.0 ** -149
    mixed = [g, torch.zeros(3000, device="cuda"), torch.full((2,), std * 100, device="cuda")]
    n64 = _norm64(mixed, 2.0)
    assert abs(float(layer.gradient_norm(mixed)) - n64) <= 5 * U * n64 + 2.0 ** -149


@pytest.mark.parametrize("kind", [2.0, INF])
def test_nothing_is_hidden(layer, kind):
    for bad in (float("nan"), INF, -INF):
        g = [_rnd(3000), _rnd(70, dtype=BF16)]
        g[0][1234] = bad
        norm = layer.clip_gradients(g, 1.0, norm_type=kind)
        want = [torch.full_like(t, float("nan")) if bad != bad else t for t in g]
        if bad != bad:
            assert bool(norm.isnan()) and all(bool(t.isnan().all()) for t in g)
        else:       # c = 0: what was finite is 0, infinity times 0 is NaN
            assert float(norm) == INF and bool(g[0][1234].isnan()) and int(g[0].count_nonzero()) == 1 and not g[1].any()
        del want


def test_limits(layer):
    g = [_rnd(100)]
    keep = g[0].clone()
    assert float(layer.clip_gradients(g, INF)) > 0 and torch.equal(g[0], keep)
    layer.clip_gradients(g, 0.0)
    assert not g[0].any()
    assert float(layer.clip_gradients(g, 0.0, eps=0.0)) == 0 and bool(g[0].isnan().all())      # 0 / 0, as the formula says
    for empty in ([], [None, None], [torch.empty(0, device="cuda")], ()):
        norm = layer.clip_gradients(empty, 1.0)
        assert norm.shape == () and norm.is_cuda and float(norm) == 0 and float(layer.gradient_norm(empty)) == 0
    one = _rnd(50, 3)
    n64 = _norm64([one], 2.0)
    assert abs(float(layer.clip_gradients(one, 0.5)) - n64) <= 5 * U * n64 and abs(_norm64([one], 2.0) - 0.5) < 1e-5
    with pytest.raises(ValueError):
        layer.clip_gradients([_rnd(3)], -1.0)
    with pytest.raises(ValueError):
        layer.clip_gradients([_rnd(3)], float("nan"))
    with pytest.raises(TypeError):
        layer.clip_gradients([_rnd(3).half()], 1.0)
    with pytest.raises(ValueError, match="every gradient"):
        layer.clip_gradients([_rnd(3), _rnd(3)], 1.0, out=[_rnd(3), None])


def test_the_same_twice_and_another_stream(layer):
    make = lambda: [_rnd(300, 70, seed=[5]), _rnd(5000, dtype=BF16, seed=[6])]
    a, b, c = make(), make(), make()
    na, nb = layer.clip_gradients(a, 0.3), layer.clip_gradients(b, 0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        nc = layer.clip_gradients(c, 0.3)
    torch.cuda.synchronize()
    assert torch.equal(na, nb) and torch.equal(na, nc) and all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(a, b, c))


def test_a_graph_that_saved_a_tensor_notices(layer):
    x = torch.ones(4, device="cuda", requires_grad=True)
    g = _rnd(4)
    y = (x * g).sum()
    layer.clip_gradients([g], 0.1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


_CAPTURE = r"""
import torch
from paper_1911_04070_b200 import layer
grads = [torch.randn(300, 200, device="cuda"), torch.randn(999, device="cuda").bfloat16()]
out = [torch.empty(g.shape, device="cuda") for g in grads]
step = lambda: layer.clip_gradients(grads, 0.7, out=out)
side = torch.cuda.Stream()
with torch.cuda.stream(side):
    step()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    norm = step()
for g in grads:
    g.normal_()
graph.replay()
got = [norm.clone()] + [o.clone() for o in out]
assert torch.equal(step(), got[0]) and all(torch.equal(a, b) for a, b in zip(out, got[1:]))
print("done")
"""


def test_capture():
    r = subprocess.run([sys.executable, "-c", _CAPTURE], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stderr[-2000:]


def test_more_elements_than_32_bits_count(layer):
    g = torch.zeros(2 ** 32 + 5, dtype=BF16, device="cuda")
    g[-1], g[0], g[2 ** 31 + 1] = 3, 4, 12
    assert float(layer.clip_gradients([g], 6.5, eps=0.0)) == 13
    assert float(g[-1]) == 1.5 and float(g[0]) == 2 and float(g[2 ** 31 + 1]) == 6 and int(torch.count_nonzero(g)) == 3
