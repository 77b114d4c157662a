"""layer.clip_gradients where the norm or the factor leaves float32's normal numbers: finite gradients stay what the formula makes of them.

Bounds, u = 2^-24.  Factor from a float64 norm, rounded once or with its quotient by a power of two, and a product that is exact in its first step: 4 u at
most with the 8 squares of the norm (5 u) behind it, 9 u in all; and the rounding of the result's type.  Below 2^-126 results
come in steps of 2^-149 (bf16 2^-133), and a product of two roundings is off by one and a half of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


def _check(layer, grads, most, eps=1e-6, into=None):
    before = [g.double() for g in grads]
    out = None if into is None else [torch.empty(g.shape, device="cuda", dtype=into) for g in grads]
    n64 = float(torch.cat([b.view(-1) for b in before]).square().sum().sqrt())
    f32 = lambda v: float(torch.tensor(v, dtype=F32))
    c = min(1.0, f32(most) / (n64 + f32(eps)))
    norm = float(layer.clip_gradients(grads, most, eps=eps, out=out))
    assert norm == float("inf") if n64 > 3.403e38 else abs(norm - n64) <= 5 * U * n64 + 2.0 ** -149
    for b, got in zip(before, grads if out is None else out):
        want = b * c
        half = torch.finfo(BF16).eps / 2 if got.dtype == BF16 else 0
        least = 2.0 ** -133 if got.dtype == BF16 else 2.0 ** -149
        off = (got.double() - want).abs()
        assert bool((off <= (9 * U + half) * (1 + 2.0 ** -6) * want.abs() + 1.5 * least + 2 * 2.0 ** -149).all()), float((off / want.abs()).max())


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("into", [None, F32, BF16])
@pytest.mark.parametrize("most", [1.0, 1e38, 3e38, 1e-6, 1e-20, 1e-44, 0.0])
def test_norms_beyond_float32(layer, gt, into, most):
    g = torch.Generator().manual_seed(1)
    big = (torch.rand(5000, generator=g) * 2 - 1) * 3e38
    _check(layer, [big.to("cuda", gt), torch.full((3,), 3e38, device="cuda"), torch.randn(70, generator=g).to("cuda")], most, into=into)
    _check(layer, [torch.full((2,), 3e38, device="cuda", dtype=gt)], most, into=into)


@pytest.mark.parametrize("gt", [F32, BF16])
@pytest.mark.parametrize("std,most", [(1e30, 1e-9), (1e33, 1e-12), (1e36, 1e-30), (1e20, 1e-30), (1e36, 1e-38), (1.0, 1e-41), (1e-12, 1e-40)])
def test_factors_below_the_normal_numbers(layer, gt, std, most):
    g = (torch.randn(20000, generator=torch.Generator().manual_seed(2)).double() * std).to("cuda", gt)
    _check(layer, [g], most, eps=0.0)
    wide = torch.tensor([1e38, 1.0, 1e10, 1e-30, -1e25, 2e-38, 1e-45, 0.0], device="cuda")        # far apart in one tensor
    _check(layer, [wide.to(gt)], most, eps=0.0)


@pytest.mark.parametrize("most", [1e-40, 1e-42, 1e-45])
def test_norms_below_the_normal_numbers(layer, most):
    for g in (torch.full((9,), 1e-41), torch.tensor([1e-45, 3e-45]), torch.randn(3000, generator=torch.Generator().manual_seed(3)) * 1e-42):
        _check(layer, [g.to("cuda")], most, eps=0.0)


def test_no_limit(layer):
    for big in (1.0, 3e38):
        g = torch.full((50,), big, device="cuda")
        layer.clip_gradients([g], float("inf"))
        assert bool((g == torch.tensor(big)).all())


@pytest.mark.parametrize("kind", [2.0, float("inf")])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_no_limit_scales_nothing_whatever_the_norm(layer, kind, bad):
    g = [torch.randn(3000, generator=torch.Generator().manual_seed(4)).to("cuda"), torch.randn(70, generator=torch.Generator().manual_seed(5)).to("cuda", BF16)]
    g[0][1234] = bad
    keep = [t.clone() for t in g]
    same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    norm = layer.clip_gradients(g, float("inf"), norm_type=kind)
    assert not bool(torch.isfinite(norm)) and all(same(a, b) for a, b in zip(g, keep))
    out = [torch.empty_like(t) for t in g]
    layer.clip_gradients(g, float("inf"), norm_type=kind, out=out)
    assert all(torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0)) for a, b in zip(out, keep))
