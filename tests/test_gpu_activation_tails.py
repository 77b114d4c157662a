"""The block's activations by themselves, each held to its own bound, tails included.

Weights pick g and 1 out of x and give the inner row back, so that y is act(g) rounded once to bf16 (2^-8), and dx[:, 0] its
derivative rounded once (the products that follow multiply by ones and add zeros).  Before the rounding:
  relu: exact, also in its derivative, 0 at g = 0.
  silu: relative errors only.  The exponential's argument g log2(e) carries half a step of its product and of the constant, at most
    2 * 128 * 2^-24 for |g| < 89, hence 1.1e-5 of the value; the other operations add a few 2^-22: 2^-16 in all.  s = 1 / (1 + exp(-g))
    below 2^-126 is flushed to zero: |g| 2^-126 of y, (1 + |g|) 2^-126 of the derivative s (1 + g (1 - s)), whose two terms each
    count with 2^-16.
  gelu: 1.5e-7 / 2 of the approximation of erfc, times |g| in y; the rest relative, 2^-16 as above (the density's argument is below
    2 * 128 until it is flushed).  Relative to the tail itself, from a table of the approximation's error in 64 bits."""
import pytest

pytestmark = pytest.mark.gpu
H, R, TINY = 2.0 ** -8, 2.0 ** -16, 2.0 ** -126
CDF = 0.76e-7
TAIL = ((-4.0, 5e-4), (-5.0, 1.6e-3), (-6.0, 3.6e-3), (-8.0, 1.03e-2), (-10.0, 1.98e-2), (-12.0, 3.11e-2))


def _points():
    import torch
    g = torch.cat([torch.linspace(-40, 40, 20001), torch.linspace(-13, 0, 8001), torch.linspace(-1, 1, 4001), torch.linspace(-89, -40, 2001),
                   torch.tensor([0.0, -0.0, -2.0 ** -126, 2.0 ** -126, -88.0, 88.0, -100.0, 100.0])]).bfloat16()
    return torch.unique(g).flip(0)


def _run(act, rows):
    """(g, y, dx[:, 0]) with all points in one call, or in calls of `rows`."""
    import torch
    from paper_1911_04070_b200 import binding
    pick = lambda c: torch.zeros(8, 8, dtype=torch.bfloat16).index_fill_(1, torch.tensor([c]), 1).cuda()
    eye = torch.eye(8, dtype=torch.bfloat16).cuda()
    g = _points().cuda()
    out = []
    for part in g.split(rows or len(g)):
        x = torch.zeros(len(part), 8, dtype=torch.bfloat16, device="cuda:0")
        x[:, 0], x[:, 1] = part, 1
        one = torch.zeros_like(x)
        one[:, 3] = 1
        y = binding.bpt_gated_ff_fwd(x, pick(0), pick(1), eye, act)
        assert torch.equal(y, y[:, :1].expand_as(y))
        out.append((y[:, 0], binding.bpt_gated_ff_bwd(x, pick(0), pick(1), eye, one, act)[0][:, 0]))
    y, d = (torch.cat(t).double() for t in zip(*out))
    return g.double(), y, d


@pytest.mark.parametrize("rows", [0, 60, 300])
def test_relu_is_exact(rows):
    import torch
    z, y, d = _run("relu", rows)
    assert torch.equal(y, z.clamp(min=0)) and torch.equal(d, (z > 0).double())


@pytest.mark.parametrize("rows", [0, 60, 300])
def test_silu_to_its_tails(rows):
    import torch
    z, y, d = _run("silu", rows)
    s = 1 / (1 + torch.exp(-z))
    err = (y - z * s).abs()
    assert (err <= (H + R) * (z * s).abs() + z.abs() * TINY).all(), float((err / (z * s).abs()).nan_to_num(0).max())
    want = s + z * s * (1 - s)
    err = (d - want).abs()
    assert (err <= H * want.abs() + R * s * (1 + z.abs() * (1 - s)) + (1 + z.abs()) * TINY).all(), float(err.max())


@pytest.mark.parametrize("rows", [0, 60, 300])
def test_gelu_to_its_tails(rows):
    import math
    import torch
    z, y, d = _run("gelu", rows)
    cdf = 0.5 * torch.special.erfc(-z / math.sqrt(2))
    pdf = torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    f = z * cdf
    err = (y - f).abs()
    assert (err <= (H + R) * f.abs() + CDF * z.abs()).all(), float(err.max())
    above = 0.0
    for lo, rel in TAIL:
        here = (z < above) & (z >= lo)
        assert (err[here] <= (H + R + rel) * f[here].abs() + z[here].abs() * TINY).all(), lo
        above = lo
    want = cdf + z * pdf
    err = (d - want).abs()
    assert (err <= H * want.abs() + R * (cdf + z.abs() * pdf) + CDF + (1 + z.abs()) * TINY).all(), float(err.max())
