"""layer.token_states and its gradient on the GPU: refusals that need a device, and lists of ids laid out over the ends of what the kernels cut them
into.  Bounds as for the other tests of the gradient: n places are added in fp32 in some order, each addition off by at most 2^-24 of a
partial sum of absolute values, then the scale and the rounding: (n + 2) 2^-24 sum |d_out| + eps_t / 2 |dW|."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


@pytest.mark.parametrize("train", [False, True])
@pytest.mark.parametrize("padding", [-1, -2, -5, 5, 2 ** 40])
def test_a_padding_id_outside_the_table_is_refused(layer, padding, train):
    """-1 is not the last id, as it is elsewhere, nor none: it is refused on the device as on the host."""
    ids, w = torch.zeros(3, 4, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda", requires_grad=train)
    with pytest.raises(ValueError, match="padding_idx"):
        layer.token_states(ids, w, padding_idx=padding)


def _check(layer, ids, V, D, wt=F32, dt=F32):
    g = torch.Generator("cuda").manual_seed(ids.numel() + D)
    w, d = torch.randn(V, D, generator=g, device="cuda").to(wt).requires_grad_(True), torch.randn(*ids.shape, D, generator=g, device="cuda").to(dt)
    step = lambda: torch.autograd.grad(layer.token_states(ids, w, dtype=dt), [w], d)[0]
    dw = step()
    assert torch.equal(dw, step())
    flat, rows = ids.reshape(-1), d.reshape(-1, D).double()
    sums = lambda t: torch.zeros(V, D, dtype=torch.float64, device="cuda").index_add_(0, flat, t)
    want, mag, places = sums(rows), sums(rows.abs()), torch.bincount(flat, minlength=V)[:, None]
    off = (places + 2) * 2.0 ** -24 * mag
    bound = off + torch.finfo(wt).eps / 2 * (want.abs() + off) + torch.finfo(wt).smallest_normal * (places > 0)
    worst = ((dw.double() - want).abs() - bound).max()
    assert float(worst) <= 0, float(worst)


def _runs(total, around):
    """Lengths of runs of one id each that end one place before, at and one place behind multiples of `around`, far and near, up to `total` places."""
    ends, at = [], 0
    for i in range(1, total // around):
        for e in ((-1, 0, 1), (0,), (-1,), (1,), (), (-1, 1))[i % 6]:
            ends.append(i * around + e)
    ends = sorted(set(e for e in ends if 0 < e < total)) + [total]
    return [b - a for a, b in zip([0] + ends, ends)]


# places a warp adds up in one go: 8, 16 or 32, by how much work there is; a CTA's warps take eight times that
@pytest.mark.parametrize("total,D,around", [(9000, 8, 8), (9000, 8, 64), (20000, 8, 16), (20000, 24, 128), (40000, 8, 32), (40000, 8, 256), (40000, 201, 256),
                                            (20000, 300, 256), (40000, 13, 512), (131072, 8, 256), (131073, 8, 256), (150000, 9, 32)])
@pytest.mark.parametrize("wt", [F32, BF16])
def test_runs_that_end_around_the_ends_of_tiles(layer, total, D, around, wt):
    runs = _runs(total, around)
    ids = torch.repeat_interleave(torch.arange(len(runs)) * 2 + 1, torch.tensor(runs))      # in order, and shuffled: the sorted list is the same
    V = 2 * len(runs) + 4
    _check(layer, ids.to("cuda"), V, D, wt)
    _check(layer, ids[torch.randperm(total, generator=torch.Generator().manual_seed(5))].to("cuda"), V, D, wt)


# beyond one launch of a cluster and beyond two passes of 9 bits: three passes, the list changing places three times; and four
@pytest.mark.parametrize("total,V,D", [(131073, 262144, 8), (200001, 300000, 9), (140000, 2 ** 24, 1), (140000, 2 ** 27, 1), (150000, 262143, 8)])
def test_sorts_of_many_passes(layer, total, V, D):
    g = torch.Generator().manual_seed(V)
    ids = torch.cat([torch.randint(0, V, (total - 40000,), generator=g), torch.full((20000,), V - 1), torch.randint(V - 300, V, (20000,), generator=g)])
    ids = ids[torch.randperm(total, generator=g)].to("cuda")
    if V * D <= 2 ** 22:
        return _check(layer, ids, V, D)
    d = torch.randint(-8, 9, (total, D), generator=g).float().to("cuda")         # whole numbers: every order gives the same sum
    w = torch.zeros(V, D, device="cuda", requires_grad=True)
    dw, = torch.autograd.grad(layer.token_states(ids, w), [w], d)
    assert torch.equal(dw, torch.zeros(V, D, device="cuda").index_add_(0, ids, d))


def test_forward_mode_over_the_backward_pass_is_refused(layer):
    from torch.autograd import forward_ad
    ids, w = torch.zeros(3, 4, dtype=torch.int64, device="cuda"), torch.zeros(5, 8, device="cuda", requires_grad=True)
    with forward_ad.dual_level():
        y = layer.token_states(ids, w)
        up = forward_ad.make_dual(torch.ones_like(y), torch.ones_like(y))
        with pytest.raises(NotImplementedError, match="forward-mode"):
            torch.autograd.grad(y, w, up)
