"""layer.adjust_logits on the GPU against plain float64.

Bound, u = 2^-24: a setting given as a number is rounded to fp32 (1 u), and each of division or product, penalty, and three sums rounds
once: 6 u of the sum of the absolute values that enter an element; and half a step of the result's type."""
import subprocess
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


def _oracle(x, history=None, lengths=None, prompt_lengths=None, repetition=1.0, presence=0.0, frequency=0.0, bias=None, bias_ids=None, bias_values=None,
            allowed=None):
    """Element by element of the history in Python integers; returns the result and the sum of absolute values behind each element."""
    B, V = x.shape
    y, mag = x.double().cpu().clone(), torch.zeros(B, V, dtype=torch.float64)
    num = lambda v, b: float(v[b]) if isinstance(v, torch.Tensor) else float(v)
    for b in range(B):
        row = [] if history is None else history[b].tolist()
        n = len(row) if lengths is None else min(max(int(lengths[b]), 0), len(row))
        p = 0 if prompt_lengths is None else min(max(int(prompt_lengths[b]), 0), n)
        seen, times = torch.zeros(V, dtype=torch.bool), torch.zeros(V, dtype=torch.float64)
        for t, v in enumerate(row[:n]):
            if 0 <= v < V:
                seen[v] = True
                times[v] += t >= p
        r, f, pr = num(repetition, b), num(frequency, b), num(presence, b)
        y[b] = torch.where(seen, torch.where(y[b] > 0, y[b] / r, y[b] * r), y[b])
        mag[b] = y[b].abs() + abs(f) * times + abs(pr) * (times > 0)
        y[b] -= f * times + pr * (times > 0)
        if bias is not None:
            z = (bias if bias.dim() == 1 else bias[b % bias.shape[0]]).double().cpu()
            y[b] += z
            mag[b] += z.abs()
        if bias_ids is not None:
            last = {v: float(w) for v, w in zip(bias_ids[b].tolist(), bias_values[b].tolist()) if 0 <= v < V}
            for v, w in last.items():
                y[b, v] += w
                mag[b, v] += abs(w)
        if allowed is not None:
            words = (allowed if allowed.dim() == 1 else allowed[b % allowed.shape[0]]).cpu().long() & 0xffffffff
            ok = ((words[:, None] >> torch.arange(32)) & 1).bool().reshape(-1)[:V]
            y[b] = torch.where(ok, y[b], torch.full_like(y[b], -float("inf")))
    return y, mag


def _check(layer, x, out=None, **kw):
    keep = x.clone()
    y64, mag = _oracle(x, **kw)
    y = layer.adjust_logits(x, out=out, **kw)
    assert out is None or y is out
    assert y.shape == x.shape and y.dtype == (x.dtype if out is None else out.dtype)
    if out is not x:
        assert torch.equal(x.contiguous().view(torch.uint8), keep.contiguous().view(torch.uint8))      # NaN, too
    got = y.double().cpu()
    fine = torch.isfinite(y64)
    assert torch.equal(torch.isfinite(got), fine) and torch.equal(got[~fine].isnan(), y64[~fine].isnan())
    solid = ~fine & ~y64.isnan()
    assert torch.equal(got[solid], y64[solid])
    off, bound = (got - y64).abs()[fine], (6 * U * mag * (1 + 2.0 ** -6) + torch.finfo(y.dtype).eps / 2 * (y64.abs() + 6 * U * mag) + 2.0 ** -126)[fine]
    assert bool((off <= bound).all()), float((off - bound).max())
    return y


class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator().manual_seed(seed)

    def logits(self, B, V, dtype=F32):
        return (torch.randn(B, V, generator=self.g) * 3).to("cuda", dtype)

    def ids(self, lo, hi, *shape, dtype=torch.int64):
        return torch.randint(lo, hi, shape, generator=self.g).to("cuda", dtype)

    def real(self, *shape, lo=0.0, hi=1.0, dtype=F32):
        return (torch.rand(*shape, generator=self.g) * (hi - lo) + lo).to("cuda", dtype)

    def bits(self, *shape):
        return torch.randint(-2 ** 31, 2 ** 31, shape, generator=self.g).to(torch.int32).to("cuda")


# one id, odd rows, the ends of words of the mask and of pieces of 2048 and 8192 elements
@pytest.mark.parametrize("B,V", [(1, 1), (3, 7), (5, 31), (2, 33), (4, 256), (1, 2047), (2, 2048), (3, 2049), (2, 8193), (160, 16411)])
@pytest.mark.parametrize("lt", [F32, BF16])
@pytest.mark.parametrize("ot", [F32, BF16])
def test_all_together(layer, B, V, lt, ot):
    d = _Draw(B * V)
    T, K = 50, min(V, 9)
    out = torch.full((B, V), 7.0, device="cuda", dtype=ot)
    _check(layer, d.logits(B, V, lt), out=out, history=d.ids(0, V, B, T), lengths=d.ids(0, T + 1, B, dtype=torch.int32),
           prompt_lengths=d.ids(0, T + 1, B, dtype=torch.int32), repetition=d.real(B, lo=0.5, hi=2), presence=d.real(B, lo=-1), frequency=d.real(B, lo=-0.5),
           bias=d.real(B, V, lo=-2, hi=2, dtype=ot), bias_ids=d.ids(0, V, B, K), bias_values=d.real(B, K, lo=-9, hi=9), allowed=d.bits(B, (V + 31) // 32))


@pytest.mark.parametrize("kw", ["history", "prompt", "bias", "bias row", "ids", "mask", "mask row", "nothing"])
@pytest.mark.parametrize("lt", [F32, BF16])
def test_each_alone(layer, kw, lt):
    d = _Draw(7)
    B, V, T = 3, 2501, 4000
    x = d.logits(B, V, lt)
    h = dict(history=d.ids(0, 300, B, T, dtype=torch.int32), repetition=1.3, presence=0.25, frequency=0.0625)
    _check(layer, x, **{"history": h, "prompt": dict(h, prompt_lengths=torch.tensor([0, 4000, 1700], dtype=torch.int32, device="cuda")),
                        "bias": dict(bias=d.real(V)), "bias row": dict(bias=d.real(1, V, dtype=BF16)),
                        "ids": dict(bias_ids=d.ids(0, V, B, 700, dtype=torch.int32), bias_values=d.real(B, 700)),
                        "mask": dict(allowed=d.bits(B, 79)), "mask row": dict(allowed=d.bits(79)), "nothing": {}}[kw])


@pytest.mark.parametrize("setting", [dict(repetition=1.5), dict(presence=-0.5), dict(frequency=0.3)])
def test_one_setting_alone(layer, setting):
    d = _Draw(8)
    _check(layer, d.logits(2, 100), history=d.ids(0, 100, 2, 60), **setting)


def test_lengths_are_clamped_and_what_is_behind_is_not_looked_at(layer):
    d = _Draw(9)
    x, h = d.logits(6, 50), d.ids(0, 50, 6, 20)
    lengths = torch.tensor([0, 5, 20, 25, -3, 1], dtype=torch.int32, device="cuda")
    prompts = torch.tensor([4, 9, 3, 22, 1, -7], dtype=torch.int32, device="cuda")
    want = _check(layer, x, history=h, lengths=lengths, prompt_lengths=prompts, repetition=2.0, presence=1.0, frequency=0.5)
    for b, n in enumerate(lengths.clamp(0, 20).tolist()):
        h[b, n:] = 3
    assert torch.equal(want, layer.adjust_logits(x, h, lengths, prompts, 2.0, 1.0, 0.5))
    assert torch.equal(x, layer.adjust_logits(x, h[:, :0], repetition=2.0, presence=1.0))


def test_ids_outside_the_vocabulary_count_for_nothing(layer):
    d = _Draw(10)
    for V in (13, 50, 2048):
        for lt in (F32, BF16):
            flat = d.logits(1, 3 * V + 9, lt)[0]
            for first in (0, 1, 5):
                x = flat[first:first + 2 * V].view(2, V)
                h = d.ids(0, V, 2, 40)
                h[0, ::3] = torch.tensor([-1, -2, -7, V, V + 1, 2 ** 40, -2 ** 63, 2 ** 63 - 1, 2 ** 32, 2 ** 31, -2 ** 31, V + 2048, 4, -8], device="cuda")
                bi = torch.tensor([[-1, V, 2 ** 63 - 1, -2 ** 63, 2], [V + 3, -7, 0, -1, 2 ** 32]], device="cuda")
                _check(layer, x, history=h, repetition=1.5, presence=2.0, frequency=0.5, bias_ids=bi, bias_values=d.real(2, 5))


def test_masked_rows_infinities_and_nan(layer):
    d = _Draw(11)
    inf, nan = float("inf"), float("nan")
    x = d.logits(4, 70)
    x[0, :6] = torch.tensor([inf, -inf, nan, 0.0, -0.0, torch.finfo(F32).min / 4], device="cuda")
    x[1] = torch.finfo(F32).min
    x[3] = nan
    h = torch.arange(70, device="cuda").repeat(4, 1)
    h[1] = -1                                                               # twice the lowest value would be -inf
    allowed = torch.full((4, 3), -1, dtype=torch.int32, device="cuda")
    allowed[2:] = 0
    y = _check(layer, x, history=h[:, :6], repetition=2.0, presence=0.5, allowed=allowed)
    assert bool((y[2:] == -inf).all()) and bool(y[0, 2].isnan())
    allowed[0, 0] = ~4
    assert float(layer.adjust_logits(x, allowed=allowed)[0, 2]) == -inf
    bias = torch.zeros(70, device="cuda")
    bias[3], bias[0], bias[1] = -inf, -inf, inf
    _check(layer, x, bias=bias)
    _check(layer, x.to(BF16), history=h, repetition=2.0)


def test_the_same_biased_id_twice(layer):
    x = torch.zeros(2, 500, device="cuda")
    ids = torch.full((2, 400), 77, device="cuda")
    ids[1, 200:] = 5
    values = torch.arange(800.0, device="cuda").view(2, 400)
    y = _check(layer, x, bias_ids=ids, bias_values=values)
    assert float(y[0, 77]) == 399 and float(y[1, 77]) == 599 and float(y[1, 5]) == 799


def test_counts_of_one_id(layer):
    x = torch.full((1, 64), 100000.0, device="cuda")
    h = torch.full((1, 60001), 9, device="cuda")
    h[0, 5] = 8
    y = layer.adjust_logits(x, h, prompt_lengths=torch.tensor([1], dtype=torch.int32, device="cuda"), frequency=1.0)
    assert float(y[0, 9]) == 100000 - 59999 and float(y[0, 8]) == 99999 and float(y[0, 7]) == 100000


def test_views(layer):
    d = _Draw(12)
    big = d.logits(5, 3 * 101, BF16)
    keep = big.clone()
    h, kw = d.ids(0, 100, 30, 5).t(), dict(repetition=1.5, frequency=0.25)
    for cut in (slice(0, 100), slice(101, 201), slice(3, 103)):
        x = big[:, cut]
        want = _check(layer, x, history=h, bias=d.real(200, 5).t()[:, 50:150], allowed=d.bits(5, 9)[:, 2:6], **kw)
        assert torch.equal(want, _check(layer, x.t().contiguous().t(), history=h, **kw)) is False
        into = torch.full((5, 120), 3.0, device="cuda", dtype=BF16)
        got = _check(layer, x, out=into[:, 7:107], history=h, **kw)
        assert torch.equal(got, layer.adjust_logits(x, h, **kw)) and bool((into[:, :7] == 3).all()) and bool((into[:, 107:] == 3).all())
    side = _check(layer, big[:, 1:101], out=big[:, 201:301], history=h, **kw)     # side by side in one tensor
    assert torch.equal(side, layer.adjust_logits(keep[:, 1:101], h, **kw)) and torch.equal(big[:, :201], keep[:, :201])
    with pytest.raises(ValueError, match="overlaps"):
        layer.adjust_logits(big[:, 1:101], out=big[:, 100:200])
    big.copy_(keep)
    want = layer.adjust_logits(big[:, 101:201], h, **kw)
    x = big[:, 101:201]
    got = _check(layer, x, out=x, history=h, **kw)                          # in place, in the middle of a larger tensor
    assert torch.equal(got, want) and torch.equal(big[:, :101], keep[:, :101]) and torch.equal(big[:, 201:], keep[:, 201:])
    assert torch.equal(_check(layer, d.logits(1, 9).expand(4, 9), history=h[:4].contiguous() % 9, **kw), _check(layer, _Draw(12).logits(1, 1).new_zeros(4, 9))) is False
    last = d.logits(3 * 6, 40).view(3, 6, 40)[:, -1]
    _check(layer, last, history=h[:3] % 40, **kw)


def test_refusals_on_the_device(layer):
    d = _Draw(13)
    x, h, i32 = d.logits(3, 40), d.ids(0, 40, 3, 8), torch.int32
    for kw, what in ((dict(history=h.float()), "history"), (dict(history=h[0]), "history"), (dict(history=h[:2]), "history"), (dict(lengths=d.ids(0, 8, 3, dtype=i32)), "history"),
                     (dict(history=h, lengths=d.ids(0, 8, 3)), "lengths"), (dict(history=h, prompt_lengths=d.ids(0, 8, 2, dtype=i32)), "prompt_lengths"),
                     (dict(history=h, repetition=0.0), "repetition"), (dict(history=h, presence=float("nan")), "presence"),
                     (dict(history=h, frequency=d.real(2)), "frequency"), (dict(history=h, repetition=d.real(3).double()), "repetition"),
                     (dict(bias=d.real(39)), "bias"), (dict(bias=d.real(2, 40)), "bias"), (dict(bias_ids=h), "together"), (dict(bias_values=d.real(3, 8)), "together"),
                     (dict(bias_ids=h, bias_values=d.real(3, 7)), "bias_ids"), (dict(bias_ids=h.float(), bias_values=d.real(3, 8)), "bias_ids"),
                     (dict(allowed=d.bits(3, 1)), "allowed"), (dict(allowed=d.bits(3, 2).long()), "allowed"), (dict(out=x[:, :39]), "out"),
                     (dict(out=d.logits(40, 3).t()), "out"), (dict(history=h.cpu()), "history")):
        with pytest.raises(ValueError, match=what):
            layer.adjust_logits(x, **kw)
    big = d.logits(1, 200)[0]
    with pytest.raises(ValueError, match="overlaps"):
        layer.adjust_logits(big[:120].view(3, 40), out=big[8:128].view(3, 40))
    for name in ("bias", "bias_values"):
        z = d.real(3, 40)
        with pytest.raises(ValueError, match="another argument"):
            layer.adjust_logits(x, **{"bias_ids": d.ids(0, 40, 3, 40)} if name == "bias_values" else {}, **{name: z}, out=z)
    with pytest.raises(TypeError):
        layer.adjust_logits(x, out=x.half())
    with pytest.raises(TypeError):
        layer.adjust_logits(x, bias=d.real(40).half())
    with pytest.raises(NotImplementedError, match="derivative"):
        layer.adjust_logits(x, h, repetition=d.real(3).requires_grad_(True))
    assert layer.adjust_logits(x[:0], h[:0], repetition=2.0, bias_ids=h[:0], bias_values=d.real(0, 8)).shape == (0, 40)


def test_another_stream(layer):
    d = _Draw(14)
    x, h = d.logits(4, 5000), d.ids(0, 5000, 4, 300)
    want = layer.adjust_logits(x, h, repetition=1.2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer.adjust_logits(x, h, repetition=1.2)
    torch.cuda.synchronize()
    assert torch.equal(want, got)


# rows of several pieces each, more of them than run at once: ids of the histories are listed apart
@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("lt,ot", [(BF16, BF16), (F32, F32), (BF16, F32)])
def test_large_batches(layer, in_place, lt, ot):
    if in_place and lt != ot:
        pytest.skip("another type cannot be written in place")
    d = _Draw(15)
    B, V, T, K = 200, 32801, 60, 9
    x = d.logits(B, V, lt)
    h, bi = d.ids(-2, V + 2, B, T), d.ids(-1, V + 1, B, K)
    h[0], h[1, ::2], bi[1, 3:] = 7, V - 1, 11
    kw = dict(history=h, lengths=d.ids(0, T + 1, B, dtype=torch.int32), prompt_lengths=d.ids(0, T + 1, B, dtype=torch.int32), repetition=d.real(B, lo=0.5, hi=2),
              presence=d.real(B, lo=-1), frequency=d.real(B, lo=-0.5))
    full = dict(kw, bias=d.real(V, lo=-2, hi=2), bias_ids=bi, bias_values=d.real(B, K, lo=-9, hi=9), allowed=d.bits(B, (V + 31) // 32))
    want = _check(layer, x, out=torch.empty(B, V, device="cuda", dtype=ot), **full)
    some = _check(layer, x, out=torch.empty(B, V, device="cuda", dtype=ot), **kw)
    if in_place:
        y, z = x.clone(), x
        assert torch.equal(layer.adjust_logits(y, out=y, **full), want) and torch.equal(layer.adjust_logits(z, out=z, **kw), some)


def test_long_histories_of_large_batches(layer):
    """As many different ids as the table of a row takes, and one more than that."""
    d = _Draw(16)
    B, V = 190, 32768
    x = d.logits(B, V)
    for T in (12288, 12289):
        h = torch.stack([torch.randperm(V, generator=d.g)[:T] for _ in range(3)]).repeat(64, 1)[:B].to("cuda")
        y = layer.adjust_logits(x, h, presence=1.0, repetition=2.0)
        r = torch.where(x > 0, x / 2, x * 2) - 1
        want = x.clone().scatter_(1, h, r.gather(1, h))
        assert torch.equal(y, want)


_CAPTURE = r"""
import torch
from paper_1911_04070_b200 import layer
x, h = torch.randn(4, 3001, device="cuda"), torch.randint(0, 3001, (4, 200), device="cuda")
n = torch.tensor([5, 0, 200, 77], dtype=torch.int32, device="cuda")
rep, out = torch.rand(4, device="cuda") + 1, torch.empty(4, 3001, device="cuda")
step = lambda: layer.adjust_logits(x, h, lengths=n, repetition=rep, frequency=0.1, out=out)
step()
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    step()
x.normal_(); n.add_(3); h.random_(0, 3001)
graph.replay()
got = out.clone()
assert torch.equal(step(), got)
print("done")
"""


def test_capture():
    r = subprocess.run([sys.executable, "-c", _CAPTURE], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "done" in r.stdout, r.stderr[-2000:]


def test_offsets_past_32_bits(layer):
    B, V = 3, 2 ** 30 - 1
    x = torch.zeros(B, V, dtype=BF16, device="cuda")
    h = torch.tensor([[V - 1], [0], [V - 2]], device="cuda")
    y = layer.adjust_logits(x, h, presence=2.0, out=x)
    assert float(y[2, -2]) == -2 and float(y[0, -1]) == -2 and float(y[1, 0]) == -2 and int(torch.count_nonzero(y)) == 3
