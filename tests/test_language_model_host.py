"""What BPTLanguageModel does around its stack, on the CPU: the stack itself, whose kernels need a device, is replaced by given logits."""
import pytest
import torch

from paper_1911_04070_b200 import layer


class _Given:
    """Stands for a model: its logits are given."""

    def __init__(self, logits):
        self.x, self.vocab = logits, logits.shape[-1]

    def __call__(self, ids, lengths=None):
        return self.x


@pytest.mark.parametrize("dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("bad", [[7], [-1], [-100], [7, -1, 2 ** 31 - 1, -2 ** 31]])
def test_ids_outside_the_vocabulary_are_no_targets(dtype, ragged, bad):
    g = torch.Generator().manual_seed(1)
    x, ids = torch.randn(3, 9, 7, generator=g, requires_grad=True), torch.randint(0, 7, (3, 9), generator=g).to(dtype)
    lengths = torch.tensor([9, 5, 1], dtype=torch.int32) if ragged else None
    on = torch.ones(3, 8, dtype=torch.bool) if lengths is None else torch.arange(1, 9) < lengths[:, None]
    for i, v in enumerate(bad):
        ids[i % 2, 2 * i + 1] = v
        on[i % 2, 2 * i] = False
    ids[2, 0] = bad[0]                          # the first id is no target
    loss = layer.BPTLanguageModel.loss(_Given(x), ids, lengths)
    # -log softmax of the targets that there are, in float64
    p = x.detach().double()[:, :-1].log_softmax(-1)
    want = -p[on].gather(1, ids[:, 1:][on].long()[:, None]).mean()
    # log_softmax over 7 and a mean over up to 24 values in float32: no more than 50 roundings of values up to the largest one
    assert abs(float(loss) - float(want)) <= 50 * 2.0 ** -24 * float(p.abs().max())
    dx, = torch.autograd.grad(loss, [x])
    assert bool(torch.isfinite(dx).all()) and not dx[:, -1].any() and not dx[:, :-1][~on].any() and bool((dx[:, :-1][on].abs().sum(-1) > 0).all())


class _Steps:
    """Stands for a model in generate: step by step, the logits are given for every last id and row."""

    def __init__(self, table):          # [steps at most, B, V]
        self.table, self.vocab, self.scale, self.padding_idx, self.embedding, self.encoder = table, table.shape[-1], 1.0, None, torch.zeros(1), self
        self.n, self.t = table.shape[0], 0

    def step(self, state):
        self.t += 1
        return self.table[self.t - 1]

    def logits(self, state):
        return state.clone()


def _masked(x, history, lengths, prompts, allowed=None, bias=None, out=None, **settings):
    if allowed is None:
        return
    words = allowed.expand(x.shape[0], -1).long() & 0xffffffff
    ok = ((words[:, torch.arange(x.shape[1]) // 32] >> (torch.arange(x.shape[1]) % 32)) & 1).bool()
    out.copy_(torch.where(ok, x, torch.full_like(x, -float("inf"))))


def _generate(monkeypatch, table, prompt, steps, **kw):
    m = _Steps(table)
    monkeypatch.setattr(layer, "BPTDecoder", lambda encoder, B, dtype: m)
    monkeypatch.setattr(layer, "token_states", lambda ids, weight, scale: ids)
    monkeypatch.setattr(layer, "adjust_logits", _masked)
    return layer.BPTLanguageModel.generate(m, prompt, steps, **kw)


@pytest.mark.parametrize("temperature", [0.0, 0.7])
def test_a_sequence_without_an_allowed_id_has_ended(monkeypatch, temperature):
    """Row 1 has nothing allowed at the third id of the answer, and something again from the fifth on; rows 0 and 2 always do."""
    g = torch.Generator().manual_seed(3)
    table, prompt = torch.randn(12, 3, 20, generator=g), torch.randint(0, 20, (3, 2), generator=g)

    def grammar(ids):
        w = torch.full((3, 1), 0b11111111110, dtype=torch.int32)
        if ids.shape[1] == 4 or ids.shape[1] == 5:
            w[1] = 0
        return w

    call = lambda **kw: _generate(monkeypatch, table, prompt, 8, temperature=temperature, generator=torch.Generator().manual_seed(7), **kw)
    got = call(allowed=grammar, end_id=19)
    free = call(allowed=torch.tensor([0b11111111110], dtype=torch.int32))       # the same draws, nothing ever forbidden altogether
    assert torch.equal(got[0], free[0]) and torch.equal(got[2], free[2]) and torch.equal(got[1, :4], free[1, :4])
    assert bool((got[1, 4:] == 19).all())
    with pytest.raises(ValueError, match="end_id"):
        call(allowed=grammar)
    assert torch.equal(call(allowed=torch.tensor([0b11111111110], dtype=torch.int32), end_id=0), free)
    for bad in (-1, 20):
        with pytest.raises(ValueError, match="end_id"):
            call(allowed=grammar, end_id=bad)


@pytest.mark.parametrize("call", [lambda t: layer.clip_gradients([t], 1.0), lambda t: layer.clip_gradients([t], 1.0, out=[t]), lambda t: layer.gradient_norm(t)])
def test_clipping_is_not_traced(call):
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(call, (torch.ones(4),), check_trace=False)


def _checked(draw):
    def multinomial(p, *a, **k):
        assert bool((p >= 0).all()) and bool(torch.isfinite(p).all()) and bool((p.sum(-1) > 0).all())
        return draw(p, *a, **k)
    return multinomial


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("masked", [False, True])
def test_nothing_is_drawn_from_logits_that_are_not_finite(monkeypatch, what, masked):
    """Said in words, and not by the draw's own check on the device; a temperature that takes logits beyond float32 does the same."""
    monkeypatch.setattr(torch, "multinomial", _checked(torch.multinomial))
    g = torch.Generator().manual_seed(3)
    table, prompt = torch.randn(12, 3, 20, generator=g), torch.randint(0, 20, (3, 2), generator=g)
    kw = dict(allowed=torch.tensor([0b11111111110], dtype=torch.int32)) if masked else {}
    call = lambda t, temperature: _generate(monkeypatch, t, prompt, 8, temperature=temperature, generator=torch.Generator().manual_seed(7), **kw)
    assert call(table, 0.7).shape == (3, 10)
    broken = table.clone()
    broken[4, 1, 5] = what
    with pytest.raises(ValueError, match="not finite"):
        call(broken, 0.7)
    with pytest.raises(ValueError, match="not finite"):
        call(table, 1e-42)


def test_a_temperature_that_takes_all_logits_below_float32_ends_nothing(monkeypatch):
    table = -1 - torch.rand(12, 3, 20, generator=torch.Generator().manual_seed(3))
    with pytest.raises(ValueError, match="not finite"):
        _generate(monkeypatch, table, torch.zeros(3, 2, dtype=torch.int64), 8, temperature=1e-42, end_id=3)


@pytest.mark.parametrize("temperature", [0.0, 0.7])
@pytest.mark.parametrize("steps", [0, 1, 5])
def test_a_mask_that_allows_nothing_from_the_first_step_on(monkeypatch, temperature, steps):
    """Given for one row of three; the other rows' ids do not show it."""
    table, prompt = torch.randn(12, 3, 20, generator=torch.Generator().manual_seed(3)), torch.ones(3, 2, dtype=torch.int64)
    mask = torch.full((3, 1), 0xfffff, dtype=torch.int32)
    call = lambda **kw: _generate(monkeypatch, table, prompt, steps, temperature=temperature, generator=torch.Generator().manual_seed(7), allowed=mask, **kw)
    free = call()
    mask[1] = 0
    got = call(end_id=4)
    assert got.shape == (3, 2 + steps) and torch.equal(got[::2], free[::2]) and bool((got[1, 2:] == 4).all()) and bool((got[:, :2] == 1).all())
    if steps:
        with pytest.raises(ValueError, match="end_id"):
            call()
