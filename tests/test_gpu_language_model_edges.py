"""BPTLanguageModel on the GPU with the inputs at the edge of what its calls define."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def _model(vocab=37, n=32, k=3, seed=3, **form):
    from paper_1911_04070_b200 import layer
    torch.manual_seed(seed)
    return layer.BPTLanguageModel(vocab, n, k, 64, 2, 96, 2, device="cuda:0", **form).to("cuda:0")


@pytest.mark.parametrize("bad", [37, -1, -100, 2 ** 40])
def test_an_id_outside_the_table_in_a_training_step(bad):
    """Reported, not a target, and the parameters' gradients are those of a loss without it."""
    from paper_1911_04070_b200 import binding, layer
    m = _model()
    opt = torch.optim.SGD(m.parameters(), lr=0.0)
    ids = torch.randint(0, 37, (3, 32), generator=torch.Generator().manual_seed(1)).to("cuda:0")
    ids[1, 5] = bad
    while binding.bpt_check_device():
        pass
    loss, norm = layer.training_step(m, opt, ids, max_norm=1e9)
    assert binding.bpt_check_device() == 8 and binding.bpt_check_device() == 0
    assert bool(torch.isfinite(loss)) and bool(torch.isfinite(norm)) and all(bool(torch.isfinite(p.grad).all()) for p in m.parameters())
    p = m(ids)[:, :-1].detach().double().log_softmax(-1)
    on = torch.ones(3, 31, dtype=torch.bool, device="cuda:0")
    on[1, 4] = False
    want = -p[on].gather(1, ids[:, 1:][on][:, None]).mean()
    # as on the host: at most 7 + 37 + 93 roundings of values up to the largest one
    assert abs(float(loss) - float(want)) <= 150 * 2.0 ** -24 * float(p.abs().max())


@pytest.mark.parametrize("temperature", [0.0, 1.5])
@torch.no_grad()
def test_a_sequence_that_its_grammar_ends(temperature):
    """Sequence 1 has nothing allowed at its third id, sequence 0 and 2 go on as if it were not there."""
    m = _model()
    prompt = torch.randint(0, 37, (3, 4), generator=torch.Generator().manual_seed(2)).to("cuda:0")
    always = torch.tensor([0x7ffffffe, 0], dtype=torch.int32, device="cuda:0")

    def grammar(ids):
        w = always.repeat(3, 1)
        if ids.shape[1] == 6:
            w[1] = 0
        return w

    call = lambda **kw: m.generate(prompt, 10, temperature, torch.Generator("cuda:0").manual_seed(5), repetition=1.1, **kw)
    got, free = call(allowed=grammar, end_id=36), call(allowed=always)
    assert torch.equal(got[::2], free[::2]) and torch.equal(got[1, :6], free[1, :6]) and bool((got[1, 6:] == 36).all())
    assert bool((free[:, 4:] >= 1).all()) and bool((free[:, 4:] < 31).all())
    with pytest.raises(ValueError, match="end_id"):
        call(allowed=grammar)
    ban = torch.full((37,), -float("inf"), device="cuda:0")         # a bias that leaves nothing, from the first step on
    assert bool((call(bias=ban, end_id=0)[:, 4:] == 0).all())


@torch.no_grad()
def test_logits_that_are_not_finite_are_not_drawn_from():
    """Said in words; the device takes calls as before."""
    prompt = torch.randint(0, 37, (3, 4), generator=torch.Generator().manual_seed(2)).to("cuda:0")
    m = _model(tied=False)
    want = m.generate(prompt, 6, 1.0, torch.Generator("cuda:0").manual_seed(5))
    keep = m.head.weight[5].clone()
    for bad in (float("nan"), float("inf")):
        m.head.weight[5] = bad
        with pytest.raises(ValueError, match="not finite"):
            m.generate(prompt, 6, 1.0, torch.Generator("cuda:0").manual_seed(5))
    m.head.weight[5] = keep
    with pytest.raises(ValueError, match="not finite"):
        m.generate(prompt, 6, 1e-42, torch.Generator("cuda:0").manual_seed(5))
    assert torch.equal(m.generate(prompt, 6, 1.0, torch.Generator("cuda:0").manual_seed(5)), want)
