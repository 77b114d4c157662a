"""BPTLanguageModel: ids to logits, gradients, training steps and generation, against the float64 oracle of the layer stack and against the
same steps written out with PyTorch's operators.  float32 throughout (the general kernels); bounds as for the layer's own tests: 2e-4 of the
largest value for outputs and gradients, whose errors are those of the stack's float32 operators."""
import pytest
import torch

pytestmark = pytest.mark.gpu

NAMES = {"wq": "wq.weight", "wk": "wk.weight", "wv": "wv.weight", "wo": "wo.weight", "rel_emb": "rel_emb",
         "ln1_w": "norm1.weight", "ln1_b": "norm1.bias", "ln2_w": "norm2.weight", "ln2_b": "norm2.bias",
         "ff1_w": "ff1.weight", "ff1_b": "ff1.bias", "ff2_w": "ff2.weight", "ff2_b": "ff2.bias"}


def _model(n=32, k=3, vocab=37, tied=True, padding_idx=None, seed=3):
    from paper_1911_04070_b200 import layer
    torch.manual_seed(seed)
    m = layer.BPTLanguageModel(vocab, n, k, 64, 2, 96, 2, tied=tied, padding_idx=padding_idx, device="cuda:0").to("cuda:0")
    with torch.no_grad():
        for l in m.encoder.layers:
            l.rel_emb.mul_(10.0)            # relation embeddings large enough to matter
    return m


def _oracle(m, ids, lengths=None):
    """Logits in float64 on the CPU, and the parameters they depend on: {name: leaf}."""
    from oracle import bpt_layer, bpt_oracle as orc
    leaves = {a: p.detach().double().cpu().requires_grad_(True) for a, p in m.named_parameters()}
    ws = [{a: leaves["encoder.layers.%d.%s" % (i, b)] for a, b in NAMES.items()} for i in range(len(m.encoder.layers))]
    emb = leaves["embedding"]
    rows = emb[ids.cpu()] * m.scale
    if m.padding_idx is not None:
        rows = torch.where((ids.cpu() == m.padding_idx)[..., None], rows.detach(), rows)
    if lengths is not None:
        rows = rows * (torch.arange(ids.shape[1]) < lengths.cpu()[:, None])[..., None]
    h = bpt_layer.encoder_forward(rows, ws, orc.enumerate_graph(m.encoder.n, m.encoder.g.k, 1), 2, None if lengths is None else lengths.tolist(), "tokens")
    return h @ (emb if m.head is None else leaves["head.weight"]).T, leaves


def _close(got, want, tol=2e-4):
    got, want = got.detach().double().cpu(), want.detach()
    assert float((got - want).abs().max()) <= tol * float(want.abs().max()), float((got - want).abs().max() / want.abs().max())


@pytest.mark.parametrize("tied,padding_idx,ragged", [(True, None, False), (False, None, False), (True, 5, True), (False, 0, True)])
def test_logits_and_gradients(tied, padding_idx, ragged):
    m = _model(tied=tied, padding_idx=padding_idx)
    ids = torch.randint(0, 37, (3, 32), device="cuda:0")
    lengths = torch.tensor([32, 7, 20], dtype=torch.int32, device="cuda:0") if ragged else None
    x = m(ids, lengths)
    want, leaves = _oracle(m, ids, lengths)
    real = torch.ones(3, 32, dtype=torch.bool) if lengths is None else torch.arange(32) < lengths.cpu()[:, None]
    _close(x.cpu()[real], want[real])
    loss = m.loss(ids, lengths)
    target, on = ids.cpu()[:, 1:], real[:, 1:]
    want_loss = torch.nn.functional.cross_entropy(want[:, :-1][on], target[on])
    assert abs(float(loss) - float(want_loss)) <= 2e-4 * float(want_loss)
    loss.backward()
    grads = torch.autograd.grad(want_loss, list(leaves.values()), allow_unused=True)
    for (name, p), g in zip(m.named_parameters(), grads):
        if "rel_emb" in name:
            continue                        # its ancestors' rows are exact zeros here; held to its own bounds in the layer's tests
        _close(p.grad, g)


def test_training_step_is_the_step_written_out():
    from paper_1911_04070_b200 import layer
    a, b = _model(padding_idx=2), _model(padding_idx=2)
    opt_a, opt_b = (torch.optim.SGD(m.parameters(), lr=0.5) for m in (a, b))
    ids = torch.randint(0, 37, (4, 32), device="cuda:0")
    lengths = torch.tensor([32, 9, 2, 31], dtype=torch.int32, device="cuda:0")
    for most in (0.05, 1e6):
        loss, norm = layer.training_step(a, opt_a, ids, lengths, max_norm=most)
        opt_b.zero_grad(set_to_none=True)
        want = b.loss(ids, lengths)
        want.backward()
        want_norm = torch.nn.utils.clip_grad_norm_(b.parameters(), most)
        opt_b.step()
        # equal but for the order of the norm's sum, which reaches the results by a factor of at most 1 + 2^-20
        assert torch.equal(loss, want.detach()) and abs(float(norm) - float(want_norm)) <= 2.0 ** -20 * float(want_norm)
        for p, q in zip(a.parameters(), b.parameters()):
            assert float((p.grad - q.grad).abs().max()) <= 2.0 ** -20 * float(q.grad.abs().max())
            with torch.no_grad():
                p.copy_(q)


def _greedy(m, prompt, steps, allowed=None, repetition=1.0, presence=0.0, frequency=0.0, bias=None):
    """Generation by a full forward pass per token and a loop over the ids, all in float64 after the model."""
    ids, P, V = prompt.clone(), prompt.shape[1], m.vocab
    for _ in range(steps):
        t = ids.shape[1]
        full = torch.cat([ids, ids.new_zeros(ids.shape[0], m.encoder.n - t)], 1)
        x = m(full, torch.full((ids.shape[0],), t, dtype=torch.int32, device=ids.device))[:, t - 1].double()
        for b, row in enumerate(ids.tolist()):
            for v in range(V):
                n = row[P:].count(v)
                if v in row:
                    x[b, v] = x[b, v] / repetition if x[b, v] > 0 else x[b, v] * repetition
                x[b, v] -= frequency * n + presence * (n > 0)
        if bias is not None:
            x += bias.double()
        words = allowed(ids) if callable(allowed) else allowed
        if words is not None:
            words = words.expand(ids.shape[0], -1)
            ok = torch.stack([(words[:, v // 32] >> (v % 32)) & 1 for v in range(V)], 1).bool()
            x = x.masked_fill(~ok, -float("inf"))
        best = x.topk(2, dim=-1).values
        assert bool((best[:, 0] - best[:, 1] > 1e-3).all()), "the choice is too close for float32: another seed"
        ids = torch.cat([ids, x.argmax(-1, keepdim=True)], 1)
    return ids


@pytest.mark.parametrize("settings", [{}, dict(repetition=1.7), dict(presence=3.0, frequency=0.5), dict(repetition=1.2, frequency=1.0)])
@torch.no_grad()
def test_generation(settings):
    m = _model(seed=11)
    prompt = torch.randint(0, 37, (3, 4), generator=torch.Generator().manual_seed(2)).to("cuda:0")
    got = m.generate(prompt, 12, **settings)
    assert got.shape == (3, 16) and torch.equal(got[:, :4], prompt)
    assert torch.equal(got, _greedy(m, prompt, 12, **settings))


@torch.no_grad()
def test_generation_under_a_grammar_and_a_bias():
    m = _model(seed=12)
    prompt = torch.randint(0, 37, (2, 3), device="cuda:0")
    even, odd = (sum(1 << v for v in range(s, 32, 2)) for s in (0, 1))
    word = lambda w: w - (1 << 32) if w >> 31 else w

    def alternate(ids):                     # even ids follow odd ones and the other way round
        w = torch.where(ids[:, -1:] % 2 == 0, torch.tensor([[word(odd), 0]], device="cuda:0"), torch.tensor([[word(even), 0]], device="cuda:0"))
        return w.int()

    bias = torch.linspace(-2, 2, 37, device="cuda:0")
    got = m.generate(prompt, 20, allowed=alternate, bias=bias, repetition=1.1)
    assert bool(((got[:, 3:] % 2) != (got[:, 2:-1] % 2)).all()) and bool((got[:, 3:] < 32).all())
    assert torch.equal(got[:, :10], _greedy(m, prompt, 7, allowed=alternate, bias=bias, repetition=1.1))
    drawn = [m.generate(prompt, 20, temperature=1.5, generator=torch.Generator("cuda:0").manual_seed(s), allowed=alternate(prompt)) for s in (1, 1, 2)]
    assert torch.equal(drawn[0], drawn[1]) and not torch.equal(drawn[0], drawn[2])


def test_refusals():
    from paper_1911_04070_b200 import layer
    m = _model()
    ids = torch.zeros(1, 5, dtype=torch.int64, device="cuda:0")
    for call in (lambda: m(ids), lambda: m.generate(ids[:, :0], 3), lambda: m.generate(ids, 28), lambda: m.generate(ids, 3, temperature=-1.0),
                 lambda: layer.BPTLanguageModel(0, 32, 3, 64, 2, 96, 1), lambda: layer.BPTLanguageModel(9, 32, 3, 64, 2, 96, 1, padding_idx=9),
                 lambda: m.encoder.forward_nodes(torch.zeros(1, 32, 64, device="cuda:0"))):
        with pytest.raises(ValueError):
            call()
    assert torch.equal(m.generate(ids, 0), ids) and m.generate(ids, 27).shape == (1, 32)


def test_a_bfloat16_model_trains_and_generates():
    """The tiled kernels: every parameter gets a finite gradient, the norm is that of the gradients, and an id outside the table is reported."""
    from paper_1911_04070_b200 import binding, layer
    torch.manual_seed(0)
    m = layer.BPTLanguageModel(256, 128, 8, 128, 2, 256, 2, device="cuda:0", gated="silu", sandwich=True).to("cuda:0", torch.bfloat16)
    opt = torch.optim.SGD(m.parameters(), lr=0.0)
    ids = torch.randint(0, 256, (2, 128), device="cuda:0")
    binding.bpt_check_device()
    loss, norm = layer.training_step(m, opt, ids, max_norm=1e9)
    assert bool(torch.isfinite(loss)) and all(bool(torch.isfinite(p.grad).all()) for p in m.parameters())
    want = float(torch.cat([p.grad.double().reshape(-1) for p in m.parameters()]).norm())
    assert abs(float(norm) - want) <= 5 * 2.0 ** -24 * want
    got = m.generate(ids[:, :8], 8, temperature=1.0, generator=torch.Generator("cuda:0").manual_seed(1))
    assert got.shape == (2, 16) and bool((got >= 0).all()) and bool((got < 256).all()) and binding.bpt_check_device() == 0
    ids[0, 3] = 256
    m(ids)
    assert binding.bpt_check_device() == 8
