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
