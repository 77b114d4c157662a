"""layer.adjust_logits on the GPU with arguments that lie beside one another in memory, and the passes of one launch over several pieces of rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def layer():
    from paper_1911_04070_b200 import layer
    return layer


def test_results_beside_other_arguments_in_one_buffer(layer):
    """Apart from all other arguments is apart: rows between the rows of another argument are; rows that share an element with one are refused."""
    buf = torch.randn(4, 400, generator=torch.Generator().manual_seed(1)).to("cuda")
    x, bias, out = buf[:, :100], buf[:, 100:200], buf[:, 200:300]
    keep, want = buf.clone(), x + bias
    assert torch.equal(layer.adjust_logits(x, bias=bias, out=out), want) and torch.equal(buf[:, :200], keep[:, :200]) and torch.equal(buf[:, 300:], keep[:, 300:])
    for into in (buf[:, 199:299], buf[:, 50:150], buf[:, 99:199]):
        with pytest.raises(ValueError, match="overlaps"):
            layer.adjust_logits(x, bias=bias, out=into)
    # rows at another distance than the logits': the first one ends before them, the second begins behind the third of them
    flat = torch.randn(2000, generator=torch.Generator().manual_seed(2)).to("cuda")
    x, out = flat[100:820].view(2, 360)[:, :100], flat.as_strided((2, 100), (1000, 1), 0)
    want = x.clone()
    assert torch.equal(layer.adjust_logits(x, out=out), want)
    with pytest.raises(ValueError, match="overlaps"):
        layer.adjust_logits(x, out=flat.as_strided((2, 100), (1000, 1), 1))


# the pass alone (no history, no ids of a row's own): pieces of 4096 elements, from a 16-byte boundary of the logits on
@pytest.mark.parametrize("V", [4088, 4095, 4096, 4097, 4104, 8191, 8192, 8193, 12300])
@pytest.mark.parametrize("lt", [F32, BF16])
@pytest.mark.parametrize("bt", [F32, BF16])
def test_pieces_of_a_pass_without_a_history(layer, V, lt, bt):
    g = torch.Generator("cuda").manual_seed(V)
    for first in (0, 1, 3, 7):
        buf = torch.randn(3 * V + 20, generator=g, device="cuda").to(lt)
        x = buf[first:first + 3 * V].view(3, V)             # rows of an odd V start anywhere
        bias = torch.randn(3 * V + 9, generator=g, device="cuda").to(bt)[first:first + 3 * V].view(3, V)
        words = torch.randint(-2 ** 31, 2 ** 31, (3, (V + 31) // 32), generator=g, device="cuda").to(torch.int32)
        words[1] = 0
        ok = ((words[..., None] >> torch.arange(32, device="cuda")) & 1).bool().view(3, -1)[:, :V]
        masked = lambda t: torch.where(ok, t, torch.full_like(t, -float("inf"))).to(lt)
        # one addition in float32 and one rounding: the same bits
        for kw, want in ((dict(bias=bias), (x.float() + bias.float()).to(lt)), (dict(allowed=words), masked(x.float())),
                         (dict(bias=bias, allowed=words), masked(x.float() + bias.float())), (dict(bias=bias[0]), (x.float() + bias[0].float()).to(lt)), ({}, x)):
            want = want.clone()
            assert torch.equal(layer.adjust_logits(x, **kw), want)
            into = torch.full((3, V + 5), 7.0, device="cuda", dtype=lt)
            assert torch.equal(layer.adjust_logits(x, out=into[:, first % 5:first % 5 + V], **kw), want) and int((into == 7).sum()) >= 15
            keep = buf.clone()
            assert torch.equal(layer.adjust_logits(x, out=x, **kw), want)
            assert torch.equal(buf[:first], keep[:first]) and torch.equal(buf[first + 3 * V:], keep[first + 3 * V:])
            buf.copy_(keep)
