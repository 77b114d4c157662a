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
