"""Host side of bpt_adjust_logits: refusals before anything is launched, and what layer.adjust_logits refuses.  No GPU needed."""
import ctypes

import pytest
import torch
from torch.autograd import forward_ad


@pytest.fixture(scope="module")
def lib():
    from paper_1911_04070_b200 import build, binding
    build.build()
    return binding.load_library()


def _args(**kw):
    from paper_1911_04070_b200 import binding
    a = dict(rows=3, vocab=100, logits_stride=100, out_stride=100, dtype=1, out_dtype=1, logits=4096, repetition=1.0, history_bytes=8, bias_id_bytes=8)
    a.update(kw)
    return binding.LogitsArgs(**a)


H = dict(history=4096, history_len=5, history_stride=5)


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(vocab=0), 1), (dict(dtype=2), 1), (dict(out_dtype=-1), 1), (dict(logits=None), 1), (dict(logits=4097), 1),
                                       (dict(logits_stride=99), 1), (dict(out_stride=99), 1), (dict(history_len=-1), 1), (dict(history_len=5), 1),
                                       (dict(H, history_bytes=2), 1), (dict(H, history=4100), 1), (dict(H, history_stride=-5), 1), (dict(H, lengths=4097), 1),
                                       (dict(H, prompt_lengths=4098), 1), (dict(H, repetition=0.0), 1), (dict(H, repetition=-1.0), 1),
                                       (dict(H, repetition=float("nan")), 1), (dict(H, presence=float("inf")), 1), (dict(H, frequency=float("nan")), 1),
                                       (dict(H, presence_rows=4097), 1), (dict(bias=4096, bias_dtype=3), 1), (dict(bias=4097), 1),
                                       (dict(bias=4096, bias_stride=50), 1), (dict(bias_count=-1), 1), (dict(bias_count=2), 1),
                                       (dict(bias_count=2, bias_ids=4096), 1), (dict(bias_count=2, bias_ids=4100, bias_values=4096), 1),
                                       (dict(bias_count=2, bias_ids=4096, bias_values=4096, bias_id_bytes=1), 1), (dict(allowed=4098), 1),
                                       (dict(allowed=4096, allowed_stride=3), 1), (dict(vocab=1 << 30, logits_stride=1 << 30, out_stride=1 << 30), 2),
                                       (dict(rows=1 << 29, vocab=1 << 14, logits_stride=1 << 14, out_stride=1 << 14), 2)])
def test_refusals(lib, kw, status):
    assert lib.bpt_adjust_logits(ctypes.byref(_args(**kw)), 8192, 16384, 1 << 50, None) == status


def test_more_refusals(lib):
    call = lambda a, out=8192, ws=16384, n=1 << 50: lib.bpt_adjust_logits(a if a is None else ctypes.byref(a), out, ws, n, None)
    need = lambda a: lib.bpt_adjust_logits_workspace_bytes(a if a is None else ctypes.byref(a))
    assert call(None) == 1 and need(None) == 0
    assert call(_args(), out=None) == 1 and call(_args(), out=8193) == 1
    assert call(_args(rows=0, logits=None, history_len=4, bias_count=3), out=None) == 0
    # many pieces of rows with a history: listed apart, in a workspace
    big = dict(H, rows=3000, vocab=50000, logits_stride=50000, out_stride=50000, presence=1.0)
    assert need(_args()) == 0 and need(_args(**dict(big, presence=0.0))) == 0 and need(_args(**dict(big, history_len=20000))) == 0
    a = _args(**big)
    assert need(a) >= 3000 * (5 * 8 + 4)
    assert call(a, ws=None) == 3 and call(a, n=need(a) - 1) == 3 and call(a, ws=16392) == 1


def test_python_refusals(lib):
    from paper_1911_04070_b200 import layer
    x = torch.zeros(2, 40)
    with pytest.raises(ValueError, match="CUDA"):
        layer.adjust_logits(x)
    with pytest.raises(TypeError, match="float32 and bfloat16"):
        layer.adjust_logits(x.half())
    with pytest.raises(NotImplementedError, match="derivative"):
        layer.adjust_logits(x.clone().requires_grad_(True))
    with pytest.raises(NotImplementedError, match="derivative"):
        layer.adjust_logits(x, bias=torch.zeros(40, requires_grad=True))
    with forward_ad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
        layer.adjust_logits(forward_ad.make_dual(x, x))
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(layer.adjust_logits, (x,), check_trace=False)
