"""Host side of bpt_grad_norm / bpt_clip_grads: refusals before anything is launched (the overlaps among them), the workspace query, and
what layer.clip_gradients refuses.  No GPU needed."""
import ctypes

import pytest
import torch
from torch.autograd import forward_ad


@pytest.fixture(scope="module")
def lib():
    from paper_1911_04070_b200 import build, binding
    build.build()
    return binding.load_library()


def _list(*entries):
    from paper_1911_04070_b200 import binding
    return (binding.Grad * len(entries))(*(binding.Grad(*e) for e in entries)), len(entries)


def _clip(lib, *entries, kind=0, most=1.0, eps=1e-6, norm=4096, ws=8192, n=1 << 40):
    a, k = _list(*entries)
    return lib.bpt_clip_grads(a, k, kind, most, eps, norm, ws, n, None)


# (grad, out, numel, dtype, out_dtype): float32 tensors of 16 elements take 64 bytes
A, B = (65536, None, 16, 0, 0), (131072, None, 16, 1, 0)


@pytest.mark.parametrize("entries", [((65536, None, -1, 0, 0),), ((None, None, 4, 0, 0),), ((65538, None, 4, 0, 0),), ((65537, None, 4, 1, 0),),
                                     ((65536, None, 4, 2, 0),), ((65536, 131073, 4, 0, 1),), ((65536, 131072, 4, 0, 3),)])
def test_refused_entries(lib, entries):
    assert _clip(lib, *entries) == 1
    assert _clip(lib, A, *entries) == 1


def test_refusals(lib):
    assert _clip(lib, A, kind=2) == 1 and _clip(lib, A, most=-1.0) == 1 and _clip(lib, A, most=float("nan")) == 1 and _clip(lib, A, eps=-1e-6) == 1
    assert _clip(lib, A, norm=None) == 1 and _clip(lib, A, norm=4098) == 1
    assert _clip(lib, A, ws=None) == 3 and _clip(lib, A, n=0) == 3 and _clip(lib, A, ws=8200) == 1
    assert _clip(lib, (65536, None, (1 << 40) + 1, 0, 0)) == 2
    assert lib.bpt_clip_grads(None, 1, 0, 1.0, 1e-6, 4096, 8192, 1 << 30, None) == 1 and lib.bpt_clip_grads(None, -1, 0, 1.0, 1e-6, 4096, 8192, 1 << 30, None) == 1
    a, n = _list(A)
    assert lib.bpt_grad_norm(a, n, 5, 4096, 8192, 1 << 30, None) == 1 and lib.bpt_grad_norm(a, n, 0, None, 8192, 1 << 30, None) == 1


@pytest.mark.parametrize("entries", [(A, A), (A, B, A), (A, (65536 + 60, None, 16, 0, 0)), ((65536 - 60, None, 16, 0, 0), A),
                                     ((65536, None, 1000, 0, 0), (65540, None, 1, 0, 0), B),                # one inside another
                                     ((65536, 131072, 16, 0, 0), (196608, 131072 + 32, 16, 0, 0)),           # two results
                                     ((65536, 131072, 16, 0, 0), (131072 + 4, 196608, 16, 0, 0)),           # a result over another's gradient
                                     ((65536, 131072, 16, 0, 0), (65536, 196608, 16, 0, 0), (196608, None, 16, 0, 0)),
                                     ((65536, 65536, 16, 0, 1),), ((65536, 65536 + 4, 16, 0, 0),)])
def test_overlaps(lib, entries):
    assert _clip(lib, *entries) == 1
    assert _clip(lib, *reversed(entries)) == 1


def test_workspace_query(lib):
    q = lambda *e: lib.bpt_grad_norm_workspace_bytes(*_list(*e))
    assert q() >= 16 and q((None, None, 0, 0, 0)) >= 16 and q((None, None, 5, 0, 0)) == 0
    assert q(*[(65536, None, 1 << 30, 0, 0)] * 2000) <= 3 * 148 * 8 * 8


def test_python_refusals(lib):
    from paper_1911_04070_b200 import layer
    t = torch.zeros(4)
    with pytest.raises(ValueError, match="CUDA"):
        layer.clip_gradients([t], 1.0)
    with pytest.raises(ValueError, match="CUDA"):
        layer.gradient_norm(t)
    with pytest.raises(ValueError, match="norm_type"):
        layer.clip_gradients([t], 1.0, norm_type=1.0)
    with pytest.raises(ValueError, match="every gradient"):
        layer.clip_gradients([t], 1.0, out=[])
    with forward_ad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
        layer.clip_gradients([forward_ad.make_dual(t, t)], 1.0)
