"""Host side of bpt_embed: refusals before anything is launched, the workspace query, and what layer.token_states refuses.  No GPU needed."""
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
    a = dict(batch=2, tokens=8, out_rows=15, vocab=100, padding_idx=-1, D=32, id_bytes=8, weight_dtype=1, out_dtype=1, scale=1.0, ids=4096, weight=4096)
    a.update(kw)
    return binding.EmbedArgs(**a)


@pytest.mark.parametrize("kw,status", [(dict(batch=-1), 1), (dict(tokens=-1), 1), (dict(out_rows=7), 1), (dict(vocab=0), 1), (dict(D=0), 1), (dict(id_bytes=2), 1),
                                       (dict(weight_dtype=2), 1), (dict(out_dtype=-1), 1), (dict(scale=float("nan")), 1), (dict(scale=float("inf")), 1),
                                       (dict(padding_idx=100), 1), (dict(padding_idx=-2), 1), (dict(vocab=1 << 30), 2), (dict(D=(1 << 20) + 1), 2),
                                       (dict(batch=1 << 20, out_rows=1 << 20), 2), (dict(batch=1, tokens=1, out_rows=1 << 29, D=1 << 20), 2),
                                       (dict(ids=None), 1), (dict(ids=4100), 1), (dict(lengths=4098), 1)])
def test_refusals(lib, kw, status):
    a = _args(**kw)
    assert lib.bpt_embed_fwd(ctypes.byref(a), 8192, None) == status
    assert lib.bpt_embed_bwd(ctypes.byref(a), 8192, 8192, 8192, 1 << 50, None) == status
    if status == 2 or kw.keys() & {"batch", "tokens", "out_rows", "D"}:
        assert lib.bpt_embed_bwd_workspace_bytes(ctypes.byref(a)) == 0


def test_more_refusals(lib):
    a = _args()
    assert lib.bpt_embed_fwd(None, 8192, None) == 1 and lib.bpt_embed_fwd(ctypes.byref(a), None, None) == 1
    assert lib.bpt_embed_fwd(ctypes.byref(a), 8193, None) == 1                                   # out off its element
    assert lib.bpt_embed_fwd(ctypes.byref(_args(weight=None)), 8192, None) == 1
    assert lib.bpt_embed_fwd(ctypes.byref(_args(weight=4097)), 8192, None) == 1
    bwd = lambda a=a, d=8192, w=8192, ws=8192, n=1 << 50: lib.bpt_embed_bwd(a if a is None else ctypes.byref(a), d, w, ws, n, None)
    assert bwd(None) == 1 and bwd(d=None) == 1 and bwd(w=None) == 1 and bwd(d=8193) == 1 and bwd(w=8193) == 1
    assert bwd(ws=None) == 3 and bwd(n=lib.bpt_embed_bwd_workspace_bytes(ctypes.byref(a)) - 1) == 3 and bwd(ws=8200) == 1


def test_nothing_to_do(lib):
    assert lib.bpt_embed_fwd(ctypes.byref(_args(batch=0, ids=None, weight=None)), None, None) == 0
    assert lib.bpt_embed_fwd(ctypes.byref(_args(tokens=0, out_rows=0, ids=None, weight=None)), None, None) == 0


def test_workspace_query(lib):
    q = lambda **kw: lib.bpt_embed_bwd_workspace_bytes(ctypes.byref(_args(**kw)))
    assert q(tokens=0, out_rows=0) >= 16
    assert q(vocab=1 << 20) == q(vocab=100)              # no table of the vocabulary's length
    assert lib.bpt_embed_bwd_workspace_bytes(None) == 0


@pytest.fixture(scope="module")
def layer(lib):
    from paper_1911_04070_b200 import layer
    return layer


def test_python_refusals(layer):
    ids, w = torch.zeros(2, 4, dtype=torch.int64), torch.zeros(5, 8)
    with pytest.raises(ValueError, match="CUDA"):
        layer.token_states(ids, w)
    with pytest.raises(TypeError, match="int32 or int64"):
        layer.token_states(ids.float(), w)
    with pytest.raises(TypeError, match="float32 and bfloat16"):
        layer.token_states(ids, w.half())
    with pytest.raises(TypeError, match="float32 and bfloat16"):
        layer.token_states(ids, w, dtype=torch.float16)
    with pytest.raises(ValueError, match="weight"):
        layer.token_states(ids, w[0])
    for pad in (5, -1):
        with pytest.raises(ValueError, match="padding_idx"):
            layer.token_states(ids, w, padding_idx=pad)
    with pytest.raises(NotImplementedError, match="scale"):
        layer.token_states(ids, w, scale=torch.ones((), requires_grad=True))


def test_modes_are_refused(layer):
    ids, w = torch.zeros(2, 4, dtype=torch.int64), torch.zeros(5, 8)
    with forward_ad.dual_level(), pytest.raises(NotImplementedError, match="forward-mode"):
        layer.token_states(ids, forward_ad.make_dual(w, torch.ones_like(w)))
    with pytest.raises(NotImplementedError, match="traced"):
        torch.jit.trace(lambda t: layer.token_states(ids, t), (w,), check_trace=False)
