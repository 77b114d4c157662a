"""Host side of bpt_res_norm: refusals before anything is launched, the workspace query, and the oracle of the seam
against finite differences and against PyTorch's own float64 operators.  No GPU needed."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import bpt_layer


@pytest.fixture(scope="module")
def lib():
    from paper_1911_04070_b200 import build, binding
    build.build()
    return binding.load_library()


def _args(**kw):
    from paper_1911_04070_b200 import binding
    a = dict(rows=4, gate_groups=1, D=32, dtype=0, param_dtype=0, gate_dtype=0, norm=1, post_norm=0, alpha=1.0, eps=1e-5, h=4096, b=4096)
    a.update(kw)
    return binding.ResNormArgs(**a)


@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(D=0), 1), (dict(D=8193), 2), (dict(rows=1 << 31), 2), (dict(dtype=2), 1),
                                       (dict(param_dtype=7), 1), (dict(gate_dtype=-1), 1), (dict(norm=3), 1), (dict(post_norm=-1), 1),
                                       (dict(eps=float("nan")), 1), (dict(eps=-1.0), 1), (dict(b=None, post_norm=1), 1), (dict(b=None, gate=4096), 1),
                                       (dict(norm=0, weight=4096), 1), (dict(post_weight=4096), 1), (dict(gate=4096, gate_groups=3), 1),
                                       (dict(gate=4096, gate_groups=0), 1), (dict(h=None), 1), (dict(h=4098), 1), (dict(b=4097), 1)])
def test_refusals(lib, kw, status):
    a = _args(**kw)
    y = None if kw.get("norm") == 0 else 8192
    assert lib.bpt_res_norm_fwd(ctypes.byref(a), y, 8192, None, None) == status
    assert lib.bpt_res_norm_bwd(ctypes.byref(a), 8192, None, None, 8192, None, None, None, None, None, None, 8192, 1 << 30, None) == status


def test_more_refusals(lib):
    a = _args()
    assert lib.bpt_res_norm_fwd(None, 8192, None, None, None) == 1
    assert lib.bpt_res_norm_fwd(ctypes.byref(a), None, 8192, None, None) == 1                    # a norm without y
    assert lib.bpt_res_norm_fwd(ctypes.byref(_args(norm=0)), 8192, 8192, None, None) == 1        # y without a norm
    assert lib.bpt_res_norm_fwd(ctypes.byref(_args(norm=0)), None, None, None, None) == 1
    assert lib.bpt_res_norm_fwd(ctypes.byref(a), 8192, None, 8200, None) == 1              # stats off its boundary
    bwd = lambda a, dy=8192, ws=8192, n=1 << 30, stats=8192, **o: lib.bpt_res_norm_bwd(
        ctypes.byref(a), stats, dy, None, *[o.get(k) for k in ("dh", "db", "dw", "dc", "dpw", "dpc", "dg")], ws, n, None)
    assert bwd(a, ws=None) == 3 and bwd(a, n=0) == 3 and bwd(a, ws=8200) == 1
    assert bwd(a, stats=None) == 1 and bwd(a, stats=8196) == 1
    assert bwd(_args(norm=0)) == 1                                                         # dy without a norm
    assert bwd(_args(b=None), db=8192) == 1 and bwd(a, dw=8192) == 1 and bwd(a, dpc=8192) == 1 and bwd(a, dg=8192) == 1


def test_workspace_query(lib):
    q = lambda **kw: lib.bpt_res_norm_bwd_workspace_bytes(ctypes.byref(_args(**kw)))
    assert q(D=0) == 0 and lib.bpt_res_norm_bwd_workspace_bytes(None) == 0
    assert q(rows=0) >= 4 * 32 * 4
    assert q(rows=1 << 20) <= 148 * 2 * 4 * 32 * 4
    assert q(rows=1 << 20, gate=4096, gate_groups=2) > q(rows=1 << 20)
    assert q(rows=1 << 20, gate=4096, gate_groups=1 << 20) == q(rows=1 << 20)             # a gate per row needs no sums


def _problem(norm, post, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    x = dict(h=r(3, 4, 7), b=r(3, 4, 7), gate=r(3, 1, 7))
    for pre, kind in (("", norm), ("post_", post)):
        x[pre + "weight"] = r(7) if kind else None
        x[pre + "bias"] = r(7) if kind else None
    return x, dict(norm=norm, post_norm=post, alpha=0.7, eps=1e-3), r(3, 4, 7), r(3, 4, 7)


@pytest.mark.parametrize("norm,post", [("layer", None), ("rms", "layer"), ("layer", "rms"), (None, "layer")])
def test_oracle_against_torch_and_differences(norm, post):
    x, cfg, dy, dr = _problem(norm, post, 0)
    F = torch.nn.functional
    ref = {None: lambda v, w, c: v, "layer": lambda v, w, c: F.layer_norm(v, (7,), w, c, 1e-3), "rms": lambda v, w, c: F.rms_norm(v, (7,), w, 1e-3) + c}
    y, r = bpt_layer.res_norm(**x, **cfg)
    r_ref = 0.7 * x["h"] + x["gate"] * ref[post](x["b"], x["post_weight"], x["post_bias"])
    assert torch.allclose(r, r_ref, rtol=1e-13, atol=1e-13)
    assert torch.allclose(y, ref[norm](r_ref, x["weight"], x["bias"]), rtol=1e-12, atol=1e-12)
    loss = lambda x: float(sum((a * b).sum() for a, b in zip(bpt_layer.res_norm(**x, **cfg), (dy, dr))))
    leaf = {a: None if v is None else v.clone().requires_grad_(True) for a, v in x.items()}
    yl, rl = bpt_layer.res_norm(**leaf, **cfg)
    ((yl * dy).sum() + (rl * dr).sum()).backward()
    for name, v in x.items():
        if v is None:
            continue
        t = torch.randn(v.shape, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
        step = 1e-5
        up, down = ({**x, name: v + s * step * t} for s in (1, -1))
        want = (loss(up) - loss(down)) / (2 * step)
        got = float((leaf[name].grad * t).sum())
        assert abs(got - want) <= 1e-6 * (1 + abs(want)), (name, got, want)   # step^2 of the third derivative, and 1e-16 / step


def test_argument_struct_matches_the_header():
    from paper_1911_04070_b200 import binding
    a = binding.ResNormArgs
    assert ctypes.sizeof(a) == 8 + 8 + 4 * 6 + 8 + 7 * 8 and a.h.offset == 48 and a.gate.offset == 96
