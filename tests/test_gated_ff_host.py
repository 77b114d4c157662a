"""Host side of bpt_gated_ff: refusals before anything is launched, the workspace query, and the oracle of the block
against PyTorch's own float64 operators and against finite differences.  No GPU needed."""
import pytest
import torch

from oracle import bpt_layer

A = 1 << 12     # an aligned address that no refused call may touch


@pytest.fixture(scope="module")
def lib():
    from paper_1911_04070_b200 import build, binding
    build.build()
    return binding.load_library()


def _fwd(lib, rows=4, D=64, F=128, act=1, ws=A, n=1 << 40, **p):
    ptr = dict(x=A, w_gate=A, w_up=A, w_down=A, y=A)
    ptr.update(p)
    return lib.bpt_gated_ff_fwd(*ptr.values(), rows, D, F, act, None, ws, n, None)


def _bwd(lib, rows=4, D=64, F=128, act=1, ws=A, n=1 << 40, **p):
    ptr = dict(x=A, w_gate=A, w_up=A, w_down=A, dy=A, dx=A, dw_gate=A, dw_up=A, dw_down=A)
    ptr.update(p)
    return lib.bpt_gated_ff_bwd(*ptr.values(), rows, D, F, act, None, ws, n, None)


@pytest.mark.parametrize("call", [_fwd, _bwd])
@pytest.mark.parametrize("kw,status", [(dict(rows=-1), 1), (dict(D=0), 1), (dict(F=0), 1), (dict(act=3), 1), (dict(act=-1), 1), (dict(D=60), 2),
                                       (dict(F=4), 2), (dict(rows=(1 << 26) + 1), 2), (dict(D=32776), 2), (dict(x=None), 1), (dict(w_gate=None), 1),
                                       (dict(w_up=None), 1), (dict(w_down=None), 1), (dict(x=A + 8), 1), (dict(w_down=A + 2), 1), (dict(ws=None), 3),
                                       (dict(n=8), 3), (dict(ws=A + 128), 1)])
def test_refusals(lib, call, kw, status):
    assert call(lib, **kw) == status


def test_more_refusals(lib):
    assert _fwd(lib, y=None) == 1 and _fwd(lib, y=A + 4) == 1
    assert _bwd(lib, dy=None) == 1 and _bwd(lib, dx=A + 8) == 1
    assert _bwd(lib, dw_up=None) == 1 and _bwd(lib, dw_gate=None, dw_up=None) == 1     # three weight gradients or none
    assert _bwd(lib, dx=None, dw_gate=None, dw_up=None, dw_down=None) == 1
    assert _fwd(lib, rows=0, x=None, y=None, ws=None, n=0) == 0                         # nothing to do


def test_workspace_query(lib):
    q = lib.bpt_gated_ff_workspace_bytes
    assert q(0, 64, 128, 0) == 0 and q(4, 60, 128, 0) == 0 and q(-1, 64, 128, 1) == 0
    assert q(1000, 64, 128, 0) >= 1000 * 128 * 2
    assert q(1000, 64, 128, 1) >= 3 * 1000 * 128 * 2 + 3 * 64 * 128 * 4
    assert q(65532, 512, 2048, 1) <= 3 * 65532 * 2048 * 2 + 16 * 3 * 512 * 2048 * 4 + 4096


@pytest.mark.parametrize("act", ["relu", "silu", "gelu"])
def test_oracle_against_torch_and_differences(act):
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    v = dict(x=r(5, 6), w_gate=r(9, 6), w_up=r(9, 6), w_down=r(6, 9))
    F = torch.nn.functional
    f = {"relu": F.relu, "silu": F.silu, "gelu": F.gelu}[act]
    y = bpt_layer.gated_ff(**v, act=act)
    assert torch.allclose(y, (f(v["x"] @ v["w_gate"].T) * (v["x"] @ v["w_up"].T)) @ v["w_down"].T, rtol=1e-12, atol=1e-12)
    dy = r(5, 6)
    leaf = {a: t.clone().requires_grad_(True) for a, t in v.items()}
    (bpt_layer.gated_ff(**leaf, act=act) * dy).sum().backward()
    for name, t in v.items():
        d = r(*t.shape)
        step = 1e-6
        up, down = ((bpt_layer.gated_ff(**{**v, name: t + s * step * d}, act=act) * dy).sum() for s in (1, -1))
        want, got = float(up - down) / (2 * step), float((leaf[name].grad * d).sum())
        assert abs(got - want) <= 1e-6 * (1 + abs(want)), (name, got, want)     # 1e-16 * |loss| / step, and step^2


def test_few_rows_rule(lib):
    f = lib.bpt_gated_ff_few_rows
    assert f(1, 512, 2048) and f(128, 512, 2048) and not f(129, 512, 2048)
    assert f(16, 4096, 11008) and not f(17, 4096, 11008)         # a pass over large weights pays for sixteen rows
    assert f(384, 64, 128) and not f(385, 64, 128)
    assert not f(4, 60, 128) and not f(-1, 64, 128)              # invalid sizes
    assert lib.bpt_gated_ff_workspace_bytes(64, 512, 2048, 0) == 64 * 2048 * 4
