"""The device's failure record: what a bounded wait that ran out leaves there survives the calls that follow, is reported once, and
is what a training loop looks at, whose backward calls have no status block that it could reach.  The wait that runs out is the
library's self-test: bounded by construction, nothing faults or hangs."""
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture
def record():
    import torch
    from paper_1911_04070_b200 import binding
    block = torch.zeros(256, dtype=torch.uint8, device="cuda:0")
    binding.bpt_check_device()                  # what earlier self-tests left
    assert binding.bpt_check_device() == 0

    def give_up(arrive=False):
        binding.bpt_selftest_wait_timeout(block, 2000, arrive=arrive)
        return block
    return give_up


def _step(rows, D=64, F=128):
    import torch
    from paper_1911_04070_b200 import layer
    t = lambda *s: (torch.randn(*s, device="cuda:0") * 0.1).bfloat16().requires_grad_(True)
    x, wg, wu, wd = t(rows, D), t(F, D), t(F, D), t(D, F)
    y = layer.gated_feed_forward(x, wg, wu, wd)
    y.backward(torch.ones_like(y))
    return y


def test_reported_once(record):
    import torch
    from paper_1911_04070_b200 import binding
    block = record()
    assert binding.bpt_check(block) == 5 and binding.bpt_check(None) == 0
    assert binding.bpt_check_device() == 5
    assert binding.bpt_check_device() == 0 and binding.bpt_check_device("cuda:0") == 0
    record(arrive=True)
    assert binding.bpt_check_device(torch.device("cuda", 0)) == 0


@pytest.mark.parametrize("rows", [5, 64, 500, 3000])
def test_a_training_step_neither_sets_nor_clears_it(record, rows):
    from paper_1911_04070_b200 import binding
    y = _step(rows)
    assert binding.bpt_check_device() == 0 and binding.bpt_check(y._bpt_workspace) == 0
    record()
    y = _step(rows)                             # the calls clear their own blocks only
    assert binding.bpt_check(y._bpt_workspace) == 0
    assert binding.bpt_check_device() == 5 and binding.bpt_check_device() == 0


def test_from_another_stream(record):
    import torch
    from paper_1911_04070_b200 import binding
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        record()
        assert binding.bpt_check_device() == 5
    assert binding.bpt_check_device() == 0


_FIRST = r"""
import torch
from paper_1911_04070_b200 import binding
t = lambda *s: torch.randn(*s, device="cuda:0").bfloat16()
x, wg, wu, wd = t(500, 64), t(128, 64), t(128, 64), t(64, 128)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    y = binding.bpt_gated_ff_fwd(x, wg, wu, wd)
    g = binding.bpt_gated_ff_bwd(x, wg, wu, wd, y)
graph.replay()
torch.cuda.synchronize()
want = binding.bpt_gated_ff_fwd(x, wg, wu, wd)
assert torch.equal(y, want) and all(torch.equal(a, b) for a, b in zip(g, binding.bpt_gated_ff_bwd(x, wg, wu, wd, want)))
assert binding.bpt_check_device() == 0
print("captured")
"""


def test_the_first_calls_of_a_process_can_be_captured():
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured" in r.stdout, r.stdout + r.stderr
