"""The device's record keeps a wait that ran out and an id outside its table apart, whichever came first.  The wait that runs out is the
library's self-test, bounded by construction; an id outside the table reads nothing."""
import itertools

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("order", list(itertools.permutations(["wait", "forward", "backward"])) + [("backward", "wait", "backward")])
def test_neither_covers_the_other(order):
    import torch
    from paper_1911_04070_b200 import binding
    block = torch.zeros(256, dtype=torch.uint8, device="cuda:0")
    ids, w = torch.tensor([1, 2, 99], device="cuda:0"), torch.ones(5, 8, device="cuda:0")
    while binding.bpt_check_device():
        pass
    acts = {"wait": lambda: binding.bpt_selftest_wait_timeout(block, 2000, arrive=False), "forward": lambda: binding.bpt_embed_fwd(ids, w),
            "backward": lambda: binding.bpt_embed_bwd(ids, torch.ones(3, 8, device="cuda:0"), 5, torch.float32)}
    for a in order:
        acts[a]()
    assert [binding.bpt_check_device() for _ in range(3)] == [5, 8, 0]
    for a in order:
        if a != "wait":
            acts[a]()
    assert [binding.bpt_check_device() for _ in range(2)] == [8, 0]


def test_the_sort_beyond_one_launch_reports_too():
    import torch
    from paper_1911_04070_b200 import binding
    while binding.bpt_check_device():
        pass
    ids = torch.zeros(140000, dtype=torch.int64, device="cuda:0")
    d = torch.ones(140000, 8, device="cuda:0")
    binding.bpt_embed_bwd(ids, d, 5, torch.float32)
    assert binding.bpt_check_device() == 0
    ids[139999] = -3
    dw = binding.bpt_embed_bwd(ids, d, 5, torch.float32)
    assert [binding.bpt_check_device() for _ in range(2)] == [8, 0]
    assert bool((dw[0] == 139999).all()) and not dw[1:].any()
