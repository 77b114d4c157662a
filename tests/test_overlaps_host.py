"""Which tensors share memory, as the calls that write tensors ask: against the sets of bytes written out.  No GPU needed."""
import itertools
import random

import pytest
import torch


@pytest.fixture(scope="module")
def share():
    from paper_1911_04070_b200 import build, binding
    build.build()
    return binding.load_native().share_memory


def _bytes(t):
    """Per element, the bytes that it takes."""
    e = t.element_size()
    for at in itertools.product(*map(range, t.shape)):
        p = t.data_ptr() + e * sum(i * s for i, s in zip(at, t.stride()))
        yield range(p, p + e)


def _meet(a, b):
    return bool({x for r in _bytes(a) for x in r} & {x for r in _bytes(b) for x in r})


def _meets_itself(a):
    all_bytes = [x for r in _bytes(a) for x in r]
    return len(set(all_bytes)) < len(all_bytes)


BUF = torch.zeros(4096)


def _view(rng):
    t = BUF if rng.random() < 0.5 else BUF.view(torch.bfloat16)
    d = rng.randint(0, 4)
    size, stride = [rng.randint(0 if rng.random() < 0.03 else 1, 5) for _ in range(d)], [rng.choice([0, 1, 1, 2, 3, 4, 5, 8, 16, 17, 20, 60]) for _ in range(d)]
    return t.as_strided(size, stride, rng.randint(0, 300))


def test_random_views(share):
    rng, met = random.Random(1), 0
    for _ in range(6000):
        a, b = _view(rng), _view(rng)
        want = _meet(a, b)
        met += want
        assert share(a, b) == want and share(b, a) == want, (a.shape, a.stride(), a.storage_offset(), b.shape, b.stride(), b.storage_offset())
        assert share(a) == _meets_itself(a), (a.shape, a.stride())
    assert 500 < met < 5500         # the draw has enough of both: 592 of 6000


def test_views_of_large_tensors(share):
    """What a program does with its buffers, at sizes where elements cannot be tried one by one."""
    big = torch.empty(1 << 14, 3, 8, 128, dtype=torch.bfloat16)
    q, k, v = big.unbind(1)
    assert not share(q, k) and not share(k, v) and share(q, q.transpose(1, 2)) and share(big, v) and not share(q) and not share(big)
    assert not share(big[..., ::2], big[..., 1::2]) and share(big[..., ::2], big[..., ::3]) and not share(big[::2], big[1::2])
    wide = torch.empty(20000, 3 * 1000)
    left, middle = wide[:, :1000], wide[:, 1000:2000]
    assert not share(left, middle) and share(left, wide[:, 999:1999]) and not share(left.t(), middle.t()) and share(left.t(), wide[:, 500:700])
    assert not share(left[:, ::2], left[:, 1::2]) and share(wide[:1].expand(9, -1)) and not share(wide.t())
    assert share(wide.view(-1).as_strided((1000, 1000), (999, 1))) and not share(wide.view(-1).as_strided((1000, 1000), (1000, 1)))
    assert not share(wide[:10], wide[10:]) and not share(wide, torch.empty(5)) and not share(wide[:, :0], wide)
