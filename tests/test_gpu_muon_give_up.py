"""Waits of the products' kernel that run out: the kernel ends, the status says so once, and the calls that follow are as good as any.  No GPU fault is
involved: tasks are started while the product that they need never comes, with a short limit."""
import time

import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu
TIMEOUT = 7


def rand(shape, seed):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda")


# tiles of 128 with hi and lo parts, of 128, of 256 (many), both kinds, several tiles in the product that waits
SETS = [[(100, 130)], [(300, 700)], [(500, 700)], [(600, 700)] * 160, [(64, 100), (900, 1100)]]


@pytest.mark.parametrize("shapes", SETS, ids=range(len(SETS)))
def test_the_context_survives(shapes):
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    want, outs = ([torch.empty(s, device="cuda") for s in shapes] for _ in range(2))
    tr.orthogonalize(ins, want)
    assert tr.device_status() == 0
    tr.selftest_bounded_wait(2_000_000)  # ~1 ms
    tr.orthogonalize(ins, outs)  # the status not asked for
    assert tr.device_status() == TIMEOUT
    assert tr.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(outs, want))
    exact = ref.orthogonal(ins[-1])
    assert float((outs[-1].double() - exact).norm() / exact.norm()) <= 1e-3


def test_waits_last_as_long_as_they_may():
    tr = demo.MuonTransform([(500, 700)], lr=1e-2, weight_decay=0.1)
    tr.selftest_bounded_wait(2_000_000)
    torch.cuda.synchronize()
    t0 = time.perf_counter()
    tr.selftest_bounded_wait(40_000_000)
    torch.cuda.synchronize()
    assert time.perf_counter() - t0 > 40e6 / 2.1e9  # (the clock is below 2.1 GHz)
    assert tr.device_status() == TIMEOUT and tr.device_status() == 0


def test_limits():
    tr = demo.MuonTransform([(10, 20)], lr=1e-2, weight_decay=0.1)
    for limit in (0, -1, 2_000_000_001):
        with pytest.raises(demo.DemoError) as e:
            tr.selftest_bounded_wait(limit)
        assert e.value.status == 1
