"""Sets that go through the workspace of the iterations in several groups: thin matrices, small ones, small and larger ones side by side."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu
GROUP_BYTES, GROUP_ELEMENTS = 26 << 27, 1 << 27


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def check(shapes, look, bound):
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    first, again = ([torch.full(s, float("nan"), device="cuda") for s in shapes] for _ in range(2))
    tr.orthogonalize(ins, first)
    tr.orthogonalize(ins, again)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    for i in look:
        want = ref.orthogonal(ins[i])
        assert float((first[i].double() - want).norm() / want.norm()) <= bound(shapes[i])
    return tr


def documented(shape):
    return 1e-3 if min(shape) > 384 else 2e-5 + min(max(shape) * 2.0 ** -26, 6e-5)


# one row of 2^20 takes 145 bytes an element, of 384 x 384 24
@pytest.mark.parametrize("shapes", [[(1, 1 << 20)] * 64, [(1 << 17, 2)] * 300, [(40, 60)] * 300 + [(1, 1 << 20)] * 40], ids=["rows", "columns", "mixed"])
def test_thin_matrices_share_a_workspace(shapes):
    tr = check(shapes, [0, 1, 23, 24, len(shapes) // 2, len(shapes) - 1], documented)
    assert tr.workspace_bytes < GROUP_BYTES + (64 << 20)  # (tables, tasks)


def test_several_groups_of_small_matrices():
    shapes = [(384, 384)] * 1100 + [(100, 300)] * 3  # 162 million elements
    assert sum(a * b for a, b in shapes) > GROUP_ELEMENTS
    n = GROUP_ELEMENTS // 384 ** 2
    check(shapes, [0, n - 1, n, n + 1, 1099, 1100, 1102], documented)


def test_several_groups_of_both_kinds_side_by_side():
    shapes = [(384, 380), (3000, 2000)] * 25 + [(300, 301)] * 1500
    assert sum(a * b for a, b in shapes if min(a, b) <= 384) > GROUP_ELEMENTS and sum(a * b for a, b in shapes if min(a, b) > 384) > GROUP_ELEMENTS
    check(shapes, [0, 1, 42, 43, 44, 45, 46, 49, 50, 1000, 1446, 1500, 1549], documented)


def test_a_step_of_several_groups():
    shapes = [(384, 384)] * 1000 + [(2000, 3000)] * 24
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    g = [rand(s, i, 1e-2).bfloat16() for i, s in enumerate(shapes)]
    m, x = ([rand(s, k * 5000 + i, 1e-2) for i, s in enumerate(shapes)] for k in (1, 2))
    m0, x0 = [t.clone() for t in m], [t.clone() for t in x]
    tr.step(g, m, x)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for i in (0, 909, 910, 911, 999, 1000, 1021, 1022, 1023):
        wm, wx = ref.muon_step(g[i], m0[i], x0[i], lr=1e-2, wd=0.1)
        # momentum: a product and a sum, rounded once each; x: the update's error and its own two roundings
        assert float((m[i].double() - wm).abs().max()) <= 2 * 2.0 ** -24 * float(wm.abs().max())
        assert float((x[i].double() - wx).norm()) <= documented(shapes[i]) * float((wx - x0[i].double()).norm()) + 2 * 2.0 ** -24 * float(wx.norm())
