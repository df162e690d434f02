"""Sets whose products have one step of K: a worker's two CTAs pass tasks to each other faster than any other set makes them do."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape,count,calls", [((1, 1 << 20), 16, 12), ((1 << 17, 100), 16, 12), ((128, 128), 3000, 20), ((3, 5), 20000, 20), ((128, 30000), 40, 12)])
def test_many_tasks_of_one_step(shape, count, calls):
    shapes = [shape] * count
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    gen = torch.Generator("cuda").manual_seed(1)
    flat = torch.randn((count,) + shape, generator=gen, device="cuda")
    out = [torch.empty_like(flat) for _ in range(2)]
    lists = [list(o.unbind(0)) for o in out]
    # rows of a stack are 16-byte aligned where their size is a multiple of it; others are copied out
    ins = list(flat.unbind(0))
    if shape[0] * shape[1] % 4:
        ins = [t.clone() for t in ins]
        lists = [[t.clone() for t in l] for l in lists]
    for _ in range(calls):
        for l in lists:
            tr.orthogonalize(ins, l)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    assert all(torch.equal(a, b) for a, b in zip(*lists))
    for i in (0, count // 2, count - 1):
        want = ref.orthogonal(ins[i])
        assert float((lists[0][i].double() - want).norm() / want.norm()) <= 2e-5 + 6e-5
