"""AdamW in one launch against 64 bits: sizes, types, the step count on the device, captured graphs."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref
from tests.guards import Guarded, all_intact

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
U = 2.0 ** -24


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def tensors(shapes, dtype, guard=True):
    make = (lambda s, d, v: Guarded(s, d, "cuda", v)) if guard else (lambda s, d, v: v.to(d))
    g = [rand(s, i, 1e-2).to(dtype) for i, s in enumerate(shapes)]
    m = [make(s, F32, rand(s, 100 + i, 1e-2)) for i, s in enumerate(shapes)]
    v = [make(s, F32, rand(s, 200 + i, 1e-2).square()) for i, s in enumerate(shapes)]
    x = [make(s, F32, rand(s, 300 + i)) for i, s in enumerate(shapes)]
    return g, m, v, x


SETS = [[(1,)], [(7,), (2048,), (2049,), (3,)], [(2047, 3), (5,), (4, 4, 4, 4)], [(i % 9 + 1,) for i in range(300)], [(1000, 1001), (1,)], [(4096, 4096)]]


@pytest.mark.parametrize("shapes", SETS, ids=range(len(SETS)))
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_steps(shapes, dtype):
    tr = demo.AdamwTransform(shapes, lr=1e-2, weight_decay=0.1, beta1=0.9, beta2=0.999, grad_dtype=demo.DEMO_F32 if dtype == F32 else demo.DEMO_BF16)
    g, m, v, x = tensors(shapes, dtype)
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    for t in (1, 2, 3):
        if t == 3:
            tr.set_lr(1e-3)
        lr = 1e-3 if t == 3 else 1e-2
        want = [ref.adamw_step(gi, mi.t, vi.t, xi.t, t, lr=lr, wd=0.1, beta2=0.999) for gi, mi, vi, xi in zip(g, m, v, x)]
        tr.step(g, [i.t for i in m], [i.t for i in v], [i.t for i in x], count)
        torch.cuda.synchronize()
        assert int(count) == t
        for mi, vi, xi, (wm, wv, wx) in zip(m, v, x, want):
            # three roundings of each product and sum at most, of values no larger than these; x: those of the update (six) beside its own
            assert ((mi.t - wm).abs() <= 3 * U * (wm.abs() + 0.1)).all()
            assert ((vi.t - wv).abs() <= 4 * U * wv.abs() + 1e-38).all()
            upd = (wx - xi.t.double()).abs()
            assert (upd <= 3 * U * wx.abs() + 12 * U * lr * ((wm / (1 - 0.9 ** t)).abs() + 0.1) / ((wv / (1 - 0.999 ** t)).sqrt() + 1e-8)).all()
    assert all_intact(m + v + x)
    assert tr.launch_count == 3


def test_captured_steps_count_on():
    shapes = [(1000,), (300, 70)]
    mk = lambda: demo.AdamwTransform(shapes, lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32)  # noqa: E731
    a, b = mk(), mk()
    sa, sb = tensors(shapes, F32, False), tensors(shapes, F32, False)
    ca, cb = (torch.full((1,), 5, dtype=torch.int64, device="cuda") for _ in range(2))
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        a.step(*sa, ca)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            a.step(*sa, ca)
    for _ in range(4):
        graph.replay()
    for _ in range(5):
        b.step(*sb, cb)
    torch.cuda.synchronize()
    assert int(ca) == int(cb) == 10
    for u, w in zip(sa, sb):
        assert all(torch.equal(p, q) for p, q in zip(u, w))


def test_capture_with_new_pointers_is_refused():
    shapes = [(64,)]
    tr = demo.AdamwTransform(shapes, lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32)
    s, count = tensors(shapes, F32, False), torch.zeros(1, dtype=torch.int64, device="cuda")
    tr.step(*s, count)
    torch.cuda.synchronize()
    other = tensors(shapes, F32, False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(torch.cuda.Stream()):
        graph.capture_begin()
        with pytest.raises(demo.DemoError) as e:
            tr.step(*other, count)
        tr.step(*s, count)
        graph.capture_end()
    assert e.value.status == 1
    graph.replay()
    torch.cuda.synchronize()
    assert int(count) == 2
