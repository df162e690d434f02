"""Matrices of more than 384 rows, whose products take 11 bits, on each of the kernels that they can take: tiles of 128 and of 256, the first two iterations
one after the other and in one, beside small matrices; as outputs, as steps and as decoded payloads."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref
from tests.guards import Guarded, all_intact
from tests.muon_plan import plan
from tests.test_gpu_muon_decode import payloads_of, received

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CODE = {F32: demo.DEMO_F32, BF16: demo.DEMO_BF16}
# name: matrices, tile, first two iterations in one
SETS = {
    "128": ([(401, 777), (900, 515), (777, 401)], 128, 0),
    "128, two in one": ([(500, 4003)] * 4 + [(4001, 500)], 128, 1),
    "256": ([(401, 777)] * 40 + [(515, 900)] * 2 + [(777, 401)] * 3, 256, 0),
    "256, two in one": ([(513, 1333)] * 40 + [(1333, 514)] * 3 + [(385, 387)], 256, 1),
    "beside small ones": ([(700, 900), (64, 100), (900, 2000), (2001, 388), (384, 384)], 128, 0),
}


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def takes(name):
    shapes, tile, two = SETS[name]
    large = [g for g in plan(shapes) if not g[0]]
    assert {g[1] for g in large} == {tile} and large[0][6] == two, "the set no longer takes the way that it is here for"
    return shapes


def documented(shape):  # of full rank
    return 1e-3 if min(shape) > 384 else 2e-5 + min(max(shape) * 2.0 ** -26, 6e-5)


def look(shapes):
    """The first and the last of each size."""
    return sorted({shapes.index(s) for s in shapes} | {len(shapes) - 1 - shapes[::-1].index(s) for s in shapes})


def test_sets_take_their_ways():
    for name in SETS:
        takes(name)


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_outputs(name, dtype):
    shapes = takes(name)
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    ins = [Guarded(s, dtype, "cuda", rand(s, i)) for i, s in enumerate(shapes)]
    outs = [Guarded(s, dtype, "cuda", rand(s, 5)) for s in shapes]
    for _ in range(2):
        tr.orthogonalize([u.t for u in ins], [o.t for o in outs])
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for i in look(shapes):
        want = ref.orthogonal(ins[i].t)
        # (bf16: half a step of each value beside it)
        assert float((outs[i].t.double() - want).norm() / want.norm()) <= documented(shapes[i]) + (2.0 ** -8 if dtype == BF16 else 0)
    assert all_intact(ins + outs)


@pytest.mark.parametrize("name", SETS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nesterov,scale", [(True, demo.DEMO_SCALE_RMS), (False, demo.DEMO_SCALE_ASPECT), (True, demo.DEMO_SCALE_NONE)])
def test_steps(name, dtype, nesterov, scale):
    shapes, mu = takes(name), 0.875
    tr = demo.MuonTransform(shapes, lr=0.02, weight_decay=0.1, momentum=mu, nesterov=nesterov, scale=scale, grad_dtype=CODE[dtype])
    g = [rand(s, i, 1e-2).to(dtype) for i, s in enumerate(shapes)]
    m = [Guarded(s, F32, "cuda", rand(s, 500 + i, 1e-2)) for i, s in enumerate(shapes)]
    x = [Guarded(s, F32, "cuda", rand(s, 900 + i)) for i, s in enumerate(shapes)]
    for n in range(2):
        if n == 1:
            tr.set_lr(0.005)
        lr = 0.005 if n == 1 else 0.02
        at = look(shapes)
        before = {i: (m[i].t.clone(), x[i].t.clone()) for i in at}
        tr.step(g, [t.t for t in m], [t.t for t in x])
        torch.cuda.synchronize()
        assert tr.device_status() == 0
        for i in at:
            m0, x0 = before[i]
            wm, wx = ref.muon_step(g[i], m0, x0, lr=lr, wd=0.1, mu=mu, nesterov=nesterov, scale=scale)
            # one rounding of the momentum; x: the update's error and two roundings of its own (1 - lr wd and the sum)
            assert bool(((m[i].t.double() - wm).abs() <= 2.0 ** -24 * wm.abs() + 1e-40).all())
            assert float((x[i].t.double() - wx).norm()) <= documented(shapes[i]) * float((wx - x0.double()).norm()) + 2 * 2.0 ** -24 * float(wx.norm())
    assert all_intact(m + x)


@pytest.mark.parametrize("name", SETS)
def test_a_step_is_the_orthogonalisation(name):
    """Without momentum, decay and factor x is x - lr O(g), to the bit; in place, too."""
    shapes = takes(name)
    tr = demo.MuonTransform(shapes, momentum=0.0, nesterov=False, weight_decay=0.0, lr=1.0, scale=demo.DEMO_SCALE_NONE, grad_dtype=demo.DEMO_F32)
    g = [rand(s, i) for i, s in enumerate(shapes)]
    o, m, x = ([torch.zeros(s, device="cuda") for s in shapes] for _ in range(3))
    tr.orthogonalize(g, o)
    tr.step(g, m, x)
    assert all(torch.equal(-a, b) for a, b in zip(o, x))
    assert all(torch.equal(a, b) for a, b in zip(g, m))
    tr.orthogonalize(m, m)
    assert all(torch.equal(a, b) for a, b in zip(o, m))
    torch.cuda.synchronize()
    assert tr.device_status() == 0


@pytest.mark.parametrize("name", SETS)
def test_captured_steps(name):
    shapes = takes(name)
    tr, eager = (demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1) for _ in range(2))
    g = [rand(s, i, 1e-2).bfloat16() for i, s in enumerate(shapes)]
    state = [[rand(s, k * 100 + i, 1e-2) for i, s in enumerate(shapes)] for k in (1, 2)]
    other = [[t.clone() for t in ts] for ts in state]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        tr.step(g, *state)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            tr.step(g, *state)
        for _ in range(3):
            graph.replay()
    for _ in range(4):
        eager.step(g, *other)
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and eager.device_status() == 0
    for a, b in zip(state, other):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 8])
@pytest.mark.parametrize("name", ["128", "128, two in one", "256", "256, two in one"])
@pytest.mark.parametrize("coefficients", [ref.COEFFICIENTS, (1.875, -1.25, 0.375)])
def test_steps_and_coefficients(name, steps, coefficients):
    shapes = SETS[name][0]
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1, steps=steps, coefficients=coefficients)
    ins, outs = [rand(s, i) for i, s in enumerate(shapes)], [torch.full(s, float("nan"), device="cuda") for s in shapes]
    tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for i in look(shapes):
        want = ref.orthogonal(ins[i], steps=steps, coefficients=coefficients)
        assert float((outs[i].double() - want).norm() / want.norm()) <= ref.tolerance(shapes[i])


@pytest.mark.parametrize("chunk,shapes,tile", [(64, [(448, 576)] * 60 + [(512, 1600)] * 20 + [(1600, 448)] * 10 + [(640,)], 256),
                                               (64, [(64,), (512, 1536), (448, 448), (128, 192)], 128), (32, [(416, 1216)] * 2 + [(96,)], 128)])
def test_decoded_payloads(chunk, shapes, tile):
    matrices = [s for s in shapes if len(s) == 2]
    assert {g[1] for g in plan(matrices) if not g[0]} == {tile}
    dm = demo.DemoTransform(shapes, chunk=chunk, topk=32, beta=0.9, lr=3e-3, weight_decay=0.05, num_workers=3)
    mu = demo.MuonTransform(matrices, lr=1e-2, weight_decay=0.1)
    ps = payloads_of(dm, shapes)
    rs = received(dm, shapes, chunk, 32, ps, demo.DEMO_AGG_SUM)
    x = [Guarded(s, F32, "cuda", rand(s, 70 + i)) for i, s in enumerate(shapes)]
    at = sorted(set(look(shapes)))
    for _ in range(2):
        x0 = [t.t.double() for t in x]
        mu.decode_apply(dm, ps, [t.t for t in x])
        torch.cuda.synchronize()
        assert mu.device_status() == 0 and dm.device_status() == 0
        for i in at:
            got, w0, r = x[i].t, x0[i], rs[i]
            if got.dim() == 1:
                want = w0 - 3e-3 * (torch.sign(r) + 0.05 * w0)
                assert ((got - want).abs() <= 1e-6 * want.abs() + 1e-6 + 6.1e-3 * (r.abs() < 1e-5)).all()
            else:
                want = w0 - 1e-2 * (ref.scale_of(2, got.shape) * ref.orthogonal(r) + 0.1 * w0)
                # (a few coefficients a chunk: the rank need not be full)
                assert float((got - want).norm()) <= (2e-3 if min(got.shape) > 384 else 4e-4) * float((want - w0).norm()) + 2 * 2.0 ** -24 * float(want.norm())
    assert all_intact(x)


def test_refused_decodes_leave_everything_as_it_was():
    shapes = [(448, 512), (64,)]
    dm = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=3)
    mu = demo.MuonTransform(shapes[:1], lr=1e-2, weight_decay=0.1)
    ps, x = payloads_of(dm, shapes), [rand(s, i) for i, s in enumerate(shapes)]
    before = [t.clone() for t in x]
    refused = 0
    for ctx, payloads, params in ((mu, ps[:2], x), (mu, ps, x[:1]), (mu, ps, x[::-1]), (mu, ps + ps[:1], x), (mu, ps, [x[0].bfloat16(), x[1]]),
                                  (demo.MuonTransform([(512, 448)], lr=1e-2, weight_decay=0.1), ps, x),
                                  (demo.MuonTransform(shapes[:1] * 2, lr=1e-2, weight_decay=0.1), ps, x)):
        with pytest.raises((ValueError, demo.DemoError)):
            ctx.decode_apply(dm, payloads, params)
        refused += 1
    torch.cuda.synchronize()
    assert refused == 7 and all(torch.equal(a, b) for a, b in zip(x, before))
    mu.decode_apply(dm, ps, x)
    torch.cuda.synchronize()
    assert not torch.equal(x[0], before[0]) and not torch.equal(x[1], before[1])
