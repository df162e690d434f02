"""Orthogonalised updates against 64 bits: sizes, types, scales, steps, streams, captured graphs."""
import math

import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref
from tests.guards import Guarded, all_intact

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CODE = {F32: demo.DEMO_F32, BF16: demo.DEMO_BF16}


def muon(shapes, **kw):
    args = dict(lr=1e-2, weight_decay=0.1)
    args.update(kw)
    return demo.MuonTransform(shapes, **args)


def rel(x, y):
    return float((x.double() - y).norm() / y.norm())


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def check(tr, outs, ins, out_dtype, **kw):
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for o, u in zip(outs, ins):
        want = ref.orthogonal(u, **kw)
        assert torch.isfinite(o).all()
        tol = ref.tolerance(u.shape) + (2.0 ** -8 if out_dtype == BF16 else 0.0)
        assert rel(o, want) <= tol, (tuple(u.shape), rel(o, want), tol)


SMALL = [(1, 1), (1, 7), (9, 1), (5, 3), (17, 40), (64, 64), (63, 65), (128, 130), (200, 129), (256, 512), (256, 256), (129, 1000)]
LARGE = [(257, 300), (300, 257), (512, 512), (1000, 331), (331, 1000), (640, 2048), (1531, 515)]


@pytest.mark.parametrize("shape", SMALL + LARGE)
@pytest.mark.parametrize("in_dtype,out_dtype", [(F32, F32), (BF16, BF16)])
def test_one_matrix(shape, in_dtype, out_dtype):
    tr = muon([shape])
    u = Guarded(shape, in_dtype, "cuda", rand(shape, 1))
    o = Guarded(shape, out_dtype, "cuda", rand(shape, 2))
    tr.orthogonalize([u.t], [o.t])
    check(tr, [o.t], [u.t], out_dtype)
    assert all_intact([u, o])
    assert torch.equal(u.t, rand(shape, 1).to(in_dtype))


def test_many_matrices_of_all_sizes_at_once():
    shapes = SMALL + LARGE + [(256, 1024)] * 7 + [(384, 384)] * 5
    tr = muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    outs = [Guarded(s, F32, "cuda") for s in shapes]
    for _ in range(2):
        tr.orthogonalize(ins, [o.t for o in outs])
    check(tr, [o.t for o in outs], ins, F32)
    assert all_intact(outs)


def test_more_matrices_than_one_group_holds():
    shapes = [(2048, 2048)] * 9 + [(100, 60)] * 3  # 38 million elements
    tr = muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    outs = [torch.empty(s, dtype=BF16, device="cuda") for s in shapes]
    tr.orthogonalize(ins, outs)
    check(tr, outs, ins, BF16)


@pytest.mark.parametrize("shape", [(96, 200), (600, 400)])
@pytest.mark.parametrize("kind", ["rank1", "rank8", "rows", "tiny", "huge", "spread", "one_entry", "identity"])
def test_spectra_and_scales(shape, kind):
    u = rand(shape, 3)
    if kind == "rank1":
        u = u[:, :1] @ u[:1]
    elif kind == "rank8":
        u = u[:, :8] @ u[:8]
    elif kind == "rows":
        u = u * torch.exp(2 * rand((shape[0], 1), 4))
    elif kind == "tiny":
        u = u * 1e-24
    elif kind == "huge":
        u = u * 1e24
    elif kind == "spread":  # singular values from 1 to 1e-6
        q, r = torch.linalg.qr(u.double()), torch.linalg.qr(rand(shape[::-1], 5).double())
        k = min(shape)
        s = torch.logspace(0, -6, k, dtype=torch.float64, device="cuda")
        u = ((q[0][:, :k] * s) @ r[0][:, :k].t()).float()
    elif kind == "one_entry":
        u = torch.zeros(shape, device="cuda")
        u[shape[0] // 2, 7] = -3.0
    elif kind == "identity":
        u = torch.eye(*shape, device="cuda")
    eps = 0.0 if kind == "tiny" else 1e-7
    tr = muon([shape], eps=eps)
    o = torch.empty(shape, device="cuda")
    tr.orthogonalize([u], [o])
    torch.cuda.synchronize()
    want = ref.orthogonal(u, eps=eps)
    assert torch.isfinite(o).all()
    # Rounding noise outside a low rank is not brought back to one: it grows by a = 3.44 an iteration.  X, of norm about one, is rounded to
    # 22 bits before each of them: 2^-22 (a^5 + a^4 + ... + a) = 684 * 2^-22.  E and F are rounded to r, and enter through b E X and F X:
    # r (|b| + |b| + |c|) (a^4 + ... + 1) = 198 * 11.6 r, where their entries' roundings are independent and meet min(shape) entries
    # of a singular vector of norm one: / sqrt(min(shape)).
    r = 2.0 ** -11 if min(shape) > 256 else 2.0 ** -22
    noise = 684 * 2.0 ** -22 + 198 * 11.6 * r / math.sqrt(min(shape))
    tol = ref.tolerance(shape) * float(want.norm()) + noise * (kind in ("rank1", "rank8", "spread", "one_entry"))
    assert float((o.double() - want).norm()) <= tol, (float((o.double() - want).norm()), float(want.norm()), tol)


def test_zeros_give_zeros_and_bad_values_stay_with_their_matrix():
    shapes = [(300, 400), (300, 400), (64, 32), (64, 32)]
    tr = muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    ins[0].zero_()
    ins[2][3, 4] = float("nan")
    outs = [torch.full(s, 7.0, device="cuda") for s in shapes]
    tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    assert (outs[0] == 0).all()
    check(tr, [outs[1], outs[3]], [ins[1], ins[3]], F32)
    ins[1][0, 0] = float("inf")
    ins[2].copy_(ins[3])
    tr.orthogonalize(ins, outs)
    check(tr, outs[2:], ins[2:], F32)
    zero = muon([(40, 50)], eps=0.0)
    out = torch.full((40, 50), 7.0, device="cuda")
    zero.orthogonalize([torch.zeros((40, 50), device="cuda")], [out])
    assert (out == 0).all()


@pytest.mark.parametrize("steps", [1, 2, 8])
@pytest.mark.parametrize("shape", [(100, 70), (300, 500)])
def test_steps_and_coefficients(shape, steps):
    for coefficients in (ref.COEFFICIENTS, (1.875, -1.25, 0.375)):
        tr = muon([shape], steps=steps, coefficients=coefficients)
        u, o = rand(shape, 6), torch.empty(shape, device="cuda")
        tr.orthogonalize([u], [o])
        check(tr, [o], [u], F32, steps=steps, coefficients=coefficients)


def test_in_place():
    shapes = [(300, 500), (500, 300), (30, 50)]
    tr = muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    outs = [u.clone() for u in ins]
    tr.orthogonalize(outs, outs)
    check(tr, outs, ins, F32)


def test_same_bits_again_and_in_any_set():
    shapes = [(700, 500), (256, 300), (500, 1400)]
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    first = [torch.empty(s, device="cuda") for s in shapes]
    tr = muon(shapes)
    tr.orthogonalize(ins, first)
    for _ in range(3):
        outs = [torch.empty(s, device="cuda") for s in shapes]
        tr.orthogonalize(ins, outs)
        assert all(torch.equal(a, b) for a, b in zip(first, outs))
    for i, s in enumerate(shapes):
        alone = torch.empty(s, device="cuda")
        muon([s]).orthogonalize([ins[i]], [alone])
        assert torch.equal(alone, first[i])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("nesterov", [True, False])
@pytest.mark.parametrize("scale", [demo.DEMO_SCALE_NONE, demo.DEMO_SCALE_ASPECT, demo.DEMO_SCALE_RMS])
def test_step(dtype, nesterov, scale):
    shapes = [(64, 200), (300, 64), (512, 300), (333, 777), (1, 5), (260, 257)]
    tr = muon(shapes, nesterov=nesterov, scale=scale, momentum=0.9, lr=0.02, grad_dtype=CODE[dtype])
    g = [rand(s, i, 1e-2).to(dtype) for i, s in enumerate(shapes)]
    m = [Guarded(s, F32, "cuda", rand(s, 50 + i, 1e-2)) for i, s in enumerate(shapes)]
    x = [Guarded(s, F32, "cuda", rand(s, 90 + i)) for i, s in enumerate(shapes)]
    for n in range(3):
        if n == 2:
            tr.set_lr(0.005)
        lr = 0.005 if n == 2 else 0.02
        want = [ref.muon_step(gi, mi.t, xi.t, lr=lr, wd=0.1, mu=0.9, nesterov=nesterov, scale=scale) for gi, mi, xi in zip(g, m, x)]
        before = [xi.t.clone() for xi in x]
        tr.step(g, [t.t for t in m], [t.t for t in x])
        torch.cuda.synchronize()
        assert tr.device_status() == 0
        for mi, xi, x0, (wm, wx), s in zip(m, x, before, want, shapes):
            assert float((mi.t.double() - wm).abs().max()) <= 2 * 2.0 ** -24 * float(wm.abs().max() + 1)
            # the update's error, and the rounding of x itself
            update = float((wx - x0.double()).norm())
            assert float((xi.t.double() - wx).norm()) <= ref.tolerance(s) * update + 2 * 2.0 ** -24 * float(wx.norm())
    assert all_intact(m + x)


def test_step_and_orthogonalize_agree():
    """The set's own parts: a step without momentum, decay or factor is x - lr O(g)."""
    shapes = [(320, 640), (100, 50)]
    tr = muon(shapes, momentum=0.0, nesterov=False, weight_decay=0.0, lr=1.0, scale=demo.DEMO_SCALE_NONE, grad_dtype=demo.DEMO_F32)
    g = [rand(s, i) for i, s in enumerate(shapes)]
    o, m, x = ([torch.zeros(s, device="cuda") for s in shapes] for _ in range(3))
    tr.orthogonalize(g, o)
    tr.step(g, m, x)
    assert all(torch.equal(-a, b) for a, b in zip(o, x))
    assert all(torch.equal(a, b) for a, b in zip(g, m))


def test_captured_graph_and_eager_calls():
    shapes = [(300, 400), (64, 96)]
    tr, eager = muon(shapes), muon(shapes)
    g = [rand(s, i, 1e-2).bfloat16() for i, s in enumerate(shapes)]
    state = [[rand(s, k * 10 + i, 1e-2) for i, s in enumerate(shapes)] for k in (1, 2)]
    other = [[t.clone() for t in ts] for ts in state]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        tr.step(g, *state)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            tr.step(g, *state)
    for n in range(3):
        for gi in g:
            gi.mul_(-0.5)
        graph.replay()
        outs = [torch.empty(s, device="cuda") for s in shapes]
        tr.orthogonalize(state[1], outs)  # eager calls between replays: another entry point, its own tables
        torch.cuda.synchronize()
    for gi in g:
        gi.mul_(-8.0)
    eager.step(g, *other)
    for n in range(3):
        for gi in g:
            gi.mul_(-0.5)
        eager.step(g, *other)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for a, b in zip(state, other):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_capture_with_new_pointers_is_refused():
    shapes = [(64, 96)]
    tr = muon(shapes)
    u, o = rand(shapes[0], 1), torch.empty(shapes[0], device="cuda")
    tr.orthogonalize([u], [o])
    torch.cuda.synchronize()
    new = torch.empty(shapes[0], device="cuda")
    st = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        graph.capture_begin()
        with pytest.raises(demo.DemoError) as e:
            tr.orthogonalize([u], [new])
        tr.orthogonalize([u], [o])
        graph.capture_end()
    assert e.value.status == 1
    want = o.clone()
    o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want)


def test_on_other_streams_and_two_contexts_at_once():
    shapes = [(700, 900), (300, 2000)]
    a, b = muon(shapes), muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    want = [torch.empty(s, device="cuda") for s in shapes]
    a.orthogonalize(ins, want)
    torch.cuda.synchronize()
    outs = [[torch.empty(s, device="cuda") for s in shapes] for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        for tr, o, st in zip((a, b), outs, streams):
            tr.orthogonalize(ins, o, stream=st)
    torch.cuda.synchronize()
    assert a.device_status() == 0 and b.device_status() == 0
    for o in outs:
        assert all(torch.equal(u, v) for u, v in zip(o, want))


def test_launches_are_counted_and_workspace_told():
    tr = muon([(300, 400)])
    assert tr.launch_count == 0 and tr.workspace_bytes > 300 * 400 * 8
    u, o = rand((300, 400), 1), torch.empty((300, 400), device="cuda")
    tr.orthogonalize([u], [o])
    assert tr.launch_count > 0
