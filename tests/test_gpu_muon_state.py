"""What the contexts of the orthogonalised updates and of AdamW keep between calls, and what they must not: results do not depend on the calls
before, on the stream that made the context, or on which of its captured graphs ran last."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu
F32 = torch.float32


def muon(shapes, **kw):
    return demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1, **kw)


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


# tiles of 128 with hi and lo parts, of 128, of 256 (many of them), both kinds at once, sums in parts; odd sizes, so that there are pads
@pytest.mark.parametrize("shapes", [[(65, 127)], [(129, 1000), (33, 70)], [(257, 331)], [(300, 700)], [(270, 1333)] * 160, [(147, 99), (513, 700)],
                                    [(301, 4001)], [(700, 8200)], [(3, 9001)], [(401, 555)], [(401, 1333)], [(390, 1333)] * 160, [(401, 4001)]], ids=range(13))
def test_nothing_of_a_bad_matrix_stays(shapes):
    tr, fresh = muon(shapes), muon(shapes)
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    bad = [torch.full(s, v, device="cuda") for s, v in zip(shapes, [float("nan"), float("inf")] * len(shapes))]
    outs, want = ([torch.empty(s, device="cuda") for s in shapes] for _ in range(2))
    fresh.orthogonalize(ins, want)
    tr.orthogonalize(bad, outs)
    tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and fresh.device_status() == 0
    for o, w, u in zip(outs, want, ins):
        assert torch.equal(o, w)
    for i in {0, len(shapes) - 1}:
        exact = ref.orthogonal(ins[i])
        # (sums over K of up to 9001 elements: 2^-24 for each of sqrt(K) < 128 steps of a sum in one direction)
        assert float((outs[i].double() - exact).norm() / exact.norm()) <= ref.tolerance(shapes[i]) + 16 * 128 * 2.0 ** -24


@pytest.mark.parametrize("shape", [(520, 3500), (2000, 4200), (1100, 8200), (768, 8000), (2048, 8192), (8200, 1537)])
def test_sums_in_parts(shape):
    tr, u = muon([shape]), rand(shape, 1)
    outs = [torch.full(shape, float("nan"), device="cuda") for _ in range(3)]
    for o in outs:
        tr.orthogonalize([u], [o])
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    want = ref.orthogonal(u)
    assert float((outs[0].double() - want).norm() / want.norm()) <= ref.tolerance(shape)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])  # (whichever part came last)


def test_most_steps():
    # the singular values go round in 0.7 .. 1.2 for as long as the iterations last
    shapes = [(64, 96), (300, 500)]
    tr = muon(shapes, steps=64)
    ins, outs = [rand(s, i) for i, s in enumerate(shapes)], [torch.empty(s, device="cuda") for s in shapes]
    tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for o in outs:
        s = torch.linalg.svdvals(o.double())
        assert float(s.max()) < 1.3 and float(s.min()) > 0.6
    with pytest.raises(demo.DemoError):
        muon(shapes, steps=65)


def test_first_call_on_another_stream_than_the_busy_one():
    shapes = [(300, 400), (64, 96)]
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    x = torch.randn(8192, 8192, device="cuda")
    outs, st = [torch.empty(s, device="cuda") for s in shapes], torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(20):
        x = x @ x * 1e-2
    tr, adam = muon(shapes), demo.AdamwTransform([(1000,)], lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32)
    tr.orthogonalize(ins, outs, stream=st)
    state, count = [[torch.ones(1000, device="cuda")] for _ in range(4)], torch.zeros((), dtype=torch.int64, device="cuda")
    torch.cuda.synchronize()
    adam.step(*state, count, stream=st)
    adam.step(*state, count, stream=st.cuda_stream)
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and int(count) == 2
    for o, u in zip(outs, ins):
        want = ref.orthogonal(u)
        assert float((o.double() - want).norm() / want.norm()) <= ref.tolerance(u.shape)


def test_two_graphs_of_one_context():
    shapes = [(300, 400), (64, 96), (520, 3500)]
    tr, eager = muon(shapes, grad_dtype=demo.DEMO_F32), muon(shapes, grad_dtype=demo.DEMO_F32)
    g = [rand(s, i, 1e-2) for i, s in enumerate(shapes)]
    m, x = ([rand(s, k * 10 + i, 1e-2) for i, s in enumerate(shapes)] for k in (1, 2))
    m2, x2 = [t.clone() for t in m], [t.clone() for t in x]
    o, o2 = ([torch.empty(s, device="cuda") for s in shapes] for _ in range(2))
    st = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(st):
        tr.step(g, m, x)
        tr.orthogonalize(x, o)
        st.synchronize()
        with torch.cuda.graph(graphs[0], stream=st):
            tr.step(g, m, x)
        with torch.cuda.graph(graphs[1], stream=st):
            tr.orthogonalize(x, o)
        for n in (0, 1, 0, 0, 1):
            graphs[n].replay()
    eager.step(g, m2, x2)
    for n in (0, 1, 0, 0, 1):
        eager.step(g, m2, x2) if n == 0 else eager.orthogonalize(x2, o2)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for a, b in ((m, m2), (x, x2), (o, o2)):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_types_and_places_are_checked_on_the_device():
    tr = muon([(4, 6)])
    u, o = rand((4, 6), 1), torch.empty(4, 6, device="cuda")
    for bad in (u.half(), u.cpu(), u.t(), torch.empty(4, 7, device="cuda")[:, :6], u.double()):
        with pytest.raises((ValueError, demo.DemoError)):
            tr.orthogonalize([bad], [o])
        with pytest.raises((ValueError, demo.DemoError)):
            tr.orthogonalize([u], [bad])
    off = torch.empty(25, device="cuda")[1:].view(4, 6)  # not on a 16-byte boundary
    for args in (([off], [o]), ([u], [off])):
        with pytest.raises((ValueError, demo.DemoError)):
            tr.orthogonalize(*args)
    with pytest.raises((ValueError, demo.DemoError)):
        tr.step([u], [o], [o.clone()])  # (gradients of this context are bf16)
    adam = demo.AdamwTransform([(4, 6)], lr=1e-2, weight_decay=0.0, grad_dtype=demo.DEMO_F32)
    s = [[torch.zeros(4, 6, device="cuda")] for _ in range(4)]
    for count in (torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int64), torch.zeros(2, dtype=torch.int64, device="cuda")):
        with pytest.raises((ValueError, demo.DemoError)):
            adam.step(*s, count)
    with pytest.raises((ValueError, demo.DemoError)):
        adam.step(s[0], s[1], s[2], [off], torch.zeros(1, dtype=torch.int64, device="cuda"))
    tr.orthogonalize([u], [o])
    torch.cuda.synchronize()
    assert tr.device_status() == 0 and tr.launch_count == 3 and adam.launch_count == 0


def replayed_between_calls_with_others(call, make):
    """call(a) captured; then called with b, and captured with b, too; the graphs still work on their own tensors, call by call."""
    a, b, c, want_a, want_b = (make() for _ in range(5))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    with torch.cuda.stream(st):
        call(a)
        st.synchronize()
        with torch.cuda.graph(graphs[0], stream=st):
            call(a)
        call(c)
        graphs[0].replay()
        call(b)
        st.synchronize()
        with torch.cuda.graph(graphs[1], stream=st):
            call(b)
        call(c)
        graphs[1].replay()
        graphs[0].replay()
    st.synchronize()
    for _ in range(3):
        call(want_a)
    for _ in range(2):
        call(want_b)
    call(make())
    torch.cuda.synchronize()
    for got, want in ((a, want_a), (b, want_b), (c, want_b)):
        assert all(torch.equal(u, v) for x, y in zip(got, want) for u, v in zip(x, y))


def test_a_captured_step_keeps_its_tensors():
    shapes = [(64, 96), (300, 400)]
    tr = muon(shapes, grad_dtype=demo.DEMO_F32)
    make = lambda: [[rand(s, k * 10 + i) for i, s in enumerate(shapes)] for k in range(3)]  # noqa: E731
    replayed_between_calls_with_others(lambda s: tr.step(*s), make)
    assert tr.device_status() == 0


def test_a_captured_orthogonalisation_keeps_its_tensors():
    shapes = [(64, 96), (300, 400)]
    tr = muon(shapes)
    make = lambda: [[rand(s, i) for i, s in enumerate(shapes)]]  # noqa: E731
    before = tr.workspace_bytes
    replayed_between_calls_with_others(lambda s: tr.orthogonalize(s[0], s[0]), make)  # (in place)
    assert tr.device_status() == 0 and before < tr.workspace_bytes < before + 4096


def test_a_captured_adamw_step_keeps_its_tensors():
    shapes = [(64, 96), (301,)]
    tr = demo.AdamwTransform(shapes, lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32)
    counts = []

    def make():
        s = [[rand(sh, k * 10 + i).abs() for i, sh in enumerate(shapes)] for k in range(4)]
        counts.append(torch.zeros(1, dtype=torch.int64, device="cuda"))
        return s + [[counts[-1]]]

    replayed_between_calls_with_others(lambda s: tr.step(s[0], s[1], s[2], s[3], s[4][0]), make)
    assert [int(c) for c in counts] == [3, 2, 2, 3, 2, 1]


def test_a_captured_decode_keeps_its_tensors():
    shapes = [(128, 192), (64,), (320, 384)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=2)
    tr_mu = muon([shapes[0], shapes[2]])

    def payload(seed):
        p = torch.empty(tr.payload_bytes, dtype=torch.uint8, device="cuda")
        tr.compress(0, [rand(s, seed + i).bfloat16() for i, s in enumerate(shapes)], [torch.zeros(s, device="cuda") for s in shapes], p)
        return p

    def make():
        return [[payload(1), payload(5)], [rand(s, i) for i, s in enumerate(shapes)]]

    def call(s):
        tr_mu.decode_apply(tr, s[0], s[1])
        tr.decode_apply([s[0][1], s[0][0]], [t.clone() for t in s[1]]) if not torch.cuda.is_current_stream_capturing() else None

    replayed_between_calls_with_others(call, make)
    assert tr_mu.device_status() == 0 and tr.device_status() == 0
