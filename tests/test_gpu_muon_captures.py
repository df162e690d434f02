"""Programs that capture again and again: graphs keep what they were captured with for as long as they live, and nothing grows with those that are gone."""
import gc

import pytest
import torch

import paper_2411_19870_b200 as demo

pytestmark = pytest.mark.gpu


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def captured(call, st):
    """call() once, then in a graph."""
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(st):
        call()
        st.synchronize()
        with torch.cuda.graph(graph, stream=st):
            call()
    return graph


def test_tables_of_graphs_that_are_gone_serve_again():
    shapes = [(20, 30), (400, 500)] * 50
    tr, st = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32), torch.cuda.Stream()
    sizes = []
    for n in range(12):
        sets = [[rand(s, n + k) for s in shapes] for k in range(4)]
        graphs = [captured(lambda: tr.orthogonalize(sets[3], sets[3]), st), captured(lambda: tr.step(*sets[:3]), st)]
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        del g, graphs
        gc.collect()
        sizes.append(tr.workspace_bytes)
    # for each of the two entry points (five pointers a matrix) one in use, and room for two that are still on their way back
    assert sizes[-1] <= sizes[0] + 2 * 5 * len(shapes) * 8
    assert tr.device_status() == 0


def test_graphs_that_live_keep_theirs():
    shapes = [(64, 96), (300, 410)]
    tr, st = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1), torch.cuda.Stream()
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    want = [torch.empty(s, device="cuda") for s in shapes]
    tr.orthogonalize(ins, want)
    torch.cuda.synchronize()
    alive = []
    for n in range(9):
        outs = [torch.empty(s, device="cuda") for s in shapes]
        graph = captured(lambda: tr.orthogonalize(ins, outs), st)
        if n % 3 != 1:
            alive.append((graph, outs))
        del graph
        gc.collect()
        if n == 5:  # some of those that lived go, too
            alive = alive[::2]
    with torch.cuda.stream(st):
        for _, outs in alive:
            for o in outs:
                o.zero_()
        for k in list(range(len(alive))) + list(range(len(alive)))[::-1]:
            alive[k][0].replay()
            tr.orthogonalize(ins, [torch.empty(s, device="cuda") for s in shapes])
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for _, outs in alive:
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_a_context_may_go_before_its_graphs():
    """The graph is not replayed any more, but its end still tells the context's tables."""
    st = torch.cuda.Stream()
    for _ in range(3):
        tr = demo.AdamwTransform([(100,)], lr=1e-2, weight_decay=0.1, grad_dtype=demo.DEMO_F32)
        s, count = [[torch.ones(100, device="cuda")] for _ in range(4)], torch.zeros(1, dtype=torch.int64, device="cuda")
        graph = captured(lambda: tr.step(*s, count), st)
        graph.replay()
        torch.cuda.synchronize()
        tr.close()
        del graph
        gc.collect()
        assert int(count) == 2


def test_decodes_captured_anew():
    shapes = [(128, 192), (64,), (320, 384)]
    dm = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=1)
    tr, st = demo.MuonTransform([shapes[0], shapes[2]], lr=1e-2, weight_decay=0.1), torch.cuda.Stream()
    p = torch.empty(dm.payload_bytes, dtype=torch.uint8, device="cuda")
    dm.compress(0, [rand(s, i).bfloat16() for i, s in enumerate(shapes)], [torch.zeros(s, device="cuda") for s in shapes], p)
    want = [rand(s, 9) for s in shapes]
    for _ in range(3):
        tr.decode_apply(dm, [p], want)
    torch.cuda.synchronize()
    sizes = []
    for n in range(8):
        x, q = [rand(s, 9) for s in shapes], p.clone()
        graph = captured(lambda: tr.decode_apply(dm, [q], x), st)
        graph.replay()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(x, want))
        del graph
        gc.collect()
        sizes.append(tr.workspace_bytes)
    assert sizes[-1] <= sizes[0] + 2 * 2 * 2 * 8  # (two pointers for each of two matrices)
    assert tr.device_status() == 0 and dm.device_status() == 0
