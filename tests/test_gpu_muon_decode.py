"""Payloads decoded into orthogonalised updates, and the whole set as a training program uses it."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu
W = 3


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def received(tr, shapes, chunk, k, payloads, agg):
    """R of every tensor in 64 bits, from the payloads' bytes."""
    import math

    n = torch.arange(chunk, dtype=torch.float64)
    c = torch.cos(math.pi * (2 * n + 1) * n[:, None] / (2 * chunk)) * math.sqrt(2 / chunk)
    c[0] /= math.sqrt(2)
    out = []
    for t, s in enumerate(shapes):
        first, n_chunks, k_eff = tr.payload_layout(t)
        m = chunk ** len(s)
        q, hits = torch.zeros(n_chunks, m, dtype=torch.float64), torch.zeros(n_chunks, m)
        for p in payloads:
            rec = p.cpu()[first * 8:(first + n_chunks * k_eff) * 8].view(torch.int32).view(n_chunks, k_eff, 2)
            q.scatter_add_(1, rec[..., 0].long(), rec[..., 1].contiguous().view(torch.float32).double())
            hits.scatter_add_(1, rec[..., 0].long(), torch.ones(n_chunks, k_eff))
        if agg == demo.DEMO_AGG_MEAN:
            q /= len(payloads)
        if agg == demo.DEMO_AGG_COUNT_MEAN:
            q /= hits.clamp(min=1)
        if len(s) == 1:
            out.append((q @ c).flatten())
        else:
            r = c.t() @ q.view(n_chunks, chunk, chunk) @ c
            out.append(r.view(s[0] // chunk, s[1] // chunk, chunk, chunk).permute(0, 2, 1, 3).reshape(s))
    return [r.cuda() for r in out]


def payloads_of(tr, shapes):
    ps = []
    for w in range(W):
        g = [rand(s, 10 * w + i).bfloat16() for i, s in enumerate(shapes)]
        m = [torch.zeros(s, device="cuda") for s in shapes]
        p = torch.empty(tr.payload_bytes, dtype=torch.uint8, device="cuda")
        tr.compress(w, g, m, p)
        ps.append(p)
    return ps


@pytest.mark.parametrize("chunk,k", [(8, 4), (16, 9), (32, 8), (64, 32), (128, 40)])
@pytest.mark.parametrize("agg", [demo.DEMO_AGG_SUM, demo.DEMO_AGG_MEAN, demo.DEMO_AGG_COUNT_MEAN])
def test_decode_apply(chunk, k, agg):
    shapes = [(2 * chunk, 5 * chunk), (3 * chunk,), (6 * chunk, 4 * chunk), (chunk, chunk)]
    tr = demo.DemoTransform(shapes, chunk=chunk, topk=k, beta=0.9, lr=3e-3, weight_decay=0.05, num_workers=W)
    tr.set_decode_mode(agg, demo.DEMO_PHI_SIGN)
    mu = demo.MuonTransform([s for s in shapes if len(s) == 2], lr=1e-2, weight_decay=0.1)
    ps = payloads_of(tr, shapes)
    x = [rand(s, 70 + i) for i, s in enumerate(shapes)]
    x0 = [t.double() for t in x]
    rs = received(tr, shapes, chunk, k, ps, agg)
    plain = [t.clone() for t in x]
    for n in range(2):
        mu.decode_apply(tr, ps, x)
        torch.cuda.synchronize()
        assert mu.device_status() == 0 and tr.device_status() == 0
        for xi, w0, r in zip(x, x0, rs):
            if xi.dim() == 1:
                want = w0 - 3e-3 * (torch.sign(r) + 0.05 * w0)
                assert ((xi - want).abs() <= 1e-6 * want.abs() + 1e-6 + 6.1e-3 * (r.abs() < 1e-5)).all()
            else:
                want = w0 - 1e-2 * (ref.scale_of(2, xi.shape) * ref.orthogonal(r) + 0.1 * w0)
                assert float((xi - want).norm()) <= ref.tolerance(xi.shape) * float((want - w0).norm()) + 2 * 2.0 ** -24 * float(want.norm())
        x0 = [t.double() for t in x]
    # the plain decode of the same context works as before
    other = demo.DemoTransform(shapes, chunk=chunk, topk=k, beta=0.9, lr=3e-3, weight_decay=0.05, num_workers=W)
    other.set_decode_mode(agg, demo.DEMO_PHI_SIGN)
    a, b = [t.clone() for t in plain], [t.clone() for t in plain]
    tr.decode_apply(ps, a)
    other.decode_apply(ps, b)
    assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_caller_supplied_basis():
    shapes = [(256, 384), (64,)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=4096, beta=0.9, lr=1e-2, weight_decay=0.0, num_workers=W)
    tr.set_basis(torch.linalg.qr(torch.randn(64, 64, generator=torch.Generator().manual_seed(1), dtype=torch.float64))[0].float())
    mu = demo.MuonTransform(shapes[:1], lr=1e-2, weight_decay=0.0)
    x = [rand(s, i) for i, s in enumerate(shapes)]
    before = x[0].double()
    ps = payloads_of(tr, shapes)  # every coefficient kept: R is the sum of the momenta, in any basis
    r = sum(rand(shapes[0], 10 * w).bfloat16().double() for w in range(W))
    mu.decode_apply(tr, ps, x)
    torch.cuda.synchronize()
    want = before - 1e-2 * ref.scale_of(2, shapes[0]) * ref.orthogonal(r)
    # (3xTF32 in both transforms: 2^-21 of the values, more than the orthogonalisation's own fp32 sums)
    assert float((x[0] - want).norm()) <= 4 * ref.tolerance(shapes[0]) * float((want - before).norm()) + 2 * 2.0 ** -24 * float(want.norm())


def test_captured_graph():
    shapes = [(128, 192), (64,), (320, 384)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=W)
    mu = demo.MuonTransform([shapes[0], shapes[2]], lr=1e-2, weight_decay=0.1)
    ps = payloads_of(tr, shapes)
    x = [rand(s, i) for i, s in enumerate(shapes)]
    y = [t.clone() for t in x]
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        graph = torch.cuda.CUDAGraph()
        graph.capture_begin()
        with pytest.raises(demo.DemoError):  # the first call allocates
            mu.decode_apply(tr, ps, x)
        tr2 = x[0] + 0  # (something to capture)
        graph.capture_end()
        mu.decode_apply(tr, ps, x)
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            mu.decode_apply(tr, ps, x)
    tr.decode_apply(ps, [t.clone() for t in x])  # other pointers in the plain decode's table
    graph.replay()
    graph.replay()
    torch.cuda.synchronize()
    for _ in range(3):
        mu.decode_apply(tr, ps, y)
    torch.cuda.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(x, y))
    del tr2


def test_bad_record_is_reported_and_left_out():
    shapes = [(128, 128)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=W)
    mu = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    ps = payloads_of(tr, shapes)
    a, b = rand(shapes[0], 5), rand(shapes[0], 5)
    ps[1].view(torch.int32).view(-1, 2)[31, 1] = 0  # the last record of the first chunk: a value of zero
    mu.decode_apply(tr, ps, [a])
    assert tr.device_status() == 0
    ps[1].view(torch.int32).view(-1, 2)[31, 0] = 64 * 64  # an index outside the chunk
    mu.decode_apply(tr, ps, [b])
    assert tr.device_status() == 8 and tr.device_status() == 0 and mu.device_status() == 0
    assert torch.equal(a, b)


def test_refusals():
    shapes = [(128, 128), (64,)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=32, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=W)
    x = [rand(s, i) for i, s in enumerate(shapes)]
    ps = payloads_of(tr, shapes)
    for other in ([(128, 64)], [(128, 128), (128, 128)], [(64, 128)]):
        with pytest.raises(demo.DemoError) as e:
            demo.MuonTransform(other, lr=1e-2, weight_decay=0.1).decode_apply(tr, ps, x)
        assert e.value.status == 2
    mu = demo.MuonTransform([(128, 128)], lr=1e-2, weight_decay=0.1)
    with pytest.raises(demo.DemoError) as e:
        mu.decode_apply(tr, ps[:2], x)
    assert e.value.status == 1
    nd = demo.DemoTransform([(128, 96)], chunk_shapes=[(16, 32)], topk=8, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=1)
    with pytest.raises(demo.DemoError) as e:
        demo.MuonTransform([(128, 96)], lr=1e-2, weight_decay=0.1).decode_apply(
            nd, [torch.zeros(nd.payload_bytes, dtype=torch.uint8, device="cuda")], [rand((128, 96), 1)])
    assert e.value.status == 4
    before = [t.clone() for t in x]
    assert all(torch.equal(u, v) for u, v in zip(x, before))


def test_the_set_as_a_training_program_uses_it():
    """Three steps: the matrices' gradients compressed by every worker and received as orthogonalised updates, the embedding and the
    vectors by AdamW, each against 64 bits on the payloads that it was given."""
    shapes = [(128, 256), (256, 128), (320, 320)]
    rest = [(101, 64), (64,)]
    tr = demo.DemoTransform(shapes, chunk=64, topk=64, beta=0.9, lr=1e-2, weight_decay=0.1, num_workers=W)
    mu = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    ad = demo.AdamwTransform(rest, lr=1e-2, weight_decay=0.1)
    momentum = [[torch.zeros(s, device="cuda") for s in shapes] for _ in range(W)]
    payloads = [torch.empty(tr.payload_bytes, dtype=torch.uint8, device="cuda") for _ in range(W)]
    x, y = [rand(s, i) for i, s in enumerate(shapes)], [rand(s, 9 + i) for i, s in enumerate(rest)]
    m, v = [torch.zeros(s, device="cuda") for s in rest], [torch.zeros(s, device="cuda") for s in rest]
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    for n in range(3):
        for w in range(W):
            tr.compress(w, [rand(s, 1000 * n + 10 * w + i).bfloat16() for i, s in enumerate(shapes)], momentum[w], payloads[w])
        g = [rand(s, 5000 * n + i).bfloat16() for i, s in enumerate(rest)]
        x0, old = [t.double() for t in x], [(a.clone(), b.clone(), c.clone()) for a, b, c in zip(m, v, y)]
        rs = received(tr, shapes, 64, 64, payloads, demo.DEMO_AGG_SUM)
        mu.decode_apply(tr, payloads, x)
        ad.step(g, m, v, y, count)
        torch.cuda.synchronize()
        for xi, w0, r in zip(x, x0, rs):
            want = w0 - 1e-2 * (ref.scale_of(2, xi.shape) * ref.orthogonal(r) + 0.1 * w0)
            assert float((xi - want).norm()) <= ref.tolerance(xi.shape) * float((want - w0).norm()) + 2 * 2.0 ** -24 * float(want.norm())
        for (a, b, c), gi, yi in zip(old, g, y):
            want = ref.adamw_step(gi, a, b, c, n + 1, lr=1e-2, wd=0.1)[2]
            assert float((yi - want).abs().max()) <= 12 * 2.0 ** -24 * (float(want.abs().max()) + 1)
    assert int(count) == 3
