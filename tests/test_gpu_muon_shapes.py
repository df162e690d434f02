"""The ways that a set of matrices can take: tiles of 256 and of 128, iterations one by one and in twos, several groups in one workspace,
small matrices beside larger ones; and how accurate each is where the rank is low."""
import math

import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def errors(shapes, ins, look, **kw):
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1, **kw)
    outs = [torch.full(s, float("nan"), device="cuda") for s in shapes]
    for _ in range(2):  # (the second call finds what the first left in the workspace)
        tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    assert all(bool(torch.isfinite(o).all()) for o in outs)
    return [(float((outs[i].double() - w).norm()), float(w.norm())) for i in look for w in (ref.orthogonal(ins[i], **{k: kw[k] for k in kw if k == "steps"}),)]


# Many: the set's tasks outweigh its chain of products, tiles of 256.  One: tiles of 128.
@pytest.mark.parametrize("count", [1, 160], ids=["one", "many"])
@pytest.mark.parametrize("shape", [(257, 257), (300, 420), (420, 300), (300, 700), (513, 511), (270, 1333), (640, 1280)])
@pytest.mark.parametrize("steps", [2, 3, 4, 5])
def test_every_way(shape, count, steps):
    shapes = [shape] * count
    ins = [rand(shape, i) for i in range(count)]
    look = sorted({0, count // 2, count - 1})
    for off, norm in errors(shapes, ins, look, steps=steps):
        assert off <= ref.tolerance(shape) * norm, (off / norm, ref.tolerance(shape))


@pytest.mark.parametrize("shape,count", [((400, 1200), 1), ((400, 1200), 120), ((400, 450), 120)])
@pytest.mark.parametrize("rank", [1, 5, 32])
def test_low_rank(shape, count, rank):
    u = rand((shape[0], rank), 1) @ rand((rank, shape[1]), 2)
    ins = [u * (1 + i) for i in range(count)]
    # as in test_gpu_muon.py, where the products that round B and A are those of two iterations at a time: B' B has entries of up to a^2 = 12
    # instead of |b| + |c| = 6.8, and T and A' add their roundings to it, each less than B's: three times as much
    noise = 684 * 2.0 ** -22 + 3 * 198 * 11.6 * 2.0 ** -11 / math.sqrt(min(shape))
    for off, norm in errors([shape] * count, ins, [0, count - 1]):
        assert off <= ref.tolerance(shape) * norm + noise
        assert off <= 0.02 * norm  # (what include/demo.h says, with room)


def test_several_groups_in_one_workspace():
    shapes = [(4096, 4096)] * 18  # 302 million elements
    ins = [rand(shapes[0], i).bfloat16() for i in range(18)]
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    # less than all eighteen need: X takes two fp16 copies and one fp32, A and B a copy of each, 20 bytes an element of a square matrix
    assert tr.workspace_bytes < 18 * 4096 * 4096 * 20
    outs = [torch.empty(s, dtype=torch.bfloat16, device="cuda") for s in shapes]
    tr.orthogonalize(ins, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    for i in (0, 14, 15, 16, 17):
        want = ref.orthogonal(ins[i])
        assert float((outs[i].double() - want).norm() / want.norm()) <= ref.tolerance(shapes[i]) + 2.0 ** -8


def test_small_matrices_beside_larger_ones():
    shapes = [(147, 512), (700, 900), (64, 64), (900, 2000), (33, 1000), (512, 512)]
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    for (off, norm), s in zip(errors(shapes, ins, range(len(shapes))), shapes):
        assert off <= ref.tolerance(s) * norm
    # on a side stream, too, nothing of a later call overtakes an earlier one
    tr = demo.MuonTransform(shapes, lr=1e-2, weight_decay=0.1)
    outs = [torch.empty(s, device="cuda") for s in shapes]
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        for n in range(6):
            for u in ins:
                u.mul_(-1.0)
            tr.orthogonalize(ins, outs)
    st.synchronize()
    again = [torch.empty(s, device="cuda") for s in shapes]
    tr.orthogonalize(ins, again)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, again))


def test_long_and_thin():
    shapes = [(3, 200000), (120001, 40), (300, 50304), (1, 1 << 20)]
    ins = [rand(s, i) for i, s in enumerate(shapes)]
    for (off, norm), s in zip(errors(shapes, ins, range(len(shapes))), shapes):
        # (sums over K of up to 2^20 elements in fp32: 2^-24 for each of sqrt(K) = 1024 steps in one direction, in each of the products)
        assert off <= (ref.tolerance(s) + 16 * 1024 * 2.0 ** -24) * norm
