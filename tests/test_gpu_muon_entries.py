"""Matrices with single entries that outweigh the rest, entry by entry: a rounding of such an entry has nothing to average out with."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu


def orthogonalised(shape, count, u):
    tr = demo.MuonTransform([shape] * count, lr=1e-2, weight_decay=0.1)
    outs = [torch.full(shape, float("nan"), device="cuda") for _ in range(count)]
    for _ in range(2):
        tr.orthogonalize([u] * count, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    assert all(torch.equal(o, outs[0]) for o in outs)
    return outs[0].double()


# tiles of 128 (one, two at a time), transposed, sums in parts, tiles of 256 (many), hi and lo parts; sizes within a tile's first row of blocks too
@pytest.mark.parametrize("shape,count", [((300, 301), 1), ((300, 1200), 1), ((1201, 300), 1), ((300, 4003), 1), ((300, 420), 160), ((270, 1333), 160),
                                         ((420, 300), 160), ((257, 257), 1), ((100, 130), 1),
                                         ((400, 401), 1), ((400, 1600), 1), ((1601, 400), 1), ((400, 4003), 1), ((400, 520), 160), ((390, 1533), 160),
                                         ((520, 400), 160)])
def test_one_entry_a_row(shape, count):
    gen = torch.Generator("cuda").manual_seed(1)
    m, n = min(shape), max(shape)
    values = 1 + torch.rand(m, generator=gen, device="cuda")
    x = torch.zeros(m, n, device="cuda")
    x[torch.arange(m, device="cuda"), torch.randperm(n, generator=gen, device="cuda")[:m]] = values
    u = (x if shape[0] <= shape[1] else x.t()).contiguous()
    o, want = orthogonalised(shape, count, u), ref.orthogonal(u)
    # The products off the diagonal are zero, what is left is p(p(..x..)) of each entry in fp32, with u = 2^-24: an iteration's d = x^2 is off
    # by 4 u (x^2, what its fp16 value leaves out and their sum), which B = a + b d + c d^2 passes on |(b + 2 c d) d| <= 1.6 times, d up to 1.45; its
    # three terms, up to 3.5, 6.9 and 4.3, round by 20 u; B x by |B| <= 3.5 u more: 30 u x, and twice that where two iterations are one and d
    # is a product of five roundings itself.  Earlier errors are passed on |p'(x)| times.  x itself begins three roundings off.
    a, b, c = ref.COEFFICIENTS
    v = values.double() / values.double().norm()
    off = 3 * 2.0 ** -24 * v
    for _ in range(5):
        off = (a + 3 * b * v ** 2 + 5 * c * v ** 4).abs() * off + 60 * 2.0 ** -24 * v
        v = a * v + b * v ** 3 + c * v ** 5
    assert float((o - want).abs().max()) <= float(off.max())
    assert bool((o[want == 0] == 0).all())


@pytest.mark.parametrize("shape,count", [((300, 1200), 1), ((830, 3320), 3), ((600, 600), 1), ((512, 2048), 40)])
def test_heavy_tails(shape, count):
    gen = torch.Generator("cuda").manual_seed(2)
    chi = sum(torch.randn(shape, generator=gen, device="cuda").square() for _ in range(3))
    u = torch.randn(shape, generator=gen, device="cuda") * (chi / 3).rsqrt().clamp(max=1e3)
    o, want = orthogonalised(shape, count, u), ref.orthogonal(u)
    # Where an entry x of a row has nearly all of its weight, the rounding of its fp16 value, r = 2^-11 of it, is in E along the entry's column c:
    # r x c.  Through (b + 2 c) E X of the last iteration |b + 2 c| r x |c|^2 comes back to it, |c|^2 = 1 - x^2 without the entry itself: at most
    # 0.71 r 0.39, and 1.6 times that of the iteration before, and F's and X's own rounding in F X, r |F| |c| each: 2 r 0.4 (1 + 1.6).
    assert float((o - want).abs().max()) <= (0.71 * 0.39 + 2 * 0.4) * 2.6 * 2.0 ** -11
    assert float((o - want).norm() / want.norm()) <= ref.tolerance(shape)
