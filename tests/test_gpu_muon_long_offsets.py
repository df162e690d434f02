"""Matrices and tensors of more than 2^31 elements."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu
N = 1 << 20
STEP = 1 << 16


def orthogonal_by_parts(u, look):
    """Columns `look` (slices) of O of a wide matrix in 64 bits: O = P X with P a polynomial of X X^T, which alone needs all of X."""
    a, b, c = ref.COEFFICIENTS
    m = u.shape[0]
    g = torch.zeros(m, m, dtype=torch.float64, device="cuda")
    for at in range(0, u.shape[1], STEP):
        x = u[:, at:at + STEP].double()
        g += x @ x.t()
    norm = g.diagonal().sum().sqrt() + 1e-7
    g /= norm * norm
    p = torch.eye(m, dtype=torch.float64, device="cuda")
    for _ in range(5):
        q = a * torch.eye(m, dtype=torch.float64, device="cuda") + b * g + c * g @ g
        p, g = q @ p, q @ g @ q
    return [p @ (u[:, s].double() / norm) for s in look]


@pytest.mark.parametrize("tall", [False, True])
def test_orthogonalize(tall):
    m = 2100
    shape = (N, m) if tall else (m, N)
    assert m * N > 1 << 31
    gen = torch.Generator("cuda").manual_seed(1)
    u = torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    o = torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda")
    tr = demo.MuonTransform([shape], lr=1e-2, weight_decay=0.1)
    tr.orthogonalize([u], [o])
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    wide, got = (u.t(), o.t()) if tall else (u, o)
    look = [slice(0, 4096), slice(N // 2 - 2048, N // 2 + 2048), slice(N - 4096, N)]
    for s, want in zip(look, orthogonal_by_parts(wide, look)):
        assert float((got[:, s].double() - want).norm() / want.norm()) <= 1e-3 + 2.0 ** -8  # (bf16 results)


def test_adamw():
    n = (1 << 31) + 4099
    tr = demo.AdamwTransform([(5,), (n,)], lr=1e-2, weight_decay=0.1)
    gen = torch.Generator("cuda").manual_seed(1)
    g = [torch.empty(k, dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for k in (5, n)]
    m, v, x = ([torch.full((k,), f, device="cuda") for k in (5, n)] for f in (0.5, 2.0, 1.0))
    count = torch.zeros(1, dtype=torch.int64, device="cuda")
    tr.step(g, m, v, x, count)
    torch.cuda.synchronize()
    for at in (0, (1 << 30) - 1000, (1 << 31) - 1000, n - 2000):
        part = slice(at, at + 2000)
        one = torch.ones(2000, device="cuda")
        wm, wv, wx = ref.adamw_step(g[1][part], 0.5 * one, 2 * one, one, 1, lr=1e-2, wd=0.1)
        # three roundings of m, four of v; x: three of its own and twelve of an update of up to lr (|m| / 0.1) / sqrt(v / 0.05)
        u = 2.0 ** -24
        assert bool(((m[1][part] - wm).abs() <= 3 * u * (wm.abs() + 0.5)).all())
        assert bool(((v[1][part] - wv).abs() <= 4 * u * wv).all())
        assert bool(((x[1][part] - wx).abs() <= 3 * u * wx.abs() + 12 * u * 1e-2 * (wm.abs() + 0.5) / 0.1 / (wv / 0.05).sqrt()).all())
