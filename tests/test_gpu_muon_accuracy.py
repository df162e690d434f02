"""The accuracy that include/demo.h documents for the orthogonalised updates, held as it stands there."""
import pytest
import torch

import paper_2411_19870_b200 as demo
from tests import muon_reference as ref

pytestmark = pytest.mark.gpu


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator("cuda").manual_seed(seed), device="cuda") * scale


def make(shape, kind):
    m, n = shape
    if kind == "gaussian":
        return rand(shape, 1)
    if kind == "rows":  # rows of very different sizes
        return rand(shape, 1) * torch.exp(rand((m, 1), 2))
    if kind == "positive":
        return rand(shape, 1).abs()
    if kind == "equal":
        return torch.ones(shape, device="cuda")
    if kind == "equal rows":
        return rand((1, n), 1).expand(m, n).contiguous()
    if kind == "equal columns":
        return rand((m, 1), 1).expand(m, n).contiguous()
    if kind == "blocks":  # of 8 x 8 equal entries
        return rand((-(-m // 8), -(-n // 8)), 1).repeat_interleave(8, 0).repeat_interleave(8, 1)[:m, :n].contiguous()
    if kind == "signs":
        return rand(shape, 1).sign()
    rank = int(kind)
    return rand((m, rank), 1) @ rand((rank, n), 2)


# what the header says: of full rank, of a lower one, where roundings do not average out
def documented(shape, kind):
    small, n = min(shape) <= 384, max(shape)
    if kind in ("equal", "equal rows", "equal columns", "blocks", "signs"):
        return 4e-4 if small else 3e-2
    if kind in ("gaussian", "rows", "positive"):
        return 2e-5 + min(n * 2.0 ** -26, 6e-5) if small else 1e-3
    return 4e-4 if small else 2e-3


def error(shape, count, kind, **kw):
    u = make(shape, kind)
    tr = demo.MuonTransform([shape] * count, lr=1e-2, weight_decay=0.1, **kw)
    outs = [torch.full(shape, float("nan"), device="cuda") for _ in range(count)]
    tr.orthogonalize([u] * count, outs)
    torch.cuda.synchronize()
    assert tr.device_status() == 0
    want = ref.orthogonal(u)
    off = [float((outs[i].double() - want).norm() / want.norm()) for i in {0, count - 1}]
    return max(off)


# Many: no worker is idle, so a sum is cut for its exactness alone.  One: for the idle workers, too.
LONG = [((64, 8192), 160), ((300, 8192), 60), ((8200, 257), 60), ((1, 1 << 20), 1), ((4, 36258), 160), ((400, 32768), 60), ((32700, 520), 30)]


@pytest.mark.parametrize("shape,count", LONG)
@pytest.mark.parametrize("kind", ["gaussian", "positive", "equal", "equal columns", "signs"])
def test_long_sums(shape, count, kind):
    if min(shape) == 1 and kind == "equal columns":
        kind = "equal"  # (the same)
    if min(shape) == 1 and kind in ("gaussian", "positive"):
        assert error(shape, count, kind) <= 2e-5 + 6e-5  # (one row: of full rank)
    else:
        assert error(shape, count, kind) <= documented(shape, kind)


# around the limit of the 22-bit products, and well on either side
SIZES = [((64, 64), 1), ((128, 300), 1), ((257, 257), 1), ((300, 700), 1), ((700, 301), 1), ((384, 384), 1), ((384, 1537), 1), ((1000, 383), 40),
         ((385, 385), 1), ((385, 386), 160), ((390, 1533), 1), ((390, 1533), 120), ((1201, 400), 1), ((512, 2048), 40), ((1024, 1024), 1)]


@pytest.mark.parametrize("shape,count", SIZES)
@pytest.mark.parametrize("kind", ["gaussian", "rows", "positive", "signs"])
def test_full_rank(shape, count, kind):
    if kind == "signs":  # (signs of Gaussian values: roundings of one size, but the entries' sums average them out)
        assert error(shape, count, kind) <= documented(shape, "gaussian")
    else:
        assert error(shape, count, kind) <= documented(shape, kind)


@pytest.mark.parametrize("shape,count", SIZES)
@pytest.mark.parametrize("kind", ["1", "2", "5", "32", "128"])
def test_low_rank(shape, count, kind):
    assert error(shape, count, kind) <= documented(shape, kind)


@pytest.mark.parametrize("shape,count", SIZES)
@pytest.mark.parametrize("kind", ["equal", "equal rows", "equal columns", "blocks"])
def test_equal_entries(shape, count, kind):
    assert error(shape, count, kind) <= documented(shape, kind)
