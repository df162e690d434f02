"""Orthogonalised updates and AdamW without a device: refusals, which come before any CUDA call, and the reference's own identities."""
import ctypes
import math

import pytest
import torch

import paper_2411_19870_b200 as demo
from paper_2411_19870_b200 import binding
from tests import muon_reference as ref


def _muon(shapes=((64, 32),), **kw):
    args = dict(lr=1e-2, weight_decay=0.1)
    args.update(kw)
    return demo.MuonTransform(shapes, **args)


@pytest.mark.parametrize("shapes,kw,status", [
    ([(64,)], {}, 2),
    ([(2, 3, 4)], {}, 2),
    ([(0, 4)], {}, 2),
    ([(4, (1 << 20) + 1)], {}, 2),
    ([], {}, 1),
    ([(4, 4)], {"steps": 0}, 1),
    ([(4, 4)], {"steps": 65}, 1),
    ([(4, 4)], {"eps": -1.0}, 1),
    ([(4, 4)], {"lr": float("inf")}, 1),
    ([(4, 4)], {"momentum": float("nan")}, 1),
    ([(4, 4)], {"coefficients": (1.0, float("nan"), 0.0)}, 1),
    ([(4, 4)], {"scale": 3}, 1),
    ([(4, 4)], {"nesterov": 2}, 1),
    ([(4, 4)], {"grad_dtype": 7}, 4),
    ([(4, 4)], {"device": -1}, 1),
])
def test_muon_arguments(shapes, kw, status):
    with pytest.raises(demo.DemoError) as e:
        _muon(shapes, **kw)
    assert e.value.status == status


@pytest.mark.parametrize("shapes,kw,status", [
    ([(0,)], {}, 2),
    ([((1 << 40) + 1,)], {}, 2),
    ([], {}, 1),
    ([(4,)], {"beta1": 1.0}, 1),
    ([(4,)], {"beta2": -0.1}, 1),
    ([(4,)], {"eps": -1e-8}, 1),
    ([(4,)], {"weight_decay": float("nan")}, 1),
    ([(4,)], {"grad_dtype": 2}, 4),
])
def test_adamw_arguments(shapes, kw, status):
    args = dict(lr=1e-2, weight_decay=0.1)
    args.update(kw)
    with pytest.raises(demo.DemoError) as e:
        demo.AdamwTransform(shapes, **args)
    assert e.value.status == status


def test_coefficients_are_three():
    with pytest.raises(ValueError):
        _muon(coefficients=(1.0, 2.0))


def test_null_arguments():
    lib = demo.load_library()
    assert lib.demo_muon_init(None, None, None, 0, 0) == 1
    assert lib.demo_orthogonalize(None, None, 0, None, 0, None) == 1
    assert lib.demo_muon_step(None, None, None, None, None) == 1
    assert lib.demo_muon_decode_apply(None, None, None, 0, None, None) == 1
    assert lib.demo_muon_set_lr(None, 1.0) == 1
    assert lib.demo_muon_workspace_bytes(None) == 0
    assert lib.demo_muon_launch_count(None) == 0
    assert lib.demo_muon_device_status(None, None) == 1
    lib.demo_muon_free(None)
    assert lib.demo_adamw_init(None, None, None, 0, 0) == 1
    assert lib.demo_adamw_step(None, None, None, None, None, None, None) == 1
    assert lib.demo_adamw_set_lr(None, 1.0) == 1
    assert lib.demo_adamw_launch_count(None) == 0
    lib.demo_adamw_free(None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="needs a machine without a device")
def test_no_device_no_context():
    for make in (_muon, lambda: demo.AdamwTransform([(4,)], lr=1e-2, weight_decay=0.0)):
        with pytest.raises(demo.DemoError) as e:
            make()
        assert e.value.status == 6


def test_config_layouts_match_the_header():
    assert ctypes.sizeof(binding.DemoMuonConfig) == 44
    assert ctypes.sizeof(binding.DemoAdamwConfig) == 32


@pytest.mark.parametrize("dtype,shape,contiguous", [(torch.float16, (4, 6), True), (torch.float32, (6, 4), True), (torch.float32, (4, 6), False)])
def test_tensors_are_checked(dtype, shape, contiguous):
    t = torch.zeros(shape, dtype=dtype)
    if not contiguous:
        t = torch.zeros(shape[::-1], dtype=dtype).t()
    with pytest.raises(ValueError):
        binding._checked([t], [(4, 6)], torch.float32, None, "grads")
    with pytest.raises(ValueError):
        binding._checked([], [(4, 6)], torch.float32, None, "grads")
    with pytest.raises(ValueError):  # on the host
        binding._checked([torch.zeros(4, 6)], [(4, 6)], torch.float32, 0, "grads")


def test_reference_polynomial_acts_on_singular_values():
    u = torch.randn(12, 20, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    left, s, right = torch.linalg.svd(u, full_matrices=False)
    a, b, c = ref.COEFFICIENTS
    s = s / math.sqrt(float((u * u).sum()))
    for _ in range(5):
        s = a * s + b * s ** 3 + c * s ** 5
    want = (left * s) @ right
    for x, y in ((u, want), (u.t(), want.t())):
        assert float((ref.orthogonal(x, eps=0.0) - y).abs().max()) < 1e-12
    assert float(s.min()) > 0.3 and float(s.max()) < 1.3


def test_reference_gradient_of_a_step_by_differences():
    """The converged iteration (a, b, c = 1.875, -1.25, 0.375) gives the direction of steepest descent in the spectral norm: no other
    matrix of spectral norm one has a larger product with U than the nuclear norm."""
    u = torch.randn(6, 9, generator=torch.Generator().manual_seed(2), dtype=torch.float64)
    o = ref.orthogonal(u, steps=40, coefficients=(1.875, -1.25, 0.375))
    assert abs(float((o * u).sum()) - float(torch.linalg.svdvals(u).sum())) < 1e-9
    assert abs(float(torch.linalg.matrix_norm(o, 2)) - 1) < 1e-9
