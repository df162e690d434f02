"""The native calls of the orthogonalised updates and of AdamW (csrc/calls.cpp) without a device: which they take, what reaches the library."""
import ctypes

import pytest
import torch

from paper_2411_19870_b200 import binding

vp, i32 = ctypes.c_void_p, ctypes.c_int32
ORTHOGONALIZE = ctypes.CFUNCTYPE(ctypes.c_int, vp, vp, i32, vp, i32, vp)
STEP = ctypes.CFUNCTYPE(ctypes.c_int, vp, vp, vp, vp, vp)
DECODE = ctypes.CFUNCTYPE(ctypes.c_int, vp, vp, vp, i32, vp, vp)
ADAMW = ctypes.CFUNCTYPE(ctypes.c_int, vp, vp, vp, vp, vp, vp, vp)


def at(address, n):
    return list((vp * n).from_address(address))


def ptrs(tensors):
    return [t.data_ptr() for t in tensors]


def address(f):
    return ctypes.cast(f, vp).value


class Sub(torch.Tensor):
    pass


@pytest.fixture()
def calls():
    return binding.load_calls()


# (more tensors than the lists hold without an allocation, too)
@pytest.mark.parametrize("n", [1, 5, 70])
def test_pointers_in_order(calls, n):
    shapes = [(4, 6 + i % 3) for i in range(n)]
    f32, bf16 = (calls.layouts(d, -1, shapes) for d in (torch.float32, torch.bfloat16))
    count = calls.layouts(torch.int64, -1, [(1,)])
    x, m, v = ([torch.zeros(s) for s in shapes] for _ in range(3))
    g = [torch.zeros(s, dtype=torch.bfloat16) for s in shapes]
    t = torch.zeros(1, dtype=torch.int64)
    p = [torch.zeros(16, dtype=torch.uint8) for _ in range(n + 1)]
    known = {(a.data_ptr(), a.numel()) for a in p}
    seen = []
    o = ORTHOGONALIZE(lambda *a: seen.append((a[0], at(a[1], n), a[2], at(a[3], n), a[4], a[5])) or 3)
    s = STEP(lambda *a: seen.append((a[0], at(a[1], n), at(a[2], n), at(a[3], n), a[4])) or 4)
    d = DECODE(lambda *a: seen.append((a[0], a[1], at(a[2], n + 1), a[3], at(a[4], n), a[5])) or 5)
    w = ADAMW(lambda *a: seen.append((a[0], at(a[1], n), at(a[2], n), at(a[3], n), at(a[4], n), a[5], a[6])) or 6)
    assert calls.orthogonalize(address(o), 64, bf16, g, 1, f32, tuple(x), 0, 9) == 3
    assert seen.pop() == (64, ptrs(g), 1, ptrs(x), 0, 9)
    assert calls.muon_step(address(s), 64, bf16, f32, g, m, x, 0) == 4 and seen.pop() == (64, ptrs(g), ptrs(m), ptrs(x), None)
    assert calls.muon_decode(address(d), 64, 72, known, p, f32, x, 9) == 5 and seen.pop() == (64, 72, ptrs(p), n + 1, ptrs(x), 9)
    assert calls.adamw_step(address(w), 64, bf16, f32, g, m, v, x, count, (t,), 9) == 6
    assert seen.pop() == (64, ptrs(g), ptrs(m), ptrs(v), ptrs(x), t.data_ptr(), 9)


def bad_lists(x):
    """Lists that are not what the call was made for."""
    return {"number": x + x[:1], "type": [x[0].double()] + x[1:], "shape": [x[0].view(6, 4)] + x[1:], "order": [torch.zeros(6, 4).t()] + x[1:],
            "subclass": [x[0].as_subclass(Sub)] + x[1:], "iterator": iter(x), "none": None, "not tensors": [1, 2]}


@pytest.mark.parametrize("which", sorted(bad_lists([torch.zeros(4, 6)] * 2)))
def test_what_does_not_fit_is_left_to_the_checks(calls, which):
    shapes = [(4, 6), (4, 6)]
    f32, count = calls.layouts(torch.float32, -1, shapes), calls.layouts(torch.int64, -1, [(1,)])
    x, t = [torch.zeros(s) for s in shapes], torch.zeros(1, dtype=torch.int64)
    p = torch.zeros(16, dtype=torch.uint8)
    known = {(p.data_ptr(), p.numel())}
    seen = []
    o, s, d, w = (f(lambda *a: seen.append(a) or 0) for f in (ORTHOGONALIZE, STEP, DECODE, ADAMW))

    def new():
        return bad_lists(x)[which]  # (an iterator serves once)

    for k in range(2):
        args = [x, x]
        args[k] = new()
        assert calls.orthogonalize(address(o), 64, f32, args[0], 0, f32, args[1], 0, 0) is None
    for k in range(3):
        args = [x] * 3
        args[k] = new()
        assert calls.muon_step(address(s), 64, f32, f32, *args, 0) is None
    for k in range(4):
        args = [x] * 4
        args[k] = new()
        assert calls.adamw_step(address(w), 64, f32, f32, *args, count, (t,), 0) is None
    assert calls.adamw_step(address(w), 64, f32, f32, x, x, x, x, count, new(), 0) is None
    assert calls.muon_decode(address(d), 64, 72, known, [p], f32, new(), 0) is None
    assert calls.muon_decode(address(d), 64, 72, known, new(), f32, x, 0) is None
    assert not seen


def test_unknown_payloads_and_counts_are_left_to_the_checks(calls):
    f32, count = calls.layouts(torch.float32, -1, [(4, 6)]), calls.layouts(torch.int64, -1, [(1,)])
    x, p = [torch.zeros(4, 6)], torch.zeros(16, dtype=torch.uint8)
    seen = []
    d, w = (f(lambda *a: seen.append(a) or 0) for f in (DECODE, ADAMW))
    assert calls.muon_decode(address(d), 64, 72, set(), [p], f32, x, 0) is None
    assert calls.muon_decode(address(d), 64, 72, {(p.data_ptr(), 16)}, [p[:8]], f32, x, 0) is None
    for t in (torch.zeros(1, dtype=torch.int32), torch.zeros((), dtype=torch.int64), torch.zeros(2, dtype=torch.int64)):
        assert calls.adamw_step(address(w), 64, f32, f32, x, x, x, x, count, (t,), 0) is None
    assert not seen


def test_errors_of_the_arguments_are_raised(calls):
    f32 = calls.layouts(torch.float32, -1, [(4, 6)])
    x = [torch.zeros(4, 6)]
    for name in ("orthogonalize", "muon_step", "muon_decode", "adamw_step"):
        with pytest.raises(TypeError):
            getattr(calls, name)(1, 2)
    with pytest.raises(TypeError):
        calls.orthogonalize(1, 64, f32, x, "fp32", f32, x, 0, 0)
    with pytest.raises(ValueError):
        calls.muon_step(1, 64, object(), f32, x, x, x, 0)
