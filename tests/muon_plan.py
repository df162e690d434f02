"""How a set of matrices would be worked on by a device of 148 SMs; needs none."""
import ctypes

from paper_2411_19870_b200 import binding


def plan(shapes):
    """Of each group: 22 bits or 11, tile, matrices, tasks, tasks at once, workers, whether the first matrix does the first two iterations in one."""
    lib = binding.load_library()
    cfg = binding.DemoMuonConfig(0.95, 1, 5, (ctypes.c_float * 3)(3.4445, -4.7750, 2.0315), 1e-7, 1e-3, 0.1, 2, binding.DEMO_BF16)
    descs = (binding.DemoTensorDesc * len(shapes))()
    for d, s in zip(descs, shapes):
        d.ndim, d.shape[0], d.shape[1] = 2, s[0], s[1]
    most = 64
    out = (ctypes.c_int * (7 * most))()
    n = lib.demo_muon_plan(ctypes.byref(cfg), descs, len(shapes), 148, out, most)
    assert 0 < n <= most
    return [tuple(out[7 * i:7 * i + 7]) for i in range(n)]
