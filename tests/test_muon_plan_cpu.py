"""How the workers of a device of 148 SMs are divided among the matrices of a set: the plan, made without a device."""
import pytest

from tests.muon_plan import plan

WORKERS = 148 // 2


MIXED = [[(512, 512), (64, 64)], [(1024, 1024), (10, 20)], [(700, 500), (500, 1400), (256, 300)], [(768, 512), (256, 640), (128, 128)],
         [(512, 4608)] * 2 + [(1000, 512), (512, 147)], [(1024, 1024)] * 4 + [(256, 512)], [(512, 4608)] * 4 + [(512, 147), (7511, 512)],
         [(1024, 1024)] * 2 + [(256, 1024)] * 2 + [(1024, 2816)] * 2 + [(2816, 1024)],
         [(2048, 2048)] * 2 + [(256, 2048)] * 2 + [(2048, 8192)] * 2 + [(8192, 2048)], [(400, 400)] + [(384, 384)] * 40, [(1024, 1024)] + [(256, 1024)] * 30]


@pytest.mark.parametrize("shapes", MIXED, ids=range(len(MIXED)))
def test_division_between_small_and_larger_matrices(shapes):
    groups = plan(shapes)
    small, large = ([g for g in groups if g[0] == k] for k in (1, 0))
    assert small and large
    for g in groups:
        assert 1 <= g[5] <= g[4]
    kept, given = (max(g[5] for g in k) for k in (large, small))
    assert kept + given <= WORKERS
    # the larger ones have no fewer workers than the small ones could leave them, unless the small ones are the most of the work
    tasks = [sum(g[3] for g in k) for k in (large, small)]
    if tasks[0] >= tasks[1]:
        assert kept >= min(max(g[4] for g in large), WORKERS - max(g[4] for g in small))
        assert kept >= given or kept == max(g[4] for g in large)


@pytest.mark.parametrize("shapes", [[(256, 512)], [(64, 64)] * 300, [(1024, 4096)] * 3, [(1, 7)]])
def test_one_kind_has_the_device(shapes):
    for g in plan(shapes):
        assert g[5] == min(g[4], WORKERS)


def test_groups():
    assert [g[2] for g in plan([(384, 384)] * 1100)] == [910, 190]  # 128 million elements
    assert len(plan([(1, 1 << 20)] * 20)) == 2                      # 3.5 GB
    assert [(g[0], g[2]) for g in plan([(384, 384)] * 3 + [(4096, 4096)] * 9)] == [(0, 8), (0, 1), (1, 3)]
