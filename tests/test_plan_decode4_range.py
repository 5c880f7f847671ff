"""The shapes that put a sink before every form of decoding attention over a 4-bit cache
reach each of them."""
import test_gpu_decode4_range as gpu
from test_plan_decode4 import plans  # noqa: F401  (a fixture)


def test_the_sinks_meet_every_form(plans):  # noqa: F811
    problems = [(n_q, n_kv, d, keys, n_new) for n_q, n_kv, d, _, keys, n_new, _ in gpu.SINKS]
    forms = {(p[2], g[2], g[3], g[0] > 1) for p, g in zip(problems, plans(problems))}
    want = {(d, rows, waves, split) for d in (64, 128) for split in (False, True)
            for rows in (16, 32) for waves in (4, 8)}
    assert forms >= want, sorted(want - forms)


def test_the_gpu_shapes_meet_every_merge(plans):  # noqa: F811
    """The merge of up to 8, up to 16 and more splits, for few rows and many, whole
    workgroups of rows and a part of one."""
    problems = [(n_q, n_kv, d, keys, n_new)
                for n_q, n_kv, d, _, keys, n_new, _ in gpu.SINKS + gpu.ORDINARY]
    merges = set()
    for (n_q, _, d, _, n_new), plan in zip(problems, plans(problems)):
        splits, rows = plan[0], n_q * n_new
        if splits > 1:
            groups = 1 if splits <= 8 else 2 if splits <= 16 else 1024 // d
            merges.add((d, groups))
            if groups <= 2:
                merges.add((d, groups, rows % (1024 // d // groups) != 0, rows < 256))
    for d in (64, 128):
        assert {(d, 1), (d, 2), (d, 1024 // d)} <= merges
        assert {(d, g, True, few) for g in (1, 2) for few in (False, True)} <= merges, merges
