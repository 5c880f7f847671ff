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
