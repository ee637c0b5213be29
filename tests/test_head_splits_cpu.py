"""Cuts of d hidden's contraction in runs of the vocabulary that are shorter than the run they were made for: some have no step."""
import ctypes
import random

from test_head_tiles_cpu import lib, tiles_of  # noqa: F401  (a fixture)


def test_splits_without_a_step(lib):  # noqa: F811
    rng, empty = random.Random(3), 0
    for _ in range(300):
        cg = rng.choice([1, 2])
        H, cols, rows, ctas = 8 * rng.randint(1, 100), rng.randint(1, 1500), rng.randint(1, 1000), rng.randint(1, 148 // cg)
        steps, splits = -(-cols // 64), rng.randint(1, 74)
        got = tiles_of(lib, 2, cg, H, cols, 0, False, splits, 1, 1, rows, ctas)
        hidden = {}
        for m, n, k0, ks, split, _ in (t for t in got if t[4] >= 0):
            hidden.setdefault((m, n), []).append((split, k0, ks))
        assert len(hidden) == -(-rows // (128 * cg)) * -(-H // 256)
        for parts in hidden.values():
            parts.sort()
            assert [p[0] for p in parts] == list(range(splits))              # every split's sums are written
            at = 0
            for _, k0, ks in parts:
                assert ks >= 0 and k0 == 64 * at
                at += ks
                empty += ks == 0
            assert at == steps
        weight = [t for t in got if t[4] < 0]
        assert len(weight) == len(set(weight)) == -(-cols // (128 * cg)) * -(-H // 256) and all(t[3] == -(-rows // 64) for t in weight)
    assert empty > 1000


def test_a_plan_whose_last_run_is_shorter_than_its_splits(lib):  # noqa: F811
    out = (ctypes.c_longlong * 22)()
    lib.plan(9400, 8, 1, 760351, 148, 1, out)
    cg, _, _, run, runs, splits = list(out)[:6]
    last = 760351 - (runs - 1) * run
    assert (cg, run, runs, splits, last) == (2, 14080, 55, 2, 31)
    got = tiles_of(lib, 2, 2, 8, last, 0, False, splits, 1, 1, 9400, 74)
    assert {(t[4], t[3]) for t in got if t[4] >= 0} == {(0, 0), (1, 1)}
