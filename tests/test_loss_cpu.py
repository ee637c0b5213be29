"""What of the losses needs no GPU: refusals before any CUDA call, the struct layouts, and the fp64 forms the GPU tests compare
with, pinned by a second writing and by differences."""
import ctypes

import numpy as np

import loss_oracle as lo
from paper_2502_05202_b200 import build as tli_build, tli

CALLS = (("tli_loss", tli.tli_loss_args, "_PACK_LOSS"), ("tli_loss_grad", tli.tli_loss_grad_args, "_PACK_LOSS_GRAD"),
         ("tli_head_loss", tli.tli_head_loss_args, "_PACK_HEAD_LOSS"), ("tli_head_loss_grad", tli.tli_head_loss_grad_args, "_PACK_HEAD_LOSS_GRAD"))


def test_null_arguments_are_refused():
    tli_build.build()
    lib = tli.load()
    for name, args, _ in CALLS:
        assert getattr(lib, name)(None, ctypes.byref(args()), None) == tli.TLI_ERR_ARG
        assert getattr(lib, name)(None, None, None) == tli.TLI_ERR_ARG
    assert lib.tli_head_loss_workspace_bytes(None, 1, 8, 1, 0) == 0 and lib.tli_head_loss_grad_workspace_bytes(None, 1, 8, 1, 0) == 0


def test_packed_arguments_are_laid_out_as_the_structs():
    for _, cls, pack in CALLS:
        values = [3 + 7 * i for i in range(len(cls._fields_))]
        filled = cls.from_buffer_copy(bytes(ctypes.sizeof(cls)))
        for (name, _), x in zip(cls._fields_, values):
            setattr(filled, name, x)
        assert getattr(tli, pack)(*values) == bytes(filled)


def some_rows(rng, N, V, k):
    part = rng.random(V) < 0.7
    part[0] = True
    z = rng.normal(0, 2, (N, V))
    z[rng.random((N, V)) < 0.1] = -np.inf
    z[:, 0] = 0.5
    t = rng.integers(-1, V, (N, k))
    t[:, 0] = 0
    return z, part, t, rng.normal(0, 2, (N, k)), rng.choice([0.5, 1.0, 3.0], N)


def test_the_plain_loss_against_a_second_writing():
    rng = np.random.default_rng(0)
    for _ in range(50):
        z, part, t, teacher, tau = some_rows(rng, 4, 9, 3)
        loss, stats, status, q, p, _, _ = lo.rows(z, part, t, teacher, tau)
        for n in range(4):
            w = {v: np.exp(z[n, v] / tau[n]) for v in range(9) if part[v]}
            e = [(x, np.exp(y / tau[n])) for x, y in zip(t[n], teacher[n]) if x >= 0 and part[x]]
            total = sum(y for _, y in e)
            value = 0.0
            for x, y in e:
                with np.errstate(divide="ignore"):
                    value += y / total * (np.log(y / total) - np.log(w[x] / sum(w.values())))
            assert status[n] == 0 and (loss[n] == value or abs(loss[n] - value) < 1e-12)
            assert abs(q[n].sum() - 1) < 1e-12 and abs(p[n].sum() - 1) < 1e-12 and (q[n][~part] == 0).all()
            assert abs(stats[n, 1] * np.exp(stats[n, 0] / tau[n]) - sum(w.values())) < 1e-9


def test_the_plain_gradient_against_differences():
    rng = np.random.default_rng(1)
    z, part, t, teacher, tau = some_rows(rng, 3, 8, 4)
    z = np.where(np.isfinite(z), z, -5.0)
    _, _, _, q, p, _, _ = lo.rows(z, part, t, teacher, tau)
    for v in range(8):
        e = np.zeros_like(z)
        e[:, v] = 1e-6
        d = (lo.rows(z + e, part, t, teacher, tau)[0] - lo.rows(z - e, part, t, teacher, tau)[0]) / 2e-6
        assert np.abs(d - (q - p)[:, v] / tau).max() < 1e-8


def test_rows_the_definition_leaves_out():
    z = np.array([[1.0, 2.0, 3.0]] * 5)
    z[2] = -np.inf
    z[3, 1] = np.nan
    part = np.array([True, True, False])
    t = np.array([[2, -1], [0, 1], [0, 1], [0, 1], [1, 1]])
    loss, stats, status, q, _, _, _ = lo.rows(z, part, t, np.zeros((5, 2)), np.array([1, -1, 1, 1, 1.0]))
    assert list(status) == [lo.LEFT_OUT, lo.BAD_TEMPERATURE, lo.FALLBACK, lo.NONFINITE, 0]
    assert (loss[:3] == 0).all() and np.isnan(loss[3]) and abs(loss[4] - (np.log1p(np.exp(-1)) - np.log(2))) < 1e-12    # (the same id twice: ln p is that of a half)
