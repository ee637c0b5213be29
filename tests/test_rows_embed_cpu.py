"""What of the filtered sampler and the embedding calls needs no GPU: refusals before any CUDA call, the struct layouts,
and the plain fp64 forms the GPU tests compare with, pinned by brute force."""
import ctypes

import numpy as np

import row_oracle as ro
from paper_2502_05202_b200 import build as tli_build, tli


def test_null_arguments_are_refused():
    tli_build.build()
    lib = tli.load()
    for name, args in (("tli_sample", tli.tli_sample_args), ("tli_filter", tli.tli_filter_args), ("tli_embed", tli.tli_embed_args),
                       ("tli_embed_grad", tli.tli_embed_grad_args)):
        call = getattr(lib, name)
        assert call(None, ctypes.byref(args()), None) == tli.TLI_ERR_ARG
        assert call(None, None, None) == tli.TLI_ERR_ARG
    assert lib.tli_sample_workspace_bytes(None, 1, 1, 0, 0) == 0
    assert lib.tli_filter_workspace_bytes(None, 1, 1, 0, 0) == 0
    assert lib.tli_embed_grad_workspace_bytes(None, 1, 1) == 0


def brute_kept(z, tau, k, p, mp):
    """Token by token, from the definition."""
    order = sorted((i for i in range(len(z)) if z[i] > -np.inf), key=lambda i: (-z[i], i))
    w = {i: np.exp((z[i] - z[order[0]]) / tau) for i in order}
    order = order[:k] if k > 0 else order
    total, run, kept = sum(w[i] for i in order), 0.0, []
    for n, i in enumerate(order):
        if n == 0 or ((p >= 1 or run < p * total) and (mp <= 0 or w[i] >= mp)):
            kept.append(i)
        run += w[i]
    return sorted(kept)


def test_the_plain_kept_set_against_brute_force():
    rng = np.random.default_rng(0)
    for trial in range(400):
        V = int(rng.integers(1, 9))
        z = rng.integers(-3, 4, V) * 0.75                                     # ties
        z[rng.random(V) < 0.2] = -np.inf
        if not (z > -np.inf).any():
            continue
        tau, k, p, mp = rng.choice([0.5, 1.0, 2.0]), int(rng.integers(0, 6)), rng.choice([1.0, 0.3, 0.77, 0.95]), rng.choice([0.0, 0.1, 0.6])
        ids, w, status = ro.kept_ids(z, np.ones(V, bool), tau, k, p, mp)
        assert status == 0 and list(ids) == brute_kept(z, tau, k, p, mp)
        # the whole unit interval goes to the kept ids in proportion to their weights
        us = (np.arange(4000) + 0.5) / 4000
        share = np.bincount([ro.sample_row(ids, w, u)[0] for u in us], minlength=V) / 4000
        want = np.zeros(V)
        want[ids] = w / w.sum()
        assert np.abs(share - want).max() <= 1 / 4000 + 1e-9


def test_ids_carried_between_vocabularies():
    m = np.array([3, -1, 0], np.int32)                                        # drafter 0 -> target 3, drafter 2 -> target 0
    assert list(ro.table_ids([0, 1, 2, 3, -1], m, 5, 1, 0)) == [3, -1, 0, -1, -1]
    assert list(ro.table_ids([0, 1, 3, 4, 5, -2], m, 5, 0, 1)) == [2, -1, 0, -1, -1, -1]
    assert list(ro.table_ids([0, 4, 5], m, 5, 0, 0)) == [0, 4, -1]


def test_packed_arguments_are_laid_out_as_the_structs():
    for pack, cls in ((tli._PACK_SAMPLE, tli.tli_sample_args), (tli._PACK_FILTER, tli.tli_filter_args), (tli._PACK_EMBED, tli.tli_embed_args),
                      (tli._PACK_EMBED_GRAD, tli.tli_embed_grad_args)):
        values = [1.5 if t is ctypes.c_float else 3 + 7 * i for i, (_, t) in enumerate(cls._fields_)]
        filled = cls.from_buffer_copy(bytes(ctypes.sizeof(cls)))
        for (name, _), x in zip(cls._fields_, values):
            setattr(filled, name, x)
        assert pack(*values) == bytes(filled)
