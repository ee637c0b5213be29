"""The row kernels with their threads in orders that a GPU need not show (rows_on_cpu.py): the same tokens, probabilities, kept sets and
status bits as the fp64 definition, and blocks that end, whatever runs first between two barriers."""
import numpy as np
import pytest

import row_oracle as ro
import rows_on_cpu as rc

ORDERS = range(6)


@pytest.fixture(scope="module")
def lib():
    return rc.build()


def check(lib, z, asks, dtype=0, part=None, order=0, seed=0, left=None, u=None):
    """Sampled (``u``: with this number for every row) and filtered against the definition; ``left``: how many rows the pick kernel is to leave to the
    spread kernel."""
    z = np.ascontiguousarray(z, np.float32)
    if dtype:
        z = (z.view(np.uint32) & 0xffff0000).view(np.float32)
    B, R, V = z.shape
    f = lambda i, t: np.array([asks[b % len(asks)][i] for b in range(B)], t)
    ask = f(0, np.float32), f(1, np.int32), f(2, np.float32), f(3, np.float32)
    u = np.full((B, R), u, np.float32) if u is not None else np.random.default_rng(seed).integers(0, 1 << 24, (B, R)).astype(np.float32) / np.float32(1 << 24)
    tokens, prob, status, kept = ro.rows(z.astype(np.float64), np.ones(V, bool) if part is None else part, *ask, u)
    got = rc.run(lib, z, dtype, ask, u, part, order, seed)
    np.testing.assert_array_equal(got["status"], status)
    np.testing.assert_array_equal(got["tokens"], tokens)
    np.testing.assert_allclose(got["prob"], prob, rtol=2.0 ** -24 + 1e-12, atol=2.0 ** -149)
    assert left is None or got["left"] == left
    got = rc.run(lib, z, dtype, ask, None, part, order, seed)
    np.testing.assert_array_equal(got["status"], status)
    np.testing.assert_array_equal(got["kept"][status == 0], kept[status == 0])


@pytest.mark.parametrize("order", ORDERS)
def test_lists_of_hundreds(lib, order):
    """257 to 4096 listed elements: the search begins to count in the word that the list's length was read from."""
    z = np.random.default_rng(1).normal(0, 3, (4, 1, 3000))
    check(lib, z, [(1.0, 500, 1.0, 0.0), (1.0, 0, 0.95, 0.0), (1.0, 400, 0.9, 0.0), (1.0, 2999, 1.0, 0.0)], order=order, left=0)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("scale", [1, 3])
def test_lists_of_several_warps(lib, scale, order):
    """33 to 256 listed elements: the drawn one is left in the word that the border was read from."""
    z = np.random.default_rng(scale).normal(0, scale, (12, 1, 4096))
    for seed in range(4):
        check(lib, z, [(1.0, 100, 1.0, 0.0), (1.0, 60, 1.0, 0.0), (1.0, 128, 0.9, 0.0)], order=order, seed=seed, left=0)


def tail(rng, shape, scale):
    return rng.normal(0, scale, shape) - 1.1 * np.log1p(rng.permutation(shape[-1]))


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", [0, 1])
def test_every_way_through_the_kernels(lib, dtype, order):
    """Rows without filters, of one id, of short and long lists, left to the spread kernel, settled there from the list and by digits."""
    rng = np.random.default_rng(7 + dtype)
    asks = [(1.0, 0, 1.0, 0.0), (0.0, 0, 0.9, 0.0), (1.0, 1, 1.0, 0.0), (0.8, 50, 0.9, 0.0), (1.0, 0, 1.0, 0.05), (1.3, 0, 0.9, 0.0),
            (1.0, 3000, 1.0, 0.0), (1.0, 3000, 0.9, 0.01), (1.0, 7000, 0.8, 0.0), (1.0, 0, 0.99, 1e-4), (-1.0, 0, 1.0, 0.0), (1.0, 0, np.nan, 0.0)]
    z = np.concatenate([tail(rng, (len(asks), 1, 9001), 3), rng.normal(0, 0.05, (len(asks), 1, 9001))], axis=1)
    check(lib, z, asks, dtype=dtype, order=order, seed=order)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("dtype", [0, 1])
def test_ties_masks_and_nothing(lib, dtype, order):
    rng = np.random.default_rng(9 + dtype)
    asks = [(1.0, 0, 0.5, 0.0), (1.0, 70, 1.0, 0.0), (0.7, 2000, 0.9, 0.0), (1.0, 0, 1.0, 0.5), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0)]
    V = 5003
    z = rng.integers(0, 3, (len(asks), 6, V)) * 0.5
    part = rng.random(V) < 0.6
    z[:, 1] = -np.inf
    z[:, 2][:, rng.random(V) < 0.9] = -np.inf
    z[:, 3, np.flatnonzero(part)[5]] = np.nan
    z[:, 4] = rng.normal(0, 1, (len(asks), V))
    z[:, 4, np.flatnonzero(~part)[::3]] = np.nan
    z[:, 5] = 1.0
    check(lib, z, asks, dtype=dtype, part=part, order=order, seed=order)


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("u", [0.0, 1.0 - 2.0 ** -24])
def test_the_ends_of_the_uniform(lib, u, order):
    rng = np.random.default_rng(11)
    asks = [(1.0, 100, 1.0, 0.0), (1.0, 1000, 1.0, 0.0), (1.0, 3000, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.02, 0, 0.99, 0.0), (1.0, 5000, 0.99, 0.0)]
    check(lib, rng.normal(0, 1, (len(asks), 1, 32003)), asks, order=order, u=u)


@pytest.mark.parametrize("bits", [43.1, 44.1, 45.1])
@pytest.mark.parametrize("k,V", [(8000, 9001), (8999, 9001), (30000, 40001)])
def test_top_k_by_digits_counts_small_weights(lib, k, V, bits):
    """An id of weight 1, one of 1 - d and k - 2 of 2^-bits or a little less, of 2 d in all or a little more: half of their mass is more than the first id has, so
    top-p 1/2 keeps two.  Without the small ones it keeps one.  The border lies d / 2 from the first id's mass, more than 1e-11 of the mass."""
    z = (-bits - 0.3 * np.random.default_rng(k).random((1, 1, V))) * np.log(2.0)
    d = (k - 2) * 2.0 ** (-bits - 0.3) / 2
    assert d / 4 > 1e-11
    z[0, 0, 17] = 0.0
    z[0, 0, 4001] = -d
    check(lib, z, [(1.0, k, 0.5, 0.0)], left=1)


LISTS = [(4096, 4000, 46.1, 0.3, 0), (4096, 4096, 46.1, 0.3, 0), (40001, 6000, 45.1, 3.0, 1), (40001, 5000, 45.1, 2.5, 1)]


@pytest.mark.parametrize("V,k,bits,width,left", LISTS)
def test_lists_count_small_weights(lib, V, k, bits, width, left):
    """The same among lists of thousands, in the pick kernel and settled by the spread kernel."""
    z = (-bits - width * np.random.default_rng(k).random((1, 1, V))) * np.log(2.0)
    d = (k - 2) * 2.0 ** (-bits - 0.5) / 2
    assert d / 4 > 4e-12
    z[0, 0, 17] = 0.0
    z[0, 0, 3001] = -d
    check(lib, z, [(1.0, k, 0.5, 0.0)], left=left)


@pytest.mark.parametrize("V,k,bits,width,left", LISTS)
def test_draws_among_small_weights(lib, V, k, bits, width, left):
    """All ids but the last have small weights, and the number falls among them: the drawn id owns it, up to 2e-12 of the mass."""
    z = (-bits - width * np.random.default_rng(k).random((1, 1, V))) * np.log(2.0)
    z[0, 0, V - 1] = 0.0
    z = z.astype(np.float32)
    ids, w, _ = ro.kept_ids(z[0, 0].astype(np.float64), np.ones(V, bool), 1.0, k, 1.0, 0.0)
    c = np.cumsum(w)
    u = np.float32(c[len(c) // 2] / c[-1])                                   # half of the small ones lie in front
    assert 5e-12 < u < 1e-9
    got = rc.run(lib, z, 0, (np.ones(1, np.float32), np.full(1, k, np.int32), np.ones(1, np.float32), np.zeros(1, np.float32)), np.full((1, 1), u, np.float32))
    assert got["left"] == left and got["status"][0, 0] == 0
    at = np.flatnonzero(ids == got["tokens"][0, 0])[0]
    assert c[at] - w[at] - 2e-12 * c[-1] <= float(u) * c[-1] <= c[at] + 2e-12 * c[-1]


def test_powers_of_two_to_the_stated_error(lib):
    """exp2_neg() against 2^x in 64-bit mantissas: 1.5e-13 of the value, from 0 to where the weights are cut off."""
    import ctypes
    rng = np.random.default_rng(3)
    x = np.concatenate([-1020.0 * rng.random(200000), -40.0 * rng.random(200000), -np.arange(0, 1020.0, 1 / 32), -np.geomspace(1e-300, 1.0, 5000), [0.0]])
    out = np.empty_like(x)
    lib.exp2_on_cpu(ctypes.c_void_p(x.ctypes.data), ctypes.c_void_p(out.ctypes.data), ctypes.c_int(x.size))
    assert np.finfo(np.longdouble).nmant >= 63
    error = np.abs(out.astype(np.longdouble) / np.exp2(x.astype(np.longdouble)) - 1)
    assert 1e-13 < error.max() <= 1.5e-13 and out[-1] == 1.0
