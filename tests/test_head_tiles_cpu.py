"""How the head's products are cut up and dealt out, compiled from the source for the CPU: every tile once, every element of a
contraction once, workspaces that do not overlap."""
import ctypes
import os
import random
import subprocess

import pytest

from rows_on_cpu import CSRC, _definition

HOST = """
#include <algorithm>
#include <cstddef>
#include <cstring>
#define __device__
#define __forceinline__ inline
using std::max; using std::min;
enum { TLI_MAX_TARGETS = 256 };
static size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
constexpr int kHeadK = 64, kHeadN = 256, kHeadNear = 4, kHeadMinSteps = 8;
constexpr long long kHeadRunBytes = 256ll << 20;
enum : int { HEAD_STATS = 0, HEAD_SLOPE = 1, HEAD_GRADS = 2 };
struct HeadGemm { int H, cols, bn, early, splits, want_dh, want_dw; };
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    src = open(os.path.join(CSRC, "tli_head.cu")).read()
    for line in ("constexpr int kHeadK = 64;", "constexpr int kHeadN = 256;", "constexpr long long kHeadRunBytes = 256ll << 20;", "constexpr int kHeadMinSteps = 8;",
                 "constexpr int kHeadNear = 4;"):
        assert line in src
    code = HOST + _definition(src, "struct HeadTile ") + "\n" + _definition(src, "template <int MODE, int CG> struct HeadTiles") + "\n" + \
        _definition(src, "struct HeadPlan") + "\n" + _definition(src, "HeadPlan head_plan(") + """
template <int MODE, int CG> static int tiles(const HeadGemm &P, int rows, int ctas, int *out, int most) {
    int n = 0;
    for (int c = 0; c < ctas; ++c) {
        const HeadTiles<MODE, CG> t(P, rows, c, ctas);
        HeadTile w;
        for (int i = 0; t.get(P, i, w); ++i) {
            if (n == most) return -1;
            const int one[6] = {w.m, w.n, w.k0, w.ks, w.split, c};
            std::memcpy(out + 6 * n++, one, sizeof one);
        }
    }
    return n;
}
extern "C" int all_tiles(int mode, int cg, int H, int cols, int bn, int early, int splits, int dh, int dw, int rows, int ctas, int *out, int most) {
    const HeadGemm P = {H, cols, bn, early, splits, dh, dw};
    if (mode == HEAD_GRADS) return cg == 1 ? tiles<HEAD_GRADS, 1>(P, rows, ctas, out, most) : tiles<HEAD_GRADS, 2>(P, rows, ctas, out, most);
    return cg == 1 ? tiles<HEAD_STATS, 1>(P, rows, ctas, out, most) : tiles<HEAD_STATS, 2>(P, rows, ctas, out, most);
}
extern "C" void plan(int N, int H, int k, int V, int sms, int grad, long long *out) {
    const HeadPlan L = head_plan(N, H, k, V, sms, grad != 0);
    const long long all[] = {L.cg, L.bn, L.tiles, L.run, L.runs, L.splits, (long long)L.total, (long long)L.taking, (long long)L.n_valid, (long long)L.pos, (long long)L.by_row,
                             (long long)L.rowp, (long long)L.rows, (long long)L.part, (long long)L.tid, (long long)L.tval, (long long)L.tid_of, (long long)L.tval_of,
                             (long long)L.near_id, (long long)L.near_off, (long long)L.G, (long long)L.sums};
    std::memcpy(out, all, sizeof all);
}
"""
    d = tmp_path_factory.mktemp("head")
    (d / "x.cpp").write_text(code)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wno-sign-compare", "-fPIC", "-shared", "-o", str(d / "x.so"), str(d / "x.cpp")], check=True)
    return ctypes.CDLL(str(d / "x.so"))


def tiles_of(lib, mode, cg, H, cols, bn, early, splits, dh, dw, rows, ctas):
    most = 200000
    out = (ctypes.c_int * (6 * most))()
    n = lib.all_tiles(mode, cg, H, cols, bn, early, splits, dh, dw, rows, ctas, out, most)
    assert n >= 0
    return [tuple(out[6 * i:6 * i + 6]) for i in range(n)]


def test_every_tile_of_the_logits_once(lib):
    rng = random.Random(0)
    for _ in range(300):
        cg, early = rng.choice([1, 2]), rng.random() < 0.3
        H, cols, rows, ctas = 8 * rng.randint(1, 300), rng.randint(1, 30000), rng.randint(0, 128 * cg if early else 3000), rng.randint(1, 148 // cg)
        bn = rng.choice([64, 96, 224, 256]) if cg == 1 else 256
        got = tiles_of(lib, 0, cg, H, cols, bn, early, 1, 1, 1, rows, ctas)
        blocks = 1 if early else -(-rows // (128 * cg))
        want = {(m * 128 * cg, n * bn, 0, -(-H // 64), 0) for m in range(blocks) for n in range(-(-cols // bn))}
        assert len(got) == len(want) and {t[:5] for t in got} == want


def test_every_tile_and_step_of_the_gradients_once(lib):
    rng = random.Random(1)
    for _ in range(400):
        cg, early = rng.choice([1, 2]), rng.random() < 0.3
        H, cols, rows, ctas = 8 * rng.randint(1, 300), rng.randint(1, 9000), rng.randint(0, 128 * cg if early else 3000), rng.randint(1, 148 // cg)
        steps = -(-cols // 64)
        splits = rng.randint(1, max(1, steps // 8))
        dh, dw = rng.choice([(1, 1), (1, 0), (0, 1)])
        got = tiles_of(lib, 2, cg, H, cols, 0, early, splits, dh, dw, rows, ctas)
        blocks, wide = 1 if early else -(-rows // (128 * cg)), -(-H // 256)
        weight = [t for t in got if t[4] < 0]
        want = {(m * 128 * cg, n * 256, 0, -(-rows // 64)) for m in range(-(-cols // (128 * cg))) for n in range(wide)} if dw else set()
        assert len(weight) == len(want) and {t[:4] for t in weight} == want
        hidden = {}
        for m, n, k0, ks, split, _ in (t for t in got if t[4] >= 0):
            hidden.setdefault((m, n), []).append((k0, ks, split))
        assert set(hidden) == ({(m * 128 * cg, n * 256) for m in range(blocks) for n in range(wide)} if dh else set())
        for parts in hidden.values():
            parts.sort()
            assert [p[2] for p in parts] == list(range(splits)) and parts[0][0] == 0 and sum(p[1] for p in parts) == steps
            assert all(a[0] + 64 * a[1] == b[0] and a[1] > 0 for a, b in zip(parts, parts[1:]))


def test_gradients_tiles_come_out_even(lib):
    """2000 rows, a vocabulary of 49 152, H 1024, 74 pairs: no pair has more than a tile of d weight above the mean."""
    got = tiles_of(lib, 2, 2, 1024, 49152, 0, 0, 2, 1, 1, 2000, 74)
    load = [sum(t[3] for t in got if t[5] == c) for c in range(74)]
    assert max(load) <= sum(load) / 74 + 32


def test_plans(lib):
    rng = random.Random(2)
    for _ in range(500):
        N, H, k = rng.choice([1, 5, 128, 129, 1000, 8192, 70000, 262144]), 8 * rng.randint(1, 700), rng.randint(1, 256)
        V, grad = rng.choice([1, 255, 257, 32000, 128256, 1048576]), rng.randint(0, 1)
        out = (ctypes.c_longlong * 22)()
        lib.plan(N, H, k, V, 148, grad, out)
        cg, bn, tiles, run, runs, splits, total, *off = out
        assert cg == (1 if N <= 128 else 2) and bn % 32 == 0 and 64 <= bn <= 256 and tiles == -(-V // bn)
        sizes = dict(taking=-(-N // 32) * 4, n_valid=4, pos=4 * N, by_row=16 * N, rowp=16 * N, rows=2 * N * H)
        names = ["taking", "n_valid", "pos", "by_row", "rowp", "rows", "part", "tid", "tval", "tid_of", "tval_of", "near_id", "near_off", "G", "sums"]
        at = dict(zip(names, off))
        if grad:
            assert run % 256 == 0 and (runs - 1) * run < V <= runs * run and 1 <= splits <= max(1, min(V, run) // 64 // 8 + 1)
            sizes.update(tid=4 * N * k, tval=4 * N * k, tid_of=4 * N * k, tval_of=4 * N * k, near_id=16 * N, near_off=16 * N, G=2 * N * run, sums=4 * N * H * splits)
        else:
            sizes.update(part=8 * N * tiles)
        spans = sorted((at[n], at[n] + size) for n, size in sizes.items())
        assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:])) and spans[-1][1] <= total and all(a[0] % 256 == 0 for a in spans)
