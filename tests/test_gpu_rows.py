"""tli_sample() and tli_filter() against the fp64 definition: tokens, status bits and kept sets identical, prob to one
rounding to fp32 (2^-24 relative; the fp64 sums behind it differ by less than 1e-12)."""
import ctypes

import numpy as np
import pytest
import torch

import row_oracle as ro
from paper_2502_05202_b200 import tli, workload as wl

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
INF = float("inf")

# (tau, top_k, top_p, min_p): every filter alone, together, off in every way, and at its ends
ASKS = [(1.0, 0, 1.0, 0.0), (0.7, 1, 1.0, 0.0), (1.0, 5, 1.0, 0.0), (1.3, 40, 0.9, 0.0), (0.8, 0, 0.9, 0.0),
        (1.0, 0, 0.5, 0.05), (0.0, 0, 1.0, 0.0), (0.0, 7, 0.2, 0.9), (1.0, 0, 1.0, 0.02), (2.5, 0, 0.99, 0.0),
        (1.0, 10 ** 9, 2.0, -1.0), (1.0, -3, 1.0, 1.0), (1.0, 0, 1.0, 1.5), (1.0, 0, 0.0, 0.0), (0.9, 300, 0.97, 0.01),
        (1.0, 0, 1.0 - 2.0 ** -24, 0.0), (0.05, 64, 0.95, 0.0), (1.0, 2, 1e-6, 0.0)]


def numbers(rng, shape):
    return rng.integers(0, 1 << 24, shape).astype(np.float32) / np.float32(1 << 24)


def to_dtype(z, dtype):
    t = torch.from_numpy(np.ascontiguousarray(z, dtype=np.float32))
    return t.to(torch.bfloat16) if dtype == wl.BF16 else t


def a_map(rng, V_t, V_d, f):
    m = np.full(V_d, -1, np.int32)
    on = rng.permutation(V_d)[:min(V_t, max(1, int(round(f * V_d))))]
    m[on] = rng.permutation(V_t)[:on.size]
    return m


def verifier(rng, V, side, f=0.6):
    V_other = max(3, V // 2 + 1)
    V_t, V_d = (V, V_other) if side == T else (V_other, V)
    if side == D:
        V_t = V + 5
    m = a_map(rng, V_t, V_d, f)
    return tli.Verifier(V_t, V_d, m), (np.ones(V, bool) if side == T else m >= 0)


def asks(B, table=ASKS):
    per = [table[b % len(table)] for b in range(B)]
    f = lambda i, t: np.array([a[i] for a in per], t)
    return f(0, np.float32), f(1, np.int32), f(2, np.float32), f(3, np.float32)


def check(v, side, part, z, ask, u, in_place=False):
    """z: CPU tensor [B,R,V] or a CUDA view of one; both calls against the definition.  Returns the kept mask."""
    dev = z if z.is_cuda else z.cuda()
    z64 = dev.double().cpu().numpy()
    tau, k, p, mp = ask
    dt, dk, dp, dm = (torch.from_numpy(x).cuda() for x in (tau, k, p, mp))
    tokens, prob, status, kept = ro.rows(z64, part, tau, k, p, mp, u)
    out = v.sample(dev, dt, torch.from_numpy(u).cuda(), side=side, top_k=dk, top_p=dp, min_p=dm)
    again = v.sample(dev, dt, torch.from_numpy(u).cuda(), side=side, top_k=dk, top_p=dp, min_p=dm)
    fil = v.filter(dev, dt, side=side, top_k=dk, top_p=dp, min_p=dm)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(out["status"].cpu().numpy(), status)
    np.testing.assert_array_equal(out["tokens"].cpu().numpy(), tokens)
    np.testing.assert_allclose(out["prob"].cpu().numpy(), prob, rtol=2.0 ** -24 + 1e-12, atol=2.0 ** -149)
    for name in out:
        assert torch.equal(out[name], again[name]), name
    np.testing.assert_array_equal(fil["status"].cpu().numpy(), status)
    expect = dev.clone()
    expect[torch.from_numpy(~kept).cuda()] = -INF
    same = torch.from_numpy(status & ~ro.FALLBACK != 0).cuda()
    expect[same] = dev[same]
    as_bits = lambda t: t.contiguous().view(torch.int16 if t.dtype == torch.bfloat16 else torch.int32)
    assert torch.equal(as_bits(fil["logits"]), as_bits(expect))
    if in_place:
        own = dev.clone()
        res = v.filter(own, dt, side=side, top_k=dk, top_p=dp, min_p=dm, out=own)
        assert res["logits"].data_ptr() == own.data_ptr()
        assert torch.equal(as_bits(own), as_bits(expect))
    return kept


@pytest.mark.parametrize("side", [T, D])
@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("V", [1, 2, 7, 13, 257, 1000, 4099, 33001])
def test_every_filter_on_small_and_ragged_rows(V, dtype, side):
    rng = np.random.default_rng(1000 + V + 7 * dtype + 3 * side)
    v, part = verifier(rng, V, side)
    B, R = len(ASKS), 2
    z = rng.normal(0, 3, (B, R, V)) - 1.1 * np.log1p(rng.permutation(V))
    check(v, side, part, to_dtype(z, dtype), asks(B), numbers(rng, (B, R)), in_place=True)


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("values", [1, 2, 9])
@pytest.mark.parametrize("V", [37, 3000, 40001])
def test_ties_go_to_the_lowest_ids(V, values, dtype):
    """Rows of a few distinct values: the border lies inside a run of equal logits, up to the whole row.  Zeros of both signs are equal."""
    rng = np.random.default_rng(V + values)
    v, part = verifier(rng, V, T)
    B = len(ASKS)
    z = rng.integers(0, values, (B, 1, V)) * 0.5
    z[rng.random(z.shape) < 0.3] *= -0.0
    u = numbers(rng, (B, 1))
    check(v, T, part, to_dtype(z, dtype), asks(B), u)


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("scale", [0.01, 0.3, 2.0])
def test_kept_sets_of_thousands(scale, dtype):
    """Flat rows and large k: the kept set is far larger than what is sorted."""
    rng = np.random.default_rng(int(scale * 100) + dtype)
    V = 60013
    v, part = verifier(rng, V, T)
    table = [(1.0, 0, 0.9, 0.0), (1.0, 5000, 1.0, 0.0), (1.0, 20000, 0.8, 0.0), (0.7, 0, 0.5, 0.001), (1.0, 2047, 1.0, 0.0),
             (1.0, 2049, 0.9999, 0.0), (1.0, 59999, 1.0, 0.3), (1.0, 0, 0.999, 0.0), (1.0, 0, 1.0, 0.5), (1.0, 50000, 0.01, 0.0)]
    B = len(table)
    z = rng.normal(0, scale, (B, 1, V))
    kept = check(v, T, part, to_dtype(z, dtype), asks(B, table), numbers(rng, (B, 1)))
    assert scale > 1 or kept.sum(-1).max() > 10000


@pytest.mark.parametrize("side", [T, D])
@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_top_k_of_thousands_with_top_p(dtype, side):
    """Around the lengths of the lists: as many elements as fit, one more, and far more."""
    rng = np.random.default_rng(31)
    V = 32003
    v, part = verifier(rng, V, side, f=0.9)
    table = [(1.0, k, p, m) for k in (1024, 1537, 2048, 3000, 4096, 4097, 6143, 6144, 6145, 8192, 8193) for p, m in ((0.99, 0.0), (0.6, 1e-3))]
    B = len(table)
    z = np.stack([rng.normal(0, 1, (B, V)), rng.normal(0, 0.05, (B, V))], axis=1)
    check(v, side, part, to_dtype(z, dtype), asks(B, table), numbers(rng, (B, 2)))


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("V", [40001, 128256, 300007])
def test_a_few_large_elements_over_a_heavy_tail(V, dtype):
    """Most of the mass in two or three elements, side by side or apart; the border among them, just behind them, or far down the tail."""
    rng = np.random.default_rng(V + dtype)
    v, part = verifier(rng, V, T)
    table = [(1.0, 0, p, m) for p in (0.5, 0.9, 0.915, 0.925, 0.95, 0.99) for m in (0.0, 1e-4)]
    B = len(table)
    z = rng.normal(0, 1.5, (B, 4, V))
    tail = np.log(np.exp(z).sum(-1))
    for r, (many, apart) in enumerate(((2, 1), (3, 1), (2, 5000), (3, 3))):
        for j in range(many):
            z[:, r, 9000 + j * apart] = tail[:, r] + np.log(0.92 / 0.08 / many)
    kept = check(v, T, part, to_dtype(z, dtype), asks(B, table), numbers(rng, (B, 4)))
    assert kept.sum(-1).min() <= 2 and kept.sum(-1).max() > 1000


@pytest.mark.parametrize("side", [T, D])
@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_masked_infinite_and_nan_logits(dtype, side):
    rng = np.random.default_rng(5 + dtype)
    V = 5003
    v, part = verifier(rng, V, side, f=0.5)
    lowest = torch.finfo(torch.bfloat16 if dtype == wl.BF16 else torch.float32).min
    B = 2 * len(ASKS)
    z = rng.normal(0, 2, (B, 8, V)).astype(np.float32)
    inside = np.flatnonzero(part)
    z[:, 0] = -INF                                          # nothing left
    z[:, 1] = -INF; z[:, 1, inside[len(inside) // 2]] = -7  # one id left
    z[:, 2][:, rng.random(V) < 0.9] = -INF
    z[:, 3] = lowest                                        # a mask of the type's lowest value everywhere
    z[:, 4][:, rng.random(V) < 0.9] = lowest
    z[:, 5, inside[3]] = np.nan
    z[:, 6, inside[-1]] = INF
    z[:, 7, inside[: len(inside) // 2]] = -INF
    if side == D:
        z[:, :3, np.flatnonzero(~part)[::3]] = np.nan       # outside the intersection: not examined
        z[:, 7, np.flatnonzero(~part)[::2]] = INF
    check(v, side, part, to_dtype(z, dtype), asks(B), numbers(rng, (B, 8)), in_place=True)


def test_bad_parameters_flag_the_row_and_leave_it_alone():
    rng = np.random.default_rng(9)
    v, part = verifier(rng, 700, T)
    table = [(-1.0, 3, 0.5, 0.1), (INF, 0, 1.0, 0.0), (np.nan, 0, 1.0, 0.0), (1.0, 0, np.nan, 0.0), (1.0, 0, 1.0, np.nan),
             (np.nan, 0, np.nan, 0.0), (1.0, 4, 1.0, 0.0)]
    B = len(table)
    z = to_dtype(rng.normal(0, 2, (B, 3, 700)), wl.F32)
    check(v, T, part, z, asks(B, table), numbers(rng, (B, 3)), in_place=True)


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_extreme_temperatures_and_logits(dtype):
    rng = np.random.default_rng(11)
    V = 4001
    v, part = verifier(rng, V, T)
    table = [(t, k, p, m) for t in (1e-30, 1e-4, 1e30, 3e38) for (k, p, m) in ((0, 1.0, 0.0), (9, 1.0, 0.0), (0, 0.7, 0.0), (0, 1.0, 0.5))]
    B = len(table)
    z = np.stack([rng.normal(0, 3, (B, V)), rng.normal(0, 1e38, (B, V)), rng.normal(0, 1e-38, (B, V)),
                  rng.normal(1e5, 300, (B, V))], axis=1)
    z = np.clip(z, -3e38, 3e38)
    check(v, T, part, to_dtype(z, dtype), asks(B, table), numbers(rng, (B, 4)))


@pytest.mark.parametrize("u", [0.0, 2.0 ** -24, 0.5, 1.0 - 2.0 ** -24])
def test_the_ends_of_the_uniform(u):
    rng = np.random.default_rng(12)
    V = 9000
    v, part = verifier(rng, V, D)
    B = len(ASKS)
    z = to_dtype(rng.normal(0, 4, (B, 2, V)), wl.BF16)
    check(v, D, part, z, asks(B), np.full((B, 2), u, np.float32))


@pytest.mark.parametrize("V", [600, 9000, 40000])
def test_uniforms_outside_their_range_still_draw_a_kept_id(V):
    rng = np.random.default_rng(13)
    v, part = verifier(rng, V, T)
    us = np.array([1.0, 2.0, 1e30, INF, -INF, -1.0, np.nan], np.float32)
    B = len(ASKS)
    z = rng.normal(0, 1, (B, us.size, V)).astype(np.float32)
    tau, k, p, mp = asks(B)
    dt, dk, dp, dm = (torch.from_numpy(x).cuda() for x in (tau, k, p, mp))
    _, _, status, kept = ro.rows(z.astype(np.float64), part, tau, k, p, mp, np.zeros((B, us.size), np.float32))
    out = v.sample(torch.from_numpy(z).cuda(), dt, torch.from_numpy(np.tile(us, (B, 1))).cuda(), side=T, top_k=dk, top_p=dp, min_p=dm)
    tokens = out["tokens"].cpu().numpy()
    assert (status == 0).all() and (out["status"].cpu().numpy() == 0).all()
    assert np.take_along_axis(kept, tokens[..., None].astype(np.int64), 2).all()


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
@pytest.mark.parametrize("offset", [0, 1, 3])
def test_strides_alignment_and_padding(offset, dtype):
    rng = np.random.default_rng(13 + offset)
    V, B, R, pitch = 2011, len(ASKS), 3, 2016 + offset
    v, part = verifier(rng, V, T)
    buf = to_dtype(rng.normal(0, 3, (R, B, pitch + 8)), dtype).cuda()
    z = buf[:, :, offset:offset + V].permute(1, 0, 2)        # sequences inside positions, rows off the 16-byte grid
    u = numbers(rng, (B, R))
    check(v, T, part, z, asks(B), u)
    # one row for every sequence
    check(v, T, part, z[:1].expand(B, R, V), asks(B), u)
    # an output of another alignment, whose padding stays as it was
    out = torch.full((B, R, V + 5), 7.0, dtype=z.dtype, device="cuda")
    view = out[:, :, 2:2 + V]
    tau, k, p, mp = (torch.from_numpy(x).cuda() for x in asks(B))
    ref = v.filter(z, tau, top_k=k, top_p=p, min_p=mp)["logits"]
    v.filter(z, tau, top_k=k, top_p=p, min_p=mp, out=view)
    assert torch.equal(view, ref)
    assert (out[:, :, :2] == 7).all() and (out[:, :, 2 + V:] == 7).all()


@pytest.mark.parametrize("dtype,V", [(wl.F32, tli.TLI_MAX_V), (wl.BF16, tli.TLI_MAX_V - 3), (wl.F32, 262145)])
def test_the_widest_rows(dtype, V):
    rng = np.random.default_rng(14)
    m = np.full(11, -1, np.int32)
    v = tli.Verifier(V, 11, m)
    table = [(1.0, 50, 0.9, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 0, 1.0, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 9000, 1.0, 0.0), (1.0, 0, 1.0, 0.01)]
    B = len(table)
    z = rng.normal(0, 3, (B, 1, V)).astype(np.float32)
    check(v, T, np.ones(V, bool), to_dtype(z, dtype), asks(B, table), numbers(rng, (B, 1)))


@pytest.mark.parametrize("name", ["cfg1", "cfg2", "cfg4"])
def test_rows_of_the_workloads(name):
    cfg = wl.config_by_name(name)
    batch = wl.make_batch(cfg, rows=range(4))
    v = tli.Verifier(cfg.V_t, cfg.V_d, batch["id_map"])
    rng = np.random.default_rng(15)
    table = [(0.9, 50, 1.0, 0.0), (0.7, 0, 0.9, 0.0), (1.0, 40, 0.95, 0.0), (1.0, 0, 1.0, 0.05)]
    for side, key, part in ((T, "target_logits", np.ones(cfg.V_t, bool)), (D, "drafter_logits", batch["id_map"] >= 0)):
        z = torch.from_numpy(np.ascontiguousarray(batch[key][:4, :3]))
        z = z.view(torch.bfloat16) if z.dtype == torch.uint16 else z
        check(v, side, part, z, asks(4, table), numbers(rng, (4, 3)))


def test_none_means_off():
    rng = np.random.default_rng(16)
    V, B, R = 3001, 4, 3
    v, part = verifier(rng, V, T)
    z = to_dtype(rng.normal(0, 3, (B, R, V)), wl.F32).cuda()
    tau = torch.ones(B, device="cuda")
    u = torch.from_numpy(numbers(rng, (B, R))).cuda()
    off = dict(top_k=torch.zeros(B, dtype=torch.int32, device="cuda"), top_p=torch.ones(B, device="cuda"), min_p=torch.zeros(B, device="cuda"))
    a, b = v.sample(z, tau, u), v.sample(z, tau, u, **off)
    assert all(torch.equal(a[n], b[n]) for n in a)
    assert torch.equal(v.filter(z, tau)["logits"], z)


def test_captured_replayed_and_overlapping_calls():
    """One context, calls captured into two graphs, replayed and run on two streams at once."""
    rng = np.random.default_rng(17)
    V, B, R = 32000, 16, 2
    v, part = verifier(rng, V, T)
    tau, k, p, mp = (torch.from_numpy(x).cuda() for x in asks(B))
    z = [to_dtype(rng.normal(0, 3, (B, R, V)), wl.BF16).cuda() for _ in range(2)]
    u = [torch.from_numpy(numbers(rng, (B, R))).cuda() for _ in range(2)]
    want = [v.sample(z[i], tau, u[i], top_k=k, top_p=p, min_p=mp)["tokens"] for i in range(2)]
    want_f = [v.filter(z[i], tau, top_k=k, top_p=p, min_p=mp)["logits"] for i in range(2)]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append((v.sample(z[i], tau, u[i], top_k=k, top_p=p, min_p=mp)["tokens"],
                         v.filter(z[i], tau, top_k=k, top_p=p, min_p=mp)["logits"]))
        graphs.append(g)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(3):
        for o in outs:
            o[0].fill_(-5); o[1].fill_(3)
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i][0], want[i]) and torch.equal(outs[i][1], want_f[i])
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(v.sample(z[i], tau, u[i], top_k=k, top_p=p, min_p=mp)["tokens"])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_masks_of_the_lowest_value_beside_a_large_kept_set():
    """Flat rows with most ids masked by the type's lowest value or -inf: the sample that brackets the border sees the masks too."""
    rng = np.random.default_rng(19)
    V = 70001
    v, part = verifier(rng, V, T)
    table = [(1.0, 0, 0.9, 0.0), (1.0, 0, 0.99, 0.0), (1.3, 9000, 1.0, 0.0), (1.0, 3000, 0.9, 0.0), (1.0, 12000, 0.95, 0.0), (1.0, 0, 0.97, 1e-3)]
    for dtype in (wl.F32, wl.BF16):
        lowest = torch.finfo(torch.bfloat16 if dtype == wl.BF16 else torch.float32).min
        z = rng.normal(-9, 1.5, (len(table), 3, V))
        z[:, 1][:, rng.random(V) < 0.6] = lowest
        z[:, 2][:, rng.random(V) < 0.6] = -INF
        check(v, T, part, to_dtype(z, dtype), asks(len(table), table), numbers(rng, (len(table), 3)))


def test_calls_from_several_threads():
    """Threads that share a Verifier and a stream: their kernels may interleave, their scratch may not."""
    import threading
    rng = np.random.default_rng(20)
    V, B, R = 30000, 18, 2
    v, part = verifier(rng, V, T)
    tau, k, p, mp = (torch.from_numpy(x).cuda() for x in asks(B))
    z = [to_dtype(rng.normal(0, 1 + i, (B, R, V)), wl.BF16).cuda() for i in range(4)]
    u = [torch.from_numpy(numbers(rng, (B, R))).cuda() for _ in range(4)]
    want = [v.sample(z[i], tau, u[i], top_k=k, top_p=p, min_p=mp)["tokens"] for i in range(4)]
    torch.cuda.synchronize()
    got = [[] for _ in range(4)]

    def work(i):
        for _ in range(30):
            got[i].append(v.sample(z[i], tau, u[i], top_k=k, top_p=p, min_p=mp)["tokens"])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    for i in range(4):
        assert len(got[i]) == 30 and all(torch.equal(g, want[i]) for g in got[i])


def test_output_rows_between_input_rows():
    """An output that lies in the gaps of the input's rows is fine, one that meets them is refused."""
    rng = np.random.default_rng(21)
    V, B, R = 1000, 3, 2
    v, _ = verifier(rng, V, T)
    buf = torch.from_numpy(rng.normal(0, 2, (B, R, 2, V)).astype(np.float32)).cuda()
    tau, k = torch.ones(B, device="cuda"), torch.full((B,), 7, dtype=torch.int32, device="cuda")
    want = v.filter(buf[:, :, 0].contiguous(), tau, top_k=k)["logits"]
    v.filter(buf[:, :, 0], tau, top_k=k, out=buf[:, :, 1])
    assert torch.equal(buf[:, :, 1], want)
    flat = torch.randn(B * R * V + 8, device="cuda")
    with pytest.raises(tli.TLIError):
        v.filter(flat[:B * R * V].view(B, R, V), tau, top_k=k, out=flat[8:].view(B, R, V))
    with pytest.raises(tli.TLIError):
        v.filter(flat[:R * V].view(1, R, V), tau[:1], top_k=k[:1], out=flat[V:V + R * V].view(1, R, V))


def test_refusals():
    rng = np.random.default_rng(18)
    V = 100
    v, _ = verifier(rng, V, T)
    z = torch.randn(2, 3, V, device="cuda")
    tau, u = torch.ones(2, device="cuda"), torch.rand(2, 3, device="cuda")
    tok = torch.empty(2, 3, dtype=torch.int32, device="cuda")
    ws = torch.empty(tli.tli_sample_workspace_bytes(v.ctx, 2, 3, tli.TLI_F32, T), dtype=torch.uint8, device="cuda")
    lib = tli.load()

    def sample(**change):
        a = tli.make_sample_args(v.ctx, z, tau, u, tok, ws)
        for n, x in change.items():
            setattr(a, n, x)
        return lib.tli_sample(v.ctx, ctypes.byref(a), None)

    def filt(**change):
        a = tli.make_filter_args(v.ctx, z, tau, z, ws)
        for n, x in change.items():
            setattr(a, n, x)
        return lib.tli_filter(v.ctx, ctypes.byref(a), None)

    assert sample() == tli.TLI_OK and filt() == tli.TLI_OK
    for call in (sample, filt):
        for bad in (dict(B=0), dict(R=0), dict(dtype=2), dict(side=2), dict(side=-1), dict(logits=None), dict(temperature=None),
                    dict(logits=z.data_ptr() + 2), dict(stride_b=-1), dict(stride_r=-5)):
            assert call(**bad) == tli.TLI_ERR_ARG, bad
        assert call(B=65536) == tli.TLI_ERR_UNSUPPORTED
        for bad in (dict(workspace=None), dict(workspace=ws.data_ptr() + 16), dict(workspace_bytes=ws.numel() - 1)):
            assert call(**bad) == tli.TLI_ERR_WORKSPACE, bad
    for bad in (dict(uniforms=u.data_ptr() + 2), dict(tokens=tok.data_ptr() + 1), dict(top_k=tok.data_ptr() + 2)):
        assert sample(**bad) == tli.TLI_ERR_ARG, bad
    assert sample(uniforms=None) == tli.TLI_ERR_ARG and sample(tokens=None) == tli.TLI_ERR_ARG
    for bad in (dict(out=None), dict(out=z.data_ptr() + 1), dict(out_stride_r=V - 1), dict(out_stride_b=3 * V - 1), dict(out_stride_b=-1)):
        assert filt(**bad) == tli.TLI_ERR_ARG, bad
    assert lib.tli_sample(v.ctx, None, None) == tli.TLI_ERR_ARG
    shard = tli.tli_shard_create(0, v.V_t, v.V_d, np.full(v.V_d, -1, np.int32), 2, 0)
    a = tli.make_sample_args(v.ctx, z, tau, u, tok, ws)
    assert lib.tli_sample(shard, ctypes.byref(a), None) == tli.TLI_ERR_ARG
    assert tli.tli_sample_workspace_bytes(shard, 2, 3, 0, T) == 0
    tli.tli_destroy(shard)
    with pytest.raises(ValueError):
        v.sample(z[:, :, :50], tau, u)
    with pytest.raises(ValueError):
        v.sample(z, tau, u[:, :2])
    with pytest.raises(ValueError):
        v.sample(z, tau, u, top_k=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        v.filter(z.transpose(1, 2), tau)
    with pytest.raises(ValueError):
        v.filter(z, tau, out=z.bfloat16())
    with pytest.raises(TypeError):
        v.sample(z.half(), tau, u)
