"""tli_loss() and tli_loss_grad() against fp64.

Roundings.  s = log2(e)/tau is off by 2^-23 relative (constant and quotient), so an exponent a = (z - m) s of a weight by |a| 2^-23,
its difference and its product by |a| 2^-24 each: |a| 2^-22 ln 2 = 1.4 |a| 2^-23 of the weight; ex2 adds 2^-22.  So the sum is off by
1.4 E 2^-23 relative, E the mean of |a| under q, and by what follows.  The sum itself: at most
D = V/1024 + 64 additions in a row (2^-24 each) and one ex2 for every new maximum of a thread, warp, CTA and cluster (at most B = V/8192 + 24).
    eps_sum  = 1.4 E 2^-23 + (B + 2) 2^-22 + D 2^-24
    loss     : eps_sum + 2^-22 |ln sum| + (|terms| + 1) 2^-20      (quotients, products and sums of the targets' terms: under eight
                                                                   roundings of 2^-24 each, their ex2 2^-22 and W's as much, ln W 2^-22)
    gradient : |h| (q (1.4 |a| 2^-23 + eps_sum + 2^-21) + p (2^-20 + eps_p)) and the rounding to its type, half a step.
A target's probability has an exponent of its own, b = (t - max t) s: the difference and the product round by 2^-24 each and s by 2^-23,
2^-22 ln 2 |b| in all, with |b| ln 2 = |t - max t|/tau =: far.  So a weight is off by far 2^-22 and W by the mean of far under p:
eps_p p = (p far + p mean far) 2^-22; the loss's terms, which the weights multiply, by at most (sum p far) (1 + largest term / 2) 2^-21 more
(each |x_j| p_j far_j is counted with the largest x)."""
import ctypes

import numpy as np
import pytest
import torch

import loss_oracle as lo
import row_oracle as ro
from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
STEP = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126}       # (ex2 flushes what is subnormal)


def make_map(rng, V_t, V_d, f=0.6):
    m = np.full(V_d, -1, np.int32)
    on = rng.permutation(V_d)[:max(1, min(V_t, int(f * V_d)))]
    m[on] = rng.permutation(V_t)[:on.size]
    return m


def sum_error(z, part, stats, q, tau):
    V = z.shape[1]
    a = np.where(q > 0, np.abs(np.where(np.isfinite(z), z, 0) - stats[:, :1]) / tau[:, None], 0) * 1.4427
    E = (q * a).sum(1)
    return a, 1.4 * E * 2.0 ** -23 + (V / 8192 + 26) * 2.0 ** -22 + (V / 1024 + 64) * 2.0 ** -24


def check(v, m, z, ids, teacher=None, tau=None, g=None, side=T, ids_side=T, shared=False, out=None, grad=True):
    """z, teacher: device tensors; ids int32 numpy [N] or [N,k]; tau, g: float32 numpy [N] or None."""
    N, V = z.shape
    dev = lambda x: None if x is None else torch.from_numpy(x).cuda()
    d_ids, d_tau, d_g = dev(ids), dev(tau), dev(g)
    how = dict(teacher=teacher, temperature=d_tau, side=side, ids_side=ids_side, shared=shared)
    got = v.loss(z, d_ids, **how)
    z64 = z.double().cpu().numpy()
    t = ro.table_ids(ids.reshape(N, -1), np.zeros(0, np.int32) if m is None else m, v.V_t, ids_side, side)
    part = (m >= 0) if shared else np.ones(V, bool)
    tau = np.ones(N, np.float32) if tau is None else tau
    t64 = None if teacher is None else teacher.double().cpu().numpy()
    loss, stats, status, q, p, terms, far = lo.rows(z64, part, t, t64, tau)
    np.testing.assert_array_equal(got["status"].cpu().numpy(), status)
    l, st = got["loss"].double().cpu().numpy(), got["stats"].double().cpu().numpy()
    fine = (status & lo.NONFINITE) == 0
    assert np.isnan(l[~fine]).all() and (st[status & (8 | 32 | 128) != 0] == 0).all()
    np.testing.assert_array_equal(st[fine, 0], stats[fine, 0])
    with np.errstate(invalid="ignore", divide="ignore"):
        a, eps = sum_error(z64, part, stats, q, np.where(tau > 0, tau, 1).astype(np.float64))
        assert (np.abs(st - stats)[fine, 1] <= (eps * stats[:, 1])[fine]).all()
        bound = eps + 2.0 ** -22 * np.abs(np.log(np.maximum(stats[:, 1], 1))) + (terms + 1) * 2.0 ** -20
        inf = np.isinf(loss)
        bound = bound + far.sum(1) * 2.0 ** -21 * (1 + np.where(p > 0, a * 0.7 + far / np.where(p > 0, p, 1), 0).max(1) / 2)
        assert (l[inf] == loss[inf]).all()
        ok = fine & ~inf
        assert (np.abs(l - loss)[ok] <= bound[ok]).all(), (np.abs(l - loss) - bound)[ok].max()
    if not grad:
        return got, None
    kept = z.clone()
    gr = v.loss_grad(z, d_ids, got["stats"], grad_loss=d_g, out=out, **how)["grad"]
    x = gr.double().cpu().numpy()
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        h = ((np.ones(N) if g is None else g.astype(np.float64)) / tau)[:, None]
        exact = h * (q - p)
        err = np.abs(h) * (q * (1.4 * a * 2.0 ** -23 + eps[:, None] + 2.0 ** -21) + p * 2.0 ** -20 + (far + p * far.sum(1)[:, None]) * 2.0 ** -22)
        err = err + HALF[z.dtype] * (np.abs(exact) + err) + STEP[z.dtype]
        zero = (status & (8 | 32 | 128)) != 0
        assert (x[zero] == 0).all() and np.isnan(x[~fine]).all()
        ok = fine & ~zero
        assert (np.abs(x - exact)[ok] <= err[ok]).all(), (np.abs(x - exact) - err)[ok].max()
    assert out is not None or torch.equal(z.view(torch.int16 if z.dtype == torch.bfloat16 else torch.int32),
                                          kept.view(torch.int16 if z.dtype == torch.bfloat16 else torch.int32))
    return got, gr


def inputs(rng, N, V, k, V_ids, dtype):
    z = torch.from_numpy(rng.normal(0, 3, (N, V)).astype(np.float32)).to(dtype).cuda()
    if k == 0:
        return z, rng.integers(0, V_ids, N).astype(np.int32), None
    return z, rng.integers(0, V_ids, (N, k)).astype(np.int32), torch.from_numpy(rng.normal(0, 2, (N, k)).astype(np.float32)).cuda()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("side,ids_side,shared", [(T, T, False), (T, D, False), (D, T, False), (D, D, False), (D, T, True), (D, D, True)])
@pytest.mark.parametrize("N,V_t,V_d,k", [(1, 1, 1, 0), (1, 7, 5, 3), (5, 129, 257, 0), (33, 1501, 1203, 1), (3, 32003, 50257, 20), (700, 300, 517, 256)])
def test_loss_and_gradient(N, V_t, V_d, k, side, ids_side, shared, dtype):
    rng = np.random.default_rng(N + V_t + k)
    m = make_map(rng, V_t, V_d)
    v = tli.Verifier(V_t, V_d, m)
    z, ids, teacher = inputs(rng, N, V_t if side == T else V_d, k, V_t if ids_side == T else V_d, dtype)
    ids.flat[rng.integers(0, ids.size, ids.size // 10)] = rng.choice(np.array([-1, -9, 2 ** 31 - 1, -2 ** 31, max(V_t, V_d)], np.int64)).astype(np.int32)
    tau = rng.choice(np.array([0.3, 1.0, 2.5], np.float32), N).astype(np.float32)
    g = rng.normal(0, 1, N).astype(np.float32)
    check(v, m, z, ids, teacher, tau, g, side, ids_side, shared)
    check(v, m, z, ids, None if teacher is None else teacher.bfloat16(), None, None, side, ids_side, shared)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(1, 256000), (2, 1048576), (40, 65536), (148, 33333), (1300, 4099)])
def test_rows_over_one_and_several_blocks(N, V, dtype):
    rng = np.random.default_rng(V)
    v = tli.Verifier(V, 3, np.array([0, -1, V - 1], np.int32))
    z, ids, teacher = inputs(rng, N, V, 5, V, dtype)
    ids[0, :3] = 0, V - 1, V // 2
    check(v, np.array([0, -1, V - 1], np.int32), z, ids, teacher)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_infinities_and_nan(dtype):
    rng = np.random.default_rng(3)
    V_t, V_d = 700, 900
    m = make_map(rng, V_t, V_d)
    inside, outside = np.flatnonzero(m >= 0), np.flatnonzero(m < 0)
    v = tli.Verifier(V_t, V_d, m)
    low = torch.finfo(dtype).min
    z, ids, teacher = inputs(rng, 14, V_d, 4, V_d, dtype)
    ids[:] = rng.choice(inside, ids.shape)
    z[0] = -float("inf")                                                     # nothing left
    z[1] = low
    z[2, inside] = -float("inf")
    z[3, outside] = float("nan")                                             # outside the intersection
    z[4, outside] = float("inf")
    z[5, inside[7]] = float("nan")
    z[6, inside[8]] = float("inf")
    z[7, :] = -float("inf"); z[7, inside[3]] = -1e4                          # one left
    ids[7] = inside[3]
    z[8, ids[8, 0]] = -float("inf")                                          # a target that cannot be
    z[9] = low; z[9, ids[9]] = 5.0
    ids[10] = outside[:4]; z[10] = float("nan")                              # left out, whatever it holds
    teacher[11] = -float("inf"); z[11] = float("inf")
    teacher[12, 1] = float("nan")
    teacher[13, :3] = torch.tensor([low, -float("inf"), 3.0])
    for shared in (True, False):
        check(v, m, z, ids, teacher, side=D, ids_side=D, shared=shared, grad=True)
    labels = ids[:, 0].copy()
    check(v, m, z, labels, side=D, ids_side=D, shared=True)


def test_wide_gaps_and_large_logits():
    rng = np.random.default_rng(4)
    V = 5000
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    z, ids, _ = inputs(rng, 8, V, 0, V, torch.float32)
    z *= torch.tensor([1e-30, 1e-3, 1, 10, 1e3, 1e6, 1e10, 1e20], device="cuda")[:, None]
    z[2] += 1e6
    for n in range(4, 8):
        ids[n] = int(z[n].argmax())
    check(v, None, z, ids)


def test_temperatures():
    rng = np.random.default_rng(5)
    v = tli.Verifier(600, 3, np.array([0, -1, 2], np.int32))
    tau = np.array([0.0, -1.0, np.nan, np.inf, -np.inf, 1e-45, 1e-3, 1e3, 1e38, 3e38, 1e-20], np.float32)
    z, ids, teacher = inputs(rng, tau.size, 600, 6, 600, torch.float32)
    z[10] = z[10].round()
    check(v, None, z, ids, teacher, tau=tau)
    ids[0] = -1
    check(v, None, z, ids, teacher, tau=tau)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_same_id_twice(dtype):
    rng = np.random.default_rng(6)
    v = tli.Verifier(300, 3, np.array([0, -1, 2], np.int32))
    z, ids, teacher = inputs(rng, 5, 300, 9, 300, dtype)
    ids[0] = 17
    ids[1, ::2] = 299
    ids[2, 1:3] = ids[2, 0]
    check(v, None, z, ids, teacher)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_alignment_and_in_place(dtype):
    rng = np.random.default_rng(7)
    V = 1001
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    for offset, pitch, out_offset, out_pitch in ((0, 1001, 0, 1001), (1, 1016, 1, 1016), (3, 1003, 0, 1001), (8, 1024, 8, 2048), (5, 1009, 2, 1010)):
        big = torch.from_numpy(rng.normal(0, 3, (20, pitch + 8)).astype(np.float32)).to(dtype).cuda()
        z = big.view(-1)[offset:offset + 20 * pitch].view(20, pitch)[:, :V]
        ids, g = rng.integers(0, V, 20).astype(np.int32), rng.normal(0, 1, 20).astype(np.float32)
        buf = torch.full((20 * out_pitch + 16,), 5.0, dtype=dtype, device="cuda")
        out = buf[out_offset:out_offset + 20 * out_pitch].view(20, out_pitch)[:, :V]
        _, gr = check(v, None, z, ids, g=g, out=out)
        want = gr.clone()
        rest = buf.clone()
        rest[out_offset:out_offset + 20 * out_pitch].view(20, out_pitch)[:, :V] = 5.0
        assert (rest == 5).all()
        before = big.clone()
        d_ids, stats = torch.from_numpy(ids).cuda(), v.loss(z, torch.from_numpy(ids).cuda())["stats"]
        v.loss_grad(z, d_ids, stats, grad_loss=torch.from_numpy(g).cuda(), out=z)
        assert torch.equal(z, want)
        z.copy_(before.view(-1)[offset:offset + 20 * pitch].view(20, pitch)[:, :V])
        assert torch.equal(big, before)
    one = torch.from_numpy(rng.normal(0, 3, (1, V)).astype(np.float32)).to(dtype).cuda().expand(6, V)
    check(v, None, one, rng.integers(0, V, 6).astype(np.int32))


def test_offsets_beyond_32_bits():
    V = 40000
    big = torch.empty(2 ** 31 + 2 ** 30 + 2 * V + 64, dtype=torch.bfloat16, device="cuda")
    z = big.as_strided((3, V), (2 ** 30 + 2 ** 29, 1), 3)                    # the last row begins 6 GB into the buffer
    z.copy_(torch.randn(3, V, device="cuda"))
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    ids = np.array([5, V - 1, 0], np.int32)
    check(v, None, z, ids)
    keep = z[:2].clone()
    out = big.as_strided((2, V), (2 ** 30 + 2 ** 29, 1), V + 40)
    check(v, None, z[:2], ids[:2], out=out)
    assert torch.equal(z[:2], keep)


def test_gradient_agrees_with_differences():
    """The library's gradient against central differences of the definition in fp64, step 1e-5: truncation below 1e-9, rounding 1e-10."""
    rng = np.random.default_rng(8)
    V_t, V_d = 60, 50
    m = make_map(rng, V_t, V_d)
    v = tli.Verifier(V_t, V_d, m)
    z, ids, teacher = inputs(rng, 3, V_d, 4, V_t, torch.float32)
    ids[:, 0] = m[m >= 0][:3]
    tau = np.array([0.7, 1.0, 3.0], np.float32)
    d = dict(teacher=teacher, temperature=torch.from_numpy(tau).cuda(), side=D, ids_side=T, shared=True)
    st = v.loss(z, torch.from_numpy(ids).cuda(), **d)["stats"]
    got = v.loss_grad(z, torch.from_numpy(ids).cuda(), st, **d)["grad"].double().cpu().numpy()
    z64, t = z.double().cpu().numpy(), ro.table_ids(ids, m, V_t, T, D)
    f = lambda x: lo.rows(x, m >= 0, t, teacher.double().cpu().numpy(), tau)[0]
    for x in range(V_d):
        e = np.zeros_like(z64)
        e[:, x] = 1e-5
        assert (np.abs((f(z64 + e) - f(z64 - e)) / 2e-5 - got[:, x]) <= 1e-6).all()


def test_nothing_and_one_element():
    v = tli.Verifier(1, 1, np.array([0], np.int32))
    empty = v.loss(torch.empty(0, 1, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert empty["loss"].shape == (0,) and empty["stats"].shape == (0, 2)
    assert v.loss_grad(torch.empty(0, 1, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), empty["stats"])["grad"].shape == (0, 1)
    check(v, None, torch.full((2, 1), 3.0, device="cuda"), np.array([0, 1], np.int32))


def test_captured_replayed_and_on_two_streams():
    rng = np.random.default_rng(9)
    V = 20000
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    z, ids, teacher = inputs(rng, 30, V, 8, V, torch.bfloat16)
    ids = torch.from_numpy(ids).cuda()
    both = lambda: (lambda f: (f["loss"], f["stats"], v.loss_grad(z, ids, f["stats"], teacher=teacher)["grad"]))(v.loss(z, ids, teacher=teacher))
    want = both()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = both()
    for _ in range(3):
        for x in got:
            x.fill_(9)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams * 4:
        with torch.cuda.stream(s):
            outs.append(both())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))


def test_refusals():
    V = 64
    v = tli.Verifier(V, 40, np.concatenate((np.arange(30), np.full(10, -1))).astype(np.int32))
    z, ids = torch.zeros(4, V, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    teach, ids2 = torch.zeros(4, 2, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    loss, stats, out = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.zeros(4, V, device="cuda")
    lib = tli.load()
    base = dict(N=4, k=1, dtype=0, side=0, ids_side=0, support=0, teacher_dtype=0, logits=z.data_ptr(), stride=V, ids=ids.data_ptr(), stats=stats.data_ptr())

    def call(name, cls, extra, change):
        a = cls()
        for n, x in {**base, **extra, **change}.items():
            setattr(a, n, x)
        return getattr(lib, name)(v.ctx, ctypes.byref(a), None)

    forward = lambda **c: call("tli_loss", tli.tli_loss_args, dict(loss=loss.data_ptr()), c)
    back = lambda **c: call("tli_loss_grad", tli.tli_loss_grad_args, dict(grad=out.data_ptr(), grad_stride=V), c)
    for f in (forward, back):
        assert f() == tli.TLI_OK and f(N=0) == tli.TLI_OK
        assert f(k=2, teacher=teach.data_ptr(), ids=ids2.data_ptr()) == tli.TLI_OK
        for bad in (dict(N=-1), dict(k=0), dict(k=2), dict(dtype=2), dict(side=2), dict(ids_side=-1), dict(support=2), dict(support=1),
                    dict(teacher=teach.data_ptr(), teacher_dtype=2), dict(teacher=teach.data_ptr() + 2), dict(logits=None), dict(logits=z.data_ptr() + 2),
                    dict(stride=-V), dict(ids=None), dict(ids=ids.data_ptr() + 1), dict(temperature=loss.data_ptr() + 2), dict(stats=None), dict(stats=stats.data_ptr() + 4)):
            assert f(**bad) == tli.TLI_ERR_ARG, bad
        assert f(N=tli.TLI_MAX_TOKENS + 1) == tli.TLI_ERR_UNSUPPORTED
        assert f(k=tli.TLI_MAX_TARGETS + 1, teacher=teach.data_ptr()) == tli.TLI_ERR_UNSUPPORTED
    for bad in (dict(loss=None), dict(loss=loss.data_ptr() + 1), dict(status=loss.data_ptr() + 2)):
        assert forward(**bad) == tli.TLI_ERR_ARG, bad
    for bad in (dict(grad=None), dict(grad=out.data_ptr() + 2), dict(grad_stride=V - 1), dict(grad=z.data_ptr() + 16), dict(grad=z.data_ptr(), grad_stride=V + 1),
                dict(stride=0, grad=z.data_ptr()), dict(grad_loss=loss.data_ptr() + 2)):
        assert back(**bad) == tli.TLI_ERR_ARG, bad
    for call_ in (lambda: v.loss(z[:, :-1], ids), lambda: v.loss(z, ids.long()), lambda: v.loss(z, ids2), lambda: v.loss(z, ids2, teacher=teach[:3]),
                  lambda: v.loss(z, ids, temperature=torch.ones(3, device="cuda")), lambda: v.loss(z, ids, side=2), lambda: v.loss(z.t().contiguous().t(), ids),
                  lambda: v.loss(z.cpu(), ids), lambda: v.loss_grad(z, ids, stats[:3]), lambda: v.loss_grad(z, ids, stats, out=out[:3])):
        with pytest.raises(ValueError):
            call_()
    with pytest.raises(TypeError):
        v.loss(z.half(), ids)
    with pytest.raises(tli.TLIError):
        v.loss(z, ids, shared=True)
