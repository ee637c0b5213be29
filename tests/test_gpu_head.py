"""tli_head_loss() and tli_head_loss_grad() against fp64.

A logit is a sum of H exact products of bf16 values in fp32.  The matrix unit adds 16 of them at a time and may cut what does not fit
(2^-23 of the sum of sizes A = sum |h w| per step, every step); joining parts rounds by 2^-24 each:
    dz = (H / 16 + 8) 2^-23 A
The loss on top of that: stats' m is off by dz of the largest, the sum relative to it by the mean of 2 dz / tau under q and by what
tests/test_gpu_loss.py derives for rows of logits; the targets' logits are sums in fp32 in some order (H 2^-24 A at most).
    gradients: G = g (q - p) / tau is rounded to bf16 (2^-8 of itself) and q is off by q (2 dz / tau + eps); a product's sums over n terms
    lose n / 16 + 8 times 2^-23 of sum |G w|, and the result is rounded to bf16."""
import ctypes

import numpy as np
import pytest
import torch

import loss_oracle as lo
import row_oracle as ro
from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
HALF = 2.0 ** -8


def make_map(rng, V_t, V_d, f=0.6):
    m = np.full(V_d, -1, np.int32)
    on = rng.permutation(V_d)[:max(1, min(V_t, int(f * V_d)))]
    m[on] = rng.permutation(V_t)[:on.size]
    return m


def check(v, m, h, w, ids, teacher=None, tau=None, g=None, side=T, ids_side=T, shared=False, h_out=None, w_out=None):
    """h, w, teacher: device tensors; ids int32 numpy [N] or [N,k]; tau, g: float32 numpy [N] or None."""
    N, H = h.shape
    V = w.shape[0]
    dev = lambda x: None if x is None else torch.from_numpy(x).cuda()
    d_ids, d_tau, d_g = dev(ids), dev(tau), dev(g)
    how = dict(teacher=teacher, temperature=d_tau, side=side, ids_side=ids_side, shared=shared)
    got = v.head_loss(h, w, d_ids, **how)
    again = v.head_loss(h, w, d_ids, **how)
    assert all(torch.equal(torch.nan_to_num(got[k], nan=7.0), torch.nan_to_num(again[k], nan=7.0)) for k in got)
    h64, w64 = h.double().cpu().numpy(), w.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        z, A = h64 @ w64.T, np.abs(h64) @ np.abs(w64).T
    t = ro.table_ids(ids.reshape(N, -1), np.zeros(0, np.int32) if m is None else m, v.V_t, ids_side, side)
    part = (m >= 0) if shared else np.ones(V, bool)
    tau = np.ones(N, np.float32) if tau is None else tau
    t64 = None if teacher is None else teacher.double().cpu().numpy()
    loss, stats, status, q, p, terms, far = lo.rows(z, part, t, t64, tau)
    np.testing.assert_array_equal(got["status"].cpu().numpy(), status)
    fine, zero = (status & lo.NONFINITE) == 0, (status & (8 | 32 | 128)) != 0
    ok = fine & ~zero
    l, st, at = (got[k].double().cpu().numpy() for k in ("loss", "stats", "target_logits"))
    assert np.isnan(l[~fine]).all() and (l[zero] == 0).all() and (st[zero] == 0).all()
    on = (t >= 0) & part[np.maximum(t, 0)] & ok[:, None]
    if t64 is not None:
        on &= ~(t64 < lo.MASK)
    assert (at.reshape(N, -1)[~on & ok[:, None]] == 0).all()
    rows = np.repeat(np.arange(N)[:, None], t.shape[1], 1)[on]
    assert (np.abs(at.reshape(N, -1)[on] - z[rows, t[on]]) <= (H + 8) * 2.0 ** -24 * A[rows, t[on]]).all()
    T64 = np.where(tau > 0, tau, 1).astype(np.float64)[:, None]
    with np.errstate(invalid="ignore"):
        dz = (H / 16 + 8) * 2.0 ** -23 * np.where(part, A, 0)
        a = np.where(q > 0, (stats[:, :1] - z) / T64, 0)
        high = (dz * part).max(1)
        eps = (q * (1.4 * 1.45 * a * 2.0 ** -23 + 2 * dz / T64)).sum(1) + high / T64[:, 0] + (V / 8192 + 60) * 2.0 ** -22 + (V / 1024 + 64) * 2.0 ** -24
        assert (np.abs(st - stats)[ok, 0] <= high[ok]).all()
        assert (np.abs(st - stats)[ok, 1] <= (eps * stats[:, 1])[ok]).all()
        bound = eps + 2.0 ** -22 * np.abs(np.log(np.maximum(stats[:, 1], 1))) + (terms + 1) * 2.0 ** -20 + 2 * high / T64[:, 0]
        bound = bound + far.sum(1) * 2.0 ** -21 * (1 + np.where(p > 0, a + far / np.where(p > 0, p, 1), 0).max(1) / 2)
        assert (np.abs(l - loss)[ok] <= bound[ok]).all(), (np.abs(l - loss) - bound)[ok].max()
    dh, dw = None if h_out is None else h_out, None if w_out is None else w_out
    if h_out is None and w_out is None:
        b = v.head_loss_grad(h, w, d_ids, got["stats"], got["target_logits"], grad_loss=d_g, **how)
        c = v.head_loss_grad(h, w, d_ids, got["stats"], got["target_logits"], grad_loss=d_g, **how)
        one = v.head_loss_grad(h, w, d_ids, got["stats"], got["target_logits"], grad_loss=d_g, weight_grad=False, **how)
        two = v.head_loss_grad(h, w, d_ids, got["stats"], got["target_logits"], grad_loss=d_g, hidden_grad=False, **how)
        dh, dw = b["grad_hidden"], b["grad_weight"]
        assert one["grad_weight"] is None and two["grad_hidden"] is None
        same = lambda x, y: torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))
        assert same(dh, c["grad_hidden"]) and same(dw, c["grad_weight"]) and same(dh, one["grad_hidden"]) and same(dw, two["grad_weight"])
        np.testing.assert_array_equal(b["status"].cpu().numpy() & (32 | 128), status & (32 | 128))
    else:
        ws = torch.empty(tli.tli_head_loss_grad_workspace_bytes(v.ctx, N, H, t.shape[1], side), dtype=torch.uint8, device="cuda")
        args = tli.tli_head_loss_grad_args(N, H, t.shape[1], side, ids_side, 1 if shared else 0, 0, h.data_ptr(), h.stride(0), w.data_ptr(), w.stride(0),
                                           d_ids.data_ptr(), None, None, got["stats"].data_ptr(), got["target_logits"].data_ptr(), None,
                                           dh.data_ptr(), dh.stride(0), dw.data_ptr(), dw.stride(0), None, ws.data_ptr(), ws.numel())
        assert tli.load().tli_head_loss_grad(v.ctx, ctypes.byref(args), torch.cuda.current_stream().cuda_stream) == tli.TLI_OK
    x, y = dh.double().cpu().numpy(), dw.double().cpu().numpy()
    assert (x[zero] == 0).all()
    if not fine.all():
        assert np.isnan(x[~fine]).all() and np.isnan(y[part]).all()
        return got
    s = ((np.ones(N) if g is None else g.astype(np.float64)) / T64[:, 0] * ok)[:, None]
    G = s * (q - p)
    err = np.abs(s) * (q * (2.1 * a * 2.0 ** -23 + 2 * dz / T64 + high[:, None] / T64 + eps[:, None] + 2.0 ** -21) + p * 2.0 ** -20 + (far + p * far.sum(1)[:, None]) * 2.0 ** -22)
    err = err + HALF * (np.abs(G) + err) + 2.0 ** -126
    hh, live = np.where(ok[:, None], h64, 0), int(ok.sum())
    G, err = np.where(ok[:, None], G, 0), np.where(ok[:, None], err, 0)
    for got_, exact, e, size, n in ((x, G @ w64, err @ np.abs(w64), np.abs(G) @ np.abs(w64), V), (y, G.T @ hh, err.T @ np.abs(hh), np.abs(G).T @ np.abs(hh), live)):
        e = e + (n / 16 + 8) * 2.0 ** -23 * size
        e = e + HALF * (np.abs(exact) + e) + 2.0 ** -126
        assert (np.abs(got_ - exact) <= e).all(), (np.abs(got_ - exact) - e).max()
        # two roundings to bf16, each at most 2^-8 and on average (over mantissas) 2^-8 / sqrt(3) or less
        if exact.size > 2000 and np.linalg.norm(exact) > 0:
            assert np.linalg.norm(got_ - exact) <= 2.0 ** -8 * np.linalg.norm(exact)
    return got


def inputs(rng, N, H, V, k, V_ids, scale=2.0):
    bf = lambda x: torch.from_numpy(x.astype(np.float32)).bfloat16().cuda()
    h, w = bf(rng.normal(0, 1, (N, H))), bf(rng.normal(0, scale / H ** 0.5, (V, H)))
    if k == 0:
        return h, w, rng.integers(0, V_ids, N).astype(np.int32), None
    return h, w, rng.integers(0, V_ids, (N, k)).astype(np.int32), torch.from_numpy(rng.normal(0, 2, (N, k)).astype(np.float32)).cuda()


SIDES = [(T, T, False), (T, D, False), (D, T, False), (D, D, False), (D, T, True), (D, D, True)]


@pytest.mark.parametrize("side,ids_side,shared", SIDES)
@pytest.mark.parametrize("N,H,V_t,V_d,k", [(1, 8, 1, 1, 0), (1, 64, 7, 5, 3), (2, 72, 129, 257, 0), (33, 200, 501, 403, 1), (130, 136, 1003, 1257, 20), (300, 264, 300, 517, 256)])
def test_loss_and_gradients(N, H, V_t, V_d, k, side, ids_side, shared):
    rng = np.random.default_rng(N + H + k)
    m = make_map(rng, V_t, V_d)
    v = tli.Verifier(V_t, V_d, m)
    h, w, ids, teacher = inputs(rng, N, H, V_t if side == T else V_d, k, V_t if ids_side == T else V_d)
    ids.flat[rng.integers(0, ids.size, ids.size // 8)] = rng.choice(np.array([-1, -9, 2 ** 31 - 1, -2 ** 31, max(V_t, V_d)], np.int64)).astype(np.int32)
    tau = rng.choice(np.array([0.3, 1.0, 2.5], np.float32), N).astype(np.float32)
    g = rng.normal(0, 1, N).astype(np.float32)
    check(v, m, h, w, ids, teacher, tau, g, side, ids_side, shared)
    check(v, m, h, w, ids, None if teacher is None else teacher.bfloat16(), None, None, side, ids_side, shared)


@pytest.mark.parametrize("N", [1, 7, 8, 9, 31, 32, 33, 63, 64, 65, 97, 127, 128, 129, 255, 256, 257, 385, 600])
def test_every_fill_of_a_row_block(N):
    rng = np.random.default_rng(N)
    v = tli.Verifier(700, 3, np.array([0, -1, 2], np.int32))
    h, w, ids, _ = inputs(rng, N, 128, 700, 0, 700)
    check(v, None, h, w, ids)


@pytest.mark.parametrize("V", [1, 31, 33, 63, 64, 65, 255, 256, 257, 511, 513, 40000])
@pytest.mark.parametrize("H", [8, 56, 64, 72, 248, 256, 264, 520, 1032])
def test_every_fill_of_a_tile(V, H):
    rng = np.random.default_rng(V + H)
    v = tli.Verifier(V, 1, np.array([0], np.int32))
    for N in (5, 150):
        h, w, ids, _ = inputs(rng, N, H, V, 0, V)
        check(v, None, h, w, ids)


def test_long_contractions():
    rng = np.random.default_rng(1)
    v = tli.Verifier(300, 1, np.array([0], np.int32))
    for N, H in ((3, 4096), (140, 8200)):
        h, w, ids, _ = inputs(rng, N, H, 300, 0, 300)
        check(v, None, h, w, ids)


def test_runs_of_the_vocabulary():
    """More rows than one run of G holds for the whole vocabulary; the last run is a short one."""
    rng = np.random.default_rng(2)
    V, N, k = 20000, 20000, 2
    m = make_map(rng, 6100, V, 0.3)
    v = tli.Verifier(6100, V, m)
    h, w, ids, teacher = inputs(rng, N, 64, V, k, V)
    d = dict(teacher=teacher, side=D, ids_side=D)
    d_ids = torch.from_numpy(ids).cuda()
    f = v.head_loss(h, w, d_ids, **d)
    b = v.head_loss_grad(h, w, d_ids, f["stats"], f["target_logits"], **d)
    z = h.double() @ w.double().T
    p = torch.softmax(teacher.double(), 1)
    G = torch.softmax(z, 1).scatter_add_(1, d_ids.long(), -p)
    lse = torch.logsumexp(z, 1)
    loss = (p * (p.log() - z.gather(1, d_ids.long()) + lse[:, None])).sum(1)
    assert (f["loss"].double() - loss).abs().max() <= 1e-5 * loss.abs().max()
    for got, exact in ((b["grad_hidden"], G @ w.double()), (b["grad_weight"], G.T @ h.double())):
        assert (got.double() - exact).norm() <= 2.0 ** -8 * exact.norm()


def test_rows_left_out_hold_anything():
    rng = np.random.default_rng(3)
    V_t, V_d = 400, 500
    m = make_map(rng, V_t, V_d, 0.3)
    v = tli.Verifier(V_t, V_d, m)
    for N in (70, 300):
        h, w, ids, _ = inputs(rng, N, 72, V_d, 0, V_t)
        gone = ro.table_ids(ids, m, V_t, T, D) < 0
        assert 10 < gone.sum() < N - 10
        h[torch.from_numpy(gone).cuda()] = float("nan")
        check(v, m, h, w, ids, side=D, ids_side=T)
        check(v, m, h, w, np.full(N, -1, np.int32), side=D, ids_side=T)       # all of them


def test_infinities_and_nan():
    rng = np.random.default_rng(4)
    V = 300
    m = make_map(rng, V, V)
    v = tli.Verifier(V, V, m)
    for N in (5, 200):
        h, w, ids, _ = inputs(rng, N, 64, V, 0, V)
        ids[:] = rng.choice(np.flatnonzero(m >= 0), N)
        h[3] = float("nan")
        check(v, m, h, w, ids, side=D, ids_side=D, shared=True)
        h[3, 1:] = 0
        h[3, 0] = float("inf")                                               # inf and -inf and NaN among the logits
        check(v, m, h, w, ids, side=D, ids_side=D)


def test_temperatures_and_the_same_id_twice():
    rng = np.random.default_rng(5)
    v = tli.Verifier(600, 3, np.array([0, -1, 2], np.int32))
    tau = np.array([0.0, -1.0, np.nan, np.inf, 1e-45, 0.05, 1e3, 1e30, 1.0, 1.0], np.float32)
    h, w, ids, teacher = inputs(rng, tau.size, 64, 600, 6, 600)
    ids[8] = 17
    ids[9, ::2] = 599
    check(v, None, h, w, ids, teacher, tau=tau)


def test_strides_and_alignment():
    rng = np.random.default_rng(6)
    V, H = 401, 72
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    for N in (9, 140):
        for offset, pitch, w_pitch, out_offset, out_pitch in ((0, 72, 72, 0, 72), (1, 73, 80, 3, 75), (8, 96, 128, 8, 80), (5, 72, 72, 0, 74)):
            base = torch.from_numpy(rng.normal(0, 1, N * pitch + 16).astype(np.float32)).bfloat16().cuda()
            h = base[offset:offset + N * pitch].view(N, pitch)[:, :H]
            w = torch.from_numpy(rng.normal(0, 0.2, (V, w_pitch)).astype(np.float32)).bfloat16().cuda()[:, :H]
            buf = torch.full((N * out_pitch + 16,), 5.0, dtype=torch.bfloat16, device="cuda")
            h_out = buf[out_offset:out_offset + N * out_pitch].view(N, out_pitch)[:, :H]
            w_buf = torch.full((V, w_pitch + 8), 5.0, dtype=torch.bfloat16, device="cuda")
            check(v, None, h, w, rng.integers(0, V, N).astype(np.int32), h_out=h_out, w_out=w_buf[:, 8:8 + H])
            assert (w_buf[:, :8] == 5).all() and (w_buf[:, 8 + H:] == 5).all()
            rest = buf.clone()
            rest[out_offset:out_offset + N * out_pitch].view(N, out_pitch)[:, :H] = 5.0
            assert (rest == 5).all()
        one = torch.from_numpy(rng.normal(0, 1, (1, H)).astype(np.float32)).bfloat16().cuda().expand(N, H)
        check(v, None, one, w.contiguous(), rng.integers(0, V, N).astype(np.int32))


def test_gradients_agree_with_differences():
    """The gradients against central differences of the definition in fp64 (step 1e-4, truncation below 1e-7): two roundings to bf16."""
    rng = np.random.default_rng(7)
    V, N, H = 40, 6, 16
    v = tli.Verifier(V, V, np.arange(V, dtype=np.int32))
    h, w, ids, teacher = inputs(rng, N, H, V, 3, V)
    tau, g = rng.choice(np.array([0.7, 1.0, 2.0], np.float32), N).astype(np.float32), rng.normal(0, 1, N).astype(np.float32)
    d = dict(teacher=teacher, temperature=torch.from_numpy(tau).cuda())
    d_ids = torch.from_numpy(ids).cuda()
    f = v.head_loss(h, w, d_ids, **d)
    b = v.head_loss_grad(h, w, d_ids, f["stats"], f["target_logits"], grad_loss=torch.from_numpy(g).cuda(), **d)
    h64, w64, t64 = h.double().cpu().numpy(), w.double().cpu().numpy(), teacher.double().cpu().numpy()
    value = lambda h_, w_: (lo.rows(h_ @ w_.T, np.ones(V, bool), ids, t64, tau)[0] * g).sum()
    q, p = lo.rows(h64 @ w64.T, np.ones(V, bool), ids, t64, tau)[3:5]
    G = np.abs(g[:, None] / tau[:, None] * (q - p))
    for got, x, size in ((b["grad_hidden"], 0, G @ np.abs(w64)), (b["grad_weight"], 1, G.T @ np.abs(h64))):
        got = got.double().cpu().numpy()
        for i, j in [(i, j) for i in range(got.shape[0]) for j in range(0, H, 5)]:
            e = np.zeros(got.shape)
            e[i, j] = 1e-4
            up, down = (h64 + e, h64 - e) if x == 0 else (w64 + e, w64 - e)
            diff = ((value(up, w64) - value(down, w64)) if x == 0 else (value(h64, up) - value(h64, down))) / 2e-4
            assert abs(diff - got[i, j]) <= 2.0 ** -8 * (size[i, j] + abs(got[i, j])) + 1e-6


def test_nothing():
    v = tli.Verifier(50, 1, np.array([0], np.int32))
    h, w, ids = torch.empty(0, 64, dtype=torch.bfloat16, device="cuda"), torch.ones(50, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda")
    f = v.head_loss(h, w, ids)
    b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])
    assert f["loss"].shape == (0,) and b["grad_hidden"].shape == (0, 64) and (b["grad_weight"] == 0).all()


@pytest.mark.parametrize("N", [1, 20, 33, 64, 65, 97, 130, 200, 300])
def test_scratch_that_holds_nan(N):
    """Nothing of the workspace is read that the call has not written."""
    rng = np.random.default_rng(N)
    V, H = 700, 136
    m = make_map(rng, V, V, 0.5)
    v = tli.Verifier(V, V, m)
    h, w, ids, teacher = inputs(rng, N, H, V, 3, V)
    ids[0] = np.flatnonzero(m >= 0)[:3]
    d = dict(teacher=teacher, side=D, ids_side=D, shared=True)
    d_ids = torch.from_numpy(ids).cuda()
    f = v.head_loss(h, w, d_ids, **d)
    b = v.head_loss_grad(h, w, d_ids, f["stats"], f["target_logits"], **d)
    assert all(torch.isfinite(x).all() for x in (f["loss"], f["stats"], b["grad_hidden"], b["grad_weight"]))
    v._scratch = lambda need: torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    f2 = v.head_loss(h, w, d_ids, **d)
    b2 = v.head_loss_grad(h, w, d_ids, f["stats"], f["target_logits"], **d)
    assert all(torch.equal(f[k], f2[k]) for k in f) and all(torch.equal(b[k], b2[k]) for k in b)


def test_a_first_call_that_is_captured():
    code = """
import numpy as np, torch
from paper_2502_05202_b200 import tli
v = tli.Verifier(500, 2, np.array([0, -1], np.int32))
for N in (8, 300):
    h, w = torch.randn(N, 64, device="cuda").bfloat16(), torch.randn(500, 64, device="cuda").bfloat16()
    ids = torch.arange(N, device="cuda", dtype=torch.int32)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        f = v.head_loss(h, w, ids)
        b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])
    g.replay()
    torch.cuda.synchronize()
    e = v.head_loss(h, w, ids)
    assert torch.equal(e["loss"], f["loss"]) and torch.equal(v.head_loss_grad(h, w, ids, e["stats"], e["target_logits"])["grad_weight"], b["grad_weight"])
"""
    import os
    import subprocess
    import sys
    subprocess.run([sys.executable, "-c", code], check=True, timeout=300, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))


def test_hidden_gradient_in_place():
    rng = np.random.default_rng(11)
    v = tli.Verifier(300, 2, np.array([0, -1], np.int32))
    for N in (40, 300):
        h, w, ids, _ = inputs(rng, N, 64, 300, 0, 300)
        d_ids = torch.from_numpy(ids).cuda()
        f = v.head_loss(h, w, d_ids)
        want = v.head_loss_grad(h, w, d_ids, f["stats"], f["target_logits"])
        dw = torch.empty_like(w)
        ws = torch.empty(tli.tli_head_loss_grad_workspace_bytes(v.ctx, N, 64, 1, 0), dtype=torch.uint8, device="cuda")
        a = tli.tli_head_loss_grad_args(N, 64, 1, 0, 0, 0, 0, h.data_ptr(), 64, w.data_ptr(), 64, d_ids.data_ptr(), None, None, f["stats"].data_ptr(),
                                        f["target_logits"].data_ptr(), None, h.data_ptr(), 64, dw.data_ptr(), 64, None, ws.data_ptr(), ws.numel())
        assert tli.load().tli_head_loss_grad(v.ctx, ctypes.byref(a), torch.cuda.current_stream().cuda_stream) == tli.TLI_OK
        assert torch.equal(h, want["grad_hidden"]) and torch.equal(dw, want["grad_weight"])


def test_captured_replayed_and_on_two_streams():
    rng = np.random.default_rng(8)
    V = 3000
    v = tli.Verifier(V, 3, np.array([0, -1, 2], np.int32))
    for N in (40, 500):
        h, w, ids, teacher = inputs(rng, N, 256, V, 5, V)
        ids = torch.from_numpy(ids).cuda()

        def both():
            f = v.head_loss(h, w, ids, teacher=teacher)
            b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"], teacher=teacher)
            return f["loss"], f["stats"], b["grad_hidden"], b["grad_weight"]

        want = both()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = both()
        for _ in range(3):
            for x in got:
                x.fill_(9)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
        outs = []
        for s in [torch.cuda.Stream() for _ in range(2)] * 3:
            with torch.cuda.stream(s):
                outs.append(both())
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for o in outs for a, b in zip(o, want))


def test_a_training_step():
    """Target ids into the drafter's table, one layer, the loss over the intersection, and every gradient back to the table, against fp64
    autograd of the same step on the same rounded values."""
    rng = np.random.default_rng(9)
    V_t, V_d, N, H, k = 900, 700, 200, 64, 8
    m = make_map(rng, V_t, V_d)
    v = tli.Verifier(V_t, V_d, m)
    table = torch.randn(V_d, H, device="cuda").bfloat16()
    head = (torch.randn(V_d, H, device="cuda") * 0.25).bfloat16()
    tokens = torch.from_numpy(rng.integers(0, V_t, N).astype(np.int32)).cuda()
    teacher_rows = torch.randn(N, V_t, device="cuda") * 3
    teacher, ids = teacher_rows.topk(k, dim=1)
    ids = ids.int()
    e = v.embed(tokens, table, scale=2.0, ids_side=T, table_side=D)
    f = v.head_loss(e["rows"], head, ids, teacher=teacher, side=D, ids_side=T, shared=True)
    g = torch.full((N,), 1.0 / N, device="cuda")
    b = v.head_loss_grad(e["rows"], head, ids, f["stats"], f["target_logits"], grad_loss=g, teacher=teacher, side=D, ids_side=T, shared=True)
    d_table = v.embed_grad(tokens, b["grad_hidden"], scale=2.0, ids_side=T, table_side=D, dtype=torch.float32)["grad"]
    # the same loss and the same gradient through rows of logits
    z = (e["rows"].float() @ head.float().T)
    r = v.loss(z, ids, teacher=teacher, side=D, ids_side=T, shared=True)
    assert (r["loss"] - f["loss"]).abs().max() <= 1e-5 and torch.equal(r["status"], f["status"])
    dz = v.loss_grad(z, ids, r["stats"], grad_loss=g, teacher=teacher, side=D, ids_side=T, shared=True)["grad"]
    assert (dz.double() @ head.double() - b["grad_hidden"].double()).norm() <= 2.0 ** -7 * b["grad_hidden"].double().norm()
    inv = torch.full((V_t,), -1, dtype=torch.long, device="cuda")
    mm = torch.from_numpy(m).cuda().long()
    inv[mm[mm >= 0]] = torch.nonzero(mm >= 0).flatten()
    tab, hd = table.double().requires_grad_(), head.double().requires_grad_()
    at = inv[tokens.long()]
    rows = 2.0 * tab[at.clamp(min=0)] * (at >= 0)[:, None]
    logits = (rows @ hd.T).masked_fill(mm < 0, -float("inf"))
    tid = inv[ids.long()]
    live = (tid >= 0).any(1)
    p = torch.softmax(teacher.double().masked_fill(tid < 0, -float("inf"))[live], 1)
    logq = torch.log_softmax(logits[live], 1).gather(1, tid[live].clamp(min=0))
    loss = torch.where(p > 0, p * (p.clamp(min=1e-300).log() - torch.where(p > 0, logq, 0.0)), 0.0).sum() / N
    loss.backward()
    assert abs(f["loss"].double().sum().item() / N - loss.item()) <= 1e-5 * abs(loss.item())
    for got, exact in ((d_table, tab.grad), (b["grad_weight"], hd.grad)):
        assert (got.double() - exact).norm() <= 2.0 ** -7 * exact.norm()


def test_refusals():
    V, H = 64, 16
    v = tli.Verifier(V, 40, np.concatenate((np.arange(30), np.full(10, -1))).astype(np.int32))
    h, w, ids = torch.zeros(4, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(V, H, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, dtype=torch.int32, device="cuda")
    f32, st = torch.zeros(4, device="cuda"), torch.zeros(4, 2, device="cuda")
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    need = tli.tli_head_loss_workspace_bytes(v.ctx, 4, H, 1, 0), tli.tli_head_loss_grad_workspace_bytes(v.ctx, 4, H, 1, 0)
    ws = torch.empty(max(need), dtype=torch.uint8, device="cuda")
    lib = tli.load()
    base = dict(N=4, H=H, k=1, hidden=h.data_ptr(), hidden_stride=H, weight=w.data_ptr(), weight_stride=H, ids=ids.data_ptr(), stats=st.data_ptr(),
                target_logits=f32.data_ptr(), workspace=ws.data_ptr(), workspace_bytes=ws.numel())

    def call(name, cls, extra, change):
        a = cls()
        for n, x in {**base, **extra, **change}.items():
            setattr(a, n, x)
        return getattr(lib, name)(v.ctx, ctypes.byref(a), None)

    forward = lambda **c: call("tli_head_loss", tli.tli_head_loss_args, dict(loss=f32.data_ptr()), c)
    back = lambda **c: call("tli_head_loss_grad", tli.tli_head_loss_grad_args, dict(grad_hidden=dh.data_ptr(), grad_hidden_stride=H, grad_weight=dw.data_ptr(), grad_weight_stride=H), c)
    for i, f in enumerate((forward, back)):
        assert f() == tli.TLI_OK and f(N=0) == tli.TLI_OK
        for bad in (dict(N=-1), dict(H=0), dict(H=12), dict(k=0), dict(k=2), dict(side=2), dict(ids_side=-1), dict(support=2), dict(support=1), dict(hidden=None),
                    dict(hidden=h.data_ptr() + 1), dict(hidden_stride=-H), dict(weight=None), dict(weight=w.data_ptr() + 8), dict(weight_stride=H + 4), dict(weight_stride=8),
                    dict(ids=None), dict(ids=ids.data_ptr() + 1), dict(stats=None), dict(stats=st.data_ptr() + 4), dict(target_logits=None)):
            assert f(**bad) == tli.TLI_ERR_ARG, bad
        for bad in (dict(workspace=None), dict(workspace=ws.data_ptr() + 8), dict(workspace_bytes=need[i] - 1)):
            assert f(**bad) == tli.TLI_ERR_WORKSPACE, bad
        assert f(N=tli.TLI_MAX_HEAD_TOKENS + 1) == tli.TLI_ERR_UNSUPPORTED and f(H=tli.TLI_MAX_H + 8) == tli.TLI_ERR_UNSUPPORTED
    assert forward(loss=None) == tli.TLI_ERR_ARG
    for bad in (dict(grad_hidden=None, grad_weight=None), dict(grad_hidden=dh.data_ptr() + 1), dict(grad_hidden_stride=H - 1), dict(grad_weight=dw.data_ptr() + 8),
                dict(grad_weight_stride=H + 4), dict(grad_weight_stride=8), dict(grad_weight=w.data_ptr()), dict(grad_hidden=w.data_ptr() + 32),
                dict(grad_hidden=dw.data_ptr()), dict(grad_weight=w.data_ptr() + 16 * (V - 1) * 2)):
        assert back(**bad) == tli.TLI_ERR_ARG, bad
    assert back(grad_hidden=None) == tli.TLI_OK and back(grad_weight=None) == tli.TLI_OK
    for size in (tli.tli_head_loss_workspace_bytes, tli.tli_head_loss_grad_workspace_bytes):
        assert size(v.ctx, 4, 12, 1, 0) == 0 and size(v.ctx, -1, 16, 1, 0) == 0 and size(v.ctx, 4, 16, 0, 0) == 0 and size(v.ctx, 4, 16, 1, 2) == 0
    for bad in (lambda: v.head_loss(h.float(), w, ids), lambda: v.head_loss(h, w.float(), ids), lambda: v.head_loss(h, w[:-1], ids), lambda: v.head_loss(h, w, ids.long()),
                lambda: v.head_loss(h.cpu(), w, ids), lambda: v.head_loss_grad(h, w, ids, st[:3], f32), lambda: v.head_loss_grad(h, w, ids, st, f32[:3])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(tli.TLIError):
        v.head_loss(h[:, :12].contiguous(), w[:, :12].contiguous(), ids)
