"""tli_embed() and tli_embed_grad() against fp64.

Lookup: a product in fp32 (2^-24) rounded once more to bf16 (2^-8 of half a step: eps/2 = 2^-8 relative).
Gradient: n terms added in fp32 in any order are off by at most (n-1) 2^-24 sum|g| (1 + tiny), then the scale (2^-24) and the
rounding to the output's type (eps/2); 2^-149 and 2^-133 are the smallest steps of the two types."""
import ctypes

import numpy as np
import pytest
import torch

import row_oracle as ro
from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133}
V_T, V_D = 1501, 1203


def make_map(rng, V_t=V_T, V_d=V_D, f=0.6):
    m = np.full(V_d, -1, np.int32)
    on = rng.permutation(V_d)[:min(V_t, int(f * V_d))]
    m[on] = rng.permutation(V_t)[:on.size]
    return m


def some_ids(rng, N, V):
    ids = np.minimum(np.exp(rng.random(N) * np.log(V)).astype(np.int64), V - 1).astype(np.int32)    # a few frequent ids
    if N > 4:
        ids[rng.integers(0, N, max(1, N // 20))] = rng.choice(np.array([-1, -7, V, V + 100, 2 ** 31 - 1, -2 ** 31], np.int64)).astype(np.int32)
    return ids


def check_embed(v, m, ids, table, scale, ids_side, table_side, shape=None):
    d = torch.from_numpy(ids).cuda()
    out = v.embed(d if shape is None else d.view(shape), table, scale=scale, ids_side=ids_side, table_side=table_side)
    want = ro.table_ids(ids, m, v.V_t, ids_side, table_side)
    np.testing.assert_array_equal(out["table_ids"].cpu().numpy().ravel(), want)
    t64 = table.double().cpu().numpy()
    exact = t64[np.maximum(want, 0)] * float(np.float32(scale))
    exact[want < 0] = 0
    got = out["rows"].double().cpu().numpy().reshape(exact.shape)
    assert (np.abs(got - exact) <= (HALF[table.dtype] + 2.0 ** -23) * np.abs(exact) + STEP[table.dtype]).all()
    assert (got[want < 0] == 0).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ids_side", [T, D])
@pytest.mark.parametrize("table_side", [T, D])
@pytest.mark.parametrize("N,H", [(1, 1), (1, 2048), (5, 8), (33, 129), (700, 256), (64, 4100), (300, 1000)])
def test_lookup(N, H, table_side, ids_side, dtype):
    rng = np.random.default_rng(N + H)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    table = torch.randn(V_T if table_side == T else V_D, H, device="cuda").to(dtype)
    ids = some_ids(rng, N, V_T if ids_side == T else V_D)
    check_embed(v, m, ids, table, 1.0, ids_side, table_side)
    check_embed(v, m, ids, table, -11.3, ids_side, table_side, shape=(1, N))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lookup_strides_and_alignment(dtype):
    rng = np.random.default_rng(1)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    for offset, pitch, H in ((0, 72, 64), (1, 72, 64), (8, 80, 64), (0, 67, 64), (4, 256, 200)):
        table = torch.randn(V_T, pitch + 16, device="cuda").to(dtype)[:, offset:offset + H]
        check_embed(v, m, some_ids(rng, 50, V_T), table, 2.0, T, T)
        out = torch.full((50, pitch + 9), 5.0, dtype=dtype, device="cuda")
        view = out[:, offset:offset + H]
        ids = torch.from_numpy(some_ids(rng, 50, V_D)).cuda()
        tli.tli_embed(v.ctx, tli.make_embed_args(ids, table, view, 2.0, D, T))
        assert torch.equal(view, v.embed(ids, table, 2.0, D, T)["rows"])
        assert (out[:, :offset] == 5).all() and (out[:, offset + H:] == 5).all()


def test_lookup_of_inf_nan_and_nothing():
    rng = np.random.default_rng(2)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    table = torch.randn(V_T, 16, device="cuda")
    table[3] = float("nan")
    table[4] = float("inf")
    out = v.embed(torch.tensor([3, 4, -1], dtype=torch.int32, device="cuda"), table, scale=0.5)["rows"]
    assert out[0].isnan().all() and (out[1] == float("inf")).all() and (out[2] == 0).all()
    empty = v.embed(torch.empty(0, dtype=torch.int32, device="cuda"), table)
    assert empty["rows"].shape == (0, 16) and empty["table_ids"].shape == (0,)


def check_grad(v, m, ids, grad, scale, ids_side, table_side, dtype, out=None):
    V = v.V_t if table_side == T else v.V_d
    N, H = grad.shape
    d = torch.from_numpy(ids).cuda()
    if out is None:
        got = v.embed_grad(d, grad, scale=scale, ids_side=ids_side, table_side=table_side, dtype=dtype)["grad"]
        assert torch.equal(got, v.embed_grad(d, grad, scale=scale, ids_side=ids_side, table_side=table_side, dtype=dtype)["grad"])
    else:
        ws = torch.empty(tli.tli_embed_grad_workspace_bytes(v.ctx, N, H), dtype=torch.uint8, device="cuda")
        tli.tli_embed_grad(v.ctx, tli.make_embed_grad_args(d, grad, out, ws, scale, ids_side, table_side))
        got = out
    t = ro.table_ids(ids, m, v.V_t, ids_side, table_side)
    g = grad.double().cpu().numpy()
    total, size, count = np.zeros((V, H)), np.zeros((V, H)), np.zeros(V)
    on = t >= 0
    np.add.at(total, t[on], g[on])
    np.add.at(size, t[on], np.abs(g[on]))
    np.add.at(count, t[on], 1)
    s = abs(float(np.float32(scale)))
    exact = total * float(np.float32(scale))
    bound = np.maximum(count - 1, 0)[:, None] * 2.0 ** -24 * 1.01 * size * s + (HALF[got.dtype] + 2.0 ** -23) * (np.abs(exact) + 1e-3 * size * s * (count[:, None] > 1)) + 2 * STEP[got.dtype]
    # (the roundings after the sum are relative to the computed sum, at most 1e-3 sum|g| away for fewer than 16 000 terms)
    err = np.abs(got.double().cpu().numpy() - exact)
    assert (err <= bound).all(), (err - bound).max()
    assert (got.cpu()[torch.from_numpy(count == 0)] == 0).all()


@pytest.mark.parametrize("gdtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("odtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("ids_side,table_side", [(T, T), (D, T), (T, D), (D, D)])
@pytest.mark.parametrize("N,H", [(1, 1), (1, 64), (31, 8), (33, 16), (257, 100), (2000, 72), (517, 1000), (4000, 13)])
def test_gradient(N, H, ids_side, table_side, odtype, gdtype):
    rng = np.random.default_rng(N * 7 + H)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    ids = some_ids(rng, N, V_T if ids_side == T else V_D)
    grad = torch.randn(N, H, device="cuda").to(gdtype)
    check_grad(v, m, ids, grad, 3.7, ids_side, table_side, odtype)


@pytest.mark.parametrize("kind", ["one id", "no id", "window ends", "two ids", "all once"])
def test_gradient_of_long_and_short_runs(kind):
    """Runs of one id that end at, before and after the ends of the windows the sorted tokens are cut into."""
    rng = np.random.default_rng(3)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    N = 1501
    ids = {"one id": np.full(N, 700), "no id": np.full(N, -1),
           "window ends": np.repeat([5, 6, 9, 1500, 0, 40, 41], [32, 31, 1, 64, 33, 96, 1244]),
           "two ids": rng.choice([1024, 1023], N), "all once": rng.permutation(V_T)}[kind].astype(np.int32)
    for gdtype in (torch.float32, torch.bfloat16):
        for H in (40, 7):
            check_grad(v, m, ids, torch.randn(N, H, device="cuda").to(gdtype), 1.0, T, T, torch.float32)


@pytest.mark.parametrize("N", [65535, 65536, 65537, 131072, 131073, 150001])
def test_gradient_of_many_tokens(N):
    """The sort of one cluster and of many CTAs; a vocabulary that needs both digits."""
    rng = np.random.default_rng(N)
    V_t, V_d = 70001, 5
    m = np.array([4, -1, 70000, 0, 1], np.int32)
    v = tli.Verifier(V_t, V_d, m)
    check_grad(v, m, some_ids(rng, N, V_t), torch.randn(N, 8, device="cuda"), 0.5, T, T, torch.float32)


def test_gradient_over_the_widest_vocabulary():
    rng = np.random.default_rng(4)
    V_t = tli.TLI_MAX_V
    v = tli.Verifier(V_t, 3, np.array([0, -1, V_t - 1], np.int32))
    ids = rng.integers(0, V_t, 3000).astype(np.int32)
    ids[:4] = [V_t - 1, 0, V_t - 1, 0]
    check_grad(v, np.array([0, -1, V_t - 1], np.int32), ids, torch.randn(3000, 4, device="cuda"), 1.0, T, T, torch.float32)


def test_gradient_strides_alignment_and_padding():
    rng = np.random.default_rng(5)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    ids = some_ids(rng, 300, V_D)
    for gdtype in (torch.float32, torch.bfloat16):
        for odtype in (torch.float32, torch.bfloat16):
            for offset, pitch, H in ((0, 72, 64), (1, 72, 64), (0, 67, 64)):
                grad = torch.randn(300, pitch + 8, device="cuda").to(gdtype)[:, offset:offset + H]
                buf = torch.full((V_T, pitch + 9), 5.0, dtype=odtype, device="cuda")
                check_grad(v, m, ids, grad, 2.0, D, T, odtype, out=buf[:, offset:offset + H])
                assert (buf[:, :offset] == 5).all() and (buf[:, offset + H:] == 5).all()
    one = torch.randn(1, 64, device="cuda").expand(300, 64)                  # one gradient row for every token
    check_grad(v, m, ids, one, 1.0, D, D, torch.float32)


def test_gradient_of_nothing_is_zero():
    rng = np.random.default_rng(6)
    v = tli.Verifier(V_T, V_D, make_map(rng))
    out = v.embed_grad(torch.empty(0, dtype=torch.int32, device="cuda"), torch.empty(0, 24, device="cuda"))["grad"]
    assert out.shape == (V_T, 24) and (out == 0).all()


def test_gradient_agrees_with_differences():
    """sum(out * c) as a function of the table, differenced in fp64 through the lookup's own definition (linear: exact but for rounding)."""
    rng = np.random.default_rng(7)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    ids = torch.from_numpy(some_ids(rng, 64, V_D)).cuda()
    c = torch.randn(64, 16, device="cuda")
    grad = v.embed_grad(ids, c, scale=2.0, ids_side=D, table_side=T)["grad"]
    table = torch.randn(V_T, 16, device="cuda")
    f = lambda t: (v.embed(ids, t, scale=2.0, ids_side=D, table_side=T)["rows"].double() * c.double()).sum().item()
    used = v.embed(ids, table, ids_side=D, table_side=T)["table_ids"]
    for row in used[used >= 0][:5].tolist() + [int(m.max()) - 1]:
        step = torch.zeros_like(table)
        step[row, 3] = 8.0
        diff = (f(table + step) - f(table - step)) / 16.0
        # the lookup rounds 64 rows of about |x| < 16 to 2^-24 each
        assert abs(diff - grad[row, 3].item()) <= 64 * 16 * 2 * 2.0 ** -23 + 1e-5


def test_captured_and_replayed():
    rng = np.random.default_rng(8)
    m = make_map(rng)
    v = tli.Verifier(V_T, V_D, m)
    ids = torch.from_numpy(some_ids(rng, 900, V_D)).cuda()
    table, grad = torch.randn(V_T, 128, device="cuda"), torch.randn(900, 128, device="cuda")
    want = v.embed(ids, table, 1.5, D, T)["rows"], v.embed_grad(ids, grad, 1.5, D, T)["grad"]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = v.embed(ids, table, 1.5, D, T)["rows"], v.embed_grad(ids, grad, 1.5, D, T)["grad"]
    for _ in range(3):
        got[0].fill_(9); got[1].fill_(9)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_refusals():
    rng = np.random.default_rng(9)
    v = tli.Verifier(V_T, V_D, make_map(rng))
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    table, out = torch.zeros(V_T, 16, device="cuda"), torch.zeros(4, 16, device="cuda")
    grad, dw = torch.zeros(4, 16, device="cuda"), torch.zeros(V_T, 16, device="cuda")
    ws = torch.empty(tli.tli_embed_grad_workspace_bytes(v.ctx, 4, 16), dtype=torch.uint8, device="cuda")
    lib = tli.load()

    def embed(**change):
        a = tli.make_embed_args(ids, table, out)
        for n, x in change.items():
            setattr(a, n, x)
        return lib.tli_embed(v.ctx, ctypes.byref(a), None)

    def back(**change):
        a = tli.make_embed_grad_args(ids, grad, dw, ws)
        for n, x in change.items():
            setattr(a, n, x)
        return lib.tli_embed_grad(v.ctx, ctypes.byref(a), None)

    assert embed() == tli.TLI_OK and back() == tli.TLI_OK and embed(N=0) == tli.TLI_OK
    for bad in (dict(N=-1), dict(H=0), dict(dtype=2), dict(ids_side=2), dict(table_side=-1), dict(ids=None), dict(table=None),
                dict(out=None), dict(table=table.data_ptr() + 2), dict(out_stride=15), dict(table_stride=-16)):
        assert embed(**bad) == tli.TLI_ERR_ARG, bad
    for bad in (dict(N=-1), dict(H=0), dict(grad_dtype=2), dict(out_dtype=-1), dict(ids_side=2), dict(table_side=-1), dict(ids=None),
                dict(grad=None), dict(out=None), dict(out=dw.data_ptr() + 1), dict(out_stride=15), dict(grad_stride=-16)):
        assert back(**bad) == tli.TLI_ERR_ARG, bad
    for call in (embed, back):
        assert call(N=tli.TLI_MAX_TOKENS + 1) == tli.TLI_ERR_UNSUPPORTED and call(H=tli.TLI_MAX_H + 1) == tli.TLI_ERR_UNSUPPORTED
    for bad in (dict(workspace=None), dict(workspace=ws.data_ptr() + 8), dict(workspace_bytes=ws.numel() - 1)):
        assert back(**bad) == tli.TLI_ERR_WORKSPACE, bad
    with pytest.raises(ValueError):
        v.embed(ids, table[:-1])
    with pytest.raises(ValueError):
        v.embed(ids.long(), table)
    with pytest.raises(ValueError):
        v.embed_grad(ids, grad[:3])
    with pytest.raises(TypeError):
        v.embed(ids, table.half())
