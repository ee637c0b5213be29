"""Speculative decoding under filters, the calls together as a server makes them: drafts sampled from the filtered q',
target and drafter rows filtered, verification on the filtered rows, the tokens carried into the other vocabulary's embeddings.
The emitted tokens follow the filtered target distribution (chi-square; sequences share logits and differ in uniforms)."""
import numpy as np
import pytest
import torch

import row_oracle as ro
from paper_2502_05202_b200 import tli, workload as wl
from test_gpu_lossless import chi2_ok, uniforms

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau,k,p,mp", [(1.0, 5, 1.0, 0.0), (0.8, 0, 0.75, 0.0), (1.3, 6, 0.9, 0.05)])
def test_filtered_speculation_is_lossless(tau, k, p, mp, dtype):
    rng = np.random.default_rng(21)
    V_t, V_d, K, B = 9, 11, 3, 21000
    id_map = np.array([4, -1, 0, 7, -1, 2, 8, -1, 5, 1, -1], np.int32)
    zt1 = torch.from_numpy(rng.normal(0, 1.2, (1, K + 1, V_t)).astype(np.float32)).to(dtype).cuda()
    zd1 = torch.from_numpy(rng.normal(0, 1.2, (1, K, V_d)).astype(np.float32)).to(dtype).cuda()
    full = lambda x, t: torch.full((B,), x, dtype=t, device="cuda")
    ask = dict(top_k=full(k, torch.int32), top_p=full(p, torch.float32), min_p=full(mp, torch.float32))
    one = {n: x[:1] for n, x in ask.items()}
    t = full(tau, torch.float32)
    v = tli.Verifier(V_t, V_d, id_map)
    d = v.sample(zd1.expand(B, K, V_d), t, uniforms(rng, (B, K)), side=D, **ask)
    ft = v.filter(zt1, t[:1], side=T, **one)["logits"]
    fd = v.filter(zd1, t[:1], side=D, **one)["logits"]
    out = v.verify(ft.expand(B, K + 1, V_t), fd.expand(B, K, V_d), d["tokens"], t, uniforms(rng, (B, K + 1)))
    torch.cuda.synchronize()
    ids, n, nxt = d["tokens"].cpu().numpy(), out["accepted"].cpu().numpy(), out["next_token"].cpu().numpy()
    # a zero residual cannot happen here; a draft is always inside the kept set, so its q' is the sampler's probability
    assert (out["row_status"].cpu().numpy() == 0).all() and (id_map[ids] >= 0).all()
    assert torch.allclose(out["q_draft"], d["prob"], rtol=0, atol=1e-5)
    zt, zd = zt1.double().cpu().numpy()[0], zd1.double().cpu().numpy()[0]
    reach = 1.0                                                              # probability that position j is reached
    for j in range(K + 1):
        kept, w, _ = ro.kept_ids(zt[j], np.ones(V_t, bool), np.float32(tau), k, np.float32(p), np.float32(mp))
        want = np.zeros(V_t)
        want[kept] = w / w.sum()
        reached = n >= j
        tok = np.where(n[reached] > j, id_map[ids[reached, j]], nxt[reached]) if j < K else nxt[reached]
        assert abs(reached.sum() - B * reach) <= 6 * np.sqrt(B * reach * (1 - reach)) + 1e-6
        if reached.sum() > 300:                                              # (two narrow kept sets may not overlap: no draft passes)
            chi2_ok(tok, want, "position %d" % j)
        if j < K:
            kept, w, _ = ro.kept_ids(zd[j], id_map >= 0, np.float32(tau), k, np.float32(p), np.float32(mp))
            reach *= np.minimum(want[id_map[kept]], w / w.sum()).sum()
    v.close()


@pytest.mark.parametrize("dtype", [wl.F32, wl.BF16])
def test_a_step_of_a_server(dtype):
    """One step at workload-like sizes, captured into a graph and replayed; mixed requests, some greedy."""
    cfg = wl.tiny_config(B=12, K=4, V_t=50021, V_d=30011, dtype=dtype, f_mapped=0.6, sigma_d=0.5,
                         temperatures=(0.0, 0.8, 1.0), seed=92)
    b = wl.make_batch(cfg)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    logits = lambda a: dev(a).view(torch.bfloat16) if dtype == wl.BF16 else dev(a)
    zt, zd = logits(b["target_logits"]), logits(b["drafter_logits"])
    tau, u = dev(b["temperature"]), dev(b["uniforms"])
    ud = u[:, :cfg.K].contiguous()
    ks, ps, ms = np.array([0, 50, 20, 0] * 3, np.int32), np.array([0.9, 1.0, 0.95, 1.0] * 3, np.float32), np.array([0, 0, 0, 0.05] * 3, np.float32)
    ask = dict(top_k=dev(ks), top_p=dev(ps), min_p=dev(ms))
    et, ed = torch.randn(cfg.V_t, 64, device="cuda").bfloat16(), torch.randn(cfg.V_d, 64, device="cuda").bfloat16()
    v = tli.Verifier(cfg.V_t, cfg.V_d, b["id_map"])
    v._ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def step():
        d = v.sample(zd, tau, ud, side=D, **ask)
        inputs = v.embed(d["tokens"], et, scale=8.0, ids_side=D, table_side=T)
        ft, fd = v.filter(zt, tau, **ask), v.filter(zd, tau, side=D, **ask)
        out = v.verify(ft["logits"], fd["logits"], d["tokens"], tau, u)
        back = v.embed(out["next_token"], ed, ids_side=T, table_side=D)
        return [d["tokens"], d["prob"], inputs["table_ids"], inputs["rows"], out["accepted"], out["next_token"], out["q_draft"],
                out["row_status"], back["table_ids"], back["rows"]]

    eager = [t.clone() for t in step()]
    torch.cuda.synchronize()
    tokens, prob, carried, rows, accepted, nxt, q, status, back, _ = (t.float().cpu().numpy() for t in eager)
    assert (status == 0).all()
    np.testing.assert_array_equal(carried, b["id_map"][tokens.astype(int)])
    sampled = (b["temperature"] > 0)[:, None] & np.ones_like(q, bool)
    np.testing.assert_allclose(q[sampled], prob[sampled], atol=1e-5)
    inv = ro.table_ids(nxt.astype(int), b["id_map"], cfg.V_t, 0, 1)
    np.testing.assert_array_equal(back, inv)
    # the emitted token is in the kept set of its row
    z = zt.double().cpu().numpy()
    for i in range(cfg.B):
        kept, _, _ = ro.kept_ids(z[i, int(accepted[i])], np.ones(cfg.V_t, bool), b["temperature"][i], ks[i], ps[i], ms[i])
        assert int(nxt[i]) in kept
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        outs = step()
    for _ in range(3):
        for t in outs:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        for a, e in zip(outs, eager):
            assert torch.equal(a, e)
    del g
    v.close()
