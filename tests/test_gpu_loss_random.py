"""Random calls of the losses and their gradients (sizes over their logarithm, sides, maps, masks, teachers, types, strides), every element
against fp64.

Bounds, as derived in test_gpu_loss.py and test_gpu_head.py: with dz = (H / 16 + 8) 2^-23 sum |h w| (0 for rows of logits), a = (m - z) / tau, mean and
`high` over the ids that take part,
    eps (of the sum) = mean of (2^-22 a + 2 dz / tau) under q + high / tau + (V / 8192 + 60) 2^-22 + (V / 1024 + 64) 2^-24,      high = max dz
    loss: eps + 2^-22 |ln sum| + (terms + 1) 2^-20 + 2 high / tau + the targets' share, far (1 + (a + far) / 2) 2^-21, far = max |t - max t| / tau
    G:    |g / tau| (q (2^-22 a + (2 dz + high) / tau + eps + 2^-21) + p (2^-20 + 2 far 2^-22)), then half a step of its type
          and (1 + |g / tau|) 2^-126: a weight below 2^-126 is flushed to 0 before g / (tau sum), sum >= 1, multiplies it, and the product is flushed again
    a product's sums over n terms: (n / 16 + 8) 2^-23 of sum |G w|, then half a step of bf16."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
TINY = 2.0 ** -126


def one(rng, gen):
    size = lambda low, high: int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    rand = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    head = rng.random() < 0.7
    V_t, V_d, side, ids_side = size(1, 300000), size(1, 150000), rng.choice([T, D]), rng.choice([T, D])
    shared = side == D and rng.random() < 0.5
    V, V_ids = (V_t if side == T else V_d), (V_t if ids_side == T else V_d)
    k = rng.choice([1, 1, 1, 2, 5, 33, 64, 200, 256])
    labels, H = k == 1 and rng.random() < 0.7, 8 * size(1, 1100)
    N = max(1, min(size(1, 4000), 40_000_000 // V, 30_000_000_000 // (V * H) if head else 4000))
    what = dict(head=head, N=N, H=H, V_t=V_t, V_d=V_d, side=side, ids_side=ids_side, shared=shared, k=k, labels=labels)
    np_rng = np.random.default_rng(rng.randrange(1 << 30))
    m = np.full(V_d, -1, np.int32)
    on = np_rng.permutation(V_d)[:max(1, min(V_t, int(rng.choice([0.02, 0.3, 0.9]) * V_d)))]
    m[on] = np_rng.permutation(V_t)[:on.size]
    forth = torch.from_numpy(m).cuda().long()
    back = torch.full((V_t,), -1, dtype=torch.long, device="cuda")
    back[forth[forth >= 0]] = torch.nonzero(forth >= 0).flatten()
    ids = torch.randint(0, V_ids, (N,) if labels else (N, k), device="cuda", generator=gen, dtype=torch.int32)
    if rng.random() < 0.5:
        ids.view(-1)[torch.rand(ids.numel(), device="cuda", generator=gen) < 0.1] = -1
    teacher = None if labels else (rand(N, k) * 2).to(rng.choice([torch.float32, torch.bfloat16]))
    tau = None if rng.random() < 0.5 else torch.rand(N, device="cuda", generator=gen) * 2 + 0.3
    g = None if rng.random() < 0.3 else rand(N) / N
    how = dict(teacher=teacher, temperature=tau, side=side, ids_side=ids_side, shared=shared)

    # the targets
    t = ids.view(N, -1).long()
    t = torch.where(t >= 0, t if side == ids_side else (forth if ids_side == D else back)[t.clamp(min=0)], t)
    takes = t >= 0
    if shared:
        takes &= forth[t.clamp(min=0)] >= 0
    live, at = takes.any(1), t.clamp(min=0)
    tau64 = (torch.ones(N, device="cuda") if tau is None else tau).double()[:, None]
    y = (torch.zeros(N, k, device="cuda") if labels else teacher).double().div(tau64).masked_fill(~takes, -math.inf)
    p = torch.softmax(y, 1).nan_to_num(0.0)
    far = torch.where(takes, y.amax(1, keepdim=True) - y, 0.0).amax(1)

    v = tli.Verifier(V_t, V_d, m)
    if head:
        h = rand(N, H + rng.choice([0, 0, 3, 8])).bfloat16()[:, :H]
        w = (rand(V, H) * (2 / H ** 0.5)).bfloat16()
        if rng.random() < 0.3:
            h[~live] = float("nan")
        f = v.head_loss(h, w, ids, **how)
        h64, w64 = torch.where(live[:, None], h.double(), 0.0), w.double()
        z, dz = h64 @ w64.T, (h64.abs() @ w64.abs().T) * ((H / 16 + 8) * 2.0 ** -23)
    else:
        rows = (rand(N, V + rng.choice([0, 0, 1, 5])) * 3).to(rng.choice([torch.float32, torch.bfloat16]))[:, :V]
        f = v.loss(rows, ids, **how)
        z, dz = rows.double(), torch.zeros(N, 1, dtype=torch.float64, device="cuda")
    if shared:
        z, dz = z.masked_fill(forth < 0, -math.inf), (dz * (forth >= 0) if head else dz)
    lq = torch.log_softmax(z / tau64, 1)
    q, high = lq.exp(), dz.amax(1) / tau64[:, 0]
    top = z.amax(1, keepdim=True)
    a = torch.where(q > 0, (top - z) / tau64, 0.0)
    eps = (q * (a * 2.0 ** -22 + 2 * dz / tau64)).sum(1) + high + (V / 8192 + 60) * 2.0 ** -22 + (V / 1024 + 64) * 2.0 ** -24
    lp, lq_t, a_t = torch.where(p > 0, p.clamp(min=1e-300).log(), 0.0), torch.where(takes, lq.gather(1, at), 0.0), torch.where(takes, (top - z.gather(1, at)) / tau64, 0.0)
    loss = (p * (lp - lq_t)).sum(1) * live
    terms = (p * (lp.abs() + a_t)).sum(1)
    bound = eps + 2.0 ** -22 * (lq.amax(1)).abs() + (terms + 1) * 2.0 ** -20 + 2 * high + far * (1 + (a_t.amax(1) + far) / 2) * 2.0 ** -21
    assert torch.equal(f["status"], torch.where(live, 0, tli.TLI_ROW_LEFT_OUT).int()), what
    assert ((f["loss"].double() - loss).abs() <= bound * live).all(), (what, (f["loss"].double() - loss).abs().max().item())

    scale = ((torch.ones(N, device="cuda") if g is None else g).double() * live)[:, None] / tau64
    spread = torch.zeros_like(q).scatter_add_(1, at, p)
    G = scale * (q - spread)
    err = scale.abs() * (q * (a * 2.0 ** -22 + 2 * dz / tau64 + (high + eps)[:, None] + 2.0 ** -21) + spread * (2.0 ** -20 + far[:, None] * 2.0 ** -21)) + TINY * (1 + scale.abs())
    if head:
        b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"], grad_loss=g, **how)
        err = err + 2.0 ** -8 * (G.abs() + err)
        for got, x, e, s, n in ((b["grad_hidden"], G @ w64, err @ w64.abs(), G.abs() @ w64.abs(), V), (b["grad_weight"], G.T @ h64, err.T @ h64.abs(), G.abs().T @ h64.abs(), N)):
            e = e + (n / 16 + 8) * 2.0 ** -23 * (s + e)
            e = e + 2.0 ** -8 * (x.abs() + e) + TINY
            assert ((got.double() - x).abs() <= e).all(), (what, ((got.double() - x).abs() - e).max().item())
        assert (b["grad_hidden"][~live] == 0).all()
    else:
        got = v.loss_grad(rows, ids, f["stats"], grad_loss=g, **how)["grad"]
        e = err + HALF[rows.dtype] * (G.abs() + err)
        assert ((got.double() - G).abs() <= e).all(), (what, ((got.double() - G).abs() - e).max().item())
    v.close()


@pytest.mark.parametrize("seed", range(20))
def test_random_calls(seed):
    rng, gen = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    for _ in range(25):
        one(rng, gen)
