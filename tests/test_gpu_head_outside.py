"""tli_head_loss() and tli_head_loss_grad() over the intersection, where weight rows of ids outside it hold NaN and infinities: those ids do
not take part, so every output is what it is with zeros in their place.

Everything but d hidden is the same to the bit: these ids are left out of the statistics and have G = 0, and no other sum has their weights.
d hidden's sums are formed in another order: n terms G w one after the other in fp32 lose n 2^-24 of sum |G w|, the matrix unit's (n / 16 + 8)
2^-23; both have the same G (bf16, within 2^-8 of g (q - p), so sum |G w| <= (1 + 2^-7) sum |g (q - p) w|), and both are rounded to bf16, half a
step (2^-8) each."""
import numpy as np
import pytest
import torch

import test_gpu_head as th
from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER
NONE = float("nan"), float("inf"), -float("inf")


def run(v, h, w, ids, teacher):
    how = dict(teacher=teacher, side=D, ids_side=D, shared=True)
    f = v.head_loss(h, w, ids, **how)
    b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"], **how)
    return f, b


def compare(v, m, h, clean, dirty, ids, teacher, bad_rows=()):
    inside = torch.from_numpy(m >= 0).cuda()
    (f, b), (f2, b2) = run(v, h, clean, ids, teacher), run(v, h, dirty, ids, teacher)
    same = lambda x, y: torch.equal(torch.nan_to_num(x, nan=7.0), torch.nan_to_num(y, nan=7.0))
    for k in ("loss", "stats", "target_logits", "status"):
        assert same(f[k], f2[k]), k
    assert torch.equal(b["status"], b2["status"]) and same(b["grad_weight"], b2["grad_weight"])
    fine = torch.ones(h.shape[0], dtype=torch.bool, device="cuda")
    fine[list(bad_rows)] = False
    x, y = b["grad_hidden"].double(), b2["grad_hidden"].double()
    assert torch.isnan(x[~fine]).all() and torch.isnan(y[~fine]).all()
    x, y, V = x[fine], y[fine], clean.shape[0]
    G = torch.softmax((h[fine].double() @ clean.double().T).masked_fill(~inside, -float("inf")), 1)
    k = ids.view(h.shape[0], -1)[fine].long()
    p = torch.ones_like(k, dtype=torch.float64) if teacher is None else torch.softmax(teacher[fine].double(), 1)
    G.scatter_add_(1, k, -p)
    size = G.abs() @ clean.double().abs()
    bound = 2.0 ** -8 * (x.abs() + y.abs()) + (V / 16 + V / 2 + 9) * 2.0 ** -23 * (1 + 2.0 ** -7) * size + 2.0 ** -126
    assert ((x - y).abs() <= bound).all()                                    # (false for NaN)


def inputs(N, H, V, k, share):
    rng = np.random.default_rng(N + H + V)
    m = th.make_map(rng, V, V, share)
    h, w, ids, teacher = th.inputs(rng, N, H, V, k, V)
    inside, outside = np.flatnonzero(m >= 0), np.flatnonzero(m < 0)
    ids = torch.from_numpy(rng.choice(inside, ids.shape).astype(np.int32)).cuda()
    clean = w.clone()
    clean[torch.from_numpy(outside).cuda()] = 0
    return rng, m, h, clean, ids, teacher, outside


@pytest.mark.parametrize("N", [1, 5, 129, 300])
@pytest.mark.parametrize("H,V,k,share", [(8, 3, 0, 0.4), (264, 700, 0, 0.5), (72, 5003, 3, 0.9), (520, 1500, 2, 0.05)])
def test_all_of_them(N, H, V, k, share):
    rng, m, h, clean, ids, teacher, outside = inputs(N, H, V, k, share)
    dirty = clean.clone()
    for i, v in enumerate(outside):
        dirty[v] = NONE[i % 3]
    compare(tli.Verifier(V, V, m), m, h, clean, dirty, ids, teacher)


@pytest.mark.parametrize("N,V", [(40, 900), (300, 900), (20000, 20000)])
def test_a_few_elements(N, V):
    """Some columns of d hidden are the matrix unit's and some are not; of 20000 rows and ids, several runs of the vocabulary."""
    rng, m, h, clean, ids, teacher, outside = inputs(N, 72, V, 0, 0.5)
    dirty = clean.clone()
    for i, v in enumerate(rng.choice(outside, 5, replace=False)):
        dirty[v, int(rng.choice([0, 31, 32, 71]))] = NONE[i % 3]
    compare(tli.Verifier(V, V, m), m, h, clean, dirty, ids, teacher)


@pytest.mark.parametrize("N", [7, 200])
def test_beside_a_row_that_is_nan_itself(N):
    _, m, h, clean, ids, teacher, outside = inputs(N, 136, 600, 0, 0.5)
    h[3] = float("nan")
    dirty = clean.clone()
    dirty[torch.from_numpy(outside).cuda()] = float("nan")
    compare(tli.Verifier(600, 600, m), m, h, clean, dirty, ids, teacher, (3,))
    compare(tli.Verifier(600, 600, m), m, h, clean, clean, ids, teacher, (3,))


def test_rows_none_of_which_takes_part():
    _, m, h, clean, ids, _, outside = inputs(50, 64, 400, 0, 0.5)
    ids[:] = int(outside[0])
    f, b = run(tli.Verifier(400, 400, m), h, torch.full_like(clean, float("nan")), ids, None)
    assert (f["loss"] == 0).all() and (f["status"] == tli.TLI_ROW_LEFT_OUT).all() and (b["grad_hidden"] == 0).all() and (b["grad_weight"] == 0).all()
