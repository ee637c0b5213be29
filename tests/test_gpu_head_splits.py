"""d hidden where the last run of the vocabulary is so short that one of the two splits has no step of it (55 runs of 14 080 ids, the last
of 31, on 148 SMs): zeros are added to that split's sums, not what tensor memory holds.

Two roundings to bf16 (G's and the result's), each at most 2^-8 and on average over mantissas 2^-8 / sqrt(3) or less, as everywhere for
these gradients; the sums of 760 351 terms that are all but zero beside the label's add less than 2^-16 to that."""
import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("few", [False, True])
def test_a_split_without_a_step(few):
    """few: all but 100 of the rows are left out."""
    N, H, V = 9400, 8, 760351
    v = tli.Verifier(V, 1, np.array([0], np.int32))
    v._scratch = lambda need: torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(int(few))
    h, w = torch.randn(N, H, device="cuda", generator=g).bfloat16(), (torch.randn(V, H, device="cuda", generator=g) * 0.7).bfloat16()
    ids = torch.randint(0, V, (N,), device="cuda", generator=g, dtype=torch.int32)
    ids[::2] = V - 1 - ids[::2] % 31                                         # (labels in the last run too)
    if few:
        ids[100:] = -1
    f = v.head_loss(h, w, ids)
    b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])
    assert torch.isfinite(b["grad_hidden"]).all() and torch.isfinite(b["grad_weight"]).all()
    rows = torch.arange(100 if few else N, device="cuda")[:: 1 if few else 94]
    w64, t = w.double(), ids[rows].long()
    z = h[rows].double() @ w64.T
    assert (f["loss"][rows].double() - (torch.logsumexp(z, 1) - z.gather(1, t[:, None])[:, 0])).abs().max() <= 1e-4
    d = torch.softmax(z, 1)
    d[torch.arange(rows.numel(), device="cuda"), t] -= 1
    exact = d @ w64
    assert (b["grad_hidden"][rows].double() - exact).norm() <= 2.0 ** -8 * exact.norm()
    if few:
        assert (b["grad_hidden"][100:] == 0).all()
        last = d[:, -31:].T @ h[rows].double()
        assert (b["grad_weight"][-31:].double() - last).norm() <= 2.0 ** -8 * last.norm()
