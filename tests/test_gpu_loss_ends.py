"""The losses at the ends of their ranges (most tokens, widest vocabulary, longest rows, offsets beyond 32 bits, the sizes where the row
kernels' cut changes, two threads at once), against torch in fp64.

Tolerances. A loss over rows of logits of size 8 at most: a sum of at most 16 385 terms in parts of a thread (2^-24 a step, some hundred steps)
and the rounding of lse and of the loss, together below 1e-5; over 9 elements 2e-6. The head's loss has the rounding of its products on top,
H steps of 2^-24 of the running sum at most: 1e-4. A gradient in bf16 has one rounding of half a step, 2^-8 (absolute where no element
is above 1). The head's gradients round G once and the result once, independently: each element below 2^-8, whose mean square over a
binade is a third of that, so the norm of both together stays below 2^-8."""
import threading

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu


def one_sided(V):
    return tli.Verifier(V, 1, np.array([0], np.int32))


def check_head(v, h, w, ids, grads=True):
    N = h.shape[0]
    f = v.head_loss(h, w, ids)
    b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"]) if grads else None
    dw = torch.zeros(w.shape, dtype=torch.float64, device="cuda")
    w64, step = w.double(), max(1, 100_000_000 // w.shape[0])
    live = (ids >= 0) & (ids < w.shape[0])
    worst = off = size = 0.0
    for a in range(0, N, step):
        hh, t, on = h[a:a + step].double(), ids[a:a + step].long().clamp(0, w.shape[0] - 1), live[a:a + step]
        z = hh @ w64.T
        lse = torch.logsumexp(z, 1)
        loss = torch.where(on, lse - z.gather(1, t[:, None])[:, 0], torch.zeros_like(lse))
        worst = max(worst, (f["loss"][a:a + step].double() - loss).abs().max().item())
        if grads:
            d = torch.softmax(z, 1)
            d[torch.arange(d.shape[0], device="cuda"), t] -= 1
            d *= on[:, None]
            e = d @ w64
            off += (b["grad_hidden"][a:a + step].double() - e).square().sum().item()
            size += e.square().sum().item()
            dw += d.T @ hh
    assert worst <= 1e-4
    if grads:
        assert off <= (2.0 ** -8) ** 2 * size
        assert (b["grad_weight"].double() - dw).norm() <= 2.0 ** -8 * dw.norm()


@pytest.mark.parametrize("H", [8, 72])
def test_the_most_tokens(H):
    N, V = tli.TLI_MAX_HEAD_TOKENS, 300
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") * 2 / H ** 0.5).bfloat16()
    ids = torch.randint(-1, V, (N,), device="cuda", dtype=torch.int32)
    check_head(one_sided(V), h, w, ids)


@pytest.mark.parametrize("N", [3, 200])
def test_the_widest_vocabulary(N):
    V, H = tli.TLI_MAX_V, 64
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") * 0.25).bfloat16()
    ids = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
    ids[0] = V - 1
    check_head(one_sided(V), h, w, ids)


@pytest.mark.parametrize("N", [4, 150])
def test_the_widest_rows(N):
    V, H = 300, tli.TLI_MAX_H
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") * 2 / H ** 0.5).bfloat16()
    check_head(one_sided(V), h, w, torch.randint(0, V, (N,), device="cuda", dtype=torch.int32))


def test_weight_rows_beyond_32_bits():
    V, H, pitch = 40000, 64, 65536                                           # 2.6e9 elements, 5.2 GB from the first row to the last
    big = torch.empty(V * pitch, dtype=torch.bfloat16, device="cuda")
    w = big.view(V, pitch)[:, :H]
    w.copy_(torch.randn(V, H, device="cuda") * 0.25)
    v = one_sided(V)
    for N in (5, 300):
        h = torch.randn(N, H, device="cuda").bfloat16()
        ids = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
        ids[0] = V - 1
        check_head(v, h, w, ids)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_most_rows_of_logits(dtype):
    N, V = tli.TLI_MAX_TOKENS, 9
    v = one_sided(V)
    z = torch.randn(N, V, device="cuda").to(dtype)
    ids = torch.randint(-1, V, (N,), device="cuda", dtype=torch.int32)
    f = v.loss(z, ids)
    on = ids >= 0
    want = torch.nn.functional.cross_entropy(z.double(), ids.long().clamp(min=0), reduction="none") * on
    assert (f["loss"].double() - want).abs().max() <= 2e-6 and torch.equal(f["status"], torch.where(on, 0, tli.TLI_ROW_LEFT_OUT).int())
    d = torch.softmax(z.double(), 1)
    d[torch.arange(N, device="cuda"), ids.long().clamp(min=0)] -= 1
    d *= on[:, None]
    g = v.loss_grad(z, ids, f["stats"])["grad"].double()
    assert (g - d).abs().max() <= (2e-6 if dtype is torch.float32 else 2.0 ** -8)


@pytest.mark.parametrize("V", [511, 512, 513, 2047, 2049, 4095, 4097, 8191, 8193, 16383, 16385])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_around_the_sizes_where_the_cut_changes(V, dtype):
    v = one_sided(V)
    for N, k in ((1300, 64), (1300, 65), (40, 64), (2, 1)):
        z = (torch.randn(N, V, device="cuda") * 2).to(dtype)
        ids = torch.randint(0, V, (N, k), device="cuda", dtype=torch.int32)
        teacher = torch.randn(N, k, device="cuda")
        f = v.loss(z, ids, teacher=teacher)
        p, lq = torch.softmax(teacher.double(), 1), torch.log_softmax(z.double(), 1)
        want = (p * (p.log() - lq.gather(1, ids.long()))).sum(1)
        assert (f["loss"].double() - want).abs().max() <= 1e-5
        d = lq.exp().scatter_add_(1, ids.long(), -p)
        g = v.loss_grad(z, ids, f["stats"], teacher=teacher)["grad"].double()
        assert (g - d).norm() <= (1e-5 if dtype is torch.float32 else 2.0 ** -8) * d.norm()


def test_two_threads_at_once():
    V, H = 5000, 256
    v = one_sided(V)
    jobs = []
    for N in (60, 700):
        h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") / 8).bfloat16()
        ids = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
        f = v.head_loss(h, w, ids)
        b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])
        jobs.append((h, w, ids, f["loss"].clone(), b["grad_hidden"].clone(), b["grad_weight"].clone()))
    torch.cuda.synchronize()
    bad = []

    def work(job, own_stream):
        h, w, ids, loss, dh, dw = job
        with torch.cuda.stream(torch.cuda.Stream() if own_stream else torch.cuda.current_stream()):
            for _ in range(20):
                f = v.head_loss(h, w, ids)
                b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])
                if not (torch.equal(f["loss"], loss) and torch.equal(b["grad_hidden"], dh) and torch.equal(b["grad_weight"], dw)):
                    bad.append(h.shape)

    for own_stream in (False, True):
        threads = [threading.Thread(target=work, args=(job, own_stream)) for job in jobs]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    torch.cuda.synchronize()
    assert not bad
