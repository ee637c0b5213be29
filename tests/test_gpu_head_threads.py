"""One Verifier, several threads: every call has to end and to give what it gives alone."""
from concurrent.futures import ThreadPoolExecutor

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

ROUNDS = 20


def job(v, N, H, V, shared):
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") / 8).bfloat16()
    z = (torch.randn(N, V, device="cuda") * 2).bfloat16()
    ids = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
    how = dict(side=tli.TLI_SIDE_DRAFTER, ids_side=tli.TLI_SIDE_DRAFTER, shared=shared)

    def calls():
        f = v.head_loss(h, w, ids, **how)
        b = v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"], **how)
        r = v.loss(z, ids, **how)
        return f["loss"], b["grad_hidden"], b["grad_weight"], r["loss"], v.loss_grad(z, ids, r["stats"], **how)["grad"]

    return calls


@pytest.mark.parametrize("own_stream", [False, True])
def test_threads_at_once(own_stream):
    V = 5000
    v = tli.Verifier(V, V, np.where(np.arange(V) % 3 > 0, np.arange(V), -1).astype(np.int32))
    jobs = [job(v, N, 256, V, shared) for N, shared in ((60, True), (700, False), (1, False), (130, True))]
    want = [calls() for calls in jobs]
    torch.cuda.synchronize()

    def work(i):
        done = 0
        with torch.cuda.stream(torch.cuda.Stream() if own_stream else torch.cuda.current_stream()):
            for _ in range(ROUNDS):
                assert all(torch.equal(a, b) for a, b in zip(jobs[i](), want[i]))
                done += 1
        return done

    with ThreadPoolExecutor(len(jobs)) as pool:
        results = [pool.submit(work, i) for i in range(len(jobs))]
        assert [r.result(timeout=120) for r in results] == [ROUNDS] * len(jobs)      # (result() raises what its thread raised)
