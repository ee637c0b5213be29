"""Device memory that a Verifier keeps after the losses of a training batch."""
import gc
import threading

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu


def test_the_scratch_of_a_training_batch_is_not_kept():
    N, H, V, keep = 4096, 256, 32768, 64 << 20
    v = tli.Verifier(V, 1, np.array([0], np.int32))
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") / 8).bfloat16()
    ids = torch.randint(0, V, (N,), device="cuda", dtype=torch.int32)
    assert tli.tli_head_loss_grad_workspace_bytes(v.ctx, N, H, 1, tli.TLI_SIDE_TARGET) > 4 * keep
    got, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()

    def step():
        f = v.head_loss(h, w, ids)
        return v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"])

    def other():
        with torch.cuda.stream(streams[1]):
            got.append(step())

    first = step()
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    with torch.cuda.stream(streams[0]):
        got.append(step())
    t = threading.Thread(target=other)
    t.start()
    t.join()
    torch.cuda.synchronize()
    held = sum(x.numel() * x.element_size() for g in got for x in g.values())
    assert len(got) == 2 and torch.cuda.memory_allocated() - before <= held + 2 * keep
    # ... and what the allocator hands out again behind the call is free again: the same gradients, one call after the other
    assert all(torch.equal(g[k], first[k]) for g in got for k in first)
    for _ in range(4):
        again = step()
        torch.full((100 << 20,), 0xff, dtype=torch.uint8, device="cuda")
        assert all(torch.equal(again[k], first[k]) for k in first)
