"""Device memory that a Verifier keeps for the filtered rows and the embedding gradient."""
import gc
import threading

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu


def test_close_gives_up_the_scratch_of_every_thread_and_stream():
    V, B, R = 32000, 16, 4
    v = tli.Verifier(V, 100, np.full(100, -1, np.int32))
    z, tau, u = torch.randn(B, R, V, device="cuda"), torch.ones(B, device="cuda"), torch.rand(B, R, device="cuda")
    need = tli.tli_sample_workspace_bytes(v.ctx, B, R, tli.TLI_F32, tli.TLI_SIDE_TARGET)
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    held, go = threading.Event(), threading.Event()

    def other():
        v.sample(z, tau, u)
        held.set()
        go.wait(60)                                                          # the thread lives on while the verifier is closed

    t = threading.Thread(target=other)
    t.start()
    assert held.wait(60)
    v.sample(z, tau, u)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        v.sample(z, tau, u)
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() >= before + 3 * need
    v.close()
    assert torch.cuda.memory_allocated() == before
    go.set()
    t.join()
    with pytest.raises(tli.TLIError):
        v.sample(z, tau, u)
