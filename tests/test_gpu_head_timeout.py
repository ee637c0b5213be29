"""What the head losses say after a bounded wait has run out: no kernel waits here, the host sets the word that such a wait sets."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

from rows_on_cpu import CSRC, _definition
from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

T, D = tli.TLI_SIDE_TARGET, tli.TLI_SIDE_DRAFTER


@pytest.fixture(scope="module")
def error_word(tmp_path_factory):
    """Device address of a context's word, by the context's own definition."""
    src = open(os.path.join(CSRC, "tli.cu")).read()
    assert "P.error = ctx->d_counters + 3 * (TLI_MAX_B + 1);" in src
    d = tmp_path_factory.mktemp("ctx")
    (d / "x.cpp").write_text("#include <cstdint>\nstruct float2 { float x, y; };\n" + _definition(src, "struct tli_ctx ") + "\nenum { TLI_MAX_B = %d };\n" % tli.TLI_MAX_B +
                             'extern "C" void *word(tli_ctx *ctx) { return ctx->d_counters + 3 * (TLI_MAX_B + 1); }\n')
    subprocess.run(["g++", "-std=c++17", "-fPIC", "-shared", "-o", str(d / "x.so"), str(d / "x.cpp")], check=True)
    fn = ctypes.CDLL(str(d / "x.so")).word
    fn.argtypes, fn.restype = [ctypes.c_void_p], ctypes.c_void_p
    return fn


@pytest.mark.parametrize("N,k", [(1, 0), (40, 0), (300, 0), (150, 7), (70, 40)])
def test_a_wait_that_ran_out_reaches_every_row(error_word, N, k):
    rng = np.random.default_rng(N)
    V, H = 500, 64
    m = np.where(rng.random(V) < 0.5, np.arange(V), -1).astype(np.int32)
    v = tli.Verifier(V, V, m)
    h, w = torch.randn(N, H, device="cuda").bfloat16(), (torch.randn(V, H, device="cuda") / 4).bfloat16()
    ids = torch.from_numpy(rng.integers(-1, V, (N, k) if k else N).astype(np.int32)).cuda()      # (some take part and some do not)
    teacher = torch.randn(N, k, device="cuda") if k else None
    how = dict(teacher=teacher, side=D, ids_side=T, shared=True)

    def calls():
        f = v.head_loss(h, w, ids, **how)
        both, weight, hidden = (v.head_loss_grad(h, w, ids, f["stats"], f["target_logits"], hidden_grad=a, weight_grad=b, **how)
                                for a, b in ((True, True), (False, True), (True, False)))
        return f, both, weight, hidden

    def check(got, flag):
        for a, b in zip(got, want):
            for name in b:
                if name == "status":
                    assert torch.equal(a[name], b[name] | flag)
                elif b[name] is not None:
                    assert torch.equal(a[name], b[name]), name
                else:
                    assert a[name] is None

    want = calls()
    assert (want[0]["status"] & tli.TLI_ROW_TIMEOUT == 0).all()
    torch.cuda.synchronize()
    runtime = ctypes.CDLL("libcudart.so.12")
    runtime.cudaMemset.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t]
    assert runtime.cudaMemset(error_word(v.ctx), 1, 4) == 0
    check(calls(), tli.TLI_ROW_TIMEOUT)
    check(calls(), tli.TLI_ROW_TIMEOUT)                                      # (it stays until it is reset)
    tli.tli_reset(v.ctx)
    check(calls(), 0)
