"""The row and embedding calls at the ends of their ranges: small weights that decide, the most rows, offsets beyond 32 bits, a first call that
is captured."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2502_05202_b200 import tli

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def verifier(V):
    return tli.Verifier(V, 3, np.array([0, -1, V - 1], np.int32))


@pytest.mark.parametrize("V,k,bits,width", [(4096, 4000, 46.1, 0.3), (40001, 6000, 45.1, 3.0), (9001, 8999, 43.1, 0.3), (40001, 30000, 45.1, 0.3)])
def test_small_weights_decide(V, k, bits, width):
    """An id of weight 1, one of 1 - d and k - 2 small ones of 2 d in all or a little more: top-p 1/2 keeps two ids, one without the small ones."""
    z = (-bits - width * np.random.default_rng(k).random((1, 1, V))) * np.log(2.0)
    d = (k - 2) * 2.0 ** (-bits - min(width, 0.5)) / 2
    z[0, 0, 17], z[0, 0, 3001] = 0.0, -d
    assert d / 4 > 4e-12                                                     # of the mass, from the first id's to the border
    z = torch.from_numpy(z.astype(np.float32)).cuda()
    v = verifier(V)
    out = v.filter(z, torch.ones(1, device="cuda"), top_k=torch.full((1,), k, dtype=torch.int32, device="cuda"), top_p=torch.full((1,), 0.5, device="cuda"))
    assert torch.nonzero(out["logits"][0, 0] > -float("inf")).flatten().tolist() == [17, 3001]


@pytest.mark.parametrize("B,R", [(65535, 1), (13107, 5)])
@pytest.mark.parametrize("V", [37, 4500])
def test_the_most_rows(V, B, R):
    """Every row of 65 535 against a row of the same logits in a call of its own kind of size."""
    g = torch.Generator(device="cuda").manual_seed(V + R)
    base = torch.randn(64, 1, V, device="cuda", generator=g).bfloat16()
    which = torch.randint(0, 64, (B, R), device="cuda", generator=g)
    z = base[which.flatten(), 0].view(B, R, V)
    tau = torch.full((B,), 0.9, device="cuda")
    k, p = torch.full((B,), 30, dtype=torch.int32, device="cuda"), torch.full((B,), 0.8, device="cuda")
    u = torch.rand(B, R, device="cuda", generator=g)
    v = verifier(V)
    for ask in (dict(top_k=k, top_p=p), dict(top_p=p)):
        small = v.filter(base, tau[:64], **{n: x[:64] for n, x in ask.items()})["logits"][:, 0]
        out = v.sample(z, tau, u, **ask)
        assert (out["status"] == 0).all()
        assert (small[which.flatten()].gather(1, out["tokens"].view(-1, 1).long()) > -float("inf")).all()
        assert torch.equal(v.filter(z, tau, out=z.clone(), **ask)["logits"].view(-1, V), small[which.flatten()])


def test_offsets_beyond_32_bits():
    """4.4e9 elements of 16 bits, filtered in place: the first, the middle and the last rows."""
    V, B = 152064, 29000
    v = verifier(V)
    g = torch.Generator(device="cuda").manual_seed(1)
    base = (torch.randn(50, V, device="cuda", generator=g) * 3).bfloat16()
    z = base.repeat(B // 50, 1).view(B, 1, V)
    assert z.numel() > 2 ** 32
    tau, p = torch.ones(B, device="cuda"), torch.full((B,), 0.9, device="cuda")
    u = torch.rand(B, 1, device="cuda", generator=g)
    tokens = v.sample(z, tau, u, top_p=p)["tokens"]
    want = v.filter(base.view(50, 1, V), tau[:50], top_p=p[:50])["logits"][:, 0]
    v.filter(z, tau, top_p=p, out=z)
    for first in (0, 14100, B - 50):
        assert torch.equal(z[first:first + 50, 0], want)
        assert (want.gather(1, tokens[first:first + 50].long()) > -float("inf")).all()
    v.close()


def test_embedding_offsets_beyond_32_bits():
    """A table of 2.1e9 elements and 2.2e9 of rows, and the dense gradient of that table."""
    V, H, N = 262144, 8208, 270000
    assert V * H > 2 ** 31 and N * H > 2 ** 31
    v = verifier(V)
    table = torch.empty(V, H, dtype=torch.bfloat16, device="cuda")
    table.copy_((torch.arange(V, device="cuda") % 251).view(-1, 1).bfloat16().expand(V, H))
    ids = torch.randint(0, V, (N,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))
    ids[-3:] = torch.tensor([V - 1, 0, V - 1], device="cuda")
    rows = v.embed(ids, table)["rows"]
    want = (ids % 251).bfloat16()
    for c in (0, 4100, H - 1):
        assert torch.equal(rows[:, c], want)
    del table
    grad = v.embed_grad(ids, rows.fill_(1.0), dtype=torch.bfloat16)["grad"]
    counts = torch.bincount(ids.long(), minlength=V).bfloat16()
    for c in (0, 4100, H - 1):
        assert torch.equal(grad[:, c], counts)
    v.close()


def test_the_most_tokens():
    N, V = tli.TLI_MAX_TOKENS, 50257
    v = verifier(V)
    ids = torch.randint(0, V, (N,), dtype=torch.int32, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    ids[1000:900000] = 77
    grad = v.embed_grad(ids, torch.ones(1, 8, device="cuda").expand(N, 8))["grad"]
    counts = torch.bincount(ids.long(), minlength=V).float()                 # (sums of ones are exact in fp32 up to 2^24)
    assert torch.equal(grad, counts.view(-1, 1).expand(-1, 8))


FIRST = """
import sys
sys.path.insert(0, %r)
import numpy as np, torch
from paper_2502_05202_b200 import tli
v = tli.Verifier(5000, 4000, np.arange(4000, dtype=np.int32))
z, tau = torch.randn(3, 2, 5000, device="cuda"), torch.ones(3, device="cuda")
p, u = torch.full((3,), 0.97, device="cuda"), torch.rand(3, 2, device="cuda")
table, ids = torch.randn(5000, 64, device="cuda"), torch.arange(6, dtype=torch.int32, device="cuda")
torch.cuda.synchronize()
call = lambda: [v.sample(z, tau, u, top_p=p)["tokens"], v.filter(z, tau, top_p=p)["logits"], v.embed(ids, table)["rows"], v.embed_grad(ids, table[:6])["grad"]]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = call()
g.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, call()))
print("captured first")
"""


def test_a_first_call_may_be_captured():
    r = subprocess.run([sys.executable, "-c", FIRST % ROOT], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "captured first" in r.stdout, r.stdout + r.stderr
