"""The vocabulary-side operators of a decoding or training step, as cases that can be timed and compared.

    sample      one id per row of logits after temperature, top-k, top-p and min-p, from given uniforms
    filter      the same filters as masked logits (-inf outside the kept set), what a verification of drafts
                drawn under filters takes
    embed       rows of an embedding table for ids of either vocabulary, carried through the id map, times a scale
    embed_grad  the gradient of that lookup with respect to the table, every row of it written

``run`` computes a case in plain torch operations where ``own`` is false, and with this framework's calls where it
is true.  Ids are compared exactly, so the plain form of the row operators works in 64 bits: a kept set and an
inverse CDF have a border wherever one id ends and the next begins.
"""
import math

import numpy as np
import torch

own = False

_F32, _BF16 = "float32", "bfloat16"
_TYPES = {_F32: torch.float32, _BF16: torch.bfloat16}
_SIZE = {_F32: 4, _BF16: 2}

# What a server's batch mixes: (top_k, top_p, min_p) by sequence; 0, 1 and 0 are "off".
_MIXES = {
    "none": [(0, 1.0, 0.0)],
    "k": [(64, 1.0, 0.0)],
    "p": [(0, 0.9, 0.0)],
    "min_p": [(0, 1.0, 0.05)],
    "k_p": [(50, 0.9, 0.0)],
    "mixed": [(50, 1.0, 0.0), (0, 0.9, 0.0), (40, 0.95, 0.0), (0, 1.0, 0.05), (0, 1.0, 0.0), (1000, 0.99, 0.0),
              (20, 0.8, 0.1), (0, 0.99, 0.0)],
}
_TAUS = {"one": [1.0], "warm": [0.7], "mixed": [0.5, 0.8, 1.0, 1.2], "half_greedy": [0.0, 0.9]}


def listed():
    return [
        # the next token of a single conversation, one row of a 32 000-id target: latency is all
        {"name": "sample_one_row", "op": "sample", "side": "target", "B": 1, "R": 1, "V": 32000, "V_other": 32768,
         "f": 0.7, "type": _F32, "tau": "one", "mix": "k_p"},
        # drawing the drafts of 64 sequences, one drafter forward: 16-bit rows, only ids of the intersection count
        {"name": "sample_drafts", "op": "sample", "side": "drafter", "B": 64, "R": 1, "V": 32000, "V_other": 152064,
         "f": 0.85, "type": _BF16, "tau": "mixed", "mix": "mixed"},
        # every position of a verification batch of eight sequences under nucleus sampling
        {"name": "sample_nucleus", "op": "sample", "side": "target", "B": 8, "R": 6, "V": 128256, "V_other": 49152,
         "f": 0.4, "type": _BF16, "tau": "warm", "mix": "p"},
        # a large batch of 32-bit rows with every kind of request in it
        {"name": "sample_large", "op": "sample", "side": "target", "B": 64, "R": 5, "V": 256000, "V_other": 128256,
         "f": 0.55, "type": _F32, "tau": "one", "mix": "mixed"},
        # filtering the rows that verify five drafts of one sequence
        {"name": "filter_one_sequence", "op": "filter", "side": "target", "B": 1, "R": 6, "V": 32000, "V_other": 32768,
         "f": 0.7, "type": _F32, "tau": "one", "mix": "k_p"},
        # drafter rows of an odd width (no row but the first is aligned), half of the sequences at temperature 0
        {"name": "filter_drafter_odd", "op": "filter", "side": "drafter", "B": 32, "R": 16, "V": 50257,
         "V_other": 128256, "f": 0.3, "type": _BF16, "tau": "half_greedy", "mix": "mixed"},
        # the target rows of 64 sequences with eight drafts each
        {"name": "filter_target", "op": "filter", "side": "target", "B": 64, "R": 9, "V": 152064, "V_other": 32000,
         "f": 0.85, "type": _BF16, "tau": "mixed", "mix": "mixed"},
        # the verification forward's input rows: the last token and five drafts, drafter ids into the target's table
        {"name": "embed_decode", "op": "embed", "N": 48, "H": 2048, "ids": "drafter", "table": "target",
         "V_t": 128256, "V_d": 49152, "f": 0.4, "type": _BF16, "scale": 1.0},
        # a prefill: sixteen thousand prompt tokens of the target's own vocabulary, scaled by sqrt(H)
        {"name": "embed_prefill", "op": "embed", "N": 16384, "H": 4096, "ids": "target", "table": "target",
         "V_t": 152064, "V_d": 32000, "f": 0.85, "type": _BF16, "scale": 64.0},
        # a small fine-tuning step of a drafter: odd width, 32 bits throughout
        {"name": "grad_small", "op": "embed_grad", "N": 517, "H": 1000, "ids": "drafter", "table": "drafter",
         "V_t": 32000, "V_d": 32768, "f": 0.7, "type": _F32, "out": _F32, "scale": 1.0},
        # distilling a drafter on text in the target's ids: 16-bit gradients into the drafter's 32-bit master gradient
        {"name": "grad_distil", "op": "embed_grad", "N": 16384, "H": 2048, "ids": "target", "table": "drafter",
         "V_t": 128256, "V_d": 49152, "f": 0.4, "type": _BF16, "out": _F32, "scale": 1.0},
        # a training step over a wide vocabulary, gradient kept in 16 bits
        {"name": "grad_wide", "op": "embed_grad", "N": 32768, "H": 1024, "ids": "target", "table": "target",
         "V_t": 152064, "V_d": 32000, "f": 0.85, "type": _BF16, "out": _BF16, "scale": 32.0},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["sample", "filter", "embed", "embed_grad"])
    kind = rng.choice([_F32, _BF16])
    if op in ("sample", "filter"):
        most = 20_000_000 if op == "filter" else 40_000_000
        V = _log_int(rng, 1000, 256000)
        rows = _log_int(rng, 1, max(1, min(512, most // V)))
        R = rng.randint(1, min(9, rows))
        return {"op": op, "side": rng.choice(["target", "drafter"]), "B": max(1, rows // R), "R": R, "V": V,
                "V_other": _log_int(rng, 30000, 160000), "f": round(rng.uniform(0.1, 0.9), 3), "type": kind,
                "tau": rng.choice(sorted(_TAUS)), "mix": rng.choice(sorted(_MIXES))}
    case = {"op": op, "ids": rng.choice(["target", "drafter"]), "table": rng.choice(["target", "drafter"]),
            "V_t": _log_int(rng, 1000, 150000), "V_d": _log_int(rng, 1000, 60000), "f": round(rng.uniform(0.1, 0.6), 3),
            "type": kind, "scale": rng.choice([1.0, 0.125, 45.25]), "N": _log_int(rng, 1, 16384)}
    most = 60_000_000 if op == "embed" else 80_000_000
    V = case["V_t"] if case["table"] == "target" else case["V_d"]
    case["H"] = _log_int(rng, 64, max(65, min(4096, most // max(V, case["N"]))))
    if op == "embed_grad":
        case["out"] = rng.choice([_F32, _BF16])
    return case


def _sizes(case):
    """(V_t, V_d) of a case."""
    if case["op"] in ("sample", "filter"):
        return (case["V"], case["V_other"]) if case["side"] == "target" else (case["V_other"], case["V"])
    return case["V_t"], case["V_d"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    V_t, V_d = _sizes(case)
    # drafter id -> target id, -1 outside the intersection, and the inverse
    mapped = min(max(1, round(case["f"] * V_d)), V_t, V_d)
    xs = torch.randperm(V_d, generator=g, device="cuda")[:mapped]
    ts = torch.randperm(V_t, generator=g, device="cuda")[:mapped]
    forth = torch.full((V_d,), -1, dtype=torch.int32, device="cuda")
    back = torch.full((V_t,), -1, dtype=torch.int32, device="cuda")
    forth[xs] = ts.int()
    back[ts] = xs.int()
    s = {"case": case, "forth": forth, "back": back}
    if case["op"] in ("sample", "filter"):
        B, R, V = case["B"], case["R"], case["V"]
        # noise around a power law over the ranks, as the logits of a language model fall off
        rank = torch.randperm(V, generator=g, device="cuda").float().add_(1.0)
        z = torch.empty(B, R, V, device="cuda").normal_(0.0, 3.0, generator=g)
        s["logits"] = z.sub_(1.1 * rank.log()).to(_TYPES[case["type"]])
        taus, mixes = _TAUS[case["tau"]], _MIXES[case["mix"]]
        s["tau"] = torch.tensor([taus[(b // 2) % len(taus)] for b in range(B)], dtype=torch.float32, device="cuda")
        per = [mixes[b % len(mixes)] for b in range(B)]
        s["top_k"] = torch.tensor([m[0] for m in per], dtype=torch.int32, device="cuda")
        s["top_p"] = torch.tensor([m[1] for m in per], dtype=torch.float32, device="cuda")
        s["min_p"] = torch.tensor([m[2] for m in per], dtype=torch.float32, device="cuda")
        s["u"] = torch.randint(0, 1 << 24, (B, R), generator=g, device="cuda").float() * 2.0 ** -24
    else:
        N, H = case["N"], case["H"]
        V_ids = V_t if case["ids"] == "target" else V_d
        V_tab = V_t if case["table"] == "target" else V_d
        # low ids are the frequent ones in a vocabulary ordered by merges
        r = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
        s["ids"] = torch.exp(r * math.log(V_ids)).long().sub_(1).clamp_(0, V_ids - 1).int()
        if case["op"] == "embed":
            s["table"] = torch.empty(V_tab, H, device="cuda").normal_(0.0, 0.02, generator=g).to(_TYPES[case["type"]])
        else:
            s["grad"] = torch.empty(N, H, device="cuda").normal_(0.0, 1e-3, generator=g).to(_TYPES[case["type"]])
    if own:
        from paper_2502_05202_b200 import tli
        s["v"] = tli.Verifier(V_t, V_d, forth.cpu().numpy())
    return s


def _kept(s):
    """(weights, kept set) of every row, in id order, in 64 bits."""
    z = s["logits"].double()
    if s["case"]["side"] == "drafter":
        z = z.masked_fill(s["forth"] < 0, -math.inf)
    tau, k = s["tau"].double().view(-1, 1, 1), s["top_k"].view(-1, 1, 1)
    p, least = s["top_p"].double().view(-1, 1, 1), s["min_p"].double().view(-1, 1, 1)
    sorted_z, order = torch.sort(z, dim=-1, descending=True, stable=True)  # ties: lowest id first
    w = torch.exp((sorted_z - sorted_z[..., :1]) / torch.where(tau > 0, tau, torch.ones_like(tau)))
    place = torch.arange(z.shape[-1], device=z.device)
    first = place == 0
    keep = (sorted_z > -math.inf) & ((place < k) | (k <= 0))
    w = torch.where(keep, w, torch.zeros_like(w))
    mass = w.cumsum(-1)
    keep &= (mass - w < p * mass[..., -1:]) | (p >= 1) | first
    keep &= (w >= least) | first
    keep &= (tau > 0) | first
    w = torch.where(keep, w, torch.zeros_like(w))
    return torch.zeros_like(w).scatter_(-1, order, w), torch.zeros_like(keep).scatter_(-1, order, keep)


def _table_ids(s):
    case = s["case"]
    ids = s["ids"].long()
    if case["ids"] == case["table"]:
        return ids
    return (s["forth"] if case["ids"] == "drafter" else s["back"]).long()[ids]


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2502_05202_b200 import tli
        sides = {"target": tli.TLI_SIDE_TARGET, "drafter": tli.TLI_SIDE_DRAFTER}
        v = s["v"]
        if op == "sample":
            return v.sample(s["logits"], s["tau"], s["u"], side=sides[case["side"]], top_k=s["top_k"],
                            top_p=s["top_p"], min_p=s["min_p"])
        if op == "filter":
            return v.filter(s["logits"], s["tau"], side=sides[case["side"]], top_k=s["top_k"], top_p=s["top_p"],
                            min_p=s["min_p"])
        if op == "embed":
            return v.embed(s["ids"], s["table"], scale=case["scale"], ids_side=sides[case["ids"]],
                           table_side=sides[case["table"]])
        return v.embed_grad(s["ids"], s["grad"], scale=case["scale"], ids_side=sides[case["ids"]],
                            table_side=sides[case["table"]], dtype=_TYPES[case["out"]])
    if op == "sample":
        w, kept = _kept(s)
        c = w.cumsum(-1)
        total = c[..., -1:]
        token = (c <= s["u"].double().unsqueeze(-1) * total).sum(-1, keepdim=True)
        prob = w.gather(-1, token) / total
        return {"tokens": token.squeeze(-1).int(), "prob": prob.squeeze(-1).float(), "status": torch.zeros_like(s["u"]).int()}
    if op == "filter":
        _, kept = _kept(s)
        return {"logits": s["logits"].masked_fill(~kept, -math.inf), "status": torch.zeros_like(s["u"]).int()}
    ids = _table_ids(s)
    inside = ids >= 0
    if op == "embed":
        rows = s["table"][ids.clamp(min=0)].float() * case["scale"]
        rows = rows * inside.unsqueeze(-1)
        return {"rows": rows.to(s["table"].dtype), "table_ids": ids.int()}
    V_tab = s["forth"].numel() if case["table"] == "drafter" else s["back"].numel()
    g = s["grad"].float() * inside.unsqueeze(-1)
    total = torch.zeros(V_tab, case["H"], device="cuda").index_add_(0, ids.clamp(min=0), g)
    return {"grad": (total * case["scale"]).to(_TYPES[case["out"]])}


def _distinct(V, N):
    """Expected number of distinct ids among N drawn as prepare() draws them."""
    v = np.arange(1, V + 1, dtype=np.float64)
    p = np.log1p(1.0 / v) / math.log(V + 1)
    return float(-np.expm1(N * np.log1p(-np.minimum(p, 1 - 1e-12))).sum())


def work(case):
    size = _SIZE[case["type"]]
    if case["op"] in ("sample", "filter"):
        rows, V = case["B"] * case["R"], case["V"]
        once = rows * V * size
        if case["op"] == "sample":
            return {"bytes": once + rows * 16, "flops": rows * V}
        return {"bytes": 2 * once + rows * 4, "flops": rows * V}
    N, H = case["N"], case["H"]
    V_t, V_d = _sizes(case)
    V_ids, V_tab = (V_t if case["ids"] == "target" else V_d), (V_t if case["table"] == "target" else V_d)
    hit = 1.0 if case["ids"] == case["table"] else min(1.0, case["f"] * V_d / V_ids)
    distinct = hit * _distinct(V_ids, N)
    if case["op"] == "embed":
        return {"bytes": int(distinct * H * size) + N * H * size + 8 * N, "flops": N * H}
    return {"bytes": int(hit * N * H * size) + V_tab * H * _SIZE[case["out"]] + 4 * N, "flops": N * H}


def exact(case, seed):
    s = {k: v.double().cpu().numpy() if v.is_floating_point() else v.cpu().numpy()
         for k, v in prepare(case, seed).items() if isinstance(v, torch.Tensor)}
    if case["op"] in ("sample", "filter"):
        if s["logits"].size > 90_000_000:  # about a tenth of a microsecond an entry in the sort
            return None
        B, R, V = s["logits"].shape
        tokens, prob = np.zeros((B, R), np.int32), np.zeros((B, R))
        out = np.full((B, R, V), -np.inf)
        status = np.zeros((B, R), np.int32)
        for b in range(B):
            tau, k, p, least = s["tau"][b], int(s["top_k"][b]), s["top_p"][b], s["min_p"][b]
            for r in range(R):
                z = s["logits"][b, r]
                if case["side"] == "drafter":
                    z = np.where(s["forth"] >= 0, z, -np.inf)
                if tau == 0:
                    kept, w = np.array([np.argmax(z)]), np.ones(1)
                else:
                    order = np.argsort(-z, kind="stable")
                    n = int(np.count_nonzero(z > -np.inf))
                    if k > 0:
                        n = min(n, k)
                    order = order[:n]
                    w = np.exp((z[order] - z[order[0]]) / tau)
                    if p < 1:
                        c = np.cumsum(w)
                        n = min(n, int(np.searchsorted(c, p * c[-1], side="left")) + 1)
                    n = max(1, min(n, int(np.count_nonzero(w >= least))))
                    kept = np.sort(order[:n])
                    w = np.exp((z[kept] - z[order[0]]) / tau)
                out[b, r, kept] = s["logits"][b, r, kept]
                if case["op"] == "sample":
                    c = np.cumsum(w)
                    at = min(int(np.searchsorted(c, s["u"][b, r] * c[-1], side="right")), len(kept) - 1)
                    tokens[b, r], prob[b, r] = kept[at], w[at] / c[-1]
        if case["op"] == "sample":
            return {"tokens": tokens, "prob": prob, "status": status}
        return {"logits": out, "status": status}
    ids = s["ids"].astype(np.int64)
    if case["ids"] != case["table"]:
        ids = (s["forth"] if case["ids"] == "drafter" else s["back"])[ids].astype(np.int64)
    if case["op"] == "embed":
        rows = s["table"][np.maximum(ids, 0)] * case["scale"]
        rows[ids < 0] = 0.0
        return {"rows": rows, "table_ids": ids.astype(np.int32)}
    V_tab = len(s["forth"]) if case["table"] == "drafter" else len(s["back"])
    if V_tab * case["H"] > 160_000_000:
        return None
    total = np.zeros((V_tab, case["H"]))
    inside = np.flatnonzero(ids >= 0)
    if inside.size:
        inside = inside[np.argsort(ids[inside], kind="stable")]
        starts = np.flatnonzero(np.concatenate(([True], np.diff(ids[inside]) != 0)))
        total[ids[inside][starts]] = np.add.reduceat(s["grad"][inside], starts, axis=0) * case["scale"]
    return {"grad": total}
