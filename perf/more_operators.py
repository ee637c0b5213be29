"""The losses of a training step over one of two vocabularies, as cases that can be timed and compared.

    loss            of rows of logits: cross entropy against a label, or the divergence from a teacher's top logits,
                    ids of either vocabulary carried through the id map
    loss_grad       its gradient with respect to the logits
    head_loss       the same loss from hidden rows and the output head's weight, the logits not kept
    head_loss_grad  its gradients with respect to the hidden rows and the weight

The softmax runs over the whole vocabulary, or (``shared``) over the ids that both vocabularies have.  A row none of
whose target ids takes part is left out: loss and gradient 0.  ``run`` computes a case in plain torch operations where
``own`` is false, and with this framework's calls where it is true.
"""
import math

import torch

own = False

_F32, _BF16 = "float32", "bfloat16"
_TYPES = {_F32: torch.float32, _BF16: torch.bfloat16}
_SIZE = {_F32: 4, _BF16: 2}
_LEFT_OUT = 128


def listed():
    # k = 0: labels; k > 0: a teacher's k largest logits.  ids: the vocabulary the target ids belong to.
    return [
        # scoring one token of a conversation against a 32 000-id vocabulary: latency is all
        {"name": "loss_one_row", "op": "loss", "N": 1, "V_t": 32000, "V_d": 32768, "f": 0.7, "side": "target",
         "ids": "target", "shared": False, "type": _F32, "k": 0, "tau": 1.0},
        # distilling a drafter with rows of an odd width on a target's top 20, over the ids it can draft
        {"name": "loss_distil_odd", "op": "loss", "N": 1500, "V_t": 128256, "V_d": 50257, "f": 0.3, "side": "drafter",
         "ids": "target", "shared": True, "type": _BF16, "k": 20, "tau": 0.9},
        # evaluating 4096 tokens over the widest vocabulary in 32 bits
        {"name": "loss_wide", "op": "loss", "N": 4096, "V_t": 256000, "V_d": 128256, "f": 0.55, "side": "target",
         "ids": "target", "shared": False, "type": _F32, "k": 0, "tau": 1.0},
        # an online update from the few positions of one verification
        {"name": "loss_grad_few", "op": "loss_grad", "N": 6, "V_t": 128256, "V_d": 32768, "f": 0.7, "side": "drafter",
         "ids": "drafter", "shared": False, "type": _F32, "k": 0, "tau": 1.0},
        # a distillation step of a drafter, 16-bit logits, softened on both sides
        {"name": "loss_grad_distil", "op": "loss_grad", "N": 2048, "V_t": 128256, "V_d": 49152, "f": 0.4,
         "side": "drafter", "ids": "target", "shared": True, "type": _BF16, "k": 32, "tau": 2.0},
        # a training step of 8192 tokens over a wide vocabulary
        {"name": "loss_grad_wide", "op": "loss_grad", "N": 8192, "V_t": 128256, "V_d": 49152, "f": 0.4,
         "side": "target", "ids": "target", "shared": False, "type": _BF16, "k": 0, "tau": 1.0},
        # one token's loss straight from its hidden row: the head's weight is read once
        {"name": "head_one_token", "op": "head_loss", "N": 1, "V_t": 32000, "V_d": 32768, "f": 0.7, "side": "target",
         "ids": "target", "shared": False, "H": 2048, "k": 0, "tau": 1.0},
        # a ragged batch labelled in the target's ids, most of which an odd drafter vocabulary lacks
        {"name": "head_ragged", "op": "head_loss", "N": 1111, "V_t": 128256, "V_d": 50257, "f": 0.3,
         "side": "drafter", "ids": "target", "shared": True, "H": 1000, "k": 0, "tau": 1.0},
        # the forward half of a training step
        {"name": "head_step", "op": "head_loss", "N": 8192, "V_t": 128256, "V_d": 49152, "f": 0.4, "side": "target",
         "ids": "target", "shared": False, "H": 2048, "k": 0, "tau": 1.0},
        # an online update of a drafter's head and hidden rows from a batch of 64 sequences
        {"name": "head_grad_few", "op": "head_loss_grad", "N": 64, "V_t": 152064, "V_d": 32000, "f": 0.85,
         "side": "drafter", "ids": "drafter", "shared": False, "H": 2048, "k": 0, "tau": 1.0},
        # distilling a drafter's head on a target's top 32
        {"name": "head_grad_distil", "op": "head_loss_grad", "N": 2000, "V_t": 128256, "V_d": 49152, "f": 0.4,
         "side": "drafter", "ids": "target", "shared": True, "H": 1024, "k": 32, "tau": 1.5},
        # the backward half of a training step
        {"name": "head_grad_step", "op": "head_loss_grad", "N": 8192, "V_t": 128256, "V_d": 49152, "f": 0.4,
         "side": "target", "ids": "target", "shared": False, "H": 2048, "k": 0, "tau": 1.0},
    ]


def _log_int(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["loss", "loss_grad", "head_loss", "head_loss_grad"])
    side = rng.choice(["target", "drafter"])
    V_t, V_d = _log_int(rng, 1000, 256000), _log_int(rng, 1000, 128256)
    V = V_t if side == "target" else V_d
    case = {"op": op, "V_t": V_t, "V_d": V_d, "f": round(rng.uniform(0.2, 0.9), 3), "side": side,
            "ids": rng.choice(["target", "drafter"]), "shared": side == "drafter" and rng.random() < 0.5,
            "k": rng.choice([0, 0, 1, 7, 32, rng.randint(2, 128)]), "tau": rng.choice([1.0, 1.0, 0.7, 2.0])}
    if op in ("loss", "loss_grad"):
        case["type"] = rng.choice([_F32, _BF16])
        case["N"] = _log_int(rng, 1, min(8192, 500_000_000 // V))
    else:
        case["H"] = 8 * _log_int(rng, 8, 512)
        case["N"] = _log_int(rng, 1, max(2, min(8192, 1_000_000_000_000 // (V * case["H"]))))
    return case


def _rows_of(case):
    return case["V_t"] if case["side"] == "target" else case["V_d"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    V_t, V_d, V, N, k = case["V_t"], case["V_d"], _rows_of(case), case["N"], case["k"]
    # drafter id -> target id, -1 outside the intersection, and the inverse
    mapped = min(max(1, round(case["f"] * V_d)), V_t, V_d)
    xs = torch.randperm(V_d, generator=g, device="cuda")[:mapped]
    ts = torch.randperm(V_t, generator=g, device="cuda")[:mapped]
    forth = torch.full((V_d,), -1, dtype=torch.int32, device="cuda")
    back = torch.full((V_t,), -1, dtype=torch.int32, device="cuda")
    forth[xs] = ts.int()
    back[ts] = xs.int()
    s = {"case": case, "forth": forth, "back": back, "teacher": None}
    V_ids = V_t if case["ids"] == "target" else V_d
    if k:
        # distinct ids all over the vocabulary, logits that fall off with the rank
        first = torch.randint(0, V_ids, (N, 1), generator=g, device="cuda")
        gaps = torch.randint(1, V_ids // k + 1, (N, k), generator=g, device="cuda")
        s["ids"] = ((first + gaps.cumsum(1)) % V_ids).int()
        rank = torch.arange(1, k + 1, device="cuda").float()
        noise = torch.empty(N, k, device="cuda").normal_(0.0, 0.3, generator=g)
        s["teacher"] = 12.0 - 1.5 * rank.log() + noise
    else:
        # low ids are the frequent ones in a vocabulary ordered by merges
        r = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
        s["ids"] = torch.exp(r * math.log(V_ids)).long().sub_(1).clamp_(0, V_ids - 1).int()
    s["temperature"] = None if case["tau"] == 1.0 else torch.full((N,), case["tau"], device="cuda")
    ids, on = _ids(s)
    if case["op"] in ("loss", "loss_grad"):
        # noise, and a student that has half learned what the targets are
        z = torch.empty(N, V, device="cuda").normal_(0.0, 2.0, generator=g)
        z.scatter_add_(1, ids, torch.where(on, 8.0, 0.0))
        s["logits"] = z.to(_TYPES[case["type"]])
    else:
        H = case["H"]
        s["weight"] = torch.empty(V, H, device="cuda").normal_(0.0, 2.0 / math.sqrt(H), generator=g).bfloat16()
        h = torch.empty(N, H, device="cuda").normal_(0.0, 1.0, generator=g)
        h += 2.0 * (s["weight"][ids[:, 0]].float() * on[:, :1])
        s["hidden"] = h.bfloat16()
    if case["op"].endswith("grad"):
        # the mean over a batch of weighted tokens, and what the forward call left
        s["grad_loss"] = torch.rand(N, generator=g, device="cuda").add_(0.5).div_(N)
        forward = _loss(s)
        s["stats"] = forward["stats"]
        if "hidden" in s:
            s["target_logits"] = forward["target_logits"]
    if own:
        from paper_2502_05202_b200 import tli
        s["v"] = tli.Verifier(V_t, V_d, forth.cpu().numpy())
    return s


def _ids(s):
    """The target ids in the rows' vocabulary [N, k], and which of them take part."""
    case = s["case"]
    ids = s["ids"].view(s["ids"].shape[0], -1).long()
    if case["ids"] != case["side"]:
        ids = (s["forth"] if case["ids"] == "drafter" else s["back"]).long()[ids]
    on = ids >= 0
    ids = ids.clamp(min=0)
    if case["shared"]:
        on &= s["forth"][ids] >= 0
    return ids, on


def _logits(s):
    """Logits of the ids that take part in 32 bits (-inf for the others), divided by nothing yet."""
    z = s["logits"].float() if "logits" in s else s["hidden"].float() @ s["weight"].float().t()
    return z.masked_fill(s["forth"] < 0, -math.inf) if s["case"]["shared"] else z


def _target(s, on):
    """Probabilities of the target ids [N, k] in 32 bits, 0 where one does not take part."""
    if s["teacher"] is None:
        return on.float()
    t = (s["teacher"] / s["case"]["tau"]).masked_fill(~on, -math.inf)
    w = torch.exp(t - t.amax(1, keepdim=True).clamp(min=-1e30))
    return w / w.sum(1, keepdim=True).clamp(min=1e-30)


def _loss(s):
    tau = s["case"]["tau"]
    ids, on = _ids(s)
    z = _logits(s)
    m = z.amax(1, keepdim=True)
    total = torch.exp((z - m) / tau).sum(1, keepdim=True)
    p = _target(s, on)
    at = z.gather(1, ids)
    terms = torch.where(p > 0, p * ((m - at) / tau + torch.where(p > 0, p, torch.ones_like(p)).log()), torch.zeros_like(p))
    row = on.any(1)
    out = {"loss": torch.where(row, total.log().squeeze(1) + terms.sum(1), torch.zeros_like(m[:, 0])),
           "stats": torch.cat((m, total), 1) * row.unsqueeze(1),
           "status": torch.where(row, 0, _LEFT_OUT).int()}
    if "hidden" in s:
        out["target_logits"] = at.masked_fill(~on, 0.0).view_as(s["ids"])
    return out


def _slope(s):
    """The gradient with respect to the logits in 32 bits."""
    tau = s["case"]["tau"]
    ids, on = _ids(s)
    z = _logits(s)
    g = (s["grad_loss"] / tau * on.any(1)).unsqueeze(1)
    m, total = s["stats"][:, :1], s["stats"][:, 1:]
    z.sub_(m).div_(tau).exp_().mul_(g / total.clamp(min=1e-30))
    return z.scatter_add_(1, ids, -g * _target(s, on))


def run(s):
    case = s["case"]
    op = case["op"]
    if own:
        from paper_2502_05202_b200 import tli
        sides = {"target": tli.TLI_SIDE_TARGET, "drafter": tli.TLI_SIDE_DRAFTER}
        v = s["v"]
        how = dict(teacher=s["teacher"], temperature=s["temperature"], side=sides[case["side"]],
                   ids_side=sides[case["ids"]], shared=case["shared"])
        if op == "loss":
            return v.loss(s["logits"], s["ids"], **how)
        if op == "loss_grad":
            # 32-bit rows over the whole vocabulary: the plain form works in the logits' own memory, and so does this call
            place = s["logits"] if case["type"] == _F32 and not case["shared"] else None
            return v.loss_grad(s["logits"], s["ids"], s["stats"], grad_loss=s["grad_loss"], out=place, **how)
        if op == "head_loss":
            return v.head_loss(s["hidden"], s["weight"], s["ids"], **how)
        out = v.head_loss_grad(s["hidden"], s["weight"], s["ids"], s["stats"], s["target_logits"],
                               grad_loss=s["grad_loss"], **how)
        return {"grad_hidden": out["grad_hidden"], "grad_weight": out["grad_weight"]}
    if op in ("loss", "head_loss"):
        return _loss(s)
    slope = _slope(s)
    if op == "loss_grad":
        return {"grad": slope.to(s["logits"].dtype)}
    return {"grad_hidden": (slope @ s["weight"].float()).bfloat16(),
            "grad_weight": (slope.t() @ s["hidden"].float()).bfloat16()}


def _share(case):
    """Expected share of the rows that take part, as prepare() draws them."""
    V_t, V_d = case["V_t"], case["V_d"]
    mapped = min(max(1, round(case["f"] * V_d)), V_t, V_d)
    if case["ids"] == case["side"] and not case["shared"]:
        return 1.0
    return 1.0 - (1.0 - mapped / (V_t if case["ids"] == "target" else V_d)) ** max(1, case["k"])


def work(case):
    N, V, k, share = case["N"], _rows_of(case), max(1, case["k"]), _share(case)
    small = N * k * (8 if case["k"] else 4) + 16 * N
    if case["op"] in ("loss", "loss_grad"):
        once = N * V * _SIZE[case["type"]]
        part = int(share * once)  # rows that are left out need not be read, but their gradient is written
        return {"bytes": part + small + (once if case["op"] == "loss_grad" else 0), "flops": 4 * int(share * N * V)}
    H = case["H"]
    one = 2 * int(share * N * V) * H
    matrices = 2 * V * H + 2 * int(share * N) * H
    if case["op"] == "head_loss":
        return {"bytes": matrices + small, "flops": one}
    return {"bytes": matrices + small + 2 * V * H + 2 * N * H, "flops": 3 * one}


def exact(case, seed):
    """From the definitions, row blocks in 64 bits: p against the softmax of the rows that take part."""
    s = prepare(case, seed)
    N, V, tau = case["N"], _rows_of(case), float(case["tau"])
    grads = case["op"].endswith("grad")
    head = "hidden" in s
    if head and (6 if grads else 2) * N * V * case["H"] > 1.4e13:
        return None
    table = None
    if case["ids"] != case["side"]:
        table = (s["forth"] if case["ids"] == "drafter" else s["back"]).tolist()
    shared = (s["forth"] >= 0).double().log() if case["shared"] else None  # 0 or -inf
    taking = set(torch.nonzero(s["forth"] >= 0).flatten().tolist()) if case["shared"] else None
    ids = s["ids"].reshape(N, -1).tolist()
    teacher = s["teacher"].double().tolist() if s["teacher"] is not None else [[0.0]] * N
    weight = s["weight"].double() if head else None
    loss, stats, status = torch.zeros(N, dtype=torch.float64), torch.zeros(N, 2, dtype=torch.float64), torch.zeros(N, dtype=torch.int32)
    targets = torch.zeros(N, len(ids[0]), dtype=torch.float64)
    slope_rows, dh, dw = [], [], 0.0
    block = max(1, min(N, 200_000_000 // V))
    for a in range(0, N, block):
        b = min(N, a + block)
        z = s["hidden"][a:b].double() @ weight.T if head else s["logits"][a:b].double()
        if shared is not None:
            z = z + shared
        lse = torch.logsumexp(z / tau, 1)
        top = z.max(1).values
        rows, cols, probs, out = [], [], [], torch.ones(b - a, dtype=torch.float64)
        for i in range(a, b):
            mine = [(j, (table[x] if table else x)) for j, x in enumerate(ids[i])]
            mine = [(j, x) for j, x in mine if x >= 0 and (taking is None or x in taking)]
            if not mine:
                out[i - a] = 0.0
                status[i] = _LEFT_OUT
                continue
            t = [teacher[i][j] / tau for j, _ in mine]
            most = max(t)
            total = sum(math.exp(x - most) for x in t)
            for (j, x), y in zip(mine, t):
                rows.append(i - a), cols.append((j, x)), probs.append(math.exp(y - most) / total)
        r = torch.tensor(rows, dtype=torch.long, device="cuda")
        c = torch.tensor([x for _, x in cols], dtype=torch.long, device="cuda")
        p = torch.tensor(probs, dtype=torch.float64, device="cuda")
        out = out.cuda()
        if grads:
            weigh = s["grad_loss"][a:b].double() * out / tau
            d = torch.softmax(z / tau, 1) * weigh[:, None]
            d.index_put_((r, c), -p * weigh[r], accumulate=True)
            if head:
                dh.append(d @ weight)
                dw = dw + d.T @ s["hidden"][a:b].double()
            else:
                slope_rows.append(d)
        else:
            at = z[r, c]
            each = torch.zeros(b - a, dtype=torch.float64, device="cuda")
            each.index_add_(0, r, p * (p.log() - at / tau + lse[r]))
            loss[a:b] = each.cpu()
            stats[a:b, 0] = (top * out).cpu()
            stats[a:b, 1] = (torch.exp(lse - top / tau) * out).cpu()
            targets[a + r.cpu(), torch.tensor([j for j, _ in cols], dtype=torch.long)] = at.cpu()
    if grads:
        return {"grad_hidden": torch.cat(dh), "grad_weight": dw} if head else {"grad": torch.cat(slope_rows)}
    result = {"loss": loss, "stats": stats, "status": status}
    if head:
        result["target_logits"] = targets.view(s["ids"].shape)
    return result
