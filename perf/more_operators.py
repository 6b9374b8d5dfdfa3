"""Cases of the rollout operators: inputs, plain forms, calls and exact values.

Four operators of a speculative rollout step, each with a plain form of elementary torch operations and the
framework's call:

  quantize  an LM head in bf16 -> 4-bit codes with a scale per group, and the values that they stand for
  logits    logits of a few tokens from such a head
  verify    drafted tokens against the target's distribution, from given uniforms; what is emitted, with its log-probs
  slots     block tables and the rows of new tokens in a paged store, from the requests' lengths

``own`` is False for the plain forms and True for the framework's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
RESIDUAL_FLOOR = 2.0 ** -30      # a residual with less mass than this is drawn from the target itself
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


# ------------------------------------------------------------------------------------------------ cases
def _verify(name, R, most, V, ttype, dtype, mode, temperature, **more):
    """mode: "dense" (draft distributions given), "lookup" (drafts without one), "greedy"."""
    return dict({"name": name, "op": "verify", "R": R, "most": most, "V": V, "target": ttype, "draft": dtype, "mode": mode,
                 "temperature": temperature}, **more)


def listed():
    return [
        # weight refresh of the smallest workload's head
        {"name": "quantize_small", "op": "quantize", "V": 4096, "d": 256, "group": 128},
        # weight refresh of the 7B-shaped head, once per training step
        {"name": "quantize_7b", "op": "quantize", "V": 152064, "d": 3584, "group": 128},
        # one decoded token, 7B-shaped head
        {"name": "logits_1_token", "op": "logits", "T": 1, "d": 3584, "V": 152064, "group": 128, "type": "f32"},
        # a small head and an odd batch: latency
        {"name": "logits_small", "op": "logits", "T": 5, "d": 640, "V": 5000, "group": 64, "type": "f32"},
        # one decoding step of a batch of requests, 32B-shaped head without its padded rows, fine groups
        {"name": "logits_16_32b", "op": "logits", "T": 16, "d": 5120, "V": 151643, "group": 32, "type": "bf16"},
        # a larger batch
        {"name": "logits_64_tokens", "op": "logits", "T": 64, "d": 3584, "V": 152064, "group": 128, "type": "f32"},
        # one request, four drafted tokens: latency
        _verify("verify_1_request", 1, 4, 152064, "f32", "f32", "dense", 1.0),
        # one step of a batch of requests
        _verify("verify_64", 64, 4, 152064, "bf16", "f32", "dense", 0.8),
        # a large batch, drafts copied from earlier responses, ragged
        _verify("verify_lookup", 192, 7, 152064, "bf16", "bf16", "lookup", 1.0),
        # evaluation without sampling
        _verify("verify_greedy", 33, 5, 151643, "f32", "f32", "greedy", 0.0),
        # one decoding step: a few drafted tokens each
        {"name": "slots_step", "op": "slots", "R": 64, "block": 16, "mean": 1024, "grow": 5, "fresh": False},
        # a whole store's responses placed at once, with those that they replace
        {"name": "slots_store", "op": "slots", "R": 4096, "block": 64, "mean": 300, "grow": 270, "fresh": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["quantize", "logits", "verify", "slots"])
    if op in ("quantize", "logits"):
        d, V = rng.choice([(256, 4096), (96, 1000), (640, 8200), (1024, 32768), (2080, 19001), (3584, 152064), (5120, 100003)])
        V = max(1, V - rng.randint(0, 300))
        group = rng.choice([32, 64, 128])
        if op == "quantize":
            return {"op": op, "V": V, "d": d, "group": group}
        return {"op": op, "T": _log_int(rng, 1, 64), "d": d, "V": V, "group": group, "type": rng.choice(sorted(TYPE))}
    if op == "verify":
        V = rng.choice([152064, 151643, 32000, _log_int(rng, 50, 20000)])
        most = rng.randint(0, 8)
        R = _log_int(rng, 1, min(2048, max(1, 150 * 10 ** 6 // (V * (most + 1)))))
        mode = rng.choice(["dense", "dense", "lookup", "greedy"])
        return {"op": op, "R": R, "most": most, "V": V, "target": rng.choice(sorted(TYPE)), "draft": rng.choice(sorted(TYPE)),
                "mode": mode, "temperature": 0.0 if mode == "greedy" else round(rng.uniform(0.5, 1.5), 3)}
    R = _log_int(rng, 1, 4096)
    mean = _log_int(rng, 1, min(4096, 1200000 // R))
    return {"op": op, "R": R, "block": rng.choice([1, 8, 16, 24, 64, 128]), "mean": mean, "grow": _log_int(rng, 1, mean), "fresh": rng.random() < 0.5}


def _positions(case):
    """Expected target rows looked at, from the shares of drafts that these inputs let pass."""
    rate = {"dense": 0.85, "lookup": 0.5, "greedy": 0.95}[case["mode"]]
    n = case["most"] if case["mode"] == "dense" else case["most"] / 2.0      # ragged lists are half as long on average
    return case["R"] * (1.0 - rate ** (n + 1)) / (1.0 - rate)


def work(case):
    op = case["op"]
    if op == "slots":
        tokens = case["R"] * case["grow"]
        return {"bytes": 12 * tokens + 20 * case["R"] + 8 * (tokens // case["block"] + 1), "flops": 4 * tokens}
    if op == "verify":
        rows = _positions(case)
        size = {"f32": 4, "bf16": 2}
        each = size[case["target"]] + (size[case["draft"]] if case["mode"] == "dense" else 0)
        return {"bytes": rows * case["V"] * each, "flops": 4 * rows * case["V"] * (2 if case["mode"] == "dense" else 1)}
    V, d = case["V"], case["d"]
    held = V * d // 2 + 2 * V * -(-d // case["group"])
    if op == "quantize":
        return {"bytes": 4 * V * d + held, "flops": 6 * V * d}
    T = case["T"]
    return {"bytes": held + 2 * T * d + (4 if case["type"] == "f32" else 2) * T * V, "flops": 2 * T * d * V}


# ----------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _head(g, V, d):
    """A head whose rows differ in size, with a few large weights, as trained ones have."""
    W = _normal(g, V, d) if V * d < 1 << 24 else torch.empty(V, d, dtype=torch.bfloat16, device=DEV).normal_(0.0, 1.0, generator=g)
    W *= (0.02 * torch.exp(0.3 * _normal(g, V, 1))).to(W.dtype)
    W[:, :: max(1, d // 5)] *= 4.0
    return W.to(torch.bfloat16)


def _prepare_verify(g, case, s):
    R, most, V, mode = case["R"], case["most"], case["V"], case["mode"]
    # model drafts are all of one length, the others of any up to the longest
    n = torch.full((R,), most, device=DEV) if mode == "dense" else torch.arange(R, device=DEV) % (most + 1)
    n = n[torch.randperm(R, generator=g, device=DEV)]
    s["cu"] = torch.zeros(R + 1, dtype=torch.int32, device=DEV)
    s["cu"][1:] = n.cumsum(0).int()
    D = int(s["cu"][-1])
    rows = D + R
    target = torch.empty(rows, V, dtype=TYPE[case["target"]], device=DEV)
    draft = torch.empty(D, V, dtype=TYPE[case["draft"]], device=DEV) if mode == "dense" else None
    ids = torch.empty(D, dtype=torch.int32, device=DEV)
    first = s["cu"][:-1].long()
    real = V - V // 300                                     # the last rows of a padded head are masked
    peaks = min(real, 24)
    request = torch.repeat_interleave(torch.arange(R, device=DEV), n.long() + 1)
    place = torch.arange(rows, device=DEV) - first[request] - request
    has_draft = place < n.long()[request]
    tau = case["temperature"] or 1.0
    for i in range(0, rows, 64):
        j = min(rows, i + 64)
        z = 1.8 * _normal(g, j - i, V)
        start = (real * _uniform(g, j - i, 1) ** 2).long()
        at = (start + (real // peaks) * torch.arange(peaks, device=DEV)) % real
        height = math.log(V) + 3.0 - 1.1 * torch.arange(peaks, device=DEV, dtype=torch.float32) ** 0.7
        z.scatter_(1, at, height + 0.7 * _normal(g, j - i, peaks))
        z[:, real:] = -math.inf
        target[i:j] = z.to(target.dtype)
        here = has_draft[i:j]
        k = (first[request[i:j]] + place[i:j])[here]
        if k.numel() == 0:
            continue
        near = z[here] + (0.15 if mode == "greedy" else 0.5) * _normal(g, int(here.sum()), V)
        if mode == "dense":
            draft[k] = near.to(draft.dtype)
            near = draft[k].float()
        if mode != "greedy":                                # a draw from the draft's distribution
            sharp = 4.0 if mode == "lookup" else 1.0        # a lookup proposes what the text has said before
            near = sharp * near / tau - torch.log(-torch.log(_uniform(g, *near.shape).clamp(1e-30, 1 - 2 ** -24)))
        ids[k] = near.argmax(dim=1).int()
    s["target"], s["draft"], s["ids"] = target, draft, ids
    s["u_accept"], s["u_sample"] = _uniform(g, max(D, 1))[:D], _uniform(g, R)
    s["token"] = torch.empty(rows, dtype=torch.int32, device=DEV)
    s["logp"], s["n_emitted"] = torch.empty(rows, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)


def _prepare_slots(g, case, s):
    R, block, mean = case["R"], case["block"], case["mean"]
    per = -(-(4 * mean + 2 * case["grow"]) // block) + 1    # widest table
    held_tokens = (mean * 2.0 * _uniform(g, R)).int().clamp(min=0)
    grow = torch.arange(R, device=DEV) * (2 * case["grow"] + 1) // R if case["fresh"] else torch.full((R,), case["grow"], device=DEV)
    grow = grow[torch.randperm(R, generator=g, device=DEV)].int()
    # what a step before has taken back (rejected drafts), or given up altogether (finished responses)
    length = torch.where(_uniform(g, R) < 0.9, (held_tokens - 3).clamp(min=0), torch.zeros_like(held_tokens))
    if case["fresh"]:
        length = torch.where(_uniform(g, R) < 0.7, torch.zeros_like(length), length)
    held = (held_tokens + block - 1) // block
    blocks = R * (2 * mean // block + 1) + R * (2 * case["grow"] // block + 2)
    order = torch.randperm(blocks, generator=g, device=DEV).int()
    before = held.cumsum(0) - held
    column = torch.arange(per, device=DEV)
    at = (before.long()[:, None] + column).clamp(max=blocks - 1)
    s["table"] = torch.where(column < held[:, None], order[at], torch.full_like(at, -1, dtype=torch.int32)).contiguous()
    taken = int(held.sum())
    s["free"] = torch.full((blocks,), -1, dtype=torch.int32, device=DEV)
    s["free"][: blocks - taken] = order[taken:]
    s["free_count"] = torch.tensor([blocks - taken], dtype=torch.int32, device=DEV)
    s["length"], s["grow"], s["held"] = length, grow, held.int()
    capacity = int(grow.sum()) + 64
    s["cu"], s["held_out"] = torch.empty(R + 1, dtype=torch.int32, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)
    s["free_count_out"], s["granted"] = torch.empty_like(s["free_count"]), torch.empty(R, dtype=torch.int32, device=DEV)
    s["slot"] = torch.full((capacity,), -7, dtype=torch.int64, device=DEV)
    s["position"] = torch.full((capacity,), -7, dtype=torch.int32, device=DEV)


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    s = {"case": case}
    if op == "verify":
        _prepare_verify(g, case, s)
        return s
    if op == "slots":
        _prepare_slots(g, case, s)
        return s
    V, d = case["V"], case["d"]
    groups = -(-d // case["group"])
    if op == "quantize":
        s["W"] = _head(g, V, d)
        s["codes"] = torch.empty(V, d // 8, dtype=torch.int32, device=DEV)
        s["scale"] = torch.empty(V, groups, dtype=torch.bfloat16, device=DEV)
        s["values"] = torch.empty_like(s["W"])
        return s
    s["codes"] = torch.empty(V, d // 8, dtype=torch.int32, device=DEV)
    s["codes"].random_(-(1 << 31), 1 << 31, generator=g)   # every digit: heads quantised elsewhere use -8 too
    fine = 2.0 ** -9 * (1.0 + torch.randint(0, 16, (V, groups), generator=g, device=DEV) / 16.0)       # five significant bits
    s["scale"] = (fine * 2.0 ** torch.randint(-1, 2, (V, groups), generator=g, device=DEV)).to(torch.bfloat16)
    s["H"] = _normal(g, case["T"], d).to(torch.bfloat16)
    s["logits"] = torch.empty(case["T"], V, dtype=TYPE[case["type"]], device=DEV)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_quantize(s):
    group = s["case"]["group"]
    V, d = s["W"].shape
    n = -(-d // group)
    w = torch.nn.functional.pad(s["W"], (0, n * group - d)).view(V, n, group).float()
    top = w.abs().amax(dim=2) / torch.full((V, n), 7.0, device=DEV)        # a tensor: by a number it would be a product
    mantissa = torch.frexp(top).mantissa
    power = top / torch.where(top > 0, mantissa, torch.ones_like(top))      # of two, exactly
    scale = torch.round(mantissa * 32.0) * 0.03125 * power
    unit = torch.where(scale > 0, scale, torch.ones_like(scale))[:, :, None]
    q = (w.abs() / unit + 0.5).floor_().mul_(torch.sign(w))
    values = (q * scale[:, :, None]).to(torch.bfloat16).view(V, n * group)[:, :d]
    return {"scale": scale.to(torch.bfloat16), "values": values}


def _plain_logits(s):
    codes, case = s["codes"], s["case"]
    V, d = codes.shape[0], case["d"]
    k = torch.arange(8, dtype=torch.int32, device=DEV)
    shift = 4 * (k // 2) + 16 * (k % 2)                    # even weights in a word's low half, odd ones in its high half
    q = ((codes[:, :, None] >> shift) & 15).sub_(8).view(V, d).float()
    q *= torch.repeat_interleave(s["scale"].float(), case["group"], dim=1)[:, :d]
    return {"logits": (s["H"].float() @ q.T).to(s["logits"].dtype)}


def _softmax64(z, tau):
    z = z.double() / tau
    e = torch.exp(z - z.amax(dim=1, keepdim=True))
    return e / e.sum(dim=1, keepdim=True)


def _plain_verify(s):
    """In 64 bits: acceptance is a comparison, and a draw is the place of a number among running sums of 10^5 terms."""
    case = s["case"]
    target, ids, cu = s["target"], s["ids"].long(), s["cu"].long()
    R, V = case["R"], target.shape[1]
    n = cu[1:] - cu[:-1]
    rows, D = target.shape[0], ids.numel()
    request = torch.repeat_interleave(torch.arange(R, device=DEV), n + 1, output_size=rows)
    place = torch.arange(rows, device=DEV) - cu[request] - request          # of a target row in its request
    of_draft = torch.repeat_interleave(torch.arange(R, device=DEV), n, output_size=D)
    checked = torch.arange(D, device=DEV) + of_draft                        # target row that a draft is checked against
    greedy = case["mode"] == "greedy"
    p = _softmax64(target, 1.0 if greedy else float(np.float32(case["temperature"])))
    best = target.argmax(dim=1)
    if greedy:
        accept = best[checked] == ids
    else:
        px = p[checked].gather(1, ids[:, None])[:, 0]
        if case["mode"] == "dense":
            q = _softmax64(s["draft"], float(np.float32(case["temperature"])))
            qx = q.gather(1, ids[:, None])[:, 0]
        else:
            q, qx = None, torch.ones_like(px)
        accept = s["u_accept"].double() * qx < px
    first = torch.full((R,), 1 << 30, dtype=torch.int64, device=DEV)
    spot = torch.arange(D, device=DEV) - cu[of_draft]
    first = torch.minimum(first.scatter_reduce(0, of_draft, torch.where(accept, 1 << 30, spot), "amin"), n)
    row = cu[:-1] + torch.arange(R, device=DEV) + first                     # the row that is drawn from
    rejected = first < n
    if greedy:
        drawn = best[row]
    else:
        mass = p[row]
        at = (cu[:-1] + first).clamp(max=max(D - 1, 0))                     # the rejected draft, where there is one
        if D > 0 and case["mode"] == "dense":
            left = torch.where(rejected[:, None], (mass - q[at]).clamp(min=0.0), mass)
            mass = torch.where(left.sum(dim=1, keepdim=True) > RESIDUAL_FLOOR, left, mass)
        elif D > 0:
            cut = rejected[:, None] & (torch.arange(V, device=DEV) == ids[at][:, None])
            left = torch.where(cut, torch.zeros_like(mass), mass)
            mass = torch.where(left.sum(dim=1, keepdim=True) > RESIDUAL_FLOOR, left, mass)
        running = mass.cumsum(dim=1)
        beyond = running > s["u_sample"].double()[:, None] * running[:, -1:]
        drawn = torch.where(beyond.any(dim=1), beyond.int().argmax(dim=1), (mass > 0).long().cumsum(dim=1).argmax(dim=1))
    token = torch.full((rows,), -1, dtype=torch.int64, device=DEV)
    token[checked] = ids
    token = torch.where(place < first[request], token, torch.where(place == first[request], drawn[request], -1))
    logp = torch.log(p.gather(1, token.clamp(min=0)[:, None])[:, 0])
    return {"token": token.int(), "logp": torch.where(token < 0, 0.0, logp).float(), "n_emitted": (first + 1).int()}


def _plain_slots(s):
    block = s["case"]["block"]
    length, grow, held = s["length"].long(), s["grow"].long(), s["held"].long()
    table, free, count = s["table"], s["free"], s["free_count"].long()
    R, per = table.shape
    need = (length + grow + block - 1) // block
    given, wanted = (held - need).clamp(min=0), (need - held).clamp(min=0)
    given_to, wanted_to = given.cumsum(0), wanted.cumsum(0)
    available = count + given_to[-1]
    granted = (wanted == 0) | (wanted_to <= available)
    held_out = torch.where(granted, need, held)
    left = available - torch.where(granted, wanted, 0).sum()
    # given blocks go on top of the stack, in the order of the requests and of their tables
    place = torch.arange(free.numel(), device=DEV)
    back = place - count
    owner = torch.searchsorted(given_to, back.clamp(min=0), right=True).clamp(max=R - 1)
    column = (need[owner] + back - (given_to - given)[owner]).clamp(0, per - 1)
    stack = torch.where((back >= 0) & (place < available), table[owner, column], free)
    # wanted blocks come off it
    cell = torch.arange(per, device=DEV)
    order = (wanted_to - wanted)[:, None] + cell - held[:, None]
    new = granted[:, None] & (cell >= held[:, None]) & (cell < need[:, None])
    table = torch.where(new, stack[(available - 1 - order).clamp(0, free.numel() - 1)], table)
    free = torch.where(place < left, stack, free)
    # rows of the new tokens
    cu = torch.nn.functional.pad(grow.cumsum(0), (1, 0))
    t = torch.arange(s["slot"].numel(), device=DEV)
    r = torch.searchsorted(cu, t, right=True).sub_(1).clamp(max=R - 1)
    pos = length[r] + t - cu[r]
    row = table[r, (pos // block).clamp(0, per - 1)].long() * block + pos % block
    here = t < cu[-1]
    slot = torch.where(here, torch.where(granted[r], row, -1), s["slot"])
    position = torch.where(here, pos.int(), s["position"])
    return {"table": table, "free": free, "free_count": left.int(), "held": held_out.int(), "granted": granted.int(), "cu": cu.int(),
            "slot": slot, "position": position}


PLAIN = {"quantize": _plain_quantize, "logits": _plain_logits, "verify": _plain_verify, "slots": _plain_slots}

# ------------------------------------------------------------------------------------ framework's calls
_contexts = {}


def _context():
    """The context that a program creates once per device and keeps."""
    from paper_2507_01663_b200 import Context
    if 0 not in _contexts:
        _contexts[0] = Context(0)
    return _contexts[0]


def _own(s):
    ctx, case = _context(), s["case"]
    op = case["op"]
    if op == "quantize":
        ctx.quantize_head(s["W"], s["codes"], s["scale"], group=case["group"], values=s["values"])
        return {"scale": s["scale"], "values": s["values"]}
    if op == "logits":
        ctx.quant_logits(s["H"], s["codes"], s["scale"], s["logits"], group=case["group"])
        return {"logits": s["logits"]}
    if op == "verify":
        ctx.draft_verify(s["target"], s["draft"], s["ids"], s["cu"], s["u_accept"], s["u_sample"], s["token"], s["n_emitted"],
                         logp=s["logp"], max_draft=case["most"], temperature=case["temperature"])
        return {"token": s["token"], "logp": s["logp"], "n_emitted": s["n_emitted"]}
    ctx.block_slots(s["length"], s["grow"], s["held"], s["table"], s["free"], s["free_count"], s["held_out"], s["free_count_out"],
                    s["cu"], s["slot"], block_size=case["block"], position=s["position"], granted=s["granted"])
    return {"table": s["table"], "free": s["free"], "free_count": s["free_count_out"], "held": s["held_out"], "granted": s["granted"],
            "cu": s["cu"], "slot": s["slot"], "position": s["position"]}


def run(state):
    return _own(state) if own else PLAIN[state["case"]["op"]](state)


# --------------------------------------------------------------------------------------- exact, 64 bits
def _exact_quantize(case, s):
    V, d, group = case["V"], case["d"], case["group"]
    n = -(-d // group)
    scale, values = torch.empty(V, n, dtype=torch.float64, device=DEV), torch.empty(V, d, dtype=torch.float64, device=DEV)
    for j in range(n):
        w = s["W"][:, j * group:(j + 1) * group].double()
        top = w.abs().max(dim=1).values / torch.full((V,), 7.0, dtype=torch.float64, device=DEV)
        lead = (top.view(torch.int64) & (0x7ff << 52)).view(torch.float64)      # the power of two not above
        step = torch.where(top > 0, lead / 16, 1.0)        # five significant bits; halves go to the even neighbour
        scale[:, j] = torch.round(top / step) * step
        unit = torch.where(scale[:, j] > 0, scale[:, j], 1.0)[:, None]
        below = torch.floor(w.abs() / unit)
        digit = below + (w.abs() - below * unit >= unit / 2).double()
        values[:, j * group:(j + 1) * group] = torch.where(w < 0, -digit, digit) * scale[:, j, None]
    return {"scale": scale, "values": values}


def _exact_logits(case, s):
    group, out = case["group"], []
    H = s["H"].double()
    for i in range(0, case["V"], 8192):
        words = s["codes"][i:i + 8192].long() & 0xffffffff
        total = torch.zeros(case["T"], words.shape[0], dtype=torch.float64, device=DEV)
        for k in range(8):                                 # digits of weight 8 j + k
            q = ((words // (1 << (4 * (k // 2) + 16 * (k % 2)))) % 16 - 8).double()
            at = torch.arange(k, case["d"], 8, device=DEV)
            total += H[:, at] @ (q * s["scale"][i:i + 8192].double()[:, at // group]).T
        out.append(total)
    return {"logits": torch.cat(out, dim=1)}


def _exact_verify(case, s):
    """Request by request, as the method is told: log-probs of what is emitted."""
    cu = s["cu"].tolist()
    ids, ua, us = s["ids"].tolist(), s["u_accept"].double().tolist(), s["u_sample"].double().tolist()
    tau = float(np.float32(case["temperature"])) or 1.0
    logp = torch.zeros(s["target"].shape[0], dtype=torch.float64, device=DEV)
    for r in range(case["R"]):
        base = cu[r] + r
        for i in range(cu[r + 1] - cu[r] + 1):
            z = s["target"][base + i].double() / tau
            lp = z - torch.logsumexp(z, dim=0)
            x = ids[cu[r] + i] if i < cu[r + 1] - cu[r] else None
            keep = None
            if case["mode"] == "greedy":
                y = int(z.argmax())
                accepted = x == y
            else:
                prob = torch.exp(lp)
                accepted = False
                if x is not None:
                    if case["mode"] == "dense":
                        zq = s["draft"][cu[r] + i].double() / tau
                        other = torch.exp(zq - torch.logsumexp(zq, dim=0))
                    else:
                        other = torch.zeros_like(prob)
                        other[x] = 1.0
                    accepted = ua[cu[r] + i] * float(other[x]) < float(prob[x])
                    keep = torch.relu(prob - other)
                    if case["mode"] == "lookup":
                        keep = torch.where(other > 0, 0.0, prob)
                if not accepted:
                    mass = prob if keep is None or float(keep.sum()) <= RESIDUAL_FLOOR else keep
                    run_to = torch.cumsum(mass, dim=0)
                    y = min(int(torch.searchsorted(run_to, us[r] * run_to[-1:], right=True)), case["V"] - 1)
            if accepted:
                logp[base + i] = lp[x]
                continue
            logp[base + i] = lp[y]
            break
    return {"logp": logp}


def exact(case, seed):
    if case["op"] == "slots":
        return None                                        # whole numbers
    s = prepare(case, seed)
    return {"quantize": _exact_quantize, "logits": _exact_logits, "verify": _exact_verify}[case["op"]](case, s)
