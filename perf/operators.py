"""Cases of the distillation and preference operators: inputs, plain forms, calls and exact values.

Five operators of the post-training path, each with a plain form of elementary torch operations and the
framework's call:

  score   student log-probs of K listed vocabulary ids per token (LM head, log-softmax, pick)
  grad    its gradient through the head: d_hidden and, unless the head is frozen, d_W
  loss    divergence between a teacher's and the student's log-probs of those ids, with its gradient
  update  score, loss and grad of one packed micro-batch as one step
  pairs   preference loss over pairs of packed sequences, with the gradient per token

``own`` is False for the plain forms and True for the framework's calls.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TAIL_FLOOR = 2.0 ** -16      # smallest mass of the tail outcome (support "tail")
DIVERGENCE = {"forward": 0, "reverse": 1}
SUPPORT = {"raw": 0, "renorm": 1, "tail": 2}
KIND = {"logistic": 0, "squared": 1, "hinge": 2}


# ------------------------------------------------------------------------------------------------ cases
def _head(name, op, T, d, V, K, **more):
    return dict({"name": name, "op": op, "T": T, "d": d, "V": V, "K": K}, **more)


def listed():
    return [
        # one generated token scored against a short list of alternatives (7B-shaped head)
        _head("score_1_token", "score", 1, 3584, 152064, 20),
        # one decoding step of a batch of requests
        _head("score_64_tokens", "score", 64, 3584, 152064, 20),
        # a training micro-batch against a teacher's top 64
        _head("score_7b", "score", 8192, 3584, 152064, 64),
        # launch-bound: the smallest workload's head and about its token count
        _head("grad_small", "grad", 1195, 256, 4096, 16, head=True),
        # an ordinary micro-batch, odd token count and list length
        _head("grad_7b", "grad", 4001, 3584, 152064, 50, head=True),
        # one streamed micro-batch of 32768 tokens, classic distillation at temperature 2
        {"name": "loss_micro", "op": "loss", "T": 32768, "K": 64, "B": 40, "divergence": "forward",
         "support": "renorm", "temperature": 2.0, "agg": 0},
        # a whole store at once, odd list length: on-policy distillation with a tail outcome
        {"name": "loss_store", "op": "loss", "T": 1106674, "K": 50, "B": 512, "divergence": "reverse",
         "support": "tail", "temperature": 1.0, "agg": 1},
        _head("update_small", "update", 1195, 256, 4096, 16, head=True, B=32, divergence="reverse", support="tail",
              temperature=1.0, agg=1),
        _head("update_7b", "update", 8192, 3584, 152064, 64, head=True, B=11, divergence="forward", support="renorm",
              temperature=1.0, agg=0),
        # 32B-shaped head kept frozen (adapters below it are trained)
        _head("update_32b_frozen", "update", 4100, 5120, 152064, 32, head=False, B=7, divergence="forward",
              support="renorm", temperature=1.5, agg=0),
        # one preference batch: 64 prompts, a chosen and a rejected response each
        {"name": "pairs_64", "op": "pairs", "P": 64, "mean_len": 2161, "kind": "logistic", "ref": True, "norm": False,
         "beta": 0.1, "eps": 0.0, "margin": 0.0, "nll": 0.0, "halves": False},
        # a whole epoch's pairs at once, length-normalised and reference-free with a margin
        {"name": "pairs_store", "op": "pairs", "P": 24576, "mean_len": 1024, "kind": "logistic", "ref": False, "norm": True,
         "beta": 2.0, "eps": 0.1, "margin": 1.0, "nll": 0.2, "halves": True},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "grad", "loss", "update", "pairs"])
    if op == "pairs":
        P = _log_int(rng, 1, 24576)
        return {"op": op, "P": P, "mean_len": _log_int(rng, 4, min(2048, 24576 * 1024 // P)),
                "kind": rng.choice(sorted(KIND)), "ref": rng.random() < 0.7, "norm": rng.random() < 0.5,
                "beta": round(rng.uniform(0.05, 2.0), 3), "eps": round(rng.uniform(0.0, 0.3), 3),
                "margin": round(rng.uniform(0.0, 1.5), 3), "nll": round(rng.choice([0.0, rng.uniform(0.05, 1.0)]), 3),
                "halves": rng.random() < 0.5}
    divergence, support = rng.choice(sorted(DIVERGENCE)), rng.choice(sorted(SUPPORT))
    more = {"divergence": divergence, "support": support, "agg": rng.randint(0, 1),
            "temperature": round(rng.uniform(0.5, 4.0), 3) if support == "renorm" else 1.0}
    K = _log_int(rng, 2 if support == "renorm" else 1, 256)      # one slot, renormalised, is always certain
    if op == "loss":
        T = _log_int(rng, 1, 1106674 * 50 // K)
        return dict({"op": op, "T": T, "K": K, "B": max(1, min(T, _log_int(rng, 1, 4096)))}, **more)
    d, V = rng.choice([(256, 4096), (384, 4104), (640, 8200), (1024, 32768), (3584, 152064), (3584, 152064), (5120, 152064)])
    top = min(8192, 8192 * 3584 * 152064 // (d * V))
    T = _log_int(rng, 1, top)
    if op == "score":
        return {"op": op, "T": T, "d": d, "V": V - rng.randint(0, 7), "K": K}
    if op == "grad":
        return {"op": op, "T": T, "d": d, "V": V, "K": K, "head": rng.random() < 0.7}
    return dict({"op": op, "T": T, "d": d, "V": V, "K": K, "head": rng.random() < 0.7, "B": max(1, min(T, _log_int(rng, 1, 512)))},
                **more)


def work(case):
    op = case["op"]
    if op == "pairs":
        T = 2 * case["P"] * case["mean_len"]
        return {"bytes": (4 + 4 * case["ref"] + 4) * T + 16 * case["P"], "flops": 4 * T}
    T, K = case["T"], case["K"]
    if op == "loss":
        return {"bytes": 12 * T * K + 4 * T, "flops": 12 * T * K}
    d, V = case["d"], case["V"]
    product = 2 * T * d * V
    if op == "score":
        return {"bytes": 2 * T * d + 2 * V * d + 8 * T * K + 8 * T, "flops": product}
    products = 3 if case["head"] else 2      # logits, d_hidden and, with a trained head, d_W
    moved = 4 * T * d + 2 * V * d * (2 if case["head"] else 1) + 8 * T * K
    if op == "update":
        moved += 8 * T * K + 8 * T
    return {"bytes": moved, "flops": products * product}


# ----------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 2654435761 % (1 << 62))
    return g


def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _uniform(g, *shape):
    return torch.rand(*shape, generator=g, device=DEV)


def _sequences(g, n, total):
    """cu_seqlens of ``n`` sequences of uneven length that hold ``total`` tokens."""
    cut = (_uniform(g, n - 1) * (total + 1)).long().clamp(max=total).sort().values
    cu = torch.zeros(n + 1, dtype=torch.int32, device=DEV)
    cu[1:n] = cut.int()
    cu[n] = total
    return cu


def _teacher(g, T, K):
    """Log-probs of a teacher's K best ids: steeply falling scores, about nine tenths of the mass.  Some
    lists are shorter than K (their last slots are absent) and a few are empty."""
    rank = torch.arange(K, device=DEV, dtype=torch.float32)
    score = -(0.5 + 2.0 * _uniform(g, T, 1)) * torch.log1p(rank) + 0.3 * _normal(g, T, K)
    mass = 0.8 + 0.18 * _uniform(g, T, 1)
    logp = torch.log_softmax(score, dim=1) + torch.log(mass)
    logp = logp.sort(dim=1, descending=True).values
    short = _uniform(g, T, 1) < (0.05 if T >= 16 else 0.0)      # a handful of tokens have whole lists
    kept = (_uniform(g, T, 1) * (K + 1)).floor()
    return torch.where(short & (rank >= kept), torch.full_like(logp, -math.inf), logp), short, kept, rank


def _model(g, T, d, V, K):
    """Hidden rows, a head and a teacher's lists.  A row leans towards the first few ids of its list, as the
    hidden state of a trained model does, so that the listed ids hold much of the student's mass."""
    W = torch.empty(V, d, dtype=torch.bfloat16, device=DEV).normal_(0.0, 0.02, generator=g)
    ids = (V * _uniform(g, T, K) ** 2).to(torch.int32).clamp(max=V - 1)     # frequent ids come first
    logp, short, kept, rank = _teacher(g, T, K)
    lean = min(K, 4)
    height = math.log(V) + 0.5 - 1.5 * torch.log1p(rank[:lean]) + 0.5 * _normal(g, T, lean)
    pull = (W[ids[:, :lean].long()].float() * height[:, :, None]).sum(dim=1) / (0.0004 * d)
    H = (_normal(g, T, d) + pull).to(torch.bfloat16)
    ids = torch.where(short & (rank >= kept), torch.full_like(ids, -1), ids).contiguous()
    return H, W, ids, logp.contiguous()


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    s = {"case": case}
    if op == "pairs":
        P = case["P"]
        T = 2 * P * case["mean_len"]
        s["cu"] = _sequences(g, 2 * P, T)
        s["logp"] = -_uniform(g, T) * 2.0 - 0.05
        s["ref"] = s["logp"] + 0.1 * _normal(g, T) if case["ref"] else None
        s["dlogp"] = torch.empty(T, device=DEV)
        s["pair_loss"], s["score"] = torch.empty(P, device=DEV), torch.empty(2 * P, device=DEV)
        s["out"] = torch.zeros(32, dtype=torch.uint8, device=DEV)
        return s
    T, K = case["T"], case["K"]
    if op == "loss":
        s["teacher"] = _teacher(g, T, K)[0].contiguous()
        noisy = s["teacher"].clamp(min=-20.0) + 0.5 * _normal(g, T, K)
        s["cand_logp"] = (noisy - torch.logsumexp(noisy, dim=1, keepdim=True)
                          + torch.log(0.6 + 0.35 * _uniform(g, T, 1))).contiguous()
    else:
        s["H"], s["W"], s["ids"], s["teacher"] = _model(g, T, case["d"], case["V"], K)
        s["cand_logp"] = torch.empty(T, K, device=DEV)
        s["lse"], s["entropy"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    if op == "grad":
        z_lse = []
        for rows in s["H"].split(1024):             # a forward pass has left lse behind
            z_lse.append(torch.logsumexp((rows @ s["W"].T).float(), dim=1))
        s["lse"] = torch.cat(z_lse)
        s["dcand"] = (_normal(g, T, K) / T).contiguous()
    else:
        s["dcand"] = torch.empty(T, K, device=DEV)
    if op in ("grad", "update"):
        s["d_hidden"] = torch.empty_like(s["H"])
        s["d_W"] = torch.empty_like(s["W"]) if case["head"] else None
    if op in ("loss", "update"):
        s["cu"] = _sequences(g, case["B"], T)
        s["token_loss"] = torch.empty(T, device=DEV)
        s["out"] = torch.zeros(24, dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_head(s):
    """fp32 logits, logsumexp and listed log-probs."""
    z = s["H"].float() @ s["W"].float().T
    lse = torch.logsumexp(z, dim=1)
    ids = s["ids"].long()
    lq = z.gather(1, ids.clamp(min=0)) - lse[:, None]
    return z, lse, torch.where(ids < 0, torch.full_like(lq, -math.inf), lq)


def _plain_head_gradient(s, z, lse, dcand):
    ids = s["ids"].long()
    grad = torch.where(ids < 0, torch.zeros_like(dcand), dcand)
    dz = (z - lse[:, None]).exp_().mul_(-grad.sum(dim=1, keepdim=True))
    dz.scatter_add_(1, ids.clamp(min=0), grad)
    dH = (dz @ s["W"].float()).to(torch.bfloat16)
    dW = (dz.T @ s["H"].float()).to(torch.bfloat16) if s["case"]["head"] else None
    return dH, dW


def _plain_divergence(case, lt, lq):
    """Per-token divergence and its gradient in the student's log-probs; absent slots take no part.  In 64
    bits: the tail's mass is what is left of 1, and a divergence is a difference of near terms."""
    here = lt > -math.inf
    lt, lq = lt.double(), lq.double()
    zero = torch.zeros_like(lq)
    forward = case["divergence"] == "forward"
    if case["support"] == "renorm":
        tau = case["temperature"]
        none = ~here.any(dim=1, keepdim=True)
        la = (lt / tau) - torch.logsumexp(torch.where(none, zero, lt / tau), dim=1, keepdim=True)
        lb = torch.where(here, lq / tau, zero - math.inf)
        lb = lb - torch.logsumexp(torch.where(none, zero, lb), dim=1, keepdim=True)
        a, b = torch.where(here, la.exp(), zero), torch.where(here, lb.exp(), zero)
        gap = torch.where(here, la - lb, zero)
        if forward:
            return tau * tau * (a * gap).sum(dim=1), tau * (b - a)
        mean = (b * -gap).sum(dim=1, keepdim=True)
        return (tau * tau * mean).squeeze(1), tau * b * (-gap - mean)
    p, q = torch.where(here, lt.exp(), zero), torch.where(here, lq.exp(), zero)
    gap = torch.where(here, lt - lq, zero)
    loss = (p * gap).sum(dim=1) if forward else (q * -gap).sum(dim=1)
    grad = -p if forward else q * (1.0 - gap)
    if case["support"] == "tail":
        p_left, q_left = 1.0 - p.sum(dim=1, keepdim=True), 1.0 - q.sum(dim=1, keepdim=True)
        pr, qr = p_left.clamp(min=TAIL_FLOOR), q_left.clamp(min=TAIL_FLOOR)
        free = q_left > TAIL_FLOOR
        ratio = torch.log(pr / qr)
        if forward:
            loss = loss + (pr * ratio).squeeze(1)
            grad = grad + torch.where(free, pr * q / qr, zero)
        else:
            loss = loss - (qr * ratio).squeeze(1)
            grad = grad + torch.where(free, q * (ratio - 1.0), zero)
    return loss, torch.where(here, grad, zero)


def _token_weight(case, cu, T):
    """Weight of every token in the mean, in 64 bits."""
    if case["agg"] == 1:
        return torch.full((T,), 1.0 / T, dtype=torch.float64, device=DEV)
    lengths = (cu[1:] - cu[:-1]).long()
    return torch.repeat_interleave(1.0 / (lengths.double() * lengths.numel()), lengths)


def _plain_loss(s, lq):
    case, lt = s["case"], s["teacher"]
    weight = _token_weight(case, s["cu"], lt.shape[0])
    token, grad = _plain_divergence(case, lt, lq)
    here = lt > -math.inf
    zero = torch.zeros((), dtype=torch.float64, device=DEV)
    record = torch.stack([(weight * token).sum(), torch.where(here, lt.double().exp(), zero).sum(dim=1).mean(),
                          torch.where(here, lq.double().exp(), zero).sum(dim=1).mean()])
    return record.float(), token.float(), (weight[:, None] * grad).float()


def _plain_pairs(s):
    """Sequence sums in 64 bits (thousands of terms that nearly cancel between the two responses)."""
    case, cu = s["case"], s["cu"]
    P = case["P"]
    lengths = (cu[1:] - cu[:-1]).long()
    seq = torch.repeat_interleave(torch.arange(2 * P, device=DEV), lengths)
    term = s["logp"].double() if s["ref"] is None else s["logp"].double() - s["ref"].double()
    zero = torch.zeros(2 * P, dtype=torch.float64, device=DEV)
    S, L = zero.index_add(0, seq, term), zero.index_add(0, seq, s["logp"].double())
    per = 1.0 / lengths.clamp(min=1).double()
    share = per if case["norm"] else torch.ones_like(per)
    score = case["beta"] * S * share
    first = torch.arange(P, device=DEV) * (1 if case["halves"] else 2)
    second = first + (P if case["halves"] else 1)
    x = score[first] - score[second] - case["margin"]
    if case["kind"] == "logistic":
        pair = torch.log1p(torch.exp(-x.abs())) + (-x).clamp(min=0.0) + case["eps"] * x
        slope = case["eps"] - torch.sigmoid(-x)
    elif case["kind"] == "squared":
        pair, slope = ((x - 0.5) / case["beta"]) ** 2, 2.0 * (x - 0.5) / case["beta"] ** 2
    else:
        pair, slope = (1.0 - x).clamp(min=0.0), -(x < 1.0).double()
    nll = -L[first] * per[first]
    whole = pair + case["nll"] * nll
    coef = torch.zeros_like(score)
    coef[first] = (slope * case["beta"] * share[first] - case["nll"] * per[first]) / P
    coef[second] = -(slope * case["beta"] * share[second]) / P
    better = (score[first] > score[second]).double()
    record = torch.stack([whole.mean(), pair.mean(), nll.mean(), better.mean(), score[first].mean(), score[second].mean()])
    return {"record": record.float(), "pair_loss": whole.float(), "score": score.float(), "dlogp": coef.float()[seq]}


def _plain(s):
    op = s["case"]["op"]
    if op == "pairs":
        return _plain_pairs(s)
    if op == "loss":
        record, token, grad = _plain_loss(s, s["cand_logp"])
        return {"record": record, "token_loss": token, "dcand": grad}
    if op == "grad":
        z = s["H"].float() @ s["W"].float().T
        dH, dW = _plain_head_gradient(s, z, s["lse"], s["dcand"])
        return {"d_hidden": dH, "d_W": dW}
    z, lse, lq = _plain_head(s)
    if op == "score":
        entropy = lse - ((z - lse[:, None]).exp_() * z).sum(dim=1)
        return {"cand_logp": lq, "lse": lse, "entropy": entropy}
    record, token, grad = _plain_loss(s, lq)
    dH, dW = _plain_head_gradient(s, z, lse, grad)
    return {"cand_logp": lq, "lse": lse, "record": record, "token_loss": token, "dcand": grad, "d_hidden": dH, "d_W": dW}


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
    if op == "pairs":
        ctx.preference_loss(s["logp"], s["ref"], s["cu"], s["out"], pair_loss=s["pair_loss"], seq_score=s["score"],
                            dlogp=s["dlogp"], kind=KIND[case["kind"]], beta=case["beta"], label_smoothing=case["eps"],
                            margin=case["margin"], nll_coef=case["nll"], length_norm=case["norm"],
                            pair_layout=int(case["halves"]))
        return {"record": s["out"].view(torch.float32)[:6], "pair_loss": s["pair_loss"], "score": s["score"],
                "dlogp": s["dlogp"]}
    if op == "score":
        ctx.candidate_logprob(s["H"], s["W"], s["ids"], s["cand_logp"], entropy=s["entropy"], lse=s["lse"])
        return {"cand_logp": s["cand_logp"], "lse": s["lse"], "entropy": s["entropy"]}
    if op == "grad":
        ctx.candidate_logprob_backward(s["H"], s["W"], s["ids"], s["lse"], s["dcand"], s["d_hidden"], s["d_W"])
        return {"d_hidden": s["d_hidden"], "d_W": s["d_W"]}
    how = {"divergence": DIVERGENCE[case["divergence"]], "support": SUPPORT[case["support"]],
           "temperature": case["temperature"], "agg_mode": case["agg"]}
    if op == "loss":
        ctx.distill_loss(s["cand_logp"], s["teacher"], s["cu"], s["out"], token_loss=s["token_loss"], dcand=s["dcand"], **how)
        return {"record": s["out"].view(torch.float32)[:3], "token_loss": s["token_loss"], "dcand": s["dcand"]}
    ctx.distill_update(s["H"], s["W"], s["ids"], s["teacher"], s["cu"], s["out"], s["cand_logp"], s["lse"], s["d_hidden"],
                       s["d_W"], token_loss=s["token_loss"], dcand=s["dcand"], **how)
    return {"cand_logp": s["cand_logp"], "lse": s["lse"], "record": s["out"].view(torch.float32)[:3],
            "token_loss": s["token_loss"], "dcand": s["dcand"], "d_hidden": s["d_hidden"], "d_W": s["d_W"]}


def run(state):
    return _own(state) if own else _plain(state)


# --------------------------------------------------------------------------------------- exact, 64 bits
def _exact_rows(lt, lq, case):
    """The divergences written out slot by slot from their definitions: sums over the present slots (and the
    tail), the gradient by the chain rule.  lt, lq: float64 [rows, K] on the GPU."""
    on = (lt != -math.inf).double()
    lt, lq = torch.where(on > 0, lt, 0.0), torch.where(on > 0, lq, 0.0)
    if case["support"] == "renorm":
        t = case["temperature"]
        ea, eb = on * torch.exp(lt / t), on * torch.exp(lq / t)
        za, zb = ea.sum(1, keepdim=True), eb.sum(1, keepdim=True)
        full = za > 0
        za, zb = torch.where(full, za, 1.0), torch.where(full, zb, 1.0)
        a, b = ea / za, eb / zb
        d = on * ((lt - lq) / t - torch.log(za / zb))                    # log a - log b
        if case["divergence"] == "forward":
            return t * t * (a * d).sum(1), t * (b - a)
        r = -(b * d).sum(1, keepdim=True)
        return t * t * r[:, 0], t * b * (-d - r)
    p, q = on * torch.exp(lt), on * torch.exp(lq)
    if case["divergence"] == "forward":
        loss, outer, dtail = (p * (lt - lq)).sum(1), -p, None
    else:
        loss, outer, dtail = (q * (lq - lt)).sum(1), q * (lq - lt + 1.0), None
    if case["support"] == "tail":
        a, b = 1.0 - p.sum(1), 1.0 - q.sum(1)
        a_c, b_c = torch.where(a > TAIL_FLOOR, a, TAIL_FLOOR), torch.where(b > TAIL_FLOOR, b, TAIL_FLOOR)
        if case["divergence"] == "forward":
            loss = loss + a_c * (torch.log(a_c) - torch.log(b_c))
            dtail = -a_c / b_c                                           # d loss / d b
        else:
            loss = loss + b_c * (torch.log(b_c) - torch.log(a_c))
            dtail = torch.log(b_c) - torch.log(a_c) + 1.0
        outer = outer + torch.where(b > TAIL_FLOOR, dtail, 0.0)[:, None] * -q    # d b / d lq_k = -q_k
    return loss, outer


def _exact_loss(s, lq):
    case, lt = s["case"], s["teacher"].double()
    T = lt.shape[0]
    cu = s["cu"].cpu().numpy().astype(np.int64)
    n = np.diff(cu)
    w = np.full(T, 1.0 / T) if case["agg"] == 1 else np.repeat(1.0 / (np.maximum(n, 1) * float(len(n))), n)
    w = torch.from_numpy(w).to(DEV)
    token, grad = _exact_rows(lt, lq, case)
    on = lt != -math.inf
    mass = [(torch.where(on, torch.exp(v), 0.0)).sum() / T for v in (lt, lq)]
    return torch.stack([(w * token).sum(), mass[0], mass[1]]), token, w[:, None] * grad


def _exact_pairs(s):
    case, cu = s["case"], s["cu"].long()
    P, beta = case["P"], case["beta"]
    term = s["logp"].double() - (0.0 if s["ref"] is None else s["ref"].double())
    run_s = torch.nn.functional.pad(torch.cumsum(term, 0), (1, 0))       # sums by differences of a running sum
    run_l = torch.nn.functional.pad(torch.cumsum(s["logp"].double(), 0), (1, 0))
    S, L, n = run_s[cu[1:]] - run_s[cu[:-1]], run_l[cu[1:]] - run_l[cu[:-1]], (cu[1:] - cu[:-1]).double()
    n1 = torch.where(n > 0, n, 1.0)
    f = 1.0 / n1 if case["norm"] else torch.ones_like(n1)
    r = beta * S * f
    c, j = (torch.arange(P, device=DEV), P + torch.arange(P, device=DEV)) if case["halves"] else (
        torch.arange(0, 2 * P, 2, device=DEV), torch.arange(1, 2 * P, 2, device=DEV))
    x = r[c] - r[j] - case["margin"]
    if case["kind"] == "logistic":
        e = case["eps"]
        value = (1 - e) * torch.nn.functional.softplus(-x, threshold=100) + e * torch.nn.functional.softplus(x, threshold=100)
        slope = -(1 - e) / (1 + torch.exp(x)) + e / (1 + torch.exp(-x))
    elif case["kind"] == "squared":
        value, slope = (x / beta - 1 / (2 * beta)) ** 2, 2 * (x / beta - 1 / (2 * beta)) / beta
    else:
        value, slope = torch.where(x < 1, 1 - x, 0.0), torch.where(x < 1, -1.0, 0.0)
    nll = -L[c] / n1[c]
    g = torch.zeros(2 * P, dtype=torch.float64, device=DEV)
    g[c] += slope * beta * f[c] / P - case["nll"] / n1[c] / P
    g[j] -= slope * beta * f[j] / P
    dlogp = torch.repeat_interleave(g, cu[1:] - cu[:-1])
    whole = value + case["nll"] * nll
    record = torch.stack([whole.mean(), value.mean(), nll.mean(), (r[c] > r[j]).double().mean(), r[c].mean(), r[j].mean()])
    return {"record": record, "pair_loss": whole, "score": r, "dlogp": dlogp}


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "pairs":
        return _exact_pairs(s)
    if op == "loss":
        record, token, grad = _exact_loss(s, s["cand_logp"].double())
        return {"record": record, "token_loss": token, "dcand": grad}
    W = s["W"].double()
    step = 1024
    lse, lq, entropy = [], [], []
    if op != "grad":
        for i in range(0, case["T"], step):
            z = s["H"][i:i + step].double() @ W.T
            m = z.max(1, keepdim=True).values
            e = torch.exp(z - m)
            total = e.sum(1)
            lse.append(m[:, 0] + torch.log(total))
            entropy.append(lse[-1] - (e * z).sum(1) / total)
            ids = s["ids"][i:i + step].long()
            listed_z = torch.gather(z, 1, torch.where(ids < 0, 0, ids))
            lq.append(torch.where(ids < 0, -math.inf, listed_z - lse[-1][:, None]))
            del z, e
        lse, lq, entropy = torch.cat(lse), torch.cat(lq), torch.cat(entropy)
    if op == "score":
        return {"cand_logp": lq, "lse": lse, "entropy": entropy}
    out = {}
    if op == "update":
        record, token, grad = _exact_loss(s, lq)
        out = {"cand_logp": lq, "lse": lse, "record": record, "token_loss": token, "dcand": grad}
    else:
        lse, grad = s["lse"].double(), s["dcand"].double()
    dH, dW = [], torch.zeros_like(W) if case["head"] else None
    for i in range(0, case["T"], step):
        h = s["H"][i:i + step].double()
        ids = s["ids"][i:i + step].long()
        g = torch.where(ids < 0, 0.0, grad[i:i + step])
        dz = torch.exp(h @ W.T - lse[i:i + step, None])
        dz *= -g.sum(1)[:, None]
        row = torch.arange(h.shape[0], device=DEV)[:, None].expand_as(ids)
        dz.index_put_((row, torch.where(ids < 0, 0, ids)), g, accumulate=True)
        dH.append(dz @ W)
        if dW is not None:
            dW.addmm_(dz.T, h)
        del dz
    return dict(out, d_hidden=torch.cat(dH), d_W=dW)
