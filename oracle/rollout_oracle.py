"""CPU oracle of the rollout operators.  TEST INFRASTRUCTURE ONLY.

Plain, slow restatements (numpy, fp64 or whole numbers, one group / request / block at a time) of the head in 4
bits, its logits, the verification of drafted tokens and the block tables; see the header of the C library for the
formulas.  Nothing here is shared with the CUDA path.  Pins: tests/test_oracle_rollout.py.
"""
from __future__ import annotations

import math

import numpy as np

RESIDUAL_FLOOR = 2.0 ** -30


# ---------------------------------------------------------------------------------------- head in 4 bits
def five_bits(x: float) -> float:
    """x > 0 to five significant bits, halves to the even neighbour."""
    mantissa, exponent = math.frexp(x)
    return math.ldexp(float(np.rint(mantissa * 32)), exponent - 5)


def quantize_group(w):
    """(digits q in -7..7, scale) of one group; w: float64 values."""
    w = np.asarray(w, dtype=np.float64)
    if not np.isfinite(w).all() or np.abs(w).max() > 2.0 ** 120:
        return np.zeros(w.shape, dtype=np.int64), math.nan
    top = np.abs(w).max()
    if top < 2.0 ** -100:
        return np.zeros(w.shape, dtype=np.int64), 0.0
    s = five_bits(top / 7.0)
    below = np.floor(np.abs(w) / s)                           # |w| / s < 8
    q = below + (np.abs(w) - below * s >= s / 2)
    return np.where(w < 0, -q, q).astype(np.int64), s


def quantize_head_ref(W, group):
    """(q [V, d] int64, scale [V, groups], values [V, d]) of W (float64 values of bf16 numbers)."""
    V, d = W.shape
    n = -(-d // group)
    q, scale = np.zeros((V, d), dtype=np.int64), np.zeros((V, n))
    for v in range(V):
        for j in range(n):
            part = slice(j * group, min(d, (j + 1) * group))
            q[v, part], scale[v, j] = quantize_group(W[v, part])
    return q, scale, q * np.repeat(scale, group, axis=1)[:, :d]


def place(k: int) -> int:
    """Bit of weight k of a word of eight."""
    return 4 * (k // 2) + (16 if k % 2 else 0)


def pack_digits(q):
    """int32 words [V, d / 8] of q + 8."""
    V, d = q.shape
    words = np.zeros((V, d // 8), dtype=np.int64)
    for k in range(8):
        words += (q[:, k::8] + 8) << place(k)
    return words.astype(np.uint32).view(np.int32)


def unpack_digits(words):
    w = np.asarray(words).view(np.uint32).astype(np.int64)
    q = np.zeros((w.shape[0], w.shape[1] * 8), dtype=np.int64)
    for k in range(8):
        q[:, k::8] = ((w >> place(k)) & 15) - 8
    return q


def to_bf16(x):
    """float64 values that are exact in fp32, rounded to bf16 (halves to even)."""
    bits = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    bits = (bits + 0x7fff + ((bits >> 16) & 1)) & 0xffff0000
    return np.where(np.isnan(x), x, bits.astype(np.uint32).view(np.float32).astype(np.float64))


def quant_logits_ref(H, words, scale, group):
    """(logits [T, V], sums of absolute terms) in 64 bits; a weight is scale * digit as a bf16."""
    q = unpack_digits(words)
    w = to_bf16(q * np.repeat(np.asarray(scale, dtype=np.float64), group, axis=1)[:, :q.shape[1]])
    return H @ w.T, np.abs(H) @ np.abs(w).T


# ------------------------------------------------------------------------------------ draft verification
def softmax(z, tau):
    z = np.asarray(z, dtype=np.float64) / tau
    e = np.exp(z - z.max())
    return e / e.sum()


def is_distribution(z) -> bool:
    z = np.asarray(z, dtype=np.float64)
    return not (np.isnan(z).any() or (z == math.inf).any() or (z == -math.inf).all())


def draft_verify_ref(target, draft_logits, draft, cu, u_accept, u_sample, temperature=1.0, max_draft=None):
    """Dict with token, logp, n_emitted, written (which rows are), flags (set of "range", "distribution", "cu") and
    margin: how far the nearest comparison was from going the other way, relative to its larger side.  Exact borders are not
    counted: both sides are then the same numbers."""
    target = np.asarray(target, dtype=np.float64)
    D, R, V = len(draft), len(cu) - 1, target.shape[1]
    tau = float(np.float32(temperature)) or 1.0
    token, logp = np.full(D + R, -7, dtype=np.int64), np.full(D + R, math.nan)
    n_emitted, written = np.zeros(R, dtype=np.int64), np.zeros(D + R, dtype=bool)
    flags, margin = set(), math.inf
    if cu[0] != 0 or cu[R] != D:
        flags.add("cu")

    def near(a, b):
        nonlocal margin
        if a != b:
            margin = min(margin, abs(a - b) / max(abs(a), abs(b)))

    for r in range(R):
        first, end = int(cu[r]), int(cu[r + 1])
        if not (0 <= first <= end <= D) or (max_draft is not None and end - first > max_draft):
            flags.add("cu")
            continue
        n, base = end - first, first + r
        written[base:base + n + 1] = True
        token[base:base + n + 1], logp[base:base + n + 1] = -1, 0.0
        for i in range(n + 1):
            z = target[base + i]
            if not is_distribution(z):
                flags.add("distribution")
                logp[base + i], n_emitted[r] = math.nan, i
                break
            p = softmax(z, tau)
            lp = z / tau - z.max() / tau - math.log(np.exp((z - z.max()) / tau).sum())
            x = int(draft[first + i]) if i < n else None
            if x is not None and not 0 <= x < V:
                flags.add("range")
            known = x is not None and 0 <= x < V
            if temperature == 0:
                y = int(z.argmax())
                passed = x == y
            else:
                q, passed, weights = None, False, p
                if x is not None:
                    if draft_logits is not None:
                        zq = np.asarray(draft_logits[first + i], dtype=np.float64)
                        if not is_distribution(zq):
                            flags.add("distribution")
                            logp[base + i], n_emitted[r] = math.nan, i
                            break
                        q = softmax(zq, tau)
                    else:
                        q = np.zeros(V)
                        if known:
                            q[x] = 1.0
                    if known:
                        left, right = float(u_accept[first + i]) * q[x], p[x]
                        near(left, right)
                        passed = left < right
                    rest = np.maximum(p - q, 0.0) if draft_logits is not None else np.where(q > 0, 0.0, p)
                    weights = rest if rest.sum() > RESIDUAL_FLOOR else p
                if not passed:
                    u = min(max(float(u_sample[r]), 0.0), 1.0 - 2.0 ** -24)
                    C = np.cumsum(weights)
                    y = int(np.nonzero(C > u * C[-1])[0][0])
                    near(C[y], u * C[-1])
                    if y > 0:
                        near(C[y - 1], u * C[-1])
            if passed:
                token[base + i], logp[base + i] = x, lp[x]
                continue
            token[base + i], logp[base + i], n_emitted[r] = y, lp[y], i + 1
            break
    return {"token": token, "logp": logp, "n_emitted": n_emitted, "written": written, "flags": flags, "margin": margin}


# ------------------------------------------------------------------------------------------ block tables
def block_slots_ref(length, grow, held, table, free, free_count, block_size, capacity):
    """The stack worked block by block.  Returns table, free (copies), free_count, held, granted, cu, slot, position
    (entries that are not written are None in the two lists) and flags."""
    R, max_blocks = table.shape
    table, free = table.copy(), list(free)
    n_blocks, flags = len(free), set()
    if not 0 <= free_count <= n_blocks:
        flags.add("request")
    stack = free[: min(max(int(free_count), 0), n_blocks)]
    valid, need = [], []
    for r in range(R):
        end = int(length[r]) + int(grow[r])
        ok = (length[r] >= 0 and grow[r] >= 0 and 0 <= held[r] <= max_blocks and end <= 2 ** 31 - 1 and
              end <= max_blocks * block_size)
        valid.append(ok)
        need.append(-(-end // block_size) if ok else int(held[r]))
        if not ok:
            flags.add("request")
    bottom = len(stack)
    for r in range(R):
        for j in range(need[r], int(held[r])):
            stack.append(int(table[r, j]))
    if len(stack) > n_blocks:
        flags.add("request")
        stack = stack[:n_blocks]
    available = len(stack)
    wanted_before, new_held, granted = 0, [int(h) for h in held], [0] * R
    for r in range(R):
        want = max(0, need[r] - int(held[r]))
        granted[r] = int(valid[r] and (want == 0 or wanted_before + want <= available))
        wanted_before += want
        if not granted[r]:
            flags.add("blocks" if valid[r] else "request")
            continue
        for j in range(int(held[r]), need[r]):
            table[r, j] = stack.pop()
        new_held[r] = need[r]
    for p in range(bottom, len(stack)):
        free[p] = stack[p]
    cu, slot, position = [0], [None] * capacity, [None] * capacity
    for r in range(R):
        for i in range(max(0, int(grow[r]))):
            at, pos = cu[-1] + i, int(length[r]) + i
            if at >= capacity:
                flags.add("request")
                break
            position[at] = pos
            slot[at] = int(table[r, pos // block_size]) * block_size + pos % block_size if granted[r] else -1
        cu.append(cu[-1] + max(0, int(grow[r])))
    return {"table": table, "free": free, "free_count": len(stack), "held": new_held, "granted": granted, "cu": cu, "slot": slot,
            "position": position, "flags": flags}
