"""Verification of drafted tokens and products of 4-bit integers by their definitions, in 64 bits on the CPU, one entry after another."""
import math

import numpy as np
import torch


def probabilities(row, T):
    """softmax(row / T), or None for a row that cannot be scored."""
    x = row.double().numpy()
    if np.isnan(x).any() or (x == np.inf).any() or not (x > -np.inf).any() or not (T > 0 and math.isfinite(T)):
        return None
    with np.errstate(over="ignore"):
        e = np.exp(np.maximum((x - x.max()) / T, -690.0))
    e[(x - x.max()) / T < -690.0] = 0.0
    return e / e.sum()


def first_above(weights, u):
    """The first entry at which the running sum exceeds u of the whole; the last that has any where none does; -1 where none has any."""
    u = u if u > 0 else 0.0
    some = np.nonzero(weights > 0)[0]
    if not len(some):
        return -1
    c = np.cumsum(weights)
    over = np.nonzero((c > u * c[-1]) & (weights > 0))[0]
    return int(over[0]) if len(over) else int(some[-1])


def near(weights, u, width):
    """Whether another token lies within `width` of the whole of where u falls."""
    c = np.cumsum(weights)
    return len({first_above(weights, float(v)) for v in (u - width, u, u + width)}) > 1 if c[-1] > 0 else False


def draft_verify(x, temperatures, tokens, offsets, accept_u, sample_u, draft, draft_temperatures, flags):
    """Lists of the outputs; logp NaN where a row cannot be scored."""
    MATCH, INVALID, NONFINITE = flags
    R, V = x.shape
    accepted, out, logp, fl = [], [-1] * R, [0.0] * R, [0] * R
    for b in range(len(offsets) - 1):
        k0, K = offsets[b], offsets[b + 1] - offsets[b]
        row0, i = k0 + b, 0
        while True:
            p = probabilities(x[row0 + i], temperatures[row0 + i])
            if p is None:
                fl[row0 + i], logp[row0 + i] = NONFINITE, math.nan
                break
            if i == K:
                w = p
            else:
                t = tokens[k0 + i]
                inside = 0 <= t < V
                q = np.zeros(V)
                if draft is None:
                    q[t if inside else 0] = 1.0 if inside else 0.0
                else:
                    q = probabilities(draft[k0 + i], draft_temperatures[k0 + i])
                    if q is None:
                        fl[row0 + i], logp[row0 + i] = NONFINITE, math.nan
                        break
                if inside and p[t] > 0 and accept_u[k0 + i] * q[t] < p[t]:
                    out[row0 + i], logp[row0 + i], fl[row0 + i] = t, math.log(p[t]), MATCH
                    i += 1
                    continue
                if not inside:
                    fl[row0 + i] = INVALID
                w = np.maximum(p - q, 0.0)
                if w.sum() < 2.0 ** -40:
                    w = p
            t = first_above(w, sample_u[b])
            out[row0 + i], logp[row0 + i] = t, math.log(p[t])
            break
        accepted.append(i)
    return accepted, out, logp, fl


def tree_verify(x, temperatures, tokens, parents, offsets, sample_u, flags):
    MATCH, _, NONFINITE = flags
    R, V = x.shape
    accepted, out, nodes, logp, fl = [], [-1] * R, [-1] * R, [0.0] * R, [0] * R
    for b in range(len(offsets) - 1):
        k0, K = offsets[b], offsets[b + 1] - offsets[b]
        row0, at, n = k0 + b, -1, 0
        while True:
            row = row0 + at + 1
            p = probabilities(x[row], temperatures[row])
            if p is None:
                fl[row0 + n], logp[row0 + n] = NONFINITE, math.nan
                break
            t = first_above(p, sample_u[row])
            out[row0 + n], logp[row0 + n] = t, math.log(p[t])
            kids = [j for j in range(at + 1, K) if (j - 1 if parents is None else parents[k0 + j]) == at and tokens[k0 + j] == t]
            if not kids:
                break
            fl[row0 + n], nodes[row0 + n] = MATCH, kids[0]
            at, n = kids[0], n + 1
        accepted.append(n)
    return accepted, out, nodes, logp, fl


def int4(x, group, zero_points):
    """codes uint8 [N, K / 2], scales bf16 and zeros uint8 [N, K / group], values float64 [N, K] of a float32 or bfloat16 tensor."""
    N, d = x.shape
    K = -(-d // 128) * 128
    w = np.zeros((N, K), np.float32)
    w[:, :d] = x.float().numpy()
    w = w.reshape(N, K // group, group)
    f = np.float32
    with np.errstate(all="ignore"):
        good = np.isfinite(w).all(2)
        if zero_points:
            lo, hi = np.minimum(w.min(2), f(0)), np.maximum(w.max(2), f(0))
            raw = (hi - lo) / f(15)
            good &= np.isfinite(hi - lo)
        else:
            raw = np.abs(w).max(2) / f(7)
        raw = np.where(good, raw, f(math.nan))
        scales = torch.from_numpy(raw.astype(f)).to(torch.bfloat16)
        s = scales.float().numpy()
        some = s > 0
        z = np.where(some, np.clip(np.rint(-lo / s), 0, 15), 0) if zero_points else np.full_like(s, 8)
        n = np.where(some[:, :, None], np.rint(w / s[:, :, None]), 0)
        c = np.clip(n + z[:, :, None], 0, 15)
    value = (c.astype(np.float64) - z[:, :, None]) * s[:, :, None].astype(np.float64)
    c = c.reshape(N, K).astype(np.uint8)
    return (torch.from_numpy(c[:, 0::2] | (c[:, 1::2] << 4)), scales, torch.from_numpy(z.astype(np.uint8)) if zero_points else None,
            torch.from_numpy(value.reshape(N, K)))
