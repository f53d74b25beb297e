"""The routing operators in 64 bits, row by row (numpy, shares nothing with the library).

The definitions are those of include/nimble_moe.h: choice by binary32 keys, everything else in
binary64.  Besides the values the functions give, per output, the sum of the magnitudes it is made
of, which tests scale their rounding bounds by.
"""
import numpy as np


def log_score(x, sigmoid):
    """log of the score up to the row's softmax sum: x itself, or log of the logistic function."""
    if not sigmoid:
        return x
    x = np.asarray(x, dtype=np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        tail = np.log1p(np.exp(-np.abs(x)))
        return np.where(x > 0, -tail, np.where(np.isneginf(x), -np.inf, x - tail))


def choose(x32, bias32, top_k):
    """Columns of the top_k largest keys of one row, largest first, ties to the lower one."""
    if bias32 is None:
        bias32 = np.float32(0)
    else:                                     # NaN counts as -inf, +inf as the largest number
        bias32 = np.minimum(np.where(np.isnan(bias32), -np.inf, bias32), np.finfo(np.float32).max).astype(np.float32)
    key = x32 + bias32
    ok = [e for e in range(len(x32)) if x32[e] != -np.inf and key[e] > -np.inf]
    return sorted(ok, key=lambda e: (-key[e], e))[:top_k]


def route(x, top_k, sigmoid=False, renorm=True, scale=1.0, bias=None, keep=None, ends=None):
    """x float32 [T][E] (the values of the logits).  Rows outside the segments keep index -2,
    weight NaN."""
    x = np.asarray(x, dtype=np.float32)
    T, E = x.shape
    ends = [0, T] if ends is None else ends
    S = len(ends) - 1
    out = dict(index=np.full((T, top_k), -2, dtype=np.int32), weight=np.full((T, top_k), np.nan),
               counts=np.zeros((S, E), dtype=np.int32),
               routed=np.zeros(S, dtype=np.int32), prob_sum=np.zeros((S, E)),
               prob=np.zeros((T, E)), inside=np.zeros(T, dtype=bool))
    for s in range(S):
        for t in range(ends[s], ends[s + 1]):
            out["inside"][t] = True
            out["index"][t] = -1
            out["weight"][t] = 0.0
            if keep is not None and not keep[t]:
                continue
            row = x[t]
            if np.isnan(row).any() or np.isposinf(row).any():
                out["weight"][t] = np.nan
                out["prob_sum"][s] = out["prob"][t] = np.nan
                continue
            with np.errstate(over="ignore", invalid="ignore"):
                pick = choose(row, bias, top_k)
            if not pick:
                continue
            u = log_score(row.astype(np.float64), sigmoid)
            p = np.exp(u - u.max())
            total = p.sum()
            p = p / total
            up = u[pick]
            if renorm:
                w = np.exp(up - up.max())
                w /= w.sum()
            else:
                w = np.exp(up) if sigmoid else np.exp(up - u.max()) / total
            n = len(pick)
            out["index"][t, :n] = pick
            out["weight"][t, :n] = w * scale
            out["prob"][t] = p
            out["prob_sum"][s] += p
            out["routed"][s] += 1
            out["counts"][s, pick] += 1
    return out


def balance_loss(counts, routed, prob_sum, top_k, alpha):
    S, E = np.shape(counts)
    loss = np.zeros(S)
    for s in range(S):
        if routed[s]:
            f = np.asarray(counts[s], dtype=np.float64) / routed[s]
            loss[s] = alpha * E / top_k * float((f * (np.asarray(prob_sum[s], dtype=np.float64) / routed[s])).sum())
    return loss


def route_backward(x, index, weight, sigmoid=False, renorm=True, scale=1.0, keep=None,
                   ends=None, grad_weight=None, alpha=0.0, counts=None, routed=None,
                   grad_loss=None):
    """(gradient of the logits, sum of the magnitudes of its terms); NaN in rows of no segment."""
    x = np.asarray(x, dtype=np.float64)
    T, E = x.shape
    k = index.shape[1]
    ends = [0, T] if ends is None else ends
    dx, mag = np.full((T, E), np.nan), np.full((T, E), np.nan)
    for s in range(len(ends) - 1):
        c = np.zeros(E)
        if counts is not None and routed[s]:
            c = float(grad_loss[s]) * alpha * E / (k * float(routed[s]) ** 2) * counts[s].astype(np.float64)
        for t in range(ends[s], ends[s + 1]):
            there = (index[t] >= 0) & (index[t] < E)
            if (keep is not None and not keep[t]) or not there.any():
                bad = (keep is None or keep[t]) and np.isnan(weight[t, 0])
                dx[t] = mag[t] = np.nan if bad else 0.0
                continue
            u = log_score(x[t], sigmoid)
            p = np.exp(u - u.max())
            p = p / p.sum()
            slope = np.exp(log_score(np.where(np.isneginf(x[t]), 0.0, -x[t]), True)) if sigmoid else np.ones(E)
            slope = np.where(np.isneginf(x[t]), 1.0, slope)
            w = np.where(there, weight[t], 0.0)
            g = np.where(there, grad_weight[t], 0.0) if grad_weight is not None else np.zeros(k)
            all_, all_mag = float((w * g).sum()), float(np.abs(w * g).sum())
            dense = p * (c - (p * c).sum())
            dense_mag = p * (np.abs(c) + (p * np.abs(c)).sum())
            if not sigmoid and not renorm:
                dense = dense - p * all_
                dense_mag = dense_mag + p * all_mag
            for j in range(k):
                if there[j]:
                    dense[index[t, j]] += w[j] * (g[j] - (all_ / scale if renorm else 0.0))
                    dense_mag[index[t, j]] += abs(w[j]) * (abs(g[j]) + (all_mag / scale if renorm else 0.0))
            dx[t] = dense * slope
            mag[t] = dense_mag * slope
    return dx, mag


def counts(index, experts, ends=None, place=None, n_ranks=0):
    """(slots per expert, distinct rows per rank) per segment."""
    T, k = index.shape
    ends = [0, T] if ends is None else ends
    S = len(ends) - 1
    per_expert = np.zeros((S, experts), dtype=np.int32)
    per_rank = np.zeros((S, max(n_ranks, 1)), dtype=np.int32)
    for s in range(S):
        for t in range(ends[s], ends[s + 1]):
            ranks = set()
            for e in index[t]:
                if 0 <= e < experts:
                    per_expert[s, e] += 1
                    if place is not None and 0 <= place[e] < n_ranks:
                        ranks.add(int(place[e]))
            for r in ranks:
                per_rank[s, r] += 1
    return per_expert, per_rank


def traffic(rank_tokens, bytes_per_token, src=None, dst=None, way_back=False):
    """[batch][n_comm] bytes of rank_tokens [batch][R][R]."""
    B, R, _ = rank_tokens.shape
    if src is None:
        pairs = [(s, d) for s in range(R) for d in range(R) if s != d]
    else:
        pairs = list(zip(src, dst))
    out = np.full((B, len(pairs)), np.nan)
    for b in range(B):
        for k, (s, d) in enumerate(pairs):
            if 0 <= s < R and 0 <= d < R:
                out[b, k] = float(rank_tokens[b, d, s] if way_back else rank_tokens[b, s, d]) * bytes_per_token
    return out
