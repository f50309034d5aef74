"""Oracle of drawn children, of the verification of trees and of adapted projections, test infrastructure only: the definitions of
include/mamba_hip.h on numpy arrays in float64, row by row."""
import numpy as np


def weights(x, temperature=1.0, top_p=1.0, min_p=0.0, top_k=0):
    """Weights (V) of what is kept of one row of logits, the largest as one; None where the settings are no numbers."""
    x = np.array(x, dtype=np.float64)
    if not temperature >= 0 or np.isnan(top_p) or np.isnan(min_p):
        return None
    x[np.isnan(x)] = -np.inf
    q = np.zeros(len(x))
    order = np.argsort(-x, kind="stable")                        # ties in the order of the vocabulary
    order = order[x[order] > -np.inf]
    if len(order) == 0:
        return q
    if temperature == 0:
        q[order[0]] = 1.0
        return q
    best = x[order[0]]
    with np.errstate(all="ignore"):
        w = np.where(x[order] == best, 1.0, np.exp((x[order] - best) / temperature))
    w[np.isnan(w)] = 0.0                                         # (an infinite logit beside finite ones)
    w = w[w >= min(min_p, 1.0)]
    if top_k > 0:
        w = w[:top_k]
    if top_p < 1.0:
        reached = np.flatnonzero(np.cumsum(w) >= top_p * w.sum())
        w = w[:max(1, int(reached[0]) + 1 if len(reached) else len(w))]
    q[order[:len(w)]] = w
    return q


def distribution(x, *settings, **named):
    w = weights(x, *settings, **named)
    return w if w is None or not w.any() else w / w.sum()


def draw(weights, u):
    """First index up to which the weights add up to more than u times their sum; -1 where they have none."""
    c = np.cumsum(np.asarray(weights, dtype=np.float64))
    if not c[-1] > 0:
        return -1
    u = 0.0 if not u > 0 else min(float(u), 1.0 - 2.0 ** -53)
    return min(int(np.searchsorted(c, u * c[-1], side="right")), int(np.flatnonzero(weights)[-1]))


def sample(logits, u, params, top_k=None, seq_idx=None):
    """idx (M,k), prob (M,k) and dist (M,V); rows whose settings are not known: -1, 0 and NaN."""
    (M, V), k = logits.shape, u.shape[1]
    idx, prob, dist = np.full((M, k), -1, np.int64), np.zeros((M, k)), np.zeros((M, V))
    for m in range(M):
        s = seq_idx[m] if seq_idx is not None else 0 if len(params) == 1 else m
        left = None if not 0 <= s < len(params) else weights(logits[m], *map(float, params[s]), 0 if top_k is None else int(top_k[s]))
        if left is None:
            dist[m] = np.nan
            continue
        q = dist[m] = left / left.sum() if left.any() else left
        left = left.copy()
        for j in range(k):
            v = draw(left, u[m, j])
            if v < 0:
                break
            idx[m, j], prob[m, j], left[v] = v, q[v], 0.0
    return idx, prob, dist


def tree_rows(tree):
    """Rows of every position, the root's first."""
    rows = [1]
    for n in tree:
        rows.append(rows[-1] * n)
    return rows


def verify(p, q, tokens, u_accept, u_sample, tree):
    """out (S, gamma + 1), count (S), node (S, gamma) of trees drawn without replacement."""
    S, _, V = p.shape
    rows = tree_rows(tree)
    first = np.concatenate([[0], np.cumsum(rows)])               # of a position among the nodes
    out, node, count = np.full((S, len(tree) + 1), -1), np.full((S, len(tree)), -1), np.zeros(S, int)
    for s in range(S):
        row, behind = 0, None
        for i, n in enumerate(tree):
            P, rest = p[s, first[i] + row].astype(np.float64), q[s, first[i] + row].astype(np.float64)
            Q, taken = rest.copy(), -1
            for j in range(n):
                at = first[i + 1] - 1 + row * n + j              # (the root has no token)
                c = tokens[s, at]
                if not 0 <= c < V:
                    continue
                ratio = P[c] / Q[c] if Q[c] > 0 else float(Q[c] <= 0 and P[c] > 0)
                u = float(u_accept[s, at])
                if u < 1.0 and u < ratio:                        # (a NaN accepts nothing)
                    taken = row * n + j
                    break
                gap = np.fmax(P - Q, 0.0)                        # (zero where it is NaN)
                P = gap / gap.sum() if gap.sum() > 0 else P
                rest[c] = 0.0
                Q = rest / rest.sum() if rest.sum() > 0 else rest * 0.0
            if taken < 0:
                behind = P
                break
            out[s, i], node[s, i], row, count[s] = c, taken, taken, i + 1
        if behind is None:
            behind = p[s, first[-2] + row].astype(np.float64)
        out[s, count[s]] = draw(behind, u_sample[s])
        count[s] += 1
    return out, count, node


def adapted(x, w, lora_a, lora_b, idx, scale=None, bias=None, residual=None):
    """Outputs (M,N) and, of every output, the sums of absolute values that bound its rounding errors: of the product, of the adapter."""
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    delta, delta_size = np.zeros_like(y), np.zeros_like(y)
    for a in range(len(lora_a)):
        mine = np.flatnonzero(idx == a)
        s = 1.0 if scale is None else float(scale[a])
        delta[mine] = s * (x[mine] @ lora_a[a].T) @ lora_b[a].T
        delta_size[mine] = abs(s) * (np.abs(x[mine]) @ np.abs(lora_a[a]).T) @ np.abs(lora_b[a]).T
    y = y + delta
    if bias is not None:
        y = y + bias
    if residual is not None:
        y = y + residual
    y[(idx < -1) | (idx >= len(lora_a))] = np.nan
    return y, size, delta_size
