"""Oracle of the constrained choice of children, test infrastructure only: the rules of include/mamba_hip.h on numpy arrays.  With
dtype float32 every operation is one rounded float32 operation in the order that the header gives, so that results are equal bit for bit;
with float64 it is the definition without rounding."""
import numpy as np


def token_counts(tokens, V, counts=None, prompt=False):
    out = np.zeros((tokens.shape[0], V), np.int64) if counts is None else counts.astype(np.int64)
    bit, low = (out < 0), out & 0x7fffffff
    for s, row in enumerate(tokens):
        n = np.bincount(row[(row >= 0) & (row < V)], minlength=V)
        if prompt:
            bit[s] |= n > 0
        else:
            low[s] += n
    return np.where(bit, low - (1 << 31), low).astype(np.int32)


def constrain(logits, counts=None, penalties=None, seq_idx=None, path=None, bias=None, mask=None, mask_idx=None, dtype=np.float32):
    """Adjusted logits (M,V) and which tokens are allowed; a row with an index out of range allows none."""
    x = np.array(logits, dtype=dtype)
    M, V = x.shape
    allowed = np.ones((M, V), dtype=bool)
    rows = lambda idx, n: np.asarray(idx) if idx is not None else np.zeros(M, int) if n == 1 else np.arange(M)
    n_seq = max([a.shape[0] for a in (counts, penalties) if a is not None], default=0)
    seq = rows(seq_idx, n_seq)
    grammar = rows(mask_idx, mask.shape[0]) if mask is not None else np.full(M, -1)
    for m in range(M):
        if (n_seq and not 0 <= seq[m] < n_seq) or not -1 <= grammar[m] < (0 if mask is None else mask.shape[0]):
            allowed[m] = False
            continue
        if penalties is not None:
            repetition, presence, frequency = (dtype(p) for p in penalties[seq[m]])
            c = np.zeros(V, np.int64) if counts is None else counts[seq[m]].astype(np.int64)
            prompt, c = c < 0, c & 0x7fffffff
            if path is not None:
                own = path[m][(path[m] >= 0) & (path[m] < V)]
                c = c + np.bincount(own, minlength=V)
            with np.errstate(all="ignore"):
                y = np.where(x[m] > 0, x[m] / repetition, x[m] * repetition)
                y = np.where((c > 0) | prompt, y, x[m])
                x[m] = np.where(c > 0, (y - frequency * c.astype(dtype)) - presence, y)
        if bias is not None:
            with np.errstate(all="ignore"):
                x[m] = x[m] + np.asarray(bias, dtype)
        if grammar[m] >= 0:
            words = np.ascontiguousarray(mask[grammar[m]]).view(np.uint8)
            allowed[m] = np.unpackbits(words, bitorder="little")[:V] != 0
    return x, allowed


def known_rows(M, n_seq=0, seq_idx=None, n_masks=0, mask_idx=None):
    """Rows whose indices are in range."""
    ok = np.ones(M, dtype=bool)
    if n_seq and seq_idx is not None:
        ok &= (seq_idx >= 0) & (seq_idx < n_seq)
    if n_masks and mask_idx is not None:
        ok &= (mask_idx >= -1) & (mask_idx < n_masks)
    return ok


def children(x, allowed, k, path=None):
    """Tokens (M,k), values (M,k) float32 and paths of the k best allowed ones; NaN ranks as -inf, ties to the lower index."""
    M, V = x.shape
    idx, val = np.full((M, k), -1, np.int32), np.full((M, k), -np.inf, np.float32)
    for m in range(M):
        at = np.flatnonzero(allowed[m])
        v = np.where(np.isnan(x[m, at]), -np.inf, x[m, at])
        best = np.argsort(-v, kind="stable")[:k]
        idx[m, :len(best)], val[m, :len(best)] = at[best], v[best]
    own = np.zeros((M, 0), np.int32) if path is None else path
    return idx, val, np.concatenate([np.repeat(own, k, 0), idx.reshape(-1, 1)], 1)
