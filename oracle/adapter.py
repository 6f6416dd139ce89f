"""Low-rank adapters beside a shared projection, from their definition, float64.

Test infrastructure only (see the package header).

Rows come in segments: segment s holds the rows row_start[s] .. row_start[s + 1] - 1 and uses adapter seg_adapter[s]; a number outside
0 .. adapters - 1, and a row of no segment, means no adapter.  With A (adapters, rank, I), B (adapters, rank, O), and n the row's adapter:

    forward           S = scale_n X A_n^T       Z = base + S B_n
    input gradient    dS = scale_n dZ B_n^T     dX = base + dS A_n
    weight gradients  dA_n = sum dS^T X         dB_n = sum S^T dZ       over the rows of adapter n

`apply` is the forward pass; with dZ for X and A and B exchanged it is the input gradient.  Every result comes with a bound on what float32
accumulation and the operands' split into three bf16 may cost (`_bound` results): a dot product of n terms accumulated in float32, whatever the
order and even if the adder truncates, is off by at most n 2^-23 sum |a b|; a float32 number as the sum of three bf16 by 2^-24 of itself.
"""
import numpy as np

ACCUMULATE = 2.0 ** -23          # of one addition
# The first part takes the upper 8 of 24 bits, the second the next 8, the third the rest: nothing is lost from 2^-110 up, where bf16's smallest number is the
# last bit's.  2^-24 leaves room for any way of splitting in three.
SPLIT3 = 2.0 ** -24


def rows_of(row_start, seg_adapter, adapters, T):
    """The adapter of every row, -1 where it has none."""
    ids = np.full(T, -1, dtype=np.int64)
    for s, n in enumerate(seg_adapter):
        if 0 <= n < adapters:
            ids[row_start[s]:row_start[s + 1]] = n
    return ids


def apply(X, ids, down, up, scale, base):
    """(out, S, bound of S, bound of out before its rounding)."""
    T, R, C = X.shape[0], down.shape[1], up.shape[2]
    S, eS = np.zeros((T, R)), np.zeros((T, R))
    out, eO = np.zeros((T, C)), np.zeros((T, C))
    if base is not None:
        out += base
    for n in np.unique(ids[ids >= 0]):
        at = ids == n
        s = 1.0 if scale is None else float(scale[n])
        S[at] = s * (X[at] @ down[n].T)
        eS[at] = abs(s) * ((X.shape[1] + 16) * ACCUMULATE) * (np.abs(X[at]) @ np.abs(down[n]).T)      # 16: the waves' sums, scale and its product
        out[at] += S[at] @ up[n]
        eO[at] = (eS[at] + (SPLIT3 + (3 * R + 2) * ACCUMULATE) * np.abs(S[at])) @ np.abs(up[n])
        if base is not None:
            eO[at] += ACCUMULATE * np.abs(base[at])
    return out, S, eS, eO


def outer(L, M, ids, adapters):
    """(G, bound): G_n = sum over the rows of adapter n of L^T M."""
    G, e = np.zeros((adapters, L.shape[1], M.shape[1])), np.zeros((adapters, L.shape[1], M.shape[1]))
    for n in range(adapters):
        at = ids == n
        G[n] = L[at].T @ M[at]
        e[n] = (SPLIT3 + (3 * int(at.sum()) + 8) * ACCUMULATE) * (np.abs(L[at]).T @ np.abs(M[at]))
    return G, e
