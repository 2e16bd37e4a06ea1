"""Attention of one (sequence, head) whose scores are capped, biased by distance and masked, in 64 bits, from the definitions:
S = Q K^T / sqrt(d); S = cap tanh(S / cap); S -= slope |t - u| or S += table[bucket(t - u)]; pairs of different documents or with padding
(document < 0), pairs behind the causal mask and the prefix, and pairs whose table entry is -1e30 or less are left out."""
import numpy as np

MASKED = -1e30


def bucket(n, buckets, max_distance, two_sided):
    """Bucket of the distance n = t - u (an int)."""
    side = buckets // 2 if two_sided else buckets
    if n < 0:
        return side + bucket(-n, side, max_distance, False) if two_sided else 0
    near = side // 2
    if n < near:
        return n
    k = near   # bucket near + j begins at the first whole number not below near * (max_distance / near)^(j / (side - near))
    while k + 1 < side and n >= near * (max_distance / near) ** ((k + 1 - near) / (side - near)) - 1e-9:
        k += 1
    return k


def bucket_matrix(s, buckets, max_distance, two_sided):
    line = np.array([bucket(n, buckets, max_distance, two_sided) for n in range(-(s - 1), s)])
    t = np.arange(s)
    return line[t[:, None] - t[None, :] + s - 1]


def scores(Q, K, *, causal, cap=0.0, slope=None, table=None, max_distance=0, two_sided=False, doc=None, prefix=0):
    """(S with -inf where a pair is left out, dS/d(Q K^T / sqrt(d)))."""
    Q, K = np.asarray(Q, dtype=np.float64), np.asarray(K, dtype=np.float64)
    s, d = Q.shape
    S = (Q @ K.T) / np.sqrt(d)
    grad = np.ones_like(S)
    if cap:
        th = np.tanh(S / cap)
        S, grad = cap * th, 1 - th * th
    t = np.arange(s)
    dist = t[:, None] - t[None, :]
    if slope is not None:
        S = S - slope * np.abs(dist)
    seen = np.ones((s, s), dtype=bool)
    if table is not None:
        bias = np.asarray(table, dtype=np.float64)[bucket_matrix(s, len(table), max_distance, two_sided)]
        seen &= bias > MASKED
        S = S + np.where(bias > MASKED, bias, 0)
    if doc is not None:
        seen &= (doc[:, None] == doc[None, :]) & (doc[:, None] >= 0)
    if causal:
        seen &= (dist >= 0) | (t[None, :] < prefix)
    return np.where(seen, S, -np.inf), grad


def forward(Q, K, V, **kw):
    """(O, lse, P): a row without pairs has O = 0, lse = -inf."""
    S, _ = scores(Q, K, **kw)
    m = S.max(axis=1)
    safe = np.where(np.isneginf(m), 0, m)
    E = np.exp(S - safe[:, None])
    total = E.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = safe + np.log(total)
    P = E / np.where(total == 0, 1, total)[:, None]
    return P @ np.where(P.any(axis=0)[:, None], np.asarray(V, dtype=np.float64), 0), lse, P


def backward(Q, K, V, dO, O, lse, *, table=None, max_distance=0, two_sided=False, **kw):
    """(dQ, dK, dV, d_table or None, P, dS) from a forward pass's O and lse."""
    S, grad = scores(Q, K, table=table, max_distance=max_distance, two_sided=two_sided, **kw)
    Q, K, V, dO, O = (np.asarray(x, dtype=np.float64) for x in (Q, K, V, dO, O))
    s, d = Q.shape
    seen = ~np.isneginf(S)
    P = np.where(seen, np.exp(np.where(seen, S, 0) - np.where(np.isneginf(lse), 0, lse)[:, None]), 0)
    dS = P * (dO @ V.T - (dO * O).sum(axis=1, keepdims=True))
    d_table = None
    if table is not None:
        d_table = np.bincount(bucket_matrix(s, len(table), max_distance, two_sided).reshape(-1), weights=dS.reshape(-1), minlength=len(table))
    raw = dS * grad
    return raw @ K / np.sqrt(d), raw.T @ Q / np.sqrt(d), P.T @ dO, d_table, P, dS
