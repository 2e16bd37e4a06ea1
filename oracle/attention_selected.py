"""Attention of one (sequence, head) over chosen blocks of keys, and the choice, in 64 bits, from the definitions: a query attends to its own
block and to the count - 1 others (with a causal mask: in front of it) whose mean key has the largest product with it."""
import numpy as np


def round_bf16(x):
    """fp32 -> the nearest bf16 number (ties to even)."""
    bits = np.ascontiguousarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    rounded = ((bits + 0x7FFF + ((bits >> np.uint64(16)) & np.uint64(1))) >> np.uint64(16)) << np.uint64(16)
    return rounded.astype(np.uint32).view(np.float32)


def means(K, block, length):
    """Mean keys of the blocks that hold some."""
    K = np.asarray(K, dtype=np.float64)[:length]
    rows = [K[at:at + block].sum(axis=0) / len(K[at:at + block]) for at in range(0, length, block)]
    return round_bf16(np.array(rows, dtype=np.float32).reshape(len(rows), -1)).astype(np.float64)


def choose(Q, K, *, block, count, causal, length=None):
    """int32 [s, count]: ascending, -1 behind them."""
    s = len(Q)
    length = s if length is None else min(max(int(length), 0), s)
    out = np.full((s, count), -1, dtype=np.int32)
    if length == 0:
        return out
    score = np.asarray(Q, dtype=np.float64) @ means(K, block, length).T
    score = np.where(np.isnan(score), -np.inf, score)
    for t in range(length):
        own = t // block
        others = [v for v in range(score.shape[1]) if v != own and (v < own or not causal)]
        best = sorted(others, key=lambda v: (-score[t, v], v))[:count - 1]
        chosen = sorted(best + [own])
        out[t, :len(chosen)] = chosen
    return out


def seen(selected, s, *, block, causal, length=None):
    """bool [s, s]: pairs that the attention has."""
    length = s if length is None else min(max(int(length), 0), s)
    out = np.zeros((s, s), dtype=bool)
    for t in range(length):
        for v in selected[t]:
            if 0 <= int(v) * block < length:
                out[t, int(v) * block:min(length, (int(v) + 1) * block)] = True
    return out & np.tri(s, dtype=bool) if causal else out


def forward(Q, K, V, see):
    """(O, lse, P): a row without pairs has O = 0, lse = -inf."""
    Q, K, V = (np.asarray(x, dtype=np.float64) for x in (Q, K, V))
    S = np.where(see, Q @ K.T / np.sqrt(Q.shape[1]), -np.inf)
    top = S.max(axis=1)
    top = np.where(np.isneginf(top), 0, top)
    E = np.exp(S - top[:, None])
    total = E.sum(axis=1)
    with np.errstate(divide="ignore"):
        lse = top + np.log(total)
    P = E / np.where(total == 0, 1, total)[:, None]
    return P @ V, lse, P


def backward(Q, K, V, dO, O, lse, see):
    """(dQ, dK, dV, P, dS) from a forward pass's O and lse."""
    Q, K, V, dO, O = (np.asarray(x, dtype=np.float64) for x in (Q, K, V, dO, O))
    d = Q.shape[1]
    P = np.where(see, np.exp(np.where(see, Q @ K.T / np.sqrt(d) - np.where(np.isneginf(lse), 0, lse)[:, None], 0)), 0)
    dS = P * (dO @ V.T - (dO * O).sum(axis=1, keepdims=True))
    return dS @ K / np.sqrt(d), dS.T @ Q / np.sqrt(d), P.T @ dO, P, dS
