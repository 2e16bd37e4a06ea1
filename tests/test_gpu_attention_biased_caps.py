"""GPU: capped scores over the whole range of the cap, where a few rows' scores reach it and the rows beside them stay far below.

A query row that is `LONG` has one element that is not zero, a power of two, so that Q K^T is exact in fp32; its scores lie at `share` of
the cap, their tanh in the polynomial (below a quarter) or beyond it.  What the fp32 tanh may lose:
  beyond a quarter, 1 - 2 / (exp(2u) + 1): the exponential's argument is off by two roundings, itself by a unit in the last place, together
  (2u + 1) 2^-23 sech^2(u) / 2 <= 0.79 * 2^-23 of the result; the sum's rounding and the reciprocal, refined or of one unit in the last
  place, 2 q (2^-24 + 2^-23) <= 1.2 * 2^-23 with q = 1 / (exp(2u) + 1) <= 0.39; the last rounding 2^-25.  Below 2.3 * 2^-23 of the cap.
  below it, the polynomial: a few roundings relative to the score itself, whatever the cap.
A cap up to 64 may take 1 - 2 / (exp(2u) + 1) near zero, too, where q is a half: 0.5 + 1.5 + 0.25, the same bound, 1.8e-5 of a score."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import attention_biased as oab
from workloads import round_to_bf16
from gpu_util import to_dev, to_host, empty

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -8
FP32 = 2e-5          # relative error of P: fp32 sums of 64 to 128 products, scores below 30 in units of log2
TANH = 2.3 * 2.0 ** -23
TABLE = dict(buckets=16, max_distance=40)


def _inputs(b, s, n, d, cap, shares, seed):
    """Q of ordinary rows of scores up to about 10; every 13th row long, its largest |score| about share * cap."""
    rng = np.random.default_rng(seed)
    x = round_to_bf16(rng.standard_normal((b, s, n, 3, d)).astype(np.float32))
    long_rows = np.arange(s) % 13 == 5
    share = np.array(shares)[(np.arange(s) // 13) % len(shares)]
    for t in np.flatnonzero(long_rows):
        x[:, t, :, 0] = 0
        x[:, t, :, 0, 3] = 2.0 ** np.round(np.log2(share[t] * cap * np.sqrt(d) / 3))   # |K| reaches about 3
    return x, long_rows


def _device(x, cap, causal, slopes, table, d_attn=None):
    b, s, n, _, d = x.shape
    h = n * d
    keep = [None if t is None else torch.from_numpy(t.reshape(-1)).to(DEV) for t in (slopes, table)]
    bias = opt.make_attention_bias(cap=cap, slopes=keep[0], table=keep[1], **(TABLE if table is not None else {}))
    qkv, O, L = to_dev(x, "bf16"), empty(b * s * h, "bf16"), empty(b * n * s, "fp32")
    opt.attention_biased_fwd(qkv, O, L, b, s, h, n, 1, 0, 0, causal, opt.BF16, bias)
    out = {"O": O, "L": L}
    if d_attn is not None:
        out["G"], out["T"] = empty(3 * b * s * h, "bf16"), None if table is None else empty(n * TABLE["buckets"], "fp32")
        ws = torch.empty(opt.attention_biased_workspace_bytes(b, s, h, n, 1, bias), dtype=torch.uint8, device=DEV)
        opt.attention_biased_bwd(qkv, O, L, to_dev(d_attn, "bf16"), out["G"], out["T"], b, s, h, n, 1, 0, 0, causal, opt.BF16, bias, ws)
    torch.cuda.synchronize()
    shapes = {"O": (b, s, n, d), "L": (b, n, s), "G": (b, s, n, 3, d), "T": (n, -1)}
    return {k: to_host(v).astype(np.float64).reshape(shapes[k]) for k, v in out.items() if v is not None}


def _compare(x, long_rows, cap, causal, slopes, table, got, d_attn, which):
    b, s, n, _, d = x.shape
    want_T, size_T = np.zeros((n, TABLE["buckets"])), np.zeros((n, TABLE["buckets"]))
    near = TANH * cap if cap <= 64 else 0.0
    for seq in range(b):
        for head in range(n):
            if which is not None and (seq, head) not in which:
                continue
            Q, K, V = (x[seq, :, head, k].astype(np.float64) for k in range(3))
            kw = dict(causal=causal, cap=cap)
            if slopes is not None:
                kw["slope"] = float(slopes[head])
            if table is not None:
                kw.update(table=table[head], max_distance=TABLE["max_distance"])
            O, lse, P = oab.forward(Q, K, V, **kw)
            gl, go = got["L"][seq, head], got["O"][seq, :, head]
            assert np.all(np.isfinite(go)) and np.all(np.isfinite(gl))
            off = np.abs(gl - lse) / (1e-5 * np.maximum(1, np.abs(lse)) + near)
            assert off.max() <= 1, ("log-sum-exp", seq, head, off.argmax(), off.max())
            # long rows: with scores off by E, P is off by 2E of itself; no more is asked where that is not small
            E = np.where(long_rows, (TANH + 2.0 ** -22) * cap, near)
            tol = (FP32 + 2 * E)[:, None]
            assert np.all(np.abs(go - O) <= HALF * (1.01 * np.abs(O) + P @ np.abs(V)) + tol * (P @ np.abs(V)) + 1e-30), ("attn", seq, head)
            if d_attn is None:
                continue
            dO = d_attn[seq, :, head].astype(np.float64)   # (zero in long rows: an fp32 log-sum-exp does not hold their P)
            dQ, dK, dV, dT, P, dS = oab.backward(Q, K, V, dO, go, gl, **kw)
            P = np.where(long_rows[:, None], 0, P)
            _, grad = oab.scores(Q, K, **kw)
            spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(go)).sum(1, keepdims=True))
            raw, fine = np.abs(dS * grad), (FP32 + near) * spread
            for k, (w, size, small) in enumerate(((dQ, raw @ np.abs(K) / np.sqrt(d), fine @ np.abs(K) / np.sqrt(d)),
                                                  (dK, raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                                  (dV, P.T @ np.abs(dO), (FP32 + near) * P.T @ np.abs(dO)))):
                g = got["G"][seq, :, head, k]
                bad = ~(np.abs(g - w) <= HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30)
                assert not np.any(bad), (seq, head, "QKV"[k], np.argwhere(bad)[:4])
            if table is not None:
                want_T[head] += dT
                size_T[head] += np.bincount(oab.bucket_matrix(s, TABLE["buckets"], TABLE["max_distance"], False).reshape(-1),
                                            weights=spread.reshape(-1), minlength=TABLE["buckets"])
    if d_attn is not None and table is not None and which is None:
        assert np.all(np.abs(got["T"] - want_T) <= (FP32 + near) * size_T + 1e-30)


def _bias(kind, n, rng):
    slopes = (2.0 ** (-8.0 * np.arange(1, n + 1) / n)).astype(np.float32) if kind == "slopes" else None
    table = rng.standard_normal((n, TABLE["buckets"])).astype(np.float32) if kind == "table" else None
    return slopes, table


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["none", "slopes", "table"])
@pytest.mark.parametrize("cap", [20.0, 64.0, 65.0, 1e3, 1e4, 1e5, 1e6])
def test_rows_beside_one_that_reaches_the_cap(cap, kind, d):
    """Forward and backward of ordinary rows; the long ones have no gradient of their own."""
    for causal in (True, False):
        rng = np.random.default_rng(int(cap) + d)
        slopes, table = _bias(kind, 2, rng)
        x, long_rows = _inputs(1, 193, 2, d, cap, (0.1, 0.3, 0.7, 2.0), d)
        d_attn = round_to_bf16(rng.standard_normal((1, 193, 2, d)).astype(np.float32))
        d_attn[:, long_rows] = 0
        print("cap", cap, kind, d, causal, flush=True)
        _compare(x, long_rows, cap, causal, slopes, table, _device(x, cap, causal, slopes, table, d_attn), d_attn, None)


@pytest.mark.parametrize("share", [0.05, 0.2, 0.24, 0.5, 3.0])
@pytest.mark.parametrize("cap", [1e5, 1e7, 1e10, 1e16, 1e20, 1e25, 1e30])
def test_scores_around_a_very_large_cap(cap, share):
    """Forward: scores in every part of the cap's range, products beyond 1e19 (whose squares fp32 does not hold) among them."""
    for kind in ("none", "table"):
        slopes, table = _bias(kind, 1, np.random.default_rng(3))
        x, long_rows = _inputs(1, 100, 1, 64, cap, (share,), 7)
        print("cap", cap, kind, share, flush=True)
        _compare(x, long_rows, cap, False, slopes, table, _device(x, cap, False, slopes, table), None, None)


@pytest.mark.parametrize("size", [1e6, 1e8, 1e9, 1e12, 1e20, 1e30])
def test_very_large_scores_without_a_cap(size):
    """Forward: rows of scores of every finite size beside ordinary ones, one key winning them by far, or all of them below zero."""
    for kind in ("none", "slopes", "table"):
        slopes, table = _bias(kind, 1, np.random.default_rng(3))
        x, long_rows = _inputs(1, 200, 1, 64, size, (1.0,), 8)
        x[:, 64:128, :, 1, 3] = -np.abs(x[:, 64:128, :, 1, 3])   # a block of keys that long rows see below zero
        print("size", size, kind, flush=True)
        for causal in (False, True):
            _compare(x, long_rows, 0.0, causal, slopes, table, _device(x, 0.0, causal, slopes, table), None, None)


@pytest.mark.parametrize("b,n", [(1, 1), (8, 16)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size,cap", [(1e6, 0.0), (1e9, 0.0), (1e12, 0.0), (1e30, 0.0), (1e9, 1e9), (1e30, 1e30)])
def test_gradients_beside_rows_of_very_large_scores(size, cap, d, b, n):
    """Backward: rows whose fp32 log-sum-exp holds nothing of their P, with gradients of zero, leave the others theirs.  (b, n: workgroups of
    64 rows and of 128.)"""
    for kind in ("none", "slopes", "table"):
        rng = np.random.default_rng(4)
        slopes, table = _bias(kind, n, rng)
        x, long_rows = _inputs(b, 300, n, d, size, (0.2, 1.0), 9)
        d_attn = round_to_bf16(rng.standard_normal((b, 300, n, d)).astype(np.float32))
        d_attn[:, long_rows] = 0
        print("gradients", size, cap, kind, d, b, n, flush=True)
        got = _device(x, cap, True, slopes, table, d_attn)
        assert all(np.all(np.isfinite(got[k])) for k in ("G", "T") if k in got)
        with np.errstate(over="ignore", invalid="ignore"):   # (the oracle's P of the long rows, which meets zeros)
            _gradients_of_ordinary_rows(x, long_rows, cap, slopes, table, got, d_attn, {(0, 0), (b - 1, n - 1)})


def _gradients_of_ordinary_rows(x, long_rows, cap, slopes, table, got, d_attn, which):
    """dQ of the ordinary rows, dK and dV summed over them: the oracle with the long rows taken out of the sums (their dS and dO are zero)."""
    s, d = x.shape[1], x.shape[4]
    for seq, head in which:
        Q, K, V = (x[seq, :, head, k].astype(np.float64) for k in range(3))
        kw = dict(causal=True, cap=cap)
        if slopes is not None:
            kw["slope"] = float(slopes[head])
        if table is not None:
            kw.update(table=table[head], max_distance=TABLE["max_distance"])
        go, gl, dO = got["O"][seq, :, head], got["L"][seq, head], d_attn[seq, :, head].astype(np.float64)
        S, grad = oab.scores(Q, K, **kw)
        P = np.where(long_rows[:, None] | np.isneginf(S), 0, np.exp(np.where(np.isneginf(S), 0, S) - gl[:, None]))
        dS = P * (dO @ V.T - (dO * go).sum(1, keepdims=True)) * grad
        spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(go)).sum(1, keepdims=True))
        Q = np.where(long_rows[:, None], 0, Q)   # (times dS of zero)
        raw, fine = np.abs(dS), FP32 * spread
        for k, (w, size, small) in enumerate(((dS @ K / np.sqrt(d), raw @ np.abs(K) / np.sqrt(d), fine @ np.abs(K) / np.sqrt(d)),
                                              (dS.T @ Q / np.sqrt(d), raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                              (P.T @ dO, P.T @ np.abs(dO), FP32 * P.T @ np.abs(dO)))):
            g = got["G"][seq, :, head, k]
            bad = ~(np.abs(g - w) <= HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30)
            assert not np.any(bad), (seq, head, "QKV"[k], np.argwhere(bad)[:4])


@pytest.mark.parametrize("b,s,n,d", [(8, 700, 16, 128), (16, 700, 8, 64)])
@pytest.mark.parametrize("kind", ["none", "slopes", "table"])
def test_larger_launches(b, s, n, d, kind):
    """The same in workgroups of 128 rows (width 64: the forward)."""
    cap = 1e5
    rng = np.random.default_rng(b)
    slopes, table = _bias(kind, n, rng)
    x, long_rows = _inputs(b, s, n, d, cap, (0.1, 0.3, 0.7, 2.0), 11)
    d_attn = round_to_bf16(rng.standard_normal((b, s, n, d)).astype(np.float32))
    d_attn[:, long_rows] = 0
    print("cap", b, s, n, d, kind, flush=True)
    _compare(x, long_rows, cap, True, slopes, table, _device(x, cap, True, slopes, table, d_attn), d_attn, {(0, 0), (b - 1, n - 1)})
