"""GPU: attention over chosen blocks of keys where some rows' scores are beyond 2^31.

Such a row's query is zero but for one element, a power of two, and that element of its keys is a small whole number: Q K^T is exact in fp32, equal
scores stay equal and others lie far more than a rounding apart.  Its soft-max has the same weight on every key of the largest number, none on others."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import attention_selected as oas
from gpu_util import mat_to_dev, mat_to_host, to_host
from test_gpu_attention_selected import FP32, HALF, PART, Run, form  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block,count", [(64, 3), (128, 2), (192, 2), (512, 2)])
def test_scores_beyond_the_thirty_first_power(block, count, d, causal, form):  # noqa: F811
    s, n, odd = 1000, 2, 5
    r = Run(1, s, n * d, n, 1, causal, block=block, count=count)
    x = r.qkv.reshape(s, n, 3, d)
    rng = np.random.default_rng(d + block)
    x[:, :, 1, odd] = rng.integers(-8, 9, (s, n))
    x[:, :, 0, odd] = 0                                   # ordinary rows do not look at it
    large = np.arange(s) % 7 == 3
    for t in np.flatnonzero(large):
        x[t, :, 0] = 0
        x[t, :, 0, odd] = (1 if t % 2 else -1) * 2.0 ** (30 + t % 60)   # scores from 2^30 to 2^92
    r.dQKV.copy_(mat_to_dev(r.qkv, 1, "bf16"))
    r.go()
    O, G, L = mat_to_host(r.O, s, n * d, 1).astype(np.float64), mat_to_host(r.G, s, 3 * n * d, 1).astype(np.float64), to_host(r.L).reshape(n, s)
    assert np.all(np.isfinite(O)) and np.all(np.isfinite(L)) and np.all(np.isfinite(G))
    for head in range(n):
        Q, K, V = (x[:, head, k].astype(np.float64) for k in range(3))
        see = oas.seen(r.chosen()[0, head], s, block=block, causal=causal)
        want, lse, P = oas.forward(Q, K, V, see)
        got, gl, dO = O[:, head * d:(head + 1) * d], L[head].astype(np.float64), r.d_attn[:, head * d:(head + 1) * d].astype(np.float64)
        assert np.all(np.abs(gl - lse) <= 1e-5 * np.maximum(1, np.abs(lse)))
        # P rounded, V exact, the output rounded; a block's part rounded to fp16
        assert np.all(np.abs(got - want) <= HALF * (1.01 * np.abs(want) + P @ np.abs(V)) + (FP32 + PART) * (P @ np.abs(V)) + 1e-30), head
        # gradients of the ordinary queries (those of the large rows mean nothing, nor do the sums over queries that hold them)
        dQ, _, _, P, dS = oas.backward(Q[~large], K, V, dO[~large], got[~large], gl[~large], see[~large])
        spread = P * (np.abs(dO[~large]) @ np.abs(V).T + (np.abs(dO) * np.abs(got)).sum(1, keepdims=True)[~large])
        size, small = np.abs(dS) @ np.abs(K) / np.sqrt(d), (FP32 * spread + PART * np.abs(dS)) @ np.abs(K) / np.sqrt(d)
        g = G[:, 3 * head * d:(3 * head + 1) * d][~large]
        assert np.all(np.abs(g - dQ) <= HALF * (1.01 * np.abs(dQ) + size) + 2 * small + 1e-30), head
