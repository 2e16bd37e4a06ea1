"""GPU: the attention with changed scores in every kernel that its rules can choose: width, rows of a workgroup, cap, bias, with and without
documents, with and without the table's gradient, which is compared over all sequences of a head.  The host says which kernel a
case takes; that the cases together take all of them is tested without a GPU."""
import itertools

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import attention_biased as oab
from gpu_util import mat_to_host, to_host
from test_gpu_attention_biased import FP32, Run, _packed

CAPS = {0: dict(), 1: dict(cap=5.0, stretch=3.0), 2: dict(cap=70.0, stretch=7.0)}   # the second and third with scores beyond a quarter of it
BIASES = {"none": dict(), "slopes": dict(slopes=True), "table": dict(table=True, buckets=32, max_distance=60)}
MASKS = ("causal", "full", "documents", "documents causal")
S = 330   # no multiple of 64 or 128 rows
SIZES = {(64, "few"): (2, 2), (64, "many"): (4, 22), (128, "few"): (2, 2), (128, "many"): (4, 11)}   # sequences, heads


def _rows(backward, d, size, cap, bias, mask, gradient):
    b, n = SIZES[d, size]
    kw = dict(cap=CAPS[cap].get("cap", 0.0), slopes=4096 if bias == "slopes" else None, documents=4096 if "documents" in mask else None)
    if bias == "table":
        kw.update(table=4096, buckets=32, max_distance=60)
    return opt.debug_attention_biased_rows(backward, b, S, n * d, n, 1, 0, 0, opt.make_attention_bias(**kw), gradient)


CASES = [c for c in itertools.product((64, 128), ("few", "many"), CAPS, BIASES, MASKS, (False, True)) if not c[5] or c[3] == "table"]


def test_the_cases_take_every_kernel():
    """On 256 compute units.  128-row backward kernels of width 64 are for sequences without documents."""
    assert opt.debug_attention_biased_rows(False, 1, 64, 64, 1, 1, 0, 0, opt.make_attention_bias(slopes=4096, table=4096)) == -1   # refused
    forward = {(c[0], _rows(False, *c), c[2], c[3]) for c in CASES}
    assert forward == set(itertools.product((64, 128), (64, 128), CAPS, BIASES))
    backward = {(c[0], _rows(True, *c), c[2], c[3], "documents" in c[4], c[5]) for c in CASES}
    want = {(d, rows, cap, bias, docs, gradient) for d, rows, cap, bias, docs, gradient in
            itertools.product((64, 128), (64, 128), CAPS, BIASES, (False, True), (False, True))
            if (bias == "table" or not gradient) and not (d == 64 and rows == 128 and docs)}
    assert backward == want


def _table_gradient(r, head):
    """A head's row of d_table on every device row, from all of its sequences, against the oracle."""
    b, s, h, n, q, d = r.b, r.s, r.h, r.n, r.q, r.d
    M, nb, nh = b * s, b // q, n // q
    T = to_host(r.T).reshape(q, n, -1).astype(np.float64)
    assert np.all(np.isfinite(T))
    O, L = mat_to_host(r.O, M, h, q).astype(np.float64), to_host(r.L).reshape(q, q, nb, nh, s)
    for i in range(q):
        want, size = np.zeros(T.shape[2]), np.zeros(T.shape[2])
        for seq in range(i * nb, (i + 1) * nb):
            rows = slice(seq * s, (seq + 1) * s)
            Q, K, V = (r.qkv[rows, (3 * head + k) * d:(3 * head + k + 1) * d].astype(np.float64) for k in range(3))
            dO, got, kw = r.d_attn[rows, head * d:(head + 1) * d].astype(np.float64), O[rows, head * d:(head + 1) * d], r.head(seq, head)
            dT, P = oab.backward(Q, K, V, dO, got, L[i, head // nh, seq % nb, head % nh].astype(np.float64), **kw)[3:5]
            spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(got)).sum(1, keepdims=True))
            want += dT
            size += np.bincount(oab.bucket_matrix(s, len(want), kw["max_distance"], kw["two_sided"]).reshape(-1), weights=spread.reshape(-1),
                                minlength=len(want))
        assert np.all(np.abs(T[i, head] - want) <= FP32 * size + 1e-30), (i, np.abs(T[i, head] - want).max())


@pytest.mark.gpu
@pytest.mark.parametrize("d,size,cap,bias,mask,gradient", CASES)
def test_forms(d, size, cap, bias, mask, gradient):
    b, n = SIZES[d, size]
    docs = _packed(b, S, 90, 40, seed=d) if "documents" in mask else None
    kw = dict(CAPS[cap], **BIASES[bias])
    if bias == "table" and "causal" not in mask:
        kw["two_sided"] = True
    r = Run(b, S, n * d, n, 1, "causal" in mask, seed=d + n, docs=docs, dirty=docs is not None, **kw)
    if not gradient:
        r.T = None
    r.go().check(which={(0, 0), (b - 1, n - 1)})
    if gradient:
        _table_gradient(r, n // 2)


@pytest.mark.gpu
@pytest.mark.parametrize("h,n,causal", [(1408, 22, True), (2816, 22, False), (512, 4, False)])
def test_the_tables_gradient_on_every_device_row(h, n, causal):
    """A grid of 2 x 2: each device row's partial is that of its own sequences."""
    r = Run(8, S, h, n, 2, causal, table=True, buckets=100, max_distance=500, two_sided=not causal, docs=_packed(8, S, 200, 20)).go()
    for head in (0, n - 1):
        _table_gradient(r, head)
