"""CPU: the oracle of the attention with changed scores against closed forms, the plain oracle and differences; the entry points' refusals."""
import ctypes

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import attention as oatt, attention_biased as oab


def test_buckets():
    # one side of 8: distances 0..3 alone, then 4 * 4^(k/4): 4, 5.66, 8, 11.3 (max_distance 16)
    assert [oab.bucket(n, 8, 16, False) for n in (-3, 0, 1, 2, 3, 4, 5, 6, 7, 8, 11, 12, 15, 16, 1000)] == [0, 0, 1, 2, 3, 4, 4, 5, 5, 6, 6, 7, 7, 7, 7]
    assert [oab.bucket(n, 16, 16, True) for n in (0, 1, 4, -1, -4, -8, -100)] == [0, 1, 4, 9, 12, 14, 15]
    # a power that is a whole number begins its bucket: 8 * 16^(k/8) passes 16, 32, 64 for k = 2, 4, 6
    for n, k in ((15, 9), (16, 10), (31, 11), (32, 12), (63, 13), (64, 14)):
        assert oab.bucket(n, 16, 128, False) == k, n


def _random(s, d, seed):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal((s, d)) for _ in range(4)]


def test_without_changes_it_is_the_plain_attention():
    Q, K, V, dO = _random(23, 8, 0)
    for causal in (False, True):
        O, lse, P = oab.forward(Q, K, V, causal=causal)
        O0, P0 = oatt.head_forward(Q, K, V, causal)
        assert np.allclose(O, O0, atol=1e-12) and np.allclose(P, P0, atol=1e-12) and np.allclose(lse, oatt.head_logsumexp(Q, K, causal))
        got = oab.backward(Q, K, V, dO, O, lse, causal=causal)
        for a, b in zip(got[:3], oatt.head_backward(Q, K, V, P0, dO)):
            assert np.allclose(a, b, atol=1e-12)
    # a prefix over everything lifts the causal mask, one document masks nothing, equal biases change no soft-max
    free = oab.forward(Q, K, V, causal=False)[0]
    assert np.allclose(oab.forward(Q, K, V, causal=True, prefix=23)[0], free)
    assert np.allclose(oab.forward(Q, K, V, causal=False, doc=np.full(23, 5))[0], free)
    assert np.allclose(oab.forward(Q, K, V, causal=False, table=np.full(8, 3.0), max_distance=10)[0], free)
    assert np.allclose(oab.forward(Q, K, V, causal=False, cap=1e6)[0], free, atol=1e-9)


def test_documents_are_sequences_of_their_own():
    Q, K, V, _ = _random(20, 8, 1)
    doc = np.array([0] * 7 + [1] * 9 + [-1] * 4)
    O, lse, P = oab.forward(Q, K, V, causal=True, doc=doc, slope=0.3)
    for a, b in ((0, 7), (7, 16)):
        part = oab.forward(Q[a:b], K[a:b], V[a:b], causal=True, slope=0.3)
        assert np.allclose(O[a:b], part[0]) and np.allclose(lse[a:b], part[1])
    assert not O[16:].any() and np.all(np.isneginf(lse[16:])) and not P[16:].any()


KINDS = [dict(cap=1.5), dict(slope=0.2), dict(table=np.random.default_rng(5).standard_normal(8), max_distance=10),
         dict(table=np.random.default_rng(6).standard_normal(8), max_distance=9, two_sided=True, cap=2.0),
         dict(doc=np.array([0] * 4 + [2] * 6 + [-1] * 2 + [0] * 2), cap=3.0), dict(prefix=5, slope=0.1)]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(kind, causal):
    kw = dict(KINDS[kind], causal=causal)
    Q, K, V, dO = _random(14, 6, 2)

    def loss(q, k, v, table=None):
        w = dict(kw, **({"table": table} if table is not None else {}))
        return (oab.forward(q, k, v, **w)[0] * dO).sum()

    O, lse, _ = oab.forward(Q, K, V, **kw)
    dQ, dK, dV, dT, _, _ = oab.backward(Q, K, V, dO, O, lse, **kw)
    rng, h = np.random.default_rng(3), 1e-5
    for _ in range(6):   # central differences along random directions: error h^2 and 1e-16 / h
        q, k, v = (rng.standard_normal(x.shape) for x in (Q, K, V))
        num = (loss(Q + h * q, K + h * k, V + h * v) - loss(Q - h * q, K - h * k, V - h * v)) / (2 * h)
        assert abs(num - ((dQ * q).sum() + (dK * k).sum() + (dV * v).sum())) < 1e-7
        if dT is not None:
            t = rng.standard_normal(dT.shape)
            num = (loss(Q, K, V, kw["table"] + h * t) - loss(Q, K, V, kw["table"] - h * t)) / (2 * h)
            assert abs(num - (dT * t).sum()) < 1e-7


def _rc(bwd=False, b=4, s=64, h=256, n=4, q=2, i=0, j=0, causal=1, dtype=1, ptr=True, ws=4096, ws_bytes=1 << 30, d_table=None, bias=None, null_bias=False):
    one = ctypes.c_void_p(4096)
    bias = opt.make_attention_bias(**(bias or {}))
    ref = None if null_bias else ctypes.byref(bias)
    q_ptr = one if ptr else None
    if bwd:
        return opt.lib().optimus_attention_biased_bwd(q_ptr, one, one, one, one, d_table, b, s, h, n, q, i, j, causal, dtype, ref, ws, ws_bytes, None)
    return opt.lib().optimus_attention_biased_fwd(q_ptr, one, one, b, s, h, n, q, i, j, causal, dtype, ref, ws, ws_bytes, None)


T = dict(table=4096, buckets=32, max_distance=128)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("kw,code", [
    (dict(ptr=False), "EINVAL"), (dict(null_bias=True), "EINVAL"), (dict(dtype=0), "EDTYPE"), (dict(b=3), "ESHAPE"), (dict(n=3), "ESHAPE"),
    (dict(h=64), "ESHAPE"), (dict(s=0), "ESHAPE"), (dict(s=(1 << 20) + 1), "ESHAPE"), (dict(i=2), "ECOORD"), (dict(i=-1, j=0), "ECOORD"),
    (dict(bias=dict(cap=-1.0)), "EINVAL"), (dict(bias=dict(cap=float("nan"))), "EINVAL"), (dict(bias=dict(cap=float("inf"))), "EINVAL"), (dict(bias=dict(cap=1e-4)), "EINVAL"), (dict(bias=dict(cap=1e31)), "EINVAL"),
    (dict(bias=dict(T, slopes=4096)), "EINVAL"), (dict(bias=dict(prefix=4096), causal=0), "EINVAL"),
    (dict(bias=dict(T, buckets=1)), "ESHAPE"), (dict(bias=dict(T, buckets=129)), "ESHAPE"), (dict(bias=dict(T, buckets=7, two_sided=True)), "ESHAPE"),
    (dict(bias=dict(T, buckets=2, two_sided=True)), "ESHAPE"), (dict(bias=dict(T, max_distance=16)), "ESHAPE"), (dict(bias=dict(T, max_distance=1025)), "ESHAPE"),
    (dict(bias=dict(documents=4096), ws=None), "EWORKSPACE"), (dict(bias=dict(documents=4096), ws_bytes=64), "EWORKSPACE"),
    (dict(bias=dict(documents=4096), ws=4104), "EWORKSPACE"),
    (dict(b=65536, n=2, h=128, s=1, q=1), "ESHAPE"), (dict(b=2, q=1, n=512, h=512 * 64, s=1 << 20), "ESHAPE")])
def test_refusals(bwd, kw, code):
    assert _rc(bwd=bwd, **kw) == getattr(opt, code)


def test_refusals_of_the_backward():
    assert _rc(bwd=True, ws=None) == opt.EWORKSPACE and _rc(bwd=True, ws_bytes=1) == opt.EWORKSPACE
    assert _rc(bwd=True, d_table=4096) == opt.EINVAL     # no table, no gradient of one


def test_workspace_bytes():
    w = lambda **kw: opt.attention_biased_workspace_bytes(4, 100, 256, 4, 2, opt.make_attention_bias(**kw))   # noqa: E731
    rows = 4 * 4 * 100 * 4
    assert w() >= rows and w(documents=4096) >= rows + 4 * 2 * 16 and w(**T) >= rows + 4 * 4 * 2 * 32 * 4
    assert w(cap=-1.0) == 0 and opt.attention_biased_workspace_bytes(4, 100, 64, 4, 2, opt.make_attention_bias()) == 0
