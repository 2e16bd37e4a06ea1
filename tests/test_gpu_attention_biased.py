"""GPU parity: the attention with changed scores, forward, backward and the table's gradient, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import attention_biased as oab
from workloads import round_to_bf16
from gpu_util import to_host, mat_to_dev, mat_to_host, empty

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -8     # a rounding to bf16, relative
FP32 = 2e-5          # relative error of P: fp32 sums of 64 to 128 products, scores below 30 in units of log2


class Run:
    """Forward and backward on the device and what the oracle makes of the same inputs (of the device's own attn and lse, backward)."""

    def __init__(self, b, s, h, n, q, causal, seed=0, cap=0.0, slopes=None, table=None, buckets=0, max_distance=0, two_sided=False,
                 docs=None, prefix=None, stretch=1.0, dirty=False, at=(-1, -1)):
        rng = np.random.default_rng(seed * 7919 + s)
        self.b, self.s, self.h, self.n, self.q, self.causal, self.at = b, s, h, n, q, causal, at
        M, d = b * s, h // n
        self.d = d
        qkv = rng.standard_normal((M, 3 * h)).astype(np.float32)
        qkv.reshape(M, n, 3, d)[:, :, 0] *= stretch
        d_attn = rng.standard_normal((M, h)).astype(np.float32)
        qkv, d_attn = round_to_bf16(qkv), round_to_bf16(d_attn)
        self.docs, self.prefix = docs, prefix
        self.slopes = (2.0 ** (-8.0 * np.arange(1, n + 1) / n)).astype(np.float32) if slopes is True else slopes
        self.table = rng.standard_normal((n, buckets)).astype(np.float32) if table is True else table
        self.kw = dict(causal=causal, cap=cap, max_distance=max_distance, two_sided=two_sided)
        self.qkv, self.d_attn = qkv, d_attn
        if dirty:   # what lies in rows of padding
            pad = docs.reshape(-1) < 0
            qkv, d_attn = qkv.copy(), d_attn.copy()
            qkv[pad] = np.where(rng.random((pad.sum(), 3 * h)) < 0.5, np.nan, np.inf)
            d_attn[pad] = np.nan
        up = lambda x, t: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(t).reshape(-1)   # noqa: E731
        self.keep = [up(self.slopes, torch.float32), up(self.table, torch.float32), up(docs, torch.int32), up(prefix, torch.int32)]
        self.bias = opt.make_attention_bias(cap=cap, slopes=self.keep[0], table=self.keep[1], buckets=buckets, max_distance=max_distance,
                                            two_sided=two_sided, documents=self.keep[2], prefix=self.keep[3])
        self.dQKV, self.dO = mat_to_dev(qkv, q, "bf16"), mat_to_dev(d_attn, q, "bf16")
        self.nmat = (b // q) * (n // q)
        self.O, self.L, self.G = empty(M * h, "bf16"), empty(q * q * self.nmat * s, "fp32"), empty(M * 3 * h, "bf16")
        self.T = empty(q * n * buckets, "fp32") if buckets else None
        nbytes = opt.attention_biased_workspace_bytes(b, s, h, n, q, self.bias)
        self.ws = torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV)

    def forward(self):
        opt.attention_biased_fwd(self.dQKV, self.O, self.L, self.b, self.s, self.h, self.n, self.q, *self.at, self.causal, opt.BF16, self.bias,
                                 self.ws if self.docs is not None else None)

    def backward(self):
        opt.attention_biased_bwd(self.dQKV, self.O, self.L, self.dO, self.G, self.T, self.b, self.s, self.h, self.n, self.q, *self.at, self.causal,
                                 opt.BF16, self.bias, self.ws)

    def go(self):
        print("biased attention", self.b, self.s, self.h, self.n, self.q, self.causal, flush=True)
        self.forward()
        self.backward()
        torch.cuda.synchronize()
        return self

    def head(self, seq, head):
        kw = dict(self.kw)
        if self.slopes is not None:
            kw["slope"] = float(self.slopes[head])
        if self.table is not None:
            kw["table"] = self.table[head]
        if self.docs is not None:
            kw["doc"] = self.docs[seq]
        if self.prefix is not None:
            kw["prefix"] = int(min(max(self.prefix[seq], 0), self.s))
        return kw

    def check(self, which=None):
        b, s, h, n, q, d = self.b, self.s, self.h, self.n, self.q, self.d
        M, nb, nh = b * s, b // q, n // q
        O, G = mat_to_host(self.O, M, h, q).astype(np.float64), mat_to_host(self.G, M, 3 * h, q).astype(np.float64)
        L = to_host(self.L).reshape(q, q, nb, nh, s)
        T = to_host(self.T).reshape(q, n, -1).astype(np.float64) if self.T is not None else None
        want_T = np.zeros_like(T) if T is not None else None
        size_T = np.zeros_like(T) if T is not None else None
        for seq in range(b):
            for head in range(n):
                if which is not None and (seq, head) not in which:
                    continue
                rows, cols = slice(seq * s, (seq + 1) * s), slice(head * d, (head + 1) * d)
                Q, K, V = (self.qkv[rows, (3 * head + k) * d:(3 * head + k + 1) * d].astype(np.float64) for k in range(3))
                dO, kw = self.d_attn[rows, cols].astype(np.float64), self.head(seq, head)
                want, lse, P = oab.forward(Q, K, V, **kw)
                got, gl = O[rows, cols], L[seq // nb, head // nh, seq % nb, head % nh]
                empty_rows = np.isneginf(lse)
                assert np.array_equal(np.isneginf(gl), empty_rows) and not got[empty_rows].any()
                some = ~empty_rows
                assert np.all(np.abs(gl[some] - lse[some]) <= 1e-5 * np.maximum(1, np.abs(lse[some])))
                # P rounded, V exact, the output rounded
                assert np.all(np.abs(got - want) <= HALF * (1.01 * np.abs(want) + P @ np.abs(V)) + FP32 * (P @ np.abs(V)) + 1e-30), (seq, head)
                dQ, dK, dV, dT, P, dS = oab.backward(Q, K, V, dO, got, gl.astype(np.float64), **kw)
                _, grad = oab.scores(Q, K, **kw)
                spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(got)).sum(1, keepdims=True))   # what dS is a difference of
                raw, fine = np.abs(dS * grad), FP32 * spread
                for k, (w, size, small) in enumerate(((dQ, raw @ np.abs(K) / np.sqrt(d), fine @ np.abs(K) / np.sqrt(d)),
                                                      (dK, raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                                      (dV, P.T @ np.abs(dO), FP32 * P.T @ np.abs(dO)))):
                    g = G[rows, (3 * head + k) * d:(3 * head + k + 1) * d]
                    bad = np.abs(g - w) > HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30
                    assert not np.any(bad) and not np.any(np.isnan(g)), (seq, head, "QKV"[k], np.argwhere(bad | np.isnan(g))[:4])
                    if self.docs is not None:
                        assert not g[self.docs[seq] < 0].any()
                if T is not None:
                    want_T[seq // nb, head] += dT
                    size_T[seq // nb, head] += np.bincount(oab.bucket_matrix(s, T.shape[2], kw["max_distance"], kw["two_sided"]).reshape(-1),
                                                           weights=spread.reshape(-1), minlength=T.shape[2])
        if T is not None and which is None:
            assert np.all(np.abs(T - want_T) <= FP32 * size_T + 1e-30), np.abs(T - want_T).max()
        return self


def _packed(b, s, mean, pad, seed=0):
    rng = np.random.default_rng(seed)
    docs = np.full((b, s), -1, dtype=np.int32)
    for row in docs:
        at, k, end = 0, 0, s - int(rng.integers(0, pad + 1))
        while at < end:
            n = 1 + int(rng.exponential(mean))
            row[at:min(end, at + n)] = k
            at, k = at + n, k + 1
    return docs


BUCKETS = dict(table=True, buckets=32, max_distance=128)
KINDS = {
    "cap": dict(cap=5.0, stretch=3.0), "small cap": dict(cap=50.0), "slopes": dict(slopes=True), "cap+slopes": dict(cap=20.0, slopes=True),
    "buckets": BUCKETS, "cap+buckets": dict(BUCKETS, cap=10.0, stretch=4.0), "few buckets": dict(table=True, buckets=3, max_distance=7),
    "many buckets": dict(table=True, buckets=100, max_distance=1000),
}


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("b,s,h,n,q", [(2, 1, 128, 2, 1), (2, 70, 256, 2, 2), (4, 328, 256, 4, 2)])
def test_scores(b, s, h, n, q, kind, causal):
    Run(b, s, h, n, q, causal, **KINDS[kind]).go().check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("s", [2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 193, 257])
def test_block_boundaries(s, d):
    """Both sides of the table, and documents with padding, around the 32-row, 64-row and 128-row tiles."""
    Run(2, s, 2 * d, 2, 1, False, table=True, buckets=16, max_distance=20, two_sided=True, cap=15.0, docs=_packed(2, s, 25, s // 4)).go().check()


@pytest.mark.parametrize("two_sided", [True, False])
@pytest.mark.parametrize("buckets,max_distance", [(4, 3), (32, 128), (64, 500), (128, 1024)])
def test_tables_without_a_mask(buckets, max_distance, two_sided):
    Run(2, 450, 128, 2, 1, False, table=True, buckets=buckets, max_distance=max_distance, two_sided=two_sided).go().check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("layout", ["packed", "short", "pad only", "one", "mixed order", "gaps"])
def test_documents(layout, causal):
    b, s = 4, 391
    rng = np.random.default_rng(5)
    docs = {"packed": _packed(b, s, 100, 60), "short": _packed(b, s, 3, 5), "pad only": np.full((b, s), -7, dtype=np.int32),
            "one": np.full((b, s), 2 ** 31 - 1, dtype=np.int32), "mixed order": rng.integers(-1, 4, (b, s)).astype(np.int32),
            "gaps": np.where(rng.random((b, s)) < 0.1, -1, np.arange(s) // 50).astype(np.int32)}[layout]
    docs[1] = np.where(np.arange(s) < 64, -1, docs[1])   # a whole block of padding in front
    Run(b, s, 256, 4, 2, causal, slopes=True, docs=docs).go().check()
    Run(b, s, 256, 2, 2, causal, docs=docs, dirty=True, **BUCKETS).go().check()


@pytest.mark.parametrize("docs", [False, True])
@pytest.mark.parametrize("kind", ["slopes", "buckets", "cap"])
def test_prefix(kind, docs):
    s = 300
    prefix = np.array([0, 1, 63, 64, 65, 150, 299, 300, 1000, -5], dtype=np.int32)
    Run(10, s, 128, 2, 1, True, prefix=prefix, docs=_packed(10, s, 120, 20) if docs else None, **KINDS[kind]).go().check()


@pytest.mark.parametrize("b,s,h,n,q,kind", [(8, 1100, 1024, 8, 1, "cap+slopes"), (8, 1024, 512, 8, 1, "buckets"), (16, 520, 1024, 16, 1, "cap"),
                                            (4, 2100, 512, 8, 1, "cap+buckets"), (32, 200, 2048, 16, 1, "slopes")])
@pytest.mark.parametrize("causal", [True, False])
def test_larger_launches(b, s, h, n, q, kind, causal):
    """Enough workgroups for every form of the kernels; a few matrices against the oracle."""
    docs = _packed(b, s, 300, 100) if causal else None
    Run(b, s, h, n, q, causal, docs=docs, **KINDS[kind]).go().check(which={(0, 0), (b - 1, n - 1), (b // 2, 1)})


def test_table_gradient_of_a_larger_launch():
    """Every matrix counts in the table's gradient: 16 matrices of 600."""
    for causal, two in ((True, False), (False, True)):
        Run(4, 600, 256, 4, 1, causal, table=True, buckets=32, max_distance=128, two_sided=two).go().check()


def test_masking_tables():
    """-infinity and the lowest number mask; rows without a pair are zeros, their gradients too."""
    for low in (-np.inf, np.finfo(np.float32).min, -1e30):
        table = np.random.default_rng(0).standard_normal((2, 8)).astype(np.float32)
        table[0, :3] = low            # head 0: distances 0, 1, 2 masked: causal rows 0 .. 2 see nothing
        table[1, :] = low             # head 1: nothing at all
        r = Run(2, 150, 128, 2, 1, True, table=table, buckets=8, max_distance=30).go().check()
        assert np.all(np.isneginf(to_host(r.L).reshape(2, 2, 150)[:, 1])) and np.all(np.isneginf(to_host(r.L).reshape(2, 2, 150)[:, 0, :3]))


@pytest.mark.parametrize("cap", [1e-3, 0.02, 1e30])
def test_caps_at_the_ends_of_their_range(cap):
    """Scores all at the cap, and a cap that changes nothing."""
    Run(2, 150, 256, 2, 1, True, cap=cap, stretch=4.0).go().check()
    Run(2, 150, 128, 2, 1, False, cap=cap, stretch=4.0, **dict(BUCKETS, buckets=16)).go().check()


def test_without_changes_it_is_the_fused_attention():
    """No cap, no bias, no mask: what the attention without changes computes, to its own accuracy."""
    r = Run(4, 300, 256, 4, 2, True).go().check()
    O, L = empty(r.O.numel(), "bf16"), empty(r.L.numel(), "fp32")
    opt.attention_fused_fwd(r.dQKV, O, L, r.b, r.s, r.h, r.n, r.q, -1, -1, True, opt.BF16)
    torch.cuda.synchronize()
    assert torch.allclose(L, r.L, atol=1e-5, rtol=1e-6) and (O.float() - r.O.float()).norm() <= 2e-3 * O.float().norm()


@pytest.mark.parametrize("h", [256, 512])
def test_one_device_has_the_bits_of_the_grid(h):
    docs = _packed(4, 330, 90, 30)
    for kind in ("cap+slopes", "buckets"):
        full = Run(4, 330, h, 4, 2, True, docs=docs, **KINDS[kind]).go()
        for dev in ((0, 1), (1, 0)):
            one = Run(4, 330, h, 4, 2, True, docs=docs, at=dev, **KINDS[kind])
            one.forward()
            one.O.copy_(full.O), one.L.copy_(full.L)
            alone = Run(4, 330, h, 4, 2, True, docs=docs, at=dev, **KINDS[kind])
            alone.forward()
            one.backward()
            torch.cuda.synchronize()
            k = dev[0] * 2 + dev[1]
            for name in ("O", "L", "G", "T"):
                x, y = getattr(full, name), getattr(one if name in "GT" else alone, name)
                if x is None:
                    continue
                x, y = x.view(4, -1), y.view(4, -1)
                assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), name
                assert torch.isnan(y[[e for e in range(4) if e != k]]).all(), name     # nothing else is written


def test_same_call_same_bits():
    a, b = (Run(4, 1000, 512, 8, 1, True, docs=_packed(4, 1000, 200, 50), **KINDS["cap+buckets"]).go() for _ in range(2))
    for name in "OLGT":
        assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name


def test_without_the_tables_gradient():
    r = Run(2, 200, 256, 4, 1, True, **BUCKETS).go()
    G, r.T = r.G.clone(), None
    r.G.fill_(float("nan"))
    r.backward()
    torch.cuda.synchronize()
    assert torch.equal(G.view(torch.int16), r.G.view(torch.int16))


def test_captured_and_on_another_stream():
    """A graph of both passes replayed with other inputs, eager work and synchronisations between, and the same on a stream of its own."""
    r = Run(2, 500, 256, 4, 1, True, docs=_packed(2, 500, 100, 30), **KINDS["cap+buckets"]).go()
    first = [x.clone() for x in (r.O, r.L, r.G, r.T)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.forward()
        r.backward()
    other = torch.roll(r.dQKV, 8 * 64)
    saved = r.dQKV.clone()
    for k in range(4):
        r.dQKV.copy_(saved if k % 2 == 0 else other)
        for x in (r.O, r.L, r.G, r.T):
            x.fill_(float("nan"))
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (r.O, r.L, r.G, r.T)]
        r.forward()
        r.backward()
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, (r.O, r.L, r.G, r.T)))
        assert (k % 2 == 1) != all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, first))
    st = torch.cuda.Stream()
    r.dQKV.copy_(saved)
    r.G.fill_(float("nan"))
    torch.cuda.synchronize()
    opt.attention_biased_bwd(r.dQKV, r.O, r.L, r.dO, r.G, r.T, r.b, r.s, r.h, r.n, r.q, 0, 0, True, opt.BF16, r.bias, r.ws, stream=st)
    st.synchronize()
    assert not torch.isnan(r.G).any()


@pytest.mark.parametrize("d", [64, 128])
def test_long_packed_sequence(d):
    """A sequence of 70001 tokens: documents of about 80 are attentions of their own, whose oracle is small."""
    s, lengths, rng = 70001, [], np.random.default_rng(9)
    while sum(lengths) < s:
        lengths.append(int(rng.integers(1, 160)))
    lengths[-1] -= sum(lengths) - s
    docs = np.repeat(np.arange(len(lengths)), lengths).astype(np.int32)[None, :]
    ends = np.cumsum(lengths)
    for k in (100, 500):   # two documents are padding
        docs[0, ends[k] - lengths[k]:ends[k]] = -1
    r = Run(1, s, d, 1, 1, True, docs=docs, slopes=True).go()
    O, G, L = (to_host(x).reshape(s, -1).astype(np.float64) for x in (r.O, r.G, r.L))
    assert not np.isnan(O).any() and not np.isnan(G).any()
    for k in list(range(0, len(lengths), 7)) + [100, 500, len(lengths) - 1]:
        rows = slice(ends[k] - lengths[k], ends[k])
        Q, K, V = (r.qkv[rows, c * d:(c + 1) * d].astype(np.float64) for c in range(3))
        if docs[0, rows.start] < 0:
            assert not O[rows].any() and not G[rows].any() and np.all(np.isneginf(L[rows]))
            continue
        want, lse, P = oab.forward(Q, K, V, causal=True, slope=float(r.slopes[0]))
        dO = r.d_attn[rows].astype(np.float64)
        assert np.all(np.abs(L[rows, 0] - lse) <= 1e-5 * np.maximum(1, np.abs(lse)))
        assert np.all(np.abs(O[rows] - want) <= HALF * (1.01 * np.abs(want) + P @ np.abs(V)) + FP32 * (P @ np.abs(V)))
        dQ, dK, dV, _, P, dS = oab.backward(Q, K, V, dO, O[rows], L[rows, 0], causal=True, slope=float(r.slopes[0]))
        for c, (w, size) in enumerate(((dQ, np.abs(dS) @ np.abs(K) / np.sqrt(d)), (dK, np.abs(dS).T @ np.abs(Q) / np.sqrt(d)), (dV, P.T @ np.abs(dO)))):
            # (dS is a difference: its fp32 error is one of the two terms', which are of the size of sqrt(d) values)
            assert np.all(np.abs(G[rows, c * d:(c + 1) * d] - w) <= HALF * (1.01 * np.abs(w) + size) + 100 * FP32)


def test_bits_do_not_depend_on_the_launch():
    """Few and many matrices take kernels of 64 and of 128 rows: the forward's bits are the same."""
    one = Run(1, 1100, 128, 1, 1, True, **KINDS["cap+slopes"])
    many = Run(64, 1100, 128, 1, 1, True, **KINDS["cap+slopes"])
    many.dQKV[:one.dQKV.numel()].copy_(one.dQKV)
    one.forward(), many.forward()
    torch.cuda.synchronize()
    assert torch.equal(one.O, many.O[:one.O.numel()]) and torch.equal(one.L, many.L[:one.L.numel()])
