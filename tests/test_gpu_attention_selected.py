"""GPU parity: the choice of blocks, and the attention over chosen blocks, forward and backward, against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import attention_selected as oas
from workloads import round_to_bf16
from gpu_util import to_host, mat_to_dev, mat_to_host, empty

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF = 2.0 ** -8     # a rounding to bf16, relative
FP32 = 2e-5          # relative error of P: fp32 sums of 64 to 128 products, scores below 30 in units of log2
PART = 2.0 ** -12    # with lists, a block's part of an output or of dQ is rounded to fp16


@pytest.fixture(params=["mask", "lists"])
def form(request):
    """Both ways to compute: all blocks with a mask, and lists of the queries of each block."""
    opt.debug_set_attention_selected_form(1 if request.param == "mask" else 0)
    yield
    opt.debug_set_attention_selected_form(-1)


@pytest.fixture
def lists():
    opt.debug_set_attention_selected_form(0)
    yield
    opt.debug_set_attention_selected_form(-1)


class Run:
    """Choice, forward and backward on the device, and what the oracle makes of the same inputs (of the device's own attn and lse, backward).
    selected: a choice to attend to instead of the device's own, [b, n, s, count]."""

    def __init__(self, b, s, h, n, q, causal, block=64, count=3, lengths=None, selected=None, seed=0, at=(-1, -1), dirty=False, keys=None, stretch=1.0):
        rng = np.random.default_rng(seed * 7919 + s)
        self.b, self.s, self.h, self.n, self.q, self.causal, self.block, self.count = b, s, h, n, q, causal, block, count
        M, d = b * s, h // n
        self.d, self.at = d, at
        qkv = rng.standard_normal((M, 3 * h)).astype(np.float32)
        qkv.reshape(M, n, 3, d)[:, :, 0] *= stretch
        if keys is not None:
            keys(qkv.reshape(b, s, n, 3, d), rng)
        d_attn = rng.standard_normal((M, h)).astype(np.float32)
        qkv, d_attn = round_to_bf16(qkv), round_to_bf16(d_attn)
        self.qkv, self.d_attn, self.lengths = qkv, d_attn, None if lengths is None else np.asarray(lengths, dtype=np.int32)
        if dirty:   # what lies behind a sequence's end
            behind = (np.arange(s)[None] >= np.clip(self.lengths, 0, s)[:, None]).reshape(-1)
            qkv, d_attn = qkv.copy(), d_attn.copy()
            qkv[behind] = np.where(rng.random((behind.sum(), 3 * h)) < 0.5, np.nan, np.inf)
            d_attn[behind] = np.nan
        self.keep = None if lengths is None else torch.from_numpy(self.lengths).to(DEV)
        self.sel = opt.make_selection(block, count, self.keep)
        self.dQKV, self.dO = mat_to_dev(qkv, q, "bf16"), mat_to_dev(d_attn, q, "bf16")
        self.O, self.L, self.G = empty(M * h, "bf16"), empty(b * n * s, "fp32"), empty(M * 3 * h, "bf16")
        self.S = torch.full((b * n * s * count,), -123, dtype=torch.int32, device=DEV)
        self.given = selected is not None
        if self.given:
            dev = np.asarray(selected, dtype=np.int32).reshape(q, b // q, q, n // q, s, count).transpose(0, 2, 1, 3, 4, 5)
            self.S.copy_(torch.from_numpy(np.ascontiguousarray(dev)).reshape(-1))
        self.ws = torch.full((opt.attention_selected_workspace_bytes(b, s, h, n, q, *at, self.sel),), 0xFF, dtype=torch.uint8, device=DEV)
        self.args = (b, s, h, n, q, *at, causal, opt.BF16, self.sel, self.ws)

    def choose(self, **kw):
        opt.attention_select(self.dQKV, self.S, *self.args, **kw)

    def forward(self, **kw):
        opt.attention_selected_fwd(self.dQKV, self.S, self.O, self.L, *self.args, **kw)

    def backward(self, **kw):
        opt.attention_selected_bwd(self.dQKV, self.S, self.O, self.L, self.dO, self.G, *self.args, **kw)

    def go(self):
        print("selected attention", self.b, self.s, self.h, self.n, self.q, self.causal, self.block, self.count, flush=True)
        if not self.given:
            self.choose()
        self.forward()
        self.backward()
        torch.cuda.synchronize()
        return self

    def chosen(self):
        """[b, n, s, count]"""
        q, b, n = self.q, self.b, self.n
        x = self.S.cpu().numpy().reshape(q, q, b // q, n // q, self.s, self.count)
        return x.transpose(0, 2, 1, 3, 4, 5).reshape(b, n, self.s, self.count)

    def check(self, which=None):
        b, s, h, n, q, d = self.b, self.s, self.h, self.n, self.q, self.d
        M, nb, nh = b * s, b // q, n // q
        O, G = mat_to_host(self.O, M, h, q).astype(np.float64), mat_to_host(self.G, M, 3 * h, q).astype(np.float64)
        L, chosen = to_host(self.L).reshape(q, q, nb, nh, s), self.chosen()
        for seq in range(b):
            for head in range(n):
                if which is not None and (seq, head) not in which:
                    continue
                rows, cols = slice(seq * s, (seq + 1) * s), slice(head * d, (head + 1) * d)
                Q, K, V = (self.qkv[rows, (3 * head + k) * d:(3 * head + k + 1) * d].astype(np.float64) for k in range(3))
                dO, length = self.d_attn[rows, cols].astype(np.float64), None if self.lengths is None else self.lengths[seq]
                sel = chosen[seq, head]
                if not self.given:
                    want = oas.choose(Q, K, block=self.block, count=self.count, causal=self.causal, length=length)
                    assert np.array_equal(sel, want), (seq, head, np.argwhere((sel != want).any(1))[:4])
                see = oas.seen(sel, s, block=self.block, causal=self.causal, length=length)
                want, lse, P = oas.forward(Q, K, V, see)
                got, gl = O[rows, cols], L[seq // nb, head // nh, seq % nb, head % nh]
                empty_rows = np.isneginf(lse)
                assert np.array_equal(np.isneginf(gl), empty_rows) and not got[empty_rows].any()
                some = ~empty_rows
                assert np.all(np.abs(gl[some] - lse[some]) <= 1e-5 * np.maximum(1, np.abs(lse[some])))
                # P rounded, V exact, the output rounded
                assert np.all(np.abs(got - want) <= HALF * (1.01 * np.abs(want) + P @ np.abs(V)) + (FP32 + PART) * (P @ np.abs(V)) + 1e-30), (seq, head)
                dQ, dK, dV, P, dS = oas.backward(Q, K, V, dO, got, gl.astype(np.float64), see)
                spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(got)).sum(1, keepdims=True))   # what dS is a difference of
                raw, fine = np.abs(dS), FP32 * spread
                for k, (w, size, small) in enumerate(((dQ, raw @ np.abs(K) / np.sqrt(d), (fine + PART * raw) @ np.abs(K) / np.sqrt(d)),
                                                      (dK, raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                                      (dV, P.T @ np.abs(dO), FP32 * P.T @ np.abs(dO)))):
                    g = G[rows, (3 * head + k) * d:(3 * head + k + 1) * d]
                    bad = np.abs(g - w) > HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30
                    assert not np.any(bad) and not np.any(np.isnan(g)), (seq, head, "QKV"[k], np.argwhere(bad | np.isnan(g))[:4])
                    if length is not None:
                        assert not g[min(max(int(length), 0), s):].any()
        return self


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("s", [1, 2, 31, 33, 63, 64, 65, 127, 128, 129, 193, 257, 400])
def test_block_boundaries(s, d, causal, form):
    Run(2, s, 2 * d, 2, 1, causal, block=64, count=3).go().check()
    Run(2, s, 2 * d, 2, 1, causal, block=128, count=2).go().check()
    Run(2, s, 2 * d, 2, 1, causal, block=192, count=2).go().check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("block,count,s", [(64, 1, 300), (64, 2, 700), (64, 5, 1000), (64, 64, 1500), (128, 4, 1111), (192, 3, 1200), (256, 2, 1030), (512, 3, 2100),
                                           (4096, 2, 5000), (64, 12, 2300)])
def test_blocks_and_counts(block, count, s, causal, form):
    for d in (64, 128):
        Run(1, s, 2 * d, 2, 1, causal, block=block, count=count).go().check()


@pytest.mark.parametrize("b,s,h,n,q", [(4, 328, 256, 4, 2), (8, 150, 1024, 8, 2), (4, 200, 512, 4, 4), (3, 500, 640, 5, 1)])
def test_grids(b, s, h, n, q, form):
    Run(b, s, h, n, q, True, block=64, count=3).go().check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths(d, causal, form):
    """Padded batches: what lies behind a sequence's end is full of NaN and infinities."""
    lengths = [500, 0, 1, 63, 64, 65, 130, 499, 1000, -5]
    for block, count in ((64, 3), (128, 2), (256, 2)):
        Run(10, 500, 2 * d, 2, 1, causal, block=block, count=count, lengths=lengths, dirty=True).go().check()


def _given(b, n, s, count, low, high, seed=0):
    return np.random.default_rng(seed).integers(low, high, (b, n, s, count))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("block", [64, 128, 256])
def test_choices_of_the_callers_own(block, causal, form):
    """Any entries: repeated, unsorted, out of range on both sides, none at all, all queries the same block."""
    b, n, s, count = 2, 2, 700, 5
    for low, high in ((-3, 14), (0, 2), (-1, 0), (-2 ** 31, 2 ** 31 - 1)):
        Run(b, s, n * 64, n, 1, causal, block=block, count=count, selected=_given(b, n, s, count, low, high)).go().check()
    sel = np.full((b, n, s, count), 1)
    sel[0, 0, ::3] = -1                       # rows that see nothing among others
    Run(b, s, n * 128, n, 1, causal, block=block, count=count, selected=sel, lengths=[650, 100]).go().check()


def test_equal_scores():
    """Keys that repeat: equal means, the lower block is chosen; no queries at all: every score zero."""
    def same(x, rng):
        x[:, :, :, 1] = x[:, :64, :, 1].repeat(x.shape[1] // 64, axis=1)

    def pairs(x, rng):
        x[:, 128:256, :, 1] = x[:, :128, :, 1]
        x[:, 640:768, :, 1] = x[:, :128, :, 1]

    def nothing(x, rng):
        x[:, :, :, 0] = 0

    for keys in (same, pairs, nothing):
        for causal in (True, False):
            Run(1, 1024, 256, 2, 1, causal, block=64, count=6, keys=keys).go().check()
            Run(1, 1024, 128, 2, 1, causal, block=64, count=2, keys=keys).go().check()


def test_scores_that_fp32_does_not_tell_apart():
    """Means whose products with the queries differ by less than fp32 sums resolve: the order is that of the exact products."""
    def close(x, rng):
        base = rng.standard_normal(x.shape[-1]) * 8
        x[:, :, :, 1] = base + rng.standard_normal((x.shape[1] // 64, 1, x.shape[-1])).repeat(64, 1).reshape(x.shape[1], 1, -1) * 0.03
        x[:, :, :, 0] += 20 * rng.standard_normal(x.shape[-1])
    for d in (64, 128):
        r = Run(1, 2048, 2 * d, 2, 1, True, block=64, count=8, keys=close)
        r.choose()
        torch.cuda.synchronize()
        for head in range(2):
            Q, K = (r.qkv[:, (3 * head + k) * d:(3 * head + k + 1) * d].astype(np.float64) for k in range(2))
            assert np.array_equal(r.chosen()[0, head], oas.choose(Q, K, block=64, count=8, causal=True))


def test_scores_that_are_not_finite():
    """NaN below every number, infinities in their order; every list in range and ascending."""
    r = Run(1, 1024, 128, 2, 1, False, block=64, count=5)
    x = r.dQKV.view(1024, 2, 3, 64)
    x[100, 0, 1, 3] = float("nan")           # a key of block 1, head 0
    x[300, 0, 1, 5] = float("inf")           # of block 4
    x[700, 1, 0, 7] = float("nan")           # a query of head 1
    r.qkv = x.float().cpu().numpy().reshape(1024, -1)
    r.choose()
    torch.cuda.synchronize()
    for head in range(2):
        Q, K = (r.qkv[:, (3 * head + k) * 64:(3 * head + k + 1) * 64].astype(np.float64) for k in range(2))
        with np.errstate(all="ignore"):
            want = oas.choose(Q, K, block=64, count=5, causal=False)
        assert np.array_equal(r.chosen()[0, head], want)


@pytest.mark.parametrize("scale", [1e-3, 30.0, 1e4])
def test_scores_of_any_size(scale, form):
    """The forward at small and large scores: lse and the largest weights."""
    r = Run(1, 600, 128, 1, 1, True, block=64, count=3, stretch=scale)
    r.choose()
    r.forward()
    torch.cuda.synchronize()
    Q, K, V = (r.qkv[:, k * 128:(k + 1) * 128].astype(np.float64) for k in range(3))
    see = oas.seen(r.chosen()[0, 0], 600, block=64, causal=True)
    want, lse, P = oas.forward(Q, K, V, see)
    # an fp32 score is off by 128 * 2^-24 of its products' sizes, and so is P in the exponent
    off = 128 * 2.0 ** -24 * (np.abs(Q) @ np.abs(K).T / np.sqrt(128)).max(1, keepdims=True)
    L = to_host(r.L).astype(np.float64)
    assert np.all(np.abs(L - lse) <= 1e-5 * np.maximum(1, np.abs(lse)) + off[:, 0])
    bound = HALF * (1.01 * np.abs(want) + P @ np.abs(V)) + (FP32 + PART + 2 * np.expm1(np.minimum(2 * off, 1))) * np.abs(V).max()
    assert np.all(np.abs(mat_to_host(r.O, 600, 128, 1) - want) <= bound)


@pytest.mark.parametrize("b,s,h,n,block,count", [(8, 1024, 1024, 8, 64, 6), (4, 2048, 1024, 16, 128, 5), (2, 3000, 512, 4, 256, 4)])
def test_larger_launches(b, s, h, n, block, count):
    Run(b, s, h, n, 1, True, block=block, count=count).go().check(which={(0, 0), (b - 1, n - 1), (b // 2, 1)})


def test_one_device_has_the_bits_of_the_grid(form):
    for h, block in ((256, 64), (512, 128), (256, 256)):
        full = Run(4, 520, h, 4, 2, True, block=block, count=3, lengths=[520, 300, 1, 519]).go()
        for dev in ((0, 1), (1, 0)):
            one = Run(4, 520, h, 4, 2, True, block=block, count=3, lengths=[520, 300, 1, 519], at=dev).go()
            k = dev[0] * 2 + dev[1]
            for name in "SOLG":
                x, y = getattr(full, name).view(4, -1), getattr(one, name).view(4, -1)
                assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), name
                rest = y[[e for e in range(4) if e != k]]
                assert (rest == -123).all() if name == "S" else torch.isnan(rest).all(), name     # nothing else is written


def test_same_call_same_bits(form):
    a, b = (Run(4, 1000, 512, 8, 1, True, block=64, count=6).go() for _ in range(2))
    b.ws.fill_(0x55)
    b.go()
    for name in "SOLG":
        assert torch.equal(getattr(a, name).view(torch.uint8), getattr(b, name).view(torch.uint8)), name


def test_captured_and_on_another_stream(form):
    """A graph of all three replayed with other inputs and lengths, eager work and synchronisations between, and the same on a stream of its own."""
    r = Run(2, 700, 256, 4, 1, True, block=64, count=4, lengths=[700, 600]).go()
    first = [x.clone() for x in (r.S, r.O, r.L, r.G)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.choose()
        r.forward()
        r.backward()
    saved, other = r.dQKV.clone(), torch.roll(r.dQKV, 8 * 64)
    for k in range(4):
        r.dQKV.copy_(saved if k % 2 == 0 else other)
        r.keep.copy_(torch.tensor([700, 600] if k % 2 == 0 else [333, 700], dtype=torch.int32))
        for x in (r.O, r.L, r.G):
            x.fill_(float("nan"))
        r.S.fill_(-9)
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (r.S, r.O, r.L, r.G)]
        r.go()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, (r.S, r.O, r.L, r.G)))
        assert (k % 2 == 1) != all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, first))
    st = torch.cuda.Stream()
    for x in (r.O, r.L, r.G):
        x.fill_(float("nan"))
    torch.cuda.synchronize()
    r.choose(stream=st)
    r.forward(stream=st)
    r.backward(stream=st)
    st.synchronize()
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, (r.S, r.O, r.L, r.G)))


def test_portions(lists):
    """Partial results beyond the workspace's portion: more (sequence, head)s than go at a time, the same bits as one device's alone."""
    b, s, n, d = 8, 8192, 4, 128
    many = Run(b, s, n * d, n, 2, True, block=128, count=8).go()          # 32 times 36 MB and more
    one = Run(b, s, n * d, n, 2, True, block=128, count=8, at=(1, 0)).go()
    for name in "SOLG":
        assert torch.equal(getattr(one, name).view(4, -1)[2].view(torch.uint8), getattr(many, name).view(4, -1)[2].view(torch.uint8)), name


def test_a_long_sequence():
    """70001 tokens, 1094 - more than 1024 - blocks of 64 are refused, blocks of 128 run: some queries against the oracle of their own row, some
    keys' gradients against the queries that saw them."""
    s, d = 70001, 64
    with pytest.raises(opt.OptimusError):
        Run(1, s, d, 1, 1, True, block=64, count=4).go()
    r = Run(1, s, d, 1, 1, True, block=128, count=6).go()
    Q, K, V = (r.qkv[:, k * d:(k + 1) * d].astype(np.float64) for k in range(3))
    chosen, O, G = r.chosen()[0, 0], mat_to_host(r.O, s, d, 1).astype(np.float64), mat_to_host(r.G, s, 3 * d, 1).astype(np.float64)
    L, dO = to_host(r.L).astype(np.float64), r.d_attn.astype(np.float64)
    mean = oas.means(K, 128, s)
    for t in [0, 1, 127, 128, 5000, 33333, 65535, 65536, s - 1]:
        score = mean[:t // 128] @ Q[t]
        best = sorted(range(t // 128), key=lambda v: (-score[v], v))[:5] + [t // 128]
        assert list(chosen[t][:len(best)]) == sorted(best)
        keys = np.concatenate([np.arange(v * 128, min((v + 1) * 128, t + 1)) for v in sorted(best)])
        x = K[keys] @ Q[t] / 8
        p = np.exp(x - x.max())
        lse, p = x.max() + np.log(p.sum()), p / p.sum()
        assert abs(L[t] - lse) <= 1e-5 * max(1, abs(lse))
        assert np.all(np.abs(O[t] - p @ V[keys]) <= HALF * (1.01 * np.abs(p @ V[keys]) + p @ np.abs(V[keys])) + (FP32 + PART) * (p @ np.abs(V[keys])))
        ds = p * (V[keys] @ dO[t] - (dO[t] * O[t]).sum())
        want, size = ds @ K[keys] / 8, np.abs(ds) @ np.abs(K[keys]) / 8
        # (dS is a difference: its fp32 error is one of the two terms', which are of the size of sqrt(d) values)
        assert np.all(np.abs(G[t, :d] - want) <= HALF * (1.01 * np.abs(want) + size) + PART * size + 100 * FP32)
    for u in [0, 200, 40000, s - 1]:
        rows = np.nonzero((chosen == u // 128).any(1) & (np.arange(s) >= u))[0]
        p = np.exp(Q[rows] @ K[u] / 8 - L[rows])
        ds = p * (dO[rows] @ V[u] - (dO[rows] * O[rows]).sum(1))
        for got, w, size in ((G[u, d:2 * d], ds @ Q[rows] / 8, np.abs(ds) @ np.abs(Q[rows]) / 8), (G[u, 2 * d:], p @ dO[rows], p @ np.abs(dO[rows]))):
            assert np.all(np.abs(got - w) <= HALF * (1.01 * np.abs(w) + size) + 100 * FP32)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("s", [1025, 1087, 1088, 1089, 1119, 1120, 1121, 1151, 1152, 1153])
def test_block_boundaries_with_lists(s, d, lists):
    """Few of many blocks: lists of queries, around the tiles of 32, 64 and 128 rows and keys."""
    for block, count, causal in ((64, 2, True), (64, 4, False), (128, 1, True), (128, 2, False), (192, 1, True), (192, 1, False)):
        r = Run(2, s, 2 * d, 2, 1, causal, block=block, count=count, lengths=[s, 700])
        r.go().check(which={(0, 0), (1, 1)})


@pytest.mark.parametrize("block", [64, 128, 256])
def test_choices_of_the_callers_own_with_lists(block, lists):
    """More blocks than a third of them named: repeated, unsorted, out of range, none, all queries the same one."""
    b, n, s, count = 2, 2, 26 * block + 17, 2
    for causal in (True, False):
        for low, high in ((-3, 29), (0, 2), (-1, 0), (-2 ** 31, 2 ** 31 - 1)):
            r = Run(b, s, n * 64, n, 1, causal, block=block, count=count, selected=_given(b, n, s, count, low, high))
            r.go().check(which={(0, 0), (1, 1)} if block == 64 else {(1, 0)})


def test_grids_and_lengths_with_lists(lists):
    full = Run(4, 1300, 256, 4, 2, True, block=64, count=2, lengths=[1300, 700, 0, 1299], dirty=True).go().check(which={(0, 0), (1, 3), (2, 1), (3, 2)})
    for dev in ((0, 1), (1, 0)):
        one = Run(4, 1300, 256, 4, 2, True, block=64, count=2, lengths=[1300, 700, 0, 1299], dirty=True, at=dev).go()
        k = dev[0] * 2 + dev[1]
        for name in "SOLG":
            x, y = getattr(full, name).view(4, -1), getattr(one, name).view(4, -1)
            assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), name
            rest = y[[e for e in range(4) if e != k]]
            assert (rest == -123).all() if name == "S" else torch.isnan(rest).all(), name


def test_captured_with_lists(lists):
    r = Run(2, 1300, 256, 4, 1, True, block=64, count=2, lengths=[1300, 1100]).go()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.choose()
        r.forward()
        r.backward()
    saved, other = r.dQKV.clone(), torch.roll(r.dQKV, 8 * 64)
    for k in range(4):
        r.dQKV.copy_(saved if k % 2 == 0 else other)
        r.keep.copy_(torch.tensor([1300, 1100] if k % 2 == 0 else [333, 1300], dtype=torch.int32))
        for x in (r.O, r.L, r.G):
            x.fill_(float("nan"))
        r.S.fill_(-9)
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (r.S, r.O, r.L, r.G)]
        r.ws.fill_(0x55)
        r.go()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(got, (r.S, r.O, r.L, r.G)))


def test_gradients_of_any_size_with_lists(lists):
    """Rows of dO from 2^-60 to 2^60 beside each other: a part of dQ is scaled by its row, so that a small row is as exact as a large one."""
    s, d = 1300, 128
    r = Run(1, s, d, 1, 1, True, block=64, count=4)
    rows = 2.0 ** np.random.default_rng(5).integers(-60, 61, (s, 1))
    r.d_attn = (r.d_attn * rows).astype(np.float32)      # (powers of two: bf16 still)
    r.dO.copy_(mat_to_dev(r.d_attn, 1, "bf16"))
    r.go()
    Q, K, V = (r.qkv[:, k * d:(k + 1) * d].astype(np.float64) for k in range(3))
    see = oas.seen(r.chosen()[0, 0], s, block=64, causal=True)
    O, dO = mat_to_host(r.O, s, d, 1).astype(np.float64), r.d_attn.astype(np.float64)
    want, _, _, P, dS = oas.backward(Q, K, V, dO, O, to_host(r.L).astype(np.float64), see)
    spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(O)).sum(1, keepdims=True))
    raw = np.abs(dS) @ np.abs(K) / np.sqrt(d)
    small = (FP32 * spread + PART * np.abs(dS)) @ np.abs(K) / np.sqrt(d)
    got = mat_to_host(r.G, s, 3 * d, 1).astype(np.float64)[:, :d]
    # (the first query sees itself alone: its dS, a difference of equal numbers, may be all rounding)
    assert np.all(np.abs(got - want) <= HALF * (1.01 * np.abs(want) + raw) + 2 * small)


def test_most_blocks_and_entries():
    """1024 blocks and 64 of them, the most of both, captured too: more LDS than a launch has without asking."""
    s, d = 65536, 64
    r = Run(1, s, d, 1, 1, True, block=64, count=64)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.choose()
    g.replay()
    torch.cuda.synchronize()
    first = r.chosen()[0, 0].copy()
    r.S.fill_(-9)
    r.go()
    assert np.array_equal(first, r.chosen()[0, 0])
    Q, K, V = (r.qkv[:, k * d:(k + 1) * d].astype(np.float64) for k in range(3))
    O, L, mean = mat_to_host(r.O, s, d, 1).astype(np.float64), to_host(r.L).astype(np.float64), oas.means(K, 64, s)
    for t in [0, 63, 64, 64 * 63, 64 * 64, 64 * 65, 30001, 65472, s - 1]:
        score = mean[:t // 64] @ Q[t]
        best = sorted(sorted(range(t // 64), key=lambda v: (-score[v], v))[:63] + [t // 64])
        assert list(first[t]) == best + [-1] * (64 - len(best))
        keys = np.concatenate([np.arange(v * 64, min((v + 1) * 64, t + 1)) for v in best])
        x = K[keys] @ Q[t] / 8
        p = np.exp(x - x.max())
        lse, p = x.max() + np.log(p.sum()), p / p.sum()
        assert abs(L[t] - lse) <= 1e-5 * max(1, abs(lse))
        assert np.all(np.abs(O[t] - p @ V[keys]) <= HALF * (1.01 * np.abs(p @ V[keys]) + p @ np.abs(V[keys])) + (FP32 + PART) * (p @ np.abs(V[keys])))


@pytest.mark.parametrize("form_of,block", [(0, 128), (0, 512), (1, 512)])
def test_rows_past_four_gigabytes(form_of, block):
    """131072 rows of 64 heads of 128: a matrix' last rows lie 6 GB behind its first.  A query attends to its own block and the one in front;
    the last blocks' outputs and gradients against their own rows."""
    s, n, d, count = 131072, 64, 128, 2
    torch.manual_seed(3)
    x = torch.randn(s, n, 3, d, dtype=torch.bfloat16, device=DEV)
    dO = torch.randn(s, n, d, dtype=torch.bfloat16, device=DEV)
    O, G, L = torch.empty_like(dO), torch.full_like(x, float("nan")), torch.empty(n, s, dtype=torch.float32, device=DEV)
    own = torch.arange(s, dtype=torch.int32, device=DEV) // block
    S = torch.stack((own - 1, own), 1).expand(n, s, count).contiguous()
    sel = opt.make_selection(block, count)
    ws = torch.empty(opt.attention_selected_workspace_bytes(1, s, n * d, n, 1, -1, -1, sel), dtype=torch.uint8, device=DEV)
    args = (1, s, n * d, n, 1, -1, -1, True, opt.BF16, sel, ws)
    opt.debug_set_attention_selected_form(form_of)
    try:
        print("far rows", form_of, block, flush=True)
        opt.attention_selected_fwd(x, S, O, L, *args)
        opt.attention_selected_bwd(x, S, O, L, dO, G, *args)
        torch.cuda.synchronize()
    finally:
        opt.debug_set_attention_selected_form(-1)
    assert not torch.isnan(G).any()
    chosen = torch.empty_like(S)
    opt.attention_select(x, chosen, *args)
    torch.cuda.synchronize()
    rows = 2 * block                                    # keys of the first of them are those of queries in front, too
    lo = s - rows
    q = np.arange(s - rows, s)
    see = (q[:, None] >= q[None]) & (q[:, None] // block - q[None] // block <= 1)
    for head in (0, 31, 63):
        Q, K, V = (x[lo:, head, k].cpu().float().numpy().astype(np.float64) for k in range(3))
        half = slice(block, rows)                       # queries that see these two blocks alone, keys that only they see
        g, o = dO[lo:, head].cpu().float().numpy().astype(np.float64), O[lo:, head].cpu().float().numpy().astype(np.float64)
        want, lse, P = oas.forward(Q, K, V, see)
        size = P @ np.abs(V)
        assert np.all(np.abs(L[head, lo:].cpu().numpy() - lse)[half] <= 1e-5 * np.maximum(1, np.abs(lse[half])))
        assert np.all((np.abs(o - want) <= HALF * (1.01 * np.abs(want) + size) + (FP32 + PART) * size)[half])
        dQ, dK, dV, P, dS = oas.backward(Q, K, V, g, o, L[head, lo:].cpu().numpy().astype(np.float64), see)
        spread = P * (np.abs(g) @ np.abs(V).T + (np.abs(g) * np.abs(o)).sum(1, keepdims=True))
        raw, fine = np.abs(dS), FP32 * spread
        for k, (w, size, small) in enumerate(((dQ, raw @ np.abs(K) / np.sqrt(d), (fine + PART * raw) @ np.abs(K) / np.sqrt(d)),
                                              (dK, raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                              (dV, P.T @ np.abs(g), FP32 * P.T @ np.abs(g)))):
            got = G[lo:, head, k].cpu().float().numpy().astype(np.float64)
            assert np.all((np.abs(got - w) <= HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30)[half]), (head, "QKV"[k])
        # the choice: the last row's, by its own scores
        mean = oas.means(x[:, head, 1].cpu().float().numpy(), block, s)
        score = mean[:-1] @ Q[-1]
        best = int(np.argmax(score))
        assert chosen[head, -1].tolist() == [best, (s - 1) // block]


def test_two_calls_at_once_and_graphs_that_share_a_workspace(form):
    """Two streams with a workspace each; two graphs over one workspace, replayed in turn."""
    a, b = (Run(2, 1500, 256, 4, 1, True, block=64, count=4, seed=k, lengths=[1500, 900 + k]) for k in range(2))
    want = [[x.clone() for x in (r.S, r.O, r.L, r.G)] for r in (a.go(), b.go())]
    same = lambda r, w: all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((r.S, r.O, r.L, r.G), w))

    def clear():
        for r in (a, b):
            r.S.fill_(-9)
            for x in (r.O, r.L, r.G):
                x.fill_(float("nan"))
        torch.cuda.synchronize()

    streams = [torch.cuda.Stream() for _ in range(2)]
    clear()
    for step in ("choose", "forward", "backward"):
        for r, st in zip((a, b), streams):
            getattr(r, step)(stream=st)
    torch.cuda.synchronize()
    assert same(a, want[0]) and same(b, want[1])
    b.args = b.args[:-1] + (a.ws,)
    graphs = []
    for r in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r.choose()
            r.forward()
            r.backward()
        graphs.append(g)
    for k in range(3):
        clear()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert same(a, want[0]) and same(b, want[1])


@pytest.mark.parametrize("block", [64, 128, 256])
def test_captured_at_width_128(block, lists):
    """The passes whose LDS is sized at launch, captured and replayed, against eager calls."""
    r = Run(2, 1100, 512, 4, 1, True, block=block, count=3, lengths=[1100, 777]).go()
    want = [x.clone() for x in (r.S, r.O, r.L, r.G)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.choose()
        r.forward()
        r.backward()
    for k in range(3):
        r.S.fill_(-9)
        for x in (r.O, r.L, r.G):
            x.fill_(float("nan"))
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip((r.S, r.O, r.L, r.G), want))
