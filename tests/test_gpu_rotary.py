"""GPU parity: rotary positions of one to four axes and their gradient against the oracle in 64 bits.

An angle's whole turns go in 64 bits, so an angle is off by the rounding of its remainder to fp32, pi * 2^-25, cosine and sine by two units in
the last place (2 * 2^-23), the two products and their sum by a rounding each: (|x| + |y|) * 8 * 2^-24 in all, and a bf16 result by 2^-8 of itself."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import rotary as orot
from workloads import round_to_bf16
from gpu_util import empty, mat_to_dev, mat_to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HALF, FP32 = 2.0 ** -8, 8 * 2.0 ** -24


def _sizes(x, n, pairs, interleaved):
    """|x| + |y| of the pair that an element belongs to (0: it does not turn)."""
    rows, P = x.shape[0], sum(pairs)
    a = np.abs(x.astype(np.float64)).reshape(rows, n, 3, -1)
    out = np.zeros_like(a)
    e, f = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if interleaved else (slice(0, P), slice(P, 2 * P))
    both = a[:, :, :2, e] + a[:, :, :2, f]
    out[:, :, :2, e] = out[:, :, :2, f] = both
    return out.reshape(rows, -1)


class Run:
    def __init__(self, b, s, h, n, q, pairs, dtype="bf16", at=(-1, -1), start=0, seed=0, scale=None, base=10000.0, **kw):
        rng = np.random.default_rng(seed + s)
        self.args, self.n, self.q, self.pairs, self.dtype, self.kw = (b, s, h, n, q, *at, opt.BF16 if dtype == "bf16" else opt.FP32), n, q, pairs, dtype, kw
        self.x = rng.standard_normal((b * s, 3 * h)).astype(np.float32)
        if dtype == "bf16":
            self.x = round_to_bf16(self.x)
        self.pos = (rng.integers(-3, 2000, (len(pairs), b * s)) + start).astype(np.int32)
        self.dev, self.dpos = mat_to_dev(self.x, q, dtype), torch.from_numpy(self.pos).to(DEV)
        self.scale, self.base = scale, base
        self.axes = opt.make_rotary(self.dpos, pairs, base=base, scale=scale, interleaved=kw.get("interleaved", False),
                                    in_turn=kw.get("in_turn", False), shared=kw.get("shared", False))

    def want(self, back=False):
        return orot.rotate(self.x, self.pos, self.n, self.pairs, scale=self.scale, base=self.base, back=back, **self.kw)

    def close(self, y, back=False):
        got, want = mat_to_host(y, *self.x.shape, self.q).astype(np.float64), self.want(back)
        size = _sizes(self.x, self.n, self.pairs, self.kw.get("interleaved", False))
        assert np.all(np.abs(got - want) <= np.where(size > 0, FP32 * size + (HALF * np.abs(want) * (1 + FP32) if self.dtype == "bf16" else 0), 0))

    def go(self):
        print("rotary", self.args, self.pairs, self.kw, flush=True)
        for back, call in ((False, opt.rotary), (True, opt.rotary_bwd)):
            y = empty(self.x.size, self.dtype)
            call(self.dev, y, *self.args, self.axes)
            z = self.dev.clone()
            call(z, z, *self.args, self.axes)
            torch.cuda.synchronize()
            self.close(y, back)
            assert torch.equal(y.view(torch.uint8), z.view(torch.uint8))       # in place: the same bits
        return self


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("b,s,h,n,q,pairs", [(1, 1, 64, 1, 1, (32,)), (8, 1, 256, 4, 1, (16, 16)), (4, 37, 256, 4, 2, (8, 12, 12)), (2, 130, 160, 4, 2, (20,)),
                                             (2, 19, 160, 4, 2, (3, 5, 7, 1)), (3, 50, 36, 3, 1, (2, 3)), (2, 33, 512, 2, 1, (64, 40, 24)),
                                             (4, 300, 512, 8, 2, (1,)), (1, 5, 1000, 500, 1, (1,)), (2, 700, 2048, 16, 1, (32, 16, 16)),
                                             (1, 3, 4096, 1, 1, (100, 28)), (4, 6, 8, 4, 4, (1,)), (2, 9, 42, 3, 1, (5,))])
def test_against_the_oracle(b, s, h, n, q, pairs, dtype, interleaved):
    Run(b, s, h, n, q, pairs, dtype, interleaved=interleaved).go()


def test_odd_heads():
    Run(2, 21, 27, 3, 1, (2, 1), "bf16").go()
    Run(2, 21, 27, 3, 1, (4,), "fp32").go()


@pytest.mark.parametrize("kw", [dict(in_turn=True), dict(shared=True), dict(in_turn=True, shared=True), dict(in_turn=True, interleaved=True),
                                dict(scale=[0.25, 3.0, 1e-3]), dict(base=1e6), dict(base=0.5)])
def test_ladders(kw):
    for dtype in ("bf16", "fp32"):
        Run(2, 60, 256, 2, 1, (10, 30, 24), dtype, **kw).go()


@pytest.mark.parametrize("start", [10 ** 6, 2 ** 31 - 3000, -2 ** 31 + 3])
def test_far_positions(start):
    """64-bit products of up to 2^31 and a frequency of 1 / (2 pi) are right to 2^-24 of a turn: the bound has room for that."""
    Run(2, 60, 128, 2, 1, (12, 20), "fp32", start=start).go()
    Run(2, 60, 128, 2, 1, (12, 20), "bf16", start=start, interleaved=True).go()


def test_one_device_writes_its_block():
    for dtype in ("bf16", "fp32"):
        full = Run(4, 45, 256, 4, 2, (8, 20), dtype).go()
        whole = empty(full.x.size, dtype)
        opt.rotary(full.dev, whole, *full.args, full.axes)
        for dev in ((0, 1), (1, 0)):
            one = Run(4, 45, 256, 4, 2, (8, 20), dtype, at=dev)
            y = empty(one.x.size, dtype)
            opt.rotary(one.dev, y, *one.args, one.axes)
            torch.cuda.synchronize()
            k = 2 * dev[0] + dev[1]
            assert torch.equal(y.view(4, -1)[k], whole.view(4, -1)[k]) and torch.isnan(y.view(4, -1)[[e for e in range(4) if e != k]]).all()


def test_matrices_that_start_at_any_element():
    for dtype, pairs, interleaved in (("bf16", (64,), False), ("fp32", (40, 24), True)):
        r = Run(2, 70, 256, 2, 1, pairs, dtype, interleaved=interleaved)
        room = torch.zeros(r.x.size + 3, dtype=r.dev.dtype, device=DEV)
        room[1:-2] = r.dev
        y = empty(r.x.size + 5, dtype)
        opt.rotary(room[1:], y[3:], *r.args, r.axes)
        torch.cuda.synchronize()
        r.close(y[3:-2])
        assert torch.isnan(y[:3]).all() and torch.isnan(y[-2:]).all()


def test_values_that_are_not_finite_stay_in_their_pair():
    r = Run(2, 40, 128, 2, 1, (16,), "bf16")
    r.dev.view(80, 2, 3, 64)[3, 1, 0, 5] = float("inf")
    r.dev.view(80, 2, 3, 64)[4, 0, 2, 7] = float("nan")     # a value: moved, not turned
    y = empty(r.x.size, "bf16")
    opt.rotary(r.dev, y, *r.args, r.axes)
    torch.cuda.synchronize()
    bad = torch.nonzero(~torch.isfinite(y.view(80, 2, 3, 64).float())).tolist()
    assert all(e in ([3, 1, 0, 5], [3, 1, 0, 21], [4, 0, 2, 7]) for e in bad) and [4, 0, 2, 7] in bad


def test_captured_and_on_another_stream():
    r = Run(2, 300, 256, 4, 1, (16, 16), "bf16")
    y, z = empty(r.x.size, "bf16"), empty(r.x.size, "bf16")
    opt.rotary(r.dev, y, *r.args, r.axes)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.rotary(r.dev, y, *r.args, r.axes)
        opt.rotary_bwd(y, z, *r.args, r.axes)
    for k in range(4):
        r.dpos += 17 * k
        r.pos += 17 * k
        y.fill_(float("nan")), z.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        r.close(y)
        assert (z.float() - r.dev.float()).abs().max() <= 3 * HALF * 6      # there and back: two roundings of numbers below 6 * sqrt(2)
    st = torch.cuda.Stream()
    y.fill_(float("nan"))
    torch.cuda.synchronize()
    opt.rotary(r.dev, y, *r.args, r.axes, stream=st)
    st.synchronize()
    r.close(y)


def test_a_matrix_of_more_than_2_to_the_32_bytes():
    """2^20 rows of 6144 elements: rows at the ends and in the middle against a call of those rows alone."""
    s, h, n, pairs = 1 << 20, 2048, 16, (24, 40)
    x = torch.empty(s * 3 * h, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)
    for at in range(0, x.numel(), 1 << 28):
        x[at:at + (1 << 28)] = torch.randn(min(1 << 28, x.numel() - at), generator=gen, device=DEV)
    pos = torch.randint(0, 1 << 20, (2, s), generator=gen, device=DEV, dtype=torch.int32)
    y = torch.empty_like(x)
    opt.rotary(x, y, 1, s, h, n, 1, 0, 0, opt.BF16, opt.make_rotary(pos, pairs))
    torch.cuda.synchronize()
    for at in (0, 349520, 700000, s - 50):
        part = pos[:, at:at + 50].contiguous()
        rows = slice(at * 3 * h, (at + 50) * 3 * h)
        few = empty(50 * 3 * h, "bf16")
        opt.rotary(x[rows], few, 1, 50, h, n, 1, 0, 0, opt.BF16, opt.make_rotary(part, pairs))
        torch.cuda.synchronize()
        assert torch.equal(few, y[rows])
