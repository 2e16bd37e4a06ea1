"""GPU parity: the AdamW step over many tensors against the oracle in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import adamw as oad
from gpu_util import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def _cfg(step, seed=0, **kw):
    return opt.AdamwCfg(H["lr"], H["beta1"], H["beta2"], H["eps"], step, seed, **kw)


class Case:
    """One tensor: host values in 64 bits (exactly those on the device) and device buffers, `at` elements into larger ones."""

    def __init__(self, rng, n, param="fp32", master=False, eight=False, grad="fp32", parts=1, decay=0.0, at=0):
        td = {"fp32": torch.float32, "bf16": torch.bfloat16}
        self.n, self.parts, self.decay, self.eight, self.at = n, parts, decay, eight, at

        def dev(x, dtype):
            whole = torch.full((at + x.size + 8,), 77, dtype=dtype, device=DEV)
            whole[at:at + x.size] = torch.from_numpy(np.ascontiguousarray(x)).to(DEV).to(dtype)
            return whole, whole[at:at + x.size]

        w = rng.standard_normal(n).astype(np.float32)
        g = (rng.standard_normal(parts * n) * np.exp(rng.standard_normal(parts * n))).astype(np.float32)
        self.whole = {}
        self.whole["param"], self.param = dev(w, td[param])
        self.whole["grad"], self.grad = dev(g, td[grad])
        self.master = None
        if master:
            self.whole["master"], self.master = dev(w, torch.float32)
        self.m_scale = self.v_scale = None
        if eight:
            codes = rng.integers(0, 256, (2, n)).astype(np.uint8)
            codes[0][(codes[0] & 127) == 127] = 0
            codes[1] &= 127
            codes[1][codes[1] == 127] = 126
            groups = -(-n // 128)
            self.whole["m"], self.m = dev(codes[0], torch.uint8)
            self.whole["v"], self.v = dev(codes[1], torch.uint8)
            self.whole["m_scale"], self.m_scale = dev(rng.integers(117, 121, groups).astype(np.uint8), torch.uint8)
            self.whole["v_scale"], self.v_scale = dev(rng.integers(114, 121, groups).astype(np.uint8), torch.uint8)
        else:
            self.whole["m"], self.m = dev(rng.standard_normal(n).astype(np.float32), torch.float32)
            self.whole["v"], self.v = dev(rng.standard_normal(n).astype(np.float32) ** 2, torch.float32)

    def entry(self):
        return dict(param=self.param, master=self.master, grad=self.grad, m=self.m, v=self.v, m_scale=self.m_scale, v_scale=self.v_scale,
                    n=self.n, grad_parts=self.parts, weight_decay=self.decay)

    def moments(self):
        if self.eight:
            return [oad.unpack(c.cpu().numpy(), s.cpu().numpy()) for c, s in ((self.m, self.m_scale), (self.v, self.v_scale))]
        return to_host(self.m).astype(np.float64), to_host(self.v).astype(np.float64)

    def want(self, t, grad_scale=1.0):
        w = to_host(self.master if self.master is not None else self.param).astype(np.float64)
        m, v = self.moments()
        return oad.step(w, m, v, to_host(self.grad).astype(np.float64).reshape(self.parts, self.n), t=t, decay=self.decay, grad_scale=grad_scale, **H)

    def check(self, want, index, t, seed):
        """fp32: m and v take at most parts + 4 roundings of terms that do not cancel beyond |b1 m| + |c1 g|; w's update is lr times a
        quotient of them.  bf16: half a step to nearest, else one of the two neighbours that the random bits name."""
        w, m, v = want
        eps = 2.0 ** -24 * (self.parts + 8)
        gm = np.abs(to_host(self.grad).astype(np.float64).reshape(self.parts, self.n)).sum(0)
        got = to_host(self.master if self.master is not None else self.param).astype(np.float64)
        size = np.abs(w) + 2 * H["lr"] * (np.abs(m) + gm) / (np.sqrt(np.maximum(v, 1e-30)) * 1.0) / (1 - H["beta1"] ** t)
        bits = oad.random_bits(seed, t, index, self.n)
        if self.master is not None:
            assert np.all(np.abs(got - w) <= 4 * eps * size)
            p = to_host(self.param).astype(np.float64)
            assert np.all(np.abs(p - got) <= 2.0 ** -8 * np.abs(got))
            assert torch.equal(self.param, self.master.to(torch.bfloat16))
        elif self.param.dtype == torch.bfloat16:
            p = oad.round_bf16_random(w, oad.mix(bits ^ np.uint64(0x6A09E667)) & np.uint64(0xFFFF))
            off = np.abs(got - p)
            assert np.all(off <= 2.0 ** -7 * np.abs(w) + 4 * eps * size)
            # the other neighbour only where fp32's own error, a 2^-14th of a step or so, decides
            assert np.mean(off > 0) <= 2e-3 + 2.0 / self.n
        else:
            assert np.all(np.abs(got - w) <= 4 * eps * size)
        if not self.eight:
            old_m, old_v = gm, gm * gm
            assert np.all(np.abs(to_host(self.m) - m) <= 4 * eps * (np.abs(m) + old_m))
            assert np.all(np.abs(to_host(self.v) - v) <= 4 * eps * (np.abs(v) + old_v))
            return
        for code, byte, x, dither, positive in ((self.m, self.m_scale, m, bits >> np.uint64(16), False),
                                                (self.v, self.v_scale, v, bits & np.uint64(0xFFFF), True)):
            val, scale = oad.pack(x, dither, positive)
            b = byte.cpu().numpy().astype(np.int64)
            assert np.mean(b != scale) <= 1e-3 + (0 if self.n > 1000 else 0), "scales"
            got = oad.e4m3_values()[code.cpu().numpy()]
            same = np.repeat(b == scale, 128)[:self.n]
            off = np.abs(got - val)[same]
            assert np.all(off <= np.maximum(np.abs(val[same]) / 4, 2.0 ** -9))   # a neighbour at most
            assert np.mean(off > 0) <= 1e-3 + 1.0 / self.n                        # m's fp32 error is some 1e-5 of a step, more where it cancels

    def untouched(self):
        for name, whole in self.whole.items():
            used = getattr(self, name).numel()
            assert torch.all(whole[:self.at] == 77) and torch.all(whole[self.at + used:] == 77), name


KINDS = [dict(), dict(param="bf16", master=True), dict(param="bf16"), dict(param="bf16", grad="bf16", decay=0.1), dict(eight=True),
         dict(param="bf16", eight=True, decay=0.1), dict(param="bf16", master=True, eight=True, grad="bf16"), dict(parts=4, decay=0.1),
         dict(parts=3, eight=True, grad="bf16")]


@pytest.mark.parametrize("kind", range(len(KINDS)))
@pytest.mark.parametrize("n", [1, 7, 8, 127, 128, 129, 2048, 5003])
def test_one_tensor(n, kind):
    """Every combination of types at sizes around a lane's, a scale's and a workgroup's share; aligned and at odd elements."""
    for at in (0, 1, 3):
        rng = np.random.default_rng(n * 100 + kind * 10 + at)
        c = Case(rng, n, at=at, **KINDS[kind])
        t, seed = 1 + kind, 5 + (kind << 33)
        want = c.want(t)
        print("adamw", n, KINDS[kind], at, flush=True)
        opt.adamw_step(_cfg(t, seed), opt.make_adamw_tensors([c.entry()]))
        torch.cuda.synchronize()
        c.check(want, 0, t, seed)
        c.untouched()


def test_many_tensors_of_all_kinds():
    """More than one launch's worth, sizes mixed; gradients scaled by a number on the device."""
    rng = np.random.default_rng(1)
    cases = [Case(rng, int(rng.integers(1, 6000)), **KINDS[k % len(KINDS)]) for k in range(95)]
    gs = torch.tensor([0.25], device=DEV)
    want = [c.want(9, 0.25) for c in cases]
    opt.adamw_step(_cfg(9, 77, grad_scale=gs.data_ptr()), opt.make_adamw_tensors([c.entry() for c in cases]))
    torch.cuda.synchronize()
    for k, (c, w) in enumerate(zip(cases, want)):
        c.check(w, k, 9, 77)
        c.untouched()


def test_same_call_same_bits():
    rng = np.random.default_rng(2)
    runs = []
    for _ in range(2):
        rng = np.random.default_rng(2)
        cases = [Case(rng, 3001, **k) for k in KINDS]
        opt.adamw_step(_cfg(3, 11), opt.make_adamw_tensors([c.entry() for c in cases]))
        torch.cuda.synchronize()
        runs.append([c.whole[k].view(torch.uint8) for c in cases for k in c.whole])
    assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_zeroed_state_and_zero_gradients():
    for kind in (dict(), dict(eight=True), dict(param="bf16", eight=True)):
        rng = np.random.default_rng(3)
        c = Case(rng, 1000, **kind)
        for x in (c.m, c.v, c.grad) + ((c.m_scale, c.v_scale) if c.eight else ()):
            x.zero_()
        before = c.param.clone()
        opt.adamw_step(_cfg(1), opt.make_adamw_tensors([c.entry()]))
        torch.cuda.synchronize()
        assert torch.equal(c.param, before) and not c.m.any() and not c.v.any()


@pytest.mark.parametrize("eps", [1e-30, 1e-42])
def test_an_eps_next_to_zero(eps):
    """Gradients whose v is below the smallest normal number, 2^-126: the first step is still lr * sign(g), as long as g^2 keeps its digits.
    From 10^-19.5 on v is at least 1e-41; its two roundings of at most half of 2^-149 are 7e-5 of that, half as much of its root.  The
    decay and w take four roundings more.  A gradient of zero leaves its weight alone."""
    n = 1000
    g = np.logspace(-19.5, -16.5, n).astype(np.float32) * np.where(np.arange(n) % 3, 1, -1).astype(np.float32)
    g[::10] = 0
    w = torch.linspace(-1, 1, n, device=DEV)
    old, m, v = to_host(w).astype(np.float64), torch.zeros_like(w), torch.zeros_like(w)
    cfg = opt.AdamwCfg(H["lr"], H["beta1"], H["beta2"], eps, 1, 0)
    opt.adamw_step(cfg, opt.make_adamw_tensors([dict(param=w, grad=torch.from_numpy(g).to(DEV), m=m, v=v)]))
    torch.cuda.synchronize()
    want = oad.step(old, np.zeros(n), np.zeros(n), g[None].astype(np.float64), **dict(H, eps=eps), t=1, decay=0.0)[0]
    assert np.all(np.abs(to_host(w) - want) <= H["lr"] * 4e-5 + 2.0 ** -22 * (np.abs(old) + H["lr"]))
    assert np.array_equal(to_host(w)[::10], old[::10].astype(np.float32))


def test_gradient_that_is_not_finite():
    """fp32: its own element turns NaN or infinite.  8 bits: its group of 128; every other weight, moment and scale keeps its value."""
    for bad in (float("nan"), float("inf"), -float("inf")):
        for kind in (dict(), dict(eight=True), dict(eight=True, param="bf16")):
            c, d = (Case(np.random.default_rng(4), 700, **kind) for _ in range(2))
            c.grad[300] = bad
            opt.adamw_step(_cfg(2), opt.make_adamw_tensors([c.entry()]))
            opt.adamw_step(_cfg(2), opt.make_adamw_tensors([d.entry()]))
            torch.cuda.synchronize()
            mine, clean = torch.arange(700, device=DEV) != 300, None
            assert not torch.isfinite(c.param[300]) and torch.equal(c.param[mine], d.param[mine])
            group = torch.arange(700, device=DEV) // 128 != 2
            clean = group if c.eight else mine
            assert torch.equal(c.m[clean], d.m[clean]) and torch.equal(c.v[clean], d.v[clean])
            m, v = c.moments()
            assert not np.isfinite(m[300]) and not np.isfinite(v[300])
            if c.eight:
                assert np.all(np.isnan(m[256:384])) and np.all(np.isfinite(np.delete(m, np.arange(256, 384))))


def test_captured_step_with_its_numbers_on_the_device():
    """A graph replayed with another step, rate and gradient scale each time leaves the bits of eager calls with those numbers."""
    kinds = [dict(), dict(eight=True), dict(param="bf16", eight=True, decay=0.1), dict(param="bf16", master=True, decay=0.1)]
    a, b = ([Case(np.random.default_rng(50 + k), 4000 + k, **kw) for k, kw in enumerate(kinds)] for _ in range(2))
    step = torch.tensor([1], dtype=torch.int64, device=DEV)
    lr, gs = torch.tensor([1e-2], device=DEV), torch.tensor([1.0], device=DEV)
    cfg = _cfg(0, 9, grad_scale=gs.data_ptr(), lr_on_device=lr.data_ptr(), step_on_device=step.data_ptr())
    ta, tb = (opt.make_adamw_tensors([c.entry() for c in x]) for x in (a, b))
    opt.adamw_step(_cfg(1), opt.make_adamw_tensors([Case(np.random.default_rng(0), 10).entry()]))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.adamw_step(cfg, ta)
    for k in range(1, 5):
        step.fill_(k), lr.fill_(0.01 / k), gs.fill_(1.0 / k)
        g.replay()
        opt.adamw_step(cfg, tb)
        torch.cuda.synchronize()
        for x, y in zip(a, b):
            assert all(torch.equal(x.whole[n].view(torch.uint8), y.whole[n].view(torch.uint8)) for n in x.whole), k
    # the same numbers from the host: the correction terms are computed in 64 bits on either side
    c, d = (Case(np.random.default_rng(60), 3000) for _ in range(2))
    step.fill_(1000), lr.fill_(H["lr"]), gs.fill_(1.0)
    opt.adamw_step(cfg, opt.make_adamw_tensors([c.entry()]))
    opt.adamw_step(_cfg(1000, 9), opt.make_adamw_tensors([d.entry()]))
    torch.cuda.synchronize()
    assert torch.equal(c.m, d.m) and torch.allclose(c.param, d.param, rtol=2.0 ** -22, atol=2.0 ** -22)


def test_moments_of_8_bits_follow_those_of_32():
    """Two hundred steps of steady noisy gradients: v's 8-bit numbers, an eighth apart, keep moving (to nearest they would stand still at a
    change of a hundredth a step); their mean over 2^14 elements follows the 32-bit ones.  A step's rounding adds a variance of at most
    (v/8)^2/4, of which beta2 = 0.99 remembers 1 / (1 - 0.99^2) = 50: standard deviation of one element 0.44 v, of the mean 0.44 / 2^7 =
    0.0035 v, five of them 0.018."""
    n = 1 << 14
    rng = np.random.default_rng(6)
    a, b = Case(np.random.default_rng(7), n), Case(np.random.default_rng(7), n, eight=True)
    for c in (a, b):
        c.m.zero_(), c.v.zero_()
    b.m_scale.zero_(), b.v_scale.zero_()
    ta, tb = opt.make_adamw_tensors([a.entry()]), opt.make_adamw_tensors([b.entry()])
    for t in range(1, 201):
        g = torch.from_numpy((rng.standard_normal(n) * (1.0 if t <= 100 else 0.1)).astype(np.float32)).to(DEV)
        a.grad.copy_(g), b.grad.copy_(g)
        opt.adamw_step(_cfg(t, 3), ta)
        opt.adamw_step(_cfg(t, 3), tb)
    torch.cuda.synchronize()
    v32, v8 = a.moments()[1], b.moments()[1]
    assert abs(v8.mean() / v32.mean() - 1) < 0.018
    assert np.all(v8 > 0)


def test_other_stream():
    c, d = (Case(np.random.default_rng(8), 50000, eight=True) for _ in range(2))
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    opt.adamw_step(_cfg(2), opt.make_adamw_tensors([c.entry()]), stream=st)
    opt.adamw_step(_cfg(2), opt.make_adamw_tensors([d.entry()]))
    torch.cuda.synchronize()
    assert torch.equal(c.param, d.param) and torch.equal(c.m, d.m)
