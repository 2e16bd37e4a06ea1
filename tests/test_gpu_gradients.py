"""GPU parity: the norm of many gradients and the clipping by it against the oracle.

Squares and sums are 64 bits: a norm is off by its rounding to fp32, 2^-24 (with parts, whose sum is fp32: by (parts - 1) * 2^-24 of the sum of
their magnitudes as well); a clipped gradient by its rounding, 2^-24 or 2^-8 of itself, from the scale that the device holds."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import gradients as og
from workloads import round_to_bf16
from gpu_util import to_dev, to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = 2.0 ** -24


class Run:
    """kinds: (n, parts, dtype) each."""

    def __init__(self, kinds, seed=0, size=1.0, in_place=False, slack=0):
        rng = np.random.default_rng(seed)
        self.host, self.dev, entries = [], [], []
        for n, parts, dtype in kinds:
            g = (rng.standard_normal((parts, n)) * size * np.exp(rng.standard_normal())).astype(np.float32)
            g = round_to_bf16(g) if dtype == "bf16" else g
            t = to_dev(np.concatenate([np.full(slack, 7.0, dtype=np.float32), g.reshape(-1)]), dtype)[slack:]
            out = t if in_place else torch.full((n + slack,), float("nan"), dtype=t.dtype, device=DEV)[slack:]
            self.host.append(g), self.dev.append((t, out))
            entries.append(dict(grad=t, n=n, parts=parts, clipped=out))
        self.kinds, self.list = kinds, opt.make_gradients(entries)
        self.ws = torch.full((opt.gradient_norm_workspace_bytes(self.list),), 0xFF, dtype=torch.uint8, device=DEV)
        self.norm, self.scale, self.norms = (torch.full((k,), float("nan"), device=DEV) for k in (1, 1, len(kinds)))

    def go(self, max_norm, stream=None):
        print("gradients", len(self.kinds), self.kinds[:4], max_norm, flush=True)
        opt.gradient_norm(self.list, max_norm, self.norm, self.scale, self.norms, self.ws, stream=stream)
        opt.gradient_clip(self.list, self.scale, stream=stream)
        (stream or torch.cuda).synchronize()
        return self

    def check(self, max_norm):
        total, each = og.norm(self.host)
        err = np.array([U * (p - 1) * np.linalg.norm(np.abs(g.astype(np.float64)).sum(0)) for g, (_, p, _) in zip(self.host, self.kinds)])
        near = 1.01 * U
        assert np.all(np.abs(self.norms.cpu().numpy() - each) <= near * each + 1.01 * err)
        off = near * total + 1.01 * np.linalg.norm(err)
        assert abs(self.norm.item() - total) <= off
        want, got = og.scale(total, max_norm), self.scale.item()
        if abs(total - max_norm) > off:
            assert abs(got - want) <= want * (near + off / total) + 2.0 ** -149      # (the least number above zero)
        for g, (n, p, dtype), (_, out) in zip(self.host, self.kinds, self.dev):
            y, w = to_host(out[:n]).astype(np.float64), g.astype(np.float64).sum(0) * got
            half = 2.0 ** -8 if dtype == "bf16" else U
            assert np.all(np.abs(y - w) <= half * 1.01 * np.abs(w) + 1.01 * U * p * np.abs(g).sum(0) * abs(got) + 1e-45)
        return self


SIZES = (1, 2, 7, 8, 9, 2047, 2048, 2049, 4095, 4097, 8191, 8192, 8193, 16390, 100001)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("parts", [1, 2, 5])
def test_sizes(parts, dtype, in_place):
    for n in SIZES:
        Run([(n, parts, dtype)], seed=n, in_place=in_place).go(0.5).check(0.5)


@pytest.mark.parametrize("in_place", [False, True])
def test_lists(in_place):
    """Mixed types and parts at odd places, more tensors than one launch holds."""
    rng = np.random.default_rng(3)
    kinds = [(int(rng.choice(SIZES)) + k % 3, int(rng.choice([1, 1, 1, 2, 4])), str(rng.choice(["fp32", "bf16"]))) for k in range(300)]
    for slack in (0, 1, 3):
        Run(kinds, seed=slack, in_place=in_place, slack=slack).go(2.0).check(2.0)


def test_many_small_and_one_large():
    Run([(3, 1, "fp32")] * 5000 + [(20000003, 1, "bf16")] + [(64, 4, "fp32")] * 40).go(1.0).check(1.0)


@pytest.mark.parametrize("max_norm", [1e-20, 1.0, 1e30, float("inf")])
@pytest.mark.parametrize("size", [1e-30, 1.0, 1e25])
def test_ranges(size, max_norm):
    """Gradients whose squares fp32 does not hold."""
    Run([(5000, 1, "fp32"), (300, 2, "fp32"), (777, 1, "bf16")], size=size).go(max_norm).check(max_norm)


def test_a_scale_of_one_leaves_gradients_as_they_are():
    for in_place in (False, True):
        r = Run([(5000, 1, "fp32"), (300, 2, "fp32"), (777, 1, "bf16")], in_place=in_place).go(1e6)
        assert r.scale.item() == 1.0
        assert np.array_equal(to_host(r.dev[0][1][:5000]), r.host[0][0]) and np.array_equal(to_host(r.dev[2][1][:777]), r.host[2][0])
        assert np.array_equal(to_host(r.dev[1][1][:300]), r.host[1][0] + r.host[1][1])


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan")])
def test_gradients_that_are_not_finite(what):
    r = Run([(5000, 1, "fp32"), (4000, 1, "bf16")])
    r.dev[1][0][1234] = what
    r.go(1.0)
    assert not np.isfinite(r.norm.item()) and np.isnan(r.scale.item())
    each = r.norms.cpu().numpy()
    assert np.isfinite(each[0]) and not np.isfinite(each[1])
    assert torch.isnan(r.dev[0][1]).all() and torch.isnan(r.dev[1][1]).all()


def test_zero_gradients():
    r = Run([(5000, 1, "fp32"), (4000, 1, "bf16")], size=0.0).go(1.0)
    assert r.norm.item() == 0.0 and r.scale.item() == 1.0 and not r.norms.any() and not r.dev[0][1].any()


def test_without_scale_and_norms_and_the_same_bits():
    kinds = [(100001, 1, "fp32"), (300, 2, "fp32"), (70007, 1, "bf16")]
    a, b = Run(kinds).go(0.1), Run(kinds).go(0.1)
    for x, y in ((a.norm, b.norm), (a.scale, b.scale), (a.norms, b.norms), (a.dev[2][1], b.dev[2][1])):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    n = torch.zeros(1, device=DEV)
    opt.gradient_norm(a.list, 0.1, n, ws=a.ws)
    torch.cuda.synchronize()
    assert torch.equal(n, a.norm)
    # the place of a list's sum in its workspace does not matter, nor a larger one
    ws = torch.full((a.ws.numel() + 800,), 0xFF, dtype=torch.uint8, device=DEV)
    opt.gradient_norm(a.list, 0.1, n, ws=ws[8:])
    torch.cuda.synchronize()
    assert torch.equal(n, a.norm)


def test_captured_and_on_another_stream():
    kinds = [(100001, 1, "fp32"), (300, 3, "fp32"), (70007, 1, "bf16")]
    r = Run(kinds).go(0.1)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        opt.gradient_norm(r.list, 0.1, r.norm, r.scale, r.norms, r.ws)
        opt.gradient_clip(r.list, r.scale)
    for k in range(4):
        for h, (t, _) in zip(r.host, r.dev):
            h *= 2.0 ** (k - 4)
            t *= 2.0 ** (k - 4)
        for x in (r.norm, r.scale, r.norms, *(o for _, o in r.dev)):
            x.fill_(float("nan"))
        r.ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        r.check(0.1)
    st = torch.cuda.Stream()
    for x in (r.norm, r.scale, r.norms):
        x.fill_(float("nan"))
    torch.cuda.synchronize()
    r.go(0.1, stream=st).check(0.1)


def test_the_update_clips_by_the_scale():
    """optimus_adamw_step with grad_scale has the bits of a step from gradients clipped before (fp32: a product each)."""
    n, gen = 10007, torch.Generator(device=DEV)
    gen.manual_seed(0)
    made = lambda: torch.randn(n, generator=gen, device=DEV)   # noqa: E731
    p, g, m, v = made(), made(), made(), made().abs()
    grads = opt.make_gradients([dict(grad=g, clipped=torch.empty_like(g))])
    clipped = torch.empty_like(g)
    grads[0].clipped = clipped.data_ptr()
    norm, scale = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
    opt.gradient_norm(grads, 0.5, norm, scale, ws=torch.empty(opt.gradient_norm_workspace_bytes(grads), dtype=torch.uint8, device=DEV))
    opt.gradient_clip(grads, scale)
    left, right = ([x.clone() for x in (p, m, v)] for _ in range(2))
    for (w, a, b), grad, s in ((left, g, scale), (right, clipped, None)):
        cfg = opt.AdamwCfg(lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8, step=3, seed=1, grad_scale=s.data_ptr() if s is not None else None)
        opt.adamw_step(cfg, opt.make_adamw_tensors([dict(param=w, grad=grad, m=a, v=b)]))
    torch.cuda.synchronize()
    assert scale.item() < 0.01 and all(torch.equal(x, y) for x, y in zip(left, right))


def test_more_than_2_to_the_32_elements():
    n = (1 << 32) + 100003
    g = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    where = [0, (1 << 31) + 5, (1 << 32) - 1, 1 << 32, n - 1]
    for k, at in enumerate(where):
        g[at] = k + 1.0
    small = torch.full((1000,), 0.5, device=DEV)
    grads = opt.make_gradients([dict(grad=g), dict(grad=small)])
    norm, scale, norms = (torch.zeros(k, device=DEV) for k in (1, 1, 2))
    opt.gradient_norm(grads, 0.25, norm, scale, norms, torch.empty(opt.gradient_norm_workspace_bytes(grads), dtype=torch.uint8, device=DEV))
    opt.gradient_clip(grads, scale)
    torch.cuda.synchronize()
    total = np.sqrt(1 + 4 + 9 + 16 + 25 + 250)
    assert abs(norm.item() - total) <= 2 * U * total and abs(scale.item() - 0.25 / total) <= 2 * U * 0.25 / total
    got = torch.stack([g[at] for at in where]).float().cpu().numpy()
    want = np.arange(1, 6) * scale.item()
    assert np.all(np.abs(got - want) <= 2.0 ** -8 * want) and int((g != 0).sum()) == 5
