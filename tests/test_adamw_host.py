"""CPU: the oracle of the AdamW step against hand-computed steps, its 8-bit numbers, its random bits; the entry point's refusals."""
import ctypes

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import adamw as oad


def test_step_by_hand():
    # first step from zero moments: both corrected moments are g and g^2, so the update is lr * sign(g) (eps aside)
    w, m, v = oad.step(np.array([1.0, -2.0]), np.zeros(2), np.zeros(2), [[0.5, -3.0]], lr=0.1, beta1=0.9, beta2=0.99, eps=0.0, t=1, decay=0.0)
    assert np.allclose(w, [0.9, -1.9], atol=1e-15) and np.allclose(m, [0.05, -0.3]) and np.allclose(v, [0.0025, 0.09])
    # two parts and a scale are one gradient; the decay is apart from the moments
    a = oad.step(np.array([2.0]), [0.1], [0.2], [[1.0], [3.0]], lr=0.1, beta1=0.5, beta2=0.5, eps=1e-3, t=2, decay=0.25, grad_scale=0.5)
    b = oad.step(np.array([2.0]), [0.1], [0.2], [[2.0]], lr=0.1, beta1=0.5, beta2=0.5, eps=1e-3, t=2, decay=0.0)
    assert np.allclose(a[0], b[0] - 0.1 * 0.25 * 2.0) and np.allclose(a[1], b[1]) and np.allclose(a[2], b[2])
    # m = 1.05, v = 2.1; / 0.75: 1.4 / (sqrt(2.8) + 1e-3)
    assert np.allclose(b[0], 2.0 - 0.1 * 1.4 / (np.sqrt(2.8) + 1e-3))


def test_eight_bit_numbers():
    v = oad.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x7E] == 448 and v[0x38] == 1.0 and v[0xB8] == -1.0 and np.isnan(v[0x7F])
    torch = pytest.importorskip("torch")
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(np.nan_to_num(t, nan=-1e9), np.nan_to_num(v, nan=-1e9))
    rng = np.random.default_rng(0)
    x = rng.standard_normal(1000) * np.exp(3 * rng.standard_normal(1000))
    for positive in (False, True):
        y = np.abs(x) if positive else x
        up = oad.pack(y, np.full(1000, 65535, dtype=np.uint64), positive)
        down = oad.pack(y, np.zeros(1000, dtype=np.uint64), positive)
        assert np.array_equal(up[1], down[1])
        scale = np.repeat(2.0 ** (up[1] - 127.0), 128)[:1000]
        assert np.all(np.isin(up[0], v)) and np.all(np.isin(down[0], v))
        assert np.all(np.abs(up[0]) * scale >= np.abs(y) * (1 - 1e-4)) and np.all(np.abs(up[0]) <= 448)
        assert np.all((np.abs(down[0]) * scale <= np.abs(y)) | (positive & (down[0] == 2.0 ** -9)))
        assert np.all(np.abs(up[0] - down[0]) <= np.maximum(np.abs(down[0]) / 8, 2.0 ** -9))
    assert np.all(oad.pack(np.full(128, 1e-30), np.zeros(128, dtype=np.uint64), True)[0] > 0)
    assert list(oad.pack(np.array([1.0] * 128 + [np.nan] + [2.0] * 5), np.zeros(134, dtype=np.uint64), False)[1]) == [127 - 8, 255]


def test_random_bits_round_without_bias():
    """The mean of a value rounded at random many times is the value: 2^20 draws of a 16-bit number that is uniform have a mean within
    5 standard deviations, 5 / sqrt(12 * 2^20) of the step; the 16 high and low bits and the second hash are tested alike."""
    n = 1 << 20
    h = oad.random_bits(seed=12345678901, step=7, tensor=3, n=n)
    second = oad.mix(h ^ np.uint64(0x6A09E667)) & np.uint64(0xFFFF)
    bound = 5 / np.sqrt(12 * n)
    for bits in (h >> np.uint64(16), h & np.uint64(0xFFFF), second):
        f = bits.astype(np.float64) / 65536
        assert abs(f.mean() - (0.5 - 0.5 / 65536)) < bound
        for place in (0.001, 0.3, 0.9):     # share that is rounded up
            assert abs(np.floor(place + f).mean() - place) < 5 * np.sqrt(place * (1 - place) / n) + 1 / 65536
        assert abs(np.corrcoef(f[:-1], f[1:])[0, 1]) < 5 / np.sqrt(n)
    a, b = (oad.random_bits(seed=1, step=s, tensor=0, n=n) >> np.uint64(16) for s in (1, 2))
    assert abs(np.corrcoef(a.astype(float), b.astype(float))[0, 1]) < 5 / np.sqrt(n)
    far = oad.random_bits(seed=1, step=1, tensor=0, n=4096, first=1 << 32)
    assert np.mean(far == oad.random_bits(seed=1, step=1, tensor=0, n=4096)) < 0.01


def _tensor(**kw):
    t = opt.AdamwTensor(param=4096, master=None, grad=8192, m=12288, v=16384, m_scale=None, v_scale=None, n=100, param_dtype=opt.FP32,
                        grad_dtype=opt.FP32, grad_parts=1, weight_decay=0.0)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _rc(cfg, tensors, count=None):
    arr = (opt.AdamwTensor * max(1, len(tensors)))(*tensors)
    return opt.lib().optimus_adamw_step(ctypes.byref(cfg) if cfg is not None else None, arr, len(tensors) if count is None else count, None)


@pytest.mark.parametrize("change,code", [
    (dict(param=None), opt.EINVAL), (dict(grad=None), opt.EINVAL), (dict(m=None), opt.EINVAL), (dict(v=None), opt.EINVAL),
    (dict(m_scale=4096), opt.EINVAL), (dict(v_scale=4096), opt.EINVAL), (dict(n=0), opt.ESHAPE), (dict(n=-5), opt.ESHAPE),
    (dict(n=(1 << 34) + 1), opt.ESHAPE), (dict(param_dtype=2), opt.EDTYPE), (dict(grad_dtype=-1), opt.EDTYPE),
    (dict(grad_parts=0), opt.ESHAPE), (dict(master=32768), opt.EINVAL), (dict(weight_decay=float("nan")), opt.EINVAL),
    (dict(param=4098), opt.EINVAL), (dict(grad=8193), opt.EINVAL), (dict(m=12290), opt.EINVAL), (dict(v=16385), opt.EINVAL),
    (dict(param_dtype=opt.BF16, param=4097), opt.EINVAL), (dict(param_dtype=opt.BF16, master=32770), opt.EINVAL)])
def test_refuses_tensors(change, code):
    assert _rc(opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, 1, 0), [_tensor(**change)]) == code


@pytest.mark.parametrize("change", [dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=float("nan")), dict(eps=0.0),
                                    dict(eps=float("inf")), dict(eps=1e-50), dict(step=0)])
def test_refuses_settings(change):
    cfg = opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, 1, 0)
    for k, v in change.items():
        setattr(cfg, k, v)
    assert _rc(cfg, [_tensor()]) == opt.EINVAL


def test_refuses_lists():
    cfg = opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, 1, 0)
    assert _rc(None, [_tensor()]) == opt.EINVAL
    assert opt.lib().optimus_adamw_step(ctypes.byref(cfg), None, 1, None) == opt.EINVAL
    assert _rc(cfg, [], 0) == opt.ESHAPE and _rc(cfg, [_tensor()], -1) == opt.ESHAPE
    # the same parameter twice, or two that share elements, also in long lists
    assert _rc(cfg, [_tensor(), _tensor()]) == opt.EINVAL
    assert _rc(cfg, [_tensor(), _tensor(param=4096 + 396)]) == opt.EINVAL
    many = [_tensor(param=1 << 20 | k << 12) for k in range(100)] + [_tensor(param=(1 << 20) + 399 & ~3)]
    assert _rc(cfg, many) == opt.EINVAL


def test_stack_step_refusals():
    """Before anything is enqueued, without a GPU."""
    cfg = opt.LayerCfg(4, 64, 128, 4, 2, 1e-5, 1, opt.BF16, 0)
    assert opt.stack_adamw_elements(cfg) == 12 * 128 * 128 + 13 * 128
    assert opt.stack_adamw_elements(opt.LayerCfg(3, 64, 128, 4, 2, 1e-5, 1, opt.BF16, 0)) == 0
    elements = opt.stack_adamw_elements(opt.LayerCfg(1, 8, 40, 1, 1, 1e-5, 1, opt.BF16, 0))   # vectors of 40 start 128 apart
    assert elements == sum(-(-n // 128) * 128 for n in (4800, 1600, 6400, 6400, 120, 40, 160, 40, 40, 40, 40, 40))
    adamw, place = opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, 1, 0), iter(range(1 << 20, 1 << 40, 1 << 20))

    def layer():
        return opt.LayerParams(*[next(place) for _ in opt.LAYER_PARAM_FIELDS])

    def rc(params, states=None, cfg=cfg, adamw=adamw, grad=next(place), buf=None):
        pa = (opt.LayerParams * len(params))(*params)
        states = states or [opt.AdamwState(next(place), next(place), None, None, None) for _ in params]
        sa = (opt.AdamwState * len(states))(*states)
        buf = buf or opt.StackBuffers(*[next(place) for _ in range(5)])
        return opt.lib().optimus_stack_bwd_adamw(ctypes.byref(cfg), len(params), pa, sa, ctypes.byref(adamw), 0.1, grad, next(place), ctypes.byref(buf),
                                                 next(place), None)

    a, b = layer(), layer()
    assert rc([a, b], cfg=opt.LayerCfg(3, 64, 128, 4, 2, 1e-5, 1, opt.BF16, 0)) == opt.ESHAPE
    assert rc([a, b], adamw=opt.AdamwCfg(1e-3, 1.0, 0.99, 1e-8, 1, 0)) == opt.EINVAL
    assert rc([a, b], grad=None) == opt.EINVAL
    assert rc([a, a]) == opt.EINVAL                       # layers that share parameters
    b.w2 = a.w1
    assert rc([a, b]) == opt.EINVAL
    b.w2 = None
    assert rc([a, b]) == opt.EINVAL
    assert rc([a], states=[opt.AdamwState(next(place), None, None, None, None)]) == opt.EINVAL
    assert rc([a], states=[opt.AdamwState(next(place), next(place), next(place), None, None)]) == opt.EINVAL
    assert rc([a], buf=opt.StackBuffers(next(place), None, next(place), next(place), next(place))) == opt.EINVAL
    with pytest.raises(opt.OptimusError):
        opt.stack_bwd_adamw(cfg, [a], [], adamw, 0.1, 4096, 4096, opt.StackBuffers(), 4096)
