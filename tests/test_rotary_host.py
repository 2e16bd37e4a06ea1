"""CPU: the oracle of the rotary positions against closed forms, and the entry points' refusals."""
import ctypes

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import rotary as orot


def test_ladder():
    assert orot.ladder([4]) == [(0, 1.0), (0, 10000.0 ** -0.25), (0, 10000.0 ** -0.5), (0, 10000.0 ** -0.75)]
    assert orot.ladder([2, 1], base=100.0) == [(0, 1.0), (0, 0.1), (1, 1.0)]
    assert orot.ladder([1, 3, 2], base=64.0, in_turn=True) == [(0, 1.0), (1, 1.0), (2, 1.0), (1, 0.25), (2, 0.125), (1, 64.0 ** (-2 / 3))]
    assert [f for _, f in orot.ladder([1, 3], base=16.0, shared=True)] == [1.0, 0.5, 0.25, 0.125]
    assert [a for a, _ in orot.ladder([2, 2], in_turn=True, shared=True)] == [0, 1, 0, 1]


def test_products_depend_on_differences_only():
    """q . k after the turn is that of the difference of positions; values and further elements stay; the gradient turns back."""
    rng = np.random.default_rng(0)
    n, d, pairs = 2, 12, [2, 3]
    x = rng.standard_normal((1, 3 * n * d))
    for interleaved in (False, True):
        def dots(t, u):
            y = orot.rotate(np.repeat(x, 2, 0), np.array([[t[0], u[0]], [t[1], u[1]]]), n, pairs, interleaved=interleaved).reshape(2, n, 3, d)
            return np.einsum("he,he->h", y[0, :, 0], y[1, :, 1])
        assert np.allclose(dots((5, -3), (2, 4)), dots((105, 17), (102, 24)), atol=1e-12)
        assert not np.allclose(dots((5, -3), (2, 4)), dots((5, -3), (2, 5)), atol=1e-3)
        y = orot.rotate(x, np.array([[7], [9]]), n, pairs, interleaved=interleaved)
        assert np.array_equal(y.reshape(1, n, 3, d)[:, :, 2], x.reshape(1, n, 3, d)[:, :, 2])
        assert np.array_equal(y.reshape(1, n, 3, d)[..., 10:], x.reshape(1, n, 3, d)[..., 10:])
        assert np.allclose(orot.rotate(y, np.array([[7], [9]]), n, pairs, interleaved=interleaved, back=True), x, atol=1e-14)
    # one pair, a quarter of a turn
    y = orot.rotate(np.array([[1.0, 2.0, 3.0, 4.0, 5.0, 6.0]]), np.array([[1]]), 1, [1], scale=[np.pi / 2])
    assert np.allclose(y, [[-2.0, 1.0, -4.0, 3.0, 5.0, 6.0]])


def test_gradient_is_the_transpose():
    rng = np.random.default_rng(1)
    x, g = rng.standard_normal((2, 5, 3 * 2 * 8))
    pos = rng.integers(-50, 50, (2, 5))
    kw = dict(in_turn=True, interleaved=True, shared=True)
    assert np.isclose((orot.rotate(x, pos, 2, [1, 2], **kw) * g).sum(), (x * orot.rotate(g, pos, 2, [1, 2], back=True, **kw)).sum())


def _axes(**kw):
    a = opt.make_rotary(4096, kw.pop("pairs", (16,)))
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _rc(axes, x=1 << 20, y=1 << 24, b=4, s=10, h=128, n=4, q=2, i=0, j=1, dtype=opt.BF16):
    f, g = opt.lib().optimus_rotary, opt.lib().optimus_rotary_bwd
    a = ctypes.byref(axes) if axes is not None else None
    codes = {k(x, y, b, s, h, n, q, i, j, dtype, a, None) for k in (f, g)}
    assert len(codes) == 1
    return codes.pop()


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), opt.EINVAL), (dict(y=None), opt.EINVAL), (dict(dtype=2), opt.EDTYPE), (dict(b=3), opt.ESHAPE), (dict(n=6), opt.ESHAPE),
    (dict(h=130), opt.ESHAPE), (dict(s=0), opt.ESHAPE), (dict(q=0), opt.ESHAPE), (dict(i=2), opt.ECOORD), (dict(i=-1), opt.ECOORD),
    (dict(h=48), opt.ESHAPE), (dict(x=(1 << 20) + 1), opt.EINVAL), (dict(y=(1 << 24) + 2, dtype=opt.FP32), opt.EINVAL),
    (dict(y=(1 << 20) + 2), opt.EINVAL), (dict(y=(1 << 20) - 2, i=-1, j=-1), opt.EINVAL), (dict(h=4 * 4104), opt.ESHAPE),
    (dict(h=1 << 19, n=1 << 14), opt.ESHAPE)])
def test_refuses_calls(kw, code):
    assert _rc(_axes(), **kw) == code


def test_refuses_axes():
    assert _rc(None) == opt.EINVAL
    for kw, code in ((dict(positions=None), opt.EINVAL), (dict(positions=4098), opt.EINVAL), (dict(axes=0), opt.EINVAL), (dict(axes=5), opt.EINVAL),
                     (dict(base=0.0), opt.EINVAL), (dict(base=float("nan")), opt.EINVAL), (dict(base=float("inf")), opt.EINVAL), (dict(pairs=(17,)), opt.ESHAPE),
                     (dict(pairs=(8, 0)), opt.ESHAPE), (dict(pairs=(8, -1)), opt.ESHAPE), (dict(pairs=(2, 2, 2, 11)), opt.ESHAPE)):
        assert _rc(_axes(**kw)) == code, kw
    bad = _axes(pairs=(4, 4))
    bad.scale[1] = float("inf")
    assert _rc(bad) == opt.EINVAL
    bad.scale[1] = 1e7                                    # a position of 2^31 would have no turn behind the point
    assert _rc(bad) == opt.EINVAL and _rc(_axes(base=1e-9)) == opt.EINVAL
    assert _rc(_axes(pairs=(129,)), h=4 * 512) == opt.ESHAPE
    assert _rc(_axes(pairs=(3,), interleaved=1), h=4 * 9) == opt.ESHAPE        # a head of odd width
    for pairs, scale in (((), None), ((1, 1, 1, 1, 1), None), ((4, 4), [1.0])):
        with pytest.raises(opt.OptimusError) as e:
            opt.make_rotary(4096, pairs, scale=scale)
        assert e.value.code == opt.EINVAL


def test_refuses_tensors():
    torch = pytest.importorskip("torch")
    for t, code in ((torch.zeros(2, 8, dtype=torch.int64), opt.EDTYPE), (torch.zeros(2, 8), opt.EDTYPE), (torch.zeros(8, 2, dtype=torch.int32).t(), opt.EINVAL)):
        with pytest.raises(opt.OptimusError) as e:
            opt.make_rotary(t, (4, 4))
        assert e.value.code == code


@pytest.mark.parametrize("kw", [dict(b=65536, s=1, n=65536, h=65536 * 32, q=65536, i=-1, j=-1), dict(b=46341, s=1, n=46341, h=46341 * 32, q=46341, i=0, j=0),
                                dict(b=8192, s=1, n=8192 * 2, h=8192 * 87382, q=8192, i=0, j=0)])
def test_refuses_sizes_past_32_bits(kw):
    """Grids of 2^31 devices and more, rows of 2^31 columns."""
    assert _rc(_axes(), **kw) == opt.ESHAPE
