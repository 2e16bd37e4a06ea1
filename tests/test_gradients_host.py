"""CPU: the oracle of the gradients' norm, the entry points' refusals."""
import ctypes

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import gradients as og

torch = pytest.importorskip("torch")


def test_oracle():
    total, each = og.norm([np.array([[3.0, 0.0], [0.0, 4.0]]), np.array([[1.0, -2.0, 2.0]])])
    assert np.isclose(total, np.sqrt(34)) and np.allclose(each, [5.0, 3.0])
    assert og.scale(10.0, 2.0) == 0.2 and og.scale(1.0, 2.0) == 1.0 and og.scale(5.0, np.inf) == 1.0 and np.isnan(og.scale(np.inf, 1.0))


def _g(**kw):
    g = opt.Gradient(1 << 20, 1 << 24, 100, opt.FP32, 1)
    for k, v in kw.items():
        setattr(g, k, v)
    return g


def _norm(gs, count=None, max_norm=1.0, norm=4096, ws=8192, nbytes=1 << 20):
    arr = (opt.Gradient * max(1, len(gs)))(*gs)
    return opt.lib().optimus_gradient_norm(arr, len(gs) if count is None else count, max_norm, norm, None, None, ws, nbytes, None)


def _clip(gs, count=None, scale=4096):
    arr = (opt.Gradient * max(1, len(gs)))(*gs)
    return opt.lib().optimus_gradient_clip(arr, len(gs) if count is None else count, scale, None)


@pytest.mark.parametrize("change,code", [(dict(grad=None), opt.EINVAL), (dict(n=0), opt.ESHAPE), (dict(n=(1 << 34) + 1), opt.ESHAPE), (dict(parts=0), opt.ESHAPE),
                                         (dict(parts=65537), opt.ESHAPE), (dict(dtype=2), opt.EDTYPE), (dict(grad=(1 << 20) + 2), opt.EINVAL),
                                         (dict(grad=(1 << 20) + 1, dtype=opt.BF16), opt.EINVAL)])
def test_refuses_gradients(change, code):
    assert _norm([_g(**change)]) == _clip([_g(**change)]) == code
    arr = (opt.Gradient * 1)(_g(**change))
    assert opt.gradient_norm_workspace_bytes(arr) == 0


def test_refuses_calls():
    assert _norm([], 0) == _clip([], 0) == opt.ESHAPE and _norm([_g()], -1) == opt.ESHAPE
    assert _norm([_g()], max_norm=0.0) == _norm([_g()], max_norm=-1.0) == _norm([_g()], max_norm=float("nan")) == opt.EINVAL
    assert _norm([_g()], norm=None) == opt.EINVAL and _clip([_g()], scale=None) == opt.EINVAL
    assert _norm([_g()], norm=4098) == _clip([_g()], scale=4097) == opt.EINVAL
    need = opt.gradient_norm_workspace_bytes((opt.Gradient * 1)(_g()))
    assert need >= 16
    assert _norm([_g()], nbytes=need - 1) == _norm([_g()], ws=None) == _norm([_g()], ws=8196) == opt.EWORKSPACE
    lib = opt.lib()
    assert lib.optimus_gradient_norm(None, 1, 1.0, 4096, None, None, 8192, 1 << 20, None) == opt.EINVAL
    assert lib.optimus_gradient_clip(None, 1, 4096, None) == opt.EINVAL and lib.optimus_gradient_norm_workspace_bytes(None, 1) == 0


def test_refuses_clipped_gradients_that_meet():
    far = iter(range(1 << 26, 1 << 40, 1 << 20))
    apart = lambda **kw: _g(grad=next(far), clipped=next(far), **kw)   # noqa: E731
    assert _clip([_g(clipped=None)]) == _clip([_g(clipped=(1 << 24) + 2)]) == opt.EINVAL
    for bad in ([_g(clipped=(1 << 20) + 4)], [_g(clipped=(1 << 20) - 4)], [_g(parts=3, clipped=(1 << 20) + 400)],       # its own gradient, moved
                [_g(), _g(grad=1 << 28)], [_g(), _g(grad=1 << 28, clipped=(1 << 24) + 396)],                              # another clipped
                [_g(), _g(grad=(1 << 24) + 396, clipped=1 << 28)],                                                        # another's gradient
                [_g(clipped=1 << 20), _g(clipped=1 << 20)]):                                                              # the same one twice, in place
        assert _clip(bad) == opt.EINVAL
        assert _clip([apart() for _ in range(40)] + bad) == opt.EINVAL                                                    # in a long list too


def test_make_gradients():
    a, b = torch.zeros(6, 10), torch.zeros(30, dtype=torch.bfloat16)
    g = opt.make_gradients([dict(grad=a, parts=3), dict(grad=b, clipped=torch.zeros(40, dtype=torch.bfloat16), n=20)])
    assert (g[0].n, g[0].parts, g[0].dtype, g[0].grad, g[0].clipped) == (20, 3, opt.FP32, a.data_ptr(), a.data_ptr())
    assert (g[1].n, g[1].parts, g[1].dtype) == (20, 1, opt.BF16) and g[1].clipped != g[1].grad
    for bad, code in ((dict(grad=a.double()), opt.EDTYPE), (dict(grad=a.half()), opt.EDTYPE), (dict(grad=a, clipped=b), opt.EDTYPE), (dict(grad=a, n=61), opt.ESHAPE),
                      (dict(grad=a, n=21, parts=3), opt.ESHAPE), (dict(grad=a, clipped=torch.zeros(59)), opt.ESHAPE), (dict(grad=a.t()), opt.EINVAL),
                      (dict(grad=a[:, ::2]), opt.EINVAL), (dict(grad=a, clipped=torch.zeros(120)[::2]), opt.EINVAL)):
        with pytest.raises(opt.OptimusError) as e:
            opt.make_gradients([bad])
        assert e.value.code == code
    for kw, code in ((dict(norm=torch.zeros(1).double()), opt.EDTYPE), (dict(norm=torch.zeros(1), norms=torch.zeros(1)), opt.ESHAPE),
                     (dict(norm=torch.zeros(0)), opt.ESHAPE), (dict(norm=torch.zeros(1), scale=torch.zeros(1, dtype=torch.bfloat16)), opt.EDTYPE),
                     (dict(norm=torch.zeros(1), norms=torch.zeros(4)[::2]), opt.EINVAL)):
        with pytest.raises(opt.OptimusError) as e:
            opt.gradient_norm(g, 1.0, **kw)
        assert e.value.code == code
    with pytest.raises(opt.OptimusError) as e:
        opt.gradient_clip(g, torch.zeros(1).double())
    assert e.value.code == opt.EDTYPE


def test_workspace():
    """A piece a workgroup, an entry a tensor; a long list's pieces are longer."""
    many = (opt.Gradient * 1000)(*[_g() for _ in range(1000)])
    assert opt.gradient_norm_workspace_bytes(many) == 16000
    long = (opt.Gradient * 1)(_g(n=1 << 34))
    assert 8 * 1000 <= opt.gradient_norm_workspace_bytes(long) <= 8 * 10000
    assert ctypes.sizeof(opt.Gradient) == 32
