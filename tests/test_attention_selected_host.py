"""CPU: the oracle of the attention over chosen blocks against closed forms, the plain oracle and differences; the entry points' refusals."""
import ctypes

import numpy as np
import pytest

import paper_2104_05343_amd as opt
from oracle import attention as oatt, attention_selected as oas


def _random(s, d, seed):
    rng = np.random.default_rng(seed)
    return [rng.standard_normal((s, d)) for _ in range(4)]


def test_rounding():
    x = np.array([1.0, 1.00390625, 1.01171875, 1.0039065, -2.5, 3.4e38], dtype=np.float32)
    assert list(oas.round_bf16(x)[:5]) == [1.0, 1.0, 1.015625, 1.0078125, -2.5] and np.isinf(oas.round_bf16(x)[5])


def test_choice():
    """Blocks of 2 keys whose means are known numbers along one axis."""
    mean = np.array([3.0, 1.0, 2.0, 3.0, 0.0])
    K = np.stack([np.repeat(mean, 2) + np.tile([0.5, -0.5], 5), np.zeros(10)], 1)
    Q = np.tile([[1.0, 0.0]], (10, 1))
    got = oas.choose(Q, K, block=2, count=3, causal=True)
    assert got.tolist()[::2] == [[0, -1, -1], [0, 1, -1], [0, 1, 2], [0, 2, 3], [0, 3, 4]]
    got = oas.choose(-Q, K, block=2, count=2, causal=True)
    assert got.tolist()[::2] == [[0, -1], [0, 1], [1, 2], [1, 3], [1, 4]]
    got = oas.choose(Q, K, block=2, count=2, causal=False)
    assert got.tolist()[::2] == [[0, 3], [0, 1], [0, 2], [0, 3], [0, 4]]        # equal scores: the lower block
    got = oas.choose(Q, K, block=2, count=9, causal=False, length=7)
    assert got.tolist() == [[0, 1, 2, 3] + [-1] * 5] * 7 + [[-1] * 9] * 3
    assert oas.choose(0 * Q, K, block=2, count=3, causal=True).tolist()[8] == [0, 1, 4]
    assert np.allclose(oas.means(K, 2, 7)[:, 0], [3.0, 1.0, 2.0, 3.5])


def test_all_blocks_are_the_plain_attention():
    Q, K, V, dO = _random(23, 8, 0)
    for causal in (False, True):
        see = oas.seen(oas.choose(Q, K, block=4, count=6, causal=causal), 23, block=4, causal=causal)
        O, lse, P = oas.forward(Q, K, V, see)
        O0, P0 = oatt.head_forward(Q, K, V, causal)
        assert np.allclose(O, O0, atol=1e-12) and np.allclose(P, P0, atol=1e-12) and np.allclose(lse, oatt.head_logsumexp(Q, K, causal))
        for a, b in zip(oas.backward(Q, K, V, dO, O, lse, see)[:3], oatt.head_backward(Q, K, V, P0, dO)):
            assert np.allclose(a, b, atol=1e-12)


def test_pairs():
    sel = np.array([[0, -1], [0, 0], [5, 0], [1, 0], [2, 1], [0, -7]])
    see = oas.seen(sel, 6, block=2, causal=False)
    assert see.sum(1).tolist() == [2, 2, 2, 4, 4, 2]
    assert oas.seen(sel, 6, block=2, causal=True).sum(1).tolist() == [1, 2, 2, 4, 3, 2]
    assert oas.seen(sel, 6, block=2, causal=False, length=5).sum(1).tolist() == [2, 2, 2, 4, 3, 0]


@pytest.mark.parametrize("causal", [False, True])
def test_gradients_against_differences(causal):
    Q, K, V, dO = _random(14, 4, 3)
    sel = oas.choose(Q, K, block=3, count=2, causal=causal, length=12)
    sel[5] = -1                                      # a row that sees nothing
    see = oas.seen(sel, 14, block=3, causal=causal, length=12)
    O, lse, _ = oas.forward(Q, K, V, see)
    assert not O[5].any() and np.isneginf(lse[5]) and not O[12:].any()
    grads = oas.backward(Q, K, V, dO, O, lse, see)[:3]
    f = lambda: (oas.forward(Q, K, V, see)[0] * dO).sum()   # noqa: E731
    for x, g in zip((Q, K, V), grads):
        for at in [(0, 0), (4, 1), (5, 2), (9, 3), (11, 0), (13, 1)]:
            keep, eps = x[at], 1e-6
            x[at] = keep + eps
            hi = f()
            x[at] = keep - eps
            lo = f()
            x[at] = keep
            assert abs((hi - lo) / (2 * eps) - g[at]) <= 1e-7


def _rc(what, sel, qkv=1 << 20, selected=1 << 22, attn=1 << 24, lse=1 << 26, d_attn=1 << 28, d_qkv=1 << 30, b=4, s=200, h=256, n=4, q=2, i=0, j=1,
        dtype=opt.BF16, ws=1 << 32, nbytes=1 << 40):
    L, p = opt.lib(), ctypes.byref(sel) if sel is not None else None
    tail = (b, s, h, n, q, i, j, 1, dtype, p, ws, nbytes, None)
    if what == "select":
        return L.optimus_attention_select(qkv, selected, *tail)
    if what == "fwd":
        return L.optimus_attention_selected_fwd(qkv, selected, attn, lse, *tail)
    return L.optimus_attention_selected_bwd(qkv, selected, attn, lse, d_attn, d_qkv, *tail)


@pytest.mark.parametrize("kw,code", [
    (dict(qkv=None), opt.EINVAL), (dict(selected=None), opt.EINVAL), (dict(dtype=opt.FP32), opt.EDTYPE), (dict(b=3), opt.ESHAPE), (dict(n=3, h=384), opt.ESHAPE),
    (dict(h=320), opt.ESHAPE), (dict(s=0), opt.ESHAPE), (dict(s=(1 << 20) + 1), opt.ESHAPE), (dict(q=0), opt.ESHAPE), (dict(i=2), opt.ECOORD),
    (dict(j=-1), opt.ECOORD), (dict(ws=None), opt.EWORKSPACE), (dict(ws=(1 << 32) + 16), opt.EWORKSPACE), (dict(nbytes=100), opt.EWORKSPACE),
    (dict(s=1 << 17), opt.ESHAPE), (dict(b=1 << 17), opt.ESHAPE), (dict(b=1 << 15, i=-1, j=-1), opt.ESHAPE)])
def test_refuses_calls(kw, code):
    sel = opt.make_selection(64, 3)
    for what in ("select", "fwd", "bwd"):
        assert _rc(what, sel, **kw) == code, what


def test_refuses_more():
    for what in ("select", "fwd", "bwd"):
        assert _rc(what, None) == opt.EINVAL
        for block, count in ((0, 2), (32, 2), (96, 2), (-64, 2), (4160, 2), (64, 0), (64, 65)):
            assert _rc(what, opt.make_selection(block, count)) == opt.ESHAPE
        assert _rc(what, opt.make_selection(64, 2, 4098)) == opt.EINVAL
        for kw in (dict(qkv=(1 << 20) + 8), dict(selected=(1 << 22) + 2)):
            assert _rc(what, opt.make_selection(64, 2), **kw) == opt.EINVAL
    for kw in (dict(attn=(1 << 24) + 8), dict(lse=(1 << 26) + 2), dict(d_attn=(1 << 28) + 2), dict(d_qkv=(1 << 30) + 4)):
        assert _rc("bwd", opt.make_selection(64, 2), **kw) == opt.EINVAL
    assert _rc("fwd", opt.make_selection(64, 2), attn=None) == _rc("fwd", opt.make_selection(64, 2), lse=None) == opt.EINVAL
    assert _rc("bwd", opt.make_selection(64, 2), d_attn=None) == _rc("bwd", opt.make_selection(64, 2), d_qkv=None) == opt.EINVAL


@pytest.fixture
def form():
    yield opt.debug_set_attention_selected_form
    opt.debug_set_attention_selected_form(-1)


def test_workspace(form):
    size = lambda *a, sel=opt.make_selection(64, 3): opt.attention_selected_workspace_bytes(*a, sel)   # noqa: E731
    one, all_of = size(4, 200, 256, 4, 2, 0, 1), size(4, 200, 256, 4, 2, -1, -1)
    assert 4 * 200 * 4 <= one < all_of
    assert size(3, 200, 256, 4, 2, 0, 1) == size(4, 200, 320, 4, 2, 0, 1) == size(4, 200, 256, 4, 2, 0, 2) == 0
    assert size(4, 200, 256, 4, 2, 0, 1, sel=opt.make_selection(63, 3)) == 0
    form(0)
    assert size(4, 5000, 256, 4, 2, 0, 1) >= 4 * 5000 * 3 * (64 * 2 + 12)               # lists: partial results of all pairs
    form(-1)
    # of one (sequence, head) where 384 MiB do not hold them, not of all of them
    long = size(1, 1 << 18, 1024, 8, 1, 0, 0, sel=opt.make_selection(256, 16))
    assert (1 << 18) * 16 * (128 * 2 + 12) <= long < 2 * (1 << 18) * 16 * (128 * 2 + 12)


def test_form(form):
    """All blocks with a mask where queries choose much of what they could, or little is to do, at most 256 blocks; else lists."""
    def masked(s, block, count, causal, backward=False, b=1, h=2048, n=16):
        return opt.debug_attention_selected_masked(backward, b, s, h, n, 1, 0, 0, causal, opt.make_selection(block, count))
    for backward in (False, True):
        assert masked(1, 64, 1, True, backward) and masked(200, 64, 3, False, backward) and masked(4096, 128, 8, True, backward) != backward
        assert not masked(32768, 128, 16, True, backward) and not masked(8192, 128, 4, True, backward)
        assert masked(16384, 64, 64, True, backward) != backward and not masked(16385, 64, 64, True, backward)  # 256 and 257 blocks
        # the same for one device, whatever the launch covers
        sel = opt.make_selection(64, 6)
        for s in (500, 1000, 2000, 3000):
            assert len({opt.debug_attention_selected_masked(backward, 8, s, 2048, 16, 2, i, i, True, sel) for i in (-1, 0, 1)}) == 1
        for forced in (0, 1):
            form(forced)
            assert masked(1, 64, 1, True, backward) == bool(forced) and not masked(16385, 64, 64, True, backward)
        form(-1)
    with pytest.raises(opt.OptimusError):
        masked(200, 65, 3, True)


def test_refuses_tensors():
    torch = pytest.importorskip("torch")
    for t, code in ((torch.zeros(4, dtype=torch.int64), opt.EDTYPE), (torch.zeros(8, dtype=torch.int32)[::2], opt.EINVAL)):
        with pytest.raises(opt.OptimusError) as e:
            opt.make_selection(64, 2, t)
        assert e.value.code == code
    sel, x = opt.make_selection(64, 2), 1 << 20
    for t, code in ((torch.zeros(4, dtype=torch.int64), opt.EDTYPE), (torch.zeros(8, dtype=torch.int32)[::2], opt.EINVAL)):
        for call in (lambda: opt.attention_select(x, t, 4, 200, 256, 4, 2, 0, 1, True, opt.BF16, sel, None, stream=0),
                     lambda: opt.attention_selected_fwd(x, t, x, x, 4, 200, 256, 4, 2, 0, 1, True, opt.BF16, sel, None, stream=0),
                     lambda: opt.attention_selected_bwd(x, t, x, x, x, x, 4, 200, 256, 4, 2, 0, 1, True, opt.BF16, sel, None, stream=0)):
            with pytest.raises(opt.OptimusError) as e:
                call()
            assert e.value.code == code


@pytest.mark.parametrize("kw", [dict(b=65536, s=1, n=65536, h=65536 * 64, q=65536, i=-1, j=-1), dict(b=46341, s=1, n=46341, h=46341 * 64, q=46341, i=0, j=0),
                                dict(b=200, s=1, n=200 * 60000, h=200 * 60000 * 64, q=200, i=0, j=0)])
def test_refuses_sizes_past_32_bits(kw):
    """Grids of 2^31 devices and more, rows of 2^31 columns."""
    for what in ("select", "fwd", "bwd"):
        assert _rc(what, opt.make_selection(64, 2), **kw) == opt.ESHAPE, what
    assert opt.attention_selected_workspace_bytes(*(kw[k] for k in "b s h n q i j".split()), opt.make_selection(64, 2)) == 0
