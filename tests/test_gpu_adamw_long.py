"""GPU: the AdamW step over a tensor of more than 2^32 elements (26 GB with bf16 weights and gradients and 8-bit moments): elements, scales and
random bits on both sides of 2^32 and at the end against the oracle."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import adamw as oad
from gpu_util import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
H = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


def test_more_than_2_to_the_32_elements():
    n, t, seed = (1 << 32) + 5003, 3, 77
    windows = [(0, 4096), ((1 << 31) - 2048, 4096), ((1 << 32) - 2048, 4096), ((1 << 32) + 2048, n - (1 << 32) - 2048)]   # from multiples of 128 on
    print("adamw", n, flush=True)
    new = lambda size, dtype: torch.zeros(size, dtype=dtype, device=DEV)   # noqa: E731
    param, grad, m, v = new(n, torch.bfloat16), new(n, torch.bfloat16), new(n, torch.uint8), new(n, torch.uint8)
    m_scale, v_scale = new(-(-n // 128), torch.uint8), new(-(-n // 128), torch.uint8)
    rng, want = np.random.default_rng(5), []
    for at, size in windows:
        param[at:at + size] = torch.from_numpy(rng.standard_normal(size).astype(np.float32)).to(DEV).to(torch.bfloat16)
        grad[at:at + size] = torch.from_numpy(rng.standard_normal(size).astype(np.float32)).to(DEV).to(torch.bfloat16)
        codes = rng.integers(0, 120, (2, size)).astype(np.uint8)
        bytes_ = rng.integers(114, 121, (2, -(-size // 128))).astype(np.uint8)
        m[at:at + size], v[at:at + size] = (torch.from_numpy(c).to(DEV) for c in codes)
        m_scale[at // 128:at // 128 + bytes_.shape[1]], v_scale[at // 128:at // 128 + bytes_.shape[1]] = (torch.from_numpy(c).to(DEV) for c in bytes_)
        w, g = (to_host(x[at:at + size]).astype(np.float64) for x in (param, grad))
        want.append(oad.step(w, oad.unpack(codes[0], bytes_[0]), oad.unpack(codes[1], bytes_[1]), g[None], t=t, decay=0.1, **H))
    opt.adamw_step(opt.AdamwCfg(H["lr"], H["beta1"], H["beta2"], H["eps"], t, seed),
                   opt.make_adamw_tensors([dict(param=param, grad=grad, m=m, v=v, m_scale=m_scale, v_scale=v_scale, weight_decay=0.1)]))
    torch.cuda.synchronize()
    for (at, size), (w, mw, vw) in zip(windows, want):
        bits = oad.random_bits(seed, t, 0, size, first=at)
        p = oad.round_bf16_random(w, oad.mix(bits ^ np.uint64(0x6A09E667)) & np.uint64(0xFFFF))
        off = np.abs(to_host(param[at:at + size]) - p)
        # the other neighbour only where fp32's own error, a 2^-14th of a step or so, decides
        assert np.all(off <= 2.0 ** -7 * np.abs(w) + 1e-6) and np.mean(off > 0) <= 2e-3, at
        for code, byte, x, dither, positive in ((m, m_scale, mw, bits >> np.uint64(16), False), (v, v_scale, vw, bits & np.uint64(0xFFFF), True)):
            val, scale = oad.pack(x, dither, positive)
            got_scale = byte[at // 128:at // 128 + len(scale)].cpu().numpy()
            assert np.array_equal(got_scale, scale), at
            off = np.abs(oad.e4m3_values()[code[at:at + size].cpu().numpy()] - val)
            assert np.all(off <= np.maximum(np.abs(val) / 4, 2.0 ** -9)) and np.mean(off > 0) <= 2e-3, at
    # what lies between had no gradient, no moments and weights of zero
    for x in (param, m, v):
        assert not x[4096:1 << 20].any() and not x[(1 << 31) + 2048:(1 << 31) + (1 << 20)].any()
    del param, grad, m, v
    torch.cuda.empty_cache()
