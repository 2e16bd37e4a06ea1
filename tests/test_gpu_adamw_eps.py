"""GPU: the AdamW step where an eps that is not small in itself is, beside sqrt(1 - beta2): the first steps divide a root of tiny moments by
that, and what the root loses below 2^-63 is no longer nothing beside eps."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import adamw as oad
from gpu_util import to_host

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("on_device", [False, True])
@pytest.mark.parametrize("eps,beta2", [(1e-15, 0.999), (1e-15, 0.9999), (1.1e-15, 0.999999), (1e-14, 0.99999999), (1e-12, 0.999999999999),
                                       (7e-12, 0.999), (1e-11, 0.999)])
def test_roots_of_tiny_moments(eps, beta2, on_device):
    """v on both sides of 2^-126, weights that start at zero, so that they are the update.  From v = 1e-41 on its rounding of at most half
    of 2^-149 is 7e-5 of it, 3.5e-5 of its root; what the root may lose is 2^-21 of the denominator, and there are some ten roundings."""
    n, lr = 1000, 1e-2
    g = np.logspace(-20.5, -17.5, n) / np.sqrt(1 - beta2)
    g = (g * np.where(np.arange(n) % 3, 1, -1)).astype(np.float32)
    w, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    step = torch.tensor([1], dtype=torch.int64, device=DEV)
    cfg = opt.AdamwCfg(lr, 0.9, beta2, eps, 0 if on_device else 1, 0)
    if on_device:
        cfg.step_on_device = step.data_ptr()
    print("adamw", eps, beta2, on_device, flush=True)
    opt.adamw_step(cfg, opt.make_adamw_tensors([dict(param=w, grad=torch.from_numpy(g).to(DEV), m=m, v=v)]))
    torch.cuda.synchronize()
    want = oad.step(np.zeros(n), np.zeros(n), np.zeros(n), g[None].astype(np.float64), lr=lr, beta1=0.9, beta2=beta2, eps=eps, t=1, decay=0.0)[0]
    off = np.abs(to_host(w) - want) / np.abs(want)
    assert off.max() <= 3.5e-5 + 2.0 ** -21 + 10 * 2.0 ** -24, (off.argmax(), off.max())
