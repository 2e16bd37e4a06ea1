"""GPU: attention over chosen blocks of keys with blocks of a thousand keys and more, and over sequences of hundreds of thousands of tokens."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import attention_selected as oas
from test_gpu_attention_selected import DEV, FP32, HALF, PART, Run, lists  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block,count,s", [(1024, 3, 4200), (1088, 2, 3300), (2048, 2, 4200)])
def test_large_blocks_in_several_pieces(block, count, s, d, causal, lists):  # noqa: F811
    """A block's list is cut in pieces of some 256 queries, each with sums of its own of all keys."""
    Run(2, s, d, 1, 1, causal, block=block, count=count, lengths=[s, s - 700]).go().check()


def own_blocks(s, n, d, block):
    """A long sequence whose queries attend to their own block alone; what the forward and the backward pass give."""
    torch.manual_seed(s + d)
    x = torch.randn(s, n, 3, d, dtype=torch.bfloat16, device=DEV)
    dO = torch.randn(s, n, d, dtype=torch.bfloat16, device=DEV)
    O, G, L = torch.full_like(dO, float("nan")), torch.full_like(x, float("nan")), torch.full((n, s), float("nan"), dtype=torch.float32, device=DEV)
    S = (torch.arange(s, dtype=torch.int32, device=DEV) // block).expand(n, s).contiguous()
    sel = opt.make_selection(block, 1)
    ws = torch.full((opt.attention_selected_workspace_bytes(1, s, n * d, n, 1, 0, 0, sel),), 0xFF, dtype=torch.uint8, device=DEV)
    args = (1, s, n * d, n, 1, 0, 0, True, opt.BF16, sel, ws)
    print("own blocks", s, n, d, block, flush=True)
    opt.attention_selected_fwd(x, S, O, L, *args)
    opt.attention_selected_bwd(x, S, O, L, dO, G, *args)
    torch.cuda.synchronize()
    return x, dO, O, L, G


def check_block(out, head, lo, hi):
    x, dO, O, L, G = (t.cpu().float().numpy().astype(np.float64) for t in [out[0][lo:hi, head], out[1][lo:hi, head], out[2][lo:hi, head],
                                                                          out[3][head, lo:hi], out[4][lo:hi, head]])
    d = x.shape[-1]
    Q, K, V = (x[:, k] for k in range(3))
    see = np.tri(hi - lo, dtype=bool)
    want, lse, P = oas.forward(Q, K, V, see)
    size = P @ np.abs(V)
    assert np.all(np.abs(L - lse) <= 1e-5 * np.maximum(1, np.abs(lse)))
    assert np.all(np.abs(O - want) <= HALF * (1.01 * np.abs(want) + size) + (FP32 + PART) * size)
    dQ, dK, dV, P, dS = oas.backward(Q, K, V, dO, O, L, see)
    spread = P * (np.abs(dO) @ np.abs(V).T + (np.abs(dO) * np.abs(O)).sum(1, keepdims=True))
    raw, fine = np.abs(dS), FP32 * spread
    for k, (w, size, small) in enumerate(((dQ, raw @ np.abs(K) / np.sqrt(d), (fine + PART * raw) @ np.abs(K) / np.sqrt(d)),
                                          (dK, raw.T @ np.abs(Q) / np.sqrt(d), fine.T @ np.abs(Q) / np.sqrt(d)),
                                          (dV, P.T @ np.abs(dO), FP32 * P.T @ np.abs(dO)))):
        assert np.all(np.abs(G[:, k] - w) <= HALF * (1.01 * np.abs(w) + size) + 2 * small + 1e-30), (lo, "QKV"[k])


@pytest.mark.parametrize("d", [64, 128])
def test_pieces_that_the_workspace_makes_longer(d, lists):  # noqa: F811
    """262144 queries in blocks of 4096: pieces as many as fill the device would leave more than 1 GiB of sums, at width 128."""
    s, block = 1 << 18, 4096
    out = own_blocks(s, 1, d, block)
    assert not torch.isnan(out[4]).any()
    for lo in (0, 33 * block, s - block):
        check_block(out, 0, lo, lo + block)
