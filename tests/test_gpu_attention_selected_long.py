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


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d,s,block", [(64, 96 * 256, 128), (64, 96 * 256 + 1, 128), (128, 25000, 128), (64, 40000, 192)])
def test_lists_of_many_chunks(d, s, block, causal, lists):  # noqa: F811
    """A sequence's queries come 256 at a time; beyond 96 times their counts are added up apart.  Choices of any order, some of them void, against the
    definitions in 64 bits (a row of one key among them: its dS is a difference of equal numbers, and dQ the rounding of their terms)."""
    count, n = 6, 2
    rng = np.random.default_rng(s)
    selected = rng.integers(-1, s // block + 2, (1, n, s, count)).astype(np.int32)
    r = Run(1, s, n * d, n, 1, causal, block=block, count=count, selected=selected, lengths=[s - 300]).go()
    O, G, L = r.O.view(s, n, d).double(), r.G.view(s, n, 3, d).double(), r.L.view(n, s).double()
    u = torch.arange(s, device=DEV)
    for head in range(n):
        Q, K, V = (r.dQKV.view(s, n, 3, d)[:, head, k].double() for k in range(3))
        dO, chosen = r.dO.view(s, n, d)[:, head].double(), torch.from_numpy(selected[0, head]).to(DEV).long()
        sums = [torch.zeros_like(Q) for _ in range(6)]     # dK, dV; what their rounding to bf16, and that to fp32, is of
        for lo in range(0, s, 4096):
            t = slice(lo, min(s, lo + 4096))
            has = torch.zeros(len(u[t]), s // block + 3, dtype=torch.bool, device=DEV).scatter_(1, torch.where(chosen[t] < 0, s // block + 2, chosen[t]), True)
            see = has[:, u // block] & (u < s - 300)[None] & (u[t] < s - 300)[:, None]
            if causal:
                see &= u[None] <= u[t][:, None]
            S = (Q[t] @ K.T / d ** 0.5).masked_fill(~see, -float("inf"))
            lse = torch.logsumexp(S, 1)
            some = ~torch.isinf(lse)
            assert torch.equal(some, ~torch.isinf(L[head, t]))
            assert ((L[head, t] - lse)[some].abs() <= 1e-5 * lse[some].abs().clamp_min(1)).all()
            P = torch.where(see, torch.exp(S - torch.where(some, lse, 0)[:, None]), 0)
            want, size = P @ V, P @ V.abs()
            assert ((O[t, head] - want).abs() <= HALF * (1.01 * want.abs() + size) + (FP32 + PART) * size + 1e-30).all(), (head, lo)
            P = torch.where(see, torch.exp(S - torch.where(some, L[head, t], 0)[:, None]), 0)
            dS = P * (dO[t] @ V.T - (dO[t] * O[t, head]).sum(1, keepdim=True))
            fine = FP32 * P * (dO[t].abs() @ V.abs().T + (dO[t] * O[t, head]).abs().sum(1, keepdim=True))
            want, size = dS @ K / d ** 0.5, dS.abs() @ K.abs() / d ** 0.5
            small = (fine + PART * dS.abs()) @ K.abs() / d ** 0.5
            assert ((G[t, head, 0] - want).abs() <= HALF * (1.01 * want.abs() + size) + 2 * small + 1e-30).all(), (head, lo)
            for x, y in zip(sums, (dS.T @ Q[t] / d ** 0.5, P.T @ dO[t], dS.abs().T @ Q[t].abs() / d ** 0.5, P.T @ dO[t].abs(),
                                   fine.T @ Q[t].abs() / d ** 0.5, FP32 * P.T @ dO[t].abs())):
                x += y
        for k in range(2):
            want, size, small = sums[k], sums[2 + k], sums[4 + k]
            assert ((G[:, head, 1 + k] - want).abs() <= HALF * (1.01 * want.abs() + size) + 2 * small + 1e-30).all(), (head, "KV"[k])


def test_lists_grow_with_the_sequence(lists):  # noqa: F811
    """Four times the sequence takes no more than eight times as long: a choice without entries leaves lists and sums alone."""
    took = []
    for s, block in ((1 << 18, 256), (1 << 20, 1024)):
        x, O, L = (torch.zeros(s * k, dtype=t, device=DEV) for k, t in ((3 * 64, torch.bfloat16), (64, torch.bfloat16), (1, torch.float32)))
        S = torch.full((s,), -1, dtype=torch.int32, device=DEV)
        sel = opt.make_selection(block, 1)
        ws = torch.empty(opt.attention_selected_workspace_bytes(1, s, 64, 1, 1, 0, 0, sel), dtype=torch.uint8, device=DEV)
        best = float("inf")
        for _ in range(6):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            torch.cuda.synchronize()
            start.record()
            opt.attention_selected_fwd(x, S, O, L, 1, s, 64, 1, 1, 0, 0, True, opt.BF16, sel, ws)
            end.record()
            torch.cuda.synchronize()
            best = min(best, start.elapsed_time(end) * 1e3)
        assert not O.any() and torch.isneginf(L).all()
        took.append(best)
    print("us", took)
    assert took[1] <= 8 * took[0]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [64, 128])
def test_same_gradients_beside_other_traffic(d, block, lists):  # noqa: F811
    """The pass for all three gradients hands tiles of queries from iteration to iteration: the same bits whatever else the memory is busy with."""
    r = Run(1, 6000, 4 * d, 4, 1, True, block=block, count=8).go()
    want = r.G.clone()
    a, b = (torch.zeros(1 << 28, dtype=torch.uint8, device=DEV) for _ in range(2))
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(12):
        with torch.cuda.stream(other):
            for _ in range(4):
                b.copy_(a)
        r.G.fill_(float("nan"))
        r.backward()
        torch.cuda.synchronize()
        assert torch.equal(r.G.view(torch.uint8), want.view(torch.uint8))
