"""GPU: the operators of a training step together: a stack's backward pass that updates its layers against the backward pass and the
steps one by one; attention with a learned bias, its products and the update of both, step after step, against the oracle."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import adamw as oad, attention_biased as oab
from oracle.metrics import rel_frobenius
from workloads import LayerShape, layer_inputs, round_to_bf16
from gpu_util import mat_to_dev, mat_to_host, to_host, vec_to_dev, empty
from layer_util import TOL_BEHIND_LOGITS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
MATS = ("w_qkv", "w_o", "w1", "w2")
ORDER = ("w_qkv", "w_o", "w1", "w2", "b_qkv", "b_o", "b1", "b2", "ln1_g", "ln1_b", "ln2_g", "ln2_b")


def _stack(shp, L, fused, eight, master, seed=3):
    """Parameters, states (with something in them), buffers: everything that a training step of a stack holds."""
    cfg = opt.LayerCfg(shp.b, shp.s, shp.h, shp.n, shp.q, 1e-5, 1, opt.BF16, 1 if fused else 0)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    elements, d = opt.stack_adamw_elements(cfg), {"cfg": cfg, "params": [], "states": []}
    for l in range(L):
        inp = layer_inputs(seed + l, shp, "bf16", perturb_affine=True)
        if l == 0:
            d["x"], d["d_out"] = mat_to_dev(inp["x"], shp.q, "bf16"), mat_to_dev(inp["d_out"], shp.q, "bf16")
        p = {k: mat_to_dev(inp[k], shp.q, "bf16") if k in MATS else vec_to_dev(inp[k]) for k in ORDER}
        if eight:
            s = {"m": torch.randint(0, 120, (elements,), generator=gen, device=DEV, dtype=torch.uint8),
                 "v": torch.randint(0, 120, (elements,), generator=gen, device=DEV, dtype=torch.uint8),
                 "m_scale": torch.full((elements // 128,), 110, dtype=torch.uint8, device=DEV),
                 "v_scale": torch.full((elements // 128,), 100, dtype=torch.uint8, device=DEV)}
        else:
            s = {"m": torch.randn(elements, generator=gen, device=DEV), "v": torch.rand(elements, generator=gen, device=DEV)}
        if master:
            s["master"] = torch.cat([p[k].float() for k in MATS])
        d["params"].append(p), d["states"].append(s)
    sz = opt.stack_sizes(cfg, L)
    raw = {k: torch.full((max(1, getattr(sz, k)),), 0xFF, dtype=torch.uint8, device=DEV)
           for k in ("workspace", "forward", "backward", "conjunction", "checkpoint", "param_grad")}
    d["raw"], d["buf"] = raw, opt.make_stack_buffers(raw["workspace"], raw["forward"], raw["backward"], raw["conjunction"], raw["checkpoint"])
    M = shp.M * shp.h
    d["out"], d["d_x"] = empty(M, "bf16"), empty(M, "bf16")
    return d


def _same(a, b):
    for x, y in zip(a["params"] + a["states"], b["params"] + b["states"]):
        for k in x:
            assert torch.equal(x[k].view(torch.uint8), y[k].view(torch.uint8)), k
    assert torch.equal(a["d_x"].view(torch.int16), b["d_x"].view(torch.int16))


@pytest.mark.parametrize("shp,L,fused,eight,master", [(LayerShape(b=4, s=64, h=128, n=4, q=2), 3, False, True, False),
                                                      (LayerShape(b=2, s=72, h=256, n=4, q=2), 2, True, False, True),
                                                      (LayerShape(b=1, s=24, h=40, n=5, q=1), 2, False, True, True)])
def test_stack_step_is_the_backward_pass_and_the_steps(shp, L, fused, eight, master):
    """Bit for bit what optimus_stack_bwd with a gradient buffer per layer and optimus_adamw_step afterwards leave, two steps in a row."""
    a, b = (_stack(shp, L, fused, eight, master) for _ in range(2))
    decay = 0.1
    grads, glist = [], []
    for _ in range(L):
        grads.append(torch.full_like(a["raw"]["param_grad"], 0xFF))
        glist.append(opt.layer_grads_in(a["cfg"], grads[-1]))
    for step in (1, 2):
        adamw = opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, step, 5)
        for d in (a, b):
            opt.stack_fwd(d["cfg"], [opt.make_layer_params(p) for p in d["params"]], d["x"], d["buf"], d["out"])
        opt.stack_bwd_adamw(a["cfg"], [opt.make_layer_params(p) for p in a["params"]], [opt.make_adamw_state(**s) for s in a["states"]], adamw, decay,
                            a["raw"]["param_grad"], a["d_out"], a["buf"], a["d_x"])
        opt.stack_bwd(b["cfg"], [opt.make_layer_params(p) for p in b["params"]], glist, b["d_out"], b["buf"], b["d_x"])
        for l in range(L):
            p, s, g = b["params"][l], b["states"][l], glist[l]
            tensors, at, m_at = [], 0, 0
            for k in ORDER:
                n, matrix = p[k].numel(), k in MATS
                offset = getattr(g, "d_" + k) - grads[l].data_ptr()
                parts = 1 if matrix else shp.q
                tensors.append(dict(param=p[k], grad=grads[l][offset:offset + 4 * n * parts].view(torch.float32), m=s["m"][at:at + n], v=s["v"][at:at + n],
                                    grad_parts=parts, n=n, weight_decay=decay if matrix else 0.0,
                                    master=s["master"][m_at:m_at + n] if matrix and master else None))
                if eight:
                    tensors[-1].update(m_scale=s["m_scale"][at // 128:], v_scale=s["v_scale"][at // 128:])
                at, m_at = at + -(-n // 128) * 128, m_at + n
            opt.adamw_step(opt.AdamwCfg(1e-3, 0.9, 0.99, 1e-8, step, 5 + l), opt.make_adamw_tensors(tensors))
        torch.cuda.synchronize()
        _same(a, b)
    assert not torch.isnan(a["params"][0]["w_qkv"]).any()


def test_stack_step_captured():
    """The whole step as a graph, its number on the device: replays leave the bits of eager calls."""
    shp, L = LayerShape(b=4, s=64, h=128, n=4, q=2), 2
    a, b = (_stack(shp, L, False, True, False) for _ in range(2))
    step, lr = torch.tensor([1], dtype=torch.int64, device=DEV), torch.tensor([1e-3], device=DEV)
    adamw = opt.AdamwCfg(0.0, 0.9, 0.99, 1e-8, 0, 7, lr_on_device=lr.data_ptr(), step_on_device=step.data_ptr())

    def one(d):
        params = [opt.make_layer_params(p) for p in d["params"]]
        opt.stack_fwd(d["cfg"], params, d["x"], d["buf"], d["out"])
        opt.stack_bwd_adamw(d["cfg"], params, [opt.make_adamw_state(**s) for s in d["states"]], adamw, 0.1, d["raw"]["param_grad"], d["d_out"], d["buf"], d["d_x"])

    one(_stack(shp, L, False, True, False))   # the library's stream exists from here on
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        one(a)
    for k in range(1, 4):
        step.fill_(k), lr.fill_(1e-3 / k)
        g.replay()
        torch.cuda.synchronize()
        one(b)
        torch.cuda.synchronize()
        _same(a, b)


def test_attention_with_a_learned_bias_learns():
    """x -> qkv = x W -> attention with buckets, packed documents and padding -> gradients of W and the table -> AdamW, four steps.  Every
    step's gradients against the oracle from the device's own weights, every update against the oracle from the device's own gradients."""
    b, s, h, n, q, buckets = 4, 150, 256, 4, 2, 16
    M, d = b * s, h // n
    rng = np.random.default_rng(11)
    x = round_to_bf16(rng.standard_normal((M, h)).astype(np.float32))
    d_attn = round_to_bf16(rng.standard_normal((M, h)).astype(np.float32))
    docs = np.full((b, s), -1, dtype=np.int32)
    for k in range(b):
        docs[k, :s - 7 * k] = np.arange(s - 7 * k) // (40 + k)
    W0 = (rng.standard_normal((h, 3 * h)) * 1.5 / np.sqrt(h)).astype(np.float32)
    X, dO, docs_d = mat_to_dev(x, q, "bf16"), mat_to_dev(d_attn, q, "bf16"), torch.from_numpy(docs.reshape(-1)).to(DEV)
    W = mat_to_dev(round_to_bf16(W0), q, "bf16")
    master, table = W.float(), torch.from_numpy(rng.standard_normal(n * buckets).astype(np.float32)).to(DEV)
    qkv, attn, d_qkv = empty(M * 3 * h, "bf16"), empty(M * h, "bf16"), empty(M * 3 * h, "bf16")
    lse, d_W, d_table = empty(b * n * s, "fp32"), empty(3 * h * h, "fp32"), empty(q * n * buckets, "fp32")
    bias = opt.make_attention_bias(cap=20.0, table=table, buckets=buckets, max_distance=64, documents=docs_d)
    ws = torch.empty(opt.attention_biased_workspace_bytes(b, s, h, n, q, bias), dtype=torch.uint8, device=DEV)
    state = [torch.zeros(k, device=DEV) for k in (3 * h * h, 3 * h * h, n * buckets, n * buckets)]
    tensors = opt.make_adamw_tensors([dict(param=W, master=master, grad=d_W, m=state[0], v=state[1], weight_decay=0.01),
                                      dict(param=table, grad=d_table, grad_parts=q, m=state[2], v=state[3])])
    settings = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)
    for t in range(1, 5):
        W_now, table_now = mat_to_host(W, h, 3 * h, q).astype(np.float64), to_host(table).astype(np.float64).reshape(n, buckets)
        before = [to_host(k).astype(np.float64) for k in (master, table, *state)]
        opt.summa_ab(X, W, qkv, M, h, 3 * h, q, -1, -1, opt.BF16)
        opt.attention_biased_fwd(qkv, attn, lse, b, s, h, n, q, -1, -1, True, opt.BF16, bias, ws)
        opt.attention_biased_bwd(qkv, attn, lse, dO, d_qkv, d_table, b, s, h, n, q, -1, -1, True, opt.BF16, bias, ws)
        opt.summa_ex("atb", X, d_qkv, d_W, h, M, 3 * h, q, -1, -1, opt.BF16, out_fp32=True)
        opt.adamw_step(opt.AdamwCfg(step=t, **settings), tensors)
        torch.cuda.synchronize()
        # the oracle's gradients, nothing rounded
        full = x.astype(np.float64) @ W_now
        g_qkv, g_table = np.zeros((M, 3 * h)), np.zeros((n, buckets))
        for seq in range(b):
            rows = slice(seq * s, (seq + 1) * s)
            for head in range(n):
                Q, K, V = (full[rows, (3 * head + k) * d:(3 * head + k + 1) * d] for k in range(3))
                kw = dict(causal=True, cap=20.0, table=table_now[head], max_distance=64, doc=docs[seq])
                O, L, _ = oab.forward(Q, K, V, **kw)
                dq, dk, dv, dt, _, _ = oab.backward(Q, K, V, d_attn[rows, head * d:(head + 1) * d].astype(np.float64), O, L, **kw)
                g_qkv[rows, 3 * head * d:3 * (head + 1) * d] = np.concatenate([dq, dk, dv], axis=1)
                g_table[head] += dt
        # (gradients behind the logits of bf16 operands: the layer tests' bound)
        assert rel_frobenius(mat_to_host(d_W, h, 3 * h, q), x.T.astype(np.float64) @ g_qkv) <= TOL_BEHIND_LOGITS
        got_table = to_host(d_table).astype(np.float64).reshape(q, n, buckets)
        assert rel_frobenius(got_table.sum(0), g_table) <= 2 * TOL_BEHIND_LOGITS   # sums of dS, where the rounding of attn in rowsum(dO attn) counts too
        # the update, from the device's gradients: fp32 against 64 bits
        for k, (grad, parts, decay) in enumerate(((d_W, 1, 0.01), (d_table, q, 0.0))):
            w, m, v = oad.step(before[k], before[2 + 2 * k], before[3 + 2 * k], to_host(grad).astype(np.float64).reshape(parts, -1), t=t, decay=decay, **settings)
            for got, want in ((master if k == 0 else table, w), (state[2 * k], m), (state[2 * k + 1], v)):
                assert rel_frobenius(to_host(got), want) <= 1e-6
        assert torch.equal(W, master.to(torch.bfloat16))
