"""GPU: the operators of a training step on long sequences together, as they are used: projection, rotary positions in place, choice of blocks,
attention over them, and back through all of it to the weights' gradient, its norm, and the update that clips by it."""
import numpy as np
import pytest
import torch

import paper_2104_05343_amd as opt
from oracle import adamw as oad, attention_selected as oas, gradients as og, rotary as orot
from oracle.metrics import rel_frobenius
from workloads import round_to_bf16
from gpu_util import mat_to_dev, mat_to_host, to_host, empty
from layer_util import TOL_BEHIND_LOGITS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SETTINGS = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8)


class Step:
    def __init__(self, b, s, h, n, q, pairs, block, count, lengths, max_norm, seed=11):
        self.b, self.s, self.h, self.n, self.q, self.pairs, self.count, self.block, self.max_norm = b, s, h, n, q, pairs, count, block, max_norm
        M = b * s
        rng = np.random.default_rng(seed)
        self.x = round_to_bf16(rng.standard_normal((M, h)).astype(np.float32))
        self.d_attn = round_to_bf16(rng.standard_normal((M, h)).astype(np.float32))
        self.lengths = np.asarray(lengths, dtype=np.int32)
        t = np.arange(s)
        grid = np.stack([t // 36, t // 6 % 6, t % 6])   # frames of six rows and columns
        self.pos = np.tile(grid, (1, b)).astype(np.int32)
        self.X, self.dO = mat_to_dev(self.x, q, "bf16"), mat_to_dev(self.d_attn, q, "bf16")
        self.W = mat_to_dev(round_to_bf16((rng.standard_normal((h, 3 * h)) * 1.5 / np.sqrt(h)).astype(np.float32)), q, "bf16")
        self.master = self.W.float()
        self.qkv, self.attn, self.d_qkv = empty(M * 3 * h, "bf16"), empty(M * h, "bf16"), empty(M * 3 * h, "bf16")
        self.lse, self.d_W = empty(b * n * s, "fp32"), empty(3 * h * h, "fp32")
        self.selected = torch.full((b * n * s * count,), -5, dtype=torch.int32, device=DEV)
        self.m, self.v = torch.zeros(3 * h * h, device=DEV), torch.zeros(3 * h * h, device=DEV)
        self.keep = torch.from_numpy(self.pos).to(DEV), torch.from_numpy(self.lengths).to(DEV)
        self.axes = opt.make_rotary(self.keep[0], pairs, interleaved=True)
        self.sel = opt.make_selection(block, count, self.keep[1])
        self.ws = torch.full((opt.attention_selected_workspace_bytes(b, s, h, n, q, -1, -1, self.sel),), 0xFF, dtype=torch.uint8, device=DEV)
        self.grads = opt.make_gradients([dict(grad=self.d_W)])
        self.norm, self.scale = torch.zeros(1, device=DEV), torch.zeros(1, device=DEV)
        self.norm_ws = torch.empty(opt.gradient_norm_workspace_bytes(self.grads), dtype=torch.uint8, device=DEV)
        self.tensors = opt.make_adamw_tensors([dict(param=self.W, master=self.master, grad=self.d_W, m=self.m, v=self.v, weight_decay=0.01)])

    def run(self, t, step=None):
        b, s, h, n, q = self.b, self.s, self.h, self.n, self.q
        M, shape = b * s, (b, s, h, n, q, -1, -1)
        opt.summa_ab(self.X, self.W, self.qkv, M, h, 3 * h, q, -1, -1, opt.BF16)
        opt.rotary(self.qkv, self.qkv, *shape, opt.BF16, self.axes)
        opt.attention_select(self.qkv, self.selected, *shape, True, opt.BF16, self.sel, self.ws)
        opt.attention_selected_fwd(self.qkv, self.selected, self.attn, self.lse, *shape, True, opt.BF16, self.sel, self.ws)
        opt.attention_selected_bwd(self.qkv, self.selected, self.attn, self.lse, self.dO, self.d_qkv, *shape, True, opt.BF16, self.sel, self.ws)
        opt.rotary_bwd(self.d_qkv, self.d_qkv, *shape, opt.BF16, self.axes)
        opt.summa_ex("atb", self.X, self.d_qkv, self.d_W, h, M, 3 * h, q, -1, -1, opt.BF16, out_fp32=True)
        opt.gradient_norm(self.grads, self.max_norm, self.norm, self.scale, ws=self.norm_ws)
        opt.adamw_step(opt.AdamwCfg(step=t, grad_scale=self.scale.data_ptr(), step_on_device=None if step is None else step.data_ptr(), **SETTINGS),
                       self.tensors)

    def all(self):
        return self.qkv, self.selected, self.attn, self.lse, self.d_qkv, self.d_W, self.norm, self.scale, self.W, self.master, self.m, self.v


@pytest.mark.parametrize("case", [dict(b=2, s=400, h=256, n=4, q=2, pairs=(8, 12, 12), block=64, count=3, lengths=[400, 333], max_norm=5.0),
                                  dict(b=1, s=700, h=256, n=2, q=1, pairs=(16, 20, 20), block=128, count=2, lengths=[650], max_norm=1e9)])
@pytest.mark.parametrize("form", [0, 1])
def test_steps(case, form):
    """Every step's gradients against the oracle from the device's own weights and choices, the norm and the update from the device's own
    gradients, four steps."""
    opt.debug_set_attention_selected_form(form)
    try:
        r = Step(**case)
        b, s, h, n, q, d = r.b, r.s, r.h, r.n, r.q, r.h // r.n
        for t in range(1, 5):
            W_now = mat_to_host(r.W, h, 3 * h, q).astype(np.float64)
            before = [to_host(k).astype(np.float64) for k in (r.master, r.m, r.v)]
            r.run(t)
            torch.cuda.synchronize()
            chosen = r.selected.cpu().numpy().reshape(q, q, b // q, n // q, s, r.count).transpose(0, 2, 1, 3, 4, 5).reshape(b, n, s, r.count)
            turned = mat_to_host(r.qkv, b * s, 3 * h, q)
            full = orot.rotate(r.x.astype(np.float64) @ W_now, r.pos, n, r.pairs, interleaved=True)
            g_qkv = np.zeros((b * s, 3 * h))
            for seq in range(b):
                rows = slice(seq * s, (seq + 1) * s)
                for head in range(n):
                    cols = slice(3 * head * d, 3 * (head + 1) * d)
                    Q, K, _ = np.split(turned[rows, cols].astype(np.float64), 3, axis=1)
                    assert np.array_equal(chosen[seq, head], oas.choose(Q, K, block=r.block, count=r.count, causal=True, length=r.lengths[seq]))
                    Q, K, V = np.split(full[rows, cols], 3, axis=1)
                    see = oas.seen(chosen[seq, head], s, block=r.block, causal=True, length=r.lengths[seq])
                    O, L, _ = oas.forward(Q, K, V, see)
                    g_qkv[rows, cols] = np.concatenate(oas.backward(Q, K, V, r.d_attn[rows, head * d:(head + 1) * d], O, L, see)[:3], axis=1)
            g_qkv = orot.rotate(g_qkv, r.pos, n, r.pairs, interleaved=True, back=True)
            # gradients behind the logits of bf16 operands: the layer tests' bound, qkv and d_qkv rounded twice here
            assert rel_frobenius(mat_to_host(r.d_W, h, 3 * h, q), r.x.T.astype(np.float64) @ g_qkv) <= np.sqrt(2) * TOL_BEHIND_LOGITS
            grad = to_host(r.d_W).astype(np.float64)
            total, _ = og.norm([grad.reshape(1, -1)])
            assert abs(r.norm.item() - total) <= 2.0 ** -23 * total
            assert abs(r.scale.item() - og.scale(total, r.max_norm)) <= 2.0 ** -22 and (r.scale.item() < 1) == (r.max_norm < 100)
            w, m, v = oad.step(*before, grad.reshape(1, -1), t=t, decay=0.01, grad_scale=r.scale.item(), **SETTINGS)
            for got, want in ((r.master, w), (r.m, m), (r.v, v)):
                assert rel_frobenius(to_host(got), want) <= 1e-6
            assert torch.equal(r.W, r.master.to(torch.bfloat16))
    finally:
        opt.debug_set_attention_selected_form(-1)


def test_a_captured_step():
    """The whole step replayed, the step's number on the device, against eager steps: the same bits, step after step."""
    case = dict(b=2, s=400, h=256, n=4, q=2, pairs=(8, 12, 12), block=64, count=3, lengths=[400, 333], max_norm=5.0)
    a, e, warm = Step(**case), Step(**case), Step(**case)
    step = torch.ones(1, dtype=torch.int64, device=DEV)
    warm.run(1, step)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        a.run(1, step)
    for t in range(1, 5):
        step.fill_(t)
        a.ws.fill_(0x55)
        g.replay()
        torch.cuda.synchronize()
        e.run(t, step)
        torch.cuda.synchronize()
        for x, y in zip(a.all(), e.all()):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
