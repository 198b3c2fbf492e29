"""The calls together, as a training program uses them: a linear layer with a bias multiplied in 8 bits, its weight updated
through low-rank cores, its bias with AdamW, the gradients of both clipped by their norm."""
import numpy as np
import pytest
import torch

import synth_inputs as si

pytestmark = pytest.mark.gpu


def test_a_layer_in_8_bits_with_low_rank_and_dense_updates():
    import paper_2602_08007_amd as tsr
    tokens, h, f, r, p = 384, 256, 200, 32, 8
    E4, E5 = torch.float8_e4m3fn, torch.float8_e5m2
    dev = lambda shape, *key: si.normal(shape, si.stream_key(*key)).cuda()
    W, bias, X, target = dev((f, h), 1) * 0.05, torch.zeros(f, device="cuda"), dev((tokens, h), 2), dev((tokens, f), 3)
    W0 = W.clone()
    U, V = torch.empty(f, r, device="cuda"), torch.empty(h, r, device="cuda")
    C, D, M, Vm = (torch.zeros(r, r, device="cuda") for _ in range(4))
    omega = dev((h, r + p), 4)
    bm, bv = torch.zeros(f).to(E4).cuda(), torch.zeros(f).to(E5).cuda()
    bms, bvs = torch.zeros(1, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.uint8, device="cuda")
    G, gb = torch.empty(f, h, device="cuda", dtype=torch.bfloat16), torch.empty(f, device="cuda")
    Y, dX = torch.empty(tokens, f, device="cuda", dtype=torch.bfloat16), torch.empty(tokens, h, device="cuda", dtype=torch.bfloat16)
    norm, coef = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    x, xt = tsr.fp8_matrix(tokens, h, E4), tsr.fp8_matrix(h, tokens, E4)
    w, wt = tsr.fp8_matrix(f, h, E4, 128), tsr.fp8_matrix(h, f, E4, 128)
    dy, dyt = tsr.fp8_matrix(tokens, f, E5), tsr.fp8_matrix(f, tokens, E5)
    gradients = tsr.TensorSet([dict(g=G), dict(g=gb)])
    dense = tsr.TensorSet([dict(p=bias, g=gb, m=bm, v=bv, m_scale=bms, v_scale=bvs, wd_scale=0.0)])
    loss = []
    for t in range(1, 9):
        tsr.tsr_fp8_quantize(W, *w, *wt, block_rows=128)
        tsr.tsr_fp8_quantize(X, *x, *xt)
        tsr.tsr_fp8_matmul(*x, *w, Y)
        dY = (Y.float() + bias - target) / tokens
        loss.append(0.5 * tokens * dY.square().sum().item())
        tsr.tsr_fp8_quantize(dY, *dy, *dyt)
        tsr.tsr_fp8_matmul(*dy, *wt, dX)
        tsr.tsr_fp8_matmul(*dyt, *xt, G)
        gb.copy_(dY.sum(0))
        # the products against fp32 ones of the unrounded operands: half a step of e4m3 (2^-4) and e5m2 (2^-3) of the values, of
        # random signs, is under a tenth of the norm
        if t == 1:
            for got, want in ((Y, X @ W.t()), (dX, dY @ W), (G, dY.t() @ X)):
                assert torch.linalg.norm(got.float() - want) < 0.1 * torch.linalg.norm(want)
        tsr.tsr_grad_norm_batched(gradients, 0.25, norm, coef)
        want = np.sqrt(G.double().square().sum().item() + gb.double().square().sum().item())
        assert abs(norm.item() / want - 1) < 1e-6 and abs(coef.item() / min(1.0, 0.25 / want) - 1) < 1e-6
        if t == 1:
            tsr.tsr_refresh_rsvd(G, omega, r, p, 1, U, V)
        tsr.tsr_project_core(G, U, V, C)
        C.mul_(coef)                                       # clipping is linear, so it may act on the core
        before = bias.clone()
        tsr.tsr_adam_core(C, M, Vm, D, t)
        tsr.tsr_backproject_apply(W, U, V, D, 1e-3)
        tsr.tsr_adamw_batched(dense, t, 1e-2, g_scale=coef, seed=11)
        torch.cuda.synchronize()
        if t == 1:                                         # the first step of AdamW is lr times the sign of the gradient
            big = gb.abs() * coef > 1e-5
            assert torch.allclose((bias - before)[big], -1e-2 * torch.sign(gb)[big], rtol=2e-3)
    assert torch.isfinite(W).all() and torch.isfinite(bias).all() and all(np.isfinite(loss))
    assert not torch.equal(W, W0) and int(bms) > 0 and int(bvs) > 0
