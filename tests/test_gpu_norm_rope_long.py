"""Gradients of the head norms' weights where a workgroup of the backward takes many blocks of tokens.

Tolerance. A workgroup adds trips x heads terms of a feature and token row in a row, then its rows (16 of 128 features, 32 of 64); the weights' sums add
at most 8 of the 512 workgroups in a row and then 64 slices: so many additions of 2^-24 of the terms' magnitudes, and 48 more for a term
itself (test_gpu_norm_rope.py)."""
import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb
from tests.test_gpu_norm_rope import EPS, fused, near, pair_length, positions, turned, weights

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,N,H,Hk,d,halves", [(1, 40_007, 3, 1, 128, False), (3, 27_001, 2, 2, 128, True), (1, 120_011, 4, 2, 64, True), (2, 50_001, 1, 3, 64, False)])
def test_weights_gradients_over_many_blocks(B, N, H, Hk, d, halves, dtype):
    """2,501 to 5,064 blocks of tokens, the last of them partly filled; the gradients are all of one sign in part, so that the sums grow."""
    (q, k, v), _ = fused(B, N, H, Hk, d, dtype)
    wq, wk = weights(d, 5)
    plan = mb.rope_plan(positions(N, 3, 50), (10, 5, 3), halves=halves)
    dz = [(mi.randn((B, h, N, d), 11 + i, "cuda")).to(dtype) for i, h in enumerate((H, Hk, Hk))]
    dz[0] += mb.qk_norm_rope(q, None, None, None, None, plan, EPS)[0]       # dy = n, and what is random
    got = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan, EPS)
    rows = 2048 // d
    blocks = -(-B * N // rows)
    assert blocks >= 2400 and B * N % rows
    adds = -(-blocks // 512) * (H + Hk) + rows + 8 + 64 + 48
    for x, w, g, dx, dw in ((q, wq, dz[0], got[0], got[3]), (k, wk, dz[1], got[1], got[4])):
        dy = turned(g.double(), plan, inverse=True).transpose(1, 2)
        r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)
        n, dn = x.double() * r, dy * w.double()
        size = (pair_length(g.double().transpose(1, 2), halves) * n.abs()).sum((0, 1, 2))
        off = (dw.double() - (dy * n).sum((0, 1, 2))).abs() / (adds * STEP * size)
        print(f"[dw] {float(off.max()):.3f} of the bound", flush=True)
        assert (off <= 1).all()
        slack = r * (pair_length(g.double().transpose(1, 2), halves) * w.abs().double() + n.abs() * (dn * n).abs().mean(-1, keepdim=True))
        near(dx, r * (dn - n * (dn * n).mean(-1, keepdim=True)), slack, dtype)
    assert torch.equal(got[2], dz[2].transpose(1, 2))
    # any head count a workgroup's share: the last tokens alone give the same rows
    tail = mb.qk_norm_rope_bwd(q[:, -5:], k[:, -5:], *(g[:, :, -5:].contiguous() for g in dz), wq, wk,
                               mb.rope_plan(plan.positions[-5:].contiguous(), (10, 5, 3), halves=halves), EPS)
    assert all(torch.equal(a[:, -5:], b) for a, b in zip(got[:3], tail))
