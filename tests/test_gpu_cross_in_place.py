"""Cross attention whose outputs take the place of inputs: o over q, dq over o, dk over k and dv over v, in calls of each way the sums are cut."""
import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,H,Hk,N,M,S", [(1, 2, 1, 1, 700, 1), (2, 4, 2, 333, 130, 1), (2, 3, 3, 333, 40, 3), (1, 24, 12, 6000, 777, 2), (1, 1, 1, 40, 20_000, 1)])
def test_in_place(B, H, Hk, N, M, S, d, dtype):
    q, k, v, d_o = (mi.randn(s, 7 * i, "cuda").to(dtype) for i, s in enumerate(((B, H, N, d), (B, Hk, M, d), (B, Hk, M, d), (B, H, N, d))))
    offs = [N * s // S for s in range(S + 1)]
    ranges = torch.tensor([[(M * s // (2 * S), M) for s in range(S)]] * B, dtype=torch.int32, device="cuda")
    kw = dict(kv_ranges=ranges, q_offsets=offs)
    o, lse = mb.cross_attn_fwd(q, k, v, **kw)
    grads = mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw)
    got, lse2 = q.clone(), torch.empty_like(lse)
    mb.cross_attn_fwd(got, k, v, out=(got, lse2), **kw)
    assert torch.equal(got, o) and torch.equal(lse2, lse)
    k2, v2 = k.clone(), v.clone()
    mb.cross_attn_bwd(q, k2, v2, got, lse, d_o, out=(got, k2, v2), **kw)
    assert all(torch.equal(x, y) for x, y in zip((got, k2, v2), grads))
    with pytest.raises(mb.MocError):
        mb.cross_attn_bwd(q, k, v, o, lse, d_o, out=(q, k2, v2), **kw)
