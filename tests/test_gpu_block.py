"""A block's attention as it would be used: the fused projection through head norms and rotation, routing and sparse attention over the
stream, cross attention of every shot to its own caption's states, and the whole way back to the projections' gradients. Each step is
compared with its own 64-bit reference on the very tensors that the step before handed over."""
import numpy as np
import pytest
import torch

import moc_inputs as mi
from oracle import moc_oracle as mo
from paper_2508_21058_amd import binding as mb
from tests import test_gpu_cross as tc
from tests import test_gpu_norm_rope as tn
from tests.test_gpu_parity import check_close

pytestmark = pytest.mark.gpu


def grid_positions(lay, shots, text, frames, gh, gw):
    out = []
    for s in range(shots):
        out += [(s * frames, 0, 0)] * text
        out += [(s * frames + f, y, x) for f in range(frames) for y in range(gh) for x in range(gw)]
    assert len(out) == lay.N
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def test_block_forward_and_backward():
    shots, text, frames, gh, gw, topk = 3, 20, 3, 8, 12, 2
    B, H, d, M = 1, 2, 128, 3 * 40
    bf16 = torch.bfloat16
    lay = mi.multishot_layout(shots, text, frames, gh * gw, 32, "frame")
    N = lay.N
    meta = mb.chunk_meta(lay.offsets, lay.shot, lay.window, lay.text_spans)
    plan = mb.rope_plan(grid_positions(lay, shots, text, frames, gh, gw), (22, 21, 21))
    qkv = mi.randn((B, N, 3 * H, d), 1, "cuda").to(bf16)
    q0, k0, v0 = qkv.split((H, H, H), dim=2)
    wq, wk = tn.weights(d, 4)

    q, k, v = mb.qk_norm_rope(q0, k0, v0, wq, wk, plan)
    for x, w, z in ((q0, wq, q), (k0, wk, k)):
        y = tn.normed(x, w)
        tn.near(z, tn.turned(y, plan), tn.pair_length(y, False), bf16)
    pooled, sel = mb.route(meta, q, k, topk, True)
    ws = mb.attn_workspace(meta, B, H, d, topk, bf16, True)
    o, lse = mb.attn_fwd(meta, q, k, v, sel, workspace=ws)

    # cross attention: queries from a projection of the layer's output (here the output itself, token-major), states of each shot's caption
    x1 = o.transpose(1, 2).contiguous()
    states = mi.randn((B, M, 2 * H, d), 2, "cuda").to(bf16)
    ck0, cv0 = states.split((H, H), dim=2)
    cq, _, _ = mb.qk_norm_rope(x1, q_weight=wk)
    _, ck, cv = mb.qk_norm_rope(None, ck0, cv0, k_weight=wq)
    per = N // shots
    offs, ranges = [per * s for s in range(shots + 1)], [[(40 * s, 40 * s + 11 + 9 * s) for s in range(shots)]]
    kw = dict(kv_ranges=tc.device_ranges(ranges), q_offsets=offs)
    co, clse = mb.cross_attn_fwd(cq, ck, cv, **kw)
    d_co = mi.randn(co.shape, 9, "cuda").to(bf16)
    ref = tc.reference(cq, ck, cv, d_co, ranges, offs, d ** -0.5)
    tc.near("o", co, ref["o"])

    # and back
    dcq, dck, dcv = mb.cross_attn_bwd(cq, ck, cv, co, clse, d_co, **kw)
    for n, g in zip(("dq", "dk", "dv"), (dcq, dck, dcv)):
        tc.near(n, g, ref[n])
    dx1, _, _, dw, _ = mb.qk_norm_rope_bwd(x1, None, dcq, None, q_weight=wk)
    _, dck0, dcv0, _, _ = mb.qk_norm_rope_bwd(None, ck0, None, dck, dcv, k_weight=wq)
    d_o = dx1.transpose(1, 2).contiguous()
    dq, dk, dv = mb.attn_bwd(meta, q, k, v, o, lse, d_o, sel, workspace=ws, after_fwd=True)
    grad = torch.empty_like(qkv)
    mb.qk_norm_rope_bwd(q0, k0, dq, dk, dv, wq, wk, plan, out=grad.split((H, H, H), dim=2))

    # the layer against the oracle on the rotated queries and keys, with the selection it made
    L = mo.OracleLayout.from_layout(lay)
    layer = mo.moc_layer(L, *(t.float().cpu().numpy().astype(np.float64) for t in (q, k, v)), topk, True,
                         d_o.float().cpu().numpy().astype(np.float64))
    assert (np.sort(sel.cpu().numpy(), -1) == np.sort(layer["sel"], -1)).all()
    for n, got in (("o", o), ("dq", dq), ("dk", dk), ("dv", dv)):
        check_close(n, got.float().cpu().numpy(), layer[n])
    # the norms' gradients by automatic differentiation in 64 bits
    for x, w, g, rope, got, axis_w in ((q0, wq, dq, plan, grad[:, :, :H], None), (k0, wk, dk, plan, grad[:, :, H:2 * H], None),
                                       (x1, wk, dcq, None, dx1, dw), (ck0, wq, dck, None, dck0, None)):
        x64, w64 = x.double().requires_grad_(), w.double().requires_grad_()
        y = tn.normed(x64, w64)
        y = y if rope is None else tn.turned(y, rope)
        want, want_w = torch.autograd.grad(y, (x64, w64), g.double())
        off = (got.double() - want).norm() / want.norm()
        assert float(off) < 2.0 ** -8            # one rounding to bf16, half a step at most
        if axis_w is not None:
            assert float((axis_w.double() - want_w).norm() / want_w.norm()) < 1e-5
    assert torch.equal(grad[:, :, 2 * H:], dv.transpose(1, 2)) and torch.equal(dcv0, dcv.transpose(1, 2))
    meta.close()


def test_two_streams_at_once():
    """The same operators on two streams that are not ordered, each with its own workspace, against one after the other."""
    B, N, H, d, M = 1, 3000, 6, 128, 300
    bf16 = torch.bfloat16
    plan = mb.rope_plan(torch.randint(0, 50, (N, 3), dtype=torch.int32, device="cuda"), [22, 21, 21])
    sets = []
    for s in range(2):
        x = mi.randn((B, N, 3 * H, d), 7 + s, "cuda").to(bf16)
        k, v = (mi.randn((B, H, M, d), 17 + s + 2 * i, "cuda").to(bf16) for i in range(2))
        sets.append((x, k, v, mb.cross_attn_workspace(B, H, H, N, M, d, bf16, True), mb.qk_norm_rope_workspace(B, N, H, H, d, bf16)))

    def block(x, k, v, ws, ws_norm):
        q, kk, vv = mb.qk_norm_rope(*x.split(H, 2), rope=plan)
        o, lse = mb.cross_attn_fwd(q, k, v, workspace=ws)
        dq, dk, dv = mb.cross_attn_bwd(q, k, v, o, lse, q, workspace=ws)
        return (o, lse, dq, dk, dv, *mb.qk_norm_rope_bwd(*x.split(H, 2)[:2], dq, kk, vv, rope=plan, workspace=ws_norm))

    want = [block(*s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [[], []]
    for _ in range(4):
        for i, (stream, s) in enumerate(zip(streams, sets)):
            with torch.cuda.stream(stream):
                got[i].append(block(*s))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(a, b) for a, b in zip(g, want[i]))
