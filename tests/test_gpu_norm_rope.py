"""Head norms with rotation, and the rotation alone, against their formulas in 64 bits.

Tolerances. Forward: the product chain x r w (r from a sum of d squares, its adds in a tree of at most 12 levels, halved by the root),
a sine and a cosine of an angle reduced to float (half a step of a turn, 2 pi 2^-25, and one of the function) and the two products and
one sum of the rotation stay within 32 steps of 2^-24 of |y0| + |y1|; 48 steps of the pair's length are allowed. Then one rounding to
the storage type, half a step of the result. Backward: the same chain once more, of r (|dn| + |n| mean|dn n|). Weights' gradients:
sums of at most 256 adds in a row, 2^-24 each, of the terms' magnitudes."""
import numpy as np
import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: STEP}
EPS = 1e-6


def positions(N, axes=3, t0=0, seed=0):
    g = np.random.default_rng(seed)
    p = g.integers(0, 60, (N, axes)) + np.array([t0] + [0] * (axes - 1))
    return torch.from_numpy(p.astype(np.int32)).cuda()


def pairs_of(x, halves):
    """[..., d] -> [..., d/2, 2]"""
    return torch.stack(x.chunk(2, -1), -1) if halves else x.unflatten(-1, (-1, 2))


def of_pairs(z, halves):
    return torch.cat((z[..., 0], z[..., 1]), -1) if halves else z.flatten(-2)


def turned(x, plan, inverse=False):
    """x [B, heads, N, d] in 64 bits."""
    axis = np.repeat(np.arange(len(plan.axis_pairs)), plan.axis_pairs)
    a = plan.positions.double()[:, torch.from_numpy(axis).cuda()] * plan.freq
    a = torch.nn.functional.pad(a, (0, x.shape[-1] // 2 - a.shape[-1]))
    c, s = torch.cos(a), torch.sin(-a if inverse else a)
    z = pairs_of(x, plan.halves)
    return of_pairs(torch.stack((z[..., 0] * c - z[..., 1] * s, z[..., 0] * s + z[..., 1] * c), -1), plan.halves)


def normed(x, w, eps=EPS):
    """x token-major -> head-major, in 64 bits"""
    y = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + eps)
    return (y if w is None else y * w.double()).transpose(1, 2)


def pair_length(x, halves):
    n = pairs_of(x, halves).square().sum(-1).sqrt()
    return of_pairs(torch.stack((n, n), -1), halves)


def near(got, ref, scale, dtype, steps=48):
    bound = HALF[dtype] * ref.abs() + steps * STEP * scale
    off = (got.double() - ref).abs()
    assert torch.isfinite(got).all()
    assert (off <= bound).all(), f"off by {float((off / bound.clamp_min(1e-300)).max()):.2f} of the bound"


def fused(B, N, H, Hk, d, dtype, seed=1):
    """q, k, v as slices of one projection, and the projection."""
    x = mi.randn((B, N, H + 2 * Hk, d), seed, "cuda").to(dtype)
    return x.split((H, Hk, Hk), dim=2), x


def weights(d, seed):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.3 * torch.randn(d, generator=g)).cuda() for _ in range(2)]


SHAPES = [      # B, N, H, Hk, axes and pairs, first time
    (1, 1, 1, 1, (10, 5, 3), 0), (2, 33, 3, 3, (12, 10, 10), 7), (3, 257, 6, 2, (32,), 100000), (1, 1000, 5, 1, (8, 8, 8, 8), 0),
    (1, 4099, 2, 2, (0, 20, 12), 2_000_000_000 - 60),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,N,H,Hk,pairs,t0", SHAPES)
def test_forward_and_backward(B, N, H, Hk, pairs, t0, d, halves, dtype):
    (q, k, v), _ = fused(B, N, H, Hk, d, dtype)
    wq, wk = weights(d, 5)
    plan = mb.rope_plan(positions(N, len(pairs), t0), pairs, halves=halves)
    got = mb.qk_norm_rope(q, k, v, wq, wk, plan, EPS)
    for x, w, z in ((q, wq, got[0]), (k, wk, got[1])):
        y = normed(x, w)
        assert z.is_contiguous()
        near(z, turned(y, plan), pair_length(y, halves), dtype)
    assert torch.equal(got[2], v.transpose(1, 2).contiguous())

    dz = [mi.randn(z.shape, 11 + i, "cuda").to(dtype) for i, z in enumerate(got)]
    out = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan, EPS)
    for x, w, g, dx, dw in ((q, wq, dz[0], out[0], out[3]), (k, wk, dz[1], out[1], out[4])):
        dy = turned(g.double(), plan, inverse=True).transpose(1, 2)
        r = 1 / torch.sqrt(x.double().square().mean(-1, keepdim=True) + EPS)
        n, dn = x.double() * r, dy * w.double()
        ref = r * (dn - n * (dn * n).mean(-1, keepdim=True))
        slack = r * (pair_length(g.double().transpose(1, 2), halves) * w.abs().double() + n.abs() * (dn * n).abs().mean(-1, keepdim=True))
        near(dx, ref, slack, dtype)
        terms = dy * n
        off = (dw.double() - terms.sum((0, 1, 2))).abs()
        size = (pair_length(g.double().transpose(1, 2), halves) * n.abs()).sum((0, 1, 2))
        assert (off <= 256 * STEP * size).all()
    assert torch.equal(out[2], dz[2].transpose(1, 2))
    again = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan, EPS)
    assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_parts_alone_without_rotation_or_weights(dtype):
    """An encoder's keys and values: no queries, no rotation. Queries of cross attention: nothing else."""
    (q, k, v), _ = fused(2, 77, 4, 2, 128, dtype)
    _, zk, zv = mb.qk_norm_rope(None, k, v)
    near(zk, normed(k, None), normed(k, None).abs(), dtype)
    assert torch.equal(zv, v.transpose(1, 2).contiguous())
    zq, none_k, none_v = mb.qk_norm_rope(q, q_weight=weights(128, 2)[0])
    assert none_k is None and none_v is None
    near(zq, normed(q, weights(128, 2)[0]), normed(q, weights(128, 2)[0]).abs(), dtype)
    assert torch.equal(mb.qk_norm_rope(q, k, v)[1], zk)
    dz = mi.randn(zv.shape, 3, "cuda").to(dtype)
    dq, dk, dv, dqw, dkw = mb.qk_norm_rope_bwd(None, None, None, None, dz)
    assert dq is None and dk is None and dqw is None and dkw is None and torch.equal(dv, dz.transpose(1, 2))


def test_rows_of_zeros_and_of_huge_values():
    x = torch.zeros(1, 40, 2, 128, device="cuda")
    x[0, 1::3] = 1e-30
    x[0, 2::3] = 1e15                        # squares below the largest float
    z = mb.qk_norm_rope(x)[0]
    near(z, normed(x, None), normed(x, None).abs(), torch.float32)
    dz = mi.randn(z.shape, 3, "cuda")
    dx = mb.qk_norm_rope_bwd(x, None, dz, None)[0]
    assert torch.isfinite(dx).all()
    near(dx[0, 0::3], dz.transpose(1, 2)[0, 0::3].double() * 1e3, dz.transpose(1, 2)[0, 0::3].abs().double() * 1e3, torch.float32)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("halves", [False, True])
def test_rope_strides_inverse_and_in_place(halves, dtype):
    B, N, H, d = 2, 131, 5, 128
    plan = mb.rope_plan(positions(N, 3, 5000), (20, 10, 10), halves=halves)      # 24 pairs stay as they are
    x = mi.randn((B, N, H + 3, d), 4, "cuda").to(dtype)[:, :, 2:2 + H].transpose(1, 2)
    z = mb.apply_rope(x, plan)
    near(z, turned(x.double(), plan), pair_length(x.double(), halves), dtype)
    still = pairs_of(z, halves)[..., 40:, :]
    assert torch.equal(still, pairs_of(x, halves)[..., 40:, :])
    back = mb.apply_rope(x, plan, inverse=True)
    near(back, turned(x.double(), plan, True), pair_length(x.double(), halves), dtype)
    token_major = torch.empty(B, N, H, d, dtype=dtype, device="cuda")
    assert torch.equal(mb.apply_rope(x, plan, out=token_major.transpose(1, 2)), z)
    whole = torch.full((B, H, N + 2, d), 7.0, dtype=dtype, device="cuda")       # rows on either side stay as they were
    mine = whole[:, :, 1:-1]
    mine.copy_(x)
    assert mb.apply_rope(mine, plan, out=mine).data_ptr() == mine.data_ptr()
    assert torch.equal(mine, z) and (whole[:, :, 0] == 7).all() and (whole[:, :, -1] == 7).all()
    # the rotation keeps lengths, and one sample expanded over the batch is that sample
    one = x[:1].expand(3, H, N, d)
    assert torch.equal(mb.apply_rope(one, plan), z[:1].expand(3, H, N, d))


def test_gradient_against_differences():
    """Directional differences of the fp32 forward, h = 2^-6: the error of a central difference is of order h^2 of a third
    derivative of order one, and 2^-22 / h of rounding."""
    B, N, H, Hk, d = 2, 19, 3, 1, 64
    (q, k, v), x = fused(B, N, H, Hk, d, torch.float32)
    wq, wk = weights(d, 9)
    plan = mb.rope_plan(positions(N, 3, 12), (12, 10, 10), halves=True)
    dz = [mi.randn((B, h, N, d), 21 + i, "cuda") for i, h in enumerate((H, Hk, Hk))]
    grads = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan)
    flat = torch.cat([g.flatten() for g in grads]).double()

    def loss(parts):
        return sum(float((z.double() * g.double()).sum()) for z, g in zip(mb.qk_norm_rope(*parts, plan), dz))

    at, h = [q, k, v, wq, wk], 2.0 ** -6
    for seed in range(4):
        u = [mi.randn(t.shape, 40 + 7 * seed + i, "cuda") for i, t in enumerate(at)]
        diff = (loss([t + h * s for t, s in zip(at, u)]) - loss([t - h * s for t, s in zip(at, u)])) / (2 * h)
        along = float((flat * torch.cat([s.flatten() for s in u]).double()).sum())
        assert abs(diff - along) <= 2e-3 * float(flat.norm()), (diff, along)


def test_gradient_into_a_fused_projection_and_a_dirty_workspace():
    (q, k, v), x = fused(2, 300, 4, 2, 128, torch.bfloat16)
    wq, wk = weights(128, 3)
    plan = mb.rope_plan(positions(300), (22, 21, 21))
    dz = [mi.randn((2, h, 300, 128), 8 + i, "cuda").to(torch.bfloat16) for i, h in enumerate((4, 2, 2))]
    want = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan)
    grad = torch.full((2, 300, 10, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    ws = mb.qk_norm_rope_workspace(2, 300, 4, 2, 128, torch.bfloat16).fill_(255)
    got = mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan, out=grad[:, :, 1:9].split((4, 2, 2), dim=2), workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert (grad[:, :, 0] == 3).all() and (grad[:, :, 9] == 3).all()


def test_offsets_beyond_32_bits():
    """A projection of more than 2^32 elements: the last tokens of the last sample."""
    B, N, H, d = 2, 280_000, 62, 128
    x = torch.zeros(B, N, H, d, dtype=torch.bfloat16, device="cuda")
    assert x.numel() > 2 ** 32
    tail = mi.randn((B, 64, H, d), 6, "cuda").to(torch.bfloat16)
    x[:, -64:] = tail
    plan = mb.rope_plan(positions(N, 3), (22, 21, 21))
    z = mb.qk_norm_rope(x, rope=plan)[0]
    small = mb.qk_norm_rope(tail, rope=mb.rope_plan(plan.positions[-64:].contiguous(), (22, 21, 21)))[0]
    assert torch.equal(z[:, :, -64:], small)
    dx = mb.qk_norm_rope_bwd(x, None, z, None, rope=plan)[0]
    want = mb.qk_norm_rope_bwd(tail, None, small, None, rope=mb.rope_plan(plan.positions[-64:].contiguous(), (22, 21, 21)))[0]
    assert torch.equal(dx[:, -64:], want)


def test_captured_passes_and_another_stream():
    (q, k, v), x = fused(1, 500, 3, 3, 128, torch.bfloat16)
    wq, wk = weights(128, 3)
    plan = mb.rope_plan(positions(500), (22, 21, 21))
    dz = [mi.randn((1, 3, 500, 128), 8 + i, "cuda").to(torch.bfloat16) for i in range(3)]
    ws = mb.qk_norm_rope_workspace(1, 500, 3, 3, 128, torch.bfloat16)

    def both():
        return (*mb.qk_norm_rope(q, k, v, wq, wk, plan), *mb.qk_norm_rope_bwd(q, k, *dz, wq, wk, plan, workspace=ws))

    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for seed in range(3):
        x.copy_(mi.randn(x.shape, 50 + seed, "cuda"))
        want = [t.clone() for t in both()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
