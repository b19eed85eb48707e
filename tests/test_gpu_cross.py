"""Cross attention forward and backward against the formulas in 64 bits.

Tolerances, element by element. A logit is a float sum of d products: off by at most d 2^-24 sum|q k| scale, and the exponent adds three
roundings of values of the logits' size. bf16 storage rounds every probability (and every dS) to bf16 before the second product, half a
step 2^-8 each, and the result once more; delta is formed from the rounded o. Sums over states or queries stay in float: 2^-24 of the
terms' magnitudes for every add in a row, at most one per element summed."""
import math

import numpy as np
import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: STEP}


def inputs(B, H, Hk, N, M, d, dtype, seed=0):
    return [mi.randn(s, seed + 31 * i, "cuda").to(dtype) for i, s in enumerate(((B, H, N, d), (B, Hk, M, d), (B, Hk, M, d), (B, H, N, d)))]


def reference(q, k, v, d_o, ranges, offs, scale):
    """Results in 64 bits and how far each element may be off: {name: (value, bound)}."""
    B, H, N, d = q.shape
    Hk, M = k.shape[1:3]
    G, half, dt = H // Hk, HALF[q.dtype], torch.float64
    round_p = half if q.dtype == torch.bfloat16 else 0.0      # what is rounded between the products
    z = lambda *s: torch.zeros(*s, dtype=dt, device="cuda")
    val = dict(o=z(B, H, N, d), lse=torch.full((B, H, N), -math.inf, dtype=dt, device="cuda"), dq=z(B, H, N, d), dk=z(B, Hk, M, d), dv=z(B, Hk, M, d))
    tol = dict(o=z(B, H, N, d), lse=z(B, H, N), dq=z(B, H, N, d), dk=z(B, Hk, M, d), dv=z(B, Hk, M, d))
    for b in range(B):
        for h in range(H):
            for s in range(len(offs) - 1):
                a, e = ranges[b][s]
                a, e, q0, q1 = max(a, 0), min(e, M), offs[s], offs[s + 1]
                if e <= a or q1 <= q0:
                    continue
                Q, K, V, DO = (x.double() for x in (q[b, h, q0:q1], k[b, h // G, a:e], v[b, h // G, a:e], d_o[b, h, q0:q1]))
                L = Q @ K.T * scale
                el = (Q.abs() @ K.abs().T).amax(-1, keepdim=True) * scale * (d + 8) * STEP          # of a logit of the row
                P = torch.softmax(L, -1)
                O, PV = P @ V, P @ V.abs()
                adds = (e - a) * STEP
                ep = 2 * el + round_p + adds                                                        # of a probability, relative
                eo = ep * PV + half * O.abs()
                dP = DO @ V.T
                delta = (DO * O).sum(-1, keepdim=True)
                edelta = (DO.abs() * eo).sum(-1, keepdim=True) + d * STEP * (DO.abs() * O.abs()).sum(-1, keepdim=True)
                dS = P * (dP - delta)
                edS = (2 * el + round_p + 4 * STEP) * dS.abs() + P * (edelta + d * STEP * (DO.abs() @ V.abs().T)) * (1 + round_p)
                val["o"][b, h, q0:q1], tol["o"][b, h, q0:q1] = O, eo
                val["lse"][b, h, q0:q1] = torch.logsumexp(L, -1)
                tol["lse"][b, h, q0:q1] = 2 * el[:, 0] + adds + 8 * STEP * (1 + val["lse"][b, h, q0:q1].abs())
                val["dq"][b, h, q0:q1] = dS @ K * scale
                tol["dq"][b, h, q0:q1] = ((edS + adds * dS.abs()) @ K.abs()) * scale
                n = (q1 - q0) * STEP
                val["dv"][b, h // G, a:e] += P.T @ DO
                tol["dv"][b, h // G, a:e] += (P * (2 * el + round_p + n + 4 * STEP)).T @ DO.abs()
                val["dk"][b, h // G, a:e] += dS.T @ Q * scale
                tol["dk"][b, h // G, a:e] += (edS + n * dS.abs()).T @ Q.abs() * scale
    for n in ("dq", "dk", "dv"):
        tol[n] += half * val[n].abs()
    return {n: (val[n], tol[n]) for n in val}


def near(name, got, ref):
    value, bound = ref
    same = (got.double() == value)
    off = torch.where(same, torch.zeros_like(value), (got.double() - value).abs())
    assert not torch.isnan(got).any(), name
    worst = float((off / bound.clamp_min(1e-30)).max())
    print(f"[cross] {name}: {worst:.3f} of the bound, rel {float(off.norm() / value[torch.isfinite(value)].norm().clamp_min(1e-30)):.2e}")
    assert (off <= bound + 1e-30).all(), f"{name}: {worst:.2f} of the bound"


def device_ranges(ranges):
    return torch.tensor(ranges, dtype=torch.int32, device="cuda")


def check(B, H, Hk, N, M, d, dtype, ranges=None, offs=None, scale=None, seed=0):
    q, k, v, d_o = inputs(B, H, Hk, N, M, d, dtype, seed)
    cuts = [0, N] if offs is None else offs
    ref = reference(q, k, v, d_o, ranges or [[(0, M)] * (len(cuts) - 1)] * B, cuts, d ** -0.5 if scale is None else scale)
    kw = dict(kv_ranges=None if ranges is None else device_ranges(ranges), q_offsets=offs, scale=scale)
    ws = mb.cross_attn_workspace(B, H, Hk, N, M, d, dtype, True, len(cuts) - 1).fill_(255)      # whatever lies there is not read
    o, lse = mb.cross_attn_fwd(q, k, v, workspace=ws, **kw)
    near("o", o, ref["o"])
    near("lse", lse, ref["lse"])
    assert (o[(lse == -math.inf)] == 0).all()
    ws.fill_(255)
    grads = mb.cross_attn_bwd(q, k, v, o, lse, d_o, workspace=ws, **kw)
    for n, g in zip(("dq", "dk", "dv"), grads):
        near(n, g, ref[n])
    o2, lse2 = mb.cross_attn_fwd(q, k, v, **kw)
    again = mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw)
    assert torch.equal(o, o2) and torch.equal(lse, lse2) and all(torch.equal(x, y) for x, y in zip(grads, again))


WHOLE = [       # B, H, Hk, N, M
    (1, 1, 1, 1, 1), (2, 3, 3, 1, 2), (1, 2, 1, 33, 31), (2, 4, 2, 32, 64), (1, 2, 2, 129, 65), (3, 6, 2, 100, 257), (1, 1, 1, 128, 128),
    (1, 2, 2, 700, 96), (1, 24, 24, 640, 200), (4, 12, 4, 1, 8193), (1, 8, 1, 3, 1000), (1, 1, 1, 5000, 33),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,H,Hk,N,M", WHOLE)
def test_all_states(B, H, Hk, N, M, d, dtype):
    check(B, H, Hk, N, M, d, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
def test_padded_batch(d, dtype):
    """Valid lengths of a batch, one of them zero."""
    check(4, 4, 2, 150, 200, d, dtype, ranges=[[(0, 200)], [(0, 0)], [(0, 1)], [(0, 131)]])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hk", [3, 1])
def test_segments_with_their_own_ranges(Hk, dtype):
    """Segments of odd lengths (one empty), ranges that are unaligned, overlap, are empty, reversed or reach past the states."""
    offs = [0, 1, 130, 130, 300, 555]
    ranges = [[(0, 7), (5, 140), (0, 300), (140, 141), (100, 300)], [(250, 260), (30, 30), (0, 300), (200, 100), (-50, 1 << 30)]]
    check(2, 3, Hk, 555, 300, 128, dtype, ranges=ranges, offs=offs)


def test_many_segments_and_another_scale():
    """128 segments, more than a wave has lanes, each with its own states."""
    S, N, M = 128, 1000, 520
    offs = [N * s // S for s in range(S + 1)]
    ranges = [[(4 * s, 4 * s + 1 + s % 12) for s in range(S)]]
    check(1, 2, 1, N, M, 64, torch.bfloat16, ranges=ranges, offs=offs, scale=0.31)


def test_more_samples_than_a_wave_has_lanes():
    """130 samples, most of them without a state."""
    B, M = 130, 40
    ranges = [[(0, 0 if b % 3 else 1 + b % M)] for b in range(B)]
    check(B, 2, 1, 9, M, 128, torch.bfloat16, ranges=ranges)


def random_case(seed):
    g = np.random.default_rng(seed)
    B, Hk, G, S = int(g.integers(1, 4)), int(g.integers(1, 4)), int(g.integers(1, 4)), int(g.choice([1, 1, 2, 5, 40]))
    N, M = (int(2 ** g.uniform(0, top)) for top in (10, 10.5))
    d, dtype = int(g.choice([64, 128, 128])), torch.bfloat16 if g.random() < 0.7 else torch.float32
    offs = [0] + sorted(g.integers(0, N + 1, S - 1).tolist()) + [N]
    kind = g.random()
    def one(s):
        if kind < 0.3:
            return 0, int(g.integers(0, M + 1))
        if kind < 0.6:
            return M * s // S, M * (s + 1) // S
        a, b = g.integers(-3, M + 4, 2)
        return int(a), int(b)
    ranges = None if kind > 0.9 else [[one(s) for s in range(S)] for _ in range(B)]
    return dict(B=B, H=Hk * G, Hk=Hk, N=N, M=M, d=d, dtype=dtype, ranges=ranges, offs=offs if S > 1 else None, seed=seed)


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes(seed):
    check(**random_case(seed))


WIDE = ["whole", "shots", "few heads", "none", "long padded", "long overlapping", "long equal"]    # work enough for wide tiles of states in dK's and dV's pass
LARGE = {
    "whole": dict(B=2, H=12, Hk=4, N=1901, M=900),
    "padded": dict(B=4, H=8, Hk=8, N=1530, M=777, ranges=[[(0, 777)], [(0, 0)], [(0, 1)], [(0, 300)]]),
    "shots": dict(B=1, H=8, Hk=8, N=5003, M=1111, offs=[0, 300, 2000, 2003, 3700, 5003], ranges=[[(0, 77), (100, 612), (612, 615), (700, 1111), (700, 701)]]),
    "overlapping": dict(B=2, H=12, Hk=4, N=2201, M=900, offs=[0, 1, 130, 130, 1700, 2201],
                        ranges=[[(0, 7), (5, 640), (0, 900), (640, 641), (100, 900)], [(250, 260), (30, 30), (0, 900), (200, 100), (-50, 1 << 30)]]),
    "equal": dict(B=1, H=12, Hk=6, N=2900, M=1024, offs=[0, 7, 300, 301, 555, 2900], ranges=[[(3, 1001)] * 5]),
    "few heads": dict(B=1, H=2, Hk=1, N=20001, M=1500),
    "long padded": dict(B=4, H=24, Hk=24, N=3530, M=777, ranges=[[(0, 777)], [(0, 0)], [(0, 1)], [(0, 300)]]),
    "long overlapping": dict(B=2, H=12, Hk=4, N=8201, M=900, offs=[0, 1, 130, 130, 6700, 8201],
                             ranges=[[(0, 7), (5, 640), (0, 900), (640, 641), (100, 900)], [(250, 260), (30, 30), (0, 900), (200, 100), (-50, 1 << 30)]]),
    "long equal": dict(B=1, H=24, Hk=12, N=8900, M=1024, offs=[0, 7, 3000, 3001, 5055, 8900], ranges=[[(3, 1001)] * 5]),
    "long segments": dict(B=2, H=6, Hk=3, N=6210, M=500, offs=[0, 2001, 4100, 4100 + 1025, 6210], ranges=[[(3, 400)] * 4, [(0, 90), (0, 90), (90, 500), (0, 0)]]),
    "none": dict(B=1, H=12, Hk=12, N=3900, M=700, offs=[0, 450, 3900], ranges=[[(5, 5), (700, 0)]]),
}


@pytest.mark.parametrize("name", LARGE)
def test_larger_calls(name):
    mb.prof_enable(True)
    try:
        check(d=128, dtype=torch.bfloat16, **LARGE[name])
        ran = mb.prof_read()
    finally:
        mb.prof_enable(False)
    assert name not in WIDE or "cross_dkdv_wide" in ran and "cross_dkdv" not in ran, ran


@pytest.mark.parametrize("seed", range(100, 116))
def test_random_larger_shapes(seed):
    g = np.random.default_rng(seed)
    c = random_case(seed)
    N, M = (int(2 ** g.uniform(9.5, 12)) for _ in range(2))
    cut = lambda x: x * M // max(1, c["N"])
    c.update(H=c["H"] * 3, Hk=c["Hk"] * 3, N=N, M=M, d=128, dtype=torch.bfloat16)
    if c["offs"]:
        c["offs"] = [0] + sorted(g.integers(0, N + 1, len(c["offs"]) - 2).tolist()) + [N]
    if c["ranges"]:
        c["ranges"] = [[(cut(a), cut(e)) for a, e in sample] for sample in c["ranges"]]
    check(**c)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3e38])
def test_states_outside_every_range_are_never_used(junk, dtype):
    B, H, Hk, N, M, d = 2, 4, 2, 70, 190, 64
    q, k, v, d_o = inputs(B, H, Hk, N, M, d, dtype)
    offs, ranges = [0, 30, 70], [[(3, 37), (60, 129)], [(0, 0), (70, 71)]]
    kw = dict(kv_ranges=device_ranges(ranges), q_offsets=offs)

    def run():
        o, lse = mb.cross_attn_fwd(q, k, v, **kw)
        return (o, lse, *mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw))

    want = run()
    for b in range(B):
        used = torch.zeros(M, dtype=torch.bool, device="cuda")
        for a, e in ranges[b]:
            used[a:e] = True
        k[b, :, ~used] = junk
        v[b, :, ~used] = junk
    got = run()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    assert (got[0][1, :, :30] == 0).all() and (got[1][1, :, :30] == -math.inf).all() and (got[2][1, :, :30] == 0).all()
    assert (got[3][0, :, 40:60] == 0).all() and (got[4][0, :, 129:] == 0).all()


def test_peaked_and_extreme_logits():
    """Logits far apart (the running maximum moves by hundreds) and rows whose probabilities are all on one state."""
    B, H, N, M, d = 1, 2, 96, 300, 64
    q, k, v, d_o = inputs(B, H, H, N, M, d, torch.float32)
    q *= 30
    k[:, :, 250] *= 20
    scale = d ** -0.5
    ref = reference(q, k, v, d_o, [[(0, M)]], [0, N], scale)
    o, lse = mb.cross_attn_fwd(q, k, v)
    near("o", o, ref["o"])
    near("lse", lse, ref["lse"])
    for n, g in zip(("dq", "dk", "dv"), mb.cross_attn_bwd(q, k, v, o, lse, d_o)):
        near(n, g, ref[n])


def test_gradients_against_differences():
    """Central differences of the fp32 forward, h = 2^-6: h^2 of a third derivative of order one, and rounding 2^-20 / h."""
    q, k, v, d_o = inputs(2, 4, 2, 37, 29, 64, torch.float32)
    kw = dict(kv_ranges=device_ranges([[(0, 29), (3, 17)], [(5, 6), (0, 28)]]), q_offsets=[0, 20, 37])
    o, lse = mb.cross_attn_fwd(q, k, v, **kw)
    grads = mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw)
    flat, h = torch.cat([g.flatten() for g in grads]).double(), 2.0 ** -6

    def loss(*t):
        return float((mb.cross_attn_fwd(*t, **kw)[0].double() * d_o.double()).sum())

    for seed in range(4):
        u = [mi.randn(t.shape, 70 + 5 * seed + i, "cuda") for i, t in enumerate((q, k, v))]
        diff = (loss(*(t + h * s for t, s in zip((q, k, v), u))) - loss(*(t - h * s for t, s in zip((q, k, v), u)))) / (2 * h)
        along = float((flat * torch.cat([s.flatten() for s in u]).double()).sum())
        assert abs(diff - along) <= 2e-3 * float(flat.norm()), (diff, along)


def test_rows_around_the_outputs_stay_as_they_were():
    B, H, N, M, d = 1, 2, 45, 70, 128
    q, k, v, d_o = inputs(B, H, H, N, M, d, torch.bfloat16)

    def framed(n, *tail, dtype=torch.bfloat16):
        whole = torch.full((n + 2 * 64, *tail), 9.0, dtype=dtype, device="cuda")
        return whole, whole[64:64 + n]

    frames = [framed(H * n, d) for n in (N, N, M, M)] + [framed(H * N, dtype=torch.float32)]
    o, dq, dk, dv = (f[1].view(B, H, -1, d) for f in frames[:4])
    lse = frames[4][1].view(B, H, N)
    mb.cross_attn_fwd(q, k, v, out=(o, lse))
    mb.cross_attn_bwd(q, k, v, o, lse, d_o, out=(dq, dk, dv))
    for whole, _ in frames:
        assert (whole[:64] == 9).all() and (whole[-64:] == 9).all()
    assert torch.equal(o, mb.cross_attn_fwd(q, k, v)[0])


def test_offsets_beyond_32_bits():
    """Queries and states of more than 2^32 elements: the last of them."""
    d, M = 128, 70
    N = 2 ** 32 // (12 * d) + 200
    q = torch.zeros(1, 12, N, d, dtype=torch.bfloat16, device="cuda")
    k, v = inputs(1, 12, 12, 1, M, d, torch.bfloat16)[1:3]
    q[:, :, -100:] = mi.randn((1, 12, 100, d), 3, "cuda").to(torch.bfloat16)
    o, lse = mb.cross_attn_fwd(q, k, v)
    ref = reference(q[:, 10:, -100:], k[:, 10:], v[:, 10:], q[:, 10:, -100:], [[(0, M)]], [0, 100], d ** -0.5)
    near("o", o[:, 10:, -100:], ref["o"])
    dq, dk, dv = mb.cross_attn_bwd(q, k, v, o, lse, q)
    near("dq", dq[:, 10:, -100:], ref["dq"])
    near("dk", dk[:, 10:], ref["dk"])        # (the other queries and their dO are zero)
    del q, o, lse, dq
    M = 2 ** 32 // (4 * d) + 50
    k = torch.zeros(1, 4, M, d, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    q, kt, vt, d_o = inputs(1, 4, 4, 40, 90, d, torch.bfloat16)
    k[:, :, -90:], v[:, :, -90:] = kt, vt
    ranges = device_ranges([[(M - 90, M)]])
    o, lse = mb.cross_attn_fwd(q, k, v, kv_ranges=ranges)
    ref = reference(q, kt, vt, d_o, [[(0, 90)]], [0, 40], d ** -0.5)
    near("o", o, ref["o"])
    dq, dk, dv = mb.cross_attn_bwd(q, k, v, o, lse, d_o, kv_ranges=ranges)
    near("dq", dq, ref["dq"])
    near("dk", dk[:, :, -90:], ref["dk"])
    near("dv", dv[:, :, -90:], ref["dv"])
    assert not dk[:, :, :-90].any()


@pytest.mark.parametrize("N,M,S", [(900, 130, 3), (2, 3000, 1)])
def test_captured_passes_and_another_stream(N, M, S):
    B, H, Hk, d = 2, 4, 2, 128
    q, k, v, d_o = inputs(B, H, Hk, N, M, d, torch.bfloat16)
    offs = [N * s // S for s in range(S + 1)]
    ranges = device_ranges([[(M * s // S, M * (s + 1) // S) for s in range(S)]] * B)
    ws = mb.cross_attn_workspace(B, H, Hk, N, M, d, torch.bfloat16, True, S)

    def both(ws=None):
        o, lse = mb.cross_attn_fwd(q, k, v, ranges, offs, workspace=ws)
        return (o, lse, *mb.cross_attn_bwd(q, k, v, o, lse, d_o, ranges, offs, workspace=ws))

    both(ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both(ws)
    for seed in range(3):
        q.copy_(mi.randn(q.shape, 90 + seed, "cuda"))
        ranges += seed % 2
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


def ran_wide(fn):
    """fn()'s result; the call took the wide tiles of states."""
    mb.prof_enable(True)
    try:
        out = fn()
        ran = mb.prof_read()
    finally:
        mb.prof_enable(False)
    assert "cross_dkdv_wide" in ran, ran
    return out


@pytest.mark.parametrize("junk", [float("nan"), float("inf"), -3e38])
def test_wide_tiles_do_not_use_what_is_masked(junk):
    """States outside every range, and the queries (and their dO) of segments whose range is empty."""
    B, H, N, M, d = 2, 12, 4000, 700, 128
    q, k, v, d_o = inputs(B, H, H, N, M, d, torch.bfloat16)
    offs, ranges = [0, 1900, 2000, 4000], [[(3, 300), (0, 0), (333, 690)], [(0, 0), (70, 71), (64, 640)]]
    kw = dict(kv_ranges=device_ranges(ranges), q_offsets=offs)

    def run():
        o, lse = mb.cross_attn_fwd(q, k, v, **kw)
        return (o, lse, *mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw))

    want = ran_wide(run)
    for b in range(B):
        used = torch.zeros(M, dtype=torch.bool, device="cuda")
        for s, (a, e) in enumerate(ranges[b]):
            used[a:e] = True
            if e <= a:
                q[b, :, offs[s]:offs[s + 1]] = junk
                d_o[b, :, offs[s]:offs[s + 1]] = junk
        k[b, :, ~used] = junk
        v[b, :, ~used] = junk
    got = run()
    assert all(torch.equal(x, y) for x, y in zip(got, want))


def test_wide_tiles_captured():
    B, H, Hk, N, M, S, d = 1, 12, 6, 5000, 900, 3, 128
    q, k, v, d_o = inputs(B, H, Hk, N, M, d, torch.bfloat16)
    offs = [N * s // S for s in range(S + 1)]
    ranges = device_ranges([[(0, 900), (10, 20), (300, 900)]])
    ws = mb.cross_attn_workspace(B, H, Hk, N, M, d, torch.bfloat16, True, S)

    def both(ws=None):
        o, lse = mb.cross_attn_fwd(q, k, v, ranges, offs, workspace=ws)
        return (o, lse, *mb.cross_attn_bwd(q, k, v, o, lse, d_o, ranges, offs, workspace=ws))

    ran_wide(lambda: both(ws))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both(ws)
    for r in ([[(0, 900), (10, 20), (300, 900)]], [[(5, 5), (0, 899), (0, 899)]], [[(0, 256), (256, 512), (512, 900)]], [[(0, 0)] * 3]):
        ranges.copy_(device_ranges(r))
        want = [t.clone() for t in both()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), r


def test_wide_tiles_of_a_key_head_of_more_than_4_gib_of_queries():
    """Eight query heads on one key head, 17.6 million queries of it: the last of them."""
    d, H, N, M = 128, 8, 2_200_000, 300
    q = torch.zeros(1, H, N, d, dtype=torch.bfloat16, device="cuda")
    k, v = inputs(1, H, 1, 1, M, d, torch.bfloat16)[1:3]
    q[:, 7:, -100:] = mi.randn((1, 1, 100, d), 3, "cuda").to(torch.bfloat16)
    o, lse = mb.cross_attn_fwd(q, k, v)
    ref = reference(q[:, 7:, -100:], k, v, q[:, 7:, -100:], [[(0, M)]], [0, 100], d ** -0.5)
    near("o", o[:, 7:, -100:], ref["o"])
    dq, dk, dv = ran_wide(lambda: mb.cross_attn_bwd(q, k, v, o, lse, q))
    near("dq", dq[:, 7:, -100:], ref["dq"])
    near("dk", dk, ref["dk"])                # (the other queries and their dO are zero)
    near("dv", dv, ref["dv"])


@pytest.mark.parametrize("junk", [float("nan"), float("inf")])
@pytest.mark.parametrize("d,dtype,N,M", [(64, torch.bfloat16, 130, 100), (128, torch.bfloat16, 130, 100), (64, torch.float32, 130, 100),
                                         (128, torch.float32, 130, 100), (128, torch.bfloat16, 130, 30), (64, torch.float32, 130, 60),
                                         (128, torch.bfloat16, 9000, 900)])
def test_a_bad_query_reaches_its_own_states_alone(junk, d, dtype, N, M):
    """NaN or infinity in one query and its dO: the gradients of states that its segment does not attend, and the other queries, keep their bits."""
    H, Hk = (24, 12) if N > 1000 else (2, 1)
    q, k, v, d_o = inputs(1, H, Hk, N, M, d, dtype)
    offs = [0, N // 3, 2 * N // 3, N]
    ranges = [[(0, M * 37 // 100), (M * 37 // 100, M * 7 // 10), (M // 2, M)]]
    kw = dict(kv_ranges=device_ranges(ranges), q_offsets=offs)

    def run():
        o, lse = mb.cross_attn_fwd(q, k, v, **kw)
        return (o, lse, *mb.cross_attn_bwd(q, k, v, o, lse, d_o, **kw))

    want = run()
    bad = N // 2
    q[:, 0, bad] = junk
    d_o[:, 0, bad] = junk
    got = run()
    a, e = ranges[0][1]
    other = torch.ones(M, dtype=torch.bool, device="cuda")
    other[a:e] = False
    for x, y in zip(got[3:], want[3:]):
        assert torch.equal(x[:, :, other], y[:, :, other]) and not torch.isfinite(x[:, 0, ~other]).all(-1).any()
        assert torch.equal(x[:, 1:], y[:, 1:])
    for x, y in zip(got[:3], want[:3]):
        x[:, 0, bad] = y[:, 0, bad] = 0
        assert torch.equal(x, y)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_padded_batch_of_few_heads(dtype, d):
    """Items of the query passes are dealt out one by one, with and without segments, a last tile that is cut and parts of the ranges."""
    check(5, 2, 1, 1030, 300, d, dtype, ranges=[[(0, 300)], [(0, 0)], [(0, 1)], [(0, 131)], [(7, 290)]])
    check(2, 3, 3, 1100, 900, d, dtype, offs=[0, 500, 1100], ranges=[[(0, 900), (0, 900)], [(3, 20), (0, 0)]])
