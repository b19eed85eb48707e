"""Cross attention where sums are so long that one float chain of them would stall: millions of states of nearly equal probability, or millions
of queries of one key head, in calls of so many tiles that nothing has to be cut to fill the chip.

The queries are four rows repeated, so the formulas in 64 bits are formed for four of them. Tolerances as in test_gpu_cross.py, but a sum counts at
most ROW additions in a row, 2^-24 of the terms' magnitudes each, however long it is (2^16 matrix additions of sixteen products in bf16, 2^14
of two in fp32), and JOIN more where its parts are added."""
import math

import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: STEP}
ROW = {torch.bfloat16: 2 ** 16, torch.float32: 2 ** 14}
JOIN = 2 ** 8
VARIANTS = 4


def formulas(q, k, v, d_o, count, scale):
    """Values in 64 bits and bounds of `count` queries of each of the rows q, d_o [4, d] against k, v [M, d]."""
    half, adds, d = HALF[q.dtype], (ROW[q.dtype] + JOIN) * STEP, q.shape[-1]
    round_p = half if q.dtype == torch.bfloat16 else 0.0
    Q, K, V, DO = (x.double() for x in (q, k, v, d_o))
    L = Q @ K.T * scale
    el = 2 * (Q.abs() @ K.abs().T).amax(-1, keepdim=True) * scale * (d + 8) * STEP
    P = torch.softmax(L, -1)
    lse = torch.logsumexp(L, -1)
    el = el + 4 * STEP * (1 + lse.abs().max())                # (lse in float, in units of log 2, in the exponent)
    O = P @ V
    eo = (el + round_p + adds) * (P @ V.abs()) + half * O.abs()
    # the backward takes o and lse as they are stored
    delta = (DO * O.to(q.dtype).double()).sum(-1, keepdim=True)
    edelta = d * STEP * (DO.abs() * O.abs()).sum(-1, keepdim=True)
    dS = P * (DO @ V.T - delta)
    edS = (el + round_p + 4 * STEP) * dS.abs() + P * (edelta + d * STEP * (DO.abs() @ V.abs().T)) * (1 + round_p)
    dq, dk, dv = dS @ K * scale, count * (dS.T @ Q) * scale, count * (P.T @ DO)
    return dict(o=(O, eo), lse=(lse, el[:, 0] + adds), dq=(dq, ((edS + adds * dS.abs()) @ K.abs()) * scale + half * dq.abs()),
                dk=(dk, count * ((edS + adds * dS.abs()).T @ Q.abs()) * scale + half * dk.abs()),
                dv=(dv, count * ((P * (el + round_p + adds)).T @ DO.abs()) + half * dv.abs()))


def near(name, got, ref):
    value, bound = ref
    worst = float(((got.double() - value).abs() / bound).max())
    print(f"[long] {name}: {worst:.3f} of the bound", flush=True)
    assert worst <= 1, f"{name}: {worst:.2f} of the bound"


def inputs(N, M, d, dtype, spread):
    q4, do4 = (mi.randn((VARIANTS, d), s, "cuda").to(dtype) for s in (1, 2))
    k = (spread * mi.randn((M, d), 3, "cuda")).to(dtype)
    v = (0.3 + 0.1 * mi.randn((M, d), 4, "cuda")).to(dtype)
    rows = lambda x: x.repeat(N // VARIANTS, 1)[None, None]
    return q4, do4, k, v, rows(q4), rows(do4)


@pytest.mark.parametrize("dtype,d,M", [(torch.bfloat16, 128, 2 ** 22), (torch.float32, 64, 2 ** 20)])
def test_many_states_of_nearly_equal_probability(dtype, d, M):
    """1,025 tiles of queries: the range is not cut to fill the chip."""
    N = 131_200
    q4, do4, k, v, q, _ = inputs(N, M, d, dtype, 0.02)
    o, lse = mb.cross_attn_fwd(q, k[None, None], v[None, None])
    ref = formulas(q4, k, v, do4, N // VARIANTS, d ** -0.5)
    for j in range(VARIANTS):
        near("lse", lse[0, 0, j::VARIANTS], (ref["lse"][0][j], ref["lse"][1][j]))
        near("o", o[0, 0, j::VARIANTS], (ref["o"][0][j], ref["o"][1][j]))


@pytest.mark.parametrize("dtype,d,N,M", [(torch.float32, 64, 2 ** 21, 2 ** 16), (torch.bfloat16, 128, 1_310_720, 200_000)])
def test_many_queries_of_a_key_head(dtype, d, N, M):
    """512 tiles of 128 states, 782 of 256: the queries are not cut to fill the chip."""
    q4, do4, k, v, q, d_o = inputs(N, M, d, dtype, 0.02)
    ref = formulas(q4, k, v, do4, N // VARIANTS, d ** -0.5)
    rows = lambda x: x.repeat(N // VARIANTS, *[1] * (x.dim() - 1))[None, None].contiguous()
    dq, dk, dv = mb.cross_attn_bwd(q, k[None, None], v[None, None], rows(ref["o"][0].to(dtype)), rows(ref["lse"][0].float()), d_o)
    for j in range(VARIANTS):
        near("dq", dq[0, 0, j::VARIANTS], (ref["dq"][0][j], ref["dq"][1][j]))
    near("dk", dk[0, 0], ref["dk"])
    near("dv", dv[0, 0], ref["dv"])
