"""Sizes at the edge of what cross attention and the head norms take: answered on the host, so no GPU is needed."""
import ctypes as C

import pytest
import torch

from paper_2508_21058_amd import binding as mb


def cross_bytes(B, H, Hk, N, M, d=128, S=1, dt=0, bwd=1):
    """Workspace bytes, or the (negative) refusal."""
    n = C.c_size_t()
    rc = mb.lib().moc_cross_attn_workspace_bytes(B, H, Hk, N, M, d, S, dt, bwd, C.byref(n))
    return n.value if rc == 0 else rc


@pytest.mark.parametrize("dt,terms", [(0, 1 << 20), (1, 1 << 15)])
def test_long_sums_are_cut_however_well_a_call_fills_the_chip(dt, terms):
    """1,025 tiles of queries, or of states: without a limit of their length such sums are one part, without room for others."""
    N = 131_200
    assert cross_bytes(1, 1, 1, N, terms, dt=dt, bwd=0) == 0
    for parts in (2, 5):
        assert cross_bytes(1, 1, 1, N, (parts - 1) * terms + 1, dt=dt, bwd=0) >= parts * N * (128 + 1) * 4
    M = 262_400
    for parts in (1, 2, 5):
        queries = max((parts - 1) * terms + 1, 1 << 14)
        stats, sums = queries * 16, parts * M * 2 * 128 * 4 if parts > 1 else 0
        assert cross_bytes(1, 1, 1, queries, M, dt=dt) - stats >= sums
    # the queries of all heads of a key head count
    assert cross_bytes(1, 8, 1, terms // 4, M, dt=dt) >= 2 * M * 2 * 128 * 4


def test_parts_that_no_launch_has_room_for():
    assert cross_bytes(1, 1024, 1, 65_000, 1 << 25, bwd=0) > 0              # 508 x 1,024 tiles in 32 parts
    assert cross_bytes(1, 1024, 1, 65_000, (1 << 25) + 1, bwd=0) == -2      # ... in 33
    assert cross_bytes(2, 65, 65, 1 << 20, 1 << 15, dt=1, bwd=0) >= 0
    assert cross_bytes(2, 65, 65, 1 << 20, (1 << 15) + 1, dt=1, bwd=0) == -2     # more rows than a launch joins
    assert cross_bytes(1, 16, 16, 1 << 15, 1 << 21, dt=1) > 0               # 2^18 tiles of states
    assert cross_bytes(1, 16, 16, 1 << 21, 1 << 21, dt=1) == -2             # ... of which each has its queries in 64 parts
    assert cross_bytes(1, 16, 16, 1 << 15, 1 << 22, dt=1) > 0
    assert cross_bytes(1, 32, 16, (1 << 14) + 1, 1 << 22, dt=1) == -2       # 2^26 states in two parts, more than a launch adds


P = 0x10000
LAST_128 = (1 << 28) - 16       # tokens of 2^24 - 1 workgroups of sixteen


def rows():
    return mb._ROWS.pack(P, 128, 128, 128)


def rope():
    return C.byref(mb._RopePlan(P, P, 1, (C.c_int32 * 4)(10, 0, 0, 0), 0))


def norm_bytes(B, N, d):
    n = C.c_size_t()
    return mb.lib().moc_qk_norm_rope_workspace_bytes(B, N, 1, 1, d, 0, C.byref(n))


def norm_forward(B, N, d):
    return mb.lib().moc_qk_norm_rope(B, N, 1, 1, d, 0, rows(), None, None, None, None, 1e-6, None, P, None, None, None)


def norm_backward(B, N, d):
    return mb.lib().moc_qk_norm_rope_bwd(B, N, 1, 1, d, 0, rows(), None, None, None, 1e-6, None, P, None, None, rows(), None, None, None, None,
                                         P, 1 << 30, None)


def turn(B, N, d):
    return mb.lib().moc_rope(B, N, 1, d, 0, rows(), rope(), 0, rows(), None)


@pytest.mark.parametrize("call", [norm_bytes, norm_forward, norm_backward, turn])
@pytest.mark.parametrize("B,N,d", [(1, LAST_128 + 1, 128), (1, (1 << 28) - 1, 128), (3, (1 << 28) // 3, 128), (1, 1 << 28, 64)])
def test_tokens_of_2_24_workgroups_are_refused(call, B, N, d):
    assert call(B, N, d) == -2


def test_tokens_that_a_launch_holds():
    assert norm_bytes(1, LAST_128, 128) == 0 and norm_bytes(1, (1 << 28) - 1, 64) == 0


# ---- tensors on top of one another: made-up addresses, far apart unless a case says otherwise. B = 2, H = 4, Hk = 2, N = 10, M = 600, 128 features, bf16
MIB = 1 << 20
Q_BYTES, K_BYTES, LSE_BYTES = 2 * 4 * 10 * 128 * 2, 2 * 2 * 600 * 128 * 2, 2 * 4 * 10 * 4
AT = {n: (i + 1) * 64 * MIB for i, n in enumerate(("q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "ranges", "ws"))}


def cross_at(backward, **moved):
    p = {**AT, **moved}
    head, mid = (2, 4, 2, 10, 600, 128, 0, p["q"], p["k"], p["v"]), (1, None, p["ranges"], 0.1)
    if backward:
        return mb.lib().moc_cross_attn_bwd(*head, p["o"], p["lse"], p["d_o"], *mid, p["dq"], p["dk"], p["dv"], p["ws"], 32 * MIB, None)
    return mb.lib().moc_cross_attn_fwd(*head, *mid, p["o"], p["lse"], p["ws"], 32 * MIB, None)


@pytest.mark.parametrize("moved", [
    dict(o=AT["q"] + 16), dict(o=AT["q"] + Q_BYTES - 16), dict(o=AT["q"] - Q_BYTES + 16), dict(o=AT["k"]), dict(o=AT["v"] + K_BYTES - 16), dict(lse=AT["q"]),
    dict(lse=AT["o"] + Q_BYTES - 16), dict(lse=AT["k"] - LSE_BYTES + 16), dict(o=AT["ranges"]), dict(lse=AT["ranges"]), dict(ws=AT["q"]), dict(ws=AT["k"] + K_BYTES - 16),
    dict(ws=AT["o"]), dict(ws=AT["ranges"]),
])
def test_cross_attention_refuses_overlaps(moved):
    assert cross_at(False, **moved) == -2
    assert b"overlap" in mb.lib().moc_last_error()


@pytest.mark.parametrize("moved", [
    dict(dq=AT["q"]), dict(dq=AT["d_o"]), dict(dq=AT["o"] + 32), dict(dq=AT["k"]), dict(dq=AT["lse"]), dict(dk=AT["q"]), dict(dk=AT["d_o"] - K_BYTES + 16), dict(dk=AT["v"]),
    dict(dk=AT["k"] + 256), dict(dv=AT["k"]), dict(dv=AT["v"] - 256), dict(dv=AT["dk"] + K_BYTES - 16), dict(dk=AT["dq"]), dict(dv=AT["dq"] + 16), dict(dq=AT["ranges"]),
    dict(ws=AT["lse"]), dict(ws=AT["dv"]), dict(ws=AT["d_o"] - 256), dict(dv=AT["ranges"]),
])
def test_cross_attention_backward_refuses_overlaps(moved):
    assert cross_at(True, **moved) == -2
    assert b"overlap" in mb.lib().moc_last_error()


# ---- outputs whose rows lie on top of one another: B = 2, N = 8, H = 2 and Hk = 2 heads of 128 features
def turn_into(out):
    return mb.lib().moc_rope(2, 8, 2, 128, 0, mb._ROWS.pack(P, 2048, 128, 256), rope(), 0, out, None)


def norm_backward_into(dq=None, dk=None, dv=None):
    far = [mb._ROWS.pack((i + 1) << 24, 2048, 128, 256) for i in range(3)]
    x = mb._ROWS.pack(P, 2048, 128, 256)
    return mb.lib().moc_qk_norm_rope_bwd(2, 8, 2, 2, 128, 0, x, x, None, None, 1e-6, None, P, P, P, dq or far[0], dk or far[1], dv or far[2], None, None,
                                         P, 1 << 30, None)


OVERLAID = [(0, 128, 256), (2048, 0, 256), (2048, 128, 0), (2048, 64, 256), (2048, 2048, 120), (-64, 128, 256)]       # strides of samples, heads, tokens


@pytest.mark.parametrize("strides", OVERLAID)
def test_output_rows_on_top_of_one_another_are_refused(strides):
    out = mb._ROWS.pack(1 << 24, *strides)
    assert turn_into(out) == -2
    for name in ("dq", "dk", "dv"):
        assert norm_backward_into(**{name: out}) == -2
    assert b"overlap" in mb.lib().moc_last_error()


def test_workspaces_count_what_lies_behind_their_address():
    whole = torch.empty(64, dtype=torch.uint8)
    assert mb._scratch(whole) == (whole.data_ptr(), 64) and mb._scratch(whole.view(torch.float32))[1] == 64
    for ws in (whole[:1].expand(1 << 20), whole[::2], whole.view(8, 8)[:, :4]):
        with pytest.raises(ValueError):
            mb._scratch(ws)
