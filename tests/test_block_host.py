"""Refusals of the operators around the layer (head norms with rotation, rotation alone, cross attention): every one is
answered on the host, before any device work, so no GPU is needed. Pointers are made up and never followed."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2508_21058_amd import binding as mb

P = 0x10000


def rows(data=P, b=1 << 20, h=128, n=1 << 12):
    return mb._ROWS.pack(data or 0, b, h, n)


def plan(positions=P, freq=P, n_axes=3, pairs=(22, 21, 21), halves=0):
    return mb._RopePlan(positions, freq, n_axes, (C.c_int32 * 4)(*pairs), halves)


def ref(x):
    return x if x is None or isinstance(x, bytes) else C.byref(x)


def norm(B=1, N=8, H=2, Hk=2, d=128, dt=0, q=rows(), k=rows(), v=rows(), wq=P, wk=P, eps=1e-6, rope=plan(), out=(P, P, P)):
    return mb.lib().moc_qk_norm_rope(B, N, H, Hk, d, dt, ref(q), ref(k), ref(v), wq, wk, eps, ref(rope), *out, None)


def norm_bwd(B=1, N=8, H=2, Hk=2, d=128, dt=0, q=rows(), k=rows(), wq=P, wk=P, eps=1e-6, rope=plan(), g=(P, P, P),
             dq=rows(), dk=rows(), dv=rows(), dwq=P, dwk=P, ws=P, nbytes=1 << 30):
    return mb.lib().moc_qk_norm_rope_bwd(B, N, H, Hk, d, dt, ref(q), ref(k), wq, wk, eps, ref(rope), *g, ref(dq), ref(dk), ref(dv),
                                         dwq, dwk, ws, nbytes, None)


def turn(B=1, N=8, H=2, d=128, dt=0, x=rows(), rope=plan(), out=rows()):
    return mb.lib().moc_rope(B, N, H, d, dt, ref(x), ref(rope), 0, ref(out), None)


def cross(B=2, H=4, Hk=2, N=10, M=6, d=128, dt=0, S=1, off=None, ranges=None, scale=0.1, t=(P,) * 5, ws=P, nbytes=1 << 30):
    off = None if off is None else np.ascontiguousarray(off, np.int32)
    return mb.lib().moc_cross_attn_fwd(B, H, Hk, N, M, d, dt, *t[:3], S, None if off is None else off.ctypes.data, ranges, scale,
                                       *t[3:], ws, nbytes, None)


def cross_bwd(t=(P,) * 6, g=(P,) * 3, ws=P, nbytes=1 << 30, scale=0.1, S=1, off=None):
    off = None if off is None else np.ascontiguousarray(off, np.int32)
    return mb.lib().moc_cross_attn_bwd(2, 4, 2, 10, 6, 128, 0, *t, S, None if off is None else off.ctypes.data, None, scale, *g, ws,
                                       nbytes, None)


@pytest.mark.parametrize("call,want", [
    (dict(d=96), -2), (dict(B=0), -2), (dict(N=0), -2), (dict(H=0), -2), (dict(Hk=-1), -2), (dict(N=1 << 30, B=2), -2), (dict(N=1 << 27, B=2, H=1, Hk=1), -2),
    (dict(N=1 << 24, H=128), -2), (dict(dt=2), -6), (dict(eps=-1e-6), -2), (dict(eps=float("nan")), -2), (dict(eps=float("inf")), -2),
    (dict(q=None, k=None, v=None, out=(None,) * 3), -1), (dict(q=None), -1), (dict(out=(P, None, P)), -1),
    (dict(q=rows(data=None)), -1), (dict(q=rows(data=P + 8)), -8), (dict(k=rows(n=132)), -8), (dict(v=rows(h=4)), -8),
    (dict(B=2, q=rows(b=12)), -8), (dict(dt=1, q=rows(n=130)), -8), (dict(out=(P, P + 4, P)), -8), (dict(wq=P + 4), -8),
    (dict(rope=plan(positions=None)), -1), (dict(rope=plan(freq=None)), -1), (dict(rope=plan(positions=P + 2)), -8),
    (dict(rope=plan(freq=P + 4)), -8), (dict(rope=plan(n_axes=0)), -2), (dict(rope=plan(n_axes=5)), -2),
    (dict(rope=plan(pairs=(22, 21, 22))), -2), (dict(rope=plan(pairs=(70, -10, 4))), -2), (dict(d=64), -2),
    (dict(rope=plan(pairs=(2**31 - 1, 2**31 - 1, 2))), -2),
])
def test_norm_rope_refuses(call, want):
    assert norm(**call) == want
    assert mb.lib().moc_last_error() != b""


@pytest.mark.parametrize("call,want", [
    (dict(d=32), -2), (dict(dt=7), -6), (dict(eps=-1.0), -2), (dict(g=(None,) * 3, q=None, k=None, dq=None, dk=None, dv=None), -1),
    (dict(dq=None), -1), (dict(q=None), -1), (dict(g=(P, P, None)), -1), (dict(dv=None), -1), (dict(g=(P + 4, P, P)), -8),
    (dict(dq=rows(data=P + 2)), -8), (dict(dk=rows(n=4)), -8), (dict(dwq=P + 4), -8), (dict(ws=None), -7), (dict(nbytes=64), -7),
    (dict(ws=P + 8), -8), (dict(q=None, dq=None, g=(None, P, P)), -1), (dict(rope=plan(n_axes=9)), -2),
])
def test_norm_rope_backward_refuses(call, want):
    assert norm_bwd(**call) == want


@pytest.mark.parametrize("call,want", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(rope=None), -1), (dict(d=100), -2), (dict(H=0), -2), (dict(dt=-1), -6),
    (dict(x=rows(n=2)), -8), (dict(out=rows(data=P + 1)), -8), (dict(rope=plan(n_axes=0)), -2),
])
def test_rope_refuses(call, want):
    assert turn(**call) == want


@pytest.mark.parametrize("call,want", [
    (dict(H=3), -2), (dict(Hk=0), -2), (dict(N=0), -2), (dict(M=0), -2), (dict(B=-1), -2), (dict(d=256), -2), (dict(dt=5), -6),
    (dict(S=0), -2), (dict(S=129, off=[0] * 129 + [10]), -2), (dict(S=2), -1), (dict(S=2, off=[0, 4, 9]), -3),
    (dict(S=2, off=[1, 4, 10]), -3), (dict(S=3, off=[0, 6, 4, 10]), -3), (dict(S=2, off=[0, 12, 10]), -3), (dict(scale=0.0), -2),
    (dict(scale=-1.0), -2), (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(B=40000), -2), (dict(M=1 << 26), -2),
    (dict(N=1 << 26), -2), (dict(N=1 << 25), -2), (dict(B=1, H=64, Hk=1, N=1 << 25), -2), (dict(B=1, H=64, Hk=64, M=1 << 25), -2),
    (dict(B=65535, H=1, Hk=1, N=1, S=128, off=[0] * 128 + [1]), -2), (dict(B=3000, H=16, Hk=16, N=40000, S=128, off=[0] * 128 + [40000]), -2),
    (dict(t=(None, P, P, P, P)), -1), (dict(t=(P, P, P, P, None)), -1), (dict(t=(P, P + 8, P, P, P)), -8), (dict(ranges=P + 4), -8),
    (dict(ws=None, M=4096), -7), (dict(nbytes=16, M=4096), -7), (dict(ws=P + 4), -8),
])
def test_cross_attention_refuses(call, want):
    assert cross(**call) == want


@pytest.mark.parametrize("call,want", [
    (dict(t=(P, P, P, P, P, None)), -1), (dict(g=(P, None, P)), -1), (dict(g=(P, P, P + 2)), -8), (dict(ws=None), -7),
    (dict(nbytes=8), -7), (dict(ws=P + 4), -8), (dict(scale=-0.5), -2), (dict(S=4), -1), (dict(S=2, off=[0, 11, 10]), -3),
])
def test_cross_attention_backward_refuses(call, want):
    assert cross_bwd(**call) == want


def test_workspace_sizes():
    lib, n = mb.lib(), C.c_size_t()
    assert lib.moc_qk_norm_rope_workspace_bytes(1, 5, 2, 2, 128, 0, C.byref(n)) == 0 and 0 < n.value <= 1 << 20
    assert lib.moc_qk_norm_rope_workspace_bytes(1, 5, 2, 2, 128, 0, None) == -1
    assert lib.moc_qk_norm_rope_workspace_bytes(1, 0, 2, 2, 128, 0, C.byref(n)) == -2

    def size(B, H, Hk, N, M, S, bwd, d=128):
        assert lib.moc_cross_attn_workspace_bytes(B, H, Hk, N, M, d, S, 0, bwd, C.byref(n)) == 0
        return n.value

    assert size(1, 24, 24, 114368, 512, 1, 0) == 0                        # enough queries: nothing is split
    assert size(4, 12, 4, 1, 8192, 1, 0) > 0
    assert size(1, 24, 24, 114368, 512, 8, 1) >= 24 * 114368 * 16         # the statistics of the backward
    assert lib.moc_cross_attn_workspace_bytes(1, 1, 1, 1, 1, 128, 1, 0, 0, None) == -1
    # partial sums stay within a bound that does not grow with the call
    for shape in [(1, 24, 24, 4_000_000, 64), (1, 1, 1, 60_000_000, 1), (3, 8, 2, 1, 2_000_000), (1, 2, 1, 33_000_000, 100), (1, 48, 48, 700_000, 9000)]:
        stats = shape[0] * shape[1] * shape[3] * 16
        assert size(*shape, 1, 1) <= stats + (600 << 20), shape


@pytest.mark.parametrize("B,N,M", [(65535, 32640, 1), (1000, 1, 2147400)])
def test_more_workgroups_than_a_launch_has(B, N, M):
    """255 tiles of queries a sample and one workgroup more of each; 16,777 tiles of 128 states of 1,000 heads."""
    n = C.c_size_t()
    assert mb.lib().moc_cross_attn_workspace_bytes(B, 1, 1, N, M, 128, 1, 0, 1, C.byref(n)) == -2
    assert mb.lib().moc_cross_attn_workspace_bytes(B // 2, 1, 1, N, M, 128, 1, 0, 1, C.byref(n)) == 0


def test_binding_refuses_on_the_host():
    x = torch.zeros(1, 4, 2, 128)
    with pytest.raises(ValueError):
        mb.qk_norm_rope(x)                                                # not on a device
    with pytest.raises(ValueError):
        mb.qk_norm_rope(None)
    with pytest.raises(ValueError):
        mb.rope_plan(torch.zeros(4, 3, dtype=torch.int64), (22, 21, 21))
    with pytest.raises(ValueError):
        mb.rope_plan(torch.zeros(4, 3, dtype=torch.int32), (22, 21))
    with pytest.raises(ValueError):
        mb.rope_plan(torch.zeros(4, 2, dtype=torch.int32), (2, 2), freq=[1.0, 0.5, 0.25])
    with pytest.raises(ValueError):
        mb.cross_attn_fwd(x, x, x[:, :, :1])
    p = mb.rope_plan(torch.zeros(4, 3, dtype=torch.int32), (22, 21, 21))
    assert torch.allclose(p.freq[22:43], 10000.0 ** (-torch.arange(21, dtype=torch.float64) / 21))
