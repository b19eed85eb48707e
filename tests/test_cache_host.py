"""Refusals of the calls on the key / value cache: every one is answered on the host, before any device work, so no GPU
is needed. Pointers are made up and never followed."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2508_21058_amd import binding as mb

P = 1 << 40
STEP = 1 << 36          # apart from each other


def cache(k=P, v=P + STEP, ke=P + 2 * STEP, ve=P + 3 * STEP, table=P + 4 * STEP, pages=100, blocks=10, Hk=2, d=128):
    return mb._Cache(k, v, ke, ve, table, pages, blocks, Hk, d)


def rows(data=P + 5 * STEP, b=1 << 20, h=128, n=1 << 12):
    return mb._ROWS.pack(data or 0, b, h, n)


def ref(c):
    return None if c is None else C.byref(c)


def write(c=cache(), B=2, N=8, dt=0, k=rows(), v=rows(P + 6 * STEP), starts=P + 7 * STEP, counts=P + 8 * STEP):
    return mb.lib().moc_cache_write(ref(c), B, N, dt, k, v, starts, counts, None)


def read(c=cache(), B=2, N=8, dt=0, starts=P + 7 * STEP, counts=P + 8 * STEP, k=P + 5 * STEP, v=P + 6 * STEP):
    return mb.lib().moc_cache_read(ref(c), B, N, dt, starts, counts, k, v, None)


def attn(c=cache(), B=2, H=4, N=10, dt=0, q=P + 5 * STEP, S=1, off=None, ranges=P + 9 * STEP, scale=0.1, o=P + 6 * STEP, lse=P + 7 * STEP, ws=P + 8 * STEP,
         nbytes=1 << 30):
    off = None if off is None else np.ascontiguousarray(off, np.int32)
    return mb.lib().moc_cache_attn(ref(c), B, H, N, dt, q, S, None if off is None else off.ctypes.data, ranges, scale, o, lse, ws, nbytes, None)


def workspace(c=cache(), B=2, H=4, N=10, S=1, dt=0):
    n = C.c_size_t()
    return mb.lib().moc_cache_attn_workspace_bytes(ref(c), B, H, N, S, dt, C.byref(n)), n.value


CACHES = [      # what is wrong with the cache itself is refused by all of them
    (None, -1), (cache(k=None), -1), (cache(v=None), -1), (cache(ke=None), -1), (cache(ve=None), -1), (cache(table=None), -1),
    (cache(k=P + 8), -8), (cache(v=P + STEP + 4), -8), (cache(table=P + 4 * STEP + 2), -8), (cache(pages=0), -2), (cache(blocks=0), -2),
    (cache(Hk=0), -2), (cache(Hk=-1), -2), (cache(d=96), -2), (cache(d=256), -2), (cache(blocks=1 << 20), -2), (cache(blocks=(1 << 31) - 1), -2),
    (cache(Hk=1 << 16), -2),
]


@pytest.mark.parametrize("c,want", CACHES)
def test_caches_refused(c, want):
    assert write(c) == want and read(c) == want and attn(c, H=4 if c is None or c.Hk < 1 else 2 * c.Hk) == want
    assert workspace(c, H=4 if c is None or c.Hk < 1 else 2 * c.Hk)[0] == want
    assert mb.lib().moc_last_error() != b""


@pytest.mark.parametrize("call,want", [
    (dict(B=0), -2), (dict(N=0), -2), (dict(N=1 << 26), -2), (dict(B=40000), -2), (dict(dt=2), -6), (dict(k=None), -1), (dict(v=None), -1),
    (dict(k=rows(data=None)), -1), (dict(k=rows(data=P + 5 * STEP + 8)), -8), (dict(k=rows(n=132)), -8), (dict(v=rows(h=4)), -8), (dict(dt=1, v=rows(n=130)), -8),
    (dict(starts=P + 2), -8), (dict(counts=P + 1), -8), (dict(N=1 << 25, B=16), -2),
    (dict(k=rows(data=P)), -2), (dict(v=rows(data=P + STEP + 1024)), -2), (dict(k=rows(data=P - (1 << 13))), -2), (dict(starts=P + 2 * STEP), -2),
    (dict(counts=P + 4096), -2), (dict(c=cache(v=P + 4096)), -2), (dict(c=cache(ke=P + 16)), -2), (dict(c=cache(ve=P + 2 * STEP + 100)), -2),
    (dict(c=cache(table=P + 64)), -2),
])
def test_write_refuses(call, want):
    assert write(**call) == want
    assert mb.lib().moc_last_error() != b""


@pytest.mark.parametrize("call,want", [
    (dict(B=0), -2), (dict(N=0), -2), (dict(dt=7), -6), (dict(k=None, v=None), -1), (dict(k=P + 5 * STEP + 4), -8), (dict(v=P + 6 * STEP + 8), -8),
    (dict(starts=P + 2), -8), (dict(N=1 << 25, B=16), -2), (dict(k=P), -2), (dict(v=P + 5 * STEP + 64), -2), (dict(v=P + 4 * STEP), -2), (dict(k=P + 7 * STEP), -2),
    (dict(k=P + 2 * STEP), -2),
])
def test_read_refuses(call, want):
    assert read(**call) == want


@pytest.mark.parametrize("call,want", [
    (dict(B=0), -2), (dict(N=0), -2), (dict(H=0), -2), (dict(H=3), -2), (dict(H=-2), -2), (dict(B=20000), -2), (dict(N=1 << 25), -2), (dict(dt=3), -6),
    (dict(q=None), -1), (dict(o=None), -1), (dict(lse=None), -1), (dict(q=P + 5 * STEP + 8), -8), (dict(o=P + 6 * STEP + 4), -8), (dict(lse=P + 7 * STEP + 4), -8),
    (dict(scale=0.0), -2), (dict(scale=float("nan")), -2), (dict(scale=float("inf")), -2), (dict(scale=-1.0), -2), (dict(S=0), -2), (dict(S=129), -2),
    (dict(S=2), -1), (dict(S=2, off=[0, 5, 9]), -3), (dict(S=2, off=[1, 5, 10]), -3), (dict(S=3, off=[0, 7, 5, 10]), -3), (dict(ranges=P + 9 * STEP + 4), -8),
    (dict(ws=None, N=1, c=cache(blocks=1000)), -7), (dict(nbytes=16, N=1, c=cache(blocks=1000)), -7), (dict(ws=P + 8 * STEP + 8), -8),
    (dict(o=P), -2), (dict(o=P + 5 * STEP + 64), -2), (dict(lse=P + 4 * STEP), -2), (dict(lse=P + 6 * STEP), -2), (dict(o=P + 9 * STEP), -2),
    (dict(ws=P + 2 * STEP, N=1, c=cache(blocks=1000)), -2), (dict(ws=P + 6 * STEP, N=1, c=cache(blocks=1000)), -2),
])
def test_attn_refuses(call, want):
    assert attn(**call) == want
    assert mb.lib().moc_last_error() != b""


def test_workspace():
    rc, small = workspace(N=1, c=cache(blocks=1))
    assert rc == 0 and small == 0
    rc, n = workspace(N=1, c=cache(blocks=1000))
    assert rc == 0 and n > 0
    assert mb.lib().moc_cache_attn_workspace_bytes(ref(cache()), 2, 4, 10, 1, 0, None) == -1
    assert workspace(S=0)[0] == -2 and workspace(S=129)[0] == -2 and workspace(H=5)[0] == -2 and workspace(dt=9)[0] == -6
    # more parts than a launch has workgroups: 65535 heads of 67M positions
    assert workspace(B=1, H=65534, N=30000, c=cache(blocks=(1 << 20) - 1))[0] == -2


# ---- the binding's own checks ------------------------------------------------------------------------------------------

def host_cache(pages=4, Hk=2, d=64, B=2, blocks=2):
    return [torch.zeros(pages, Hk, 64, d, dtype=torch.uint8).view(torch.float8_e4m3fn) for _ in range(2)] + \
        [torch.zeros(pages, Hk, dtype=torch.int8) for _ in range(2)] + [torch.zeros(B, blocks, dtype=torch.int32)]


@pytest.mark.parametrize("at,new,error", [
    (0, lambda t: t[:, :, :32], ValueError), (1, lambda t: t[:2], ValueError), (0, lambda t: t.view(torch.int8), TypeError), (2, lambda t: t.int(), TypeError),
    (3, lambda t: t[:, :1], ValueError), (4, lambda t: t.long(), TypeError), (4, lambda t: t[0], TypeError), (4, lambda t: t.t(), ValueError),
    (2, lambda t: t.t().contiguous().t(), ValueError),
])
def test_cache_of_wrong_tensors(at, new, error):
    parts = host_cache()
    mb.KVCache(*parts)
    parts[at] = new(parts[at])
    with pytest.raises(error):
        mb.KVCache(*parts)


def test_empty_cache():
    c = mb.kv_cache(3, 130, 2, 64, device="cpu")
    assert c.table.tolist() == [[0, 1, 2], [3, 4, 5], [6, 7, 8]] and c.k.shape == (9, 2, 64, 64) and float(c.k.float().abs().sum()) == 0
    c = mb.kv_cache(3, 130, 2, 64, pages=5, device="cpu")
    assert c.pages == 5 and (c.table == -1).all()
    for bad in (dict(B=0), dict(tokens=0), dict(Hk=0), dict(pages=0)):
        with pytest.raises(ValueError):
            mb.kv_cache(**{**dict(B=1, tokens=1, Hk=1, d=64, device="cpu"), **bad})


def test_calls_of_wrong_tensors():
    c = mb.KVCache(*host_cache())
    x = torch.zeros(2, 2, 5, 64, dtype=torch.bfloat16)
    one = torch.zeros(2, dtype=torch.int32)
    bad = [lambda: mb.cache_write(c, x[:1], x[:1]), lambda: mb.cache_write(c, x, x[:, :, :4]), lambda: mb.cache_write(c, x[..., :32], x[..., :32]),
           lambda: mb.cache_write(c, x, x, one.long()), lambda: mb.cache_write(c, x, x, one[:1]), lambda: mb.cache_write(c, x, x, one, torch.zeros(4, dtype=torch.int32)[::2]),
           lambda: mb.cache_write(c, x, x, one), lambda: mb.cache_read(c, 5, one.float()), lambda: mb.cache_read(c, 5, out=(None, None)), lambda: mb.cache_read(c, 5),
           lambda: mb.cache_read(c, 4, out=(x, x)), lambda: mb.cache_attn(x[:1], c), lambda: mb.cache_attn(x.transpose(1, 2), c), lambda: mb.cache_attn(x, c),
           lambda: mb.cache_attn(x, c, kv_ranges=torch.zeros(2, 2, 2, dtype=torch.int32))]
    for call in bad:
        with pytest.raises(ValueError):
            call()
    for call in (lambda: mb.cache_write(c, x, x.float()), lambda: mb.cache_write(c, x.half(), x.half()), lambda: mb.cache_attn(x.half(), c)):
        with pytest.raises(TypeError):
            call()
