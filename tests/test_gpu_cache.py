"""The key / value cache in 8 bits: writing and reading against the definition in 64 bits, bit for bit, and attention over it
against the formula in 64 bits.

Written and read values have no tolerance: exponents follow from the largest magnitude alone, a power of two scales exactly, one rounding makes the
code, and bf16 and fp32 hold every code * 2^exponent.

Tolerances of the attention, element by element. A product of a bf16 query and a code is exact in float, and so is each of the three products that an fp32
query's terms make (three times eight bits are a float's 24); a logit is a float sum of d (fp32: 3 d) of them, off by at most that many times 2^-24
sum|q k| scale, and the exponent adds three roundings of values of the logits' size. In bf16 every probability is rounded before the second product,
half a step 2^-8, in fp32 its third term, 2^-24, and the result once more, 2^-8 or 2^-24. Sums over tokens stay in float: 2^-24 of the terms'
magnitudes for every add in a row, at most one per token summed, in fp32 three."""
import math

import numpy as np
import pytest
import torch

import moc_inputs as mi
from paper_2508_21058_amd import binding as mb

pytestmark = pytest.mark.gpu

STEP = 2.0 ** -24
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: STEP}
PAGE = mb.MOC_CACHE_PAGE
BAD = (-1, 1 << 30, -(1 << 31), (1 << 31) - 1)          # page numbers that are none


# ---- the definition -------------------------------------------------------------------------------------------------

def nearest_code(x):
    """The nearest e4m3 value of x (64 bits, |x| <= 448 where finite), ties to even; NaN for what is not finite."""
    _, e = np.frexp(x)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    return np.where(np.isfinite(x), np.round(np.where(np.isfinite(x), x, 0.0) / step) * step, np.nan)


def least_exponent(amax):
    """The least whole e in [-110, 120] with amax <= 448 * 2^e."""
    e = -110
    while e < 120 and amax > math.ldexp(448.0, e):
        e += 1
    return e


class Pool:
    """The cache in 64 bits: codes [pages, Hk, 64, d] as values, exponents."""

    def __init__(self, cache):
        self.table = cache.table.cpu().numpy()
        self.codes = [x.float().cpu().numpy().astype(np.float64) for x in (cache.k, cache.v)]
        self.exps = [x.cpu().numpy().astype(np.int64) for x in (cache.k_exp, cache.v_exp)]

    def page(self, b, pos):
        if pos < 0 or pos >= self.table.shape[1] * PAGE:
            return None
        p = int(self.table[b, pos // PAGE])
        return p if 0 <= p < self.codes[0].shape[0] else None

    def write(self, x, kv, starts, counts):
        """x [B, Hk, N, d] in 64 bits."""
        B, Hk, N, _ = x.shape
        codes, exps = self.codes[kv], self.exps[kv]
        for b in range(B):
            start, count = (0 if starts is None else int(starts[b])), (N if counts is None else min(max(int(counts[b]), 0), N))
            for block in range(start // PAGE, (start + max(count, 1) - 1) // PAGE + 1):
                at = [start + n for n in range(count) if (start + n) // PAGE == block]
                p = self.page(b, block * PAGE)
                if not at or p is None:
                    continue
                for h in range(Hk):
                    new = x[b, h, at[0] - start:at[-1] + 1 - start]
                    fine = np.abs(new[np.isfinite(new)])
                    e = least_exponent(fine.max() if fine.size else 0.0)
                    kept = at[0] - block * PAGE
                    if kept:
                        e = max(e, exps[p, h])
                        if e != exps[p, h]:
                            codes[p, h, :kept] = nearest_code(np.ldexp(codes[p, h, :kept], int(exps[p, h] - e)))
                    codes[p, h, kept:kept + len(at)] = nearest_code(np.ldexp(new, -e))
                    exps[p, h] = e

    def values(self, kv, b, h, pos):
        """[len(pos), d] values, and which of the positions are there."""
        out, there = np.zeros((len(pos), self.codes[0].shape[3])), np.zeros(len(pos), bool)
        for i, t in enumerate(pos):
            p = self.page(b, t)
            if p is not None:
                out[i], there[i] = np.ldexp(self.codes[kv][p, h, t % PAGE], int(self.exps[kv][p, h])), True
        return out, there


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def check_pool(cache, pool):
    for got, exp, kv in ((cache.k, cache.k_exp, 0), (cache.v, cache.v_exp, 1)):
        assert same(got.float().cpu().numpy().astype(np.float64), pool.codes[kv])
        assert np.array_equal(exp.cpu().numpy(), pool.exps[kv])


def scattered_cache(B, tokens, Hk, d, seed=0, holes=(), spare=2, filled=True):
    """A cache whose pages are in no order; holes: (sample, block) without a page. filled: of random codes, else of zeros."""
    blocks = -(-tokens // PAGE)
    g = np.random.default_rng(seed)
    c = mb.kv_cache(B, tokens, Hk, d, pages=B * blocks + spare)
    table = g.permutation(B * blocks + spare)[:B * blocks].reshape(B, blocks).astype(np.int32)
    for i, (b, block) in enumerate(holes):
        table[b, block] = BAD[i % len(BAD)] if i % len(BAD) else -1
    c.table.copy_(torch.from_numpy(table))
    if filled:
        for x, e in ((c.k, c.k_exp), (c.v, c.v_exp)):
            u = torch.from_numpy(g.integers(0, 256, tuple(x.shape), dtype=np.uint8))
            u = torch.where((u & 0x7f) == 0x7f, u & 0xf0, u)                       # no NaN
            x.view(torch.uint8).copy_(u)
            e.copy_(torch.from_numpy(g.integers(-9, -5, tuple(e.shape), dtype=np.int8)))
    return c


def strided(x, layout):
    """x [B, Hk, N, d] in another order of memory."""
    B, Hk, N, d = x.shape
    if layout == "heads":
        return x.contiguous()
    if layout == "tokens":
        return x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    fused = torch.full((B, N, 3 * Hk + 1, d), 777.0, dtype=x.dtype, device=x.device)
    fused[:, :, Hk:2 * Hk] = x.permute(0, 2, 1, 3)
    return fused[:, :, Hk:2 * Hk].permute(0, 2, 1, 3)


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def write_both(cache, pool, k, v, starts, counts, layout="heads"):
    for kv, x in enumerate((k, v)):
        pool.write(x.double().cpu().numpy(), kv, starts, counts)
    mb.cache_write(cache, strided(k, layout), strided(v, layout), i32(starts), i32(counts))


def states(B, Hk, N, d, dtype, seed, spread=3.0):
    """Tokens of different magnitudes, so that exponents differ and grow."""
    out = []
    for s in (seed, seed + 977):
        x = mi.randn((B, Hk, N, d), s, "cuda")
        out.append((x * torch.exp2(spread * mi.randn((B, Hk, N, 1), s + 31, "cuda").clamp(-3, 3))).to(dtype))
    return out


# ---- writing --------------------------------------------------------------------------------------------------------

WRITES = [      # B, Hk, N, tokens, starts, counts
    (1, 1, 1, 1, None, None), (1, 2, 64, 64, None, None), (2, 3, 1, 200, [5, 64], None), (3, 2, 65, 300, [63, 0, 130], [65, 0, 1]),
    (2, 1, 200, 256, [1, 56], [199, 200]), (1, 4, 130, 512, [62], None), (2, 2, 100, 128, [100, -37], None), (2, 2, 77, 100, [1 << 20, -(1 << 31)], None),
    (3, 1, 70, 140, [0, 7, 70], [-3, 1000, 70]), (1, 1, 66, 192, [63], None), (2, 2, 9, 64, [(1 << 31) - 1, 60], None),
]


@pytest.mark.parametrize("layout", ["heads", "tokens", "fused"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,Hk,N,tokens,starts,counts", WRITES)
def test_write(B, Hk, N, tokens, starts, counts, d, dtype, layout):
    cache = scattered_cache(B, tokens, Hk, d, seed=N)
    pool = Pool(cache)
    k, v = states(B, Hk, N, d, dtype, N + d)
    write_both(cache, pool, k, v, starts, counts, layout)
    check_pool(cache, pool)


def test_write_leaves_out_pages_that_are_not_there():
    cache = scattered_cache(3, 400, 2, 64, holes=[(0, 1), (1, 0), (1, 6), (2, 3), (2, 4)])
    pool = Pool(cache)
    k, v = states(3, 2, 390, 64, torch.bfloat16, 3)
    write_both(cache, pool, k, v, [3, 0, 10], [390, 380, 300])
    check_pool(cache, pool)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_write_token_by_token(dtype):
    """Exponents grow as tokens come, and what a page holds follows them."""
    cache = mb.kv_cache(2, 140, 2, 64)
    pool = Pool(cache)
    for t in range(135):
        k, v = states(2, 2, 1, 64, dtype, 100 + t)
        write_both(cache, pool, k, v, [t, t + 3], [1, t % 2])
    check_pool(cache, pool)


def test_write_again_ends_the_sample_there():
    """A second write of the same positions, as every denoising step of a frame makes it, finds nothing of the first."""
    cache = mb.kv_cache(1, 256, 2, 128)
    pool = Pool(cache)
    k, v = states(1, 2, 128, 128, torch.bfloat16, 5)
    write_both(cache, pool, k * 1000, v * 1000, [64], None)
    write_both(cache, pool, k[:, :, :100], v[:, :, :100], [64], None)
    check_pool(cache, pool)
    fresh = mb.kv_cache(1, 256, 2, 128)
    mb.cache_write(fresh, k[:, :, :100].contiguous(), v[:, :, :100].contiguous(), i32([64]))
    for a, b in ((cache.k, fresh.k), (cache.v, fresh.v)):
        assert torch.equal(a[1, :, :].view(torch.uint8), b[1].view(torch.uint8)) and torch.equal(a[2, :, :36].view(torch.uint8), b[2, :, :36].view(torch.uint8))
    assert torch.equal(cache.k_exp[1:3], fresh.k_exp[1:3]) and torch.equal(cache.v_exp[1:3], fresh.v_exp[1:3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_sample_without_tokens_writes_nothing(dtype):
    """Samples that ended keep their table row; the page that they end on is another sample's by now, or holds an exponent that no write leaves."""
    cache = scattered_cache(4, 128, 2, 64)
    cache.table[1] = cache.table[0]
    cache.table[3] = cache.table[0]
    for e in (cache.k_exp, cache.v_exp):
        e[int(cache.table[2, 0])] = 125
    pool = Pool(cache)
    k, v = states(4, 2, 70, 64, dtype, 8)
    write_both(cache, pool, k * 1000, v * 1000, [3, 20, 5, 80], [70, 0, 0, -4])
    check_pool(cache, pool)


SPECIAL = {
    "zeros": [0.0, -0.0], "one": [1.0], "most": [448.0, 449.0], "just over": [448.0 * (1 + 2 ** -7)], "ties": [1.0625, 1.1875, -1.0625, 17.0, 448.0],
    "subnormal": [448.0, 2.0 ** -10, 3 * 2.0 ** -10, 2.0 ** -9, 2.0 ** -6 - 2.0 ** -11, -(2.0 ** -10)], "tiny": [2.0 ** -126, 2.0 ** -120], "denormal": [2.0 ** -133, 2.0 ** -130],
    "huge": [2.0 ** 126, -(2.0 ** 120)], "nan": [1.0, math.nan, 3.0], "infinite": [math.inf, 2.0, -math.inf], "only nan": [math.nan], "most of bf16": [3.3895313892515355e38],
}


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("name", SPECIAL)
def test_write_special_values(name, dtype):
    values = torch.tensor(SPECIAL[name], dtype=torch.float64).to(dtype)
    k = values.repeat(64 * 64)[:64 * 40].reshape(1, 1, 40, 64).cuda()
    v = k.flip(2).contiguous()
    for start in (0, 20):
        cache = mb.kv_cache(1, 64, 1, 64)
        pool = Pool(cache)
        one = torch.full((1, 1, 20, 64), 0.37, dtype=dtype, device="cuda")
        write_both(cache, pool, one, one, [0], None)
        write_both(cache, pool, k, v, [start], None)
        check_pool(cache, pool)


def test_values_that_round_beyond_float():
    """248 * 2^120 and more are nearest to the code 256 or above it, 2^128 and more: infinite when read, less than that is finite."""
    k = torch.tensor([247.0, 247.5, 249.0, 255.0]).double().mul(2.0 ** 120).float().repeat(64)[:64].reshape(1, 1, 1, 64).cuda()
    cache = mb.kv_cache(1, 64, 1, 64)
    mb.cache_write(cache, k, -k)
    for dtype in (torch.bfloat16, torch.float32):
        got = mb.cache_read(cache, 1, dtype=dtype)
        want = torch.tensor([240.0 * 2.0 ** 120, 240.0 * 2.0 ** 120, math.inf, math.inf]).repeat(16).reshape(1, 1, 1, 64)
        assert torch.equal(got[0].float().cpu(), want) and torch.equal(got[1].float().cpu(), -want)
        for N in (1, 150):                                  # attended alone: the value itself
            o, _ = mb.cache_attn(torch.zeros(1, 1, N, 64, dtype=dtype, device="cuda"), cache, kv_ranges=i32([[[0, 1]]]))
            assert not torch.isfinite(o).any()              # (0 times an infinite key is NaN)


def test_every_code_follows_a_growing_exponent():
    """All codes of both signs, and exponents that grow by 0 to 20."""
    for grow in (0, 1, 2, 5, 8, 9, 17, 20):
        cache = mb.kv_cache(1, 64, 1, 64)
        cache.k.view(torch.uint8)[0, 0, :4] = torch.arange(256, dtype=torch.uint8, device="cuda").view(4, 64)
        cache.k_exp.fill_(0)
        pool = Pool(cache)
        x = torch.full((1, 1, 1, 64), 448.0 * 2.0 ** grow, dtype=torch.bfloat16, device="cuda")
        write_both(cache, pool, x, x, [4], None)
        check_pool(cache, pool)


# ---- reading --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,Hk,N,tokens,starts,counts", WRITES)
def test_read(B, Hk, N, tokens, starts, counts, d, dtype):
    holes = [(B - 1, 1)] if tokens > PAGE else []
    cache = scattered_cache(B, tokens, Hk, d, seed=N, holes=holes)
    pool = Pool(cache)
    got = mb.cache_read(cache, N, i32(starts), i32(counts), dtype=dtype)
    for kv in range(2):
        assert got[kv].dtype == dtype
        for b in range(B):
            start, count = (0 if starts is None else starts[b]), (N if counts is None else min(max(counts[b], 0), N))
            for h in range(Hk):
                want, _ = pool.values(kv, b, h, [start + n if n < count else -1 for n in range(N)])
                assert same(got[kv][b, h].double().cpu().numpy(), want)


def test_read_one_of_the_two_and_what_was_written():
    cache = scattered_cache(2, 300, 3, 128)
    k, v = states(2, 3, 150, 128, torch.bfloat16, 9)
    mb.cache_write(cache, k, v, i32([64, 7]))
    whole = mb.cache_read(cache, 150, i32([64, 7]))
    for i in range(2):
        out = [None, None]
        out[i] = torch.empty_like(whole[i])
        assert mb.cache_read(cache, 150, i32([64, 7]), out=out)[i] is out[i]
        assert torch.equal(out[i], whole[i])
    for got, x, e in ((whole[0], k, cache.k_exp), (whole[1], v, cache.v_exp)):       # half a step of four significant bits, or of a subnormal code
        size = torch.exp2(e.amax().double())
        assert ((got.double() - x.double()).abs() <= x.double().abs() * 2.0 ** -4 + size * 2.0 ** -10).all()


# ---- attention ------------------------------------------------------------------------------------------------------

def reference(q, pool, Hk, ranges, offs, scale):
    """{name: (value in 64 bits, how far each element may be off)}."""
    B, H, N, d = q.shape
    M, G, half, f32, dt = pool.table.shape[1] * PAGE, H // Hk, HALF[q.dtype], q.dtype == torch.float32, torch.float64
    o, eo = (torch.zeros(B, H, N, d, dtype=dt, device="cuda") for _ in range(2))
    lse, el_out = torch.full((B, H, N), -math.inf, dtype=dt, device="cuda"), torch.zeros(B, H, N, dtype=dt, device="cuda")
    values = [torch.from_numpy(np.ldexp(c, e[:, :, None, None].astype(np.int32))).cuda() for c, e in zip(pool.codes, pool.exps)]
    for b in range(B):
        page = torch.from_numpy(pool.table[b].astype(np.int64)).cuda()
        ok = (page >= 0) & (page < values[0].shape[0])
        there = ok.repeat_interleave(PAGE)
        for hk in range(Hk):
            K, V = (x[torch.where(ok, page, 0), hk].reshape(M, d) for x in values)
            for s in range(len(offs) - 1):
                a, e = (0, M) if ranges is None else ranges[b][s]
                a, e, q0, q1 = max(a, 0), min(e, M), offs[s], offs[s + 1]
                if e <= a or q1 <= q0 or not bool(there[a:e].any()):
                    continue
                k, v = K[a:e][there[a:e]], V[a:e][there[a:e]]
                adds = k.shape[0] * STEP
                for h in range(hk * G, hk * G + G):
                    Q = q[b, h, q0:q1].double()
                    L = Q @ k.T * scale
                    el = (Q.abs() @ k.abs().T).amax(-1, keepdim=True) * scale * ((3 if f32 else 1) * d + 8) * STEP
                    P = torch.softmax(L, -1)
                    o[b, h, q0:q1] = P @ v
                    eo[b, h, q0:q1] = (2 * el + half + (3 if f32 else 1) * adds + 4 * STEP) * (P @ v.abs()) + half * o[b, h, q0:q1].abs()
                    lse[b, h, q0:q1] = torch.logsumexp(L, -1)
                    el_out[b, h, q0:q1] = 2 * el[:, 0] + adds + 8 * STEP * (1 + lse[b, h, q0:q1].abs())
    return {"o": (o, eo), "lse": (lse, el_out)}


def near(name, got, ref):
    value, bound = ref
    assert not torch.isnan(got).any(), name
    off = torch.where(got.double() == value, torch.zeros_like(value), (got.double() - value).abs())
    worst = float((off / bound.clamp_min(1e-30)).max())
    print(f"[cache] {name}: {worst:.3f} of the bound")
    assert (off <= bound + 1e-30).all(), f"{name}: {worst:.2f} of the bound"


def check_attn(cache, H, N, dtype, ranges=None, offs=None, scale=None, seed=0):
    B, Hk, d = cache.B, cache.Hk, cache.d
    q = mi.randn((B, H, N, d), seed, "cuda").to(dtype)
    cuts = [0, N] if offs is None else offs
    ref = reference(q, Pool(cache), Hk, ranges, cuts, d ** -0.5 if scale is None else scale)
    kw = dict(kv_ranges=None if ranges is None else i32(ranges), q_offsets=offs, scale=scale)
    ws = mb.cache_attn_workspace(cache, H, N, dtype, len(cuts) - 1).fill_(255)      # whatever lies there is not read
    o, lse = mb.cache_attn(q, cache, workspace=ws, **kw)
    near("o", o, ref["o"])
    near("lse", lse, ref["lse"])
    assert (o[lse == -math.inf] == 0).all()
    again = mb.cache_attn(q, cache, **kw)
    assert torch.equal(o, again[0]) and torch.equal(lse, again[1])
    return o, lse


WHOLE = [       # B, H, Hk, N, tokens
    (1, 1, 1, 1, 1), (2, 3, 3, 1, 64), (1, 2, 1, 33, 65), (2, 4, 2, 32, 64), (1, 2, 2, 129, 128), (3, 6, 2, 100, 257), (1, 24, 24, 200, 200),
    (4, 12, 4, 1, 4100), (1, 8, 1, 3, 1000), (1, 1, 1, 1500, 60), (2, 16, 1, 5, 700), (1, 40, 1, 1, 400), (3, 12, 4, 11, 3000), (1, 2, 2, 1, 40000),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,H,Hk,N,tokens", WHOLE)
def test_everything_that_is_there(B, H, Hk, N, tokens, d, dtype):
    check_attn(scattered_cache(B, tokens, Hk, d, seed=tokens), H, N, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [1, 7, 150])
@pytest.mark.parametrize("d", [128, 64])
def test_padded_batch(d, N, dtype):
    """Lengths that end inside a page, at its end, of one token and of none."""
    check_attn(scattered_cache(6, 400, 2, d), 4, N, dtype, ranges=[[(0, 400)], [(0, 0)], [(0, 1)], [(0, 131)], [(0, 64)], [(0, 353)]])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hk", [3, 1])
def test_segments_with_their_own_ranges(Hk, dtype):
    """Segments of odd lengths (one empty), ranges that are unaligned, overlap, are empty, reversed or reach past the cache."""
    offs = [0, 1, 130, 130, 300, 355]
    ranges = [[(0, 7), (5, 140), (0, 300), (140, 141), (100, 300)], [(250, 260), (30, 30), (0, 300), (200, 100), (-50, 1 << 30)]]
    check_attn(scattered_cache(2, 300, Hk, 128), 3, 355, dtype, ranges=ranges, offs=offs)


def test_many_segments_and_another_scale():
    S, N = 128, 300
    offs = [N * s // S for s in range(S + 1)]
    check_attn(scattered_cache(1, 520, 1, 64), 2, N, torch.bfloat16, ranges=[[(4 * s, 4 * s + 1 + s % 12) for s in range(S)]], offs=offs, scale=0.31)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [1, 140])
def test_pages_that_are_not_there(N, dtype):
    """Holes at the begin, inside and at the end of ranges, numbers that are no pages, a sample without any page."""
    holes = [(0, 0), (0, 3), (0, 4), (1, 2), (1, 9)] + [(2, i) for i in range(10)] + [(3, i) for i in range(1, 10)]
    cache = scattered_cache(4, 640, 2, 128, holes=holes)
    ranges = [[(10, 300)], [(128, 640)], [(0, 640)], [(60, 640)]]
    o, lse = check_attn(cache, 4, N, dtype, ranges=ranges)
    assert (lse[2] == -math.inf).all() and (o[2] == 0).all()
    check_attn(cache, 4, N, dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [1, 20, 140])
@pytest.mark.parametrize("d", [128, 64])
def test_what_lies_outside_is_not_used(d, N, dtype):
    """NaN codes everywhere but in the ranges: before their begin, behind their end, on pages without a number."""
    cache = scattered_cache(2, 330, 2, d, holes=[(0, 2)])
    ranges = [[(37, 301)], [(64, 65)]]
    pool = Pool(cache)
    keep = torch.zeros(cache.pages, PAGE, dtype=torch.bool)
    for b in range(2):
        for t in range(*ranges[b][0]):
            p = pool.page(b, t)
            if p is not None:
                keep[p, t % PAGE] = True
    for x in (cache.k, cache.v):
        u = x.view(torch.uint8)
        u.copy_(torch.where(keep.cuda()[:, None, :, None], u, 0x7f))
    check_attn_values = check_attn(cache, 6, N, dtype, ranges=ranges)
    assert torch.isfinite(check_attn_values[0]).all()


def test_a_nan_stays_with_those_that_attend_it():
    cache = scattered_cache(2, 256, 1, 128)
    page = int(cache.table[0, 1])
    cache.v.view(torch.uint8)[page, 0, 10, 5] = 0x7f
    q = mi.randn((2, 2, 6, 128), 3, "cuda").to(torch.bfloat16)
    offs = [0, 2, 4, 6]
    o, lse = mb.cache_attn(q, cache, kv_ranges=i32([[(0, 74), (0, 75), (75, 256)]] * 2), q_offsets=offs)
    want = torch.zeros_like(o, dtype=torch.bool)
    want[0, :, 2:4, 5] = True
    assert torch.equal(torch.isnan(o), want) and torch.isfinite(lse).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [1, 30, 150])
def test_a_nan_key_stays_with_those_that_attend_it(N, dtype):
    cache = scattered_cache(2, 500, 1, 64)
    page = int(cache.table[1, 2])
    cache.k.view(torch.uint8)[page, 0, 0, 63] = 0xff
    q = mi.randn((2, 2, 3 * N, 64), 3, "cuda").to(dtype)
    offs = [0, N, 2 * N, 3 * N]
    o, lse = mb.cache_attn(q, cache, kv_ranges=i32([[(0, 128), (0, 129), (129, 500)]] * 2), q_offsets=offs)
    want = torch.zeros_like(lse, dtype=torch.bool)
    want[1, :, N:2 * N] = True
    assert torch.equal(torch.isnan(lse), want) and torch.equal(torch.isnan(o), want[..., None].expand_as(o))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [3, 30, 150])
def test_a_query_that_is_not_finite_stays_alone(N, dtype):
    cache = scattered_cache(1, 400, 1, 128)
    q = mi.randn((1, 2, N, 128), 3, "cuda").to(dtype)
    o, lse = mb.cache_attn(q, cache)
    bad = q.clone()
    bad[0, 0, 1, 5] = math.nan
    bad[0, 1, 2, 7] = math.inf
    o2, lse2 = mb.cache_attn(bad, cache)
    keep = torch.ones(1, 2, N, dtype=torch.bool, device="cuda")
    keep[0, 0, 1] = keep[0, 1, 2] = False
    assert torch.equal(o[keep], o2[keep]) and torch.equal(lse[keep], lse2[keep])
    assert torch.isnan(o2[~keep]).all()


def test_exponents_that_no_write_leaves():
    """-128 to -111 count as -110, 121 to 127 as 120, for reading, for attention and where a write finds them. (Values of 2^120 overflow in the sums: NaN
    on both sides is the same.)"""
    for given, taken in ((-128, -110), (-111, -110), (121, 120), (127, 120)):
        caches = []
        for e in (given, taken):
            c = scattered_cache(1, 64, 1, 64)
            c.k_exp.fill_(e)
            c.v_exp.fill_(e)
            x = torch.full((1, 1, 1, 64), 448.0 * 2.0 ** (100 if taken > 0 else -109), dtype=torch.bfloat16, device="cuda")
            read = mb.cache_read(c, 64)
            out = mb.cache_attn(x * 0, c)
            mb.cache_write(c, x, x, i32([10]))
            page = c.table[0].long()                          # (the pool's other pages keep what they were given)
            caches.append([t.float() for t in (*read, *out, c.k, c.v, c.k_exp[page], c.v_exp[page])])
        assert all(torch.allclose(a, b, rtol=0, atol=0, equal_nan=True) for a, b in zip(*caches))


def test_write_of_broadcast_inputs():
    cache = mb.kv_cache(3, 64, 2, 64)
    pool = Pool(cache)
    one = mi.randn((1, 1, 1, 64), 8, "cuda").to(torch.bfloat16)
    x = one.expand(3, 2, 40, 64)
    for kv in range(2):
        pool.write(x.double().cpu().numpy(), kv, [3, 0, 24], None)
    mb.cache_write(cache, x, x, i32([3, 0, 24]))
    check_pool(cache, pool)


def test_samples_share_pages():
    """A common beginning that two samples hold once."""
    cache = scattered_cache(2, 256, 2, 64)
    cache.table[1, :2] = cache.table[0, :2]
    check_attn(cache, 4, 9, torch.bfloat16, ranges=[[(0, 200)], [(0, 250)]])


@pytest.mark.parametrize("N", [1, 200])
def test_pool_of_more_than_four_gibibytes(N):
    """Pages at both ends of a pool whose byte offsets pass 32 bits."""
    Hk, d = 24, 128
    pages = (1 << 32) // (Hk * PAGE * d) + 40
    small = scattered_cache(2, 500, Hk, d)
    big = mb.kv_cache(2, 500, Hk, d, pages=pages)
    n = small.pages
    at = torch.cat((torch.arange(n // 2, device="cuda"), torch.arange(pages - n + n // 2, pages, device="cuda")))
    for x, y in ((big.k, small.k), (big.v, small.v)):
        x.view(torch.uint8)[at] = y.view(torch.uint8)
    big.k_exp[at], big.v_exp[at] = small.k_exp, small.v_exp
    big.table.copy_(at[small.table.long()].int())
    assert int(big.table.max()) * Hk * PAGE * d > 1 << 32
    k, v = states(2, Hk, 70, d, torch.bfloat16, 1)
    for c in (small, big):
        mb.cache_write(c, k, v, i32([100, 430]))
    for a, b in zip(mb.cache_read(small, 500), mb.cache_read(big, 500)):
        assert torch.equal(a, b)
    q = mi.randn((2, Hk, N, d), 5, "cuda").to(torch.bfloat16)
    for a, b in zip(mb.cache_attn(q, small), mb.cache_attn(q, big)):
        assert torch.equal(a, b)


def random_case(seed):
    g = np.random.default_rng(seed)
    B, Hk, G, S = int(g.integers(1, 4)), int(g.integers(1, 4)), int(g.choice([1, 2, 3, 4, 8])), int(g.choice([1, 1, 2, 5, 17]))
    N, tokens = int(2 ** g.uniform(0, 8)), int(2 ** g.uniform(0, 11))
    d, dtype = int(g.choice([64, 128, 128])), torch.bfloat16 if g.random() < 0.7 else torch.float32
    offs = [0] + sorted(g.integers(0, N + 1, S - 1).tolist()) + [N]
    blocks = -(-tokens // PAGE)
    holes = [(b, i) for b in range(B) for i in range(blocks) if g.random() < 0.15] if g.random() < 0.5 else []

    def one():
        a, b = g.integers(-3, tokens + 4, 2)
        return (int(a), int(b)) if g.random() < 0.5 else (0, int(b))
    ranges = None if g.random() < 0.2 else [[one() for _ in range(S)] for _ in range(B)]
    return scattered_cache(B, tokens, Hk, d, seed=seed, holes=holes), Hk * G, N, dtype, ranges, offs if S > 1 and ranges is not None else None


@pytest.mark.parametrize("seed", range(40))
def test_random_shapes(seed):
    cache, H, N, dtype, ranges, offs = random_case(seed)
    check_attn(cache, H, N, dtype, ranges=ranges, offs=offs, seed=seed)


LARGE = [       # B, H, Hk, N, tokens, segments: more tiles of queries than the chip takes at once, whole rounds and a rest that is cut
    (2, 24, 24, 2181, 5000, 1), (1, 12, 4, 9001, 7001, 1), (2, 24, 24, 2300, 4100, 3), (1, 24, 24, 1560, 9000, 1), (1, 8, 8, 13001, 300, 1), (3, 16, 2, 1500, 3000, 7),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("B,H,Hk,N,tokens,S", LARGE)
def test_large_calls(B, H, Hk, N, tokens, S, d, dtype):
    """Ranges of all samples and segments differ, one is empty; holes."""
    g = np.random.default_rng(N)
    cache = scattered_cache(B, tokens, Hk, d, seed=N, holes=[(b, i) for b in range(B) for i in range(3 + b, -(-tokens // PAGE), 9)])
    offs = [N * s // S + 3 * s for s in range(S)] + [N]
    ranges = [[(int(g.integers(0, tokens // 3)), int(g.integers(tokens // 2, tokens + 1))) for _ in range(S)] for _ in range(B)]
    if S > 1:
        ranges[0][1] = (77, 77)
    check_attn(cache, H, N, dtype, ranges=ranges, offs=offs if S > 1 else None)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [128, 64])
def test_segments_of_very_different_lengths(d, dtype):
    """Few queries a segment on average, one segment of many: several blocks of rows of it, in the kernels for few rows."""
    for N, offs in ((60, [0, 1, 2, 59, 60]), (300, [0, 0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 290, 290, 291, 292, 300]), (100, [0, 99, 100])):
        S = len(offs) - 1
        check_attn(scattered_cache(2, 700, 2, d), 2, N, dtype, ranges=[[(7 * s, 700 - 13 * s) for s in range(S)]] * 2, offs=offs)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows", [16, 17, 32, 33, 48, 64, 65, 128, 129])
@pytest.mark.parametrize("d", [128, 64])
def test_rows_around_the_kernels_blocks(d, rows, dtype):
    """Rows of a key head: one query of many heads, and many queries of one head."""
    for H, N in ((rows, 1), (1, rows)):
        check_attn(scattered_cache(2, 1500, 1, d), H, N, dtype, ranges=[[(5, 1500)], [(0, 333)]])


@pytest.mark.parametrize("N", [1, 70])
@pytest.mark.parametrize("dtype,tokens", [(torch.bfloat16, (1 << 20) + 5000), (torch.float32, (1 << 18) + 5000)])
def test_sums_longer_than_one_chain(dtype, tokens, N):
    """Equal probabilities of more tokens than are added in a row: no sum is more than 2^16 (fp32 2^14) matrix additions, whose error stays within
    2^-8 (2^-10) of what is added, in the weighted values and in the weights' own sum alike; the result's rounding is 2^-8 (2^-24)."""
    cache = mb.kv_cache(1, tokens, 1, 64)
    cache.k.view(torch.uint8).fill_(0x38)                     # 1.0
    cache.v.view(torch.uint8).fill_(0x38)
    cache.k_exp.fill_(0)
    cache.v_exp.fill_(1)
    q = mi.randn((1, 1, N, 64), 3, "cuda").to(dtype)
    o, lse = mb.cache_attn(q, cache, kv_ranges=i32([[(0, tokens)]]))
    error = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -10
    assert float((o.double() - 2).abs().max()) <= 2 * (2 * error + HALF[dtype])
    logit = q.double().sum(-1) * 64 ** -0.5
    assert float((lse.double() - logit - math.log(tokens)).abs().max()) <= error + 2.0 ** -14


@pytest.mark.parametrize("N", [1, 130])
def test_in_place_and_given_outputs(N):
    cache = scattered_cache(2, 300, 2, 128)
    q = mi.randn((2, 4, N, 128), 5, "cuda").to(torch.bfloat16)
    o, lse = mb.cache_attn(q, cache)
    out = (q.clone(), torch.empty_like(lse))
    got = mb.cache_attn(out[0], cache, out=out)
    assert got[0] is out[0] and torch.equal(out[0], o) and torch.equal(out[1], lse)


# ---- together -------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_rollout(dtype):
    """Frames of different counts are written and attended one after the other; what the cache holds is the definition's all along."""
    B, H, Hk, d, frame = 2, 4, 2, 128, 45
    cache = scattered_cache(B, 300, Hk, d, filled=False)
    pool = Pool(cache)
    held = [0, 0]
    for step in range(5):
        counts = [frame, frame - 7 * step]
        k, v = states(B, Hk, frame, d, dtype, step, spread=1.0)
        write_both(cache, pool, k, v, held, counts, "tokens")
        held = [h + c for h, c in zip(held, counts)]
        check_pool(cache, pool)
        check_attn(cache, H, frame, dtype, ranges=[[(max(0, h - 100), h)] for h in held], seed=step)


def test_as_cross_attention_to_the_values_read_back():
    """Attention over the cache is cross attention to what reading gives, up to the order of sums."""
    B, H, Hk, N, M, d = 2, 6, 2, 200, 640, 128
    cache = scattered_cache(B, M, Hk, d)
    k, v = mb.cache_read(cache, M)
    q = mi.randn((B, H, N, d), 1, "cuda").to(torch.bfloat16)
    ranges, offs = i32([[(0, 333), (100, 640)], [(5, 6), (0, 640)]]), [0, 90, N]
    o, lse = mb.cache_attn(q, cache, kv_ranges=ranges, q_offsets=offs)
    o2, lse2 = mb.cross_attn_fwd(q, k, v, kv_ranges=ranges, q_offsets=offs)
    # (each is off by a rounding of every probability, 2^-8, and of the result: of values that are at most the largest |v|)
    assert float((o.double() - o2.double()).abs().max()) <= 4 * 2.0 ** -8 * float(v.double().abs().max())
    assert float((lse - lse2).abs().max()) <= 1e-4


def test_the_layer_on_what_is_read_back():
    """A clip goes into the cache, comes back, and the layer routes and attends it as it does the same values from elsewhere."""
    lay = mi.multishot_layout(2, 48, 2, 390, 130, "frame")
    B, H, d, topk, N = 1, 2, 128, 2, lay.N
    q, k, v = (mi.randn((B, H, N, d), s, "cuda").to(torch.bfloat16) for s in (1, 2, 3))
    cache = scattered_cache(B, N, H, d, filled=False)
    pool = Pool(cache)
    write_both(cache, pool, k, v, None, None)
    k8, v8 = mb.cache_read(cache, N)
    want = [torch.from_numpy(np.stack([pool.values(kv, 0, h, range(N))[0] for h in range(H)])[None]).cuda().to(torch.bfloat16) for kv in range(2)]
    assert torch.equal(k8, want[0]) and torch.equal(v8, want[1])
    meta = mb.chunk_meta(lay.offsets, lay.shot, lay.window, lay.text_spans)
    _, sel = mb.route(meta, q, k8, topk)
    o, lse = mb.attn_fwd(meta, q, k8, v8, sel, d ** -0.5)
    assert torch.isfinite(o).all() and torch.isfinite(lse).all()


def test_another_stream():
    cache = scattered_cache(2, 500, 2, 128)
    k, v = states(2, 2, 30, 128, torch.bfloat16, 4)
    q = mi.randn((2, 4, 1, 128), 6, "cuda").to(torch.bfloat16)
    starts = i32([100, 470])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        mb.cache_write(cache, k, v, starts)
        got = mb.cache_attn(q, cache)
        back = mb.cache_read(cache, 30, starts)
    torch.cuda.current_stream().wait_stream(side)
    again = scattered_cache(2, 500, 2, 128)
    mb.cache_write(again, k, v, starts)
    for a, b in zip(got + back, mb.cache_attn(q, again) + mb.cache_read(again, 30, starts)):
        assert torch.equal(a, b)


@pytest.mark.parametrize("N", [1, 40])
def test_captured_steps(N):
    """A step (write behind what is held, attend all of it, advance) in a graph, replayed with eager work in between; two graphs of their own
    workspaces take turns."""
    B, H, Hk, d = 2, 4, 2, 64

    def world():
        w = dict(cache=scattered_cache(B, 1500, Hk, d, filled=False), k=torch.zeros(B, Hk, N, d, dtype=torch.bfloat16, device="cuda"),
                 v=torch.zeros(B, Hk, N, d, dtype=torch.bfloat16, device="cuda"), q=torch.zeros(B, H, N, d, dtype=torch.bfloat16, device="cuda"),
                 held=i32([0, 700]), ranges=torch.zeros(B, 1, 2, dtype=torch.int32, device="cuda"))
        w["ws"] = mb.cache_attn_workspace(w["cache"], H, N, torch.bfloat16)
        w["out"] = (torch.empty_like(w["q"]), torch.empty(B, H, N, device="cuda"))
        return w

    def step(w):
        mb.cache_write(w["cache"], w["k"], w["v"], w["held"])
        w["held"].add_(N)
        w["ranges"][:, 0, 1].copy_(w["held"])
        mb.cache_attn(w["q"], w["cache"], kv_ranges=w["ranges"], workspace=w["ws"], out=w["out"])

    graphs, worlds, eager = [], [world(), world()], [world(), world()]
    for w in worlds:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step(w)
        torch.cuda.current_stream().wait_stream(side)
        w["held"].copy_(i32([0, 700]))
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            step(w)
        graphs.append(g)
    for turn in range(6):
        for i, (g, w, e) in enumerate(zip(graphs, worlds, eager)):
            for x, s in (("k", 1), ("v", 2), ("q", 3)):
                fresh = mi.randn(tuple(w[x].shape), 100 * turn + 10 * i + s, "cuda").to(torch.bfloat16)
                w[x].copy_(fresh)
                e[x].copy_(fresh)
            g.replay()
            step(e)
            torch.cuda.synchronize()
            assert torch.equal(w["out"][0], e["out"][0]) and torch.equal(w["out"][1], e["out"][1])
            assert torch.equal(w["cache"].k_exp, e["cache"].k_exp)
