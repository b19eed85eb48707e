"""Performance cases of the key / value cache of a rollout, held in 8 bits: writing it, reading it back, attention over it.

The cache is a pool of pages of 64 tokens. Page p holds for key head h the e4m3 codes k[p, h], v[p, h] [64, d] and one exponent each; a value is
code * 2^exponent. Row b of the table names the pages of sample b: tokens [64 i, 64 i + 64) are on page table[b, i], or nowhere where that is -1.

A case is a plain dict. Common: B samples, Hk key heads, d features a head, dtype of what goes in or comes out, M tokens that the table has room for.
  op "write"  k, v [B, Hk, N, d] are slices of one fused projection [B, N, 3 Hk, d] and go to the positions from start on. ragged: samples begin at
              different positions and bring different counts (the second of three none). A block's exponent is the least one with every finite
              magnitude of it at most 448 * 2^e; where tokens in front of the new ones share the block it never falls, and their codes follow it.
  op "read"   N positions from start on come back as [B, Hk, N, d]; 0 behind a sample's count or where no page is.
  op "attn"   q [B, H, N, d] against the cache; the queries are `segments` equal pieces (frames, the last takes what is left). ranges "full"
              (all that the table has room for), "padded" (valid lengths differ), "frames" (the newest N tokens of a valid length are the queries' own, a piece attends up to
              its own end) or "window" (the same, but at most `window` tokens back). holes: every seventh page is gone.
  op "step"   a write of N tokens behind what the cache holds, and attention of their queries to all of it ("padded").
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_PAGE = 64
_LEAST, _MOST = -110, 120


def _case(name, op, **kw):
    case = dict(op=op, B=1, H=24, Hk=24, d=128, dtype="bf16", N=1560, M=33272, ragged=False, holes=False, segments=1, ranges="padded", window=0)
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one further token of an autoregressive rollout, batch of eight, inside blocks that hold tokens already: latency
        _case("write_one_token", "write", B=8, H=12, Hk=4, N=1, M=8192, ragged=True),
        # three new frames of 30 x 52 tokens behind a clip
        _case("write_frames", "write", N=4680, M=24064),
        # the benchmark's eight shots (114k tokens) at once
        _case("write_eight", "write", N=114368, M=114368),
        # a padded, odd-sized batch of fp32 projections, pages missing
        _case("write_ragged_f32", "write", B=3, H=6, Hk=2, d=64, dtype="f32", N=1301, M=3001, ragged=True, holes=True),
        # a 6k-token clip read back for the sparse layer
        _case("read_clip", "read", N=6256, M=6256),
        # odd sizes, fp32 out, different lengths
        _case("read_ragged_f32", "read", B=3, H=6, Hk=2, d=64, dtype="f32", N=1301, M=3001, ragged=True, holes=True),
        # one new token a sample, twelve query heads on four key heads, up to 8k tokens held: latency
        _case("attn_one_token", "attn", B=4, H=12, Hk=4, N=1, M=8192),
        # the same far into a long rollout, batch of eight, up to 131k tokens held
        _case("attn_one_token_long", "attn", B=8, H=12, Hk=4, N=1, M=131072),
        # one frame against a 33k-token clip
        _case("attn_frame", "attn", ranges="full"),
        # three frames at once in a batch of two, each up to its own end and at most eight frames back, pages of evicted frames gone
        _case("attn_frames_window", "attn", B=2, N=4680, M=20280, segments=3, ranges="window", window=12480, holes=True),
        # odd sizes, three samples, fewer key heads, fp32
        _case("attn_ragged_f32", "attn", B=3, H=6, Hk=2, d=64, dtype="f32", N=301, M=2003),
        # write and attention of a token together, as a rollout's layer runs them
        _case("step_one_token", "step", B=8, H=12, Hk=4, N=1, M=16384),
    ]


def draw(rng):
    """One more case of the listed ranges; never more work than half of the largest listed one of its kind."""
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    while True:
        op = rng.choice(["write", "read", "attn", "attn", "attn", "step"])
        Hk = rng.choice([1, 2, 3, 4, 6, 8, 12, 24])
        H = Hk * rng.choice([1, 1, 2, 3, 4, 8])
        if H > 48:
            continue
        kw = dict(B=rng.choice([1, 1, 2, 3, 4, 8]), H=H, Hk=Hk, d=128 if rng.random() < 0.7 else 64, dtype="f32" if rng.random() < 0.25 else "bf16",
                  holes=rng.random() < 0.3)
        M = log_int(1, 131072)
        N = 1 if rng.random() < 0.3 and op in ("attn", "step") else log_int(1, min(M, 60000))
        kw.update(N=N, M=M)
        if op in ("write", "read"):
            case = _case(None, op, ragged=rng.random() < 0.5, **kw)
            if work(case)["bytes"] <= 5e8 and case["B"] * Hk * M * case["d"] < 3e8:
                return case
            continue
        if op == "attn":
            segments = rng.choice([1, 1, 2, 3, 8, 17])
            kw.update(segments=segments, ranges=rng.choice(["full", "padded", "frames", "window"]), window=log_int(1, M))
            if segments > N:
                continue
        case = _case(None, op, **kw)
        most = 3e11 / (6 if case["dtype"] == "f32" else 1)
        if work(case)["flops"] <= most and case["B"] * H * N * M <= 6e8 and case["B"] * Hk * M * case["d"] < 3e8:
            return case


# ---- sizes --------------------------------------------------------------------------------------------------------

def _rng(case):
    return np.random.default_rng([case["B"], case["N"], case["M"], case["segments"], case["Hk"]])


def _places(case):
    """(start, count) of every sample for what is written or read."""
    B, N, M = case["B"], case["N"], case["M"]
    rng, out = _rng(case), []
    for b in range(B):
        if case["op"] == "step":        # behind what is held, which differs between samples
            out.append((int(rng.integers(0, M - N + 1)), N))
        elif case["ragged"]:
            out.append((int(rng.integers(0, M - N + 1)), 0 if B > 2 and b == 1 else int(rng.integers(max(1, N // 3), N + 1))))
        else:
            out.append((M - N, N))
    return out


def _cuts(case):
    N, S = case["N"], case["segments"]
    return [N // S * i for i in range(S)] + [N]


def _ranges(case):
    """[B][segments] of (first, end): the tokens that a piece of a sample's queries attends; None: all M."""
    B, N, M = case["B"], case["N"], case["M"]
    if case["op"] == "step":
        return [[(0, start + count)] for start, count in _places(case)]
    if case["ranges"] == "full":
        return None
    rng, cut, out = _rng(case), _cuts(case), []
    for b in range(B):
        held = max(1, int(M * rng.uniform(0.3, 1.0)))
        if case["ranges"] == "padded":
            out.append([(0, 0 if B > 2 and b == 1 and N > 1 else held)] * case["segments"])
            continue
        held = max(held, N)
        ends = [held - N + c for c in cut[1:]]
        out.append([(max(0, e - case["window"]) if case["ranges"] == "window" else 0, e) for e in ends])
    return out


def _table(case):
    """Pages of the samples in no order, and how many the pool has."""
    rng = _rng(case)
    B, blocks = case["B"], -(-case["M"] // _PAGE)
    table = rng.permutation(B * blocks + 3)[:B * blocks].reshape(B, blocks).astype(np.int32)
    if case["holes"]:
        table[:, 3::7] = -1
    return table, B * blocks + 3


# ---- inputs -------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    B, H, Hk, d, N = case["B"], case["H"], case["Hk"], case["d"], case["N"]
    table, pages = _table(case)
    st = dict(case=case, table=torch.from_numpy(table).cuda())
    for x in ("k", "v"):                    # heads differ in magnitude, and so do the blocks of a clip
        values = normal(pages, Hk, _PAGE, d)
        size = torch.exp2(torch.rand(pages, Hk, generator=g, device="cuda") * 2 - 1)
        e = _exponent(values.abs().amax((2, 3)) * size)
        st[x] = (values.mul_((size * _pow2(-e))[..., None, None])).clamp_(-448, 448).to(torch.float8_e4m3fn)
        st[x + "_exp"] = e.to(torch.int8)
        del values
    if case["op"] != "attn":
        places = _places(case)
        st["starts"] = torch.tensor([s for s, _ in places], dtype=torch.int32, device="cuda")
        st["counts"] = torch.tensor([n for _, n in places], dtype=torch.int32, device="cuda") if case["ragged"] else None
    if case["op"] in ("write", "step"):
        # (now and then a token that is larger than what its block has seen)
        st["kv"] = (normal(B, N, 3 * Hk, d) * torch.exp2(torch.floor(torch.rand(B, N, 1, 1, generator=g, device="cuda") * 4.2) - 1)).to(dtype)
    if case["op"] in ("attn", "step"):
        st["q"] = normal(B, H, N, d).to(dtype)
        ranges = _ranges(case)
        st["kv_ranges"] = None if ranges is None else torch.tensor(ranges, dtype=torch.int32, device="cuda")
        st["q_offsets"] = _cuts(case) if case["segments"] > 1 else None
    if own:
        from paper_2508_21058_amd import binding as mb
        st["cache"] = mb.KVCache(st["k"], st["v"], st["k_exp"], st["v_exp"], st["table"])
        if case["op"] in ("attn", "step"):
            st["ws"] = mb.cache_attn_workspace(st["cache"], H, N, dtype, segments=case["segments"])
    return st


def _held(st):
    return dict(k=st["k"], v=st["v"], k_exp=st["k_exp"], v_exp=st["v_exp"])


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    op, Hk = case["op"], case["Hk"]
    out = {}
    if op in ("write", "step"):
        k, v = (x.permute(0, 2, 1, 3) for x in st["kv"].split(Hk, dim=2)[1:])
        if own:
            from paper_2508_21058_amd import binding as mb
            mb.cache_write(st["cache"], k, v, st["starts"], st["counts"])
        else:
            _write(st, k, "k")
            _write(st, v, "v")
        out.update(_held(st))
    if op == "read":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        if own:
            from paper_2508_21058_amd import binding as mb
            out["k"], out["v"] = mb.cache_read(st["cache"], case["N"], st["starts"], st["counts"], dtype=dtype)
        else:
            out["k"], out["v"] = _read(st, "k").to(dtype), _read(st, "v").to(dtype)
    if op in ("attn", "step"):
        if own:
            from paper_2508_21058_amd import binding as mb
            out["o"], out["lse"] = mb.cache_attn(st["q"], st["cache"], kv_ranges=st["kv_ranges"], q_offsets=st["q_offsets"], workspace=st["ws"])
        else:
            out["o"], out["lse"] = _attend(st)
    return out


# ---- plain forms --------------------------------------------------------------------------------------------------

def _pow2(e):
    """2^e of integers, exactly."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _exponent(amax):
    """The least e with amax <= 448 * 2^e = 0.875 * 2^(e + 9)."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 9 + (m > 0.875).to(x.dtype), _LEAST).clamp(_LEAST, _MOST)


def _write(st, x, name):
    case, pool, exps, table = st["case"], st[name], st[name + "_exp"], st["table"]
    B, N = case["B"], case["N"]
    start = st["starts"].long()[:, None]
    count = N if st["counts"] is None else st["counts"].long()[:, None]
    block = start // _PAGE + torch.arange((N + _PAGE - 2) // _PAGE + 1, device=x.device)                # [B, blocks touched at most]
    pos = block[..., None] * _PAGE + torch.arange(_PAGE, device=x.device)                               # [B, blocks, 64]
    n = pos - start[..., None]
    new = (n >= 0) & (n < (count if isinstance(count, int) else count[..., None]))
    page = torch.gather(table.long(), 1, block.clamp(0, table.shape[1] - 1))
    valid = new.any(-1) & (block < table.shape[1]) & (page >= 0)
    page, pos, n, new = page[valid], pos[valid], n[valid], new[valid]                                   # [blocks, ...]
    b = torch.arange(B, device=x.device)[:, None].expand(valid.shape)[valid]
    fresh = x.permute(0, 2, 1, 3)[b[:, None], n.clamp(0, N - 1)].float().permute(0, 2, 1, 3)            # [blocks, Hk, 64, d]
    mark = new[:, None, :, None]
    kept = (pos < start[b])[:, None, :, None]
    old = exps[page].int()
    need = _exponent(torch.where(mark & torch.isfinite(fresh), fresh.abs(), 0.0).amax((2, 3)))
    e = torch.where(kept.any(2)[..., 0], torch.maximum(old, need), need)
    codes = pool[page]
    values = torch.where(mark, fresh * _pow2(-e)[..., None, None], codes.float() * torch.where(kept, _pow2((old - e).clamp(-126, 0))[..., None, None], 1.0))
    pool.view(torch.uint8)[page] = values.to(torch.float8_e4m3fn).view(torch.uint8)
    exps[page] = e.to(torch.int8)


def _values(st, name):
    """All that the table names, in 32 bits: [B, Hk, blocks * 64, d], 0 where no page is."""
    table = st["table"].long()
    there = (table >= 0)[..., None, None, None]
    x = st[name].view(torch.uint8)[table.clamp(min=0)].view(torch.float8_e4m3fn).float() * _pow2(st[name + "_exp"])[table.clamp(min=0)][..., None, None]
    x = torch.where(there, x, 0.0).permute(0, 2, 1, 3, 4)
    return x.reshape(x.shape[0], x.shape[1], -1, x.shape[-1])


def _read(st, name):
    case = st["case"]
    n = torch.arange(case["N"], device="cuda")
    pos = st["starts"].long()[:, None] + n
    x = _values(st, name)
    ok = pos < x.shape[2]
    if st["counts"] is not None:
        ok = ok & (n < st["counts"][:, None])
    index = pos.clamp(max=x.shape[2] - 1)[:, None, :, None].expand(-1, x.shape[1], -1, x.shape[3])
    return torch.where(ok[:, None, :, None], torch.gather(x, 2, index), 0.0)


def _attend(st):
    case, q = st["case"], st["q"]
    B, H, Hk, N, d = case["B"], case["H"], case["Hk"], case["N"], case["d"]
    k, v = _values(st, "k"), _values(st, "v")
    M = k.shape[2]
    t = torch.arange(M, device=q.device)
    seen = (st["table"] >= 0).repeat_interleave(_PAGE, 1)[:, None]                                      # [B, 1, M]
    if st["kv_ranges"] is not None:
        cut = torch.tensor(_cuts(case)[1:], device=q.device)
        piece = torch.searchsorted(cut, torch.arange(N, device=q.device), right=True)
        r = st["kv_ranges"][:, piece]                                                                   # [B, N, 2]
        seen = seen & (t >= r[..., :1]) & (t < r[..., 1:])
    seen = seen[:, None, None]                                                                          # [B, 1, 1, N or 1, M]
    s = torch.matmul(q.float().reshape(B, Hk, H // Hk * N, d), k.transpose(2, 3).contiguous()).reshape(B, Hk, H // Hk, N, M) * d ** -0.5
    s = torch.where(seen, s, -math.inf)
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0.0, m))
    z = p.sum(-1, keepdim=True)
    o = torch.matmul((p / torch.where(z > 0, z, 1.0)).reshape(B, Hk, H // Hk * N, M), v).reshape(B, H, N, d)
    return o.to(q.dtype), (m + torch.log(z)).reshape(B, H, N)


# ---- work ---------------------------------------------------------------------------------------------------------

def _pairs(case):
    """(query, token) pairs of one head, and tokens of the samples that some query attends."""
    table, _ = _table(case)
    there = np.repeat(table >= 0, _PAGE, 1)
    held = np.concatenate((np.zeros((case["B"], 1), np.int64), np.cumsum(there, 1)), 1)
    ranges, cut, room = _ranges(case), _cuts(case), there.shape[1]
    pairs = tokens = 0
    for b in range(case["B"]):
        row = [(0, room)] * case["segments"] if ranges is None else ranges[b]
        reached = np.zeros(room, bool)
        for s, (a, e) in enumerate(row):
            e = min(e, room)
            if e > a:
                pairs += int(held[b, e] - held[b, a]) * (cut[s + 1] - cut[s])
                reached[a:e] = True
        tokens += int((reached & there[b]).sum())
    return pairs, tokens


def work(case):
    B, H, Hk, d, N, op = case["B"], case["H"], case["Hk"], case["d"], case["N"], case["op"]
    e = 4 if case["dtype"] == "f32" else 2
    bytes_ = flops = 0.0
    if op != "attn":
        tokens = sum(n for _, n in _places(case))
        cells = 2.0 * tokens * Hk * d
        bytes_ += cells + (2.0 * B * N * Hk * d * e if op == "read" else cells * e)
        flops += cells * (1 if op == "read" else 3)
    if op in ("attn", "step"):
        pairs, tokens = _pairs(case)
        bytes_ += 2.0 * tokens * Hk * d + 2.0 * B * H * N * d * e + B * H * N * 4.0
        flops += 4.0 * d * H * pairs
    return {"bytes": bytes_, "flops": flops}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _power(e):
    """2^e of whole numbers in 64 bits, exactly (exp2 and ldexp are an ulp off for some of them)."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _nearest(x):
    """The nearest e4m3 value of |x| <= 448, ties to the even one: three bits behind the leading one, steps of 2^-9 below 2^-6."""
    _, power = torch.frexp(x)
    step = _power((power - 1).clamp(min=-6) - 3)
    return torch.where(torch.isfinite(x), torch.round(x / step) * step, math.nan)


def _exact_write(case, codes, exps, x, places, table):
    """The pool after the write, block by block; x [B, N, Hk, d]."""
    for b, (start, count) in enumerate(places):
        for block in range(start // _PAGE, (start + count + _PAGE - 1) // _PAGE):
            a, z = max(start, block * _PAGE), min(start + count, block * _PAGE + _PAGE)
            if z <= a or block >= table.shape[1] or table[b, block] < 0:
                continue
            page, at = int(table[b, block]), a - block * _PAGE
            new = x[b, a - start:z - start].transpose(0, 1).double()
            amax = torch.where(torch.isfinite(new), new.abs(), 0.0).amax((1, 2))
            e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448)).clamp(_LEAST, _MOST)
            # (a logarithm next to a whole number may be off: the least exponent is looked for around it)
            e = torch.where(amax <= 448 * _power(e - 1), e - 1, e)
            e = torch.where(amax > 448 * _power(e), e + 1, e).clamp(_LEAST, _MOST)
            if at > 0:
                old = exps[page].clone()
                e = torch.maximum(e, old)
                codes[page, :, :at] = _nearest(codes[page, :, :at] * _power(old - e)[:, None, None])
            codes[page, :, at:at + z - a] = _nearest(new * _power(-e)[:, None, None])
            exps[page] = e


def exact(case, seed):
    st = prepare(case, seed)
    op, Hk, d, N = case["op"], case["Hk"], case["d"], case["N"]
    table, _ = _table(case)
    codes, exps, out = {}, {}, {}
    for x in ("k", "v"):
        codes[x], exps[x] = st[x].double(), st[x + "_exp"].double()
    if op in ("write", "step"):
        places = _places(case)
        for i, x in enumerate(("k", "v")):
            _exact_write(case, codes[x], exps[x], st["kv"][:, :, (i + 1) * Hk:(i + 2) * Hk], places, table)
            out[x], out[x + "_exp"] = codes[x], exps[x].to(torch.int64)

    def row(name, b, h):
        """Values of a sample's head, [blocks * 64, d]; 0 where no page is."""
        at = torch.from_numpy(table[b].astype(np.int64)).cuda()
        v = codes[name][at.clamp(min=0), h] * _power(exps[name][at.clamp(min=0), h])[:, None, None]
        return torch.where((at >= 0)[:, None, None], v, 0.0).reshape(-1, d)

    if op == "read":
        for x in ("k", "v"):
            out[x] = torch.zeros(case["B"], Hk, N, d, dtype=torch.float64, device="cuda")
            for b, (start, count) in enumerate(_places(case)):
                for h in range(Hk):
                    got = row(x, b, h)[start:start + count]
                    out[x][b, h, :got.shape[0]] = got
    if op in ("attn", "step"):
        G, cut, ranges = case["H"] // Hk, _cuts(case), _ranges(case)
        out["o"] = torch.zeros(st["q"].shape, dtype=torch.float64, device="cuda")
        out["lse"] = torch.full(st["q"].shape[:3], -math.inf, dtype=torch.float64, device="cuda")
        for b in range(case["B"]):
            there = torch.from_numpy(np.repeat(table[b] >= 0, _PAGE)).cuda()
            for h in range(Hk):
                k, v = row("k", b, h), row("v", b, h)
                for s in range(case["segments"]):
                    a, e = (0, k.shape[0]) if ranges is None else ranges[b][s]
                    keep = there[a:e]
                    if e <= a or not bool(keep.any()):
                        continue
                    hs, qs = slice(h * G, h * G + G), slice(cut[s], cut[s + 1])
                    logit = st["q"][b, hs, qs].double() @ k[a:e][keep].T * d ** -0.5
                    out["o"][b, hs, qs] = torch.softmax(logit, -1) @ v[a:e][keep]
                    out["lse"][b, hs, qs] = torch.logsumexp(logit, -1)
    return out
