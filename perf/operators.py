"""Performance cases of the operators around the attention layer of a video transformer block: norms of queries and keys
with the rotation by time, height and width, the rotation alone, and cross attention to an encoder's states.

A case is a plain dict. Common: B samples, H query heads, Hk key / value heads, d features a head, dtype, path.
  op "norm_rope"   q, k, v are slices of one fused projection [B, N, H + 2 Hk, d]; q and k of every head are RMS-normalised
                   with a weight of d values and rotated, and q, k, v leave head-major [B, H, N, d], as routing and attention
                   take them. path "forward", "backward" or "train" (both).
  op "rope"        rotation alone of one token-major tensor [B, N, H, d] to a head-major one. path "forward" or "inverse" (the
                   gradient of the rotation, head-major to head-major).
  op "cross"       q [B, H, N, d] against encoder states k, v [B, Hk, M, d]. The stream is `segments` equal pieces (shots, the last takes
                   what is left); a piece of a sample attends a range of the states. ranges "full", "padded" (valid lengths differ
                   between samples, one sample has none where B > 2) or "shots" (piece s attends its own caption, a part of the s-th
                   piece of the states). path "forward", "backward" or "train".
The stream of the first two ops is `shots` times (`text` caption tokens, `frames` frames of gh x gw tokens); a caption token sits at its
shot's first time step, a video token at (frame, row, column). `t0` is the time of the first frame. `pairing` is "adjacent" (features
2j, 2j+1 are a pair) or "halves" (j, j + d/2); `axes` says how many of the d/2 pairs turn with time, height and width.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_EPS = 1e-6
_BASE = 10000.0


def _case(name, op, path, **kw):
    case = dict(op=op, path=path, B=1, H=24, Hk=24, d=128, dtype="bf16")
    if op == "cross":
        case.update(N=1560, M=512, segments=1, ranges="full")
    else:
        case.update(shots=1, text=256, frames=9, gh=30, gw=52, t0=0, pairing="adjacent", axes="22,21,21")
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # the smallest layer of the repository (1,088 tokens, two heads of 64 features, fp32 storage): latency
        _case("norm_rope_tiny_f32_train", "norm_rope", "train", text=64, frames=4, gh=16, gw=16, H=2, Hk=2, d=64, dtype="f32",
              axes="12,10,10"),
        # one sampling step of a 6k-token clip (8 s at 320 x 192)
        _case("norm_rope_short_forward", "norm_rope", "forward", frames=25, gh=12, gw=20),
        # the benchmark's eight shots (114k tokens) in training: fused projection in, its gradient out
        _case("norm_rope_eight_train", "norm_rope", "train", shots=8),
        # a padded, odd-sized batch of two with fewer key heads, pairs half a head apart, far from the stream's start
        _case("norm_rope_ragged_backward", "norm_rope", "backward", B=2, shots=3, text=77, frames=10, gh=17, gw=31, H=12, Hk=4, d=64,
              pairing="halves", axes="16,8,8", t0=100000),
        # one further token of an autoregressive rollout, batch of eight: latency
        _case("rope_one_token", "rope", "forward", B=8, text=1, frames=0, H=12, Hk=12, pairing="halves", t0=4096),
        # queries of a 33k-token single-shot layer
        _case("rope_single_forward", "rope", "forward", text=512, frames=21),
        # the gradient on its way back through the rotation, fp32 storage, odd sizes
        _case("rope_ragged_f32_inverse", "rope", "inverse", B=2, shots=2, text=119, frames=8, gh=23, gw=37, H=6, Hk=6, dtype="f32"),
        # prompts of a batch of two, padded to 512 states, one sampling step of the 6k-token clip
        _case("cross_short_forward", "cross", "forward", B=2, N=6256, ranges="padded"),
        # the benchmark's eight shots, each attending its own caption's states, in training
        _case("cross_eight_train", "cross", "train", N=114368, M=4096, segments=8, ranges="shots"),
        # image and text states together (a long encoder) in the 33k-token layer's backward
        _case("cross_single_long_backward", "cross", "backward", N=33272, M=4357),
        # one new token a sample against long padded states, twelve query heads on four key heads
        _case("cross_one_token_forward", "cross", "forward", B=4, N=1, M=8192, H=12, Hk=4, ranges="padded"),
        # odd sizes, three samples (one without any state), fewer key heads, fp32 storage
        _case("cross_ragged_f32_train", "cross", "train", B=3, N=1301, M=77, H=6, Hk=2, d=64, dtype="f32", ranges="padded"),
    ]


def draw(rng):
    """One more case of the listed ranges; never more work than half of the largest listed one of its kind."""
    def log_int(lo, hi):
        return int(round(lo * (hi / lo) ** rng.random()))

    most = {"norm_rope": work(listed()[2])["bytes"] / 2, "rope": work(listed()[2])["bytes"] / 2, "cross": work(listed()[8])["flops"] / 2}
    while True:
        op = rng.choice(["norm_rope", "rope", "cross", "cross"])
        dtype = "f32" if rng.random() < 0.25 else "bf16"
        d = 128 if rng.random() < 0.7 else 64
        Hk = rng.choice([1, 2, 3, 4, 6, 8, 12, 24])
        H = Hk * rng.choice([1, 1, 1, 2, 3, 4])
        kw = dict(B=rng.choice([1, 1, 2, 3, 4]), H=H, Hk=Hk, d=d, dtype=dtype)
        if H > 48:
            continue
        if op == "cross":
            kw.update(N=log_int(1, 120000), M=log_int(1, 9000), segments=rng.choice([1, 1, 2, 3, 8, 17]),
                      ranges=rng.choice(["full", "padded", "shots"]))
            if kw["segments"] > kw["N"] or kw["segments"] > kw["M"]:
                continue
            case = _case(None, op, rng.choice(["forward", "backward", "train"]), **kw)
            if work(case)["flops"] <= (most[op] / 8 if dtype == "f32" else most[op]) and work(case)["bytes"] < 8e9:
                return case
            continue
        h, w = rng.randint(1, d // 8), rng.randint(1, d // 8)
        kw.update(shots=rng.choice([1, 1, 2, 3, 8]), text=log_int(1, 520), frames=rng.choice([0, 1, 3, 8, 21]), gh=rng.randint(5, 45),
                  gw=rng.randint(5, 80), t0=rng.choice([0, 0, 77, 5000, 1000000]), pairing=rng.choice(["adjacent", "halves"]),
                  axes="%d,%d,%d" % (d // 2 - h - w, h, w))
        path = rng.choice(["forward", "inverse"] if op == "rope" else ["forward", "backward", "train"])
        case = _case(None, op, path, **kw)
        if work(case)["bytes"] <= most[op]:
            return case


# ---- sizes --------------------------------------------------------------------------------------------------------

def _tokens(case):
    return case["shots"] * (case["text"] + case["frames"] * case["gh"] * case["gw"])


def _positions(case):
    """(time, height, width) of every token of the stream, int32 [N, 3]."""
    out, t = [], case["t0"]
    for _ in range(case["shots"]):
        out.append(np.tile(np.array([[t, 0, 0]]), (case["text"], 1)))
        f, y, x = np.meshgrid(np.arange(case["frames"]), np.arange(case["gh"]), np.arange(case["gw"]), indexing="ij")
        out.append(np.stack([t + f.reshape(-1), y.reshape(-1), x.reshape(-1)], 1))
        t += max(case["frames"], 1)
    return np.concatenate(out).astype(np.int32)


def _axes(case):
    return [int(a) for a in case["axes"].split(",")]


def _frequencies(case):
    """Angle of each pair per unit of its axis' position, and the axis it belongs to."""
    pairs = _axes(case)
    freq = np.concatenate([_BASE ** (-np.arange(n) / max(n, 1)) for n in pairs])
    return freq.astype(np.float64), np.repeat(np.arange(len(pairs)), pairs)


def _cuts(total, pieces):
    return [total // pieces * i for i in range(pieces)] + [total]


def _ranges(case):
    """[B][segments] of (first, end): the states a segment of a sample attends."""
    rng = np.random.default_rng([case["B"], case["N"], case["M"], case["segments"]])
    B, S, M = case["B"], case["segments"], case["M"]
    out = []
    for b in range(B):
        if case["ranges"] == "shots":
            cut = _cuts(M, S)
            row = [(cut[s], cut[s] + max(1, int((cut[s + 1] - cut[s]) * rng.uniform(0.2, 1.0)))) for s in range(S)]
        elif case["ranges"] == "padded":
            n = 0 if B > 2 and b == 1 else max(1, int(M * rng.uniform(0.1, 1.0)))
            row = [(0, n)] * S
        else:
            row = [(0, M)] * S
        out.append(row)
    return out


# ---- inputs -------------------------------------------------------------------------------------------------------

def prepare(case, seed):
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)

    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    st = dict(case=case)
    if case["op"] == "cross":
        N, M, S = case["N"], case["M"], case["segments"]
        st["q"], st["k"], st["v"] = normal(B, H, N, d), normal(B, Hk, M, d), normal(B, Hk, M, d)
        st["ranges"], st["q_offsets"] = _ranges(case), _cuts(N, S)
        st["kv_ranges"] = torch.tensor(st["ranges"], dtype=torch.int32, device="cuda") if case["ranges"] != "full" else None
        if case["path"] != "forward":
            st["dO"] = normal(B, H, N, d)
        if case["path"] == "backward":        # what the forward pass of the step has left
            st["o"], st["lse"] = _cross_forward(st)
        if own:
            from paper_2508_21058_amd import binding as mb
            st["ws"] = mb.cross_attn_workspace(B, H, Hk, N, M, d, dtype, with_bwd=case["path"] != "forward", segments=S)
        return st
    N = _tokens(case)
    pos = _positions(case)
    freq, axis = _frequencies(case)
    st["positions"] = torch.from_numpy(pos).cuda()
    st["freq"], st["axis"] = torch.from_numpy(freq).cuda(), torch.from_numpy(axis).cuda()
    if case["op"] == "norm_rope":
        st["qkv"] = normal(B, N, H + 2 * Hk, d)
        st["wq"], st["wk"] = (1.0 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2))
        if case["path"] != "forward":
            st["dq"], st["dk"], st["dv"] = normal(B, H, N, d), normal(B, Hk, N, d), normal(B, Hk, N, d)
    else:
        st["x"] = normal(B, N, H, d) if case["path"] == "forward" else normal(B, H, N, d)
    if own:
        from paper_2508_21058_amd import binding as mb
        st["rope"] = mb.rope_plan(st["positions"], _axes(case), freq=freq, halves=case["pairing"] == "halves")
        if case["op"] == "norm_rope" and case["path"] != "forward":
            st["ws"] = mb.qk_norm_rope_workspace(B, N, H, Hk, d, dtype)
    return st


# ---- one pass -----------------------------------------------------------------------------------------------------

def run(st):
    case = st["case"]
    if own:
        return _run_own(st)
    if case["op"] == "cross":
        out = {}
        o, lse = st.get("o"), st.get("lse")
        if case["path"] != "backward":
            o, lse = _cross_forward(st)
            out.update(o=o, lse=lse)
        if case["path"] != "forward":
            out.update(zip(("dq", "dk", "dv"), _cross_backward(st, o, lse)))
        return out
    cos, sin = _angles(st)
    if case["op"] == "rope":
        if case["path"] == "forward":
            return _rotate(st["x"].permute(0, 2, 1, 3).float(), cos, sin, case).to(st["x"].dtype)
        return _rotate(st["x"].float(), cos, -sin, case).to(st["x"].dtype)
    H, Hk, dtype = case["H"], case["Hk"], st["qkv"].dtype
    q, k, v = (st["qkv"][:, :, a:b].float() for a, b in ((0, H), (H, H + Hk), (H + Hk, H + 2 * Hk)))
    out = {}
    if case["path"] != "backward":
        for name, x, w in (("q", q, st["wq"]), ("k", k, st["wk"])):
            y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * w
            out[name] = _rotate(y.permute(0, 2, 1, 3), cos, sin, case).to(dtype).contiguous()
        out["v"] = v.permute(0, 2, 1, 3).to(dtype).contiguous()
    if case["path"] != "forward":
        for name, x, w, dz in (("q", q, st["wq"], st["dq"]), ("k", k, st["wk"], st["dk"])):
            dy = _rotate(dz.float(), cos, -sin, case).permute(0, 2, 1, 3)
            r = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
            n = x * r
            out["dw" + name] = (dy * n).sum((0, 1, 2), dtype=torch.float64).float()
            dn = dy * w
            out["d" + name] = (r * (dn - n * (dn * n).mean(-1, keepdim=True))).to(dtype)
        out["dv"] = st["dv"].permute(0, 2, 1, 3).contiguous()
    return out


def _run_own(st):
    from paper_2508_21058_amd import binding as mb
    case = st["case"]
    if case["op"] == "cross":
        out = {}
        o, lse = st.get("o"), st.get("lse")
        kw = dict(kv_ranges=st["kv_ranges"], q_offsets=st["q_offsets"] if case["segments"] > 1 else None, workspace=st["ws"])
        if case["path"] != "backward":
            o, lse = mb.cross_attn_fwd(st["q"], st["k"], st["v"], **kw)
            out.update(o=o, lse=lse)
        if case["path"] != "forward":
            out.update(zip(("dq", "dk", "dv"), mb.cross_attn_bwd(st["q"], st["k"], st["v"], o, lse, st["dO"], **kw)))
        return out
    if case["op"] == "rope":
        if case["path"] == "forward":
            return mb.apply_rope(st["x"].permute(0, 2, 1, 3), st["rope"])
        return mb.apply_rope(st["x"], st["rope"], inverse=True)
    H, Hk = case["H"], case["Hk"]
    q, k, v = st["qkv"].split((H, Hk, Hk), dim=2)
    out = {}
    if case["path"] != "backward":
        out["q"], out["k"], out["v"] = mb.qk_norm_rope(q, k, v, st["wq"], st["wk"], st["rope"], eps=_EPS)
    if case["path"] != "forward":
        grad = torch.empty_like(st["qkv"])
        dq, dk, dv = grad.split((H, Hk, Hk), dim=2)
        dwq, dwk = mb.qk_norm_rope_bwd(q, k, st["dq"], st["dk"], st["dv"], st["wq"], st["wk"], st["rope"], eps=_EPS,
                                       out=(dq, dk, dv), workspace=st["ws"])[3:]
        out.update(dq=dq, dk=dk, dv=dv, dwq=dwq, dwk=dwk)
    return out


# ---- plain forms --------------------------------------------------------------------------------------------------

def _angles(st):
    """cos and sin of every token's angles, [N, d/2] in 32 bits; the angles of far positions need 64."""
    a = st["positions"].double()[:, st["axis"]] * st["freq"]
    return torch.cos(a).float(), torch.sin(a).float()


def _rotate(x, cos, sin, case):
    """x [B, H, N, d] with each pair (a, b) turned to (a cos - b sin, a sin + b cos)."""
    if case["pairing"] == "adjacent":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack((a * cos - b * sin, a * sin + b * cos), -1).reshape(x.shape)
    a, b = x.chunk(2, -1)
    return torch.cat((a * cos - b * sin, a * sin + b * cos), -1)


def _pieces(st):
    """(sample, first query, end, first state, end, key head, first query head, end) of products of bounded size."""
    case = st["case"]
    G = case["H"] // case["Hk"]
    for b, row in enumerate(st["ranges"]):
        for s, (k0, k1) in enumerate(row):
            q0, q1 = st["q_offsets"][s], st["q_offsets"][s + 1]
            many = max(1, min(case["Hk"], (1 << 28) // max(1, (q1 - q0) * max(k1 - k0, 1) * G)))
            for h in range(0, case["Hk"], many):
                yield b, q0, q1, k0, k1, h, min(h + many, case["Hk"]), G


def _cross_forward(st):
    q, k, v = st["q"], st["k"], st["v"]
    scale = q.shape[-1] ** -0.5
    o = torch.zeros_like(q)
    lse = torch.full(q.shape[:3], -math.inf, dtype=torch.float32, device=q.device)
    for b, q0, q1, k0, k1, h0, h1, G in _pieces(st):
        if k1 <= k0:
            continue
        qs = q[b, h0 * G:h1 * G, q0:q1].float().reshape(h1 - h0, G * (q1 - q0), -1)
        s = torch.matmul(qs, k[b, h0:h1, k0:k1].float().transpose(1, 2).contiguous()) * scale
        m = s.amax(-1, keepdim=True)
        p = torch.exp(s - m)
        z = p.sum(-1, keepdim=True)
        o[b, h0 * G:h1 * G, q0:q1] = torch.matmul(p / z, v[b, h0:h1, k0:k1].float()).reshape((h1 - h0) * G, q1 - q0, -1).to(q.dtype)
        lse[b, h0 * G:h1 * G, q0:q1] = (m + torch.log(z)).reshape((h1 - h0) * G, q1 - q0)
    return o, lse


def _cross_backward(st, o, lse):
    q, k, v, d_o = st["q"], st["k"], st["v"], st["dO"]
    scale = q.shape[-1] ** -0.5
    dq = torch.zeros_like(q)
    dk, dv = (torch.zeros(k.shape, dtype=torch.float32, device=q.device) for _ in range(2))
    for b, q0, q1, k0, k1, h0, h1, G in _pieces(st):
        if k1 <= k0:
            continue
        hs, n = slice(h0 * G, h1 * G), q1 - q0
        qs, os, dos = (x[b, hs, q0:q1].float().reshape(h1 - h0, G * n, -1) for x in (q, o, d_o))
        ks, vs = k[b, h0:h1, k0:k1].float(), v[b, h0:h1, k0:k1].float()
        p = torch.exp(torch.matmul(qs, ks.transpose(1, 2).contiguous()) * scale - lse[b, hs, q0:q1].reshape(h1 - h0, G * n, 1))
        dv[b, h0:h1, k0:k1] += torch.matmul(p.transpose(1, 2).contiguous(), dos)
        dp = torch.matmul(dos, vs.transpose(1, 2).contiguous())
        ds = p * (dp - (dos * os).sum(-1, keepdim=True)) * scale
        dq[b, hs, q0:q1] = torch.matmul(ds, ks).reshape((h1 - h0) * G, n, -1).to(q.dtype)
        dk[b, h0:h1, k0:k1] += torch.matmul(ds.transpose(1, 2).contiguous(), qs)
    return dq, dk.to(k.dtype), dv.to(v.dtype)


# ---- work ---------------------------------------------------------------------------------------------------------

def work(case):
    B, H, Hk, d = case["B"], case["H"], case["Hk"], case["d"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "cross":
        N, M = case["N"], case["M"]
        cut = _cuts(N, case["segments"])
        pairs = sum((cut[s + 1] - cut[s]) * (k1 - k0) for row in _ranges(case) for s, (k0, k1) in enumerate(row))
        rows, states = float(B) * H * N * d * e, float(B) * Hk * M * d * e
        lse = B * H * N * 4.0
        bytes_ = {"forward": 2 * rows + 2 * states + lse, "backward": 4 * rows + 4 * states + lse, "train": 4 * rows + 4 * states + lse}
        flops = {"forward": 4.0, "backward": 10.0, "train": 14.0}
        return {"bytes": bytes_[case["path"]], "flops": flops[case["path"]] * d * H * pairs}
    N = _tokens(case)
    cells, extra = float(B) * N * d, N * 12.0
    if case["op"] == "rope":
        return {"bytes": 2 * cells * H * e + extra, "flops": 3 * cells * H}
    # heads read and written: q, k, v in and out; q, k and three gradients in, three gradients out; both with one reading of q and k
    heads = {"forward": 2 * H + 4 * Hk, "backward": 3 * H + 5 * Hk, "train": 4 * H + 8 * Hk}[case["path"]]
    flops = {"forward": 7, "backward": 15, "train": 22}[case["path"]]
    return {"bytes": cells * heads * e + extra, "flops": flops * cells * (H + Hk)}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _turn(x, pos, case, inverse):
    """x [..., N, d] in 64 bits as complex numbers times e^(i angle)."""
    freq, axis = _frequencies(case)
    angle = torch.from_numpy(pos.astype(np.float64)[:, axis] * freq).to(x.device)
    unit = torch.polar(torch.ones_like(angle), -angle if inverse else angle)
    half = case["d"] // 2
    z = x.reshape(*x.shape[:-1], half, 2) if case["pairing"] == "adjacent" else x.reshape(*x.shape[:-1], 2, half).transpose(-1, -2)
    z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * unit)
    return (z if case["pairing"] == "adjacent" else z.transpose(-1, -2)).reshape(x.shape)


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "cross":
        return _exact_cross(case, st)
    pos = _positions(case)
    if case["op"] == "rope":
        x = st["x"].transpose(1, 2) if case["path"] == "forward" else st["x"]
        return torch.stack([_turn(x[:, h].double(), pos, case, case["path"] == "inverse") for h in range(case["H"])], 1)
    H, Hk = case["H"], case["Hk"]
    w = {n: st["w" + n].double().requires_grad_() for n in "qk"}
    out = {n: [] for n in "qkv"}
    grad = {n: [] for n in "qkv"}
    weight = {n: 0.0 for n in "qk"}
    for n, first, count in (("q", 0, H), ("k", H, Hk), ("v", H + Hk, Hk)):
        for h in range(count):
            x = st["qkv"][:, :, first + h].double().requires_grad_()
            y = x
            if n != "v":
                y = _turn(x / torch.sqrt(x.square().mean(-1, keepdim=True) + _EPS) * w[n], pos, case, False)
            out[n].append(y.detach())
            if case["path"] != "forward":
                dz = st["d" + n][:, h].double()
                got = torch.autograd.grad(y, (x, w[n]) if n != "v" else (x,), dz)
                grad[n].append(got[0])
                if n != "v":
                    weight[n] = weight[n] + got[1]
    res = {}
    if case["path"] != "backward":
        res.update({n: torch.stack(out[n], 1) for n in "qkv"})
    if case["path"] != "forward":
        res.update({"d" + n: torch.stack(grad[n], 2) for n in "qkv"})
        res.update({"dw" + n: weight[n] for n in "qk"})
    return res


def _exact_cross(case, st):
    B, H, Hk, N, M, d = (case[n] for n in ("B", "H", "Hk", "N", "M", "d"))
    f64 = dict(dtype=torch.float64, device="cuda")
    o, lse = torch.zeros(B, H, N, d, **f64), torch.full((B, H, N), -math.inf, **f64)
    grads = case["path"] != "forward"
    dq, dk, dv = (torch.zeros(B, h, n, d, **f64) for h, n in ((H, N), (Hk, M), (Hk, M))) if grads else (None,) * 3
    for b in range(B):
        for h in range(H):
            for s in range(case["segments"]):
                (k0, k1), q0, q1 = st["ranges"][b][s], st["q_offsets"][s], st["q_offsets"][s + 1]
                if k1 <= k0:
                    continue
                q, k, v = (x.double().requires_grad_(grads) for x in (st["q"][b, h, q0:q1], st["k"][b, h * Hk // H, k0:k1],
                                                                     st["v"][b, h * Hk // H, k0:k1]))
                logits = q @ k.T / math.sqrt(d)
                y = torch.softmax(logits, -1) @ v
                o[b, h, q0:q1], lse[b, h, q0:q1] = y.detach(), torch.logsumexp(logits, -1).detach()
                if grads:
                    got = torch.autograd.grad(y, (q, k, v), st["dO"][b, h, q0:q1].double())
                    dq[b, h, q0:q1] = got[0]
                    dk[b, h * Hk // H, k0:k1] += got[1]
                    dv[b, h * Hk // H, k0:k1] += got[2]
    res = {}
    if case["path"] != "backward":
        res.update(o=o, lse=lse)
    if grads:
        res.update(dq=dq, dk=dk, dv=dv)
    return res
