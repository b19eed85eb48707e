// Cross attention backward.
//   delta_i = dO_i . o_i,  P_it = exp(scale q_i.k_t - lse_i),  dS_it = P_it (dO_i.v_t - delta_i)
//   dQ_i = scale sum_t dS_it k_t,  dV_t = sum_i P_it dO_i,  dK_t = scale sum_i dS_it q_i
//
// Two passes without atomics: dQ over the queries, as the forward goes (it forms delta on its way in and leaves the
// statistics), then dK and dV over the states: a workgroup owns 32 to 128 states of a key head, 32 a wave, and streams the queries of every
// segment whose range meets them, 32 at a time, of all the query heads that share the key head (bf16 heads of 128 features in larger calls:
// 256 states, moc_cross_dkdv.hip). The states are few and the queries many, so the queries of a tile of states are split over workgroups, whose
// sums a last launch adds in a fixed order.
//
// What bounds it: at long ranges the products (33k queries, 4,357 states, 24 heads: dQ 2.35 ms, 1,140 TFLOP/s with the scores it forms again; a
// library product of 8,192 x 8,192 matrices reaches 1,170 on this chip, which then holds less than its clock); at short ones the rows of
// q, o, dO and dQ and what an item costs besides its products (114k queries, 256 states: 718 us, 2.8 GB, 750 TFLOP/s). dK and dV in small
// tiles: 24 heads of 64 features, 114k queries, 1,024 states 1,495 us, 963 TFLOP/s; twelve fp32 heads, 33k queries, 512 states 1,575 us, 133
// TFLOP/s of the card's 157; four states, where all there is to do is to read q and dO, 160 us for 0.74 GB.
#include <cmath>

#include "moc_cross.h"

namespace moc {

// What the key-stationary pass reads of a query.
__device__ __forceinline__ void store_record(const CrossArgs &a, const CrossItem &it, size_t row, float lse2, float delta) {
    const int word = (int)((uint32_t)(row - (size_t)it.bhk * a.copies * a.N) << 5);
    *reinterpret_cast<f32x4 *>(a.stats + 4 * row) = f32x4{lse2, delta, __int_as_float(word), 0.f};
}

template <int D, typename T>
__global__ __launch_bounds__(256, D == 64 && sizeof(T) == 2 ? 3 : 2) void cross_dq_kernel(CrossArgs a) {
    typedef Ops<D, T> O;
    constexpr int BN = sizeof(T) == 2 ? 64 : 32, DB = D / 32;
    constexpr int TB = BN * O::RB;
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    // what the key-stationary pass needs besides the records: that of padding rows and, of wide tiles, the list of them
    if (blockIdx.x == 0 && tid < 4) a.stats[4 * (size_t)a.rows + tid] = tid ? 0.f : INFINITY;
    if constexpr (D == 128 && sizeof(T) == 2)
        if ((int)blockIdx.x >= a.cut_at) { cross_cut(a, blockIdx.x - a.cut_at, *reinterpret_cast<CutLds *>(smem)); return; }
    int logical;
    if (!cross_logical(a, logical)) return;
    const int z = logical % a.split;
    CrossItem it = cross_item(a, logical / a.split);
    if (it.count <= 0) return;
    cross_slice(it.first, it.end, z, a.split, BN);
    const int r = wave * 32 + l32, rc = min(r, it.count - 1);
    const bool row_valid = r < it.count;
    const size_t row = (size_t)it.row + rc;
    const bool some = it.first < it.end;
    const T *kb = static_cast<const T *>(a.k) + (size_t)it.bhk * a.M * D, *vb = static_cast<const T *>(a.v) + (size_t)it.bhk * a.M * D;
    auto issue = [&](int pos, int buf) {
        const int valid = min(BN, it.end - pos);
        copy_tile<D, T, BN>(kb + (size_t)pos * D, valid, smem + buf * 2 * TB, wave, lane);
        copy_tile<D, T, BN>(vb + (size_t)pos * D, valid, smem + buf * 2 * TB + TB, wave, lane);
    };
    if (some) issue(it.first, 0);
    // All of the item's loads go out before anything waits for one: left to the compiler, the products of delta came between them
    // (114k queries of 24 heads, 256 states: 836 us, this way 718). In float with 128 features q, o, dO and dQ are 64 registers each, and 30 of
    // the kernel's go through scratch memory on its way in.
    typename O::Frag qf[O::KS], dof[O::KS];
    float delta = 0.f, lse2;
    {
        const T *qrow = static_cast<const T *>(a.q) + row * D, *dorow = static_cast<const T *>(a.d_o) + row * D;
        const T *orow = static_cast<const T *>(a.o_in) + row * D;
        typename O::Frag of[O::KS];
        lse2 = a.lse_in[row] * kLog2e;
#pragma unroll
        for (int s = 0; s < O::KS; ++s) {
            of[s] = O::row_frag(orow, s, half);
            dof[s] = O::row_frag(dorow, s, half);
        }
#pragma unroll
        for (int s = 0; s < O::KS; ++s) qf[s] = O::row_frag(qrow, s, half);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < O::KS; ++s) delta += O::dot(dof[s], of[s]);
        delta = xhalf_sum(delta);
    }
    const float c = a.scale_log2;
    if (z == 0 && row_valid && half == 0) store_record(a, it, row, lse2, delta);
    f32x16 dq[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) dq[b] = zero16();
    if (some) {
        O ops;
        ops.init(lane);
        auto tile = [&](auto which, int pos) {                // (as in the forward)
            constexpr int BUF = decltype(which)::value;
            wait_vmcnt<0>();
            __syncthreads();
            if (pos + BN < it.end) issue(pos + BN, BUF ^ 1);
            if (wave * 32 >= it.count) return;
            const char *kt = smem + BUF * 2 * TB, *vt = kt + TB;
            const int valid = it.end - pos;
#pragma unroll
            for (int k32 = 0; k32 < BN; k32 += 32) {
                if (k32 >= valid) break;
                ops.pin();
                f32x16 s = zero16(), dp = zero16();
#pragma unroll
                for (int i = 0; i < O::KS; ++i) s = O::mma(ops.frag(kt, k32, i), qf[i], s);
#pragma unroll
                for (int i = 0; i < O::KS; ++i) dp = O::mma(ops.frag(vt, k32, i), dof[i], dp);
                if (valid >= k32 + 32) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse2)) * (dp[i] - delta);
                } else {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(s[i], c, -lse2));
                        s[i] = k32 + (i >> 2) * 8 + half * 4 + (i & 3) < valid ? p * (dp[i] - delta) : 0.f;
                    }
                }
#pragma unroll
                for (int ks = 0; ks < O::RS; ++ks) {
                    const typename O::Frag f = O::pack(s, ks);
#pragma unroll
                    for (int b = 0; b < DB; ++b) dq[b] = O::mma(ops.tfrag(kt, k32, b, ks), f, dq[b]);
                }
            }
        };
        for (int pos = it.first; pos < it.end; pos += 2 * BN) {
            tile(IC<0>{}, pos);
            if (pos + BN < it.end) tile(IC<1>{}, pos + BN);
        }
    }
    if (a.split > 1) {
        if (row_valid) store_rows_f32<D>(dq, a.scale, a.part + ((size_t)z * a.rows + row) * D, half);
    } else if constexpr (sizeof(T) == 4) {
        if (row_valid) store_rows_f32<D>(dq, a.scale, static_cast<float *>(a.dq) + row * D, half);
    } else {
        __syncthreads();
        store_rows_bf16<D>(smem, wave, lane, dq, a.scale, row_valid ? r : -1, static_cast<bf16_t *>(a.dq) + (size_t)it.row * D);
    }
}

// The queries that a tile of states streams: the segments whose ranges meet it, neighbours that attend the same of its states as one run, cut
// into tiles of 32.
struct CrossStream {
    int n, tile_at[MOC_MAX_CROSS_SEGMENTS + 1], query[MOC_MAX_CROSS_SEGMENTS], rows[MOC_MAX_CROSS_SEGMENTS], first[MOC_MAX_CROSS_SEGMENTS],
        end[MOC_MAX_CROSS_SEGMENTS];
};
constexpr int kStreamRows = 32;
// (the first wave; a barrier before anyone else reads it)
__device__ __forceinline__ void make_stream(const CrossArgs &a, int b, int key0, int key1, CrossStream &s, int lane) {
    int n = 0, at = 0;
    for (int s0 = 0; s0 < a.n_seg; s0 += 64) {
        const int i = s0 + lane;
        int first = 0, end = 0;
        if (i < a.n_seg) {
            const CrossRange r = cross_range(a, b, i);
            first = max(r.first, key0);
            end = min(r.end, key1);
        }
        const bool in = first < end;
        const int f = __shfl_up(first, 1, 64), e = __shfl_up(end, 1, 64);
        const unsigned long long joined = __ballot(in && lane > 0 && f == first && e == end);       // goes on with the run before it
        int rows = 0;
        if (in && !(joined >> lane & 1)) {
            const unsigned long long rest = lane < 63 ? ~(joined >> (lane + 1)) : 1ull;
            const int last = i + (rest ? __ffsll(rest) - 1 : 63 - lane);
            rows = a.q_off[last + 1] - a.q_off[i];
        }
        const int tiles = (rows + kStreamRows - 1) / kStreamRows;
        int sum = tiles;
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) {
            const int o = __shfl_up(sum, w, 64);
            if (lane >= w) sum += o;
        }
        const unsigned long long have = __ballot(tiles > 0);
        if (tiles > 0) {
            const int j = n + __popcll(have & ((1ull << lane) - 1));
            s.tile_at[j] = at + sum - tiles;
            s.query[j] = a.q_off[i];
            s.rows[j] = rows;
            s.first[j] = first;
            s.end[j] = end;
        }
        n += __popcll(have);
        at += __shfl(sum, 63, 64);
    }
    if (lane == 0) { s.n = n; s.tile_at[n] = at; }
}

// KW: waves of a workgroup, 32 states each
template <int D, typename T, int KW>
__global__ __launch_bounds__(64 * KW, D == 128 || KW * sizeof(T) == 4 ? 1 : KW * sizeof(T) == 8 && KW == 4 ? 3 : 2) void cross_dkdv_kernel(CrossArgs a) {
    typedef Ops<D, T> O;
    constexpr int DB = D / 32, TB = kStreamRows * O::RB, KEYS = 32 * KW;
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB];          // Q, dO, twice
    __shared__ __attribute__((aligned(16))) float stat[2][2 * kStreamRows];
    __shared__ CrossStream cs;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    const int ktiles = (a.M + KEYS - 1) / KEYS;
    int logical;
    if (!xcd_remap((long long)ktiles * a.BHk * a.split, logical)) return;
    const int i = logical / (ktiles * a.split), bhk = dealt_head(a, i), rest = logical - i * ktiles * a.split;      // tiles of states that stream the
    const int z = rest / ktiles, key0 = (rest - z * ktiles) * KEYS;                             // same queries are neighbours
    if (wave == 0) make_stream(a, bhk / a.Hk, key0, min(key0 + KEYS, a.M), cs, lane);
    __syncthreads();
    const int per_copy = __builtin_amdgcn_readfirstlane(cs.tile_at[cs.n]);
    const long long total = (long long)per_copy * a.copies;
    const int t0 = (int)(total * z / a.split), t1 = (int)(total * (z + 1) / a.split);
    const int key = key0 + wave * 32 + l32, keyc = min(key, a.M - 1);
    const bool active = key0 + wave * 32 < a.M;
    typename O::Frag kf[O::KS], vf[O::KS];
    {
        const size_t krow = ((size_t)bhk * a.M + keyc) * D;
#pragma unroll
        for (int s = 0; s < O::KS; ++s) {
            kf[s] = O::row_frag(static_cast<const T *>(a.k) + krow, s, half);
            vf[s] = O::row_frag(static_cast<const T *>(a.v) + krow, s, half);
        }
    }
    f32x16 dk[DB], dv[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) { dk[b] = zero16(); dv[b] = zero16(); }
    O ops;
    ops.init(lane);
    const float c = a.scale_log2;
    unsigned long long poisoned = 0;                // lanes whose results are NaN
    // the next tile to copy: query head `copy` of the group, entry si of the stream, tile u of the copy
    int copy = 0, u = 0, si = 0;
    if (t0 < t1) {
        copy = t0 / per_copy;
        u = t0 - copy * per_copy;
        while (cs.tile_at[si + 1] <= u) ++si;
    }
    auto issue = [&](int buf) {
        const int done = (u - __builtin_amdgcn_readfirstlane(cs.tile_at[si])) * kStreamRows;
        const int valid = min(kStreamRows, __builtin_amdgcn_readfirstlane(cs.rows[si]) - done);
        const size_t row = ((size_t)bhk * a.copies + copy) * a.N + __builtin_amdgcn_readfirstlane(cs.query[si]) + done;
        copy_tile<D, T, kStreamRows, KW>(static_cast<const T *>(a.q) + row * D, valid, smem + buf * 2 * TB, wave, lane);
        copy_tile<D, T, kStreamRows, KW>(static_cast<const T *>(a.d_o) + row * D, valid, smem + buf * 2 * TB + TB, wave, lane);
        if (wave == 0)       // rows past the segment get (+inf, 0): no probability
            async_copy4_at(a.stats + 4 * (lane / 2 < valid ? row + lane / 2 : (size_t)a.rows) + (lane & 1), lds_address(stat[buf]));
    };
    if (t0 < t1) issue(0);
    auto tile = [&](auto which, int t) {
        constexpr int buf = decltype(which)::value;
        wait_vmcnt<0>();
        if (KW == 1) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // (the reads of the other buffer: a wave alone has no barrier)
        __syncthreads();
        const int first = __builtin_amdgcn_readfirstlane(cs.first[si]), end = __builtin_amdgcn_readfirstlane(cs.end[si]);
        if (++u == cs.tile_at[si + 1]) {
            if (++si == cs.n) { si = 0; u = 0; ++copy; }
        }
        if (t + 1 < t1) issue(buf ^ 1);
        const int kw = key0 + wave * 32;
        if (!active || first >= kw + 32 || end <= kw) return;
        ops.pin();
        const bool ok = key >= first && key < end;
        const char *qt = smem + buf * 2 * TB, *dot = qt + TB;
        f32x16 s = zero16(), dp = zero16();
#pragma unroll
        for (int i = 0; i < O::KS; ++i) s = O::mma(ops.frag(qt, 0, i), kf[i], s);
#pragma unroll
        for (int i = 0; i < O::KS; ++i) dp = O::mma(ops.frag(dot, 0, i), vf[i], dp);
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const f32x4 st0 = *reinterpret_cast<const f32x4 *>(&stat[buf][2 * (g * 8 + half * 4)]);
            const f32x4 st1 = *reinterpret_cast<const f32x4 *>(&stat[buf][2 * (g * 8 + half * 4) + 4]);
            const float l2[4] = {st0[0], st0[2], st1[0], st1[2]}, dl[4] = {st0[1], st0[3], st1[1], st1[3]};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i = 4 * g + e;
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -l2[e]));
                dp[i] = s[i] * (dp[i] - dl[e]);
            }
        }
        if (first > kw || end < kw + 32) {      // (a lane's key is in the range or not, for all of the queries. Heads of 64, as above: 720 us always masked, 655 so)
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = ok ? s[i] : 0.f;
                dp[i] = ok ? dp[i] : 0.f;
                all = fmaf(dp[i], 0.f, all);
            }
            // Zero times a NaN or an infinity of a query is not zero: its products would reach the lanes of states that it does not attend. Those that
            // attend it come out as NaN, whatever the tile's other queries add, and the others have nothing of this tile.
            if (__any(!(all == 0.f))) {
                poisoned |= __ballot(ok);
                return;
            }
        }
#pragma unroll
        for (int ks = 0; ks < O::RS; ++ks) {
            const typename O::Frag pf = O::pack(s, ks), df = O::pack(dp, ks);
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                dv[b] = O::mma(ops.tfrag(dot, 0, b, ks), pf, dv[b]);
                dk[b] = O::mma(ops.tfrag(qt, 0, b, ks), df, dk[b]);
            }
        }
    };
    for (int t = t0; t < t1; t += 2) {
        tile(IC<0>{}, t);
        if (t + 1 < t1) tile(IC<1>{}, t + 1);
    }
    if (key >= a.M) return;
    if (poisoned) {
        const float poison = poisoned >> lane & 1 ? NAN : 0.f;
#pragma unroll
        for (int b = 0; b < DB; ++b) {
            dk[b] += poison;
            dv[b] += poison;
        }
    }
    const size_t krow = (size_t)bhk * a.M + key;
    if (a.split > 1) {
        float *p = a.kpart + (((size_t)z * a.BHk * a.M) + krow) * 2 * D;
        store_rows_f32<D>(dk, a.scale, p, half);
        store_rows_f32<D>(dv, 1.f, p + D, half);
    } else {
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const size_t at = krow * D + b * 32 + g * 8 + half * 4;
                Io<T>::store4(static_cast<T *>(a.dk) + at, dk[b][4 * g] * a.scale, dk[b][4 * g + 1] * a.scale, dk[b][4 * g + 2] * a.scale,
                              dk[b][4 * g + 3] * a.scale);
                Io<T>::store4(static_cast<T *>(a.dv) + at, dv[b][4 * g], dv[b][4 * g + 1], dv[b][4 * g + 2], dv[b][4 * g + 3]);
            }
    }
}

// out = sum of the splits' rows in their order: dQ (one output of n words of four features) or dK and dV (rows of two)
template <int D, typename T>
__global__ __launch_bounds__(256) void cross_sum_kernel(const float *__restrict__ part, int split, long long rows, T *out0, T *out1) {
    constexpr int W = D / 4;
    const long long words = rows * W * (out1 ? 2 : 1), i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= words) return;
    f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int z = 0; z < split; ++z) s += *reinterpret_cast<const f32x4 *>(part + (z * words + i) * 4);
    const long long row = out1 ? i / (2 * W) : i / W;
    const int x = (int)(out1 ? i % (2 * W) : i % W);
    T *out = x < W ? out0 : out1;
    Io<T>::store4(out + row * D + (x % W) * 4, s[0], s[1], s[2], s[3]);
}

template <int D, typename T> static void bwd_dispatch(CrossArgs a, const CrossPlan &p, hipStream_t st) {
    cross_tiles(a);
    a.split = p.split_q;
    {
        MOC_PROF("cross_dq", st);
        a.cut_at = xcd_grid((long long)a.tiles * a.copies * a.BHk * a.split);
        cross_dq_kernel<D, T><<<a.cut_at + (p.wide ? a.BHk / a.Hk : 0), 256, 0, st>>>(a);
    }
    if (a.split > 1) {
        MOC_PROF("cross_sum", st);
        cross_sum_kernel<D, T><<<(unsigned)((a.rows * (D / 4) + 255) / 256), 256, 0, st>>>(a.part, a.split, a.rows, static_cast<T *>(a.dq),
                                                                                        static_cast<T *>(nullptr));
    }
    a.split = p.split_kv;
    const long long states = (long long)a.BHk * a.M;
    if (p.wide) {
        launch_cross_dkdv_wide(a, st);
    } else {
        MOC_PROF("cross_dkdv", st);
        auto launch = [&](auto waves) {
            constexpr int KW = decltype(waves)::value, KEYS = 32 * KW;
            cross_dkdv_kernel<D, T, KW><<<xcd_grid((long long)((a.M + KEYS - 1) / KEYS) * a.BHk * a.split), 64 * KW, 0, st>>>(a);
        };
        if (p.key_waves == 1) launch(IC<1>{});
        else if (p.key_waves == 2) launch(IC<2>{});
        else launch(IC<4>{});
    }
    if (a.split > 1) {
        MOC_PROF("cross_sum", st);
        cross_sum_kernel<D, T><<<(unsigned)((states * 2 * (D / 4) + 255) / 256), 256, 0, st>>>(a.kpart, a.split, states, static_cast<T *>(a.dk),
                                                                                             static_cast<T *>(a.dv));
    }
}

hipError_t launch_cross_bwd(CrossArgs a, const CrossPlan &p, int d, int dtype, hipStream_t st) {
    if (d == 128 && dtype == MOC_BF16) bwd_dispatch<128, bf16_t>(a, p, st);
    else if (d == 128) bwd_dispatch<128, float>(a, p, st);
    else if (dtype == MOC_BF16) bwd_dispatch<64, bf16_t>(a, p, st);
    else bwd_dispatch<64, float>(a, p, st);
    return hipGetLastError();
}

// ---- how a call is cut ----------------------------------------------------------------------------
CrossPlan cross_plan(int B, int H, int Hk, int N, int M, int d, int S, int dtype, bool with_bwd) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    CrossPlan p;
    const bool bf16 = dtype == MOC_BF16;
    const long long rows = (long long)B * H * N, states = (long long)B * Hk * M, per_head = (long long)N * (H / Hk);
    // However well a call fills the chip, a sum is no longer than kChainTerms: a growing float sum rounds the same number the same way for a long time, so
    // that its error is not a random walk's (4 million states of nearly equal probability in one chain: the softmax's sum 1.1 % off).
    const long long chain = bf16 ? kChainTerms : kChainTermsF32, least_q = (M + chain - 1) / chain, least_kv = (per_head + chain - 1) / chain;
    // Forward and dQ: parts of the ranges of states, of 128 states at least. Workgroups spread over the compute units in whole numbers; one takes 6 us
    // and `one` for 32 states, two on a unit take `two` (float: twice as long, one fills the matrix pipes), and parts cost their sums. Forward, join,
    // dQ and sum together, for at least 256 workgroups / this way: 24 heads of bf16, 309 queries, 300 states 46 / 33 us, 1,000 states 60 / 58, 16,000
    // states 270 / 229; 1,000 queries, 1,000 states 86 / 72; twelve fp32 heads, 311 queries, 2,800 states 262 / 207 (36 tiles in eight
    // parts are 32 units with two workgroups). Ranges of segments are all the states or each its own, as for dK and dV below.
    {
        const long long heads = (long long)B * (S == 1 ? Hk : H), len = S == 1 ? (long long)N * (H / Hk) : N;
        const long long tiles = heads * ((len + kCrossRows - 1) / kCrossRows), own_tiles = tiles + heads * (S - 1);
        const double one = (bf16 ? 0.7 : 3.5) * d / 128, two = (bf16 ? 1.1 : 7.) * d / 128, sums = (double)B * H * N * d * 8 / 6e6, stages = M / 32.;
        auto time = [&](long long s, long long n, double work) {
            const long long w = (n * s + kComputeUnits - 1) / kComputeUnits;
            return (w / 2 * two + w % 2 * one) * std::max(1., work / s) + (w + 1) / 2 * 6 + (s > 1 ? s * sums + 6 : 0);
        };
        double best = 0;
        const long long most = std::max(std::min({256LL, (M + 127LL) / 128, 4 * kComputeUnits / tiles + 1}), least_q > 1 && tiles <= 4 * kComputeUnits ? least_q + 3 : least_q);
        for (long long s = least_q; s <= most; ++s) {
            const double us = time(s, tiles, stages) + (S > 1 ? time(s, own_tiles, stages / S) : 0);
            if (s == least_q || us < best) { best = us; p.split_q = (int)s; }
        }
    }
    p.max_items = M / kWideTile + 2 * S + 1;
    p.key_waves = M <= 32 ? 1 : M <= 64 ? 2 : 4;
    // dK and dV: parts of the queries that workgroups of one tile of states share, and (bf16, 128 features) which tiles. Rounds of workgroups on
    // the chip are whole, a workgroup takes `begin` to begin and end and `stage` for 32 queries, and parts cost their sums, written and read again.
    // Microseconds, fitted to calls of 16 to 114k queries. 24 heads, small / wide tiles: 64 queries, 1,024 states 16 / 29 us; 128 queries, 4,096
    // states 54 / 58; 1,000 queries, 512 states 45 / 50; 8,000 queries, 77 states 47 / 67; 2,000 queries, 512 states 88 / 60. Small tiles, 12 fp32 heads of
    // 33k queries, 512 states (48 tiles) in 11 / 16 parts (2.06 / 3 rounds of the chip) 2,300 / 1,620. Wide tiles, 24 heads of 33k queries, 4,357 states
    // (432 tiles) in 1 / 2 / 3 / 4 / 8 parts 3,112 / 3,488 / 3,508 / 3,597 / 3,373. What the ranges of segments are is not known here: either all
    // of them are all the states or each has its own, and the sum of both times is made small. (The sums of the parts may take half a gigabyte, of parts that are
    // there for the length of the sums more.)
    // (a copy's last 32 queries, or a segment's, are not whole ones: 36 fp32 heads on twelve, nine queries in two segments 57 us with one part, 22 with six and their sum)
    const long long copies = S == 1 ? 1 : H / Hk, len = per_head / copies;
    const double stages = (double)(copies * ((len + 31) / 32)), apart = (double)(copies * S * (((len + S - 1) / S + 31) / 32));
    const double sums = (double)states * d * 16 / 6e6;
    const long long heads = (long long)B * Hk;
    auto cut = [&](int keys, int per_unit, double stage, double begin, bool pieces, int &parts) {
        const long long tiles = heads * ((M + keys - 1) / keys), units = (long long)kComputeUnits * per_unit;
        // with ranges of their own the wide tiles are cut at them; the others meet the queries of every range that reaches into them
        const long long own_tiles = pieces ? std::max(tiles, heads * S) : tiles;
        const double own_stages = pieces ? apart / S : apart * std::min(1., (keys + M / S) / (double)M);
        auto time = [&](long long s, long long n, double work) {
            // (a round with units to spare runs at a higher clock: full rounds of matrix instructions take 1.2 times as long per item)
            const double rounds = std::max((double)((n * s + units - 1) / units), pieces ? 1.2 * n * s / units : 0);
            return rounds * (stage * std::max(1., work / s) + begin) + (s > 1 ? s * sums + 5 : 0);
        };
        // (from the least number of parts on, since that one may be a bad number of rounds: 24 heads in fp32, 46k queries each of two, 1,827 states in 2 / 3 / 7
        // parts 34.3 / 37.7 / 32.7 ms)
        const long long most = std::max(std::min({1024LL, (long long)std::ceil(std::max(stages, own_stages) / (bf16 ? 2 : 1)), 3 * units / tiles + 1}), least_kv > 1 ? 3 * least_kv : 1);
        double best = 0;
        for (long long s = least_kv; s <= most && (s == least_kv || (s * states * d * 8 <= 512 << 20 && heads * p.max_items * s < 1 << 20));
             s += 1 + s / 64) {
            const double us = time(s, tiles, stages) + (S > 1 ? time(s, own_tiles, own_stages) : 0);
            if (s == least_kv || us < best) { best = us; parts = (int)s; }
        }
        return best;
    };
    // (waves on a compute unit: four, with heads of 64 features eight, in bf16 in fours twelve; or what its 160 KiB of LDS hold. 24 heads of 64 features,
    // 114k queries, 300 states: planned for eight 655 us, for twelve 580.)
    const int lds = 4 * kStreamRows * d * (bf16 ? 2 : 4) + (int)sizeof(CrossStream) + 512;
    const int per_unit = std::min(163840 / lds, (d == 128 ? 4 : bf16 && p.key_waves == 4 ? 12 : 8) / p.key_waves);
    const double stage = (bf16 ? 1.5 : 8.) * d / 128 * std::max(1., per_unit * p.key_waves / 4.);
    const double us = cut(32 * p.key_waves, per_unit, stage, 10, false, p.split_kv);
    p.wide = false;
    if (d == 128 && bf16) {
        int parts;
        p.wide = cut(kWideTile, 1, 1.5, 25, true, parts) < us;
        if (p.wide) p.split_kv = parts;
    }
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t x = at; at += up(bytes); return x; };
    p.part = take(p.split_q > 1 ? (size_t)p.split_q * rows * d * 4 : 0);
    p.part_lse = take(p.split_q > 1 ? (size_t)p.split_q * rows * 4 : 0);
    p.stats = take(with_bwd ? (size_t)(rows + 1) * 16 : 0);
    p.kpart = take(with_bwd && p.split_kv > 1 ? (size_t)p.split_kv * states * 2 * d * 4 : 0);
    p.items = take(with_bwd && p.wide ? (size_t)B * p.max_items * sizeof(CrossKeys) : 0);
    p.item_counts = take(with_bwd && p.wide ? (size_t)B * sizeof(CrossCount) : 0);
    p.total = at;
    // A launch has fewer than 2^32 threads. (The query passes take workgroups of 256 threads, one a tile of queries and part, dQ's one more a sample;
    // the passes over the states one a tile and part, the wide one 16 more; joins and sums 256 / (d / 4) rows.)
    const long long most = (1 << 24) - 1024, words = d / 4, keys = 32 * p.key_waves;
    const long long q_wgs = ((long long)B * H * ((N + kCrossRows - 1) / kCrossRows + S - 1)) * p.split_q + B;
    const long long kv_wgs = heads * (p.wide ? p.max_items : (M + keys - 1) / keys) * p.split_kv;
    p.fits = q_wgs < most && (p.split_q == 1 || rows * words / 256 < most) &&
             (!with_bwd || (kv_wgs < most && (p.split_kv == 1 || states * 2 * words / 256 < most)));
    return p;
}

}  // namespace moc
