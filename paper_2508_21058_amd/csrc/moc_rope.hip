// Norms of queries and keys with the rotation by several axes, forward and backward, and the rotation alone.
//
//   forward   r = 1/sqrt(mean x^2 + eps), y = w x r, out = R y, R turning pair (a, b) of features by
//             (a cos - b sin, a sin + b cos)
//   backward  dy = R^T g, dw = sum dy x r, with dn = dy w:  dx = r (dn - x r^2 mean(dn x))
//
// Bound by HBM: every row is read once and written once. A thread owns eight features (four pairs) of one token and walks
// the heads: the angles of a token, which cost a double product, a reduction to a turn and a sine and cosine each, are formed
// once for all of its heads of q and of k. d/8 neighbouring lanes hold a row, so a row's sums are three or four lane exchanges.
// A workgroup reads 16 (d = 128) or 32 tokens whole, contiguous in a fused projection, and writes 4 KB pieces of every head.
#include "moc_block.h"
#include "moc_device.h"

namespace moc {

constexpr int kRowThreads = 256;
// Workgroups wanted. The forward takes many short ones, so that the last round of the chip is short, but at least eight heads each where there are
// enough tokens, since each forms the angles anew: 33k tokens of 24 heads 91 us with a workgroup per 16 tokens (2,080 of them, 2,048 at a time),
// 85 with three, 83 with eight; 6k tokens (q, k and v) 41.5 with three, 43.5 with 18, 55.5 with 36. The backward's, of
// which two fit a compute unit (174 to 181 registers), take several blocks of tokens one after the other, all of them in one round, so that the weights'
// partial sums are few: 512, 1,024, 1,536 of them 53.5, 60.5, 66 us (two samples of 16k tokens, twelve and four heads of 64), 351, 357, 353
// (33k tokens of 24 heads of 128). Whole blocks of tokens each: calls of a few blocks more than a round's take a round more for them (24 heads of
// 128: 4,096 / 4,099 tokens 42 / 56 us, 8,192 / 8,200 88 / 110, 12,288 / 12,300 129 / 138; 6,256 tokens 73, 4.2 TB/s).
constexpr int kRowWgs = 6144, kRowWgsFew = 512, kRowHeadsMin = 8, kRowWgsBwd = 512;

RowGrid row_grid(int B, int N, int heads_total, int d, bool bwd) {
    RowGrid g;
    g.tokens = kRowThreads / (d / 8);
    g.blocks = (int)(((long long)B * N + g.tokens - 1) / g.tokens);
    auto groups = [&](int want, int most) { return std::max(1, std::min(most, (want + g.blocks - 1) / g.blocks)); };
    g.groups = bwd ? groups(kRowWgsBwd, heads_total)
                   : std::max(groups(kRowWgs, heads_total / kRowHeadsMin), groups(kRowWgsFew, heads_total));
    g.per_group = (heads_total + g.groups - 1) / g.groups;
    g.groups = (heads_total + g.per_group - 1) / g.per_group;
    g.grid_x = bwd ? std::min(g.blocks, std::max(1, kRowWgsBwd / g.groups)) : g.blocks;
    return g;
}

// (no call has more than kRowWgsBwd workgroups that sum)
size_t rows_partial_bytes(int d) { return (size_t)kRowWgsBwd * 2 * d * sizeof(float); }

// Sum over the LPR (8 or 16) neighbouring lanes of a row, in all of them.
template <int CTRL> __device__ __forceinline__ float lane_add(float v) {
    const int i = __float_as_int(v);
    return v + __int_as_float(__builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, true));
}
template <int LPR> __device__ __forceinline__ float row_sum(float v) {
    static_assert(LPR == 8 || LPR == 16, "a row is half or all of a 16-lane group");
    if (LPR == 16) v = lane_add<0x140>(v);      // mirrored within 16 lanes
    v = lane_add<0x141>(v);                     // mirrored within 8
    v = lane_add<0x4E>(v);                      // lane ^ 2
    return lane_add<0xB1>(v);                   // lane ^ 1
}

// A thread's eight features as four pairs f[2 i], f[2 i + 1]: neighbours, or half a head apart.
template <int D, bool HALVES, typename T> struct PairIo {
    static __device__ __forceinline__ void load(const T *row, int c, float *f) {
        if constexpr (!HALVES) {
            Io<T>::load8f(row + 8 * c, f);
        } else if constexpr (sizeof(T) == 4) {
            const f32x4 a = *reinterpret_cast<const f32x4 *>(row + 4 * c), b = *reinterpret_cast<const f32x4 *>(row + D / 2 + 4 * c);
#pragma unroll
            for (int i = 0; i < 4; ++i) { f[2 * i] = a[i]; f[2 * i + 1] = b[i]; }
        } else {
            const u32x2 a = *reinterpret_cast<const u32x2 *>(row + 4 * c), b = *reinterpret_cast<const u32x2 *>(row + D / 2 + 4 * c);
            f[0] = bf16_lo(a[0]); f[2] = bf16_hi(a[0]); f[4] = bf16_lo(a[1]); f[6] = bf16_hi(a[1]);
            f[1] = bf16_lo(b[0]); f[3] = bf16_hi(b[0]); f[5] = bf16_lo(b[1]); f[7] = bf16_hi(b[1]);
        }
    }
    static __device__ __forceinline__ void store(T *row, int c, const float *f) {
        if constexpr (!HALVES) {
            Io<T>::store8(row + 8 * c, f);
        } else {
            Io<T>::store4(row + 4 * c, f[0], f[2], f[4], f[6]);
            Io<T>::store4(row + D / 2 + 4 * c, f[1], f[3], f[5], f[7]);
        }
    }
};

// Cosines and sines of the thread's four pairs at token n.
template <int D>
__device__ __forceinline__ void token_angles(const RowArgs &a, int n, int c, const double *turns, const int *axis, float *cs, float *sn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const double p = axis[i] >= 0 ? (double)a.positions[(size_t)n * a.n_axes + axis[i]] : 0.0;
        const double t = p * turns[i];
        sincospif(2.f * (float)(t - rint(t)), &sn[i], &cs[i]);      // a turn is 2 pi
        sn[i] *= a.sign;
    }
}
template <int D> __device__ __forceinline__ void thread_turns(const RowArgs &a, int c, double *turns, int *axis) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int j = 4 * c + i;
        axis[i] = -1;
        for (int x = a.n_axes - 1; x >= 0; --x)
            if (j < a.axis_end[x]) axis[i] = x;
        turns[i] = axis[i] >= 0 ? a.freq[j] * 0.15915494309189533577 : 0.0;
    }
}

// f(Count<n>, h) for heads h0 .. h1 - 1, n of them at a time: four rows in flight a thread, what is left two and one
template <int N> struct Count { static constexpr int value = N; };
template <typename F> __device__ __forceinline__ void each_row(int h0, int h1, F f) {
    int h = h0;
    for (; h + 4 <= h1; h += 4) f(Count<4>{}, h);
    if (h + 2 <= h1) { f(Count<2>{}, h); h += 2; }
    if (h < h1) f(Count<1>{}, h);
}

template <int D, typename T, bool HALVES, bool NORM>
__global__ __launch_bounds__(kRowThreads) void rows_kernel(RowArgs a) {
    constexpr int LPR = D / 8, TOK = kRowThreads / LPR;
    typedef PairIo<D, HALVES, T> P;
    const int c = threadIdx.x % LPR;
    const int t = blockIdx.x * TOK + threadIdx.x / LPR;
    const bool valid = t < a.n_tokens;
    const int tc = valid ? t : a.n_tokens - 1;
    const int b = tc / a.N, n = tc - b * a.N;
    const int first = blockIdx.y * a.heads_per_group, last = min(first + a.heads_per_group, a.heads_total);
    float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.positions && first < a.part[0].heads + a.part[1].heads) {
        double turns[4];
        int axis[4];
        thread_turns<D>(a, c, turns, axis);
        token_angles<D>(a, n, c, turns, axis, cs, sn);
    }
    int base = 0;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        const HeadPart &hp = a.part[p];
        const int h0 = max(first - base, 0), h1 = min(last - base, hp.heads);
        base += hp.heads;
        if (h0 >= h1) continue;
        const T *x = static_cast<const T *>(hp.x) + b * hp.x_b + n * hp.x_n;
        T *o = static_cast<T *>(hp.out) + b * hp.o_b + n * hp.o_n;
        float w[8];
        if (NORM && p < 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 1.f;
            if (hp.weight) PairIo<D, HALVES, float>::load(hp.weight, c, w);
        }
        auto rows = [&](auto count, int h) {
            constexpr int U = decltype(count)::value;
            float f[U][8];
#pragma unroll
            for (int u = 0; u < U; ++u) P::load(x + (h + u) * hp.x_h, c, f[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (p < 2) {
                    float r = 1.f;
                    if (NORM) {
                        float s = 0.f;
#pragma unroll
                        for (int i = 0; i < 8; ++i) s = fmaf(f[u][i], f[u][i], s);
                        r = rsqrtf(row_sum<LPR>(s) * (1.f / D) + a.eps);
#pragma unroll
                        for (int i = 0; i < 8; ++i) f[u][i] *= r * w[i];
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float y0 = f[u][2 * i], y1 = f[u][2 * i + 1];
                        f[u][2 * i] = y0 * cs[i] - y1 * sn[i];
                        f[u][2 * i + 1] = y0 * sn[i] + y1 * cs[i];
                    }
                }
                if (valid) P::store(o + (h + u) * hp.o_h, c, f[u]);
            }
        };
        each_row(h0, h1, rows);
    }
}

constexpr int kRowHeads = 4;      // of the backward, whose last rows are loaded again where four do not divide (in steps of four, two, one: more registers, 1 to 5 % slower)

template <int D, typename T, bool HALVES>
__global__ __launch_bounds__(kRowThreads) void rows_bwd_kernel(RowArgs a) {
    constexpr int LPR = D / 8, TOK = kRowThreads / LPR;
    typedef PairIo<D, HALVES, T> P;
    __shared__ float sums[TOK][D];
    const int c = threadIdx.x % LPR, trow = threadIdx.x / LPR;
    const int first = blockIdx.y * a.heads_per_group, last = min(first + a.heads_per_group, a.heads_total);
    const bool turned = a.positions && first < a.part[0].heads + a.part[1].heads;
    double turns[4];
    int axis[4];
    if (turned) thread_turns<D>(a, c, turns, axis);
    float w[2][8], dw[2][8];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
#pragma unroll
        for (int i = 0; i < 8; ++i) { w[p][i] = 1.f; dw[p][i] = 0.f; }
        if (a.part[p].weight) PairIo<D, HALVES, float>::load(a.part[p].weight, c, w[p]);
    }
    for (int blk = blockIdx.x; blk < a.blocks; blk += gridDim.x) {
        const int t = blk * TOK + trow;
        const bool valid = t < a.n_tokens;
        const int tc = valid ? t : a.n_tokens - 1;
        const int b = tc / a.N, n = tc - b * a.N;
        float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
        if (turned) token_angles<D>(a, n, c, turns, axis, cs, sn);
        int base = 0;
#pragma unroll
        for (int p = 0; p < 3; ++p) {
            const HeadPart &hp = a.part[p];
            const int h0 = max(first - base, 0), h1 = min(last - base, hp.heads);
            base += hp.heads;
            if (h0 >= h1) continue;
            const T *g = static_cast<const T *>(hp.g) + ((size_t)b * hp.heads * a.N + n) * D;
            const T *x = static_cast<const T *>(hp.x) + b * hp.x_b + n * hp.x_n;
            T *o = static_cast<T *>(hp.out) + b * hp.o_b + n * hp.o_n;
            for (int h = h0; h < h1; h += kRowHeads) {
                float f[kRowHeads][8], y[kRowHeads][8];
#pragma unroll
                for (int u = 0; u < kRowHeads; ++u) {
                    const int hc = min(h + u, h1 - 1);
                    P::load(g + (size_t)hc * a.N * D, c, f[u]);
                    if (p < 2) P::load(x + hc * hp.x_h, c, y[u]);
                }
#pragma unroll
                for (int u = 0; u < kRowHeads; ++u) {
                    const bool mine = valid && h + u < h1;
                    if (p < 2) {
                        float s = 0.f, m = 0.f;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float g0 = f[u][2 * i], g1 = f[u][2 * i + 1];
                            f[u][2 * i] = g0 * cs[i] + g1 * sn[i];
                            f[u][2 * i + 1] = g1 * cs[i] - g0 * sn[i];
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            s = fmaf(y[u][i], y[u][i], s);
                            m = fmaf(f[u][i] * w[p][i], y[u][i], m);
                        }
                        const float r = rsqrtf(row_sum<LPR>(s) * (1.f / D) + a.eps);
                        m = row_sum<LPR>(m) * r * (1.f / D);            // mean(dn * n)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float nrm = y[u][i] * r;
                            if (mine) dw[p][i] = fmaf(f[u][i], nrm, dw[p][i]);
                            f[u][i] = r * (f[u][i] * w[p][i] - nrm * m);
                        }
                    }
                    if (mine) P::store(o + (h + u) * hp.o_h, c, f[u]);
                }
            }
        }
    }
    // the workgroup's sums for the weights' gradients, its tokens in their order
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        if (p) __syncthreads();
        PairIo<D, HALVES, float>::store(sums[trow], c, dw[p]);
        __syncthreads();
        if (threadIdx.x < D) {
            float s = 0.f;
            for (int r = 0; r < TOK; ++r) s += sums[r][threadIdx.x];
            a.partial[(((size_t)blockIdx.y * gridDim.x + blockIdx.x) * 2 + p) * D + threadIdx.x] = s;
        }
    }
}

// dw[p][e] = sum of the workgroups' sums: 16 features a workgroup, 64 slices of the partials side by side, both in a fixed order.
constexpr int kDwFeat = 16, kDwSlices = 64;
__global__ __launch_bounds__(kDwFeat *kDwSlices) void weight_grad_kernel(const float *__restrict__ partial, int count, int d, float *dq_w, float *dk_w) {
    __shared__ float sums[kDwSlices][kDwFeat];
    const int e = threadIdx.x % kDwFeat, sl = threadIdx.x / kDwFeat;
    const int per_part = d / kDwFeat, p = blockIdx.x / per_part, col = (blockIdx.x % per_part) * kDwFeat + e;
    float *out = p ? dk_w : dq_w;
    if (!out) return;
    float s = 0.f;
#pragma unroll 4
    for (int i = sl; i < count; i += kDwSlices) s += partial[((size_t)i * 2 + p) * d + col];
    sums[sl][e] = s;
    __syncthreads();
    if (sl == 0) {
        for (int i = 1; i < kDwSlices; ++i) s += sums[i][e];
        out[col] = s;
    }
}

static void fill_grid(RowArgs &a, const RowGrid &g) {
    a.heads_per_group = g.per_group;
    a.blocks = g.blocks;
}

template <int D, typename T> static void rows_dispatch(const RowArgs &a, dim3 grid, bool norm, bool halves, hipStream_t st) {
    if (norm && halves) rows_kernel<D, T, true, true><<<grid, kRowThreads, 0, st>>>(a);
    else if (norm) rows_kernel<D, T, false, true><<<grid, kRowThreads, 0, st>>>(a);
    else if (halves) rows_kernel<D, T, true, false><<<grid, kRowThreads, 0, st>>>(a);
    else rows_kernel<D, T, false, false><<<grid, kRowThreads, 0, st>>>(a);
}

hipError_t launch_rows(RowArgs a, int B, int d, int dtype, bool norm, bool halves, hipStream_t st) {
    const RowGrid g = row_grid(B, a.N, a.heads_total, d, false);
    fill_grid(a, g);
    const dim3 grid(g.grid_x, g.groups);
    MOC_PROF(norm ? "qk_norm_rope" : "rope", st);
    if (d == 128 && dtype == MOC_BF16) rows_dispatch<128, bf16_t>(a, grid, norm, halves, st);
    else if (d == 128) rows_dispatch<128, float>(a, grid, norm, halves, st);
    else if (dtype == MOC_BF16) rows_dispatch<64, bf16_t>(a, grid, norm, halves, st);
    else rows_dispatch<64, float>(a, grid, norm, halves, st);
    return hipGetLastError();
}

template <int D, typename T> static void rows_bwd_dispatch(const RowArgs &a, dim3 grid, bool halves, hipStream_t st) {
    if (halves) rows_bwd_kernel<D, T, true><<<grid, kRowThreads, 0, st>>>(a);
    else rows_bwd_kernel<D, T, false><<<grid, kRowThreads, 0, st>>>(a);
}

hipError_t launch_rows_bwd(RowArgs a, int B, int d, int dtype, bool halves, float *dq_weight, float *dk_weight, hipStream_t st) {
    const RowGrid g = row_grid(B, a.N, a.heads_total, d, true);
    fill_grid(a, g);
    const dim3 grid(g.grid_x, g.groups);
    {
        MOC_PROF("qk_norm_rope_bwd", st);
        if (d == 128 && dtype == MOC_BF16) rows_bwd_dispatch<128, bf16_t>(a, grid, halves, st);
        else if (d == 128) rows_bwd_dispatch<128, float>(a, grid, halves, st);
        else if (dtype == MOC_BF16) rows_bwd_dispatch<64, bf16_t>(a, grid, halves, st);
        else rows_bwd_dispatch<64, float>(a, grid, halves, st);
    }
    if (dq_weight || dk_weight) {
        MOC_PROF("weight_grad", st);
        weight_grad_kernel<<<2 * d / kDwFeat, kDwFeat * kDwSlices, 0, st>>>(a.partial, g.grid_x * g.groups, d, dq_weight, dk_weight);
    }
    return hipGetLastError();
}

}  // namespace moc
