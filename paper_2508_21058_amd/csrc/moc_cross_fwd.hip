// Cross attention forward: o = softmax(q K^T scale) V over the range of encoder states that a query's segment attends.
//
// One pass with a running maximum and sum. A workgroup owns 128 queries, four waves of 32, and streams the range's states through LDS in
// double-buffered tiles. S^T = K Q^T and O^T = V^T P^T, so that a lane owns a query: its statistics are scalars and the scores feed the second
// product from the registers they are in. Calls of few query tiles split the range over workgroups, whose results a second launch joins.
//
// In bf16 three workgroups share a compute unit (168 registers, tiles of 32 states): 114k queries of 24 heads, eight shots of captions of 100 to 512
// states 569 -> 506 us against two of 64-state tiles (of 32: 594), 33k queries against 4,357 states 1,886 -> 1,835
// (cards differ by 7 %: on another one tile buffers as constants took the latter from 1,790 to 1,723).
//
// What bounds it: at long ranges the products (the latter stands at 1,640 to 1,650 us, 1,080 TFLOP/s, near what the chip's power allows); at short ones
// products and vector work, which share a SIMD's issue (39 % of the cycles each), and the rows of q and o, 130 of the 506 us.
#include "moc_cross.h"

namespace moc {

template <int D, typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 3 : 2) void cross_fwd_kernel(CrossArgs a) {
    typedef Ops<D, T> O;
    constexpr int BN = 32, DB = D / 32;
    constexpr int TB = BN * O::RB;
    constexpr int PATCH = sizeof(T) == 2 ? 4 * (32 * (D + 4) + 64) * 2 : 0;      // what store_rows_bf16 takes
    __shared__ __attribute__((aligned(1024))) char smem[4 * TB > PATCH ? 4 * TB : PATCH];      // K, V, twice
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, l32 = lane & 31;
    int logical;
    if (!cross_logical(a, logical)) return;
    const int z = logical % a.split;
    CrossItem it = cross_item(a, logical / a.split);
    if (it.count <= 0) return;
    cross_slice(it.first, it.end, z, a.split, BN);
    const int r = wave * 32 + l32, rc = min(r, it.count - 1);
    const bool row_valid = r < it.count;
    const size_t row = (size_t)it.row + rc;
    T *out = static_cast<T *>(a.o) + row * D;
    float *pout = a.split > 1 ? a.part + ((size_t)z * a.rows + row) * D : nullptr;
    float *lout = a.split > 1 ? a.part_lse + (size_t)z * a.rows + row : a.lse + row;
    f32x16 oacc[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b) oacc[b] = zero16();
    float m_run = -INFINITY, l_run = 0.f;
    if (it.first < it.end) {
        const T *kb = static_cast<const T *>(a.k) + (size_t)it.bhk * a.M * D, *vb = static_cast<const T *>(a.v) + (size_t)it.bhk * a.M * D;
        O ops;
        ops.init(lane);
        const float c = a.scale_log2;
        auto issue = [&](int pos, int buf) {
            const int valid = min(BN, it.end - pos);
            copy_tile<D, T, BN>(kb + (size_t)pos * D, valid, smem + buf * 2 * TB, wave, lane);
            copy_tile<D, T, BN>(vb + (size_t)pos * D, valid, smem + buf * 2 * TB + TB, wave, lane);
        };
        issue(it.first, 0);
        const T *qrow = static_cast<const T *>(a.q) + row * D;
        typename O::Frag qf[O::KS];
#pragma unroll
        for (int s = 0; s < O::KS; ++s) qf[s] = O::row_frag(qrow, s, half);
        // One tile; the buffers take turns in a loop unrolled by two, so that LDS addresses are constants beside the lane's offsets.
        auto tile = [&](auto which, int pos) {
            constexpr int BUF = decltype(which)::value;
            wait_vmcnt<0>();
            __syncthreads();
            if (pos + BN < it.end) issue(pos + BN, BUF ^ 1);
            if (wave * 32 >= it.count) return;
            ops.pin();
            const char *kt = smem + BUF * 2 * TB, *vt = kt + TB;
            const int valid = it.end - pos;
            f32x16 s = zero16();
#pragma unroll
            for (int i = 0; i < O::KS; ++i) s = O::mma(ops.frag(kt, 0, i), qf[i], s);
            if (valid < BN) {
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if ((i >> 2) * 8 + half * 4 + (i & 3) >= valid) s[i] = -INFINITY;
            }
            float mx = s[0];
#pragma unroll
            for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
            const float m_new = fmaxf(m_run, xhalf_max(mx));
            if (pos == it.first) {
                m_run = m_new;
            } else if (__any((m_new - m_run) * c > 8.f)) {      // moved, and the sums rescaled, only when it has grown by 2^8
                const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * c);
                l_run *= alpha;
#pragma unroll
                for (int b = 0; b < DB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) oacc[b][i] *= alpha;
                m_run = m_new;
            }
            const float mc = m_run * c;
            float l_tile = 0.f;                // (on its own first: a long range adds few large numbers)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], c, -mc));
                l_tile += s[i];
            }
            l_run += l_tile;
#pragma unroll
            for (int ks = 0; ks < O::RS; ++ks) {
                const typename O::Frag pf = O::pack(s, ks);
#pragma unroll
                for (int b = 0; b < DB; ++b) oacc[b] = O::mma(ops.tfrag(vt, 0, b, ks), pf, oacc[b]);
            }
        };
        for (int pos = it.first; pos < it.end; pos += 2 * BN) {
            tile(IC<0>{}, pos);
            if (pos + BN < it.end) tile(IC<1>{}, pos + BN);
        }
    }
    const float l = xhalf_sum(l_run);
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;      // nothing attended: o = 0, lse = -inf
    const float lse = l > 0.f || l != l ? m_run * a.scale + logf(l) : -INFINITY;
    if (row_valid && half == 0) *lout = lse;
    if (a.split > 1) {
        if (row_valid && it.first < it.end) store_rows_f32<D>(oacc, inv, pout, half);
    } else if constexpr (sizeof(T) == 4) {
        if (row_valid) store_rows_f32<D>(oacc, inv, out, half);
    } else {
        __syncthreads();
        store_rows_bf16<D>(smem, wave, lane, oacc, inv, row_valid ? r : -1, static_cast<bf16_t *>(a.o) + (size_t)it.row * D);
    }
}

// Joins the results of split calls: lse = log sum_z exp(lse_z), o = sum_z exp(lse_z - lse) o_z; a split without states has lse_z = -inf and no o_z.
// SL slices of threads share a row: slice j takes every SL-th split, four features a thread, and the slices are joined in their order. (48 rows of
// 32 splits: one slice 21 us, eight 7; 51k rows of two splits: a workgroup of eight slices a row 43 us, of eight rows 15. Where
// rows fill the chip by themselves, as in calls cut for the length of their sums, one slice: 131k rows of 64 features, nine splits, eight slices 158 us, one 70.)
constexpr int kJoinThreads = 256, kJoinFew = 4, kJoinRows = 1 << 16;
template <int D, typename T, int SL> __global__ __launch_bounds__(kJoinThreads) void cross_join_kernel(CrossArgs a) {
    constexpr int LPR = D / 4, ROWS = kJoinThreads / (LPR * SL);
    __shared__ __attribute__((aligned(16))) float part[ROWS * SL][D + 4];
    const size_t rows = (size_t)a.rows;
    const int c = threadIdx.x % LPR * 4, j = threadIdx.x / LPR % SL, mine = threadIdx.x / (LPR * SL);
    const size_t row = min((size_t)blockIdx.x * ROWS + mine, rows - 1);       // (a row too many is the last one again: same values)
    float mx = -INFINITY;
#pragma unroll 4
    for (int z = j; z < a.split; z += SL) {
        const float x = a.part_lse[z * rows + row];
        mx = x != x ? INFINITY : fmaxf(mx, x);              // (a NaN makes the weights NaN: inf - inf)
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    float sum = 0.f;
#pragma unroll 4
    for (int z = j; z < a.split; z += SL) {
        const float x = a.part_lse[z * rows + row];
        const f32x4 part_o = *reinterpret_cast<const f32x4 *>(a.part + (z * rows + row) * D + c);      // (asked for before x is looked at)
        if (x == -INFINITY) continue;
        const float w = expf(x - mx);
        sum += w;
        o += w * part_o;
    }
    if (SL > 1) {
        *reinterpret_cast<f32x4 *>(&part[mine * SL + j][c]) = o;
        if (c == 0) { part[mine * SL + j][D] = sum; part[mine * SL + j][D + 1] = mx; }
        __syncthreads();
        if (j > 0) return;
        for (int i = 1; i < SL; ++i) mx = fmaxf(mx, part[mine * SL + i][D + 1]);
        o = f32x4{0.f, 0.f, 0.f, 0.f};
        sum = 0.f;
        for (int i = 0; i < SL; ++i) {
            const float m = part[mine * SL + i][D + 1];
            if (m == -INFINITY) continue;
            const float w = expf(m - mx);
            sum += w * part[mine * SL + i][D];
            o += w * *reinterpret_cast<const f32x4 *>(&part[mine * SL + i][c]);
        }
    }
    if (c == 0) a.lse[row] = mx > -INFINITY ? mx + logf(sum) : -INFINITY;
    const float inv = mx > -INFINITY ? 1.f / sum : 0.f;
    Io<T>::store4(static_cast<T *>(a.o) + row * D + c, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
}

template <int D, typename T> static void fwd_dispatch(CrossArgs &a, hipStream_t st) {
    cross_tiles(a);
    {
        MOC_PROF("cross_fwd", st);
        cross_fwd_kernel<D, T><<<xcd_grid((long long)a.tiles * a.copies * a.BHk * a.split), 256, 0, st>>>(a);
    }
    if (a.split > 1) {
        MOC_PROF("cross_join", st);
        constexpr int SL = kJoinThreads / (D / 4);
        if (a.split <= kJoinFew || a.rows >= kJoinRows) cross_join_kernel<D, T, 1><<<(unsigned)((a.rows + SL - 1) / SL), kJoinThreads, 0, st>>>(a);
        else cross_join_kernel<D, T, SL><<<(unsigned)a.rows, kJoinThreads, 0, st>>>(a);
    }
}

hipError_t launch_cross_fwd(CrossArgs a, int d, int dtype, hipStream_t st) {
    if (d == 128 && dtype == MOC_BF16) fwd_dispatch<128, bf16_t>(a, st);
    else if (d == 128) fwd_dispatch<128, float>(a, st);
    else if (dtype == MOC_BF16) fwd_dispatch<64, bf16_t>(a, st);
    else fwd_dispatch<64, float>(a, st);
    return hipGetLastError();
}

// ---- how the queries are cut ----------------------------------------------------------------------
void cross_tiles(CrossArgs &a) {
    a.tiles = 0;
    a.joined = false;
    for (int s = 0; s < a.n_seg; ++s) {
        const int rows = a.q_off[s + 1] - a.q_off[s];
        a.tile_at[s] = a.tiles;
        a.tiles += (rows + kCrossRows - 1) / kCrossRows;
        a.joined |= a.n_seg > 1 && rows < kCrossJoin;
    }
    a.tile_at[a.n_seg] = a.tiles;
    a.dealt = a.ranges && a.BHk > a.Hk && a.Hk < kXcds && a.tiles >= kXcds;
}

}  // namespace moc
