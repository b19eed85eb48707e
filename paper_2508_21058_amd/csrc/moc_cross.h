// Tiles and work items shared by the cross attention kernels.
#pragma once
#include "moc_attn_common.h"
#include "moc_block.h"

namespace moc {

constexpr int kCrossRows = 128;      // queries of a workgroup in the query-stationary passes: four waves of 32

// What the kernels need of a storage type: T = bf16 runs on 32x32x16 matrix instructions, T = float on 32x32x2 ones. A tile in
// LDS is row-major without padding, its 16-byte groups XOR-swizzled by the row (SwTile for bf16).
//   frag(tile, row0, s)      row operand: rows row0 .. row0 + 31, features of step s
//   tfrag(tile, row0, b, s)  transposed operand: feature block b (32), rows of step s behind row0
//   pack(acc, s)             a step of rows of an accumulator as the other operand of a product with tfrag
//   mma                      the product of one step
// KS: steps of a row's features. RS: steps of 32 rows.
template <int D, typename T> struct Ops;
template <int D> struct Ops<D, bf16_t> {
    typedef bf16x8 Frag;
    static constexpr int KS = D / 16, RS = 2, RB = D * 2;
    LaneOffs<D> lo;
    __device__ __forceinline__ void init(int lane) { lo.init(lane); }
    __device__ __forceinline__ void pin() { lo.pin(); }      // (see LaneOffs)
    __device__ __forceinline__ Frag frag(const char *tile, int row0, int s) const {
        return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(tile + lo.row[s] + row0 * RB));
    }
    __device__ __forceinline__ Frag tfrag(const char *tile, int row0, int b, int s) const {
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        const char *p = tile + (row0 + 16 * s) * RB;
        s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + lo.tr[2 * b]));
        s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p + lo.tr[2 * b + 1]));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        s16x8 r = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
        return __builtin_bit_cast(bf16x8, r);
    }
    // P and dS are rounded to bf16 here, half a step 2^-8 each: the second products run on bf16 matrix cores, sixteen times the rate of the float ones.
    // (Results are 2.2e-3 to 2.4e-3 of their norm off, of which their own rounding is 1.7e-3.)
    static __device__ __forceinline__ Frag pack(const f32x16 &acc, int s) { return acc_to_frag(acc, s); }
    static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) { return mfma32(a, b, c); }
    // the same operand of a row in memory
    static __device__ __forceinline__ Frag row_frag(const bf16_t *row, int s, int half) { return Io<bf16_t>::load8(row + 16 * s + 8 * half); }
    static __device__ __forceinline__ float dot(Frag a, Frag b) {
        const u32x4 x = __builtin_bit_cast(u32x4, a), y = __builtin_bit_cast(u32x4, b);
        float r = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) r = fmaf(bf16_lo(x[i]), bf16_lo(y[i]), fmaf(bf16_hi(x[i]), bf16_hi(y[i]), r));
        return r;
    }
    static __device__ __forceinline__ int swizzle(int row) { return SwTile<D>::sw(row); }
};
template <int D> struct Ops<D, float> {
    typedef f32x4 Frag;
    static constexpr int KS = D / 8, RS = 4, RB = D * 4;
    // Lane-dependent byte offsets; what depends on the step, the block or the tile goes into the instruction.
    int row[8];      // row operand of steps s and s + 8
    int tr[4];       // transposed operand, element e of any step: the swizzle's low bits are the lane's, bit 3 flips neighbouring blocks
    __device__ __forceinline__ void init(int lane) {
        const int l32 = lane & 31, half = lane >> 5;
#pragma unroll
        for (int s = 0; s < 8; ++s) row[s] = l32 * RB + (((2 * s + half) ^ (l32 & 15)) << 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) tr[e] = (4 * half + e) * RB + (((l32 >> 2) ^ (4 * half + e)) << 4) + (l32 & 3) * 4;
    }
    __device__ __forceinline__ void pin() {
#pragma unroll
        for (int s = 0; s < 8; ++s) asm volatile("" : "+v"(row[s]));
#pragma unroll
        for (int e = 0; e < 4; ++e) asm volatile("" : "+v"(tr[e]));
    }
    static __device__ __forceinline__ int swizzle(int row) { return row & 15; }
    // step s: features 8 s + 4 half .. + 4, one for each of four matrix instructions
    __device__ __forceinline__ Frag frag(const char *tile, int row0, int s) const {
        return *reinterpret_cast<const f32x4 *>(tile + row[s & 7] + row0 * RB + (s >> 3) * 256);
    }
    // rows 8 s + 4 half + e, the rows of accumulator registers 4 s + e
    __device__ __forceinline__ Frag tfrag(const char *tile, int row0, int b, int s) const {
        f32x4 r;
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const float *>(tile + tr[e] + (row0 + 8 * s) * RB + (b ^ (s & 1)) * 128);
        return r;
    }
    static __device__ __forceinline__ Frag pack(const f32x16 &acc, int s) { return f32x4{acc[4 * s], acc[4 * s + 1], acc[4 * s + 2], acc[4 * s + 3]}; }
    static __device__ __forceinline__ f32x16 mma(Frag a, Frag b, f32x16 c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b[e], c, 0, 0, 0);
        return c;
    }
    static __device__ __forceinline__ Frag row_frag(const float *row, int s, int half) { return *reinterpret_cast<const f32x4 *>(row + 8 * s + 4 * half); }
    static __device__ __forceinline__ float dot(Frag a, Frag b) { return fmaf(a[0], b[0], fmaf(a[1], b[1], fmaf(a[2], b[2], a[3] * b[3]))); }
};

// A wave's share of the asynchronous copy of `valid` rows (the others repeat the last of them) to a tile of ROWS rows; the base is
// in scalar registers that a vector instruction may just have written, hence the wait states in front of the load.
__device__ __forceinline__ void cross_copy16(const void *base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %0, %1"
                 :: "v"(off), "s"(uniform_ptr(base)), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory", "m0");
}
template <int D, typename T, int ROWS, int NW = 4>
__device__ __forceinline__ void copy_tile(const T *first, int valid, char *tile, int wave, int lane) {
    constexpr int RB = D * (int)sizeof(T), GR = RB / 16, RPI = 64 / GR, NI = ROWS / RPI;
    static_assert(NI % NW == 0, "rows divide evenly among the waves");
    const uint32_t at = lds_address(tile);
#pragma unroll
    for (int p = 0; p < NI / NW; ++p) {
        const int n = wave + NW * p, row = n * RPI + lane / GR;
        const uint32_t off = (uint32_t)min(row, valid - 1) * RB + (((lane % GR) ^ Ops<D, T>::swizzle(row)) << 4);
        cross_copy16(first, off, at + n * 1024);
    }
}

// Where a segment has fewer queries, neighbours with the same range are looked for, since their tiles are better cut as one run's (a padded batch in
// many segments). Where all are long that gains nothing, and an item would wait for the ranges before its first load (eight segments of 14k queries,
// 24 heads: forward 506 us, 495 without, dQ 832 and 814).
constexpr int kCrossJoin = 8 * kCrossRows;
// Work item of the query-stationary passes: up to kCrossRows queries of one segment of one query head.
struct CrossItem {
    int bhk, count, first, end;      // key head of all samples, queries, range of states
    long long row;                   // first query in [B * H * N]
};
__device__ __forceinline__ CrossRange cross_range(const CrossArgs &a, int b, int s) {
    CrossRange r = {0, a.M};
    if (a.ranges) {
        r = a.ranges[(size_t)b * a.n_seg + s];
        r.first = max(r.first, 0);
        r.end = min(r.end, a.M);
    }
    return r;
}
// Which segments of a sample attend what the segment before them attends (bit s of the 128): in a padded batch all do. Every lane of a
// wave has to be here.
struct SegmentBits {
    unsigned long long lo, hi;
    __device__ __forceinline__ bool at(int s) const { return ((s < 64 ? lo >> s : hi >> (s - 64)) & 1) != 0; }
};
__device__ __forceinline__ SegmentBits same_as_before(const CrossArgs &a, int b) {
    const int lane = threadIdx.x & 63;
    auto range = [&](int s) {
        CrossRange r = {0, 0};
        if (s < a.n_seg) r = cross_range(a, b, s);
        if (r.end <= r.first) r.first = r.end = 0;
        return r;
    };
    // (the exchanges are outside the conditions: lanes that skip one would hand nothing on)
    const CrossRange r = range(lane);
    const int rf = __shfl_up(r.first, 1, 64), re = __shfl_up(r.end, 1, 64);
    SegmentBits m = {__ballot(lane > 0 && lane < a.n_seg && rf == r.first && re == r.end), 0};
    if (a.n_seg > 64) {
        const CrossRange q = range(lane + 64);
        int qf = __shfl_up(q.first, 1, 64), qe = __shfl_up(q.end, 1, 64);
        const int f = __shfl(r.first, 63, 64), e = __shfl(r.end, 63, 64);
        if (lane == 0) { qf = f; qe = e; }
        m.hi = __ballot(lane + 64 < a.n_seg && qf == q.first && qe == q.end);
    }
    return m;
}
// The i-th key head of all samples in the order in which items are dealt out: sample after sample for each head, so that the slices of the XCDs
// have items of every sample. (In a padded batch ranges differ, and the XCDs of the short ones would idle: three samples of 11k queries, 36 heads on
// twelve, ranges of 539, 0 and 816 states, forward 486 us, this way 325, dQ 716 and 539.)
__device__ __forceinline__ int dealt_head(const CrossArgs &a, int i) {
    if (a.BHk == a.Hk) return i;
    const int B = a.BHk / a.Hk, hk = i / B;
    return (i - hk * B) * a.Hk + hk;
}
// Items of the query-stationary passes in slices of the XCDs, whose L2 then holds the states of a few heads. Samples of fewer heads than XCDs fill whole
// slices all the same: where their ranges may differ and a head has queries enough, items are dealt one by one (four samples of 30k queries, two
// heads, ranges of 498, 0, 81 and 380 states: forward 73 us, this way 52, dQ 112 and 83; one query a sample, where the order of reading decides, 13 and 16).
__device__ __forceinline__ bool cross_logical(const CrossArgs &a, int &logical) {
    const long long total = (long long)a.tiles * a.copies * a.BHk * a.split;
    if (a.dealt) {
        logical = blockIdx.x;
        return logical < total;
    }
    return xcd_remap(total, logical);
}
// Neighbouring segments with one range are one run of queries, cut into whole tiles; the tiles that are then too many have no queries.
__device__ __forceinline__ CrossItem cross_item(const CrossArgs &a, int logical) {
    CrossItem it;
    const int per_head = a.tiles * a.copies;
    const int i = logical / per_head;
    it.bhk = dealt_head(a, i);
    const int b = it.bhk / a.Hk;
    const int rest = logical - i * per_head, copy = rest / a.tiles, t = rest - copy * a.tiles;
    int s = 0, e = 0;
    if (a.n_seg > 1) {
        int hi = a.n_seg;                                      // the last segment with tile_at <= t
        while (hi - s > 1) {
            const int mid = (s + hi) >> 1;
            if (a.tile_at[mid] <= t) s = mid; else hi = mid;
        }
        e = s;
        if (a.joined) {
            const SegmentBits same = same_as_before(a, b);
            while (s > 0 && same.at(s)) --s;
            while (e + 1 < a.n_seg && same.at(e + 1)) ++e;
        }
    }
    const int q = a.q_off[s] + (t - a.tile_at[s]) * kCrossRows;
    it.count = min(kCrossRows, a.q_off[e + 1] - q);
    it.row = ((long long)it.bhk * a.copies + copy) * a.N + q;
    const CrossRange r = cross_range(a, b, s);
    it.first = __builtin_amdgcn_readfirstlane(r.first);
    it.end = __builtin_amdgcn_readfirstlane(r.end);
    return it;
}
// The part of a range that split z of n takes, whole tiles of `tile` states.
__device__ __forceinline__ void cross_slice(int &first, int &end, int z, int n, int tile) {
    if (n == 1 || end <= first) return;
    const int tiles = (end - first + tile - 1) / tile, f = first;
    first = min(end, f + (int)((long long)tiles * z / n) * tile);
    end = min(end, f + (int)((long long)tiles * (z + 1) / n) * tile);
}

// Cuts the states of sample b into the tiles of the wide key-stationary pass: a workgroup of 256 threads. The tiles of segments come
// first.
constexpr int kCuts = 2 * MOC_MAX_CROSS_SEGMENTS + 2;
struct CutLds {
    int first[MOC_MAX_CROSS_SEGMENTS], end[MOC_MAX_CROSS_SEGMENTS], cut[kCuts], sorted[kCuts], tile_at[kCuts];
    uint32_t segments[kCuts][MOC_MAX_CROSS_SEGMENTS / 32];
};
__device__ __forceinline__ void cross_cut(const CrossArgs &a, int b, CutLds &m) {
    auto &first = m.first, &end = m.end;
    auto &cut = m.cut, &sorted = m.sorted, &tile_at = m.tile_at;
    auto &segments = m.segments;
    const int tid = threadIdx.x, S = a.n_seg;
    const int n = 2 * S + 2;
    if (tid < S) {
        CrossRange r = cross_range(a, b, tid);
        if (r.end <= r.first || a.q_off[tid + 1] == a.q_off[tid]) r.first = r.end = 0;
        first[tid] = cut[2 * tid] = r.first;
        end[tid] = cut[2 * tid + 1] = r.end;
    }
    if (tid == 0) { cut[n - 2] = 0; cut[n - 1] = a.M; }
    __syncthreads();
    for (int i = tid; i < n; i += 256) {
        const int x = cut[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += cut[j] < x || (cut[j] == x && j < i);
        sorted[rank] = x;
    }
    __syncthreads();
    // piece i: states [sorted[i], sorted[i + 1]), of a range or of none; its tiles from tile_at[i] on, those of ranges first
    for (int i = tid; i < n; i += 256) {
        for (int w = 0; w < MOC_MAX_CROSS_SEGMENTS / 32; ++w) {
            uint32_t in = 0;
            for (int s = 32 * w; s < min(32 * w + 32, S) && i + 1 < n; ++s)
                if (first[s] <= sorted[i] && end[s] >= sorted[i + 1]) in |= 1u << (s & 31);
            segments[i][w] = in;
        }
    }
    __syncthreads();
    auto attended = [&](int i) { return (segments[i][0] | segments[i][1] | segments[i][2] | segments[i][3]) != 0; };
    static_assert(MOC_MAX_CROSS_SEGMENTS == 128, "four words of segments");
    for (int i = tid; i + 1 < n; i += 256) {
        const bool mine = attended(i);
        int at = 0;
        for (int j = 0; j + 1 < n; ++j) {
            const bool other = attended(j);
            if (other == mine ? j < i : other) at += (sorted[j + 1] - sorted[j] + kWideTile - 1) / kWideTile;
        }
        tile_at[i] = at;
    }
    __syncthreads();
    CrossKeys *out = a.items + (size_t)b * a.max_items;
    int live = 0, total = 0;
    for (int i = 0; i + 1 < n; ++i) {
        const int tiles = (sorted[i + 1] - sorted[i] + kWideTile - 1) / kWideTile;
        total += tiles;
        live += attended(i) ? tiles : 0;
        for (int t = tid; t < tiles; t += 256) {
            CrossKeys k{};
            k.start = sorted[i] + t * kWideTile;
            k.len = min(kWideTile, sorted[i + 1] - k.start);
            for (int w = 0; w < MOC_MAX_CROSS_SEGMENTS / 32; ++w) k.segments[w] = segments[i][w];
            out[tile_at[i] + t] = k;
        }
    }
    if (tid == 0) a.item_counts[b] = CrossCount{live, total - live};
}

// A wave's 32 x D transposed accumulator (lane: row l32, four-feature pieces) times `scale` to the float rows at `out`.
template <int D> __device__ __forceinline__ void store_rows_f32(const f32x16 *acc, float scale, float *row, int half) {
#pragma unroll
    for (int b = 0; b < D / 32; ++b)
#pragma unroll
        for (int g = 0; g < 4; ++g)
            Io<float>::store4(row + b * 32 + g * 8 + half * 4, acc[b][4 * g] * scale, acc[b][4 * g + 1] * scale, acc[b][4 * g + 2] * scale,
                              acc[b][4 * g + 3] * scale);
}

}  // namespace moc
