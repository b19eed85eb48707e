// dK / dV of cross attention on tiles of 256 states, heads of 128 features in bf16: the key-stationary pass of moc_dkdv_wide.h.
//
// That pass has no masks: every query of its stream attends every key of its tile. So a sample's states are cut where a range of one
// of its segments begins or ends, and the pieces into tiles; a tile streams the queries of the segments whose ranges hold it, all of
// them or, where the call has few tiles, one part in `split`. States of no range are tiles without segments, whose gradients are zero.
// Ranges are on the device, so the cutting is too (cross_cut).
#include "moc_block.h"
#include "moc_dkdv_wide.h"

namespace moc {

namespace wide {
// Pieces of contiguous queries: the segments of a tile, neighbours as one, for every query head of the group in turn, of them `stages` stages.
struct PieceSource {
    int n_direct, q_start, q_len;                       // the first piece, in queries of the key head
    const CrossArgs &a;
    const CrossKeys &keys;
    const char *inf_rec, *records;                      // (records of the key head)
    const char *rec_ptr;
    int first, rec_left, copy, seg, stages;             // of the piece: its first query and queries left; stages left behind it
    __device__ __forceinline__ PieceSource(const CrossArgs &args, const CrossKeys &k) : a(args), keys(k) {}
    __device__ __forceinline__ bool has(int s) const { return (keys.segments[s >> 5] >> (s & 31) & 1u) != 0; }
    __device__ __forceinline__ int next_segment(int s) const {      // the first segment of the tile from s on, or n_seg
        while (s < a.n_seg && !has(s)) ++s;
        return s;
    }
    __device__ __forceinline__ int piece_end(int s) const {         // behind the last segment of the piece that begins at s
        while (s < a.n_seg && has(s)) ++s;
        return s;
    }
    __device__ __forceinline__ int stages_of(int s) const { return (a.q_off[piece_end(s)] - a.q_off[s] + R - 1) / R; }
    // the piece at (copy, seg) from its stage `skip` on
    __device__ __forceinline__ void enter(int skip) {
        first = copy * a.N + a.q_off[seg] + skip * R;
        rec_left = a.q_off[piece_end(seg)] - a.q_off[seg] - skip * R;
        const int n = (rec_left + R - 1) / R;
        if (n > stages) rec_left = stages * R;
        stages -= min(n, stages);
        rec_ptr = records + (size_t)first * 16;
    }
    __device__ __forceinline__ void advance() {
        seg = next_segment(piece_end(seg));
        if (seg == a.n_seg) { ++copy; seg = next_segment(0); }
        enter(0);
    }
    __device__ __forceinline__ void issue(uint32_t dst, uint32_t rec_off, int rec_row, int rec_sel) {
        if (rec_left >= R) {
            copy4(rec_ptr, rec_off, dst);
        } else {
            if (rec_left <= 0 && stages > 0) advance();
            // (past the last stage rec_left - 1 is negative and leads back to the last record)
            const char *const at = rec_ptr + (min(rec_row, rec_left - 1) * 16 + rec_sel);
            copy4(rec_row >= rec_left && rec_sel == 0 ? inf_rec : at, dst);
        }
        rec_ptr += RECB;
        rec_left -= R;
    }
};
}  // namespace wide

template <bool BIG>
__global__ __launch_bounds__(256, 1) void cross_dkdv_wide_kernel(CrossArgs a) {
    using namespace wide;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];
    // Tiles that stream come first, then those without a segment, both in slices of the XCDs. (Were they mixed, tiles that end at
    // once would take every second or fourth workgroup, and the shader engines that these go to would idle: one live tile of four,
    // 114k queries of 24 heads, 256 states 2,300 us, packed 722.)
    int l, bhk, z, item;
    {
        const int lane = threadIdx.x & 63, B = a.BHk / a.Hk;
        auto units = [&](int b, bool live) {
            if (b >= B) return 0;
            const CrossCount n = a.item_counts[b];
            return live ? n.live * a.split * a.Hk : n.idle * a.Hk;
        };
        int total[2] = {0, 0};
        for (int b = lane; b < B; b += 64) { total[0] += units(b, true); total[1] += units(b, false); }
#pragma unroll
        for (int w = 1; w < 64; w <<= 1) { total[0] += __shfl_xor(total[0], w, 64); total[1] += __shfl_xor(total[1], w, 64); }
        const int x = blockIdx.x % kXcds, p = blockIdx.x / kXcds, per_live = (total[0] + kXcds - 1) / kXcds, per_idle = (total[1] + kXcds - 1) / kXcds;
        const bool live = p < per_live;
        l = live ? x * per_live + p : x * per_idle + p - per_live;
        if (l >= total[live ? 0 : 1] || (!live && p - per_live >= per_idle)) return;
        int b0 = 0, mine, at;
        while (true) {                                       // the sample of unit l
            if (b0 >= B) return;
            mine = units(b0 + lane, live);
            at = mine;
#pragma unroll
            for (int w = 1; w < 64; w <<= 1) {
                const int o = __shfl_up(at, w, 64);
                if (lane >= w) at += o;
            }
            const int all = __shfl(at, 63, 64);
            if (l < all) break;
            l -= all;
            b0 += 64;
        }
        const int who = __ffsll((unsigned long long)__ballot(l < at)) - 1;
        l -= __shfl(at - mine, who, 64);
        const CrossCount n = a.item_counts[b0 + who];
        const int per = live ? n.live * a.split : n.idle;
        const int hk = l / per, rest = l - hk * per;
        z = live ? rest / n.live : 0;
        item = live ? rest - z * n.live : n.live + rest;
        bhk = (b0 + who) * a.Hk + hk;
        bhk = __builtin_amdgcn_readfirstlane(bhk);
        z = __builtin_amdgcn_readfirstlane(z);
        item = __builtin_amdgcn_readfirstlane(item);
    }
    const CrossKeys &keys = a.items[(size_t)(bhk / a.Hk) * a.max_items + item];
    const int key_start = __builtin_amdgcn_readfirstlane(keys.start), key_len = __builtin_amdgcn_readfirstlane(keys.len);
    const size_t head = (size_t)bhk * a.M + key_start;
    auto store = [&](int kr, int col, const f32x4 &k4, const f32x4 &v4) {
        if (a.split == 1) {
            Io<bf16_t>::store4(static_cast<bf16_t *>(a.dk) + (head + kr) * D + col, k4[0], k4[1], k4[2], k4[3]);
            Io<bf16_t>::store4(static_cast<bf16_t *>(a.dv) + (head + kr) * D + col, v4[0], v4[1], v4[2], v4[3]);
        } else {
            float *p = a.kpart + ((size_t)z * a.BHk * a.M + head + kr) * 2 * D + col;
            *reinterpret_cast<f32x4 *>(p) = k4;
            *reinterpret_cast<f32x4 *>(p + D) = v4;
        }
    };
    PieceSource src(a, keys);
    int per_copy = 0;
    for (int s = src.next_segment(0); s < a.n_seg; s = src.next_segment(src.piece_end(s))) per_copy += src.stages_of(s);
    const long long total = (long long)per_copy * a.copies;
    const int s0 = (int)(total * z / a.split), n_st = (int)(total * (z + 1) / a.split) - s0;
    if (n_st == 0) {
        const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
        for (; z < a.split; z = per_copy ? a.split : z + 1)      // (a tile without segments is one item for all parts)
        for (int i = threadIdx.x; i < key_len * (D / 4); i += 256) store(i / (D / 4), i % (D / 4) * 4, zero, zero);
        return;
    }
    src.copy = s0 / per_copy;
    int skip = s0 - src.copy * per_copy;
    src.seg = src.next_segment(0);
    while (skip >= src.stages_of(src.seg)) {
        skip -= src.stages_of(src.seg);
        src.seg = src.next_segment(src.piece_end(src.seg));
    }
    const size_t rows = (size_t)bhk * a.copies * a.N;
    src.records = reinterpret_cast<const char *>(a.stats) + rows * 16;
    src.inf_rec = reinterpret_cast<const char *>(a.stats) + (size_t)a.rows * 16;
    src.stages = n_st;
    src.enter(skip);
    src.q_start = src.first;
    src.q_len = src.rec_left;
    src.n_direct = (src.q_len + R - 1) / R;
    const char *const qbase = static_cast<const char *>(uniform_ptr(static_cast<const char *>(a.q) + rows * RB));
    const char *const dobase = static_cast<const char *>(uniform_ptr(static_cast<const char *>(a.d_o) + rows * RB));
    const size_t states = (size_t)bhk * a.M * RB;
    dkdv_wide<BIG>(smem, src, n_st, qbase, dobase, static_cast<const char *>(a.k) + states, static_cast<const char *>(a.v) + states, key_start,
                   key_len, a.scale, a.scale_log2, store);
}

void launch_cross_dkdv_wide(const CrossArgs &a, hipStream_t st) {
    MOC_PROF("cross_dkdv_wide", st);
    const int grid = xcd_grid((long long)a.max_items * a.BHk * a.split) + 2 * kXcds;      // (each kind rounds its slices up)
    if ((long long)a.copies * a.N * wide::RB >= (1ll << 32)) cross_dkdv_wide_kernel<true><<<grid, 256, 0, st>>>(a);
    else cross_dkdv_wide_kernel<false><<<grid, 256, 0, st>>>(a);
}

}  // namespace moc
