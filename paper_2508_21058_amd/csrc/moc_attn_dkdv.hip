// dK / dV of whole key tiles (256 keys of one chunk, or its last 160 to 255), heads of 128 features: the key-stationary pass for calls with
// many of them. The ragged rest of such calls, heads of 64 features and small calls take attn_bwd_dkdv_pipe_kernel.
//
// A workgroup is four waves, one per SIMD with all 512 of its registers: a wave owns 64 keys, holds their dK^T and dV^T
// (the 256 accumulation registers) and the operands of K (64 vector registers), and streams every query that attends
// them past, 16 at a time. P and dS never leave the wave: the scores are formed as 16 x 16 blocks (queries x keys), whose
// accumulators become operands of the gradient products by exchanging half of their words with the lanes 16 away. Against
// two roles of waves of 32 keys (the other kernel) a tile row is read from LDS once per 64 keys instead of 32, nothing waits for
// another wave's P, and a chunk's queries are fetched once per 256 keys instead of 128. dK/dV of 24 heads, the other kernel
// alone / with this one: 181,760 tokens, 1,280- to 10,240-key chunks 154.4 / 140.5 ms (1,120 -> 1,230 TFLOP/s), 114k tokens,
// 260-key chunks (whose last four keys stay with the other kernel) 17.05 / 16.22, 33k tokens 3.20 / 3.04, six heads of 457k
// tokens in 130-key chunks (captions only) 36.6 / 34.6.
//
// What bounds it is that a SIMD has one wave to issue from, an instruction every four cycles at best: 16 queries against 64
// keys are 1,024 cycles of the matrix pipe and 225 instructions (900 cycles of issue), 48 of them its own, and take 1,550. On
// 181,760 tokens it issues 56 % of its cycles, has an instruction that the pipe or its operands hold back 32 % and waits for copies
// or a barrier 12 %; the matrix pipe is busy 66 % (63 % on 114k tokens of 260-key chunks, whose items are shorter). Hence the step
// is written out in slots, and what is issued in the shadow of which product matters: scheduling left to the compiler within a slot
// 13 % slower; LDS reads behind the 16-cycle score products instead of the 32-cycle gradient product 3 %; a barrier every 16 queries
// instead of every 32 1 %. Without the exponentials a timing-only build takes 5 % less, without the reads of V 6 %.
#include "moc_attn_bwd.h"
#include "moc_dkdv_wide.h"

namespace moc {

namespace wide {
// The window's queries in their order, then the chunk's list.
struct ListSource {
    int n_direct, q_start, q_len;
    const char *rec_ptr, *rec_list, *inf_rec;
    int rec_left, rec_more;
    __device__ __forceinline__ void issue(uint32_t dst, uint32_t rec_off, int rec_row, int rec_sel) {
        if (rec_left >= R) {
            copy4(rec_ptr, rec_off, dst);
        } else {
            if (rec_left <= 0 && rec_more > 0) { rec_ptr = rec_list; rec_left = rec_more; rec_more = 0; }
            // (past the last stage rec_left - 1 is negative and leads back to the last record)
            const char *const at = rec_ptr + (min(rec_row, rec_left - 1) * 16 + rec_sel);
            copy4(rec_row >= rec_left && rec_sel == 0 ? inf_rec : at, dst);
        }
        rec_ptr += RECB;
        rec_left -= R;
    }
};
}  // namespace wide

// OT: storage type of dK and dV. BIG: rows beyond the reach of 32-bit byte offsets
template <typename OT, bool BIG>
__global__ __launch_bounds__(256, 1) void attn_bwd_dkdv_wide_kernel(KvArgs a) {
    using namespace wide;
    __shared__ __attribute__((aligned(1024))) char smem[LDS];     // stages; records; V
    int bh, item_no;
    if (!kv_item(a.n_items, a.n_text, a.BH, bh, item_no)) return;
    // scalars before any address is made of them (see TileIter::start)
    bh = __builtin_amdgcn_readfirstlane(bh);
    item_no = __builtin_amdgcn_readfirstlane(item_no);
    const bool caption = item_no < a.n_text;
    KvItem item = a.items[caption ? item_no + item_no / a.text_tiles * (a.join - 1) * a.text_tiles : item_no - a.n_text + a.video_at];
    if (caption) item.q_len = min(a.text_seg, a.N - item.q_start);
    const int N = a.N;

    const bool routed = item.chunk >= 0 && a.topk > 0;
    const int32_t *loff = a.list_off + (size_t)bh * (a.C + 1);
    const int lbeg = __builtin_amdgcn_readfirstlane(routed ? loff[item.chunk] : 0);
    const int n_list = __builtin_amdgcn_readfirstlane(routed ? loff[item.chunk + 1] : 0) - lbeg;
    const int n_win = (item.q_len + R - 1) / R;                   // stages of the window's queries; the list's follow
    const int n_st = n_win + (n_list + R - 1) / R;
    if (n_st == 0) return;

    ListSource src;
    src.n_direct = n_win;
    src.q_start = item.q_start;
    src.q_len = item.q_len;
    src.inf_rec = reinterpret_cast<const char *>(a.stats2) + (size_t)a.BH * N * 16;
    src.rec_ptr = reinterpret_cast<const char *>(a.stats2) + ((size_t)bh * N + item.q_start) * 16;
    src.rec_list = reinterpret_cast<const char *>(a.gstats2) + ((size_t)bh * N * a.topk + lbeg) * 16;
    src.rec_left = item.q_len;
    src.rec_more = n_list;
    const size_t head = (size_t)bh * N * RB;
    const char *const qbase = static_cast<const char *>(uniform_ptr(static_cast<const char *>(a.q) + head));
    const char *const dobase = static_cast<const char *>(uniform_ptr(static_cast<const char *>(a.d_o) + head));
    dkdv_wide<BIG>(smem, src, n_st, qbase, dobase, static_cast<const char *>(a.k) + head, static_cast<const char *>(a.v) + head, item.key_start,
                   item.key_len, a.scale, a.scale_log2, [&](int kr, int col, const f32x4 &k4, const f32x4 &v4) {
        if (item.partial < 0) {
            const size_t row = ((size_t)bh * N + item.key_start + kr) * D + col;
            Io<OT>::store4(static_cast<OT *>(a.dk) + row, k4[0], k4[1], k4[2], k4[3]);
            Io<OT>::store4(static_cast<OT *>(a.dv) + row, v4[0], v4[1], v4[2], v4[3]);
        } else {
            const size_t row = (((size_t)bh * a.n_partials + item.partial) * a.key_tile + kr) * D + col;
            *reinterpret_cast<f32x4 *>(a.tpart_k + row) = k4;
            *reinterpret_cast<f32x4 *>(a.tpart_v + row) = v4;
        }
    });
}

hipError_t launch_dkdv_wide(const KvArgs &kv, int dtype, hipStream_t st) {
    const dim3 grid(kv_grid(kv.n_items, kv.n_text, kv.BH)), block(256);
    const bool big = (long long)kv.N * wide::RB >= (1ll << 32);
    if (dtype == MOC_BF16) {
        if (big) attn_bwd_dkdv_wide_kernel<bf16_t, true><<<grid, block, 0, st>>>(kv);
        else attn_bwd_dkdv_wide_kernel<bf16_t, false><<<grid, block, 0, st>>>(kv);
    } else {
        if (big) attn_bwd_dkdv_wide_kernel<float, true><<<grid, block, 0, st>>>(kv);
        else attn_bwd_dkdv_wide_kernel<float, false><<<grid, block, 0, st>>>(kv);
    }
    return hipGetLastError();
}

}  // namespace moc
