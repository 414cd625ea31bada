// kv_repack_q8: codes and scales moved between two layouts of an 8-bit cache, byte for byte.  A group of B_base tokens of a head is the
// same in every layout and has one scale, so nothing is rounded.
//
// Bound by reading and writing what moves.  As in kv_repack, a token's rows for a run of consecutive heads are contiguous in every
// arrangement: the unit is a 16-byte piece of such a run, consecutive lanes on consecutive pieces.  A workgroup moves 8 KiB, or one group of
// B_base tokens where that is more (from 3 common heads of 128 and B_base = 16 on), two pieces a lane or 8 KiB at a time: they are requested
// before the first of them is stored.  With 64 KiB and four pieces at a time, moving 128 sequences around 4096 tokens from DP to TP4 (2 common
// heads: 8 KiB) took 114 us, with 16 KiB 106, now 104 (4.8 TB/s; runs of 256 bytes are read), and one sequence 8.2 us, now 5.6 (its launch).
// Larger groups lose nothing by their rounds: 4 and 8 common heads, 32 KiB a group, 5.0 TB/s, and B_base = 64, 128 KiB, 5.1.
#include "kv_q8.h"

using namespace kvq8;

namespace {

constexpr int kThreads = 256;
constexpr int kUnroll = 2;
constexpr int kPayload = 8 * 1024;

struct repack_args {
    uint8_t* pool;
    float* scales;
    const int32_t *src_table, *dst_table;
    int64_t src_stride, dst_stride;
    const int32_t* n_tokens;
    kv_view_dev src, dst;
    q8_view sx, dx;
    int32_t src_head, dst_head;   // of the first common head, among those exposed
    int32_t heads;                // common ones
    int32_t run_chunks;           // 16-byte pieces in one token's run of them (one plane)
    int32_t run_shift;            // log2 or -1
    int32_t tokens_per_wg;        // a multiple of B_base
};

__device__ __forceinline__ int64_t block_of(const kv_view_dev& v, const int32_t* __restrict__ row, int t, int& slot)
{
    int j;
    kv_split_token(v, t, j, slot);
    return row[j];
}

__global__ __launch_bounds__(kThreads) void repack_kernel(repack_args a)
{
    const int s = blockIdx.y, n = a.n_tokens[s], t0 = blockIdx.x * a.tokens_per_wg;
    if (t0 >= n) return;
    const int t1 = min(n, t0 + a.tokens_per_wg);
    const int32_t* srow = a.src_table + (int64_t)s * a.src_stride;
    const int32_t* drow = a.dst_table + (int64_t)s * a.dst_stride;
    // scales: of every group that has a token
    const int B = a.sx.base_tokens, groups = (t1 - t0 + B - 1) / B, per_group = 2 * a.heads;
    float scale = 0.f;
    int64_t scale_to = 0;
    auto load_scale = [&](int i) {
        const int g = i / per_group, rem = i - g * per_group, plane = rem / a.heads, h = rem - plane * a.heads;
        int from, to;
        const int64_t sb = block_of(a.src, srow, t0 + g * B, from), db = block_of(a.dst, drow, t0 + g * B, to);
        scale = a.scales[q8_scale_at(a.sx, sb, from, a.src_head + h) + plane * (a.sx.block_scales / 2)];
        scale_to = q8_scale_at(a.dx, db, to, a.dst_head + h) + plane * (a.dx.block_scales / 2);
    };
    const int n_scales = groups * per_group;
    if ((int)threadIdx.x < n_scales) load_scale(threadIdx.x);   // (stored after the codes)
    const int per_tok = 2 * a.run_chunks, total = (t1 - t0) * per_tok;
    const int64_t s_off = a.src.head_off + a.src_head * a.src.head_dim, d_off = a.dst.head_off + a.dst_head * a.dst.head_dim;
    for (int base = threadIdx.x; base < total; base += kThreads * kUnroll) {
        kv_u32x4 val[kUnroll];
        int64_t to[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int idx = base + u * kThreads;
            to[u] = -1;
            if (idx < total) {
                int tt, plane, c;
                if (a.run_shift >= 0) {
                    tt = idx >> (a.run_shift + 1);
                    const int rem = idx & (per_tok - 1);
                    plane = rem >> a.run_shift;
                    c = rem & (a.run_chunks - 1);
                } else {
                    tt = idx / per_tok;
                    const int rem = idx - tt * per_tok;
                    plane = rem / a.run_chunks;
                    c = rem - plane * a.run_chunks;
                }
                int from_slot, to_slot;
                const int64_t sb = block_of(a.src, srow, t0 + tt, from_slot), db = block_of(a.dst, drow, t0 + tt, to_slot);
                const int64_t from = sb * a.src.block_elems + (int64_t)from_slot * a.src.token_stride + plane * a.src.plane_elems + s_off + c * 16;
                to[u] = db * a.dst.block_elems + (int64_t)to_slot * a.dst.token_stride + plane * a.dst.plane_elems + d_off + c * 16;
                val[u] = __builtin_nontemporal_load(reinterpret_cast<const kv_u32x4*>(a.pool + from));
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (to[u] >= 0) __builtin_nontemporal_store(val[u], reinterpret_cast<kv_u32x4*>(a.pool + to[u]));
    }
    for (int i = threadIdx.x; i < n_scales; i += kThreads) {
        if (i >= kThreads) load_scale(i);
        a.scales[scale_to] = scale;
    }
}

}  // namespace

extern "C" int kv_repack_q8(void* kv_pool, float* scales, int64_t n_pool_blocks, const kv_view* src_view, const kv_view* dst_view,
                            const int32_t* src_block_table, int64_t src_stride, const int32_t* dst_block_table, int64_t dst_stride,
                            const int32_t* n_tokens, int n_seqs, int max_tokens, void* hip_stream)
{
    if (!kv_view_ok(src_view) || !kv_view_ok(dst_view)) return KV_ERR_INVALID_ARG;
    const kv_geometry &g = src_view->geom, &o = dst_view->geom;
    if (g.n_q_heads != o.n_q_heads || g.n_kv_heads != o.n_kv_heads || g.head_dim != o.head_dim || g.base_block_size != o.base_block_size)
        return KV_ERR_INVALID_ARG;
    if (n_seqs < 0 || max_tokens < 0 || n_pool_blocks < 0 || src_stride < 0 || dst_stride < 0) return KV_ERR_INVALID_ARG;
    if (n_seqs == 0 || max_tokens == 0) return KV_OK;
    if (!kv_pool || !scales || !src_block_table || !dst_block_table || !n_tokens) return KV_ERR_INVALID_ARG;
    const int64_t need_src = ((int64_t)max_tokens + src_view->block_tokens - 1) / src_view->block_tokens;
    const int64_t need_dst = ((int64_t)max_tokens + dst_view->block_tokens - 1) / dst_view->block_tokens;
    if (src_stride < need_src || dst_stride < need_dst) return KV_ERR_INVALID_ARG;
    if (g.head_dim % 16 != 0 || g.base_block_size % 16 != 0 || !kv_aligned(kv_pool, 16) || !kv_aligned(scales, 4)) return KV_ERR_UNSUPPORTED;

    // heads exposed by both views
    const int lo = src_view->kv_head0 > dst_view->kv_head0 ? src_view->kv_head0 : dst_view->kv_head0;
    const int s_hi = src_view->kv_head0 + src_view->n_kv_local, d_hi = dst_view->kv_head0 + dst_view->n_kv_local;
    const int hi = s_hi < d_hi ? s_hi : d_hi;
    if (hi <= lo) return KV_OK;   // nothing in common: nothing moves
    repack_args a = {};
    a.pool = (uint8_t*)kv_pool;
    a.scales = scales;
    a.src_table = src_block_table;
    a.dst_table = dst_block_table;
    a.src_stride = src_stride;
    a.dst_stride = dst_stride;
    a.n_tokens = n_tokens;
    a.src = kv_view_to_dev(src_view);
    a.dst = kv_view_to_dev(dst_view);
    a.sx = q8_view_of(src_view);
    a.dx = q8_view_of(dst_view);
    a.src_head = lo - src_view->kv_head0;
    a.dst_head = lo - dst_view->kv_head0;
    a.heads = hi - lo;
    a.run_chunks = a.heads * g.head_dim / 16;
    a.run_shift = -1;
    for (int s = 0; s < 31; ++s)
        if ((1 << s) == a.run_chunks) a.run_shift = s;
    // about kPayload bytes per workgroup, whole groups: one at least, however long a token's run is
    const int B = g.base_block_size;
    int tokens = kPayload / (2 * a.run_chunks * 16);
    tokens = tokens < 1 ? B : (tokens + B - 1) / B * B;
    a.tokens_per_wg = tokens;
    const int64_t gx = ((int64_t)max_tokens + tokens - 1) / tokens;
    if (gx > 0x7fffffff || n_seqs > 65535) return KV_ERR_INVALID_ARG;
    hipLaunchKernelGGL(repack_kernel, dim3((unsigned)gx, (unsigned)n_seqs), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return kv_record_hip_error(hipGetLastError(), "kv_repack_q8 launch");
}
