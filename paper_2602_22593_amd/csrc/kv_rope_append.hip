// kv_rope_append: the new tokens' queries and keys are rotated by their positions, the queries go to an array, keys and values
// into the pool under a layout view.
//
// With frequencies f_0 .. f_{R/2 - 1} and an axis for each, the pair (x, y) of number i becomes (x cos a - y sin a, y cos a + x sin a),
// a = position on axis(i) * f_i.  Elements from R on pass as they are, and so do the values.
//
// Bound by reading and writing every row once: 17000 tokens of 32 query and 8 KV heads of 128, 420 MB, take 81 us (5.2 TB/s; a
// byte-for-byte copy of as much takes 67).  Stores past the caches: 8 prompts of 500 to 1000 tokens 23 us in place of 28, 2 of 3000 to
// 4000 29 in place of 38 (whoever reads the rows next does so through another die's L2).  A workgroup takes one or two tokens: their cosines and sines go into LDS once and serve all heads; then every
// lane moves items of two 16-byte pieces, the two halves of eight pairs, so that a rotation needs nothing of another
// lane.  D / 16 items a head, consecutive lanes on consecutive pieces.  Small workgroups with one item a lane at a time hide the
// chain before the rows (lengths, positions, cosines) behind each other: eight tokens and four items 105 us, four and two 91; rows
// requested before that chain, two or three items a lane, 86 to 94.
#include "kv_internal.h"

#include "decode_common.h"

using namespace kvdec;

namespace {

constexpr int kThreads = 256;
constexpr int kMostTokens = 2;    // per workgroup
constexpr int kMostPairs = 128;   // of a head

struct rope_args {
    const uint16_t *q, *k, *v_new;
    int64_t q_stride, k_stride, v_stride;   // elements between tokens
    uint16_t* out;                          // [total][n_q_local][D]
    uint16_t* pool;
    int64_t n_pool_blocks;
    const int32_t* positions;               // [axes][position_stride]
    int64_t position_stride;
    const float* inv_freq;
    const int32_t* table;
    int64_t table_stride;
    const int32_t *ctx_lens, *q_off;
    int32_t* token_pos;                     // [batch][n_kv_local][token_pos_stride] or null
    int64_t token_pos_stride;
    int64_t total;
    kv_view_dev v;
    int32_t batch, pairs, adjacent, tokens;
    uint32_t axis[kMostPairs / 16];         // two bits a pair
    float* weights;                         // [batch][n_kv_local][weights_stride], where the kernel has them
    int64_t weights_stride;
};

// The sequence whose rows hold row i, or -1: the last one that starts at or before it, 64 probes at a time (all lanes alike).
__device__ __forceinline__ int row_sequence(const rope_args& a, int64_t i, int lane)
{
    int s = 0;
    for (int span = a.batch; span > 1;) {
        const int step = (span + 63) >> 6, probe = lane * step;
        const bool ok = probe < span && a.q_off[s + min(probe, span - 1)] <= i;
        const unsigned long long which = __builtin_amdgcn_ballot_w64(ok);
        const int c = which ? 63 - __builtin_clzll(which) : 0;
        s += c * step;
        span = min(step, span - c * step);
    }
    s = __builtin_amdgcn_readfirstlane(s);
    return a.q_off[s] <= i && i < a.q_off[s + 1] ? s : -1;
}

// WEIGHTS: also clears the weights of the tokens written (a kernel of its own: the chain before the rows grows by it, 80.3 us for the prompts
// above become 82.0).
template <bool WEIGHTS>
__global__ __launch_bounds__(kThreads) void kv_rope_append_kernel(rope_args a)
{
    __shared__ float2 s_turn[kMostTokens][kMostPairs];
    __shared__ int64_t s_place[kMostTokens];   // of the token's row in the pool, -1: none, -2: not a token
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const kv_view_dev& v = a.v;
    const int64_t i0 = (int64_t)blockIdx.x * a.tokens;
    const int n = (int)min((int64_t)a.tokens, a.total - i0);
    for (int x = wave; x < n; x += kThreads / 64) {
        const int64_t i = i0 + x;
        int s = (int)i, j = 0, q_len = 1;
        if (a.q_off) {
            s = row_sequence(a, i, lane);
            if (s >= 0) {
                j = (int)(i - a.q_off[s]);
                q_len = a.q_off[s + 1] - a.q_off[s];
            }
        }
        int64_t place = -2;
        if (s >= 0) {
            const int t = a.ctx_lens[s] - q_len + j;
            int b, slot;
            kv_split_token(v, max(t, 0), b, slot);
            place = -1;
            if (t >= 0 && b < a.table_stride) {
                const int32_t id = a.table[(int64_t)s * a.table_stride + b];
                if (id >= 0 && id < a.n_pool_blocks) place = (int64_t)id * v.block_elems + (int64_t)slot * v.token_stride + v.head_off;
                if (place >= 0 && a.token_pos && t < a.token_pos_stride)
                    for (int h = lane; h < v.n_kv_local; h += 64)
                        a.token_pos[((int64_t)s * v.n_kv_local + h) * a.token_pos_stride + t] = a.positions[i];
                if (WEIGHTS && place >= 0 && t < a.weights_stride)
                    for (int h = lane; h < v.n_kv_local; h += 64) a.weights[((int64_t)s * v.n_kv_local + h) * a.weights_stride + t] = 0.f;
            }
        }
        if (lane == 0) s_place[x] = place;
    }
    // An angle may be many thousand turns: its fraction of a turn is taken in 64 bits, where a position of 31 bits and a frequency of
    // 24 leave an error of 2^-22 turns at most; from there 32 bits do.
    for (int x = tid; x < n * a.pairs; x += kThreads) {
        const int j = x / a.pairs, f = x - j * a.pairs;
        const int axis = (a.axis[f >> 4] >> (2 * (f & 15))) & 3;
        const double turns = (double)a.positions[axis * a.position_stride + i0 + j] * (double)a.inv_freq[f] * 0.15915494309189533577;
        const float part = (float)(turns - rint(turns));
        float sn, cs;
        sincospif(2.f * part, &sn, &cs);
        s_turn[j][f] = make_float2(cs, sn);
    }
    __syncthreads();

    const int per_head = v.head_dim >> 4, heads = v.n_q_local + 2 * v.n_kv_local, per_token = heads * per_head;
    const int rotated = a.pairs >> 3;   // items of a head that turn
    const int items = n * per_token;
    for (int x = tid; x < items; x += kThreads) {
        const int j = x / per_token, y = x - j * per_token, h = y / per_head, c = y - h * per_head;
        const int64_t place = s_place[j], i = i0 + j;
        const bool query = h < v.n_q_local, value = h >= v.n_q_local + v.n_kv_local;
        if (place == -2 || (!query && place < 0)) continue;
        const bool turns = !value && c < rotated, halves = turns && !a.adjacent;
        const int at = halves ? 8 * c : 16 * c, apart = halves ? a.pairs : 8;   // of the item's two pieces
        const int hk = value ? h - v.n_q_local - v.n_kv_local : h - v.n_q_local;
        const uint16_t* src = (query ? a.q + i * a.q_stride + h * v.head_dim : (value ? a.v_new + i * a.v_stride : a.k + i * a.k_stride) + hk * v.head_dim) + at;
        uint16_t* to = (query ? a.out + (i * v.n_q_local + h) * v.head_dim : a.pool + place + (value ? v.plane_elems : 0) + hk * v.head_dim) + at;
        kv_u32x4 lo = *reinterpret_cast<const kv_u32x4*>(src), hi = *reinterpret_cast<const kv_u32x4*>(src + apart);
        if (turns) {
            const float2* turn = &s_turn[j][8 * c];
            if (a.adjacent) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 t = turn[e], t2 = turn[4 + e];
                    const float xa = bf16_lo(lo[e]), ya = bf16_hi(lo[e]), xb = bf16_lo(hi[e]), yb = bf16_hi(hi[e]);
                    lo[e] = pack_bf16x2(xa * t.x - ya * t.y, ya * t.x + xa * t.y);
                    hi[e] = pack_bf16x2(xb * t2.x - yb * t2.y, yb * t2.x + xb * t2.y);
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 t = turn[2 * e], t2 = turn[2 * e + 1];
                    const float xa = bf16_lo(lo[e]), xb = bf16_hi(lo[e]), ya = bf16_lo(hi[e]), yb = bf16_hi(hi[e]);
                    lo[e] = pack_bf16x2(xa * t.x - ya * t.y, xb * t2.x - yb * t2.y);
                    hi[e] = pack_bf16x2(ya * t.x + xa * t.y, yb * t2.x + xb * t2.y);
                }
            }
        }
        __builtin_nontemporal_store(lo, reinterpret_cast<kv_u32x4*>(to));
        __builtin_nontemporal_store(hi, reinterpret_cast<kv_u32x4*>(to + apart));
    }
}

bool strided_ok(const void* p, int64_t stride, int64_t row) { return !((uintptr_t)p & 15u) && stride % 8 == 0 && stride >= row; }

}  // namespace

extern "C" int kv_rope_append(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const void* q, int64_t q_stride,
                              const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                              const int32_t* positions, int64_t position_stride, int n_axes, const float* inv_freq,
                              int rotary_dim, const int32_t* axis_of_pair, int pairs, const int32_t* block_table,
                              int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets, int batch,
                              int64_t total, int32_t* token_pos, int64_t token_pos_stride, void* hip_stream)
{
    return kv_rope_append_tracked(kv_pool, n_pool_blocks, view, q, q_stride, k, k_stride, v, v_stride, q_out, positions, position_stride, n_axes,
                                  inv_freq, rotary_dim, axis_of_pair, pairs, block_table, block_table_stride, ctx_lens, q_offsets, batch, total,
                                  token_pos, token_pos_stride, nullptr, 0, hip_stream);
}

extern "C" int kv_rope_append_tracked(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const void* q, int64_t q_stride,
                                      const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                      const int32_t* positions, int64_t position_stride, int n_axes, const float* inv_freq,
                                      int rotary_dim, const int32_t* axis_of_pair, int pairs, const int32_t* block_table,
                                      int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets, int batch,
                                      int64_t total, int32_t* token_pos, int64_t token_pos_stride, float* weights,
                                      int64_t weights_stride, void* hip_stream)
{
    if (!kv_view_ok(view) || n_pool_blocks < 0 || block_table_stride < 0 || batch < 0 || total < 0 || rotary_dim < 0 ||
        position_stride < 0 || token_pos_stride < 0 || weights_stride < 0 || (pairs != KV_ROPE_HALVES && pairs != KV_ROPE_ADJACENT) || n_axes < 1)
        return KV_ERR_INVALID_ARG;
    const int d = view->geom.head_dim, half = rotary_dim / 2;
    if (rotary_dim > d || position_stride < total || (!q_offsets && total != batch)) return KV_ERR_INVALID_ARG;
    if (axis_of_pair)
        for (int i = 0; i < half; ++i)
            if (axis_of_pair[i] < 0 || axis_of_pair[i] >= n_axes) return KV_ERR_INVALID_ARG;
    if (batch == 0 || total == 0) return KV_OK;
    if (!kv_pool || !q || !k || !v || !q_out || !positions || (half && !inv_freq) || !block_table || !ctx_lens) return KV_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)view->n_q_local * d, k_row = (int64_t)view->n_kv_local * d;
    if (q_stride < q_row || k_stride < k_row || v_stride < k_row || (q_out == q && q_stride != q_row)) return KV_ERR_INVALID_ARG;
    if (d % 16 != 0 || rotary_dim % 16 != 0 || half > kMostPairs || n_axes > 4) return KV_ERR_UNSUPPORTED;
    if (!strided_ok(q, q_stride, q_row) || !strided_ok(k, k_stride, k_row) || !strided_ok(v, v_stride, k_row) || ((uintptr_t)q_out & 15u) ||
        ((uintptr_t)kv_pool & 15u))
        return KV_ERR_UNSUPPORTED;
    rope_args a = {};
    a.q = (const uint16_t*)q;
    a.k = (const uint16_t*)k;
    a.v_new = (const uint16_t*)v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out = (uint16_t*)q_out;
    a.pool = (uint16_t*)kv_pool;
    a.n_pool_blocks = n_pool_blocks;
    a.positions = positions;
    a.position_stride = position_stride;
    a.inv_freq = inv_freq;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.q_off = q_offsets;
    a.token_pos = token_pos;
    a.token_pos_stride = token_pos_stride;
    a.weights = weights;
    a.weights_stride = weights_stride;
    a.total = total;
    a.v = kv_view_to_dev(view);
    a.batch = batch;
    a.pairs = half;
    a.adjacent = pairs == KV_ROPE_ADJACENT;
    for (int i = 0; i < half; ++i) a.axis[i >> 4] |= (uint32_t)(axis_of_pair ? axis_of_pair[i] : 0) << (2 * (i & 15));
    int64_t tokens = total / 1024;   // workgroups for four rounds of the chip before a workgroup takes several tokens
    a.tokens = (int32_t)(tokens < 1 ? 1 : tokens > kMostTokens ? kMostTokens : tokens);
    const int64_t grid = (total + a.tokens - 1) / a.tokens;
    if (grid > 0x7fffffff) return KV_ERR_UNSUPPORTED;
    if (weights) hipLaunchKernelGGL(kv_rope_append_kernel<true>, dim3((unsigned)grid), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL(kv_rope_append_kernel<false>, dim3((unsigned)grid), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return kv_record_hip_error(hipGetLastError(), "kv_rope_append launch");
}
