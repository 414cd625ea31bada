// kv_rope_append_q8: the new tokens' queries and keys are rotated by their positions, the queries go to an array, keys and values
// into a pool of 8-bit codes under a layout view, with a scale for every B_base tokens of a head (a group).
//
// A group's scale s is the smallest power of two with max |x| <= s times the largest code, over the new tokens in it, and no smaller than
// before where the group holds older tokens; x / s goes to the nearest code.  Where the scale grows, the older codes are divided by the
// same power and rounded again: exact for e4m3 (but for what falls below its normal range), off by half a step for int8, a step in all
// since the steps at least double.  A number that is not finite makes the scale NaN, and with it what the group's head reads as.
// Powers of two cost int8 half a bit on average, e4m3 nothing, and values are exact in bf16.
// Keys are rotated in fp32 and rounded once, from there to 8 bits.
// Bound by reading the rows and writing queries and codes: 8 prompts of 300 to 4000 tokens, 32 heads on 8, 70 us (372 MB, 5.3 TB/s); one token of
// 128 sequences, keys and values of 8 heads, 4 us, a chain of trips to memory.
#include "kv_q8.h"

using namespace kvq8;

namespace {

constexpr int kThreads = 256;
constexpr int kMostPairs = 64;    // of a head
constexpr int kMostBase = 128;    // tokens of a group
constexpr int kMostQueries = 16;  // tokens of a workgroup that rotates queries

struct append_args {
    const uint16_t *q, *k, *v_new;
    int64_t q_stride, k_stride, v_stride;   // elements between tokens
    uint16_t* out;                          // [total][n_q_local][D]
    uint8_t* pool;
    float* scales;
    int64_t n_pool_blocks;
    const int32_t* positions;               // [axes][position_stride]
    int64_t position_stride;
    const float* inv_freq;
    const int32_t* table;
    int64_t table_stride;
    const int32_t *ctx_lens, *q_off;
    int64_t total;
    kv_view_dev v;
    q8_view x;
    int32_t batch, pairs, adjacent, heads_q;   // heads_q: query heads to rotate, 0 where there are no queries
    int32_t parts;                             // workgroups that share a group's heads
    int32_t query_tokens;                      // of a workgroup that rotates queries: a row for D / 16 lanes
    uint32_t slots;                            // groups at most, see first_slot()
    uint32_t axis[kMostPairs / 16];            // two bits a pair
};

// Cosine and sine of pair f of row i, in 64 bits and rounded once: a key's code depends on which side of a boundary its value falls, and
// sines that are two steps of fp32 off put half as many codes again on the wrong one.  The angle as a fraction r of a turn from the nearest quarter,
// |r| <= 1/8, then the Taylor series: the first terms left out are (pi / 4)^13 / 13! = 7e-12 and (pi / 4)^14 / 14! = 4e-13.
__device__ __forceinline__ float2 turn_of(const append_args& a, int64_t i, int f)
{
    const int axis = (a.axis[f >> 4] >> (2 * (f & 15))) & 3;
    const double turns = (double)a.positions[axis * a.position_stride + i] * (double)a.inv_freq[f] * 0.15915494309189533577;
    const double quarters = rint(4. * (turns - rint(turns)));
    const double x = (turns - rint(turns) - 0.25 * quarters) * 6.28318530717958647693, y = x * x;
    const double sn = x + x * y * (-1. / 6 + y * (1. / 120 + y * (-1. / 5040 + y * (1. / 362880 - y * (1. / 39916800)))));
    const double cs = 1. + y * (-0.5 + y * (1. / 24 + y * (-1. / 720 + y * (1. / 40320 + y * (-1. / 3628800 + y * (1. / 479001600))))));
    const int k = (int)quarters;
    const float c = (float)((k & 1) ? sn : cs), s = (float)((k & 1) ? cs : sn);
    return make_float2(((k + 1) & 2) ? -c : c, (k & 2) ? -s : s);
}

// A lane's sixteen elements of a row are two pieces of eight, the two halves of eight pairs where the row is rotated by halves, so that
// a rotation needs nothing of another lane.  Where they start, and how far apart they lie:
struct pieces {
    int at, apart;
    bool turns;
};
__device__ __forceinline__ pieces pieces_of(const append_args& a, int c, bool rotated)
{
    const bool turns = rotated && 8 * c < a.pairs, halves = turns && !a.adjacent;
    return {halves ? 8 * c : 16 * c, halves ? a.pairs : 8, turns};
}
__device__ __forceinline__ void load_row(const uint16_t* row, const pieces& p, const float2* turn, bool adjacent, float (&x)[16])
{
    const kv_u32x4 lo = *reinterpret_cast<const kv_u32x4*>(row + p.at), hi = *reinterpret_cast<const kv_u32x4*>(row + p.at + p.apart);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[2 * e] = bf16_lo(lo[e]);
        x[2 * e + 1] = bf16_hi(lo[e]);
        x[8 + 2 * e] = bf16_lo(hi[e]);
        x[9 + 2 * e] = bf16_hi(hi[e]);
    }
    if (!p.turns) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma clang fp contract(off)
        const int i = adjacent ? 2 * e : e, j = adjacent ? 2 * e + 1 : 8 + e;
        const float2 t = turn[e];
        const float u = x[i], w = x[j];
        x[i] = u * t.x - w * t.y;
        x[j] = w * t.x + u * t.y;
    }
}
__device__ __forceinline__ void store_bf16(uint16_t* row, const pieces& p, const float (&x)[16])
{
    kv_u32x4 lo, hi;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lo[e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
        hi[e] = pack_bf16x2(x[8 + 2 * e], x[9 + 2 * e]);
    }
    __builtin_nontemporal_store(lo, reinterpret_cast<kv_u32x4*>(row + p.at));
    __builtin_nontemporal_store(hi, reinterpret_cast<kv_u32x4*>(row + p.at + p.apart));
}
__device__ __forceinline__ uint32_t top_of(const float (&x)[16])
{
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 16; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    return top;
}
template <int FMT>
__device__ __forceinline__ void store_codes(uint8_t* row, const pieces& p, const float (&x)[16], float inverse)
{
    kv_u32x2 c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const float* y = x + 8 * h + 4 * w;
            // (inverse 0: the scale is NaN, and so may the numbers be)
            c[h][w] = inverse == 0.f ? 0u : four_codes<FMT>(y[0] * inverse, y[1] * inverse, y[2] * inverse, y[3] * inverse);
        }
    *reinterpret_cast<kv_u32x2*>(row + p.at) = c[0];
    *reinterpret_cast<kv_u32x2*>(row + p.at + p.apart) = c[1];
}
// The codes of sixteen elements, times `ratio`, rounded again.
template <int FMT>
__device__ __forceinline__ void round_again(uint8_t* at, float ratio)
{
    kv_u32x4 c = *reinterpret_cast<const kv_u32x4*>(at);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const f32x2 lo = two_f32<FMT, false>(c[w]), hi = two_f32<FMT, true>(c[w]);
        c[w] = four_codes<FMT>(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
    }
    *reinterpret_cast<kv_u32x4*>(at) = c;
}

// The scale of a group whose new tokens go up to `top`, and that of its older ones (0 where it has none) times what its older codes are to be
// multiplied with.
struct group_scale {
    float scale, inverse, ratio;
};
template <int FMT>
__device__ __forceinline__ group_scale scale_of_group(uint32_t top, bool some_old, float before)
{
    float s = scale_for<FMT>(top);
    group_scale g = {s, 0.f, 1.f};
    if (some_old) {
        const float b = fabsf(before);
        if (!(b < INFINITY)) s = __uint_as_float(kNaNBits);   // (NaN too)
        if (s == s) {
            s = fmaxf(s, b);
            g.ratio = before / s;
        }
        g.scale = s;
    }
    if (s == s) g.inverse = 1.f / s;
    return g;
}

// Block and slot of token t of sequence s; false where it has none.
__device__ __forceinline__ bool place_of(const append_args& a, int s, int t, int64_t& block, int& slot)
{
    if (t < 0) return false;
    int b;
    kv_split_token(a.v, t, b, slot);
    if (b >= a.table_stride) return false;
    block = a.table[(int64_t)s * a.table_stride + b];
    return block >= 0 && block < a.n_pool_blocks;
}

// Lanes xor 1, 2, 4 (, 8) hold one row between them.
template <int LANES>
__device__ __forceinline__ uint32_t row_max(uint32_t x)
{
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, d));
    return x;
}

// One new token per sequence: a workgroup takes a sequence, D / 16 lanes a row (query heads, then keys, then values), each row of a key
// or value a group of its own.
template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void append_one_kernel(append_args a)
{
    __shared__ float2 s_turn[kMostPairs];
    constexpr int kLanes = D / 16, kRows = kThreads / kLanes;
    const int s = blockIdx.x, tid = threadIdx.x, c = tid % kLanes;
    const kv_view_dev& v = a.v;
    const int t = a.ctx_lens[s] - 1;
    int64_t block = 0;
    int slot = 0;
    const bool placed = place_of(a, s, t, block, slot);
    if (tid < a.pairs) s_turn[tid] = turn_of(a, s, tid);
    __syncthreads();
    const int heads = a.heads_q + 2 * v.n_kv_local;
    for (int r = blockIdx.y * kRows + tid / kLanes; r < heads; r += gridDim.y * kRows) {
        const bool query = r < a.heads_q, value = r >= a.heads_q + v.n_kv_local;
        const int h = query ? r : value ? r - a.heads_q - v.n_kv_local : r - a.heads_q;
        const pieces p = pieces_of(a, c, !value);
        float x[16];
        load_row((query ? a.q + s * a.q_stride : value ? a.v_new + s * a.v_stride : a.k + s * a.k_stride) + h * D, p, s_turn + 8 * c, a.adjacent, x);
        if (query) {
            store_bf16(a.out + ((int64_t)s * v.n_q_local + h) * D, p, x);
            continue;
        }
        if (!placed) continue;
        const uint32_t top = row_max<kLanes>(top_of(x));
        const int64_t at = q8_scale_at(a.x, block, slot, h) + (value ? a.x.block_scales / 2 : 0);
        const int old = slot % a.x.base_tokens;   // older tokens of the group
        const group_scale g = scale_of_group<FMT>(top, old > 0, old > 0 ? a.scales[at] : 0.f);
        uint8_t* row = a.pool + block * v.block_elems + (value ? v.plane_elems : 0) + (int64_t)slot * v.token_stride + v.head_off + h * D;
        store_codes<FMT>(row, p, x, g.inverse);
        if (g.inverse != 0.f && g.ratio != 1.f)
            for (int i = 1; i <= old; ++i) round_again<FMT>(row - (int64_t)i * v.token_stride + 16 * c, g.ratio);
        if (c == 0) a.scales[at] = g.scale;
    }
}

// Groups are numbered without the lengths: q_len new tokens lie in at most floor(q_len / B) + 2 groups, those of sequence s from here on.
__device__ __forceinline__ int64_t first_slot(const append_args& a, int s)
{
    const int at = a.q_off[s];
    return (a.x.base_shift >= 0 ? at >> a.x.base_shift : at / a.x.base_tokens) + 2 * (int64_t)s;
}
// The last sequence with from(s) <= i: 64 probes at a time (all lanes alike).
template <class From>
__device__ __forceinline__ int last_from(int batch, int64_t i, int lane, From from)
{
    int s = 0;
    for (int span = batch; span > 1;) {
        const int step = (span + 63) >> 6, probe = lane * step;
        const bool ok = probe < span && from(s + min(probe, span - 1)) <= i;
        const unsigned long long which = __builtin_amdgcn_ballot_w64(ok);
        const int n = which ? 63 - __builtin_clzll(which) : 0;
        s += n * step;
        span = min(step, span - n * step);
    }
    return __builtin_amdgcn_readfirstlane(s);
}

// Several: the first a.slots * a.parts workgroups take groups, a wavefront a key or value head of one at a time, the others queries.
template <int D, int FMT>
__global__ __launch_bounds__(kThreads) void append_many_kernel(append_args a)
{
    extern __shared__ float2 s_turns[];   // [tokens][pairs]
    constexpr int kLanes = D / 16, kRows = 64 / kLanes, kTimes = 16 / kRows;   // rows of a wavefront, and how often for 16 tokens
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = tid % kLanes;
    const kv_view_dev& v = a.v;
    const uint32_t groups = a.slots * (uint32_t)a.parts;
    if (blockIdx.x >= groups) {
        const int64_t i0 = (int64_t)(blockIdx.x - groups) * a.query_tokens;
        const int n = (int)min((int64_t)a.query_tokens, min(a.total, (int64_t)a.q_off[a.batch]) - i0);
        for (int x = tid; x < n * a.pairs; x += kThreads) {
            const int j = x / a.pairs;
            s_turns[x] = turn_of(a, i0 + j, x - j * a.pairs);
        }
        __syncthreads();
        for (int r = tid / kLanes; r < n * a.heads_q; r += kThreads / kLanes) {
            const int j = r / a.heads_q, h = r - j * a.heads_q;
            const pieces p = pieces_of(a, c, true);
            float x[16];
            load_row(a.q + (i0 + j) * a.q_stride + h * D, p, s_turns + j * a.pairs + 8 * c, a.adjacent, x);
            store_bf16(a.out + ((i0 + j) * v.n_q_local + h) * D, p, x);
        }
        return;
    }
    const int64_t slot_no = blockIdx.x / (uint32_t)a.parts;
    const int part = (int)(blockIdx.x - (uint32_t)slot_no * a.parts);
    const int s = last_from(a.batch, slot_no, lane, [&](int i) { return first_slot(a, i); });
    const int q0 = a.q_off[s], q_len = a.q_off[s + 1] - q0, n = a.ctx_lens[s], first = n - q_len, B = a.x.base_tokens;
    const int g0 = (max(first, 0) / B + (int)(slot_no - first_slot(a, s))) * B;   // the group's first token
    if (q_len <= 0 || g0 >= n || g0 < 0) return;
    const int t0 = max(g0, first), t1 = min(g0 + B, n);   // its new tokens (first < 0: those before token 0 have no place)
    int64_t block;
    int slot;
    if (!place_of(a, s, g0, block, slot)) return;
    const int new0 = t0 - g0, new1 = t1 - g0;             // places of the new tokens in the group
    const int64_t row0 = (int64_t)q0 + (g0 - first);      // row of the group's first token, were it new
    const int units = 2 * v.n_kv_local;
    if (part * (kThreads / 64) < v.n_kv_local) {          // (parts past the keys rotate nothing)
        for (int x = tid; x < (new1 - new0) * a.pairs; x += kThreads) {
            const int j = x / a.pairs;
            s_turns[new0 * a.pairs + x] = turn_of(a, row0 + new0 + j, x - j * a.pairs);
        }
    }
    __syncthreads();
    const int r = lane / kLanes;
    // A group of 16's numbers stay in registers; longer ones are read and rotated a second time for their codes (the prompts above 69.5 us with groups of
    // 16, of 32 75, of 64 96, of 128 146).
    const bool once = B == 16;
    for (int u = part * (kThreads / 64) + wave; u < units; u += a.parts * (kThreads / 64)) {
        const bool value = u >= v.n_kv_local;
        const int h = value ? u - v.n_kv_local : u;
        const pieces p = pieces_of(a, c, !value);
        const uint16_t* src = (value ? a.v_new : a.k) + h * D;
        const int64_t stride = value ? a.v_stride : a.k_stride;
        uint8_t* rows = a.pool + block * v.block_elems + (value ? v.plane_elems : 0) + (int64_t)slot * v.token_stride + v.head_off + h * D;
        const int64_t at = q8_scale_at(a.x, block, slot, h) + (value ? a.x.block_scales / 2 : 0);
        const float before = new0 > 0 ? a.scales[at] : 0.f;
        float x[kTimes][16];
        auto fetch = [&](int chunk) {
#pragma unroll
            for (int i = 0; i < kTimes; ++i) {
                const int j = 16 * chunk + kRows * i + r;
                if (j >= new0 && j < new1) {
                    load_row(src + (row0 + j) * stride, p, s_turns + j * a.pairs + 8 * c, a.adjacent, x[i]);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) x[i][e] = 0.f;
                }
            }
        };
        uint32_t top = 0;
        for (int chunk = new0 >> 4; chunk < (new1 + 15) >> 4; ++chunk) {
            fetch(chunk);
#pragma unroll
            for (int i = 0; i < kTimes; ++i) top = max(top, top_of(x[i]));
        }
        const group_scale g = scale_of_group<FMT>(row_max<64>(top), new0 > 0, before);
        for (int chunk = new0 >> 4; chunk < (new1 + 15) >> 4; ++chunk) {
            if (!once) fetch(chunk);
#pragma unroll
            for (int i = 0; i < kTimes; ++i) {
                const int j = 16 * chunk + kRows * i + r;
                if (j >= new0 && j < new1) store_codes<FMT>(rows + (int64_t)j * v.token_stride, p, x[i], g.inverse);
            }
        }
        if (g.inverse != 0.f && g.ratio != 1.f)
            for (int j = r; j < new0; j += kRows) round_again<FMT>(rows + (int64_t)j * v.token_stride + 16 * c, g.ratio);
        if (lane == 0) a.scales[at] = g.scale;
    }
}

bool strided_ok(const void* p, int64_t stride, int64_t row) { return kv_aligned(p, 16) && stride % 8 == 0 && stride >= row; }

}  // namespace

extern "C" int kv_rope_append_q8(void* kv_pool, float* scales, int format, int64_t n_pool_blocks, const kv_view* view, const void* q,
                                 int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* q_out,
                                 const int32_t* positions, int64_t position_stride, int n_axes, const float* inv_freq, int rotary_dim,
                                 const int32_t* axis_of_pair, int pairs, const int32_t* block_table, int64_t block_table_stride,
                                 const int32_t* ctx_lens, const int32_t* q_offsets, int batch, int64_t total, void* hip_stream)
{
    if (!kv_view_ok(view) || !q8_format_ok(format) || n_pool_blocks < 0 || block_table_stride < 0 || batch < 0 || total < 0 || rotary_dim < 0 ||
        position_stride < 0 || (pairs != KV_ROPE_HALVES && pairs != KV_ROPE_ADJACENT) || n_axes < 1)
        return KV_ERR_INVALID_ARG;
    const int d = view->geom.head_dim, half = rotary_dim / 2;
    if (rotary_dim > d || (half && position_stride < total) || (!q_offsets && total != batch) || !q != !q_out) return KV_ERR_INVALID_ARG;
    if (axis_of_pair)
        for (int i = 0; i < half; ++i)
            if (axis_of_pair[i] < 0 || axis_of_pair[i] >= n_axes) return KV_ERR_INVALID_ARG;
    if (batch == 0 || total == 0) return KV_OK;
    if (!kv_pool || !scales || !k || !v || (half && (!positions || !inv_freq)) || !block_table || !ctx_lens) return KV_ERR_INVALID_ARG;
    const int64_t q_row = (int64_t)view->n_q_local * d, k_row = (int64_t)view->n_kv_local * d;
    if ((q && (q_stride < q_row || (q_out == q && q_stride != q_row))) || k_stride < k_row || v_stride < k_row) return KV_ERR_INVALID_ARG;
    const int B = view->geom.base_block_size;
    if ((d != 64 && d != 128) || rotary_dim % 16 != 0 || n_axes > 4 || B % 16 != 0 || B > kMostBase) return KV_ERR_UNSUPPORTED;
    if ((q && !strided_ok(q, q_stride, q_row)) || !strided_ok(k, k_stride, k_row) || !strided_ok(v, v_stride, k_row) ||
        (q && !kv_aligned(q_out, 16)) || !kv_aligned(kv_pool, 16) || !kv_aligned(scales, 4))
        return KV_ERR_UNSUPPORTED;
    append_args a = {};
    a.q = (const uint16_t*)q;
    a.k = (const uint16_t*)k;
    a.v_new = (const uint16_t*)v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.out = (uint16_t*)q_out;
    a.pool = (uint8_t*)kv_pool;
    a.scales = scales;
    a.n_pool_blocks = n_pool_blocks;
    a.positions = positions;
    a.position_stride = position_stride;
    a.inv_freq = inv_freq;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.q_off = q_offsets;
    a.total = total;
    a.v = kv_view_to_dev(view);
    a.x = q8_view_of(view);
    a.batch = batch;
    a.pairs = half;
    a.adjacent = pairs == KV_ROPE_ADJACENT;
    a.heads_q = q ? view->n_q_local : 0;
    for (int i = 0; i < half; ++i) a.axis[i >> 4] |= (uint32_t)(axis_of_pair ? axis_of_pair[i] : 0) << (2 * (i & 15));
    const bool e4m3 = format == kE4M3;
    hipStream_t st = (hipStream_t)hip_stream;
    if (!q_offsets) {
        const int rows = a.heads_q + 2 * view->n_kv_local, at_once = kThreads / (d / 16);
        const dim3 grid((unsigned)batch, batch < 512 ? (unsigned)((rows + at_once - 1) / at_once) : 1u);
        auto* f = d == 64 ? (e4m3 ? append_one_kernel<64, kE4M3> : append_one_kernel<64, kInt8>)
                          : (e4m3 ? append_one_kernel<128, kE4M3> : append_one_kernel<128, kInt8>);
        hipLaunchKernelGGL(f, grid, dim3(kThreads), 0, st, a);
    } else {
        const int64_t slots = total / B + 2 * (int64_t)batch;
        const int per_part = kThreads / 64, most_parts = (2 * view->n_kv_local + per_part - 1) / per_part;
        int64_t parts = (1024 + slots - 1) / slots;
        a.parts = (int32_t)(parts < 1 ? 1 : parts > most_parts ? most_parts : parts);
        // (32 heads of 128, 8 prompts of 2048 tokens: 70 us with one token a workgroup, 72 with two, 75 with four)
        const int at_once = q ? kThreads / (d / 16) / a.heads_q : 0;
        a.query_tokens = at_once < 1 ? 1 : at_once > kMostQueries ? kMostQueries : at_once;
        const int64_t queries = q ? (total + a.query_tokens - 1) / a.query_tokens : 0, grid = slots * a.parts + queries;
        if (grid > 0x7fffffff) return KV_ERR_UNSUPPORTED;
        a.slots = (uint32_t)slots;
        const int tokens = B > a.query_tokens ? B : a.query_tokens;
        auto* f = d == 64 ? (e4m3 ? append_many_kernel<64, kE4M3> : append_many_kernel<64, kInt8>)
                          : (e4m3 ? append_many_kernel<128, kE4M3> : append_many_kernel<128, kInt8>);
        hipLaunchKernelGGL(f, dim3((unsigned)grid), dim3(kThreads), (size_t)tokens * half * sizeof(float2), st, a);
    }
    return kv_record_hip_error(hipGetLastError(), "kv_rope_append_q8 launch");
}
