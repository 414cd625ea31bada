// Decode attention over a cache held in 8 bits: one query token a sequence, every head's codes read once.
//
//   out = sum_t softmax_t(c q . sK[t] k_t) sV[t] v_t,  k_t and v_t the codes of token t, sK and sV the scales of its group
//
// Bound by reading codes and scales: 2 d + 8 / B_base bytes a token and head.
//
// A wavefront takes 32 tokens of a KV head at a time (a tile), its G <= 16 query rows as the 16 columns of the products, and needs nothing
// of LDS or of other wavefronts until it is through.  Lane l = (m = l % 16, g = l / 16), products of 16 x 16 x 32 in bf16:
//   S^T[token][row] = K . q^T   A: lane holds token m of 16, 16 bytes at 16 g of each 64 of the row; q's columns are ordered alike
//   O^T[dim][row] += V^T . P    A: lane holds d / 16 dims (from d / 16 m on) of tokens 4 g .. 4 g + 3 of both halves of the tile: what a
//                               lane loads of a token is a run of bytes, and product j takes dim d / 16 m + j from every lane
// The scores come out with tokens 4 g .. 4 g + 3 of each half in lane (row, g): the B operand of the second product as it is.  Codes
// become bf16 exactly (e4m3 by the conversion instruction, int8 over fp32), K's scale goes to the score, V's to the weight.
// Softmax by a running reference that lags up to 2^8 behind the maximum; the denominator sums the weights as they are rounded to bf16.
#include "kv_q8.h"

#include <algorithm>

using namespace kvq8;

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kTile = 32;

struct decode_args {
    const uint16_t* q;
    uint16_t* out;
    const uint8_t* pool;
    const float* scales;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* ctx_lens;
    kv_view_dev v;
    q8_view x;
    float scale_log2e;
    int32_t group, batch;
    int32_t head_sets;     // n_kv_local / HPW
    int32_t whole;         // a workgroup takes a whole pair (sequence, set of heads)
    float* part_o;         // [2 * workgroups][HPW * G][D] sums of a cut pair's piece
    float* part_ml;        // [2 * workgroups][HPW * G][2] (reference in exponent units, sum of weights)
    int2* ends;            // [batch * head_sets] workgroups that hold a pair's first and last piece
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float uniform(float x) { return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, x))); }

typedef const __attribute__((address_space(4))) int32_t* const_ints;
typedef const __attribute__((address_space(4))) float* const_floats;

// Steps of the pairs lie on one axis, sequence by sequence, in each its sets of heads in turn.  Thread i of the workgroup sums the steps of
// sequences [i k, (i + 1) k), k = batch / 256 rounded up; s_incl are the inclusive sums over the threads.
struct axis_sums {
    long long total;
    int per;   // k
};
template <int STEP>
__device__ __forceinline__ int steps_of(int n) { return n > 0 ? (n + STEP - 1) / STEP : 0; }

template <int STEP>
__device__ __forceinline__ axis_sums sum_axis(const decode_args& a, long long* s_incl)
{
    const int tid = threadIdx.x, per = (a.batch + kThreads - 1) / kThreads;
    long long mine = 0;
    for (int i = 0; i < per; ++i) {
        const int s = tid * per + i;
        if (s < a.batch) mine += steps_of<STEP>(a.ctx_lens[s]);
    }
    // inclusive sum over the wavefront, then over the workgroup
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const long long y = __shfl_up(mine, d);
        if ((tid & 63) >= d) mine += y;
    }
    s_incl[tid] = mine;
    __syncthreads();
    long long before = 0;
    for (int w = 0; w < (tid >> 6); ++w) before += s_incl[64 * w + 63];
    __syncthreads();
    s_incl[tid] = mine + before;
    __syncthreads();
    return {s_incl[kThreads - 1], per};
}

// V^T operands of one dword (dims 4 w .. 4 w + 3) of eight tokens: operand b of dim 4 w + b holds the eight tokens' values.
template <int FMT>
__device__ __forceinline__ void dims_of(const uint32_t (&t)[8], bf16x8 (&to)[4])
{
    kv_u32x4 d[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t lo = __builtin_amdgcn_perm(t[2 * p + 1], t[2 * p], 0x05010400u), hi = __builtin_amdgcn_perm(t[2 * p + 1], t[2 * p], 0x07030602u);
        d[0][p] = two_bf16<FMT, false>(lo);
        d[1][p] = two_bf16<FMT, true>(lo);
        d[2][p] = two_bf16<FMT, false>(hi);
        d[3][p] = two_bf16<FMT, true>(hi);
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) to[b] = as_bf16x8(d[b]);
}

// HPW: heads that the wavefronts of a workgroup take side by side; the others follow each other in the tokens.
template <int D, int FMT, int HPW>
__global__ __launch_bounds__(kThreads) void decode_q8_kernel(decode_args a)
{
    constexpr int kLoads = D / 64;          // of 16 bytes of a K row
    constexpr int kWords = D / 64;          // dwords of a V row in a lane
    constexpr int kDims = D / 16;           // dims of a lane's V
    constexpr int kSubs = kWaves / HPW;     // wavefronts that share a head
    constexpr int kStep = kTile * kSubs;    // tokens of a step
    constexpr int kPad = D + 4;
    __shared__ long long s_incl[kThreads];
    __shared__ float s_o[kWaves][16][kPad];
    __shared__ float s_ml[kWaves][16][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), m = lane & 15, g = lane >> 4;
    const kv_view_dev& v = a.v;
    const int G = a.group;
    // rows of sequences without tokens are zeros
    for (int s = blockIdx.x; s < a.batch; s += gridDim.x)
        if (a.ctx_lens[s] <= 0)
            for (int i = tid; i < v.n_q_local * D / 8; i += kThreads)
                reinterpret_cast<kv_u32x4*>(a.out + (int64_t)s * v.n_q_local * D)[i] = kv_u32x4{0u, 0u, 0u, 0u};

    int s, set, step;             // where the workgroup's steps start
    long long left;               // and how many they are
    if (a.whole) {
        s = (int)blockIdx.x / a.head_sets;
        set = (int)blockIdx.x - s * a.head_sets;
        step = 0;
        left = steps_of<kStep>(a.ctx_lens[s]);
    } else {
        const axis_sums sums = sum_axis<kStep>(a, s_incl);
        // (no workgroup without a step among those that have some: the pieces of a pair lie in consecutive ones)
        const long long total = sums.total * a.head_sets, W = min((long long)gridDim.x, total);
        if (blockIdx.x >= W) return;
        const long long from = total * blockIdx.x / W, to = total * (blockIdx.x + 1) / W;
        left = to - from;
        // the thread in whose sequences it lies, then the sequence
        int at = 0;
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w)
            at += __builtin_popcountll(__builtin_amdgcn_ballot_w64(s_incl[64 * w + lane] * a.head_sets <= from));
        long long in = from - (at > 0 ? s_incl[at - 1] : 0) * a.head_sets;
        s = uniform(at * sums.per);
        for (;; ++s) {
            const long long n = (long long)steps_of<kStep>(a.ctx_lens[s]) * a.head_sets;
            if (in < n) break;
            in -= n;
        }
        const int steps = steps_of<kStep>(a.ctx_lens[s]);
        set = uniform((int)(in / steps));
        step = uniform((int)(in - (long long)set * steps));
    }

    const int hw = HPW == 1 ? 0 : wave % HPW, sub = HPW == 1 ? wave : wave / HPW;
    const uint32_t row_bytes = (uint32_t)v.token_stride;
    while (left > 0) {
        const int n = uniform(a.ctx_lens[s]), steps = steps_of<kStep>(n);
        if (steps == 0) {   // (of a sequence without tokens)
            ++s;
            continue;
        }
        const int end = (int)min((long long)steps, step + left);
        const int h = set * HPW + hw;   // this wavefront's local KV head
        const const_ints ids = (const_ints)(a.table + (int64_t)s * a.table_stride);
        const int last16 = (n - 1) & ~15;

        // q, columns past the group zeros; dims in the order of K's bytes
        bf16x8 qb[2 * kLoads];
        {
            const uint16_t* row = a.q + ((int64_t)s * v.n_q_local + h * G + min(m, G - 1)) * D + 16 * g;
#pragma unroll
            for (int i = 0; i < 2 * kLoads; ++i) {
                kv_u32x4 x = *reinterpret_cast<const kv_u32x4*>(row + 64 * (i >> 1) + 8 * (i & 1));
                if (m >= G) x = kv_u32x4{0u, 0u, 0u, 0u};
                qb[i] = as_bf16x8(x);
            }
        }
        f32x4 o[kDims];
#pragma unroll
        for (int j = 0; j < kDims; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        float ref = kLowest, l = 0.f;

        struct tile {
            kv_u32x4 k[2][kLoads];
            uint32_t v[8][kWords];
            float sk[2], sv[2];
        };
        // Tokens past the end are replaced by the last one of its 16 (finite, masked later).
        auto request = [&](int t0, tile& x) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int t = min(t0 + 16 * half, last16);
                int b, slot;
                kv_split_token(v, t, b, slot);
                const int64_t id = ids[b];
                const uint8_t* base = a.pool + id * v.block_elems + (int64_t)slot * row_bytes + v.head_off + h * D;
                const int most = n - 1 - t;   // the last row that there is
                const uint32_t kr = (uint32_t)min(m, most) * row_bytes + 16 * g;
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
                    x.k[half][i] = __builtin_nontemporal_load(reinterpret_cast<const kv_u32x4*>(base + kr + 64 * i));
                const uint8_t* vb = base + v.plane_elems;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t vr = (uint32_t)min(4 * g + e, most) * row_bytes + kDims * m;
                    if constexpr (kWords == 2) {
                        const kv_u32x2 y = __builtin_nontemporal_load(reinterpret_cast<const kv_u32x2*>(vb + vr));
                        x.v[4 * half + e][0] = y[0];
                        x.v[4 * half + e][1] = y[1];
                    } else {
                        x.v[4 * half + e][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(vb + vr));
                    }
                }
                const const_floats sc = (const_floats)(a.scales + q8_scale_at(a.x, id, slot, h));
                x.sk[half] = sc[0];
                x.sv[half] = sc[a.x.block_scales / 2];
            }
        };
        auto take = [&](int t0, const tile& x) {
            float u[8];   // scores in units of the exponent
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 sc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 2 * kLoads; ++i) {
                    const uint32_t w0 = x.k[half][i >> 1][2 * (i & 1)], w1 = x.k[half][i >> 1][2 * (i & 1) + 1];
                    const kv_u32x4 ka = {two_bf16<FMT, false>(w0), two_bf16<FMT, true>(w0), two_bf16<FMT, false>(w1), two_bf16<FMT, true>(w1)};
                    sc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(ka), qb[i], sc, 0, 0, 0);
                }
                const float c = x.sk[half] * a.scale_log2e;
#pragma unroll
                for (int i = 0; i < 4; ++i) u[4 * half + i] = sc[i] * c;
            }
            if (t0 + kTile > n) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (t0 + 16 * (i >> 2) + 4 * g + (i & 3) >= n) u[i] = kNegInf;
            }
            float top = u[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, u[i]);
            if (__builtin_amdgcn_ballot_w64(top - ref > 8.f) != 0) {
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float to = fmaxf(ref, top), alpha = fast_exp2(ref - to);
                l *= alpha;
#pragma unroll
                for (int j = 0; j < kDims; ++j) o[j] *= alpha;
                ref = to;
            }
            kv_u32x4 pb;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w0 = fast_exp2(u[2 * i] - ref), w1 = fast_exp2(u[2 * i + 1] - ref), sv = x.sv[i >> 1];
                const uint32_t w = pack_bf16x2(w0, w1);
                l = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, w), __builtin_bit_cast(bf16x2, 0x3f803f80u), l, false);
                pb[i] = pack_bf16x2(w0 * sv, w1 * sv);
            }
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                uint32_t t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) t[e] = x.v[e][w];
                bf16x8 va[4];
                dims_of<FMT>(t, va);
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    o[4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[b], as_bf16x8(pb), o[4 * w + b], 0, 0, 0);
            }
        };
        {
            int t = step * kStep + sub * kTile;
            const int t_end = min(end * kStep, n);
            tile x, y;
            if (t < t_end) request(t, x);
            while (t < t_end) {
                if (t + kStep < t_end) request(t + kStep, y);
                take(t, x);
                t += kStep;
                if (t >= t_end) break;
                if (t + kStep < t_end) request(t + kStep, x);
                take(t, y);
                t += kStep;
            }
        }
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);

        // the piece's rows: sums of the wavefronts that share a head
        if (m < G) {
            // lane (row m, g): element i of product j is dim kDims (4 g + i) + j
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kDims; j += 4)
                    *reinterpret_cast<f32x4*>(&s_o[wave][m][kDims * (4 * g + i) + j]) = f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
            if (g == 0) {
                s_ml[wave][m][0] = ref;
                s_ml[wave][m][1] = l;
            }
        }
        __syncthreads();
        const bool starts = step == 0, ends = end == steps;
        const int64_t pair = (int64_t)s * a.head_sets + set;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (starts && !ends ? 1 : 0);
        const int rows = HPW * G;
        for (int i = tid; i < rows * (D / 4); i += kThreads) {
            const int row = i / (D / 4), d4 = i % (D / 4), hh = row / G, r = row - hh * G;
            float top = kLowest, sum = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kSubs; ++w) top = fmaxf(top, s_ml[w * HPW + hh][r][0]);
#pragma unroll
            for (int w = 0; w < kSubs; ++w) {
                const float f = fast_exp2(s_ml[w * HPW + hh][r][0] - top);
                sum += s_ml[w * HPW + hh][r][1] * f;
                acc += *reinterpret_cast<const f32x4*>(&s_o[w * HPW + hh][r][4 * d4]) * f;
            }
            if (starts && ends) {
                const float inv = 1.f / sum;
                *reinterpret_cast<kv_u32x2*>(a.out + ((int64_t)s * v.n_q_local + set * rows + row) * D + 4 * d4) =
                    kv_u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
            } else {
                *reinterpret_cast<f32x4*>(a.part_o + (slot * rows + row) * D + 4 * d4) = acc;
                if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * rows + row) * 2) = make_float2(top, sum);
            }
        }
        if (!a.whole && tid == 0) {
            if (starts) a.ends[pair].x = blockIdx.x;
            if (ends) a.ends[pair].y = blockIdx.x;
        }
        __syncthreads();
        left -= end - step;
        step = 0;
        if (++set == a.head_sets) {
            set = 0;
            ++s;
        }
    }
}

// Row r of a cut pair: the sum of its pieces.  D / 4 lanes a slice of the list, the slices then over LDS.
template <int D>
__global__ __launch_bounds__(kThreads) void merge_q8_kernel(decode_args a, int rows)
{
    constexpr int kSlices = kThreads / (D / 4);
    __shared__ f32x4 s_o[kSlices][D / 4];
    __shared__ float2 s_ml[kSlices];
    const int pair = blockIdx.x, row = blockIdx.y, s = pair / a.head_sets, set = pair - s * a.head_sets;
    if (a.ctx_lens[s] <= 0) return;
    const int first = a.ends[pair].x, last = a.ends[pair].y;
    if (first == last) return;
    const int slice = threadIdx.x / (D / 4), d4 = threadIdx.x % (D / 4);
    float top = kLowest, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w = first + slice; w <= last; w += kSlices) {
        const int64_t rec = (2 * (int64_t)w + (w == first ? 1 : 0)) * rows + row;
        const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + rec * 2);
        const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + rec * D + 4 * d4);
        const float to = fmaxf(top, ml.x), f = fast_exp2(top - to), e = fast_exp2(ml.x - to);
        acc = acc * f + o * e;
        sum = sum * f + ml.y * e;
        top = to;
    }
    s_o[slice][d4] = acc;
    if (d4 == 0) s_ml[slice] = make_float2(top, sum);
    __syncthreads();
    if (slice != 0) return;
    for (int i = 0; i < kSlices; ++i) top = fmaxf(top, s_ml[i].x);
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < kSlices; ++i) {
        const float f = fast_exp2(s_ml[i].x - top);
        sum += s_ml[i].y * f;
        acc += s_o[i][d4] * f;
    }
    const float inv = 1.f / sum;
    *reinterpret_cast<kv_u32x2*>(a.out + ((int64_t)s * a.v.n_q_local + set * rows + row) * D + 4 * d4) =
        kv_u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
}

constexpr int kMostWorkgroups = 512;   // two for each of 256 compute units

// How a call is cut: the same for the workspace and the launch.
struct decode_plan {
    int hpw, head_sets, workgroups;
    bool whole;
    size_t o_bytes, ml_bytes, bytes;
};
decode_plan plan_of(const kv_view* view, int batch, int max_ctx_len)
{
    decode_plan p;
    const int hl = view->n_kv_local;
    p.hpw = hl % 4 == 0 ? 4 : hl % 2 == 0 ? 2 : 1;
    p.whole = max_ctx_len <= 512;
    if (p.whole) p.hpw = 1;
    p.head_sets = hl / p.hpw;
    const int step = kTile * kWaves / p.hpw;
    const int64_t pairs = (int64_t)batch * p.head_sets, steps = pairs * (((int64_t)max_ctx_len + step - 1) / step);
    p.workgroups = (int)(p.whole ? pairs : std::min<int64_t>(steps, kMostWorkgroups));
    const int rows = p.hpw * view->group;
    p.o_bytes = p.whole ? 0 : (size_t)2 * p.workgroups * rows * view->geom.head_dim * 4;
    p.ml_bytes = p.whole ? 0 : (size_t)2 * p.workgroups * rows * 8;
    p.bytes = p.whole ? 0 : p.o_bytes + p.ml_bytes + (size_t)pairs * sizeof(int2);
    return p;
}

template <int D, int FMT>
void launch(const decode_plan& p, const decode_args& a, hipStream_t st)
{
    auto* f = p.hpw == 4 ? decode_q8_kernel<D, FMT, 4> : p.hpw == 2 ? decode_q8_kernel<D, FMT, 2> : decode_q8_kernel<D, FMT, 1>;
    hipLaunchKernelGGL(f, dim3((unsigned)p.workgroups), dim3(kThreads), 0, st, a);
    if (!p.whole)
        hipLaunchKernelGGL(merge_q8_kernel<D>, dim3((unsigned)(a.batch * p.head_sets), (unsigned)(p.hpw * a.group)), dim3(kThreads), 0, st, a, p.hpw * a.group);
}

}  // namespace

extern "C" size_t paged_decode_attn_q8_workspace_bytes(const kv_view* view, int batch, int max_ctx_len)
{
    if (!kv_view_ok(view) || batch <= 0 || max_ctx_len <= 0) return 0;
    return plan_of(view, batch, max_ctx_len).bytes;
}

extern "C" int paged_decode_attn_q8(const void* q, void* out, const void* kv_pool, const float* scales, int format, int64_t n_pool_blocks,
                                    const int32_t* block_table, int64_t block_table_stride, const int32_t* ctx_lens, int batch,
                                    int max_ctx_len, const kv_view* view, float scale, void* workspace, size_t workspace_bytes,
                                    void* hip_stream)
{
    if (!kv_view_ok(view) || !q8_format_ok(format) || batch < 0 || max_ctx_len < 0 || n_pool_blocks < 0 || block_table_stride < 0)
        return KV_ERR_INVALID_ARG;
    if (batch == 0) return KV_OK;
    if (!q || !out || !ctx_lens || (max_ctx_len > 0 && (!kv_pool || !scales || !block_table))) return KV_ERR_INVALID_ARG;
    if (block_table_stride < ((int64_t)max_ctx_len + view->block_tokens - 1) / view->block_tokens) return KV_ERR_INVALID_ARG;
    const int d = view->geom.head_dim, G = view->group;
    if ((d != 64 && d != 128) || G > 16 || view->geom.base_block_size % 16 != 0) return KV_ERR_UNSUPPORTED;
    if (!kv_aligned(q, 16) || !kv_aligned(out, 16) || !kv_aligned(kv_pool, 16) || !kv_aligned(scales, 4)) return KV_ERR_UNSUPPORTED;
    if ((int64_t)batch * view->n_q_local > 0x7fffffff || max_ctx_len > 0x7fffff00) return KV_ERR_UNSUPPORTED;
    const decode_plan p = plan_of(view, batch, max_ctx_len > 0 ? max_ctx_len : 1);
    if (p.bytes) {
        if (!workspace || !kv_aligned(workspace, 256)) return KV_ERR_INVALID_ARG;
        if (workspace_bytes < p.bytes) return KV_ERR_WORKSPACE;
    }
    decode_args a = {};
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.pool = (const uint8_t*)kv_pool;
    a.scales = scales;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.v = kv_view_to_dev(view);
    a.x = q8_view_of(view);
    a.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.group = G;
    a.batch = batch;
    a.head_sets = p.head_sets;
    a.whole = p.whole;
    a.part_o = (float*)workspace;
    a.part_ml = (float*)((char*)workspace + p.o_bytes);
    a.ends = (int2*)((char*)workspace + p.o_bytes + p.ml_bytes);
    hipStream_t st = (hipStream_t)hip_stream;
    if (d == 64) {
        if (format == kE4M3) launch<64, kE4M3>(p, a, st);
        else launch<64, kInt8>(p, a, st);
    } else {
        if (format == kE4M3) launch<128, kE4M3>(p, a, st);
        else launch<128, kInt8>(p, a, st);
    }
    return kv_record_hip_error(hipGetLastError(), "paged_decode_attn_q8 launch");
}
