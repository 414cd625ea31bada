// Decode attention over a cache held in 8 bits: one query token a sequence, every head's codes read once.
//
//   out = sum_t softmax_t(c q . sK[t] k_t) sV[t] v_t,  k_t and v_t the codes of token t, sK and sV the scales of its group
//
// Bound by reading codes and scales: 2 d + 8 / B_base bytes a token and head.  Measured: 64 sequences around 2048 tokens, 8 heads, 56 us
// (308 MB read at 5.8 TB/s, 6.3 between 64 and 192 sequences, and 4.6 us of second launch; the same cache in bf16 97); 256 around 1024,
// one head, 44 (70); 8 long and short ones, 2 heads, 32 (53).  Without its arithmetic the kernel takes 2 to 8 % less.
//
// A wavefront takes 32 tokens of a KV head at a time (a tile), its G <= 16 query rows as the 16 columns of the products, and needs nothing
// of LDS or of other wavefronts until it is through.  Lane l = (m = l % 16, g = l / 16), products of 16 x 16 x 32 in bf16:
//   S^T[token][row] = K . q^T   A: lane holds token m of 16, 16 bytes at 16 g of each 64 of the row; q's columns are ordered alike
//   O^T[dim][row] += V^T . P    A: lane holds d / 16 dims (from d / 16 m on) of tokens 4 g .. 4 g + 3 of both halves of the tile: what a
//                               lane loads of a token is a run of bytes, and product j takes dim d / 16 m + j from every lane
// The scores come out with tokens 4 g .. 4 g + 3 of each half in lane (row, g): the B operand of the second product as it is.  Codes
// become bf16 exactly (e4m3 by the conversion instruction, int8 over fp32), K's scale goes to the score, V's to the weight.
// Softmax by a running reference that lags up to 2^8 behind the maximum.  The weights go to the products as two bf16, the rounded value and
// what the rounding left: that costs 1 % of the time (the reads bound it), and the error against 64 bits is that of the output's own
// rounding, where single bf16 weights made it 1.2 to 1.4 times that.
#include "kv_q8.h"

#include <algorithm>

using namespace kvq8;

namespace {

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
    int32_t last_block;    // of a row of the table, by the bound of the lengths
    int32_t unit_shift, start_units;   // of the axis that is cut
    uint32_t inverse;      // 2^32 / workgroups
    float* part_o;         // [2 * workgroups][HPW * G][D] sums of a cut pair's piece
    float* part_ml;        // [2 * workgroups][HPW * G][2] (reference in exponent units, sum of weights)
    int2* ends;            // [batch * head_sets] workgroups that hold a pair's first and last piece
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

typedef const __attribute__((address_space(1))) uint8_t* global_bytes;
typedef const __attribute__((address_space(4))) int32_t* const_ints;
typedef const __attribute__((address_space(4))) float* const_floats;

// The pairs lie on one axis, sequence by sequence, in each its sets of heads in turn: a pair's start counts start_units, each of its steps
// 2^unit_shift.  Workgroup i takes the steps between two positions on it, which all workgroups work out alike.  (A start costs about what a step does:
// lengths of the pieces are then as unequal as whole steps make them and no more.)
__device__ __forceinline__ int steps_of(int n, int step) { return n > 0 ? (int)(((unsigned)n + step - 1) / (unsigned)step) : 0; }

template <int CTRL>
__device__ __forceinline__ int dpp_shr(int x) { return __builtin_amdgcn_update_dpp(0, x, CTRL, 0xf, 0xf, true); }
// Inclusive sum over the 64 lanes.
__device__ __forceinline__ int inclusive_sum(int x, int lane)
{
    x += dpp_shr<0x111>(x);
    x += dpp_shr<0x112>(x);
    x += dpp_shr<0x114>(x);
    x += dpp_shr<0x118>(x);
    const int t0 = __builtin_amdgcn_readlane(x, 15), t1 = t0 + __builtin_amdgcn_readlane(x, 31), t2 = t1 + __builtin_amdgcn_readlane(x, 47);
    const int row = lane >> 4;
    return x + (row == 0 ? 0 : row == 1 ? t0 : row == 2 ? t1 : t2);
}
struct axis_place {
    int s, set, step;
};
// Steps of sequences s0 + 4 lane .. + 3 of a run of 256, their sum over the lanes so far, and that of those with any.
struct axis_run {
    int n[4], steps[4], sum, some, sum_incl, some_incl;
};
// The length of sequence s of a run that starts at s0.
__device__ __forceinline__ int length_in(const axis_run& r, int s, int s0)
{
    const int i = (s - s0) & 3;
    return __builtin_amdgcn_readlane(i == 0 ? r.n[0] : i == 1 ? r.n[1] : i == 2 ? r.n[2] : r.n[3], (s - s0) >> 2);
}
__device__ __forceinline__ axis_run run_of(const decode_args& a, int s0, int lane, int step)
{
    axis_run r;
    r.sum = r.some = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) r.n[i] = a.ctx_lens[min(s0 + 4 * lane + i, a.batch - 1)];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        r.steps[i] = s0 + 4 * lane + i < a.batch ? steps_of(r.n[i], step) : 0;   // (loads without branches: all at once)
        r.sum += r.steps[i];
        r.some += r.steps[i] > 0;
    }
    r.sum_incl = inclusive_sum(r.sum, lane);
    r.some_incl = inclusive_sum(r.some, lane);
    return r;
}
// The step that starts at or behind position x of a run (x less than what the run counts).
__device__ __forceinline__ axis_place place_in(const decode_args& a, const axis_run& r, int s0, int x, int start_units, int lane)
{
    const int hs = a.head_sets;
    const int mine = hs * ((r.sum << a.unit_shift) + start_units * r.some);
    const int incl = hs * ((r.sum_incl << a.unit_shift) + start_units * r.some_incl);
    const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > x));
    x -= __builtin_amdgcn_readlane(incl - mine, at);
    int i = 0, n = __builtin_amdgcn_readlane(r.steps[0], at), per_pair = n > 0 ? (n << a.unit_shift) + start_units : 0;
#pragma unroll
    for (int k = 1; k < 4; ++k) {
        const int next = __builtin_amdgcn_readlane(r.steps[k], at);
        if (i == k - 1 && x >= hs * per_pair) {
            x -= hs * per_pair;
            i = k;
            n = next;
            per_pair = n > 0 ? (n << a.unit_shift) + start_units : 0;
        }
    }
    int set = 0;
    if (hs > 1) {   // x / per_pair, less than hs
        set = uniform((int)((float)x * __builtin_amdgcn_rcpf((float)per_pair)));
        set += (set + 1) * per_pair <= x ? 1 : 0;
        set -= set * per_pair > x ? 1 : 0;
    }
    const int in = x - set * per_pair - start_units;
    return {s0 + 4 * at + i, set, in <= 0 ? 0 : (in + (1 << a.unit_shift) - 1) >> a.unit_shift};
}
__device__ __forceinline__ axis_place place_at(const decode_args& a, axis_run r, int x, int start_units, int lane, int step)
{
    for (int s0 = 0;;) {
        const int all = a.head_sets * ((__builtin_amdgcn_readlane(r.sum_incl, 63) << a.unit_shift) + start_units * __builtin_amdgcn_readlane(r.some_incl, 63));
        if (x < all) return place_in(a, r, s0, x, start_units, lane);
        x -= all;
        s0 += 256;
        if (s0 >= a.batch) return {a.batch, 0, 0};
        r = run_of(a, s0, lane, step);
    }
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

// HPW: heads that the wavefronts of a workgroup take side by side; the others follow each other in the tokens.  8 heads have 8 wavefronts: a
// workgroup then reads whole token rows of 1 KiB as one stream (8 heads, 64 sequences around 2048 tokens: 56 us, 59 us as 4 heads and 4).
// Two tiles at a time, or two heads a wavefront, with one wavefront a SIMD: 58 us there, the same or up to 2 % better elsewhere.
// WHOLE: a workgroup takes a pair (sequence, head).  Trips to memory are what counts then: the length, the blocks of the wavefront's first 32 tiles
// and q are asked for together, scales beside the first tile.
constexpr int waves_of(int hpw) { return hpw == 8 ? 8 : 4; }   // of a workgroup
template <int D, int FMT, int HPW, bool WHOLE>
__global__ __launch_bounds__(64 * waves_of(HPW), 2) void decode_q8_kernel(decode_args a)
{
    constexpr int kWaves = waves_of(HPW), kThreads = 64 * kWaves;
    constexpr int kLoads = D / 64;          // of 16 bytes of a K row
    constexpr int kWords = D / 64;          // dwords of a V row in a lane
    constexpr int kDims = D / 16;           // dims of a lane's V
    constexpr int kSubs = kWaves / HPW;     // wavefronts that share a head
    constexpr int kStep = kTile * kSubs;    // tokens of a step
    constexpr int kPad = D + 4;
    __shared__ float s_o[kWaves][16][kPad];
    __shared__ float s_ml[kWaves][16][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), m = lane & 15, g = lane >> 4;
    const kv_view_dev& v = a.v;
    const int G = a.group;
    const int hw = wave % HPW, sub = wave / HPW;
    axis_place at, to;   // where the workgroup's steps start, and where they end
    int known = -1;      // length of the first sequence
    int whole_id = 0, whole_t = 0, whole_slot = 0;   // a lane's 16 tokens of those that the wavefront takes first, their block and place in it
    if constexpr (WHOLE) {
        at.s = (int)blockIdx.x / a.head_sets;
        at.set = (int)blockIdx.x - at.s * a.head_sets;
        at.step = 0;
        whole_t = (lane >> 1) * kStep + sub * kTile + 16 * (lane & 1);
        int b;
        kv_split_token(v, whole_t, b, whole_slot);
        // (no branch around the load: it would be waited for before the length is asked for)
        whole_id = *(a.last_block >= 0 ? a.table + (int64_t)at.s * a.table_stride + min(b, a.last_block) : a.ctx_lens);
        const int n = a.ctx_lens[at.s];
        known = n;
        if (n <= 0 || a.last_block < 0) {   // zeros
            for (int i = tid; i < G * D / 8; i += kThreads)
                reinterpret_cast<kv_u32x4*>(a.out + ((int64_t)at.s * v.n_q_local + at.set * G) * D)[i] = kv_u32x4{0u, 0u, 0u, 0u};
            return;
        }
        to = {at.s, at.set, steps_of(n, kStep)};
    } else {
        // every wavefront for itself, four lengths a lane: no barrier stands between the lengths and the first tiles
        const axis_run first = run_of(a, 0, lane, kStep);
        int all = __builtin_amdgcn_readlane(first.sum_incl, 63), some = __builtin_amdgcn_readlane(first.some_incl, 63);
        for (int s0 = 256; s0 < a.batch; s0 += 256) {
            const axis_run r = run_of(a, s0, lane, kStep);
            all += __builtin_amdgcn_readlane(r.sum_incl, 63);
            some += __builtin_amdgcn_readlane(r.some_incl, 63);
        }
        all *= a.head_sets;
        some *= a.head_sets;
        // (no workgroup without a step among those that have some: the pieces of a pair lie in consecutive ones)
        const int W = min((int)gridDim.x, all), i = (int)blockIdx.x;
        if (i >= W) return;
        const int least = (1 << a.unit_shift) + a.start_units;
        const int start_units = (all << a.unit_shift) + a.start_units * some >= 3 * least * W ? a.start_units : 0;
        const int total = (all << a.unit_shift) + start_units * some;
        auto cut = [&](int k) -> int {
            return k == W ? total : W == all ? k << a.unit_shift : (int)(((uint64_t)(uint32_t)total * ((uint32_t)k * a.inverse)) >> 32);
        };
        const int from = cut(i), until = cut(i + 1);
        if (a.batch <= 256) {
            at = place_in(a, first, 0, from, start_units, lane);
            to = place_in(a, first, 0, until == total ? 0 : until, start_units, lane);
            if (until == total) to = {a.batch, 0, 0};
            known = length_in(first, at.s, 0);
        } else {
            at = place_at(a, first, from, start_units, lane, kStep);
            to = place_at(a, first, until, start_units, lane, kStep);
        }
    }

    const uint32_t row_bytes = (uint32_t)v.token_stride;
    for (; at.s < a.batch; at.step = 0, ++at.set, at.s += at.set == a.head_sets, at.set = at.set == a.head_sets ? 0 : at.set) {
        const int s = at.s, set = at.set, step = at.step;
        const int n = known >= 0 ? known : uniform(a.ctx_lens[s]), steps = steps_of(n, kStep);
        known = -1;
        const bool last_pair = s == to.s && set == to.set;
        const int end = last_pair ? to.step : steps;
        if (step >= end) {   // (a sequence without tokens, a start at a pair's end, an end at its start)
            if (last_pair) break;
            continue;
        }
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

        const int t_first = step * kStep + sub * kTile, t_end = min(end * kStep, n);
        // WHOLE: where the groups lie, and (asked for beside the first tile) their scales
        uint64_t whole_at = 0;
        float whole_k = 0.f, whole_v = 0.f;
        auto group_of = [&](int t) -> int { return t / kStep * 2 + (t >> 4 & 1); };   // the lane that has it
        if constexpr (WHOLE)
            whole_at = reinterpret_cast<uint64_t>(a.pool) + (uint64_t)(whole_id * v.block_elems + (int64_t)whole_slot * row_bytes + v.head_off + h * D);
        struct tile {
            kv_u32x4 k[2][kLoads];
            uint32_t v[8][kWords];
            float sk[2], sv[2];
        };
        // Tokens past the end are replaced by the last one of its 16 (finite, masked later).
        // WHOLE: no branch is in the way where there is no tile at t0, and nothing is read: the descriptor is of no bytes.  (Loads behind a branch are
        // waited for as if they were not there, and with them the tile before.  Where pairs are cut that costs nothing, 2048 wavefronts have
        // enough under way, and ordinary loads behind a branch are 2 % faster than these.)
        auto request = [&](int t0, tile& x) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int t = min(t0 + 16 * half, last16), most = n - 1 - t;   // the last row that there is
                const uint32_t kr = (uint32_t)min(m, most) * row_bytes + 16 * g;
                uint32_t vr[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) vr[e] = (uint32_t)min(4 * g + e, most) * row_bytes + kDims * m;
                if constexpr (WHOLE) {
                    const int i = group_of(t), bytes = t0 < t_end ? 0x7ffffff0 : 0;
                    const uint64_t at = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)whole_at, i) |
                                        (uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(whole_at >> 32), i) << 32;
                    const __amdgpu_buffer_rsrc_t kb = __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(at), 0, bytes, 0x00020000);
                    const __amdgpu_buffer_rsrc_t vb =
                        __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<char*>(at + (uint64_t)v.plane_elems), 0, bytes, 0x00020000);
                    constexpr int kPast = 2;   // (non-temporal)
#pragma unroll
                    for (int i = 0; i < kLoads; ++i) x.k[half][i] = __builtin_amdgcn_raw_buffer_load_b128(kb, kr + 64 * i, 0, kPast);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (kWords == 2) {
                            const kv_u32x2 y = __builtin_bit_cast(kv_u32x2, __builtin_amdgcn_raw_buffer_load_b64(vb, vr[e], 0, kPast));
                            x.v[4 * half + e][0] = y[0];
                            x.v[4 * half + e][1] = y[1];
                        } else {
                            x.v[4 * half + e][0] = __builtin_amdgcn_raw_buffer_load_b32(vb, vr[e], 0, kPast);
                        }
                    }
                } else {
                    int b, slot;
                    kv_split_token(v, t, b, slot);
                    const int64_t id = ids[b];
                    const global_bytes kb = (global_bytes)(reinterpret_cast<uint64_t>(a.pool) +
                                                           (uint64_t)(id * v.block_elems + (int64_t)slot * row_bytes + v.head_off + h * D));
                    const global_bytes vb = kb + v.plane_elems;
#pragma unroll
                    for (int i = 0; i < kLoads; ++i)
                        x.k[half][i] = __builtin_nontemporal_load((const __attribute__((address_space(1))) kv_u32x4*)(kb + kr + 64 * i));
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (kWords == 2) {
                            const kv_u32x2 y = __builtin_nontemporal_load((const __attribute__((address_space(1))) kv_u32x2*)(vb + vr[e]));
                            x.v[4 * half + e][0] = y[0];
                            x.v[4 * half + e][1] = y[1];
                        } else {
                            x.v[4 * half + e][0] = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint32_t*)(vb + vr[e]));
                        }
                    }
                    const const_floats sc = (const_floats)(a.scales + q8_scale_at(a.x, id, slot, h));
                    x.sk[half] = sc[0];
                    x.sv[half] = sc[a.x.block_scales / 2];
                }
            }
        };
        auto take = [&](int t0, tile& x) {
            if constexpr (WHOLE) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int i = group_of(min(t0 + 16 * half, last16));
                    x.sk[half] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(whole_k), i));
                    x.sv[half] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(whole_v), i));
                }
            }
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
                const float c = (WHOLE ? x.sk[half] : key_scale(x.sk[half])) * a.scale_log2e;
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
            kv_u32x4 pb, pr;   // weights in bf16, and what that rounding left
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float w0 = fast_exp2(u[2 * i] - ref), w1 = fast_exp2(u[2 * i + 1] - ref), sv = x.sv[i >> 1];
                l += w0 + w1;
                pb[i] = pack_bf16x2(w0 * sv, w1 * sv);
                pr[i] = pack_bf16x2(w0 * sv - __uint_as_float(pb[i] << 16), w1 * sv - __uint_as_float(pb[i] & 0xffff0000u));
            }
#pragma unroll
            for (int w = 0; w < kWords; ++w) {
                uint32_t t[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) t[e] = x.v[e][w];
                bf16x8 va[4];
                dims_of<FMT>(t, va);
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    o[4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[b], as_bf16x8(pr), o[4 * w + b], 0, 0, 0);
                    o[4 * w + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va[b], as_bf16x8(pb), o[4 * w + b], 0, 0, 0);
                }
            }
        };
        if (t_first < t_end) {
            int t = t_first;
            tile x, y;
            request(t, x);
            if constexpr (WHOLE) {
                // scales (a lane without tokens takes any)
                const float* sc = whole_t <= last16 ? a.scales + q8_scale_at(a.x, whole_id, whole_slot, h) : a.scales;
                whole_k = sc[0];
                whole_v = sc[a.x.block_scales / 2];
                __builtin_amdgcn_sched_barrier(0);   // (in this order: the loop waits for the last of x on the way into it as in it)
                request(t + kStep, y);
                asm volatile("" : "+v"(whole_k), "+v"(whole_v));   // (waited for here and not in the loop)
                whole_k = key_scale(whole_k);
                // (one way out of the loop: with a second one between the tiles, loads on the way to it are waited for as if they were not there)
                for (; t + kStep < t_end; t += 2 * kStep) {
                    __builtin_amdgcn_sched_barrier(0);
                    take(t, x);
                    request(t + 2 * kStep, x);
                    __builtin_amdgcn_sched_barrier(0);
                    take(t + kStep, y);
                    request(t + 3 * kStep, y);
                }
                if (t < t_end) take(t, x);
            } else {
                for (;;) {
                    if (t + kStep < t_end) request(t + kStep, y);
                    __builtin_amdgcn_sched_barrier(0);   // (all of the next tile is asked for before anything waits for this one)
                    take(t, x);
                    t += kStep;
                    if (t >= t_end) break;
                    if (t + kStep < t_end) request(t + kStep, x);
                    __builtin_amdgcn_sched_barrier(0);
                    take(t, y);
                    t += kStep;
                    if (t >= t_end) break;
                }
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
            if (WHOLE || (starts && ends)) {
                const float inv = 1.f / sum;
                *reinterpret_cast<kv_u32x2*>(a.out + ((int64_t)s * v.n_q_local + set * rows + row) * D + 4 * d4) =
                    kv_u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
            } else {
                *reinterpret_cast<f32x4*>(a.part_o + (slot * rows + row) * D + 4 * d4) = acc;
                if (d4 == 0) *reinterpret_cast<float2*>(a.part_ml + (slot * rows + row) * 2) = make_float2(top, sum);
            }
        }
        if (!WHOLE && tid == 0) {
            if (starts) a.ends[pair].x = blockIdx.x;
            if (ends) a.ends[pair].y = blockIdx.x;
        }
        if (WHOLE || last_pair) break;
        __syncthreads();
    }
}

// A row of a cut pair: the sum of its pieces; zeros where the sequence has no tokens.  D / 4 lanes a slice of the list of pieces, BATCH pieces of each
// requested at a time, the slices then over LDS.  WAVES: of a row.
template <int D, int WAVES, int BATCH>
__global__ __launch_bounds__(64 * WAVES) void merge_q8_kernel(decode_args a, int rows)
{
    constexpr int kLanes = D / 4, kSlices = 64 / kLanes * WAVES, kBatch = BATCH;
    __shared__ f32x4 s_o[WAVES][kLanes];
    __shared__ float2 s_ml[WAVES];
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int pair = blockIdx.x, row = blockIdx.y, s = pair / a.head_sets, set = pair - s * a.head_sets;
    const int slice = threadIdx.x / kLanes, d4 = lane % kLanes;
    kv_u32x2* const out = reinterpret_cast<kv_u32x2*>(a.out + ((int64_t)s * a.v.n_q_local + set * rows + row) * D + 4 * d4);
    const int n = a.ctx_lens[s], first = a.ends[pair].x, last = a.ends[pair].y;   // (one trip for all)
    if (n <= 0) {
        if (slice == 0) *out = kv_u32x2{0u, 0u};
        return;
    }
    if (first == last) return;
    float top = kLowest, sum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float m, float l, const f32x4& o, float to) {
        const float f = fast_exp2(m - to);
        sum += l * f;
        acc += o * f;
    };
    for (int w0 = first + slice; w0 <= last; w0 += kBatch * kSlices) {
        float2 ml[kBatch];
        f32x4 o[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {   // (past the end: the last one again, not used)
            const int w = min(w0 + u * kSlices, last);
            const int64_t rec = (2 * (int64_t)w + (w == first ? 1 : 0)) * rows + row;
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + rec * 2);
            o[u] = *reinterpret_cast<const f32x4*>(a.part_o + rec * D + 4 * d4);
        }
        float to = top;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (w0 + u * kSlices > last) ml[u] = make_float2(kLowest, 0.f);
            to = fmaxf(to, ml[u].x);
        }
        const float keep = fast_exp2(top - to);
        acc *= keep;
        sum *= keep;
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (w0 + u * kSlices <= last) add(ml[u].x, ml[u].y, o[u], to);
        top = to;
    }
    // the wavefront's slices, then the wavefronts
#pragma unroll
    for (int d = kLanes; d < 64; d *= 2) {
        const float m = __shfl_xor(top, d), l = __shfl_xor(sum, d), to = fmaxf(top, m);
        const f32x4 o = {__shfl_xor(acc[0], d), __shfl_xor(acc[1], d), __shfl_xor(acc[2], d), __shfl_xor(acc[3], d)};
        const float keep = fast_exp2(top - to);
        acc *= keep;
        sum *= keep;
        add(m, l, o, to);
        top = to;
    }
    if (lane < kLanes) s_o[wave][d4] = acc;
    if (lane == 0) s_ml[wave] = make_float2(top, sum);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) top = fmaxf(top, s_ml[i].x);
    sum = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < WAVES; ++i) add(s_ml[i].x, s_ml[i].y, s_o[i][d4], top);
    const float inv = 1.f / sum;
    if (lane < kLanes) *out = kv_u32x2{pack_bf16x2(acc[0] * inv, acc[1] * inv), pack_bf16x2(acc[2] * inv, acc[3] * inv)};
}

constexpr int kMostWaves = 2048;   // two for each SIMD of 256 compute units
constexpr int kUnitShift = 3, kStartUnits = 8;   // a start counts as much as a step
// Up to which bound of the lengths a workgroup takes a whole pair: cutting costs a second launch, 4 us and more, and pieces to write and read;
// not cutting leaves a workgroup 0.8 us for each 128 tokens, and from 256 pairs on compute units with two.  (Lengths from 0.3 of the bound to it, us
// whole and cut: 16 pairs, 700: 7.4, 9.8; 1000: 10.2, 9.9; 96 pairs, 1000: 11.3, 14.3; 192 pairs, 1000: 15.7, 18.9; 1700: 23.7, 21.4; 384 pairs, 500:
// 14.4, 16.0; 700: 19.2, 19.2; 1000: 25.9, 23.9; 768 pairs, 500: 21.2, 24.5; 700: 27.8, 27.4; 1520 pairs, 300: 25.4, 27.3; 500: 36.6, 34.6.
// Between 256 and about 400 the rule loses up to 7 % for more than 1024 pairs: 1520 pairs at 300.)
int whole_bound(int64_t pairs) { return pairs >= 96 && pairs <= 256 ? 1024 : pairs <= 512 ? 704 : pairs <= 1024 ? 512 : 256; }
constexpr int kLeastCut = 256;   // no pair is cut up to this bound

// How a call is cut: the same for the workspace and the launch.
struct decode_plan {
    int hpw, head_sets, workgroups;
    bool whole;
    size_t o_bytes, ml_bytes, bytes;
};
int step_tokens(int hpw) { return kTile * waves_of(hpw) / hpw; }
decode_plan plan_of(const kv_view* view, int batch, int max_ctx_len)
{
    decode_plan p;
    const int hl = view->n_kv_local;
    p.hpw = hl % 8 == 0 ? 8 : hl % 4 == 0 ? 4 : hl % 2 == 0 ? 2 : 1;
    // (the room asked for does not depend on it: what serves large calls is to serve all smaller ones)
    const bool never_cut = max_ctx_len <= kLeastCut;   // (and there is no room for pieces)
    p.whole = never_cut || max_ctx_len <= whole_bound((int64_t)batch * hl);
    p.head_sets = hl / p.hpw;
    const int step = step_tokens(p.hpw);
    const int64_t pairs = (int64_t)batch * p.head_sets, steps = pairs * (((int64_t)max_ctx_len + step - 1) / step);
    p.workgroups = (int)std::min<int64_t>(steps, kMostWaves / waves_of(p.hpw));
    const int rows = p.hpw * view->group;
    p.o_bytes = never_cut ? 0 : (size_t)2 * p.workgroups * rows * view->geom.head_dim * 4;
    p.ml_bytes = never_cut ? 0 : (size_t)2 * p.workgroups * rows * 8;
    p.bytes = never_cut ? 0 : p.o_bytes + p.ml_bytes + (size_t)pairs * sizeof(int2);
    if (p.whole) {
        p.hpw = 1;
        p.head_sets = hl;
        p.workgroups = batch * hl;
    }
    return p;
}

template <int D, int FMT>
void launch(const decode_plan& p, const decode_args& a, hipStream_t st)
{
    auto* f = p.whole      ? decode_q8_kernel<D, FMT, 1, true>
              : p.hpw == 8 ? decode_q8_kernel<D, FMT, 8, false>
              : p.hpw == 4 ? decode_q8_kernel<D, FMT, 4, false>
              : p.hpw == 2 ? decode_q8_kernel<D, FMT, 2, false>
                           : decode_q8_kernel<D, FMT, 1, false>;
    hipLaunchKernelGGL(f, dim3((unsigned)p.workgroups), dim3(64 * waves_of(p.hpw)), 0, st, a);
    if (!p.whole) {
        const int pairs = a.batch * p.head_sets, rows = p.hpw * a.group;
        // By the pieces of a pair, where all are alike.  One of 20000 tokens, 8 heads, 256 pieces: 16.5 us, with 4 wavefronts a row 27; 9 of 600 to 4700, one
        // head, 57 pieces: 9.8, as many with 4, with one piece at a time 10.4; 256 around 1024, 2 pieces: 44.4, with four at a time 45.5.
        // (One long sequence among many short ones has far more pieces than this average, and its list is walked one piece at a time: 64 of 100 to 1000
        // tokens, one head, 9.4 us, with 131072 tokens in place of one of them 32.3.)
        const int pieces = p.workgroups / pairs;
        auto* f = pieces > 32 ? merge_q8_kernel<D, 16, 4> : pieces > 8 ? merge_q8_kernel<D, 4, 4> : merge_q8_kernel<D, 4, 1>;
        hipLaunchKernelGGL(f, dim3((unsigned)pairs, (unsigned)rows), dim3(pieces > 32 ? 1024 : 256), 0, st, a, rows);
    }
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
    a.last_block = max_ctx_len > 0 ? (max_ctx_len - 1) / view->block_tokens : -1;
    // (32 bits hold the axis: bounds that would pass them are cut by whole steps)
    const bool fine = (double)batch * p.head_sets * (max_ctx_len / step_tokens(p.hpw) + 2.0) < (double)(1 << 26);
    a.unit_shift = fine ? kUnitShift : 0;
    a.start_units = fine ? kStartUnits : 0;
    a.inverse = (uint32_t)((1ull << 32) / (unsigned)p.workgroups);
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
