// Attention of few query rows per sequence to a paged KV pool through a layout view, in two entry points that share a kernel:
//
//   paged_tree_attn            the last q_len tokens of a sequence are drafted; each sees everything before them and the
//                              drafted tokens that its mask names (its ancestors in a tree, and itself)
//   paged_decode_attn_weights  one query token per sequence; besides the output, the attention weight that every cached
//                              token got is added to a running sum per KV head
//
// A pair is (sequence, local KV head, block of 32 RW query rows), its rows being the sequence's new tokens x the G query
// heads of the KV head; a tile is 32 cached tokens of a pair.  The tiles of one head lie on one axis that is cut into equal
// shares, so that the work is even whatever the lengths.  A team of workgroups takes a share for all heads, so that the
// whole row of a token is asked for at about one time (64 sequences of 512 to 4096, 8 heads, drafts of up to 8: 128 us in place of
// 145).  A pair that lies in one share is finished there, the pieces of a cut one leave (reference, sum of weights, sums of values)
// in the workspace for a second launch.
//
// What bounds it: reading K and V, 4 D bytes a token and KV head, as long as the rows are few: 32 rows x 32 keys take
// 2 D / 16 + 2 D / 16 products of 32 x 32 x 16, 512 cycles at D = 128, and bring 16 KiB, for which HBM takes 1440 cycles of one
// compute unit's share.  RW wavefronts share a tile, each with 32 rows: K and V pass through LDS once per workgroup.  Four of them
// (RW = 4) are the general form, two workgroups of which fill a compute unit, also where rows leave some without work: a piece asks for its
// first four tiles at once.  Every later step asks for one tile more and ends with a barrier, at which the compiler waits for all loads into
// LDS, so that one tile is under way beside the one in hand.  Large batches of up to 64 rows take the wavefronts for other heads (HW = 4
// or 2), which reads rows of several heads in one piece; large ones of many rows have eight to a tile (RW = 8).  With sums of weights
// there are 32 rows, and where heads are not side by side the wavefronts take different tiles (KW = 4) and each stores its scores.
//
// Reached: 64 sequences of 512 to 4096, 8 heads of 128, drafts of up to 8 tokens 108 us (5.7 TB/s), up to 16 124, up to 32 145, 33 to
// 64 200.  With 256 rows a tile takes 1.1 us of a compute unit, of which the products are 0.43 at the matrix units' rate and the
// vector instructions of the softmax 0.45 (75 of 4 cycles and 16 exponentials of 16 for each wavefront): they overlap in part only.
//
// Per tile, lane l = (c = l % 32, half = l / 32):
//   S^T[token][c] = K[token][:] . q[c][:]     A operand = K rows from LDS, B operand = q
//   O^T[e][c]     = sum_t V[t][e] P[c][t]     A operand = V^T by the transposing LDS read
// Weights of drafted rows enter the second product in bf16, the type of the values that the matrix units multiply them with: off by 2^-8 of
// themselves at most, each on its own, against one rounding of the output (measured against 64 bits, 2-norms: 2.3e-3 with, 1.7e-3 with
// weights of 32 bits, of which 1.7e-3 is the output's own rounding).  What the rounding leaves out as a second operand would take four drafts of
// up to 256 102 us in place of 81, 32 of up to 64 107 in place of 92.  With sums of weights, which are handed out in 32 bits, it is added (64
// sequences of 512 to 4096 141.6 us in place of 139.9, four of up to 300 12.9 in place of 12.7): the output then is that of these weights,
// 2^-16 off.  All sums are fp32.
// Register 4 a + i of S^T holds token 8 a + 4 half + i; contraction index 8 half + 4 a' + i of step c' of the second product
// stands for token 16 c' + 8 a' + 4 half + i, so weights stay in their lane.
#include <algorithm>
#include <type_traits>

#include "decode_common.h"

using namespace kvdec;

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short bits16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bits16x4* lds_bits16x4_ptr;
typedef __attribute__((address_space(3))) void* lds_ptr;

constexpr int kKeys = 32;
constexpr float kUnset = 1e30f;   // exponent addend of a column that has seen no key yet
constexpr int kCus = 256;
// Tiles that take as long as starting and ending a piece.  us per call, shares of even length wherever those of the least do not fit / pieces
// longer than even ones by up to so many: 8 heads, 4 sequences of 2000 to 4000, drafts of up to 8 20.4 / 18.6, with sums 27.0 / 22.5; 2 of 1000
// to 8000, drafts of 150 to 256 54.0 / 46.1, 8 of them with drafts of 33 to 64 59.7 / 54.0.  Eight tiles: the same.
constexpr int kPieceTiles = 4;
constexpr int kMostNodes = 256;   // drafted tokens of a sequence
constexpr int kEdgeTiles = kMostNodes / kKeys + 1;   // tiles that they lie in

// Scores leave in four passes over 8 of 32 rows (tile x in hand, query head g): row r is x = r >> s, g = r & ((1 << s) - 1), s the log2 of the
// group rounded up.  The compiler branches around a pass in which no lane has a head: how many of the four store.
constexpr int passes_with_heads(int group)
{
    int s = 0, n = 0;
    while ((1 << s) < group) ++s;
    for (int r0 = 0; r0 < 32; r0 += 8) {
        bool any = false;
        for (int r = r0; r < r0 + 8; ++r) any = any || (r & ((1 << s) - 1)) < group;
        n += any;
    }
    return n;
}
constexpr int kMostGroup = 32;
__host__ __device__ constexpr bool stores_four(int group) { return group <= 16 || group > 24; }
constexpr bool stores_four_holds()
{
    for (int group = 1; group <= kMostGroup; ++group)
        if (stores_four(group) != (passes_with_heads(group) == 4)) return false;
    return true;
}
static_assert(stores_four_holds(), "a wait that leaves four stores under way needs four stores");

struct tree_args {
    const uint16_t* q;        // [total_q][n_q_local][D]
    uint16_t* out;
    const uint16_t* pool;
    const int32_t* table;
    int64_t table_stride;
    const int32_t* ctx_lens;
    const int32_t* q_off;     // [batch + 1], or null: one query token per sequence
    const unsigned long long* mask;   // [total_q][mask_words]
    kv_view_dev v;
    uint32_t last_block;      // n_pool_blocks - 1
    float scale_log2e;
    int32_t group, batch, max_ctx_len, max_q_len, mask_words;
    int32_t few;              // up to 64 sequences, and their tiles are counted in 32 bits
    int32_t group_shift;      // log2 of the group rounded up to a power of two
    int32_t teams, least_tiles;   // shares that the axis of tiles is cut into, and the least tiles of a share
    f32x4* part_o;            // [2 teams n_kv_local][RW][D / 8][64]: slot 2 w a piece of workgroup w that goes on a pair, 2 w + 1 one that begins it
    float* part_ml;           // [2 teams n_kv_local][32 RW][2] (reference in exponent units, sum of weights)
    int2* ends;               // [batch][blocks][n_kv_local] of every pair: the teams of its first and last piece
    int32_t most_blocks;      // row blocks of a sequence by the host's bound
    // weights:
    float* scores;            // [batch][n_q_local][score_stride] exponents: score * scale * log2(e)
    float* row_ml;            // [batch][n_q_local][2] of pairs that were not cut
    float* sums;              // [batch][n_kv_local][sum_stride]
    int64_t score_stride, sum_stride;
    int32_t chunk;            // tokens per workgroup of the launch that adds up weights
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform64(int64_t x)
{
    return (int64_t)((uint64_t)(uint32_t)uniform((int)x) | (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32);
}

// Sums over the lanes up to each one: within rows of 16, then of the row before, then of the 32 lanes before.
__device__ __forceinline__ int lane_sums(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, true);    // row_shr:1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, true);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15, 31
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
// Maximum / sum over the two lanes of a column, left in both.
__device__ __forceinline__ float half_max(float x)
{
    const uint32_t c = __builtin_bit_cast(uint32_t, x);
    const auto h = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    const uint32_t h0 = h[0], h1 = h[1];
    return fmaxf(__builtin_bit_cast(float, h0), __builtin_bit_cast(float, h1));
}
__device__ __forceinline__ float half_sum(float x)
{
    const uint32_t c = __builtin_bit_cast(uint32_t, x);
    const auto h = __builtin_amdgcn_permlane32_swap(c, c, false, false);
    const uint32_t h0 = h[0], h1 = h[1];
    return __builtin_bit_cast(float, h0) + __builtin_bit_cast(float, h1);
}
__device__ __forceinline__ float column_max(const f32x16& x)
{
    float mx = x[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, x[i]);
    return half_max(mx);
}
// l + the two bf16 values of a packed pair, summed in fp32.
__device__ __forceinline__ float add_pair(uint32_t packed, float l)
{
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, packed), __builtin_bit_cast(bf16x2, 0x3f803f80u), l, false);
}
// Whether one of the two bf16 values is an infinity or NaN.
__device__ __forceinline__ bool not_finite(uint32_t x)
{
    return (x & 0x7f800000u) == 0x7f800000u || (x & 0x7f80u) == 0x7f80u;
}

// What a sequence brings: cached tokens, new ones, tiles of a pair, row blocks of a head.
struct seq_work {
    int n, q0, q_len, tiles, blocks;
    __device__ int64_t total() const { return (int64_t)tiles * blocks; }   // of a head
};
template <int RB>
__device__ __forceinline__ seq_work work_of(const tree_args& a, int s)
{
    seq_work w;
    w.n = min(a.ctx_lens[s], a.max_ctx_len);
    w.q0 = a.q_off ? a.q_off[s] : s;
    w.q_len = a.q_off ? min(a.q_off[s + 1] - w.q0, a.max_q_len) : 1;
    if (a.q_off && w.n > 0) w.q_len = min(w.q_len, w.n);   // (both bounds are the caller's to keep; no address depends on it)
    const bool any = w.n > 0 && w.q_len > 0;
    w.tiles = any ? (w.n + kKeys - 1) / kKeys : 0;
    w.blocks = any ? (w.q_len * a.group + RB - 1) / RB : 0;
    return w;
}
__device__ __forceinline__ int64_t share_of(const tree_args& a, int64_t total)
{
    const int64_t even = (total + a.teams - 1) / a.teams;
    return even > a.least_tiles ? even : a.least_tiles;
}

// The share of this team: [from, to) on the axis, the sequence that holds `from` and its offset in it.
template <int NT, int RB>
__device__ __forceinline__ void find_share(const tree_args& a, int team, int64_t* s_sum, int64_t& from, int64_t& to, int& seq, int64_t& offset)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int each = (a.batch + NT - 1) / NT, s0 = min(tid * each, a.batch), s1 = min(s0 + each, a.batch);
    int64_t mine = 0;
    for (int s = s0; s < s1; ++s) mine += work_of<RB>(a, s).total();
    int64_t incl = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t y = __shfl_up((long long)incl, d);
        incl += lane >= d ? y : 0;
    }
    if (lane == 63) s_sum[wave] = incl;
    __syncthreads();
    int64_t total = 0, before = incl - mine;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        total += s_sum[w];
        before += w < wave ? s_sum[w] : 0;
    }
    const int64_t share = share_of(a, total);
    from = (int64_t)team * share;
    to = min(from + share, total);
    __syncthreads();
    if (from >= before && from < before + mine) {   // one thread at most
        int s = s0;
        for (int64_t w; from >= before + (w = work_of<RB>(a, s).total()); ++s) before += w;
        s_sum[0] = s;
        s_sum[1] = from - before;
    }
    __syncthreads();
    seq = uniform((int)s_sum[0]);
    offset = uniform64(s_sum[1]);
    __syncthreads();
}


template <int D, int RW, int HW, bool SUMS>
__global__ __launch_bounds__(RW == 8 ? 512 : 256, 2) void tree_kernel(tree_args a)
{
    constexpr int NW = RW < 4 ? 4 : RW, KW = NW / (RW * HW), NT = 64 * NW, RB = 32 * RW;
    constexpr int NJ = D / 32, NK = D / 16, kRow = 2 * D, kStride = HW * kRow;   // bytes of a token's row, and of the heads' rows in LDS
    constexpr int kPieces = kKeys * kStride / 16;                                 // of a staged tile, K or V
    constexpr bool kShared = RW * HW > 1;                                         // wavefronts share what is staged
    // K: piece c of row t at c ^ f(t), V: at c ^ g(t): operand reads without bank conflicts.  An array per buffer: the compiler
    // then knows that loads landing in one do not touch the operands read from another.
    constexpr int NB = RW >= 4 ? 4 : 2, kMore = NB > 2 ? KW * kPieces : 1;
    __shared__ kv_u32x4 s_k0[KW * kPieces], s_k1[KW * kPieces], s_v0[KW * kPieces], s_v1[KW * kPieces];
    __shared__ kv_u32x4 s_k2[kMore], s_k3[kMore], s_v2[kMore], s_v3[kMore];
    auto k_buf = [&](int x) { return NB == 2 ? ((x & 1) ? s_k1 : s_k0) : (x & 2) ? ((x & 1) ? s_k3 : s_k2) : ((x & 1) ? s_k1 : s_k0); };
    auto v_buf = [&](int x) { return NB == 2 ? ((x & 1) ? s_v1 : s_v0) : (x & 2) ? ((x & 1) ? s_v3 : s_v2) : ((x & 1) ? s_v1 : s_v0); };
    __shared__ float2 s_ml[KW > 1 ? NW * 32 : 1];
    __shared__ uint32_t s_seen[SUMS ? 1 : kEdgeTiles][SUMS ? 1 : RB];   // which tokens of the tiles that hold drafted ones a row sees
    __shared__ f32x4 s_out[SUMS ? NW : 1][SUMS ? 32 : 1][8];   // scores on their way out
    __shared__ int64_t s_sum[NW];

    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const int rw = wave % RW, kg = wave / RW % KW, hw = wave / (RW * KW);   // the wavefront's rows, tiles and head
    const int col = lane & 31, half = lane >> 5;
    const kv_view_dev& v = a.v;
    const int G = a.group, Hl = v.n_kv_local;

    const int sets = Hl / HW, team = (int)blockIdx.x / sets, h0 = ((int)blockIdx.x - team * sets) * HW, h = h0 + hw;
    int64_t from, to, offset;
    int s;
    // Up to 64 sequences a wavefront holds in its lanes and finds its share by itself: one trip to memory, no barriers
    const bool few = a.few != 0;
    seq_work lane_work = {0, 0, 0, 0, 0};
    if (few) {
        if (lane < a.batch) lane_work = work_of<RB>(a, lane);
        const int here = lane_work.tiles * lane_work.blocks, incl_here = lane_sums(here);
        const int total = __builtin_amdgcn_readlane(incl_here, 63), share = (int)share_of(a, total);
        // Where shares that each end with their pair are enough for the teams, a team has one piece, if they are not longer than even
        // ones by more than what a workgroup does before its first tile and after its last comes to
        int length = share, incl = 0, each = 0;
        bool fits = false;
        for (; length <= share + kPieceTiles; ++length) {
            each = (lane_work.tiles + length - 1) / length;
            incl = lane_sums(each * lane_work.blocks);
            fits = __builtin_amdgcn_readlane(incl, 63) <= a.teams;
            if (fits) break;
        }
        if (fits) {
            if (team >= __builtin_amdgcn_readlane(incl, 63)) return;
            s = __builtin_popcountll(__builtin_amdgcn_ballot_w64(incl <= team));
            const int unit = team - __builtin_amdgcn_readlane(incl - each * lane_work.blocks, s), e = __builtin_amdgcn_readlane(each, s);
            const int tiles = __builtin_amdgcn_readlane(lane_work.tiles, s), at = (unit % e) * length;
            offset = (int64_t)(unit / e) * tiles + at;
            from = 0;
            to = min(length, tiles - at);
        } else {
            from = (int64_t)team * share;
            to = min(from + share, (int64_t)total);
            s = min(__builtin_popcountll(__builtin_amdgcn_ballot_w64(incl_here <= from)), 63);
            offset = from - __builtin_amdgcn_readlane(incl_here - here, s);
        }
    } else {
        find_share<NT, RB>(a, team, s_sum, from, to, s, offset);
    }
    auto sequence = [&](int x) {
        if (!few) return work_of<RB>(a, x);
        return seq_work{__builtin_amdgcn_readlane(lane_work.n, x), __builtin_amdgcn_readlane(lane_work.q0, x),
                        __builtin_amdgcn_readlane(lane_work.q_len, x), __builtin_amdgcn_readlane(lane_work.tiles, x),
                        __builtin_amdgcn_readlane(lane_work.blocks, x)};
    };

    // ---- what does not change from piece to piece -------------------------------------------------
    const int64_t stride_bytes = (int64_t)v.token_stride * 2, block_bytes = v.block_elems * 2, plane_bytes = v.plane_elems * 2;
    const int groups_per_block = v.block_tokens >> 4;
    // staging: one instruction fills 64 consecutive pieces of 16 bytes, 512 / D rows; a wavefront fills NP of the D / 16
    // such parts of K and of V (at D = 64 under RW = 8 the lower four wavefronts K, the others V)
    constexpr bool kSplitPlanes = NK < RW;
    constexpr int NP = kSplitPlanes ? 1 : NK / RW;
    constexpr int kTokenPieces = kStride / 16, kRowsEach = 64 / kTokenPieces;
    const int first_part = kSplitPlanes ? (rw & (NK - 1)) : (hw * RW + rw) * NP;
    // (rows of 128 bytes fill half the banks: with four heads side by side odd tokens have the heads of a pair exchanged)
    auto head_place = [](int head, int token) { return D == 64 && HW > 1 ? head ^ (token & 1) : head; };
    uint32_t k_lane[NP], v_lane[NP];
    const int row_first = (first_part * kRowsEach & 15) + lane / kTokenPieces;   // within a group, of the first part
#pragma unroll
    for (int i = 0; i < NP; ++i) {
        const int row = ((first_part + i) * kRowsEach + lane / kTokenPieces) & 15, c = lane & (D / 8 - 1);
        const int head = head_place(lane % kTokenPieces / (D / 8), row) * (D / 8);
        const int kc = D == 128 ? c ^ row : c ^ (row >> 1), vc = D == 128 ? c ^ (4 * (row & 3)) : c ^ (4 * ((row >> 1) & 1));
        k_lane[i] = (uint32_t)(row * (int)stride_bytes + ((head + kc) << 4));
        v_lane[i] = (uint32_t)(row * (int)stride_bytes + ((head + vc) << 4));
    }
    uint32_t k_off, v_off[NJ];
    {
        const int p = lane & 15, sub = (lane >> 4) & 1;
        k_off = (uint32_t)(kg * kPieces * 16 + col * kStride + head_place(hw, col) * kRow + ((half ^ (D == 128 ? (col & 15) : ((col >> 1) & 7))) << 4));
        const int vrow = 4 * half + (p >> 2), g = D == 128 ? 4 * (vrow & 3) : 4 * ((vrow >> 1) & 1);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            v_off[j] = (uint32_t)(kg * kPieces * 16 + vrow * kStride + head_place(hw, vrow) * kRow + (((4 * j + 2 * sub + ((p & 3) >> 1)) ^ g) << 4) + (p & 1) * 8);
    }

    for (int64_t at = from; at < to;) {
        // ---- the next piece: tiles [t0, t0 + count) of block rb of sequence s -----------------------------
        const seq_work w = sequence(s);
        if (offset >= w.total()) {
            offset -= w.total();
            ++s;
            continue;
        }
        const int rb = uniform((int)(offset / w.tiles)), t0 = uniform((int)(offset - (int64_t)rb * w.tiles));
        const int count = (int)min((int64_t)(w.tiles - t0), to - at);
        const bool cut = count < w.tiles;
        at += count;
        offset += count;
        const int n = w.n, first = n - w.q_len;          // the first drafted token
        const int rows = min(w.q_len * G - rb * RB, RB);   // of the pair
        const bool idle = rw * 32 >= rows;                 // this wavefront has none of them
        // each key group takes tiles that follow each other: [kt0, kt0 + mine)
        const int mine = count / KW + (kg < count % KW ? 1 : 0), iters = (count + KW - 1) / KW;
        const int kt0 = t0 + kg * (count / KW) + min(kg, count % KW);
        const int last_group = (n - 1) >> 4;

        // where the groups of 16 tokens lie: lane l knows that of group l % 2 of this wavefront's tile 32 window + l / 2
        const int32_t* ids = a.table + (int64_t)s * a.table_stride;
        const char* pool_head = reinterpret_cast<const char*>(a.pool + v.head_off + h0 * D);
        auto group_at = [&](int window) { return min(2 * (kt0 + 32 * window + (lane >> 1)) + (lane & 1), last_group); };
        auto request_ids = [&](int window) { return (uint32_t)ids[group_at(window) / groups_per_block]; };
        auto places = [&](uint32_t id, int window) {
            const int g = group_at(window);
            return (int64_t)min(id, a.last_block) * block_bytes + (int64_t)(g % groups_per_block) * 16 * stride_bytes;
        };
        // Tiles are staged in order, K of a tile before its V: the places of the next tile's groups for each
        struct cursor {
            int i;          // tile that is fetched next
            int64_t place;  // of this window
            uint32_t id;    // of the next
        };
        cursor at_k{0, places(request_ids(0), 0), 0}, at_v;
        at_k.id = request_ids(1);
        const cursor at_start = at_k;
        at_v = at_k;
        // ---- this lane's query row, asked for before the tiles: waits count in order ----------------
        const int rho = rb * RB + min(rw * 32 + col, rows - 1);      // (padding columns repeat the last row)
        const int64_t qrow = (int64_t)(w.q0 + rho / G);
        const int64_t orow = (qrow * v.n_q_local + h * G + rho % G) * D;
        const int srow = rw * 32 + col;
        const bool real = srow < rows;
        bf16x8 qb[NK];
#pragma unroll
        for (int kk = 0; kk < NK; ++kk)
            qb[kk] = as_bf16x8(*reinterpret_cast<const kv_u32x4*>(a.q + orow + half * 8 + kk * 16));

        const int first_edge = (SUMS ? n : first) >> 5;   // tiles from there on hold drafted tokens or the end of the sequence
        if constexpr (!SUMS) {
            if (t0 + count > first_edge) {
                // The windows of 32 tokens that the tiles are, cut out of the rows' mask words; what lies before the draft is seen
                if ((int)threadIdx.x < rows) {
                    const uint32_t* words = reinterpret_cast<const uint32_t*>(a.mask) +
                                            ((int64_t)w.q0 + (rb * RB + (int)threadIdx.x) / G) * 2 * a.mask_words;
                    const int shift = first & 31;
                    uint32_t before = ~0u;
#pragma unroll
                    for (int e = 0; e < kEdgeTiles; ++e) {
                        const int here = n - kKeys * (first_edge + e);   // tokens of the tile that exist
                        if (here <= 0) break;
                        const uint32_t word = e < 2 * a.mask_words ? words[e] : 0u;
                        const uint32_t window = (uint32_t)((((uint64_t)word << 32 | before) << shift) >> 32);
                        s_seen[e][threadIdx.x] = here >= 32 ? window : window & ((1u << here) - 1u);
                        before = word;
                    }
                }
            }
        }

        auto stage = [&](cursor& x, const uint32_t (&at_lane)[NP], int64_t plane, kv_u32x4* dst, auto sure) {
            const int i = x.i++;
            if (!decltype(sure)::value && i >= mine) return;
            if ((i & 31) == 0 && i > 0) {
                x.place = places(x.id, i >> 5);
                x.id = request_ids((i >> 5) + 1);
            }
            const int tile = kt0 + i;
            auto rows_of = [&](int g) {
                const int l = 2 * (i & 31) + g;
                const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)x.place, l);
                const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(x.place >> 32), l);
                return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(pool_head + plane + (int64_t)((uint64_t)lo | (uint64_t)hi << 32)), 0,
                                                         0x7ffffff0, 0x00020000);
            };
            // (a wavefront that fills parts of both groups looks two places up, the others one)
            constexpr bool kBoth = NP * kRowsEach > 16;
            const __amdgpu_buffer_rsrc_t r0 = rows_of(first_part * kRowsEach >> 4), r1 = kBoth ? rows_of(1) : r0;
            auto fill = [&](auto end) {
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    const int g = kBoth ? p * kRowsEach >> 4 : first_part * kRowsEach >> 4;
                    uint32_t off = at_lane[p];
                    if constexpr (decltype(end)::value) {   // rows past the end of the sequence are its last one again (masked later)
                        const int limit = n - 1 - 16 * min(2 * tile + g, last_group), row = (p * kRowsEach & 15) + row_first;
                        off -= (uint32_t)(max((row & 15) - limit, 0) * (int)stride_bytes);
                    }
                    // (non-temporal where one block of rows is all there is; several read the tile again)
                    const __amdgpu_buffer_rsrc_t source = kBoth && g ? r1 : r0;
                    const lds_ptr to_lds = (lds_ptr)(dst + kg * kPieces + (first_part + p) * 64);
                    if (RW < 4 || (RW == 4 && w.blocks == 1)) __builtin_amdgcn_raw_ptr_buffer_load_lds(source, to_lds, 16, off, 0, 0, 2);
                    else __builtin_amdgcn_raw_ptr_buffer_load_lds(source, to_lds, 16, off, 0, 0, 0);
                }
            };
            if (2 * tile + 1 < last_group) fill(std::false_type());
            else fill(std::true_type());
        };
        auto stage_k = [&](kv_u32x4* dst, auto sure) {
            if (!kSplitPlanes || rw < NK) stage(at_k, k_lane, 0, dst, sure);
        };
        auto stage_v = [&](kv_u32x4* dst, auto sure) {
            if (!kSplitPlanes || rw >= NK) stage(at_v, v_lane, plane_bytes, dst, sure);
        };
        // This wavefront's loads have landed, and then those of the wavefronts that share its tiles; but for the last so many.  (In front of a
        // barrier the count holds where the compiler can follow what is under way: in straight code, at the start of a piece under RW = 4.)
        auto staged = [&](auto under_way) {
            constexpr int kLeft = decltype(under_way)::value;
            __builtin_amdgcn_s_waitcnt(0x0f70 | (kLeft & 15) | (kLeft >> 4) << 14);   // vmcnt
            if constexpr (kShared) __syncthreads();
            else asm volatile("" ::: "memory");
        };
        // Of several tiles the first scores need K of two and V of one; the others land beside them
        constexpr int kRing = (NB - 2) * (kSplitPlanes ? 1 : 2) * NP;
        auto start = [&](auto sure) {
#pragma unroll
            for (int x = 0; x < NB - 1; ++x) {
                stage_k(k_buf(x), sure);
                stage_v(v_buf(x), sure);
            }
            stage_k(k_buf(NB - 1), sure);
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) asm volatile("" : "+v"(qb[kk]));   // (q has come before: waited for here, where what is under way is known)
            staged(std::integral_constant<int, decltype(sure)::value ? kRing : 0>());
        };
        if (NB > 2 && mine >= NB) start(std::true_type());
        else start(std::false_type());

        float neg_m, l;
        bool unset;
        f32x16 o[NJ];
        auto clear = [&]() {
            neg_m = kUnset;
            l = 0.f;
            unset = true;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
        };
        clear();

        auto k_operand = [&](const kv_u32x4* sk, int kk) {
            uint32_t off = k_off;   // (opaque: the compiler would keep an offset per step in registers)
            if (kk > 0) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(off) : "i"(32 * kk), "v"(k_off));
            return as_bf16x8(*reinterpret_cast<const kv_u32x4*>(reinterpret_cast<const char*>(sk) + off));
        };
        auto v_operand = [&](const kv_u32x4* sv, int u) {   // u = NJ c + j
            const char* const p = reinterpret_cast<const char*>(sv) + v_off[u % NJ] + (u / NJ) * 16 * kStride;
            const bits16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_bits16x4_ptr)p);
            const bits16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_bits16x4_ptr)(p + 8 * kStride));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        f32x16 sc, ex;    // scores of a tile, then exponents: score scale log2(e) - reference
        uint32_t pw[8], pf[SUMS ? 8 : 1];   // weights, and what their rounding leaves out
        auto zero = [&]() {
            f32x16 x;
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.f;
            return x;
        };
        auto weights = [&](int u) {   // two of the sixteen
            const float e0 = fast_exp2(ex[2 * u]), e1 = fast_exp2(ex[2 * u + 1]);
            pw[u] = pack_bf16x2(e0, e1);
            if constexpr (SUMS) {   // no rounding above or below the fraction
                pf[u] = pack_bf16x2(e0 - bf16_lo(pw[u]), e1 - bf16_hi(pw[u]));
                l += e0 + e1;
            } else {   // the same rounding above and below
                l = add_pair(pw[u], l);
            }
        };
        auto weight_operand = [&](int c) { return as_bf16x8(kv_u32x4{pw[4 * c], pw[4 * c + 1], pw[4 * c + 2], pw[4 * c + 3]}); };
        auto rest_operand = [&](int c) {
            if constexpr (SUMS) return as_bf16x8(kv_u32x4{pf[4 * c], pf[4 * c + 1], pf[4 * c + 2], pf[4 * c + 3]});
            else return bf16x8{};
        };
        // Scores of as many tiles as make 32 rows leave together, through LDS, whole lines at a time.  (The loads of later tiles are
        // counted in order with the stores, whose way out is long: storing every tile's takes 64 sequences of 512 to 4096
        // 131 us in place of 129, at heads of 64 83 in place of 81.)  Returns whether it stored four times,
        // neither fewer nor more: the wait after it leaves as many requests under way.
        auto keep_scores = [&](int i) -> bool {
            if constexpr (SUMS) {
                const int slots = 32 >> a.group_shift, slot = i & (slots - 1);
                if (real) {
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        s_out[wave][(slot << a.group_shift) + col][2 * u + half] =
                            f32x4{sc[4 * u] * a.scale_log2e, sc[4 * u + 1] * a.scale_log2e, sc[4 * u + 2] * a.scale_log2e, sc[4 * u + 3] * a.scale_log2e};
                }
                if (slot < slots - 1 && i < mine - 1) return false;
                float* dst = a.scores + ((int64_t)s * v.n_q_local + h * G) * a.score_stride;
#pragma unroll
                for (int r0 = 0; r0 < 32; r0 += 8) {
                    const int r = r0 + (lane >> 3), x = r >> a.group_shift, g = r & ((1 << a.group_shift) - 1);
                    if (x <= slot && g < G)
                        *reinterpret_cast<f32x4*>(dst + g * a.score_stride + kKeys * (kt0 + i - slot + x) + 4 * (lane & 7)) = s_out[wave][r][lane & 7];
                }
                return slot == slots - 1 && stores_four(G);
            }
            return false;
        };
        // A column without a key yet has no reference; its first key sets it.
        auto first_reference = [&]() {
            if (unset) {
                const float mx = column_max(sc);
                if (neg_m == kUnset && mx != kNegInf) neg_m = -mx * a.scale_log2e;
                unset = __builtin_amdgcn_ballot_w64(neg_m == kUnset) != 0;
            }
        };
        // The reference may lag behind the running maximum by 2^8 (weights up to 2^8 are as exact), so that the accumulators are
        // rescaled rarely.
        constexpr float kLag = 8.0f;
        auto move_reference = [&](float top) {
            if (__builtin_amdgcn_ballot_w64(top > kLag) != 0) {
                // (from the scores again: exponents far above the old reference have lost the digits that the new one needs)
                const float next = fminf(neg_m, -column_max(sc) * a.scale_log2e), alpha = fast_exp2(next - neg_m);
                l *= alpha;
#pragma unroll
                for (int j = 0; j < NJ; ++j) o[j] *= alpha;
                neg_m = next;
#pragma unroll
                for (int x = 0; x < 16; ++x) ex[x] = __builtin_fmaf(sc[x], a.scale_log2e, neg_m);
            }
        };
        auto exponents = [&]() {
            float top = kNegInf;
#pragma unroll
            for (int x = 0; x < 16; ++x) {
                ex[x] = __builtin_fmaf(sc[x], a.scale_log2e, neg_m);
                top = fmaxf(top, ex[x]);
            }
            move_reference(top);
        };
        auto scores = [&](const kv_u32x4* sk) {
            bf16x8 ka[NK];
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) ka[kk] = k_operand(sk, kk);
            __builtin_amdgcn_sched_barrier(0);
            sc = zero();
#pragma unroll
            for (int kk = 0; kk < NK; ++kk) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[kk], qb[kk], sc, 0, 0, 0);
        };
        auto values = [&](const kv_u32x4* sv) {
            bf16x8 va[2 * NJ];
#pragma unroll
            for (int u = 0; u < 2 * NJ; ++u) va[u] = v_operand(sv, u);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int u = 0; u < 2 * NJ; ++u) {
                o[u % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], weight_operand(u / NJ), o[u % NJ], 0, 0, 0);
                if constexpr (SUMS) o[u % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], rest_operand(u / NJ), o[u % NJ], 0, 0, 0);
            }
        };
        // The tokens of a tile (with a mask: from first_edge on) that this lane's row sees
        auto seen_of = [&](int tile) -> uint32_t {
            if constexpr (SUMS) return n - kKeys * tile >= 32 ? ~0u : (1u << (n - kKeys * tile)) - 1u;
            else return s_seen[tile - first_edge][srow];
        };
        // Sums of values where a token that a row does not see may hold an infinity or NaN, which its weight of 0 would turn into NaN:
        // token by token, without those.  (One that the row sees counts whatever its weight: 0 times infinity is NaN then.)  And where
        // weights have two parts: an infinity is multiplied with their sum, not with each.
        auto add_values_one_by_one = [&](const kv_u32x4* sv, uint32_t seen) {
#pragma unroll 1
            for (int t = 0; t < 32; ++t) {
                const int u = 2 * (t >> 3) + ((t & 3) >> 1);
                auto of_token = [&](const uint32_t* pairs) {
                    uint32_t two = pairs[0];
#pragma unroll
                    for (int x = 1; x < 8; ++x) two = u == x ? pairs[x] : two;
                    two = (uint32_t)__shfl((int)two, col + 32 * ((t >> 2) & 1));
                    return (t & 1) ? bf16_hi(two) : bf16_lo(two);
                };
                float wt = of_token(pw);
                if constexpr (SUMS) wt += of_token(pf);
                const char* row = reinterpret_cast<const char*>(sv + kg * kPieces) + t * kStride + head_place(hw, t) * kRow;
                const int g = D == 128 ? 4 * (t & 3) : 4 * ((t >> 1) & 1);
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int u4 = 0; u4 < 4; ++u4) {   // elements 32 j + 8 u4 + 4 half ..
                        const kv_u32x2 x = *reinterpret_cast<const kv_u32x2*>(row + (((4 * j + u4) ^ g) << 4) + 8 * half);
                        if ((seen >> t) & 1) {
                            o[j][4 * u4 + 0] += wt * bf16_lo(x[0]);
                            o[j][4 * u4 + 1] += wt * bf16_hi(x[0]);
                            o[j][4 * u4 + 2] += wt * bf16_lo(x[1]);
                            o[j][4 * u4 + 3] += wt * bf16_hi(x[1]);
                        }
                    }
            }
        };
        auto hide = [&](int tile) {   // scores of tokens that the row does not see
            if (tile < first_edge) return;
            const uint32_t seen = seen_of(tile) >> (4 * half);
#pragma unroll
            for (int x = 0; x < 16; ++x) sc[x] = (seen >> (8 * (x >> 2) + (x & 3))) & 1 ? sc[x] : kNegInf;
        };
        auto whole_step = [&](auto careful, int i, const kv_u32x4* sk, const kv_u32x4* sv) {
            const int tile = kt0 + i;
            scores(sk);
            hide(tile);
            keep_scores(i);
            first_reference();
            exponents();
#pragma unroll
            for (int u = 0; u < 8; ++u) weights(u);
            if (decltype(careful)::value && (SUMS || tile >= first_edge)) add_values_one_by_one(sv, seen_of(tile));
            else values(sv);
        };
        // The chain of a tile is cut across tiles: the weights of tile i are made beside the score products of tile i + 1, its
        // output products run beside the exponents of tile i + 1.  The order is pinned: a product, the vector
        // instructions that fit under it, the operand read of the second product after it.  The loads of one tile, the
        // NB - 1st after it, are under way meanwhile.
        constexpr int kAhead = 2;
        auto step = [&](auto phase, int i) {
            constexpr int B = decltype(phase)::value;   // i % NB
            kv_u32x4* const k_next = k_buf(B + 1);
            kv_u32x4* const v_now = v_buf(B);
            stage_v(v_buf(B + NB - 1), std::false_type());
            stage_k(k_buf(B), std::false_type());
            bool stored = false;
            if (!idle) {
                bf16x8 ka[NK], va[2 * NJ];
#pragma unroll
                for (int kk = 0; kk < kAhead; ++kk) ka[kk] = k_operand(k_next, kk);
                __builtin_amdgcn_sched_barrier(0);
                sc = zero();
#pragma unroll
                for (int kk = 0; kk < NK; ++kk) {
                    sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[kk], qb[kk], sc, 0, 0, 0);
                    if (kk + kAhead < NK) ka[kk + kAhead] = k_operand(k_next, kk + kAhead);
                    else va[kk + kAhead - NK] = v_operand(v_now, kk + kAhead - NK);
#pragma unroll
                    for (int u = kk * 8 / NK; u < (kk + 1) * 8 / NK; ++u) {
                        weights(u);
                        asm volatile("" : "+v"(pw[u]), "+v"(l));   // (else moved to where they are used)
                        if constexpr (SUMS) asm volatile("" : "+v"(pf[u]));
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                const bf16x8 pb[2] = {weight_operand(0), weight_operand(1)}, pr[2] = {rest_operand(0), rest_operand(1)};
                const int tile = kt0 + i + 1;
                hide(tile);
                stored = keep_scores(i + 1);
                first_reference();
                float top = kNegInf;
#pragma unroll
                for (int u = 0; u < 2 * NJ; ++u) {
                    o[u % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], pb[u / NJ], o[u % NJ], 0, 0, 0);
                    if constexpr (SUMS) o[u % NJ] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], pr[u / NJ], o[u % NJ], 0, 0, 0);
                    if (u + kAhead < 2 * NJ) va[u + kAhead] = v_operand(v_now, u + kAhead);
                    // (the first two give the last score product time to finish)
#pragma unroll
                    for (int x = u < 2 ? 16 : 16 * (u - 2) / (2 * NJ - 2); x < (u < 2 ? 0 : 16 * (u - 1) / (2 * NJ - 2)); ++x) {
                        ex[x] = __builtin_fmaf(sc[x], a.scale_log2e, neg_m);
                        top = fmaxf(top, ex[x]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                move_reference(top);
            }
            // (a wavefront that shares no tile has no barrier, and its four stores of scores may go on)
            if (!kShared && stored) staged(std::integral_constant<int, 4>());
            else staged(std::integral_constant<int, 0>());
        };
        const int common = count / KW;   // tiles that every key group has
        int i = 0;
        if (common > 0) {
            if (!idle) {
                scores(s_k0);
                hide(kt0);
                keep_scores(0);
                first_reference();
                exponents();
            }
            if constexpr (kShared) __syncthreads();   // (K of tile 0 is read, its buffer may be filled again)
            for (; i + NB < common; i += NB) {
                step(std::integral_constant<int, 0>(), i);
                step(std::integral_constant<int, 1>(), i + 1);
                if constexpr (NB > 2) {
                    step(std::integral_constant<int, 2>(), i + 2);
                    step(std::integral_constant<int, 3>(), i + 3);
                }
            }
            if (i + 1 < common) {
                step(std::integral_constant<int, 0>(), i);
                ++i;
                if (NB > 2 && i + 1 < common) {
                    step(std::integral_constant<int, 1>(), i);
                    ++i;
                    if (NB > 2 && i + 1 < common) {
                        step(std::integral_constant<int, 2>(), i);
                        ++i;
                    }
                }
            }
            // the last one
            if constexpr (KW > 1) stage_v(v_buf(i + 1), std::false_type());
            if (!idle) {
#pragma unroll
                for (int u = 0; u < 8; ++u) weights(u);
                values(v_buf(i));
            }
            ++i;
            if constexpr (KW > 1) staged(std::integral_constant<int, 0>());
        }
        if (KW > 1 && i < mine && !idle) whole_step(std::false_type(), i, k_buf(i), v_buf(i));   // one that only some key groups have
        // A value that is no number in a tile where rows do not see every token may have reached rows that do not see it, and one anywhere
        // has met the parts of weights apart: once more then, tile by tile, with care.
        if (SUMS || t0 + count > first_edge) {
            float probe = 0.f;
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int x = 0; x < 16; ++x) probe = __builtin_fmaf(o[j][x], 0.f, probe);   // 0, or NaN
            if (__syncthreads_or(!(probe == 0.f))) {
                clear();
                at_k = at_start;
                at_v = at_start;
#pragma unroll 1
                for (i = 0; i < iters; ++i) {
                    stage_k(s_k0, std::false_type());
                    stage_v(s_v0, std::false_type());
                    staged(std::integral_constant<int, 0>());
                    if (i < mine && !idle) whole_step(std::true_type(), i, s_k0, s_v0);
                    __syncthreads();
                }
            }
        }

        // ---- the piece's rows ----------------------------------------------------------------------
        l = half_sum(l);
        const int slot = 2 * (team * Hl + h) + (t0 == 0 ? 1 : 0);
        // groups of four accumulator registers: x = 4 j + u4 holds elements 8 x + 4 half ..
        constexpr int NX = 4 * NJ, XW = NX / KW;   // each of the KW wavefronts of a row finishes XW of them
        f32x4 acc[XW];
        float m_all, l_all;
        if constexpr (KW > 1) {
            // wavefronts that took different tiles of the same rows add up: all leave their sums in LDS
            if (half == 0) s_ml[wave * 32 + col] = make_float2(l != 0.f ? -neg_m : kNegInf, l);
            __syncthreads();   // (nobody reads a tile any more)
            auto area = [&](int x) { return x == 0 ? s_k0 : x == 1 ? s_k1 : x == 2 ? s_v0 : s_v1; };
            kv_u32x4* mine_at = area(wave) + lane;
#pragma unroll
            for (int x = 0; x < NX; ++x)
                mine_at[x * 64] = __builtin_bit_cast(kv_u32x4, f32x4{o[x >> 2][4 * (x & 3)], o[x >> 2][4 * (x & 3) + 1],
                                                                     o[x >> 2][4 * (x & 3) + 2], o[x >> 2][4 * (x & 3) + 3]});
            __syncthreads();
            m_all = kNegInf;
            l_all = 0.f;
#pragma unroll
            for (int k = 0; k < KW; ++k) m_all = fmaxf(m_all, s_ml[(k * RW + rw) * 32 + col].x);
#pragma unroll
            for (int x = 0; x < XW; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
            // (a wavefront that saw no key is left out, whatever its sums are; one that weighs nothing beside the others is not: its sums may
            // be infinite)
#pragma unroll 1
            for (int k = 0; k < KW; ++k) {
                const float2 ml = s_ml[(k * RW + rw) * 32 + col];
                const float f = ml.y != 0.f ? fast_exp2(ml.x - m_all) : 0.f;
                l_all += f * ml.y;
                const kv_u32x4* from_k = area(k * RW + rw) + kg * XW * 64 + lane;
#pragma unroll
                for (int x = 0; x < XW; ++x) {
                    const f32x4 y = __builtin_bit_cast(f32x4, from_k[x * 64]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[x][e] = ml.y != 0.f ? __builtin_fmaf(y[e], f, acc[x][e]) : acc[x][e];
                }
            }
            __syncthreads();   // (before the next piece's tiles land)
        } else {
            m_all = l != 0.f ? -neg_m : kNegInf;
            l_all = l;
#pragma unroll
            for (int x = 0; x < XW; ++x) acc[x] = f32x4{o[x >> 2][4 * (x & 3)], o[x >> 2][4 * (x & 3) + 1],
                                                        o[x >> 2][4 * (x & 3) + 2], o[x >> 2][4 * (x & 3) + 3]};
            if constexpr (kShared) __syncthreads();
        }
        if (real) {
            const int x0 = KW > 1 ? kg * XW : 0;
            if (cut) {
                // (as they lie in the registers: a store is 1 KiB in one place)
                f32x4* dst = a.part_o + (((int64_t)slot * RW + rw) * NX + x0) * 64 + lane;
#pragma unroll
                for (int x = 0; x < XW; ++x) dst[x * 64] = acc[x];
                if (kg == 0 && half == 0) *reinterpret_cast<float2*>(a.part_ml + ((int64_t)slot * RB + srow) * 2) = make_float2(m_all, l_all);
            } else {
                const float inv = 1.0f / l_all;   // (0 where the row sees nothing: zeros then; NaN stays NaN)
#pragma unroll
                for (int x = 0; x < XW; ++x) {
                    uint2 pk = make_uint2(pack_bf16x2(acc[x][0] * inv, acc[x][1] * inv), pack_bf16x2(acc[x][2] * inv, acc[x][3] * inv));
                    if (l_all == 0.f) pk = make_uint2(0u, 0u);
                    *reinterpret_cast<uint2*>(a.out + orow + 8 * (x0 + x) + 4 * half) = pk;
                }
                if (SUMS && kg == 0 && half == 0)
                    *reinterpret_cast<float2*>(a.row_ml + ((int64_t)s * v.n_q_local + h * G + rho % G) * 2) = make_float2(m_all, l_all);
            }
        }
        if (lane == 0 && rw == 0 && kg == 0 && rb < a.most_blocks) {
            int2* ends = a.ends + ((int64_t)s * a.most_blocks + rb) * Hl + h;
            if (t0 == 0) ends->x = team;
            if (t0 + count == w.tiles) ends->y = team;
        }
    }
}

// The second launch adds up the pieces of cut pairs, whose slots follow from the shares,
//   out[row] = sum_z o_z 2^(m_z - M) / sum_z l_z 2^(m_z - M),  M = max_z m_z.
// A wavefront takes 32 rows and a quarter of the workgroup's columns as the main kernel's lanes held them.  What bounds it is one
// trip to memory after another, so a lane's loads of several pieces are under way at once.  Rows of sequences without tokens are
// zeros.
struct piece_list {
    int rows, h, rb;          // rows of the pair
    int w0, w1;               // teams that hold its first and last piece
    int heads;
    __device__ int64_t slot(int z) const { return 2 * ((int64_t)(w0 + z) * heads + h) + (z == 0 ? 1 : 0); }
    __device__ int count() const { return w1 - w0 + 1; }
};
template <int RB>
__device__ __forceinline__ piece_list pieces_of(const tree_args& a, const seq_work& w, int s, int h, int rb)
{
    const int2 ends = a.ends[((int64_t)s * a.most_blocks + rb) * a.v.n_kv_local + h];
    piece_list p;
    p.rows = min(w.q_len * a.group - rb * RB, RB);
    p.h = h;
    p.rb = rb;
    p.w0 = uniform(ends.x);
    p.w1 = uniform(ends.y);
    p.heads = a.v.n_kv_local;
    return p;
}
constexpr int kGroups = 4;   // of four accumulator registers that a wavefront adds up

// (m, l, acc) and the pieces z, z + step, .. added up: up to MOST are requested at a time, the last one again past the end.
// Lane (col, half) has row 32 block + col, elements 8 (x0 + x) + 4 half ..
template <int D, int RB, int MOST>
__device__ __forceinline__ void add_pieces(const tree_args& a, const piece_list& p, int block, int x0, int z, int step, float& m, float& l,
                                           f32x4 (&acc)[kGroups])
{
    const int count = p.count(), lane = threadIdx.x & 63, row = min(32 * block + (lane & 31), p.rows - 1);
    const int from = row - 32 * block + (lane & 32);   // (lanes past the last row repeat it)
    auto add = [&](auto batch) {
        constexpr int kBatch = decltype(batch)::value;
        float2 ml[kBatch];
        f32x4 y[kBatch][kGroups];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int64_t slot = p.slot(min(z + u * step, count - 1));
            ml[u] = *reinterpret_cast<const float2*>(a.part_ml + (slot * RB + row) * 2);
            const f32x4* src = a.part_o + ((slot * (RB / 32) + block) * (D / 8) + x0) * 64 + from;
#pragma unroll
            for (int x = 0; x < kGroups; ++x) y[u][x] = src[x * 64];
        }
        float mn = m;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (z + u * step >= count) ml[u].y = 0.f;
            mn = fmaxf(mn, ml[u].y != 0.f ? ml[u].x : kNegInf);
        }
        const float keep = l != 0.f ? fast_exp2(m - mn) : 0.f;
        l *= keep;
#pragma unroll
        for (int x = 0; x < kGroups; ++x) acc[x] *= keep;
        m = mn;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (ml[u].y == 0.f) continue;
            const float f = fast_exp2(ml[u].x - mn);
            l += ml[u].y * f;
#pragma unroll
            for (int x = 0; x < kGroups; ++x) acc[x] += y[u][x] * f;
        }
        z += kBatch * step;
    };
    while (z < count) {
        if (MOST == 2 || (count - z + step - 1) / step <= 2) add(std::integral_constant<int, 2>());
        else add(std::integral_constant<int, MOST>());
    }
}
// N groups of a lane's row: zeros where it has seen nothing
template <int D, int N>
__device__ __forceinline__ void store_row(const tree_args& a, const seq_work& w, int h, int rho, int element, float l, const f32x4 (&acc)[N])
{
    const float inv = 1.0f / l;
    uint16_t* dst = a.out + ((int64_t)(w.q0 + rho / a.group) * a.v.n_q_local + h * a.group + rho % a.group) * D + element;
#pragma unroll
    for (int x = 0; x < N; ++x)
        *reinterpret_cast<uint2*>(dst + 8 * x) =
            l != 0.f ? make_uint2(pack_bf16x2(acc[x][0] * inv, acc[x][1] * inv), pack_bf16x2(acc[x][2] * inv, acc[x][3] * inv)) : make_uint2(0u, 0u);
}
// One set of columns of 32 rows by the whole workgroup, whose wavefronts share the pieces out and add up in LDS
struct merge_room {
    f32x4 acc[4][kGroups][64];
    float2 ml[4][64];
};
template <int D, int RB, int MOST>
__device__ __forceinline__ void add_together(const tree_args& a, const seq_work& w, const piece_list& p, int block, int x0, merge_room& room)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = 32 * block + (lane & 31);
    float m = kNegInf, l = 0.f;
    f32x4 acc[kGroups] = {};
    add_pieces<D, RB, MOST>(a, p, block, x0, wave, 4, m, l, acc);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kGroups; ++x) room.acc[wave][x][lane] = acc[x];
    room.ml[wave][lane] = make_float2(m, l);
    __syncthreads();
    // wavefront x finishes group x
    m = kNegInf;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = fmaxf(m, room.ml[k][lane].x);
    l = 0.f;
    f32x4 all[1] = {};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 ml = room.ml[k][lane];
        if (ml.y == 0.f) continue;
        const float f = fast_exp2(ml.x - m);
        l += ml.y * f;
        all[0] += room.acc[k][wave][lane] * f;
    }
    if (row < p.rows) store_row<D>(a, w, p.h, p.rb * RB + row, 8 * (x0 + wave) + 4 * (lane >> 5), l, all);
}
template <int D>
__device__ __forceinline__ void zero_rows(const tree_args& a, const seq_work& w, int h)
{
    constexpr int kLanes = D / 4, kRows = 256 / kLanes;
    const f32x4 none[1] = {};
    for (int x = blockIdx.z * kRows + (int)threadIdx.x / kLanes; x < w.q_len * a.group; x += gridDim.z * kRows)
        store_row<D>(a, w, h, x, 4 * ((int)threadIdx.x % kLanes), 0.f, none);
}

// Block (s, pair of s, part): 32 rows (at D = 64: 64), or TOGETHER 32 rows and 32 of their columns, where lists are long and few.
template <int D, int RB, bool TOGETHER>
__global__ __launch_bounds__(256) void tree_merge_kernel(tree_args a)
{
    constexpr int kParts = D / 8 / kGroups, kBlocks = TOGETHER ? 1 : 4 / kParts;   // column sets of a row; blocks of rows of a workgroup
    __shared__ merge_room room;   // (TOGETHER)
    const int s = blockIdx.x, pair = blockIdx.y, lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6);
    const seq_work w = work_of<RB>(a, s);
    if (w.n <= 0 && w.q_len > 0 && pair < a.v.n_kv_local) zero_rows<D>(a, w, pair);
    if (pair >= min(w.blocks, a.most_blocks) * a.v.n_kv_local) return;
    const int h = pair / w.blocks, rb = pair - h * w.blocks, part = blockIdx.z;
    const int first_block = TOGETHER ? part / kParts : part * kBlocks;
    if (32 * first_block >= w.q_len * a.group - rb * RB) return;
    const piece_list p = pieces_of<RB>(a, w, s, h, rb);
    if (p.count() == 1) return;   // written by the main kernel
    if constexpr (TOGETHER) {
        add_together<D, RB, 4>(a, w, p, first_block, part % kParts * kGroups, room);
    } else {
        const int block = first_block + wave / kParts, x0 = wave % kParts * kGroups, row = 32 * block + (lane & 31);
        if (32 * block >= p.rows) return;
        float m = kNegInf, l = 0.f;
        f32x4 acc[kGroups] = {};
        add_pieces<D, RB, 4>(a, p, block, x0, 0, 1, m, l, acc);
        if (row < p.rows) store_row<D>(a, w, h, rb * RB + row, 8 * x0 + 4 * (lane >> 5), l, acc);
    }
}

// Block (s, h, chunk of tokens): (M, L) of the pair's G rows, then sum_g 2^(score_g - M_g) / L_g to the chunk's tokens; the rows of a cut
// pair are shared out over the chunks' workgroups.
// LONG: lists of more than eight pieces, which cost registers that hide more of the rest's latency where they are short.
template <int D, bool LONG>
__global__ __launch_bounds__(256) void weights_kernel(tree_args a)
{
    constexpr int RB = 32;
    __shared__ merge_room room;
    __shared__ float2 s_row[4][32];
    const int s = blockIdx.x, h = blockIdx.y, G = a.group, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    float* sums = a.sums + ((int64_t)s * a.v.n_kv_local + h) * a.sum_stride;
    const float* scores = a.scores + ((int64_t)s * a.v.n_q_local + h * G) * a.score_stride;
    // Four tokens a thread.  Their sums and the scores of four query heads are asked for before anything is known of the sequence: what
    // bounds this launch is one trip to memory after another.  (Rows of scores are padded to whole tiles.)
    const int t = (int)blockIdx.z * a.chunk + 4 * tid;
    const bool here = 4 * tid < a.chunk && t < a.max_ctx_len;
    f32x4 e[4] = {};
    float prior[4] = {0.f, 0.f, 0.f, 0.f};
    if (here) {
#pragma unroll
        for (int y = 0; y < 4; ++y) e[y] = *reinterpret_cast<const f32x4*>(scores + min(y, G - 1) * a.score_stride + t);
#pragma unroll
        for (int c = 0; c < 4; ++c) prior[c] = sums[min(t + c, a.max_ctx_len - 1)];
    }
    const seq_work w = work_of<RB>(a, s);
    if (w.n <= 0) {
        zero_rows<D>(a, w, h);
        return;
    }
    if ((int)blockIdx.z * a.chunk >= w.n && (int)blockIdx.z >= D / 8 / kGroups) return;
    const piece_list p = pieces_of<RB>(a, w, s, h, 0);
    const bool cut = p.count() > 1;
    // lane l of a wavefront takes row l % Gp, Gp = G rounded up to a power of two, and every (256 / Gp)-th piece
    int gp = 1;
    while (gp < G) gp <<= 1;
    const int g = lane & (gp - 1);
    float m = kNegInf, l = 0.f;
    auto add = [&](float m2, float l2) {
        const float mn = fmaxf(m, m2);
        l = (l != 0.f ? l * fast_exp2(m - mn) : 0.f) + (l2 != 0.f ? l2 * fast_exp2(m2 - mn) : 0.f);
        m = mn;
    };
    if (g < G) {
        if (!cut) {
            const float2 ml = *reinterpret_cast<const float2*>(a.row_ml + ((int64_t)s * a.v.n_q_local + h * G + g) * 2);
            m = ml.x;
            l = ml.y;
        } else {
            for (int z = tid / gp; z < p.count(); z += 256 / gp) {
                const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (p.slot(z) * RB + g) * 2);
                add(ml.x, ml.y);
            }
        }
    }
    if (cut) {
        for (int d = gp; d < 64; d <<= 1) {
            const float m2 = __shfl_xor(m, d), l2 = __shfl_xor(l, d);
            add(m2, l2);
        }
        if (lane < gp) s_row[wave][g] = make_float2(m, l);
        __syncthreads();
        m = kNegInf;
        l = 0.f;
        for (int x = 0; x < 4; ++x) add(s_row[x][g].x, s_row[x][g].y);
        __syncthreads();
    }
    if (wave == 0 && lane < gp) s_row[0][g] = make_float2(m, l != 0.f ? 1.0f / l : 0.f);
    __syncthreads();
    const int end = min(((int)blockIdx.z + 1) * a.chunk, w.n);
    if (here && t < end) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        for (int y0 = 0; y0 < G; y0 += 4) {
            if (y0 > 0) {
#pragma unroll
                for (int y = 0; y < 4; ++y) e[y] = *reinterpret_cast<const f32x4*>(scores + min(y0 + y, G - 1) * a.score_stride + t);
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                if (y0 + y >= G) break;
                const float2 ml = s_row[0][y0 + y];
#pragma unroll
                for (int c = 0; c < 4; ++c) x[c] += e[y][c] == kNegInf ? 0.f : fast_exp2(e[y][c] - ml.x) * ml.y;
            }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (t + c < end) sums[t + c] = t + c == w.n - 1 ? x[c] : prior[c] + x[c];   // (the newest token has no sum yet)
    }
    if (cut)
        for (int x = blockIdx.z; x < D / 8 / kGroups; x += gridDim.z) add_together<D, RB, LONG ? 4 : 2>(a, w, p, 0, x * kGroups, room);
}

// ---- host ------------------------------------------------------------------------------------------

// Several heads to a workgroup, by the bytes of K and V by the bound: below, more and shorter pieces cost more than rows of 512 and 1024
// bytes bring.  us per call, one head / several: 8 heads, drafts of up to 8, 4 sequences of 512 to 4096 21.3 / 23.1, 8 of them
// 28.7 / 26.0, 32 71.6 / 64.8, 128 239 / 228; 4 heads, 128 sequences 128 / 120; 64 of 100 to 1000 36.4 / 27.5; drafts of up to 16
// (two heads) 128 sequences 269 / 251.  Two heads of 128 rows are slower (290 / 302).  One head of up to 64 rows is better off with
// four wavefronts to a tile than with one or two (drafts of up to 16, 8 heads, 2 sequences of 512 to 4096 18.2 / 20.6; of up to 8,
// 4 of 2000 to 4000 21.6 / 24.4; of up to 8 and one head, 16 of 3000 to 20000 31.9 / 34.0; 2 of 512 to 4096 16.9 / 15.8).
constexpr int64_t kWideBytes = 100000000;
constexpr int64_t kCacheBytes = 256 << 20;   // the cache between the dies and the memory

struct tree_plan {
    int rw, hw;   // wavefronts that share a tile's rows; heads of a workgroup
    int32_t teams, least, few;
    int32_t blocks;
    size_t part_o, part_ml, ends, bytes;
};
tree_plan plan_with(const kv_view* view, int batch, int max_ctx_len, int64_t rows, int rw, int hw)
{
    tree_plan p;
    p.rw = rw;
    p.hw = hw;
    const int rb = 32 * rw;
    const int64_t blocks = (rows + rb - 1) / rb, tiles = ((int64_t)max_ctx_len + kKeys - 1) / kKeys;
    // Shorter shares cost more in pieces than they save (us per call: weights of 2 sequences of 512 to 4096 with least tiles 4 / 8 / 16 23.4 /
    // 19.3 / 26.2; four wavefronts to a tile, least tiles 2 / 4 / 8: 2 heads, 4 sequences of 512 to 4096 15.5 / 14.2 / 15.1, 8 heads, 16 of
    // 100 to 500 20.6 / 17.8 / 18.1)
    p.least = rw == 1 ? 8 : 4;
    const int64_t most = blocks * batch * ((tiles + p.least - 1) / p.least);
    // heads that the chip holds workgroups for (four heads of 64 without sums would fit twice; the shares are made for one)
    const int fill = kCus * (rw == 2 || rw == 4 ? 2 : 1) * hw;
    p.teams = (int32_t)std::max<int64_t>(std::min<int64_t>(most, fill / view->n_kv_local), 1);
    const size_t records = (size_t)2 * p.teams * view->n_kv_local * rb;
    p.part_o = records * view->geom.head_dim * 4;
    p.part_ml = records * 8;
    p.blocks = (int32_t)blocks;
    p.few = batch <= 64 && blocks * batch * tiles < 0x40000000;
    p.ends = (size_t)batch * blocks * view->n_kv_local * 8;
    p.bytes = p.part_o + p.part_ml + p.ends;
    return p;
}
int64_t cache_bytes(const kv_view* view, int batch, int max_ctx_len)
{
    return (int64_t)batch * max_ctx_len * view->n_kv_local * view->geom.head_dim * 4;
}
bool wide(const kv_view* view, int batch, int max_ctx_len) { return cache_bytes(view, batch, max_ctx_len) >= kWideBytes; }
tree_plan plan_weights(const kv_view* view, int batch, int max_ctx_len)
{
    return plan_with(view, batch, max_ctx_len, view->group, 1, view->n_kv_local % 4 == 0 && wide(view, batch, max_ctx_len) ? 4 : 1);
}
// By the bound on a pair's rows
tree_plan plan_tree(const kv_view* view, int batch, int64_t total_q, int max_ctx_len, int max_q_len)
{
    const int64_t rows = (int64_t)max_q_len * view->group;
    const tree_plan p4 = plan_with(view, batch, max_ctx_len, rows, 4, 1), p8 = plan_with(view, batch, max_ctx_len, rows, 8, 1);
    tree_plan p = p4;
    if (rows <= 64 && wide(view, batch, max_ctx_len)) {
        if (rows <= 32 && view->n_kv_local % 4 == 0) p = plan_with(view, batch, max_ctx_len, rows, 1, 4);
        if (rows > 32 && view->n_kv_local % 2 == 0) p = plan_with(view, batch, max_ctx_len, rows, 2, 2);
    }
    // Eight wavefronts read K and V half as often as two workgroups of four, which do not wait for each other and hide more.  The former
    // where most sequences have rows for them and K and V pass the memory-side cache: us per call, four / eight, 8 heads, drafts of 33 to
    // 64 and sequences of 1000 to 8000, 8 of them 60.8 / 57.3, 32 253 / 220; drafts of 1 to 64 51.3 / 54.6, 152 / 175; drafts of 150 to
    // 256, 4 of them 92 / 101, 32 743 / 654.  (On average 130, 194 and 812 rows; 160 lies between.)
    if (rows > 128 && total_q * view->group > 160 * (int64_t)batch && cache_bytes(view, batch, max_ctx_len) > kCacheBytes) p = p8;
    // A workspace asked for with larger bounds serves smaller calls, whatever their variant.  (Teams are rounded down to whole ones: of 12
    // heads two side by side leave 85 x 64 rows each, one 42 x 128.)
    p.bytes = std::max({p.bytes, p4.bytes, p8.bytes, view->n_kv_local % 2 == 0 ? plan_with(view, batch, max_ctx_len, rows, 2, 2).bytes : 0});
    return p;
}

template <int D, int RW, int HW>
void launch(const tree_args& a, int64_t most_rows, hipStream_t st)
{
    constexpr int RB = 32 * RW, kParts = D / 8 / kGroups, kBlocks = 4 / kParts;
    const unsigned pairs = (unsigned)(a.v.n_kv_local * ((most_rows + RB - 1) / RB));
    const unsigned blocks = (unsigned)((std::min<int64_t>(most_rows, RB) + 31) / 32);
    hipLaunchKernelGGL((tree_kernel<D, RW, HW, false>), dim3((unsigned)(a.teams * (a.v.n_kv_local / HW))), dim3(RW == 8 ? 512 : 256), 0, st, a);
    // Few pairs have long lists of pieces
    if ((int64_t)a.batch * pairs * blocks <= 256)
        hipLaunchKernelGGL((tree_merge_kernel<D, RB, true>), dim3((unsigned)a.batch, pairs, blocks * kParts), dim3(256), 0, st, a);
    else
        hipLaunchKernelGGL((tree_merge_kernel<D, RB, false>), dim3((unsigned)a.batch, pairs, (blocks + kBlocks - 1) / kBlocks), dim3(256), 0, st, a);
}
template <int D>
void launch_tree(const tree_plan& p, const tree_args& a, int64_t most_rows, hipStream_t st)
{
    switch (p.rw) {
        case 1: launch<D, 1, 4>(a, most_rows, st); break;
        case 2: launch<D, 2, 2>(a, most_rows, st); break;
        case 4: launch<D, 4, 1>(a, most_rows, st); break;
        default: launch<D, 8, 1>(a, most_rows, st); break;
    }
}
template <int D>
void launch_weights(const tree_plan& p, const tree_args& a, int64_t chunks, hipStream_t st)
{
    const unsigned heads = (unsigned)a.v.n_kv_local;
    if (p.hw == 4) hipLaunchKernelGGL((tree_kernel<D, 1, 4, true>), dim3((unsigned)a.teams * heads / 4), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((tree_kernel<D, 1, 1, true>), dim3((unsigned)a.teams * heads), dim3(256), 0, st, a);
    if (a.teams > 8 * a.batch) hipLaunchKernelGGL((weights_kernel<D, true>), dim3((unsigned)a.batch, heads, (unsigned)chunks), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((weights_kernel<D, false>), dim3((unsigned)a.batch, heads, (unsigned)chunks), dim3(256), 0, st, a);
}

// The checks that both entry points make, and the arguments that they share.
int common_args(tree_args& a, const void* q, void* out, const void* kv_pool, int64_t n_pool_blocks, const int32_t* block_table,
                int64_t block_table_stride, const int32_t* ctx_lens, int batch, int max_ctx_len, const kv_view* view, float scale)
{
    if (!q || !out || !ctx_lens || !kv_pool || !block_table || n_pool_blocks < 1) return KV_ERR_INVALID_ARG;
    if (block_table_stride < ((int64_t)max_ctx_len + view->block_tokens - 1) / view->block_tokens) return KV_ERR_INVALID_ARG;
    const int d = view->geom.head_dim;
    if ((d != 64 && d != 128) || view->block_tokens % 16 != 0 || view->group > kMostGroup) return KV_ERR_UNSUPPORTED;
    if (!kv_aligned(kv_pool, 16) || !kv_aligned(q, 16) || !kv_aligned(out, 8)) return KV_ERR_UNSUPPORTED;
    if ((int64_t)view->row_heads * d * 2 * 16 > 0x7fffffff || n_pool_blocks > 0x7fffffff) return KV_ERR_UNSUPPORTED;
    a = tree_args{};
    a.q = (const uint16_t*)q;
    a.out = (uint16_t*)out;
    a.pool = (const uint16_t*)kv_pool;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.v = kv_view_to_dev(view);
    a.last_block = (uint32_t)(n_pool_blocks - 1);
    a.scale_log2e = (scale > 0.f ? scale : 1.0f / sqrtf((float)d)) * 1.4426950408889634f;
    a.group = view->group;
    while ((1 << a.group_shift) < a.group) ++a.group_shift;
    a.batch = batch;
    a.max_ctx_len = max_ctx_len;
    return KV_OK;
}

int64_t score_stride(int max_ctx_len) { return ((int64_t)max_ctx_len + kKeys - 1) / kKeys * kKeys; }

}  // namespace

extern "C" size_t paged_tree_attn_workspace_bytes(const kv_view* view, int batch, int64_t total_q, int max_ctx_len, int max_q_len)
{
    if (!kv_view_ok(view) || batch <= 0 || total_q <= 0 || max_ctx_len <= 0 || max_q_len <= 0) return 0;
    return plan_tree(view, batch, total_q, max_ctx_len, max_q_len).bytes;
}

extern "C" int paged_tree_attn(const void* q, void* out, const void* kv_pool, int64_t n_pool_blocks, const int32_t* block_table,
                               int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets,
                               const uint64_t* tree_mask, int64_t mask_words, int batch, int64_t total_q, int max_ctx_len,
                               int max_q_len, const kv_view* view, float scale, void* workspace, size_t workspace_bytes,
                               void* hip_stream)
{
    if (!kv_view_ok(view) || batch < 0 || total_q < 0 || max_ctx_len < 0 || max_q_len < 0 || n_pool_blocks < 0 ||
        block_table_stride < 0 || max_q_len > max_ctx_len || mask_words < 0)
        return KV_ERR_INVALID_ARG;
    if (batch == 0 || max_q_len == 0 || total_q == 0) return KV_OK;
    if (!q_offsets || !tree_mask || mask_words < (max_q_len + 63) / 64) return KV_ERR_INVALID_ARG;
    if (max_q_len > kMostNodes || mask_words > 0x7fffffff) return KV_ERR_UNSUPPORTED;
    tree_args a;
    if (const int rc = common_args(a, q, out, kv_pool, n_pool_blocks, block_table, block_table_stride, ctx_lens, batch, max_ctx_len,
                                   view, scale))
        return rc;
    const tree_plan p = plan_tree(view, batch, total_q, max_ctx_len, max_q_len);
    if (!workspace || ((uintptr_t)workspace & 255u)) return KV_ERR_INVALID_ARG;
    if (workspace_bytes < p.bytes) return KV_ERR_WORKSPACE;
    a.q_off = q_offsets;
    a.mask = (const unsigned long long*)tree_mask;
    a.mask_words = (int32_t)mask_words;
    a.max_q_len = max_q_len;
    a.teams = p.teams;
    a.least_tiles = p.least;
    a.few = p.few;
    a.part_o = (f32x4*)workspace;
    a.part_ml = (float*)workspace + p.part_o / 4;
    a.ends = (int2*)(a.part_ml + p.part_ml / 4);
    a.most_blocks = p.blocks;
    const int64_t rows = (int64_t)max_q_len * view->group;
    if ((rows + 31) / 32 * view->n_kv_local > 65535) return KV_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)hip_stream;
    if (view->geom.head_dim == 128) launch_tree<128>(p, a, rows, st);
    else launch_tree<64>(p, a, rows, st);
    return kv_record_hip_error(hipGetLastError(), "paged_tree_attn launch");
}

extern "C" size_t paged_decode_attn_weights_workspace_bytes(const kv_view* view, int batch, int max_ctx_len)
{
    if (!kv_view_ok(view) || batch <= 0 || max_ctx_len <= 0) return 0;
    const size_t rows = (size_t)batch * view->n_q_local;
    return plan_weights(view, batch, max_ctx_len).bytes + rows * (8 + 4 * (size_t)score_stride(max_ctx_len));
}

extern "C" int paged_decode_attn_weights(const void* q, void* out, const void* kv_pool, int64_t n_pool_blocks,
                                         const int32_t* block_table, int64_t block_table_stride, const int32_t* ctx_lens, int batch,
                                         int max_ctx_len, const kv_view* view, float scale, float* weights, int64_t weights_stride,
                                         void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!kv_view_ok(view) || batch < 0 || max_ctx_len < 0 || n_pool_blocks < 0 || block_table_stride < 0) return KV_ERR_INVALID_ARG;
    if (batch == 0) return KV_OK;
    if (!weights || weights_stride < max_ctx_len) return KV_ERR_INVALID_ARG;
    tree_args a;
    if (const int rc = common_args(a, q, out, kv_pool, n_pool_blocks, block_table, block_table_stride, ctx_lens, batch, max_ctx_len,
                                   view, scale))
        return rc;
    const tree_plan p = plan_weights(view, batch, std::max(max_ctx_len, 1));
    const size_t rows = (size_t)batch * view->n_q_local;
    if (max_ctx_len > 0) {
        if (!workspace || ((uintptr_t)workspace & 255u)) return KV_ERR_INVALID_ARG;
        if (workspace_bytes < paged_decode_attn_weights_workspace_bytes(view, batch, max_ctx_len)) return KV_ERR_WORKSPACE;
    }
    a.teams = p.teams;
    a.least_tiles = p.least;
    a.few = p.few;
    a.score_stride = score_stride(max_ctx_len);
    a.scores = (float*)workspace;   // (its rows are read and written 16 bytes at a time)
    float* const parts = a.scores + rows * a.score_stride;
    a.part_o = (f32x4*)parts;
    a.part_ml = parts + p.part_o / 4;
    a.row_ml = a.part_ml + p.part_ml / 4;
    a.ends = (int2*)(a.row_ml + 2 * rows);
    a.most_blocks = 1;
    a.sums = weights;
    a.sum_stride = weights_stride;
    // 1024 tokens a workgroup, 256 where that leaves most of the chip idle
    auto chunks_of = [&](int chunk) { return std::max<int64_t>(((int64_t)max_ctx_len + chunk - 1) / chunk, 1); };
    a.chunk = batch * (int64_t)view->n_kv_local * chunks_of(1024) < 4 * kCus ? 256 : 1024;
    const int64_t chunks = chunks_of(a.chunk);
    if (chunks > 65535 || view->n_kv_local > 65535) return KV_ERR_UNSUPPORTED;
    hipStream_t st = (hipStream_t)hip_stream;
    if (view->geom.head_dim == 128) launch_weights<128>(p, a, chunks, st);
    else launch_weights<64>(p, a, chunks, st);
    return kv_record_hip_error(hipGetLastError(), "paged_decode_attn_weights launch");
}
