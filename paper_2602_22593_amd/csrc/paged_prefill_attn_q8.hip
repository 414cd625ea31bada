// paged_prefill_attn_q8: multi-token causal attention over a cache held in 8 bits.
//
// The products, the softmax and the chain cut across tiles are paged_prefill_attn's (paged_prefill_attn.hip): a workgroup of four wavefronts
// owns 128 query rows of a (sequence, KV head), S^T = K . q^T and O^T += V^T . P in bf16 products of 32 x 32 x 16, weights of tile t beside
// the scores of t + 1, output products of t beside the exponents of t + 1.  Other is how K and V get into LDS: codes are fetched into
// registers two tiles ahead, become bf16 beside the products (a quarter of a tile a wavefront, once for all four) and are written where rows of bf16
// would lie.  Values are code times scale: exact where the scale is a power of two, as the library writes them, rounded to bf16 otherwise.
// Bound by the products and what runs beside them (matrix pipe 44 % busy, vector unit 51 %, int8 39 and 62): between long prompts 1040 TFLOP/s,
// int8 920, 1137 from rows of bf16.  8 prompts of 128 to 3000 tokens, 32 heads on 8: 194 us; converted by every wavefront for itself: 254.
// Rounding: the softmax weights enter the output products as one bf16, off by 2^-8 at most, as paged_prefill_attn's do; their sum, the
// denominator, is of the same rounded weights.  The error against 64 bits is 2.0 to 2.3e-3 in the 2-norm, where that of the output's own rounding is
// 1.65e-3.  A second product with what the rounding left, as decode has it, would make the products half as many again where they are the bound.
#include "prefill_common.h"

using namespace kvprefill;
using namespace kvq8;

namespace {

constexpr int kPerCu = 2;     // workgroups that a compute unit holds
constexpr int kPlaces = 64;
constexpr uint32_t kHalf = 16384, kTile = 8192;   // of the rings of K and V: bytes of two tiles, of one

template <bool CUT, int FMT>
__global__ __launch_bounds__(kThreads, kPerCu) void prefill_q8_kernel(prefill_args a)
{
    // Rings of four tiles: the two that are read and the two that are written between two barriers.  [row][piece], K pieces swizzled (piece c of
    // row t at c ^ (t % 16)), V pieces at c ^ (4 * (t % 4)).
    __shared__ kv_u32x4 s_k[2048], s_v[2048];
    __shared__ kv_u32x4 s_place[4 * kPlaces];
    __shared__ int2 s_slot[CUT ? kMostSlots : 1];
    __shared__ float s_cost[CUT ? kCandidates : 1];

    const int lane0 = threadIdx.x & 63;
    const int wave = uniform((int)threadIdx.x >> 6);
    const kv_view_dev& v = a.v;
    const int G = a.group;
    const int tokens_per_wg = 1 << a.tile_shift;
    work_items w;
    if (!items_of<CUT, kPerCu>(a, lane0, s_slot, s_cost, reinterpret_cast<int32_t*>(s_k), reinterpret_cast<int32_t*>(s_v), s_k + 512, s_v + 512, w)) return;
    int hl = w.hl;
    const int per_head = w.per_head, own_s = w.own_s, own_place = w.own_place;
    for (int item = w.item; item < w.item_end; item += w.item_step) {   // (the body is not indented for it)
    // what is derived from the lane number is worked out anew per item: kept across the loop it costs the
    // registers that the inner loop needs (12 spilled instead of 4, with the key range cut 15 instead of 9)
    int lane = lane0;
    asm volatile("" : "+v"(lane));
    const int col = lane & 31, half = lane >> 5;
    int slot = item, s, piece = 0, pieces = 1, record = 0;
    if constexpr (CUT) {
        hl = item / per_head;
        const int idx = item - hl * per_head;
        slot = uniform(piece_slot(s_slot, a.slots, idx, lane));
        const int end_s = uniform(s_slot[slot].x), before = slot > 0 ? uniform(s_slot[slot - 1].x) >> 10 : 0;
        record = uniform(s_slot[slot].y);
        s = end_s & 1023;
        pieces = (end_s >> 10) - before;
        piece = idx - before;
    } else {
        s = a.order != kSlots ? own_s : slot_sequence(a, slot, lane);
    }

    const int n = a.ctx_lens[s];
    const int q0 = a.q_off[s];
    const int q_len = a.q_off[s + 1] - q0;
    // longest tiles first: the last query tile of a sequence sees the most keys
    const int tile_in_seq = !CUT && a.order != kSlots ? own_place : slot - ((q0 >> a.tile_shift) + s);
    const int j0 = (((q_len + tokens_per_wg - 1) >> a.tile_shift) - 1 - tile_in_seq) << a.tile_shift;
    if (j0 < 0 || n <= 0) continue;
    const int first_pos = n - q_len;                         // position of the sequence's query 0
    const int j_last = min(j0 + tokens_per_wg, q_len) - 1;   // last query token of this tile
    const int all_tiles = (first_pos + j_last) / kKeys + 1;   // key tiles 0 .. all_tiles - 1 of the query tile
    // this workgroup's share of them: [t_begin, n_tiles)
    int t_begin = 0, n_tiles = all_tiles;
    if constexpr (CUT) {
        const int per_piece = (all_tiles + pieces - 1) / pieces;
        t_begin = piece * per_piece;
        n_tiles = min(all_tiles, t_begin + per_piece);
        record += piece * (j_last - j0 + 1) - (q0 + j0);   // record of token j: record + q0 + j
    } else {
        // a start that the compiler knows to be 0 makes it double the loop's body and spill in it (8 % slower)
        asm volatile("" : "+s"(t_begin), "+s"(n_tiles));
    }

    // ---- staging ---------------------------------------------------------------------------------------
    // A wavefront stages eight rows of a tile's K and V, all of one group of 16 (wave / 2), eight lanes a row.
    const int lane_row = lane >> 3, lane_piece = lane & 7;
    const int row8 = 8 * (wave & 1) + lane_row;               // row within the group
    const int groups_per_block = v.block_tokens >> 4;
    const int last_group = (n - 1) >> 4;
    const int32_t* const ids = a.table + (int64_t)s * a.table_stride;
    const char* pool_head = reinterpret_cast<const char*>(a.pool) + v.head_off + hl * D;
    const uint32_t group_bytes = 16u * (uint32_t)v.token_stride;
    const uint32_t code_lane = (uint32_t)(row8 * v.token_stride + 8 * lane_piece);
    const uint32_t last_lane = code_lane - (uint32_t)(max(row8 - ((n - 1) & 15), 0) * v.token_stride);   // rows past the end: the last one
    // Where the rows of a wavefront's group lie, and their scales, stands in LDS for kPlaces tiles at a time (worked out tile by tile it took
    // 80 scalar instructions a tile); each wavefront has its own list, and makes the next one where it ends.
    typedef const __attribute__((address_space(1))) char* global_bytes;
    typedef const __attribute__((address_space(1))) kv_u32x2* global_codes;
    constexpr uint32_t kExact = 1u << 31, kLast = 1u << 30;   // beside an address: both scales are powers of two; the sequence ends there
    kv_u32x4* const places = s_place + wave * kPlaces;
    int p_next = t_begin, p_first = 0;   // the tile whose place comes next, and the list's first
    // Lane i's group, of tile p_first + i: its rows (and whether it is the last one), then its scales.
    uint32_t g_lo = 0, g_hi = 0, g_k = 0, g_v = 0;
    auto request_places = [&]() __attribute__((always_inline)) {
        p_first = p_next;
        const int g = min(2 * (p_first + lane) + (wave >> 1), last_group);   // (past the end: the last group, masked or never used)
        const uint32_t blk = __umulhi(2u * (uint32_t)g, a.group_inverse) >> a.group_inverse_shift;
        const uint32_t in = (uint32_t)g - blk * (uint32_t)groups_per_block;
        const int id = ids[blk];
        const float* scale = a.scales + q8_scale_at(a.x, id, 16 * (int)in, hl);
        g_k = __float_as_uint(scale[0]);
        g_v = __float_as_uint(scale[a.x.block_scales / 2]);
        const uint64_t at = reinterpret_cast<uint64_t>(pool_head) + (uint64_t)(uint32_t)id * (uint64_t)v.block_elems + (uint64_t)in * group_bytes;
        g_lo = (uint32_t)at;
        g_hi = (uint32_t)(at >> 32) | (g == last_group ? kLast : 0u);
    };
    auto list_places = [&]() __attribute__((always_inline)) {
        // Where either scale is not finite K's is NaN: not an infinity, which may make all of a token's scores -inf and so leave the group
        // out; and in V's place, so that rows that do not see the group (whose weights are 0) keep their results.
        if ((g_k & 0x7f800000u) == 0x7f800000u || (g_v & 0x7f800000u) == 0x7f800000u) {
            g_k = kNaNBits;
            g_v = 0u;
        }
        auto power = [&](uint32_t bits) -> bool { return (bits & 0x807fffffu) == 0u && bits - 1u < 0x7f7fffffu; };
        places[lane] = kv_u32x4{g_lo, g_hi | (power(g_k) && power(g_v) ? kExact : 0u), g_k, g_v};
    };
    struct place {        // of a tile's rows of this wavefront (uniform)
        global_bytes rows;
        uint32_t k, v;    // scales
        uint32_t flags;
    };
    auto look_up = [&]() __attribute__((always_inline)) -> kv_u32x4 { return places[p_next++ - p_first]; };
    auto rows_at = [&](uint32_t lo, uint32_t hi) __attribute__((always_inline)) -> global_bytes {
        return (global_bytes)((uint64_t)lo | (uint64_t)(hi & ~(kExact | kLast)) << 32);
    };
    auto place_of = [&](const kv_u32x4& e) __attribute__((always_inline)) -> place {
        const uint32_t hi = (uint32_t)uniform((int)e[1]);
        return {rows_at((uint32_t)uniform((int)e[0]), hi), (uint32_t)uniform((int)e[2]), (uint32_t)uniform((int)e[3]), hi};
    };
    struct fetched {
        kv_u32x2 lo, hi;   // pieces c and c + 8 of the row's sixteen
        uint32_t scale;
        bool exact;
    };
    auto scaled = [&](const place& x, int plane, fetched& f) __attribute__((always_inline)) {
        f.scale = plane ? x.v : x.k;
        f.exact = (x.flags & kExact) != 0;
    };
    auto fetch = [&](const place& x, int plane, fetched& f) __attribute__((always_inline)) {
        const global_bytes rows = x.rows + (plane ? v.plane_elems : 0);
        const uint32_t at = (x.flags & kLast) ? last_lane : code_lane;
        f.lo = *(global_codes)(rows + at);
        f.hi = *(global_codes)(rows + at + 64);
        scaled(x, plane, f);
    };
    // Two of the 16 codes (u of 8) as bf16.
    auto convert = [&](const fetched& f, int u, auto exact) __attribute__((always_inline)) -> uint32_t {
        const float scale = __uint_as_float(f.scale);
        const uint32_t x = u < 4 ? f.lo[u >> 1] : f.hi[(u >> 1) & 1];
        if constexpr (exact.value) {
            return (u & 1) ? __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true))
                           : __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false));
        } else {
            const f32x2 y = (u & 1) ? two_f32<FMT, true>(x) : two_f32<FMT, false>(x);
            return pack_bf16x2(y[0] * scale, y[1] * scale);
        }
    };
    // A lane writes pieces c and c + 8 of its row: the eight lanes of a row reach different banks (two neighbouring pieces a lane: a quarter of
    // the cycles of LDS were conflicts).  Offsets in the rings: of the half that is not being read by V's products, see step().
    const uint32_t put_row = (uint32_t)(16 * (wave >> 1) + row8);
    uint32_t k_put = put_row * 256 + (lane_piece ^ (put_row & 15)) * 16, v_put = put_row * 256 + (lane_piece ^ (4 * (put_row & 3))) * 16;
    auto write_k = [&](uint32_t at, const kv_u32x4& x) __attribute__((always_inline)) { *reinterpret_cast<kv_u32x4*>(reinterpret_cast<char*>(s_k) + at) = x; };
    auto write_v = [&](uint32_t at, const kv_u32x4& x) __attribute__((always_inline)) { *reinterpret_cast<kv_u32x4*>(reinterpret_cast<char*>(s_v) + at) = x; };
    auto put = [&](const fetched& f, auto write, uint32_t at) __attribute__((always_inline)) {
        kv_u32x4 x[2];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u >> 2][u & 3] = convert(f, u, std::integral_constant<bool, false>());
        write(at, x[0]);
        write(at ^ 128u, x[1]);
    };

    float neg_mc = kUnset;   // the addend of the exponent: -r of the column, see below; kUnset while it has none
    float l = 0.f;           // sum of the weights of this lane's keys of the column
    f32x16 o[4];             // o[j][4 a + i] = O[column][32 j + 8 a + 4 half + i]
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] = 0.f;

    // codes under way before tile t, in two sets that take turns: V of t + 2 and K of t + 3, then V of t + 3 and K of t + 4 (past the end: the last
    // group again)
    fetched k_even, v_even, k_odd, v_odd;
    place last_k;   // of the K that was fetched last, whose V is the next
    fetched k0, v0, k1, v1, k2;
    request_places();
    // The first tiles' codes are asked for once the block ids are there, beside their scales.
    {
        auto first = [&](int i) __attribute__((always_inline)) -> place {
            const uint32_t hi = __builtin_amdgcn_readlane(g_hi, i);
            return {rows_at(__builtin_amdgcn_readlane(g_lo, i), hi), 0u, 0u, hi};
        };
        place x = first(0);
        fetch(x, 0, k0);
        fetch(x, 1, v0);
        x = first(1);
        fetch(x, 0, k1);
        fetch(x, 1, v1);
        x = first(2);
        fetch(x, 0, k2);
        fetch(x, 1, v_even);
        x = first(3);
        fetch(x, 0, k_even);
        fetch(x, 1, v_odd);
        x = first(4);
        fetch(x, 0, k_odd);
    }
    // ---- this lane's query row (B operand) ------------------------------------------------------
    // element offset of the row of the column in q and out, or -1 if the column is
    // padding (recomputed at the end rather than kept in registers through the loop)
    auto row_of = [&](bool or_padding) -> int64_t {
        const int rho = wave * 32 + col;   // row of the tile
        // a token takes 2^group_shift rows of the tile, the first G of which are its query heads
        const int jt = j0 + (rho >> a.group_shift), g = rho & ((1 << a.group_shift) - 1);
        const int jc = min(jt, q_len - 1);
        const int64_t row = ((int64_t)(q0 + jc) * v.n_q_local + hl * G + min(g, G - 1)) * D;
        return (or_padding || (jt < q_len && g < G)) ? row : -1;
    };
    bf16x8 qb[8];
    // position of the column's query token
    const int pos = first_pos + min(j0 + ((wave * 32 + col) >> a.group_shift), q_len - 1);
    {
        const char* qrow = reinterpret_cast<const char*>(a.q + row_of(true)) + half * 16;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) qb[kk] = as_bf16x8(*reinterpret_cast<const kv_u32x4*>(qrow + kk * 32));
    }
    // positions ascend with the column: keys up to min_pos need no mask for any column of the wavefront, tiles
    // past that of max_pos are for none
    const int min_pos = uniform(pos), max_pos = __builtin_amdgcn_readlane(pos, 31);
    const int my_tiles = min(n_tiles, max_pos / kKeys + 1);
    const int my_pos = pos - 4 * half;   // this lane's keys of a tile start 4 half on

    list_places();
    last_k = place_of(look_up());
    scaled(last_k, 0, k0);
    scaled(last_k, 1, v0);
    last_k = place_of(look_up());
    scaled(last_k, 0, k1);
    scaled(last_k, 1, v1);
    last_k = place_of(look_up());
    scaled(last_k, 0, k2);
    scaled(last_k, 1, v_even);
    last_k = place_of(look_up());
    scaled(last_k, 0, k_even);
    scaled(last_k, 1, v_odd);
    last_k = place_of(look_up());
    scaled(last_k, 0, k_odd);
    put(k0, write_k, k_put);
    put(v0, write_v, v_put);
    put(k1, write_k, k_put + kTile);
    put(v1, write_v, v_put + kTile);
    put(k2, write_k, k_put + kHalf);
    k_put += kHalf;
    v_put += kHalf;
    __syncthreads();

    // Byte offsets of this lane's operands in the ring of K and of V, in the half that holds tiles t and t + 1 (t even)
    uint32_t k_off, v_off[4];
    {
        const int p = lane & 15, sub = (lane >> 4) & 1;
        k_off = (uint32_t)(col * 256 + (half ^ p) * 16);
        asm volatile("" : "+v"(k_off));
        // V^T operand of output block j, keys 16 c + 8 a + 4 half + (p / 4): elements 32 j + 16 sub + 4 (p % 4)
        const int vrow = 4 * half + (p >> 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v_off[j] = (uint32_t)(vrow * 256 + ((4 * j + 2 * sub + ((p & 3) >> 1)) ^ (4 * (vrow & 3))) * 16 + (p & 1) * 8);
            asm volatile("" : "+v"(v_off[j]));
        }
    }
    constexpr float kLag = 8.0f;
    f32x16 sc, ex;   // scores of the next tile; exponents of the tile whose weights come next
    uint32_t pw[8];  // its weights
    constexpr int kAhead = 4;   // operand reads under way
    auto zero = [&]() {
        f32x16 x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
        return x;
    };
    // K of tile t + 1 for t even (i = 0: second tile of the half) and odd (first tile of the other half)
    auto k_operand = [&](int i, int kk) __attribute__((always_inline)) {
        uint32_t off = k_off;   // (opaque: the compiler would keep all offsets in registers that the loop needs)
        if (i == 1 || kk > 0) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(off) : "i"(32 * kk + (i == 1 ? kHalf : 0)), "v"(k_off));
        return as_bf16x8(*reinterpret_cast<const kv_u32x4*>(reinterpret_cast<const char*>(s_k) + off + (i == 0 ? kTile : 0)));
    };
    auto v_operand = [&](int i, int u) __attribute__((always_inline)) {   // of tile t; u = 4 c + j
        const char* const vt = reinterpret_cast<const char*>(s_v) + v_off[u & 3] + i * kTile + (u >> 2) * 16 * 256;
        const bits16x4 lo = lds_read_transposed(vt);
        const bits16x4 hi = lds_read_transposed(vt + 8 * 256);
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    // The causal mask, only on the tiles that reach past some query of this wavefront: one uniform branch around all of
    // it, since most tiles lie wholly before every query.  A column that has seen no key yet (with the key range
    // cut it may see none; or only scores of -inf) has no reference maximum: its addend is kUnset, its exponents are
    // -inf, and the first tile that has a key for it sets the reference.
    bool unset = false;
    auto mask = [&](int tile) {
        const int base = kKeys * tile;
        if (base + 31 > min_pos || unset) {
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[i] = (base + 8 * (i >> 2) + (i & 3) <= my_pos) ? sc[i] : kNegInf;
            if (unset) {
                const float mx = column_max(sc);
                if (neg_mc == kUnset && mx != kNegInf) neg_mc = -mx * a.scale_log2e;
                unset = __builtin_amdgcn_ballot_w64(neg_mc == kUnset) != 0;
            }
        }
    };
    // Scores stay in the products' own units; the scale is folded into the exponent: t = score scale log2(e) - r,
    // weight = 2^t.  The reference r of a column may lag behind its running maximum by up to kLag: weights then
    // reach 2^kLag at most (exact in fp32 and in the bf16 operand alike), and the accumulators are rescaled only when some
    // column's maximum has moved further than that -- rarely, after the first tiles.  Both lanes of a column hold
    // the same r, so each tests its own sixteen exponents and the maximum crosses lanes only on the rare tile that
    // moves it.
    auto move_reference = [&](float tmax) {
        if (__builtin_amdgcn_ballot_w64(tmax > kLag) != 0) {
            // (from the scores again: exponents far above the old reference have lost the digits that the new one needs)
            const float to = fminf(neg_mc, -column_max(sc) * a.scale_log2e);
            const float alpha = fast_exp2(to - neg_mc);
            l *= alpha;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] *= alpha;
            neg_mc = to;
#pragma unroll
            for (int i = 0; i < 16; ++i) ex[i] = __builtin_fmaf(sc[i], a.scale_log2e, neg_mc);
        }
    };
    auto weight_operand = [&](int c) { return as_bf16x8(kv_u32x4{pw[4 * c], pw[4 * c + 1], pw[4 * c + 2], pw[4 * c + 3]}); };
    auto weights = [&](int u) {   // two of the sixteen
        const uint32_t w = pack_bf16x2(fast_exp2(ex[2 * u]), fast_exp2(ex[2 * u + 1]));
        pw[u] = w;
        l = add_pair(w, l);   // the denominator sums the same rounded weights
    };
    // (q has arrived on every way into the loop: the products in it would wait for it again, and with it for the codes under way)
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(qb[kk]));
    if (t_begin < my_tiles) {
        sc = zero();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            const uint32_t off = k_off ^ (32u * kk);
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const kv_u32x4*>(reinterpret_cast<const char*>(s_k) + off)), qb[kk], sc, 0, 0, 0);
        }
        mask(t_begin);
        const float mx = column_max(sc);
        neg_mc = mx == kNegInf ? kUnset : -mx * a.scale_log2e;
        unset = __builtin_amdgcn_ballot_w64(mx == kNegInf) != 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) ex[i] = __builtin_fmaf(sc[i], a.scale_log2e, neg_mc);
    }
    __syncthreads();
    // Tiles go by pairs, t_begin + 2 S and the next, with a barrier after each: i is the place in the pair.  Before it the pair's V and the K of
    // the next tile and the one after are in LDS; V of tile t + 2 goes to the other half, K of tile t + 3 there too (i = 0) or to this half
    // (i = 1), where nobody reads any more.
    auto k_to = [&](int i) __attribute__((always_inline)) -> uint32_t { return i == 0 ? k_put + kTile : k_put ^ kHalf; };
    auto v_to = [&](int i) __attribute__((always_inline)) -> uint32_t { return v_put + i * kTile; };
    auto fetch_ahead = [&](const kv_u32x4& next, fetched& kf, fetched& vf) __attribute__((always_inline)) {   // V of tile t + 4, K of t + 5
        fetch(last_k, 1, vf);
        last_k = place_of(next);
        fetch(last_k, 0, kf);
    };
    auto put_ahead = [&](int i, fetched& kf, fetched& vf) __attribute__((always_inline)) {
        put(kf, write_k, k_to(i));
        put(vf, write_v, v_to(i));
        fetch_ahead(look_up(), kf, vf);
    };
    // Tile t: its weights from the exponents beside the scores of tile t + 1, its output products beside the exponents of tile t + 1, and
    // beside both the codes under way become bf16.
    auto step = [&](int t, auto i_, fetched& kf, fetched& vf) __attribute__((always_inline)) {
        constexpr int i = i_.value;
        constexpr bool kPowers = FMT == kE4M3;   // e4m3 under other scales than powers of two is converted at the step's end
        // (and so twice: the prompts above 231 us in place of 194)
        const bool in_time = !kPowers || (kf.exact && vf.exact);
        const kv_u32x4 next = look_up();
        kv_u32x4 x;
        auto put_two = [&](const fetched& f, int u, auto write, uint32_t at) __attribute__((always_inline)) {
            x[u & 3] = convert(f, u, std::integral_constant<bool, kPowers>());
            if ((u & 3) == 3) write(u == 3 ? at : at ^ 128u, x);
        };
        // The order of the instructions is pinned: beside each product two exponentials with what follows from them, or three exponents of the
        // next tile, two codes, and the read of a later product's operand after it.
        bf16x8 ka[8], va[8];
#pragma unroll
        for (int kk = 0; kk < kAhead; ++kk) ka[kk] = k_operand(i, kk);
        __builtin_amdgcn_sched_barrier(0);
        // (the scores and the weights go before the output products of the SIMD's other wavefront: 1 % less time, int8 3 %)
        __builtin_amdgcn_s_setprio(1);
        sc = zero();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[kk], qb[kk], sc, 0, 0, 0);
            if (kk + kAhead < 8) ka[kk + kAhead] = k_operand(i, kk + kAhead);
            else va[kk + kAhead - 8] = v_operand(i, kk + kAhead - 8);
            weights(kk);
            asm volatile("" : "+v"(pw[kk]), "+v"(l));   // (else moved to where they are used)
            put_two(kf, kk, write_k, k_to(i));
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        mask(t + 1);
        const bf16x8 pb[2] = {weight_operand(0), weight_operand(1)};
        float tmax = kNegInf;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            o[u & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], pb[u >> 2], o[u & 3], 0, 0, 0);
            if (u + kAhead < 8) va[u + kAhead] = v_operand(i, u + kAhead);
            // (the first two give the last score product time to finish)
#pragma unroll
            for (int e = u < 2 ? 16 : (8 * (u - 2) + 2) / 3; e < (8 * (u - 1) + 2) / 3; ++e) {
                ex[e] = __builtin_fmaf(sc[e], a.scale_log2e, neg_mc);
                tmax = fmaxf(tmax, ex[e]);
            }
            put_two(vf, u, write_v, v_to(i));
            __builtin_amdgcn_sched_barrier(0);
        }
        move_reference(tmax);
        if (!in_time) {
            put(kf, write_k, k_to(i));
            put(vf, write_v, v_to(i));
        }
        fetch_ahead(next, kf, vf);
    };
    auto last_step = [&](auto i_) __attribute__((always_inline)) {   // of the wavefront's last tile
        constexpr int i = i_.value;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) weights(kk);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            o[u & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(i, u), weight_operand(u >> 2), o[u & 3], 0, 0, 0);
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};
    auto pair_begins = [&]() __attribute__((always_inline)) {
        if (p_next - p_first > kPlaces - 2) {
            request_places();
            list_places();
        }
    };
    auto pair_ends = [&]() __attribute__((always_inline)) {
        k_off ^= kHalf;
#pragma unroll
        for (int j = 0; j < 4; ++j) v_off[j] ^= kHalf;
        k_put ^= kHalf;
        v_put ^= kHalf;
        __syncthreads();
    };
    int t = t_begin;
    for (; t + 2 < my_tiles; t += 2) {
        pair_begins();
        step(t, first, k_even, v_even);
        step(t + 1, second, k_odd, v_odd);
        pair_ends();
    }
    for (bool own = t < my_tiles; t < n_tiles; t += 2, own = false) {   // the wavefront's last pair, then those that others of the workgroup still have
        pair_begins();
        if (own && t + 1 < my_tiles) {
            step(t, first, k_even, v_even);
            last_step(second);
        } else {
            if (own) last_step(first);
            put_ahead(0, k_even, v_even);
        }
        put_ahead(1, k_odd, v_odd);
        pair_ends();
    }

    // ---- normalise and store ------------------------------------------------------------------------
    {
        const float lt = half_sum(l);
        const int64_t orow = row_of(false);
        if (CUT && orow >= 0 && pieces > 1) {
            const int64_t rec = (int64_t)record * v.n_q_local + orow / D;
            float* dst = a.part_o + rec * D + 4 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *reinterpret_cast<f32x4*>(dst + 32 * j + 8 * u) = f32x4{o[j][4 * u], o[j][4 * u + 1], o[j][4 * u + 2], o[j][4 * u + 3]};
            if (half == 0) {
                a.part_ml[rec * 2 + 0] = lt > 0.f ? -neg_mc : lt != lt ? 0.f : kNegInf;   // (no valid key: left out)
                a.part_ml[rec * 2 + 1] = lt;
            }
        } else if (orow >= 0) {
            const float inv = 1.0f / lt;
            // the two lanes of a row exchange pieces so that each stores 16 bytes at a time
            uint16_t* dst = a.out + orow + 8 * half;
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    kv_u32x4 pk;
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const auto x = __builtin_amdgcn_permlane32_swap(
                            pack_bf16x2(o[j][4 * u + 2 * w] * inv, o[j][4 * u + 2 * w + 1] * inv),
                            pack_bf16x2(o[j][4 * u + 4 + 2 * w] * inv, o[j][4 * u + 5 + 2 * w] * inv), false, false);
                        pk[w] = x[0];
                        pk[2 + w] = x[1];
                    }
                    *reinterpret_cast<kv_u32x4*>(dst + 32 * j + 8 * u) = pk;
                }
        }
    }
    }
}

}  // namespace

extern "C" size_t paged_prefill_attn_q8_workspace_bytes(const kv_view* view, int batch, int64_t total_q, int max_ctx_len, int max_q_len)
{
    if (!kv_view_ok(view) || batch <= 0 || total_q <= 0 || max_ctx_len <= 0 || max_q_len <= 0) return 0;
    return prefill_workspace(view, batch, total_q, max_ctx_len, max_q_len, kPerCu).ask;
}

extern "C" int paged_prefill_attn_q8(const void* q, void* out, const void* kv_pool, const float* scales, int format, int64_t n_pool_blocks,
                                     const int32_t* block_table, int64_t block_table_stride, const int32_t* ctx_lens,
                                     const int32_t* q_offsets, int batch, int64_t total_q, int max_ctx_len, int max_q_len,
                                     const kv_view* view, float scale, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!kv_view_ok(view) || !q8_format_ok(format) || batch < 0 || total_q < 0 || max_q_len < 0) return KV_ERR_INVALID_ARG;
    if (batch > 0 && max_q_len > 0 && total_q > 0) {
        if (!scales) return KV_ERR_INVALID_ARG;
        if (view->geom.base_block_size % 16 != 0 || !kv_aligned(kv_pool, 16) || !kv_aligned(q, 16) || !kv_aligned(out, 16) || !kv_aligned(scales, 4))
            return KV_ERR_UNSUPPORTED;
    }
    const bool e4m3 = format == kE4M3;
    return prefill_call<true>(q, out, kv_pool, scales, n_pool_blocks, block_table, block_table_stride, ctx_lens, q_offsets, batch, total_q,
                              max_ctx_len, max_q_len, view, scale, workspace, workspace_bytes, hip_stream, kPerCu,
                              [e4m3](bool cut, dim3 grid, const prefill_args& a, hipStream_t st) {
                                  auto* f = e4m3 ? (cut ? prefill_q8_kernel<true, kE4M3> : prefill_q8_kernel<false, kE4M3>)
                                                 : (cut ? prefill_q8_kernel<true, kInt8> : prefill_q8_kernel<false, kInt8>);
                                  hipLaunchKernelGGL(f, grid, dim3(kThreads), 0, st, a);
                              });
}
