// Multi-token causal attention over the paged KV pool, through a layout view: a chunk of a
// prefill, or the recompute step of Soft Preempt (Sec. 5.2.2 of the paper), both of which
// attend from several new tokens of a sequence to everything cached up to each of them.
//
// A workgroup of four wavefronts owns, for one (sequence, local KV head), a tile of 128 query rows = 128 / G
// consecutive new tokens x the G query heads that share the KV head; each wavefront holds 32 rows.  The workgroup
// walks the cached tokens in staged tiles of 32, each K and V tile going once from global memory straight into
// LDS (16 bytes per lane with the load-to-LDS instruction, no registers in between; double buffered: the next tiles land
// while the current ones are consumed); each wavefront takes its MFMA operands from LDS.
//
// Per tile, lane l = (c = l % 32, half = l / 32), products of 32 x 32 x 16:
//   S^T[token][c] = K[token][:] . q[c][:]     A operand = K rows from LDS, B operand = q
//   O^T[e][c]     = sum_t V[t][e] P[c][t]     A operand = V^T, read from the row-major V tile in
//                                             LDS with the transposing 64-bit read: a lane hands
//                                             in the address of four consecutive elements of one
//                                             row and receives one element of each of four rows
// The accumulator layout of S^T (register 4 a + i: token 8 a + 4 half + i) is the B layout of the second product if
// contraction index 8 half + 4 a' + i of its step c stands for token 16 c + 8 a' + 4 half + i, so the weights
// never leave their lane and the running maximum crosses lanes only when it moves.  Each lane sums the bf16
// weights of its own keys, the same that the numerator takes, and the two lanes of a column are added up
// once at the end.
// Column c of wavefront w is row rho = 32 w + c of the tile: token rho / Gp, head rho % Gp, Gp = G rounded up to a power
// of two (rows with head >= G are padding).  The causal mask keeps
// token t for a query at position pos iff t <= pos; since pos < ctx_len it also masks the slots
// past the end of the sequence.
#include "prefill_common.h"

using namespace kvprefill;

namespace {

// What bounds it.  Short launches: how much of a wavefront's own chain (K read -> scores -> softmax -> V read ->
// output) is exposed.  So the chain is cut across tiles: the weights of tile t are made beside the score products of tile
// t + 1, its output products run beside the exponents of tile t + 1, and the order is pinned, one product, the
// four vector instructions that fit under it and the operand read of the second product after it at a time.
// Products of 32 x 32 x 16 hide four vector instructions of 4 to 5 cycles, of the wavefront itself or of another; of
// 16 x 16 x 32 they hide two at a cost (32 products and the softmax of a tile in one wavefront 703 cycles where the
// products take 520; beside another wavefront's 32 x 32 x 16 products the softmax is free).  Long launches: the power
// that the chip may draw.  On 4 prompts of 8192 under a profiler the matrix pipe is busy 52 % of the cycles at 1.84 to 1.93 GHz
// with the tile by tile order that this replaces, and 61 % at 1.59 to 1.72 GHz with two of these wavefronts per SIMD;
// 16 x 16 x 32 products in the same order 51 % at 2.09 GHz.  All are within 4 % of each other in time, and taking out the
// loads that stage K and V (in a timing-only build) is worth 10 to 11 %, the exponentials 3 to 6 %.
// us per call, tile by tile -> now: 16 prompts of 128 to 4000 tokens, 32 query heads on 8, 756 -> 727; 6 of 500 to 3900
// 267 -> 258; one of 1000 29.4 -> 23.4; 64 of 30 to 600 136 -> 131; 4 of 8192 1920 -> 1924; 512 on 4096 to 16384 in
// four sequences, 4 heads, 204 -> 196; 70 drawn shapes 9.8 % less.
// Three workgroups per compute unit (32 KiB of LDS and at most 168 registers each; nothing is spilled in the loop): with two
// of up to 190 registers launches of many tiles are slower (tp2 chunks above 221, 64 of 30 to 600 135).  Eight
// wavefronts that share the staged tiles (half the loads) wait for each other: 16 prompts 810, 4 of 8192 1969.
// CUT: the items are the pieces of plan_pieces() instead of whole query tiles.
template <bool CUT>
__global__ __launch_bounds__(kThreads, 3) void prefill_kernel(prefill_args a)
{
    // [row][piece]: K pieces swizzled (piece c of row t at c ^ (t % 16)); V pieces at c ^ (4 * (t % 4)), which puts
    // the four rows that half a wavefront reads at once in different banks (no conflicts are counted)
    // one array per buffer: the compiler then knows that the loads landing in one buffer do not touch
    // the operands being read from the other
    __shared__ kv_u32x4 s_k0[512], s_k1[512];
    __shared__ kv_u32x4 s_v0[512], s_v1[512];
    __shared__ int2 s_slot[CUT ? kMostSlots : 1];
    __shared__ float s_cost[CUT ? kCandidates : 1];

    const int lane0 = threadIdx.x & 63;
    const int wave = uniform((int)threadIdx.x >> 6);
    const kv_view_dev& v = a.v;
    const int G = a.group;
    const int tokens_per_wg = 1 << a.tile_shift;
    work_items w;
    if (!items_of<CUT, 3>(a, lane0, s_slot, s_cost, reinterpret_cast<int32_t*>(s_k0), reinterpret_cast<int32_t*>(s_v0), s_k1, s_v1, w)) return;
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

    // ---- staging: K and V tiles go from global memory straight into LDS, 16 bytes per lane; one
    // instruction of a wavefront fills 64 consecutive 16-byte slots = 4 rows of 16 pieces, and
    // which piece of its row a lane fetches is the LDS swizzle applied on the global side.
    // A wavefront fills eight rows of a tile, all of one group of 16 (wave / 2), which lies in one block: per tile it works
    // out one address, from a block id asked for a tile before.
    const int dma_r = lane >> 4, dma_c = lane & 15;
    const int row8 = 8 * (wave & 1) + dma_r;                  // and + 4: rows within the group
    const int token_stride_bytes = v.token_stride * 2;
    const int64_t plane_bytes = v.plane_elems * 2;
    const int groups_per_block = v.block_tokens >> 4;
    const int last_group = (n - 1) >> 4;
    // Within the loop block ids come by vector loads: a scalar load under way shares the counter of the LDS reads and
    // returns out of order, so that every product would wait for all reads issued instead of its own.
    const int32_t* const ids = a.table + (int64_t)s * a.table_stride;
    const __amdgpu_buffer_rsrc_t id_row = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(ids), 0, 0x7ffffff0, 0x00020000);
    const char* pool_head = reinterpret_cast<const char*>(a.pool + v.head_off + hl * D);
    const int64_t block_bytes = (int64_t)v.block_elems * 2;
    const uint32_t group_bytes = 16u * (uint32_t)token_stride_bytes;
    uint32_t k_lane[2], v_lane[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = row8 + 4 * i;
        k_lane[i] = (uint32_t)(row * token_stride_bytes) + (uint32_t)((dma_c ^ row) << 4);
        v_lane[i] = (uint32_t)(row * token_stride_bytes) + (uint32_t)((dma_c ^ (4 * (row & 3))) << 4);
    }
    typedef __attribute__((address_space(3))) void* lds_ptr;
    // where a tile's rows of this wavefront lie, and the number of their group
    struct tile_rows {
        const char* rows;
        int group;
    };
    // the group to be fetched next: its number, place in its block, and the block's id.  Past the end it is the last one
    // (what is fetched then is masked, or of a tile past the last)
    int g_at = 2 * t_begin + (wave >> 1) - 2, g_in = 0, g_id = 0;
    auto next_block = [&]() {
        g_at = min(g_at + 2, last_group);
        const uint32_t blk = __umulhi(2u * (uint32_t)g_at, a.group_inverse) >> a.group_inverse_shift;
        g_in = g_at - (int)blk * groups_per_block;
        return blk;
    };
    auto rows_of = [&](int id) -> tile_rows {
        return {pool_head + (uint64_t)(uint32_t)id * (uint64_t)block_bytes + (uint64_t)(uint32_t)g_in * group_bytes, g_at};
    };
    auto request_id = [&](uint32_t blk) { return (int)__builtin_amdgcn_raw_buffer_load_b32(id_row, 0, 4 * blk, 0); };
    auto next_rows = [&]() {
        const tile_rows x = rows_of(uniform(g_id));
        g_id = request_id(next_block());
        return x;
    };
    // Rows past the end of the sequence are replaced by its last token (finite data, masked later).  Buffer loads: the
    // global form counts for the compiler as one that may read LDS, and while it is under way every LDS read would wait for
    // all that were issued.
    auto stage_rows = [&](const tile_rows& x, const uint32_t* at, int64_t plane, kv_u32x4* dst) {
        const __amdgpu_buffer_rsrc_t rows =
            __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(x.rows + plane), 0, 0x7ffffff0, 0x00020000);
        // ordinary (cached) loads: every query tile of the sequence reads these keys again
        if (x.group < last_group) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_ptr)(dst + (2 * wave + i) * 64), 16, at[i], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t past = (uint32_t)(max(row8 + 4 * i - (n - 1 - 16 * x.group), 0) * token_stride_bytes);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_ptr)(dst + (2 * wave + i) * 64), 16, at[i] - past, 0, 0, 0);
            }
        }
    };
    // all of this wavefront's loads have landed in LDS; then every wavefront's
    auto staged = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
        __syncthreads();
    };

    float neg_mc = kUnset;   // the addend of the exponent: -r of the column, see below; kUnset while it has none
    float l = 0.f;           // sum of the weights of this lane's keys of the column
    f32x16 o[4];             // o[j][4 a + i] = O[column][32 j + 8 a + 4 half + i]
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] = 0.f;

    // of tiles t + 1 and t + 2, see stage_ahead(); the ids of the first two come by scalar loads, in one round trip
    typedef const __attribute__((address_space(4))) int32_t* const_ids;
    const const_ids first_ids = (const_ids)ids;
    const int id0 = first_ids[next_block()];
    const int in0 = g_in, at0 = g_at;
    const int id1 = first_ids[next_block()];
    tile_rows rows2 = rows_of(id1);
    tile_rows rows1 = {pool_head + (uint64_t)(uint32_t)id0 * (uint64_t)block_bytes + (uint64_t)(uint32_t)in0 * group_bytes, at0};
    g_id = request_id(next_block());
    if (t_begin < n_tiles) {
        stage_rows(rows1, k_lane, 0, s_k0);
        stage_rows(rows1, v_lane, plane_bytes, s_v0);
    }
    if (t_begin + 1 < n_tiles) stage_rows(rows2, k_lane, 0, s_k1);
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

    staged();

    // Byte offsets of this lane's operands in a K and a V tile; buffers, halves and later columns are constants that the
    // reads carry.
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
    constexpr int kAhead = 2;   // operand reads under way
    auto zero = [&]() {
        f32x16 x;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.f;
        return x;
    };
    auto k_operand = [&](const kv_u32x4* sk, int kk) {
        uint32_t off = k_off;   // (opaque: the compiler would keep all eight offsets in registers that the loop needs)
        if (kk > 0) asm volatile("v_xor_b32 %0, %1, %2" : "=v"(off) : "i"(32 * kk), "v"(k_off));
        return as_bf16x8(*reinterpret_cast<const kv_u32x4*>(reinterpret_cast<const char*>(sk) + off));
    };
    auto v_operand = [&](const kv_u32x4* sv, int u) {   // u = 4 c + j
        const char* const vt = reinterpret_cast<const char*>(sv) + v_off[u & 3] + (u >> 2) * 16 * 256;
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
    if (t_begin < my_tiles) {
        sc = zero();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k_operand(s_k0, kk), qb[kk], sc, 0, 0, 0);
        mask(t_begin);
        const float mx = column_max(sc);
        neg_mc = mx == kNegInf ? kUnset : -mx * a.scale_log2e;
        unset = __builtin_amdgcn_ballot_w64(mx == kNegInf) != 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) ex[i] = __builtin_fmaf(sc[i], a.scale_log2e, neg_mc);
    }
    __syncthreads();
    // Tile t: its weights from the exponents beside the scores of tile t + 1, its output products beside the
    // exponents of tile t + 1.  K of tile t + 2 and V of tile t + 1 land meanwhile.
    auto stage_ahead = [&](int t, kv_u32x4* dk, kv_u32x4* dv) {
        rows1 = rows2;
        rows2 = next_rows();
        if (t + 1 < n_tiles) stage_rows(rows1, v_lane, plane_bytes, dv);
        if (t + 2 < n_tiles) stage_rows(rows2, k_lane, 0, dk);
    };
    auto step = [&](int t, kv_u32x4* k_now, kv_u32x4* k_next, kv_u32x4* v_now, kv_u32x4* v_next) {
        stage_ahead(t, k_now, v_next);
        // The order of the instructions is pinned: beside each product two exponentials with what follows from them, or
        // three exponents of the next tile, and the read of the operand of the second product after it.
        bf16x8 ka[8], va[8];
#pragma unroll
        for (int kk = 0; kk < kAhead; ++kk) ka[kk] = k_operand(k_next, kk);
        __builtin_amdgcn_sched_barrier(0);
        sc = zero();
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[kk], qb[kk], sc, 0, 0, 0);
            if (kk + kAhead < 8) ka[kk + kAhead] = k_operand(k_next, kk + kAhead);
            else va[kk + kAhead - 8] = v_operand(v_now, kk + kAhead - 8);
            weights(kk);
            asm volatile("" : "+v"(pw[kk]), "+v"(l));   // (else moved to where they are used)
            __builtin_amdgcn_sched_barrier(0);
        }
        mask(t + 1);
        const bf16x8 pb[2] = {weight_operand(0), weight_operand(1)};
        float tmax = kNegInf;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            o[u & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[u], pb[u >> 2], o[u & 3], 0, 0, 0);
            if (u + kAhead < 8) va[u + kAhead] = v_operand(v_now, u + kAhead);
            // (the first two give the last score product time to finish)
#pragma unroll
            for (int i = u < 2 ? 16 : (8 * (u - 2) + 2) / 3; i < (8 * (u - 1) + 2) / 3; ++i) {
                ex[i] = __builtin_fmaf(sc[i], a.scale_log2e, neg_mc);
                tmax = fmaxf(tmax, ex[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        move_reference(tmax);
        staged();
    };
    int t = t_begin;
    for (; t + 2 < my_tiles; t += 2) {
        step(t, s_k0, s_k1, s_v0, s_v1);
        step(t + 1, s_k1, s_k0, s_v1, s_v0);
    }
    const bool odd = t + 1 < my_tiles;
    if (odd) {
        step(t, s_k0, s_k1, s_v0, s_v1);
        ++t;
    }
    if (t < my_tiles) {   // the wavefront's last tile
        stage_ahead(t, odd ? s_k1 : s_k0, odd ? s_v0 : s_v1);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) weights(kk);
        const kv_u32x4* sv = odd ? s_v1 : s_v0;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            o[u & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v_operand(sv, u), weight_operand(u >> 2), o[u & 3], 0, 0, 0);
        staged();
        ++t;
    }
    for (; t < n_tiles; ++t) {   // tiles that other wavefronts of the workgroup still have
        const bool even = ((t - t_begin) & 1) == 0;
        stage_ahead(t, even ? s_k0 : s_k1, even ? s_v1 : s_v0);
        staged();
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
                a.part_ml[rec * 2 + 0] = lt > 0.f ? -neg_mc : kNegInf;   // (no valid key: left out)
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

extern "C" size_t paged_prefill_attn_workspace_bytes(const kv_view* view, int batch, int64_t total_q,
                                                     int max_ctx_len, int max_q_len)
{
    if (!kv_view_ok(view) || batch <= 0 || total_q <= 0 || max_ctx_len <= 0 || max_q_len <= 0) return 0;
    return prefill_workspace(view, batch, total_q, max_ctx_len, max_q_len, 3).ask;
}

extern "C" int paged_prefill_attn(const void* q, void* out, const void* kv_pool, int64_t n_pool_blocks,
                                  const int32_t* block_table, int64_t block_table_stride,
                                  const int32_t* ctx_lens, const int32_t* q_offsets, int batch,
                                  int64_t total_q, int max_ctx_len, int max_q_len, const kv_view* view,
                                  float scale, void* workspace, size_t workspace_bytes, void* hip_stream)
{
    return prefill_call<false>(q, out, kv_pool, nullptr, n_pool_blocks, block_table, block_table_stride, ctx_lens, q_offsets, batch, total_q,
                        max_ctx_len, max_q_len, view, scale, workspace, workspace_bytes, hip_stream, 3,
                        [](bool cut, dim3 grid, const prefill_args& a, hipStream_t st) {
                            if (cut) hipLaunchKernelGGL((prefill_kernel<true>), grid, dim3(kThreads), 0, st, a);
                            else hipLaunchKernelGGL((prefill_kernel<false>), grid, dim3(kThreads), 0, st, a);
                        });
}
