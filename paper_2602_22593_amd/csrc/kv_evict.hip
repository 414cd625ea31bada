// Tokens that leave the cache: kv_accept keeps the accepted ones of a sequence's drafted tokens, kv_evict the most attended
// ones of each KV head.  Both move rows inside the pool, 16 bytes at a time.
#include "kv_internal.h"

namespace {

constexpr int kThreads = 256;

// Elements from the pool's start to the first exposed head of token t; -1 where the table or the pool has no such place.
__device__ __forceinline__ int64_t row_at(const kv_view_dev& v, const int32_t* table, int64_t stride, int64_t n_pool_blocks, int t)
{
    int b, slot;
    kv_split_token(v, t, b, slot);
    if (b >= stride) return -1;
    const int32_t id = table[b];
    return id < 0 || id >= n_pool_blocks ? -1 : (int64_t)id * v.block_elems + (int64_t)slot * v.token_stride + v.head_off;
}

// ---- kv_accept ---------------------------------------------------------------------------------------
// Row first + accepted[i] goes to first + i.  The accepted nodes ascend, so a row's new place is never that of a later one's
// old row: a lane that owns one 16-byte column of the sequence's rows and goes through them in order needs no other's
// progress, and may request several before it stores them.  Latency is all there is to it: lengths, nodes, table, rows.  The values
// per token of a head (its position, its weight) are columns of 4 bytes.

struct accept_args {
    uint16_t* pool;
    int64_t n_pool_blocks;
    const int32_t* table;
    int64_t table_stride;
    const int32_t *ctx_lens, *q_off, *accepted, *n_accepted;
    int64_t accepted_stride;
    int32_t* new_lens;
    kv_view_dev v;
    uint32_t* per_token[2];      // [batch][n_kv_local][per_token_stride], the first n_per_token of them
    int64_t per_token_stride[2];
    int32_t n_per_token;
};
constexpr int kMostAccepted = 256;   // rows whose places are worked out at a time
constexpr int kRowsAhead = 8;

// VALUES: with columns of values per token (128 sequences 4.6 us without, 4.9 where one kernel serves both)
template <bool VALUES>
__global__ __launch_bounds__(kThreads) void kv_accept_kernel(accept_args a)
{
    __shared__ int64_t s_from[kMostAccepted], s_to[kMostAccepted];
    __shared__ int s_node[VALUES ? kMostAccepted : 1];
    const kv_view_dev& v = a.v;
    const int s = blockIdx.x, tid = threadIdx.x;
    const int q0 = a.q_off[s], q_len = a.q_off[s + 1] - q0, n = a.ctx_lens[s], first = n - q_len;
    const int count = (int)min((int64_t)min(max(a.n_accepted[s], 0), max(q_len, 0)), a.accepted_stride);
    if (a.new_lens && blockIdx.y == 0 && tid == 0) a.new_lens[s] = max(first + count, 0);
    if (first < 0) return;
    const int32_t* table = a.table + (int64_t)s * a.table_stride;
    const int row_pieces = v.n_kv_local * v.head_dim / 8;
    const int column = (int)blockIdx.y * kThreads + tid;
    const bool mine = column < 2 * row_pieces;
    const int plane = column >= row_pieces;
    const int64_t at = plane * v.plane_elems + (int64_t)(column - plane * row_pieces) * 8;
    // or a column of values per token
    const int value = column - 2 * row_pieces, which = value >= v.n_kv_local, head = value - which * v.n_kv_local;
    const bool has_value = VALUES && !mine && which < a.n_per_token && head < v.n_kv_local;
    const int64_t value_stride = has_value ? a.per_token_stride[which] : 0;
    uint32_t* const values = has_value ? a.per_token[which] + ((int64_t)s * v.n_kv_local + head) * value_stride : nullptr;
    for (int i0 = 0; i0 < count; i0 += kMostAccepted) {
        const int m = min(count - i0, kMostAccepted);
        __syncthreads();
        if (tid < m) {
            const int node = a.accepted[(int64_t)s * a.accepted_stride + i0 + tid];
            int64_t from = -1, to = -1;
            if (node > i0 + tid && node < q_len) {   // (node i0 + tid is in its place already)
                from = row_at(v, table, a.table_stride, a.n_pool_blocks, first + node);
                to = row_at(v, table, a.table_stride, a.n_pool_blocks, first + i0 + tid);
            }
            s_from[tid] = to < 0 ? -1 : from;
            s_to[tid] = to;
            if constexpr (VALUES) s_node[tid] = node;
        }
        __syncthreads();
        if (has_value) {
            for (int r = 0; r < m; r += kRowsAhead) {
                uint32_t x[kRowsAhead];
                auto moves = [&](int u) { return r + u < m && s_from[r + u] >= 0 && first + s_node[r + u] < value_stride; };
#pragma unroll
                for (int u = 0; u < kRowsAhead; ++u)
                    if (moves(u)) x[u] = values[first + s_node[r + u]];
#pragma unroll
                for (int u = 0; u < kRowsAhead; ++u)
                    if (moves(u)) values[first + i0 + r + u] = x[u];   // (its place lies before the old one)
            }
        }
        if (!mine) continue;
        for (int r = 0; r < m; r += kRowsAhead) {
            kv_u32x4 x[kRowsAhead];
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u)
                if (r + u < m && s_from[r + u] >= 0) x[u] = *reinterpret_cast<const kv_u32x4*>(a.pool + s_from[r + u] + at);
#pragma unroll
            for (int u = 0; u < kRowsAhead; ++u)
                if (r + u < m && s_from[r + u] >= 0) *reinterpret_cast<kv_u32x4*>(a.pool + s_to[r + u] + at) = x[u];
        }
    }
}

// ---- kv_evict ----------------------------------------------------------------------------------------
// Per (sequence, KV head), of n tokens the first k = min(n, keep) in the order (protected, larger weight, lower slot) are kept.
// Slots below k that are not kept are holes; kept tokens from slot k on fill them, the j-th the j-th.  There are as many of
// one as of the other, no row is both source and destination, and nothing else moves.
//
// The k-th weight is found by counting digits (11, 11 and 10 bits) of the weights' order-preserving integers, most
// significant first, among the protected tokens if there are k of them and among the others if not.  Then holes and sources
// are numbered in the order of their slots, by ballots of 64 and sums over those.  Up to 8192 tokens by one workgroup per
// (sequence, head) that holds them in registers (evict_select_kernel); more by parts of 4096, a launch per step, with the digits
// counted in the workspace (one workgroup for 131072 tokens took 260 us, bound by its own loads).  evict_move_kernel copies the
// rows, all independent of each other.

struct evict_args {
    uint16_t* pool;
    int64_t n_pool_blocks;
    const int32_t* table;
    int64_t table_stride;
    const int32_t *ctx_lens, *keep_lens, *next_pos;
    const float* weights;        // [batch][n_kv_local][stride]
    const int32_t* token_pos;
    float* weights_out;          // the same arrays or others
    int32_t* token_pos_out;
    int64_t stride, out_stride;
    int32_t* new_lens;
    int32_t sinks, recent, max_ctx_len;
    kv_view_dev v;
    int32_t* counts;             // [batch][n_kv_local] moves
    int32_t* lists;              // [batch][n_kv_local][2][most]: holes, sources
    int64_t most;
    // sequences of more than kAlone tokens:
    int32_t parts;               // of kPart tokens, by the host's bound
    int32_t* bins;               // [batch][n_kv_local][kAllBins], cleared first
    int4* part_counts;           // [batch][n_kv_local][parts] (over, on) below k, (over, on) from there on
};

constexpr int kDigits[3] = {11, 11, 10};
constexpr int kBins = 2048;
constexpr int kHeld = 8;                        // tokens a lane holds
constexpr int kAlone = 1024 * kHeld, kPart = 512 * kHeld;
constexpr int kAllBins = 4 * kBins + 16;   // first digit of both classes, second, third, number of protected tokens, lines
constexpr int kSecond = 2 * kBins, kThird = 3 * kBins, kProtected = 4 * kBins, kLines = kProtected + 1;

// Integers in the order of the weights; NaN below all, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (!(w == w)) return 0;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

// What a workgroup knows of its (sequence, head).
struct evict_pair {
    int n, k, s;
    int64_t sh, youngest;
    __device__ evict_pair(const evict_args& a, int s_, int h) : s(s_)
    {
        sh = (int64_t)s * a.v.n_kv_local + h;
        n = min(max(a.ctx_lens[s], 0), a.max_ctx_len);
        k = min(n, max(a.keep_lens[s], 0));
        youngest = (int64_t)a.next_pos[s] - a.recent;
    }
};

// The tokens base + NT i + thread of a workgroup: order numbers and classes (0 none, 1 ordinary, 2 protected).
template <int NT>
struct held_tokens {
    uint32_t key[kHeld];
    int cls[kHeld];
    __device__ void load(const evict_args& a, const evict_pair& p, int base)
    {
        float w[kHeld];
        int pos[kHeld];
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const int t = base + NT * i + (int)threadIdx.x;
            const int64_t at = p.sh * a.stride + min(t, p.n - 1);
            w[i] = a.weights[at];
            pos[i] = a.token_pos[at];
        }
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            key[i] = order_of(w[i]);
            cls[i] = base + NT * i + (int)threadIdx.x >= p.n ? 0 : pos[i] < a.sinks || (int64_t)pos[i] >= p.youngest ? 2 : 1;
        }
    }
    // Counts the digit of `width` bits below bit `shift` of those of the class whose upper bits are `prefix`.
    __device__ void count(int* bins, int of_class, int shift, int width, uint32_t prefix) const
    {
#pragma unroll
        for (int i = 0; i < kHeld; ++i) {
            const bool in = cls[i] == of_class && (shift == 32 || (key[i] >> (shift & 31)) == prefix);
            unsigned long long left = __builtin_amdgcn_ballot_w64(in);
            if (left == 0) continue;
            const int bin = (int)(key[i] >> (shift - width)) & ((1 << width) - 1);
            // tokens alike (many weigh nothing) are counted by one lane; the rest adds by itself
            const int leader = __builtin_ctzll(left), its = __builtin_amdgcn_readlane(bin, leader);
            const unsigned long long same = __builtin_amdgcn_ballot_w64(in && bin == its);
            if ((int)(threadIdx.x & 63) == leader) atomicAdd(&bins[its], __builtin_popcountll(same));
            if (in && bin != its) atomicAdd(&bins[bin], 1);
        }
    }
};

// Sum over the workgroup, in every thread; s_part: a word per wavefront.
template <int NT>
__device__ __forceinline__ int block_total(int x, int* s_part)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = x;
    __syncthreads();
    int t = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) t += s_part[w];
    return t;
}

// The bin that holds the rest-th of those counted, from the top, and how many of it are wanted.  Bins in LDS or in device memory.
template <int NT>
__device__ __forceinline__ void pick_bin(const int* bins, int n_bins, int& rest, int& bin, int* s_part, int* s_pick)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, each = n_bins / NT;   // consecutive bins a thread, the top first
    int mine[kBins / NT], sum = 0;
#pragma unroll
    for (int b = 0; b < kBins / NT; ++b) {
        mine[b] = b < each ? bins[n_bins - 1 - (tid * each + b)] : 0;
        sum += mine[b];
    }
    int incl = sum;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(incl, d);
        incl += lane >= d ? y : 0;
    }
    if (lane == 63) s_part[wave] = incl;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) incl += w < wave ? s_part[w] : 0;
    int before = incl - sum;
    if (before < rest && rest <= incl) {
#pragma unroll
        for (int b = 0; b < kBins / NT; ++b) {
            if (before < rest && rest <= before + mine[b]) {
                s_pick[0] = n_bins - 1 - (tid * each + b);
                s_pick[1] = rest - before;
            }
            before += mine[b];
        }
    }
    __syncthreads();
    bin = s_pick[0];
    rest = s_pick[1];
    __syncthreads();
}

// Where the line lies: `over` it stay all, `on` it the first `equals` by slot.
struct evict_line {
    int divided;       // the class that is divided; all of a higher one stay, none of a lower one
    uint32_t key;
    int equals;        // 0: nothing of the divided class stays
    __device__ bool over(uint32_t key_, int cls) const { return cls > divided || (cls == divided && equals > 0 && key_ > key); }
    __device__ bool on(uint32_t key_, int cls) const { return cls == divided && equals > 0 && key_ == key; }
};

// Kept tokens before a place, from sums over what lies before it: x, y over and on the line below slot k, z, w from there on.
__device__ __forceinline__ int kept_low(const evict_line& l, int over_low, int on_low) { return over_low + min(l.equals, on_low); }
__device__ __forceinline__ int kept_high(const evict_line& l, int on_low, int over_high, int on_high, int all_on_low)
{
    return over_high + max(min(l.equals, on_low + on_high) - min(l.equals, all_on_low), 0);
}

// Lists holes and sources among a workgroup's tokens and copies what stays, given the counts before them and of the whole pair;
// s_counts [4][NT / 64 * kHeld].  alone: the workgroup holds all of the pair's tokens, the counts before are 0 and those of the whole are its own.
template <int NT>
__device__ __forceinline__ void list_moves(const evict_args& a, const evict_pair& p, const evict_line& line, const held_tokens<NT>& x, int base, int4 before,
                                           int all_on_low, bool alone, int (*s_counts)[NT / 64 * kHeld], int* s_total)
{
    constexpr int NW = NT / 64, kSub = NW * kHeld;   // groups of 64 slots, in their order
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    unsigned long long over_b[kHeld], on_b[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int t = base + NT * i + tid;
        over_b[i] = __builtin_amdgcn_ballot_w64(line.over(x.key[i], x.cls[i]));
        on_b[i] = __builtin_amdgcn_ballot_w64(line.on(x.key[i], x.cls[i]));
        const unsigned long long low = __builtin_amdgcn_ballot_w64(t < p.k);
        if (lane < 4) {
            const unsigned long long which = (lane & 1 ? on_b[i] : over_b[i]) & (lane & 2 ? ~low : low);
            s_counts[lane][NW * i + wave] = __builtin_popcountll(which);
        }
    }
    __syncthreads();
    if (wave < 4) {   // wavefront c: exclusive sums of counts c
        int run = 0;
#pragma unroll
        for (int b = 0; b < kSub; b += 64) {
            const int y = s_counts[wave][b + lane];
            int incl = y;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int z = __shfl_up(incl, d);
                incl += lane >= d ? z : 0;
            }
            s_counts[wave][b + lane] = run + incl - y;
            run += __shfl(incl, 63);
        }
        if (lane == 0) s_total[wave] = run;
    }
    __syncthreads();
    if (alone) all_on_low = s_total[1];
    int32_t* hole_list = a.lists + p.sh * 2 * a.most;
    int32_t* source_list = hole_list + a.most;
    const bool elsewhere = a.weights_out != a.weights, pos_elsewhere = a.token_pos_out != a.token_pos;
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
        const int t = base + NT * i + tid, at = NW * i + wave;
        if (base + NT * i >= p.n) break;
        const int over_low = before.x + s_counts[0][at], on_low = before.y + s_counts[1][at];
        const int over_high = before.z + s_counts[2][at], on_high = before.w + s_counts[3][at];
        const int on_before = on_low + on_high;
        const bool is_on = on_b[i] >> lane & 1;
        const bool kept = (over_b[i] >> lane & 1) || (is_on && on_before + __builtin_popcountll(on_b[i] & below) < line.equals);
        const bool hole = t < p.k && !kept, source = t >= p.k && kept;   // (p.k <= n, and nothing past n is kept)
        const unsigned long long hole_b = __builtin_amdgcn_ballot_w64(hole), source_b = __builtin_amdgcn_ballot_w64(source);
        const int holes = min(t - lane, p.k) - kept_low(line, over_low, on_low);
        const int sources = kept_high(line, on_low, over_high, on_high, all_on_low);
        if (hole) hole_list[holes + __builtin_popcountll(hole_b & below)] = t;
        if (source) source_list[sources + __builtin_popcountll(source_b & below)] = t;
        if (t < p.k && kept && t < a.out_stride) {
            const int64_t from = p.sh * a.stride + t, to = p.sh * a.out_stride + t;
            if (elsewhere) a.weights_out[to] = a.weights[from];
            if (pos_elsewhere) a.token_pos_out[to] = a.token_pos[from];
        }
    }
    if (alone && tid == 0) a.counts[p.sh] = p.k - kept_low(line, s_total[0], s_total[1]);
}

// Nothing leaves: only copies, by `parts` workgroups.
__device__ __forceinline__ void copy_all(const evict_args& a, const evict_pair& p, int part, int parts)
{
    const bool elsewhere = a.weights_out != a.weights, pos_elsewhere = a.token_pos_out != a.token_pos;
    for (int64_t t = (int64_t)part * blockDim.x + threadIdx.x; t < min((int64_t)p.n, a.out_stride); t += (int64_t)parts * blockDim.x) {
        if (elsewhere) a.weights_out[p.sh * a.out_stride + t] = a.weights[p.sh * a.stride + t];
        if (pos_elsewhere) a.token_pos_out[p.sh * a.out_stride + t] = a.token_pos[p.sh * a.stride + t];
    }
}

template <int NT>
__global__ __launch_bounds__(NT) void evict_select_kernel(evict_args a)
{
    __shared__ int s_bins[kBins], s_part[NT / 64], s_pick[2], s_total[4];
    __shared__ int s_counts[4][NT / 64 * kHeld];
    const int tid = threadIdx.x;
    const evict_pair p(a, blockIdx.x, blockIdx.y);
    if (blockIdx.y == 0 && tid == 0 && a.new_lens) a.new_lens[p.s] = p.k;
    if (p.k == p.n) {
        if (tid == 0 && a.counts) a.counts[p.sh] = 0;
        copy_all(a, p, 0, 1);
        return;
    }
    held_tokens<NT> x;
    x.load(a, p, 0);
    int here = 0;
#pragma unroll
    for (int i = 0; i < kHeld; ++i) here += x.cls[i] == 2;
    const int shielded = block_total<NT>(here, s_part);
    evict_line line;
    line.divided = shielded >= p.k ? 2 : 1;
    line.key = 0;
    line.equals = line.divided == 2 ? p.k : p.k - shielded;
    int shift = 32;
    if (line.equals > 0) {
#pragma unroll
        for (int d = 0; d < 3; ++d) {
            for (int b = tid; b < kBins; b += NT) s_bins[b] = 0;
            __syncthreads();
            x.count(s_bins, line.divided, shift, kDigits[d], line.key);
            __syncthreads();
            int bin;
            pick_bin<NT>(s_bins, 1 << kDigits[d], line.equals, bin, s_part, s_pick);
            line.key = line.key << kDigits[d] | (uint32_t)bin;
            shift -= kDigits[d];
        }
    }
    list_moves<NT>(a, p, line, x, 0, make_int4(0, 0, 0, 0), 0, true, s_counts, s_total);
}

// ---- more than kAlone tokens: a launch per step, block (part, head, sequence)
__global__ __launch_bounds__(256) void evict_clear_kernel(int32_t* bins, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) bins[i] = 0;
}

// The line as far as the digits counted so far tell: what the launch before found, and one digit more, left for the next launch.
template <int NT>
__device__ __forceinline__ evict_line next_line(const evict_args& a, const evict_pair& p, int digit, bool writes, int* s_part, int* s_pick)
{
    int* const bins = a.bins + p.sh * kAllBins;
    int* const kept = bins + kLines;   // (divided, key, equals) after each digit
    evict_line line;
    if (digit == 0) {
        const int shielded = bins[kProtected];
        line.divided = shielded >= p.k ? 2 : 1;
        line.key = 0;
        line.equals = line.divided == 2 ? p.k : p.k - shielded;
    } else {
        line.divided = kept[3 * (digit - 1)];
        line.key = (uint32_t)kept[3 * (digit - 1) + 1];
        line.equals = kept[3 * (digit - 1) + 2];
    }
    if (digit < 3) {
        if (line.equals > 0) {
            const int at = digit == 0 ? (line.divided - 1) * kBins : digit == 1 ? kSecond : kThird;
            int bin;
            pick_bin<NT>(bins + at, 1 << kDigits[digit], line.equals, bin, s_part, s_pick);
            line.key = line.key << kDigits[digit] | (uint32_t)bin;
        }
        if (writes && threadIdx.x == 0) {
            kept[3 * digit] = line.divided;
            kept[3 * digit + 1] = (int)line.key;
            kept[3 * digit + 2] = line.equals;
        }
    }
    return line;
}

// Sums of six counts over the workgroup, in every thread.
template <int NT>
__device__ __forceinline__ void block_totals(int (&x)[6], int (*s_six)[6])
{
#pragma unroll
    for (int q = 0; q < 6; ++q)
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) x[q] += __shfl_xor(x[q], d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
        for (int q = 0; q < 6; ++q) s_six[threadIdx.x >> 6][q] = x[q];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 6; ++q) {
        x[q] = 0;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) x[q] += s_six[w][q];
    }
}

template <int STEP>   // 0, 1, 2: counts that digit; 3: counts tokens over and on the line; 4: lists the moves
__global__ __launch_bounds__(512) void evict_part_kernel(evict_args a)
{
    constexpr int NT = 512;
    __shared__ int s_bins[STEP == 0 ? 2 * kBins : STEP < 3 ? kBins : 1], s_part[NT / 64], s_pick[2], s_total[4];
    __shared__ int s_counts[4][STEP == 4 ? NT / 64 * kHeld : 64], s_six[NT / 64][6];
    const int tid = threadIdx.x, part = blockIdx.x, base = part * kPart;
    const evict_pair p(a, blockIdx.z, blockIdx.y);
    if (STEP == 0 && part == 0 && blockIdx.y == 0 && tid == 0 && a.new_lens) a.new_lens[p.s] = p.k;
    if (p.k == p.n) {
        if (STEP == 4) copy_all(a, p, part, gridDim.x);
        if (STEP == 4 && part == 0 && tid == 0) a.counts[p.sh] = 0;
        return;
    }
    if (base >= p.n) return;
    int32_t* bins = a.bins + p.sh * kAllBins;
    held_tokens<NT> x;
    x.load(a, p, base);
    if constexpr (STEP < 3) {
        evict_line line{1, 0, 1};
        if constexpr (STEP > 0) {
            line = next_line<NT>(a, p, STEP - 1, part == 0, s_part, s_pick);
            if (line.equals == 0) return;
        }
        constexpr int kCounted = STEP == 0 ? 2 * kBins : 1 << kDigits[STEP];
        for (int b = tid; b < kCounted; b += NT) s_bins[b] = 0;
        __syncthreads();
        if constexpr (STEP == 0) {
            int here = 0;
#pragma unroll
            for (int i = 0; i < kHeld; ++i) here += x.cls[i] == 2;
            const int shielded = block_total<NT>(here, s_part);
            if (tid == 0 && shielded) atomicAdd(&bins[kProtected], shielded);
            x.count(s_bins, 1, 32, kDigits[0], 0);
            x.count(s_bins + kBins, 2, 32, kDigits[0], 0);
        } else {
            x.count(s_bins, line.divided, STEP == 1 ? 32 - kDigits[0] : kDigits[2], kDigits[STEP], line.key);
        }
        __syncthreads();
        int32_t* to = bins + (STEP == 0 ? 0 : STEP == 1 ? kSecond : kThird);
        for (int b = tid; b < kCounted; b += NT)
            if (s_bins[b]) atomicAdd(&to[b], s_bins[b]);
    } else {
        const evict_line line = next_line<NT>(a, p, STEP - 1, part == 0, s_part, s_pick);
        int4* counts = a.part_counts + p.sh * a.parts;
        if constexpr (STEP == 3) {
            int c[6] = {0, 0, 0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < kHeld; ++i) {
                const int high = base + NT * i + tid >= p.k;
                const int over = line.over(x.key[i], x.cls[i]), on = line.on(x.key[i], x.cls[i]);
                c[0] += high ? 0 : over;
                c[1] += high ? 0 : on;
                c[2] += high ? over : 0;
                c[3] += high ? on : 0;
            }
            block_totals<NT>(c, s_six);
            if (tid == 0) counts[part] = make_int4(c[0], c[1], c[2], c[3]);
        } else {
            int c[6] = {0, 0, 0, 0, 0, 0};   // before this part; over and on the line below slot k in all
            const int parts = (p.n + kPart - 1) / kPart;
            for (int q = tid; q < parts; q += NT) {
                const int4 y = counts[q];
                c[4] += y.x;
                c[5] += y.y;
                if (q < part) {
                    c[0] += y.x;
                    c[1] += y.y;
                    c[2] += y.z;
                    c[3] += y.w;
                }
            }
            block_totals<NT>(c, s_six);
            if (part == 0 && tid == 0) a.counts[p.sh] = p.k - kept_low(line, c[4], c[5]);
            list_moves<NT>(a, p, line, x, base, make_int4(c[0], c[1], c[2], c[3]), c[5], false, s_counts, s_total);
        }
    }
}

// Block (x, head, sequence): moves x, x + gridDim.x, .. by groups that fill the workgroup.
__global__ __launch_bounds__(kThreads) void evict_move_kernel(evict_args a)
{
    const kv_view_dev& v = a.v;
    const int h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
    const int64_t sh = (int64_t)s * v.n_kv_local + h;
    const int count = a.counts[sh];
    const int32_t* hole_list = a.lists + sh * 2 * a.most;
    const int32_t* source_list = hole_list + a.most;
    const int32_t* table = a.table + (int64_t)s * a.table_stride;
    const int row_pieces = v.head_dim / 8, per_move = 2 * row_pieces;   // 16-byte pieces of K and V
    constexpr int kUnroll = 2;   // (four in half as many workgroups: 24 us in place of 22 for 60 MB)
    const int total = count * per_move;   // (the host keeps it below 2^31 by more than a step)
    for (int x0 = (int)blockIdx.x * kThreads * kUnroll + tid; x0 < total; x0 += (int)gridDim.x * kThreads * kUnroll) {
        kv_u32x4 val[kUnroll];
        int64_t to[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int x = x0 + u * kThreads;
            to[u] = -1;
            if (x >= total) continue;
            const int j = x / per_move, c = x - j * per_move, plane = c >= row_pieces;
            const int hole = hole_list[j], source = source_list[j];
            const int64_t in = plane * v.plane_elems + h * v.head_dim + (c - plane * row_pieces) * 8;
            const int64_t from = row_at(v, table, a.table_stride, a.n_pool_blocks, source);
            to[u] = row_at(v, table, a.table_stride, a.n_pool_blocks, hole);
            if (from < 0 || to[u] < 0) {
                to[u] = -1;
                continue;
            }
            val[u] = *reinterpret_cast<const kv_u32x4*>(a.pool + from + in);
            to[u] += in;
            if (c == 0 && hole < a.out_stride) {
                a.weights_out[sh * a.out_stride + hole] = a.weights[sh * a.stride + source];
                a.token_pos_out[sh * a.out_stride + hole] = a.token_pos[sh * a.stride + source];
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
            if (to[u] >= 0) *reinterpret_cast<kv_u32x4*>(a.pool + to[u]) = val[u];
    }
}

// Where things lie in the workspace
struct evict_room {
    int64_t heads, most, parts;
    size_t lists, bins, counts, bytes;
};
evict_room room_for(const kv_view* view, int batch, int max_ctx_len)
{
    auto whole = [](size_t x) { return (x + 255) / 256 * 256; };
    evict_room r;
    r.heads = (int64_t)batch * view->n_kv_local;
    r.most = max_ctx_len / 2 + 1;   // a hole and a source are two tokens
    r.parts = max_ctx_len > kAlone ? (max_ctx_len + kPart - 1) / kPart : 0;
    r.lists = whole(r.heads * 4);
    r.bins = r.lists + whole(r.heads * 8 * r.most);
    r.counts = r.bins + (r.parts ? whole(r.heads * 4 * kAllBins) : 0);
    r.bytes = r.counts + whole(r.heads * 16 * r.parts);
    return r;
}

}  // namespace

extern "C" int kv_accept(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const int32_t* block_table,
                         int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* accepted,
                         int64_t accepted_stride, const int32_t* n_accepted, int batch, int32_t* new_lens, void* hip_stream)
{
    return kv_accept_tracked(kv_pool, n_pool_blocks, view, block_table, block_table_stride, ctx_lens, q_offsets, accepted, accepted_stride,
                             n_accepted, batch, new_lens, nullptr, 0, nullptr, 0, hip_stream);
}

extern "C" int kv_accept_tracked(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const int32_t* block_table,
                                 int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* accepted,
                                 int64_t accepted_stride, const int32_t* n_accepted, int batch, int32_t* new_lens, int32_t* token_pos,
                                 int64_t token_pos_stride, float* weights, int64_t weights_stride, void* hip_stream)
{
    if (!kv_view_ok(view) || n_pool_blocks < 0 || block_table_stride < 0 || accepted_stride < 0 || batch < 0 || token_pos_stride < 0 ||
        weights_stride < 0)
        return KV_ERR_INVALID_ARG;
    if (batch == 0) return KV_OK;
    if (!kv_pool || !block_table || !ctx_lens || !q_offsets || !accepted || !n_accepted) return KV_ERR_INVALID_ARG;
    // (a sequence's workgroups all read what one of them would overwrite)
    if (new_lens && (kv_words_meet(new_lens, batch, ctx_lens, batch) || kv_words_meet(new_lens, batch, q_offsets, (int64_t)batch + 1) ||
                     kv_words_meet(new_lens, batch, n_accepted, batch) || kv_words_meet(new_lens, batch, accepted, batch * accepted_stride)))
        return KV_ERR_INVALID_ARG;
    if (!kv_aligned(kv_pool, 16)) return KV_ERR_UNSUPPORTED;
    accept_args a = {};
    a.pool = (uint16_t*)kv_pool;
    a.n_pool_blocks = n_pool_blocks;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.q_off = q_offsets;
    a.accepted = accepted;
    a.accepted_stride = accepted_stride;
    a.n_accepted = n_accepted;
    a.new_lens = new_lens;
    a.v = kv_view_to_dev(view);
    if (token_pos) {
        a.per_token[a.n_per_token] = (uint32_t*)token_pos;
        a.per_token_stride[a.n_per_token++] = token_pos_stride;
    }
    if (weights) {
        a.per_token[a.n_per_token] = (uint32_t*)weights;
        a.per_token_stride[a.n_per_token++] = weights_stride;
    }
    const int64_t columns = (int64_t)view->n_kv_local * (view->geom.head_dim / 4 + a.n_per_token), parts = (columns + kThreads - 1) / kThreads;
    if (parts > 65535) return KV_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)batch, (unsigned)parts);
    if (a.n_per_token) hipLaunchKernelGGL(kv_accept_kernel<true>, grid, dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    else hipLaunchKernelGGL(kv_accept_kernel<false>, grid, dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return kv_record_hip_error(hipGetLastError(), "kv_accept launch");
}

extern "C" size_t kv_evict_workspace_bytes(const kv_view* view, int batch, int max_ctx_len)
{
    if (!kv_view_ok(view) || batch <= 0 || max_ctx_len <= 0) return 0;
    return room_for(view, batch, max_ctx_len).bytes;
}

extern "C" int kv_evict(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const int32_t* block_table,
                        int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* keep_lens, int batch, int max_ctx_len,
                        const float* weights, const int32_t* token_pos, int64_t stride, const int32_t* next_pos, int sinks,
                        int recent, float* weights_out, int32_t* token_pos_out, int64_t out_stride, int32_t* new_lens,
                        void* workspace, size_t workspace_bytes, void* hip_stream)
{
    if (!kv_view_ok(view) || n_pool_blocks < 0 || block_table_stride < 0 || batch < 0 || max_ctx_len < 0 || sinks < 0 || recent < 0)
        return KV_ERR_INVALID_ARG;
    if (batch == 0) return KV_OK;
    if (!kv_pool || !block_table || !ctx_lens || !keep_lens || !weights || !token_pos || !next_pos || !weights_out || !token_pos_out)
        return KV_ERR_INVALID_ARG;
    if (new_lens && (kv_words_meet(new_lens, batch, ctx_lens, batch) || kv_words_meet(new_lens, batch, keep_lens, batch) ||
                     kv_words_meet(new_lens, batch, next_pos, batch)))
        return KV_ERR_INVALID_ARG;
    if (stride < max_ctx_len || out_stride < 0 || ((weights_out == weights || token_pos_out == token_pos) && out_stride != stride) ||
        block_table_stride < ((int64_t)max_ctx_len + view->block_tokens - 1) / view->block_tokens)
        return KV_ERR_INVALID_ARG;
    // (a list holds half of the tokens; evict_move_kernel counts 16-byte pieces of K and V, and goes past the end by a step of all its workgroups, 2^21)
    const int64_t most_pieces = ((int64_t)max_ctx_len / 2 + 1) * (view->geom.head_dim / 4);
    if (!kv_aligned(kv_pool, 16) || most_pieces > 0x7f000000 || max_ctx_len > (1 << 24) || batch > 65535 || view->n_kv_local > 65535) return KV_ERR_UNSUPPORTED;
    if (max_ctx_len > 0) {
        if (!workspace || ((uintptr_t)workspace & 255u)) return KV_ERR_INVALID_ARG;
        if (workspace_bytes < kv_evict_workspace_bytes(view, batch, max_ctx_len)) return KV_ERR_WORKSPACE;
    }
    evict_args a = {};
    a.pool = (uint16_t*)kv_pool;
    a.n_pool_blocks = n_pool_blocks;
    a.table = block_table;
    a.table_stride = block_table_stride;
    a.ctx_lens = ctx_lens;
    a.keep_lens = keep_lens;
    a.next_pos = next_pos;
    a.weights = weights;
    a.token_pos = token_pos;
    a.weights_out = weights_out;
    a.token_pos_out = token_pos_out;
    a.stride = stride;
    a.out_stride = out_stride;
    a.new_lens = new_lens;
    a.sinks = sinks;
    a.recent = recent;
    a.max_ctx_len = max_ctx_len;
    a.v = kv_view_to_dev(view);
    hipStream_t st = (hipStream_t)hip_stream;
    if (max_ctx_len == 0) {   // (no workspace: only new_lens is written)
        hipLaunchKernelGGL(evict_select_kernel<512>, dim3((unsigned)batch, (unsigned)view->n_kv_local), dim3(512), 0, st, a);
        return kv_record_hip_error(hipGetLastError(), "kv_evict launch");
    }
    const evict_room r = room_for(view, batch, max_ctx_len);
    a.counts = (int32_t*)workspace;
    a.lists = (int32_t*)((char*)workspace + r.lists);
    a.most = r.most;
    if (r.parts == 0) {
        // The smaller workgroup waits less at its barriers and shares a compute unit: us per call, 1024 threads / 512, sequences of 1000 to
        // 2000 and 8 heads, 4 of them 18.3 / 16.9, 16 27.0 / 25.8, 64 86.9 / 78.5
        const dim3 grid((unsigned)batch, (unsigned)view->n_kv_local);
        if (max_ctx_len <= 512 * kHeld) hipLaunchKernelGGL(evict_select_kernel<512>, grid, dim3(512), 0, st, a);
        else hipLaunchKernelGGL(evict_select_kernel<1024>, grid, dim3(1024), 0, st, a);
    } else {
        a.parts = (int32_t)r.parts;
        a.bins = (int32_t*)((char*)workspace + r.bins);
        a.part_counts = (int4*)((char*)workspace + r.counts);
        const int64_t words = r.heads * kAllBins;
        hipLaunchKernelGGL(evict_clear_kernel, dim3((unsigned)((words + 2047) / 2048 < 1024 ? (words + 2047) / 2048 : 1024)), dim3(256), 0, st, a.bins, words);
        const dim3 grid((unsigned)r.parts, (unsigned)view->n_kv_local, (unsigned)batch);
        hipLaunchKernelGGL(evict_part_kernel<0>, grid, dim3(512), 0, st, a);
        hipLaunchKernelGGL(evict_part_kernel<1>, grid, dim3(512), 0, st, a);
        hipLaunchKernelGGL(evict_part_kernel<2>, grid, dim3(512), 0, st, a);
        hipLaunchKernelGGL(evict_part_kernel<3>, grid, dim3(512), 0, st, a);
        hipLaunchKernelGGL(evict_part_kernel<4>, grid, dim3(512), 0, st, a);
    }
    // two workgroups for every one that the chip holds, each moving 8 tokens or more at a time
    int64_t each = (4096 + r.heads - 1) / r.heads;
    const int64_t useful = (r.most * view->geom.head_dim / 4 + kThreads * 2 - 1) / (kThreads * 2);
    if (each > useful) each = useful;
    hipLaunchKernelGGL(evict_move_kernel, dim3((unsigned)each, (unsigned)view->n_kv_local, (unsigned)batch), dim3(kThreads), 0, st, a);
    return kv_record_hip_error(hipGetLastError(), "kv_evict launch");
}
