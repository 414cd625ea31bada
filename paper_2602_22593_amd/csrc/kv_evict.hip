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
// progress, and may request several before it stores them.  Latency is all there is to it: lengths, nodes, table, rows.

struct accept_args {
    uint16_t* pool;
    int64_t n_pool_blocks;
    const int32_t* table;
    int64_t table_stride;
    const int32_t *ctx_lens, *q_off, *accepted, *n_accepted;
    int64_t accepted_stride;
    int32_t* new_lens;
    kv_view_dev v;
};
constexpr int kMostAccepted = 256;   // rows whose places are worked out at a time
constexpr int kRowsAhead = 8;

__global__ __launch_bounds__(kThreads) void kv_accept_kernel(accept_args a)
{
    __shared__ int64_t s_from[kMostAccepted], s_to[kMostAccepted];
    const kv_view_dev& v = a.v;
    const int s = blockIdx.x, tid = threadIdx.x;
    const int q0 = a.q_off[s], q_len = a.q_off[s + 1] - q0, n = a.ctx_lens[s], first = n - q_len;
    const int count = (int)min((int64_t)min(max(a.n_accepted[s], 0), max(q_len, 0)), a.accepted_stride);
    if (a.new_lens && blockIdx.y == 0 && tid == 0) a.new_lens[s] = first + count;
    if (first < 0) return;
    const int32_t* table = a.table + (int64_t)s * a.table_stride;
    const int row_pieces = v.n_kv_local * v.head_dim / 8;
    const int column = (int)blockIdx.y * kThreads + tid;
    const bool mine = column < 2 * row_pieces;
    const int plane = column >= row_pieces;
    const int64_t at = plane * v.plane_elems + (int64_t)(column - plane * row_pieces) * 8;
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
        }
        __syncthreads();
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
// kv_evict_select_kernel, a workgroup per (sequence, head): the k-th weight by counting digits of the weights' order-preserving
// integers, most significant first, among the protected tokens if there are k of them and among the others if not; then
// wavefronts that each own a range of slots number holes and sources by ballots.  kv_evict_move_kernel copies the rows.

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
};

constexpr int kSelectThreads = 1024, kWaves = kSelectThreads / 64;
constexpr int kDigit = 11, kBins = 1 << kDigit;

// Integers in the order of the weights; NaN below all, the two zeros alike.
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (!(w == w)) return 0;
    const uint32_t u = __float_as_uint(w == 0.f ? 0.f : w);
    return (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int evict_keep(const evict_args& a, int s, int n) { return min(n, max(a.keep_lens[s], 0)); }

__global__ __launch_bounds__(kSelectThreads) void kv_evict_select_kernel(evict_args a)
{
    __shared__ int s_bins[kBins];
    __shared__ int s_wave[kWaves][4];
    __shared__ int s_pick[2];
    const int s = blockIdx.x, h = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int Hl = a.v.n_kv_local;
    const int64_t sh = (int64_t)s * Hl + h;
    const int n = min(max(a.ctx_lens[s], 0), a.max_ctx_len), k = evict_keep(a, s, n);
    const float* weights = a.weights + sh * a.stride;
    const int32_t* pos = a.token_pos + sh * a.stride;
    float* weights_out = a.weights_out + sh * a.out_stride;
    int32_t* pos_out = a.token_pos_out + sh * a.out_stride;
    const bool elsewhere = a.weights_out != a.weights, pos_elsewhere = a.token_pos_out != a.token_pos;
    if (h == 0 && tid == 0 && a.new_lens) a.new_lens[s] = k;
    if (k == n) {   // nothing leaves
        if (tid == 0 && a.counts) a.counts[sh] = 0;
        for (int t = tid; t < min((int64_t)n, a.out_stride); t += kSelectThreads) {
            if (elsewhere) weights_out[t] = weights[t];
            if (pos_elsewhere) pos_out[t] = pos[t];
        }
        return;
    }
    const int64_t youngest = (int64_t)a.next_pos[s] - a.recent;
    auto is_protected = [&](int p) { return p < a.sinks || (int64_t)p >= youngest; };

    // how many are protected, and which class is divided
    int here = 0;
    for (int t = tid; t < n; t += kSelectThreads) here += is_protected(pos[t]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) here += __shfl_xor(here, d);
    if (lane == 0) s_wave[wave][0] = here;
    __syncthreads();
    int shielded = 0;
    for (int w = 0; w < kWaves; ++w) shielded += s_wave[w][0];
    const bool among = shielded >= k;            // the line lies among the protected ones
    int rest = among ? k : k - shielded;         // of the divided class these many stay
    __syncthreads();

    // the order number of the last one that stays: its digits from the top
    uint32_t prefix = 0;
    int shift = 32;
    for (int pass = 0; pass < 3 && rest > 0; ++pass) {
        const int width = pass < 2 ? kDigit : 32 - 2 * kDigit;
        for (int b = tid; b < kBins; b += kSelectThreads) s_bins[b] = 0;
        __syncthreads();
        for (int t = tid; t < n; t += kSelectThreads) {
            if (is_protected(pos[t]) != among) continue;
            const uint32_t u = order_of(weights[t]);
            if (shift < 32 && (u >> shift) != prefix) continue;
            atomicAdd(&s_bins[(u >> (shift - width)) & ((1 << width) - 1)], 1);
        }
        __syncthreads();
        // the bin that holds the rest-th from the top: lane l of the first wavefront looks at bins of 1 / 64 of the range
        if (wave == 0) {
            const int bins = 1 << width, each = bins / 64, top = bins - 1 - lane * each;
            int sum = 0;
            for (int b = 0; b < each; ++b) sum += s_bins[top - b];
            int incl = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int y = __shfl_up(incl, d);
                incl += lane >= d ? y : 0;
            }
            const int before = incl - sum;
            if (before < rest && rest <= incl) {
                int left = rest - before, b = top;
                while (s_bins[b] < left) left -= s_bins[b--];
                s_pick[0] = b;
                s_pick[1] = left;
            }
        }
        __syncthreads();
        prefix = prefix << width | (uint32_t)s_pick[0];
        rest = s_pick[1];
        shift -= width;
        __syncthreads();
    }
    // stays: above the line in the divided class, or on it among the first `rest` by slot; and all of the upper class
    const int equals = rest;
    const bool none = (among ? k : k - shielded) == 0;
    auto state = [&](int t, bool& over, bool& on) {
        over = on = false;
        if (t >= n) return;
        const bool p = is_protected(pos[t]);
        if (p != among) {
            over = p;
            return;
        }
        if (none) return;
        const uint32_t u = order_of(weights[t]);
        over = u > prefix;
        on = u == prefix;
    };
    const int each = ((n + kWaves - 1) / kWaves + 63) & ~63, t0 = min(wave * each, n), t1 = min(t0 + each, n);
    int over_low = 0, on_low = 0, over_high = 0, on_high = 0;   // in slots below k, and from there on
    for (int t = t0; t < t1; t += 64) {
        bool over, on;
        state(t + lane < t1 ? t + lane : n, over, on);
        const bool low = t + lane < k;
        over_low += __builtin_popcountll(__builtin_amdgcn_ballot_w64(over && low));
        on_low += __builtin_popcountll(__builtin_amdgcn_ballot_w64(on && low));
        over_high += __builtin_popcountll(__builtin_amdgcn_ballot_w64(over && !low));
        on_high += __builtin_popcountll(__builtin_amdgcn_ballot_w64(on && !low));
    }
    if (lane == 0) {
        s_wave[wave][0] = over_low;
        s_wave[wave][1] = on_low;
        s_wave[wave][2] = over_high;
        s_wave[wave][3] = on_high;
    }
    __syncthreads();
    int on_before = 0, holes = 0, sources = 0, all_sources = 0;   // before this wavefront's range
    {
        int seen = 0, kept_low = 0, kept_high = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) {
                on_before = seen;
                holes = min(t0, k) - kept_low;
                sources = kept_high;
            }
            const int low = min(max(equals - seen, 0), s_wave[w][1]);
            kept_low += s_wave[w][0] + low;
            seen += s_wave[w][1];
            const int high = min(max(equals - seen, 0), s_wave[w][3]);
            kept_high += s_wave[w][2] + high;
            seen += s_wave[w][3];
        }
        all_sources = kept_high;
    }
    if (tid == 0) a.counts[sh] = all_sources;
    int32_t* hole_list = a.lists + sh * 2 * a.most;
    int32_t* source_list = hole_list + a.most;
    const unsigned long long below = (1ull << lane) - 1;
    for (int t = t0; t < t1; t += 64) {
        bool over, on;
        const int at = t + lane;
        state(at < t1 ? at : n, over, on);
        const unsigned long long ons = __builtin_amdgcn_ballot_w64(on);
        const bool kept = over || (on && on_before + __builtin_popcountll(ons & below) < equals);
        on_before += __builtin_popcountll(ons);
        const bool inside = at < t1, hole = inside && at < k && !kept, source = inside && at >= k && kept;
        const unsigned long long hole_b = __builtin_amdgcn_ballot_w64(hole), source_b = __builtin_amdgcn_ballot_w64(source);
        if (hole) hole_list[holes + __builtin_popcountll(hole_b & below)] = at;
        if (source) source_list[sources + __builtin_popcountll(source_b & below)] = at;
        holes += __builtin_popcountll(hole_b);
        sources += __builtin_popcountll(source_b);
        if (inside && at < k && kept && at < a.out_stride) {
            if (elsewhere) weights_out[at] = weights[at];
            if (pos_elsewhere) pos_out[at] = pos[at];
        }
    }
}

// Block (x, head, sequence): moves x, x + gridDim.x, .. by groups that fill the workgroup.
__global__ __launch_bounds__(kThreads) void kv_evict_move_kernel(evict_args a)
{
    const kv_view_dev& v = a.v;
    const int h = blockIdx.y, s = blockIdx.z, tid = threadIdx.x;
    const int64_t sh = (int64_t)s * v.n_kv_local + h;
    const int count = a.counts[sh];
    const int32_t* hole_list = a.lists + sh * 2 * a.most;
    const int32_t* source_list = hole_list + a.most;
    const int32_t* table = a.table + (int64_t)s * a.table_stride;
    const int row_pieces = v.head_dim / 8, per_move = 2 * row_pieces;   // 16-byte pieces of K and V
    constexpr int kUnroll = 4;
    const int total = count * per_move;   // (a list is shorter than 2^24)
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

int64_t most_moves(int max_ctx_len) { return max_ctx_len / 2 + 1; }

}  // namespace

extern "C" int kv_accept(void* kv_pool, int64_t n_pool_blocks, const kv_view* view, const int32_t* block_table,
                         int64_t block_table_stride, const int32_t* ctx_lens, const int32_t* q_offsets, const int32_t* accepted,
                         int64_t accepted_stride, const int32_t* n_accepted, int batch, int32_t* new_lens, void* hip_stream)
{
    if (!kv_view_ok(view) || n_pool_blocks < 0 || block_table_stride < 0 || accepted_stride < 0 || batch < 0) return KV_ERR_INVALID_ARG;
    if (batch == 0) return KV_OK;
    if (!kv_pool || !block_table || !ctx_lens || !q_offsets || !accepted || !n_accepted || new_lens == ctx_lens) return KV_ERR_INVALID_ARG;
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
    const int64_t columns = 2 * (int64_t)view->n_kv_local * view->geom.head_dim / 8, parts = (columns + kThreads - 1) / kThreads;
    if (parts > 65535) return KV_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(kv_accept_kernel, dim3((unsigned)batch, (unsigned)parts), dim3(kThreads), 0, (hipStream_t)hip_stream, a);
    return kv_record_hip_error(hipGetLastError(), "kv_accept launch");
}

extern "C" size_t kv_evict_workspace_bytes(const kv_view* view, int batch, int max_ctx_len)
{
    if (!kv_view_ok(view) || batch <= 0 || max_ctx_len <= 0) return 0;
    return (size_t)batch * view->n_kv_local * 4 * (1 + 2 * (size_t)most_moves(max_ctx_len));
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
    if (!kv_pool || !block_table || !ctx_lens || !keep_lens || !weights || !token_pos || !next_pos || !weights_out || !token_pos_out ||
        new_lens == ctx_lens || new_lens == keep_lens)
        return KV_ERR_INVALID_ARG;
    if (stride < max_ctx_len || out_stride < 0 || ((weights_out == weights || token_pos_out == token_pos) && out_stride != stride) ||
        block_table_stride < ((int64_t)max_ctx_len + view->block_tokens - 1) / view->block_tokens)
        return KV_ERR_INVALID_ARG;
    if (max_ctx_len > (1 << 24) || batch > 65535 || view->n_kv_local > 65535) return KV_ERR_UNSUPPORTED;
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
    const int64_t heads = (int64_t)batch * view->n_kv_local;
    a.counts = (int32_t*)workspace;
    a.lists = a.counts + heads;
    a.most = most_moves(max_ctx_len);
    hipStream_t st = (hipStream_t)hip_stream;
    hipLaunchKernelGGL(kv_evict_select_kernel, dim3((unsigned)batch, (unsigned)view->n_kv_local), dim3(kSelectThreads), 0, st, a);
    if (max_ctx_len > 0) {
        // workgroups for eight rounds of the chip, each moving 8 tokens or more at a time
        int64_t each = (2048 + heads - 1) / heads;
        const int64_t useful = (a.most * view->geom.head_dim / 4 + kThreads * 4 - 1) / (kThreads * 4);
        if (each > useful) each = useful;
        hipLaunchKernelGGL(kv_evict_move_kernel, dim3((unsigned)each, (unsigned)view->n_kv_local, (unsigned)batch), dim3(kThreads), 0, st, a);
    }
    return kv_record_hip_error(hipGetLastError(), "kv_evict launch");
}
