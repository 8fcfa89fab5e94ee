// What a step that verifies drafted tokens does with its trees: tables from the parents, and what stays of the step.
//
// Tables.  A row's ancestors are its parent's and its parent; its position is its request's cached length + their number.  One workgroup per request, a thread per row: in
// round r a thread takes over the bits and the count of the row 2^r generations up, and that row's pointer, so a path of 256 rows takes 8 rounds and a tree
// of a few generations two or three (the rounds end when no pointer is left).  Latency: parents -> rounds in LDS -> store; 4.1 us for 64 requests of 4 - 32 rows, 6.7 for 256 of 16 - 256
// (an empty kernel: 4), a tenth of a megabyte.  A walk from each row to its root instead is a chain of as many dependent reads as the tree has generations.
//
// Keep.  The walk down a tree is a chain of one step per row that stays: one wave per request holds parents, tokens and choices in registers, a step
// is a ballot over the rows.  A second launch moves the rows, a workgroup per request and layer, and puts pages back: both need walks that are over.  Calls of few requests are one launch: every
// workgroup walks its own tree again, the one that sees to the pages walks all (1 - 16 requests, 2 or 32 layers: 9.5 - 11.0 us a call for 13.6 - 14.7, as
// a launch less is issued; captured, where issue does not count, 6.6 - 7.8 for 5.3 - 6.4.  With room for walks of 32 requests: 12.0 captured for 16 of them, 12.3 - 14.8 for 32).
// Kept row i comes from row path[i] >= i, and path ascends, so no row is read behind a store to it (a thread moves its bytes of all rows, in their order).
// Latency: 64 requests, 32 layers (31 MB read and written, at 5 TB/s 6 us) captured 9.9 us; the places of all rows are looked up beside the walk, or beside what it left.
#include "fr_internal.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr int N_MAX = FR_TREE_MAX_ROWS, WORDS = N_MAX / 32;
constexpr int TB = 256;
static_assert(N_MAX == TB, "a thread per row");
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

struct Rows { int first, n, all; };   // of a request: its first row, how many count, how many there are
__device__ __forceinline__ Rows rows_of(const int32_t* q_offsets, int b, int T, int max_new) {
    const int lo = max(min(q_offsets[b], T), 0), hi = max(min(q_offsets[b + 1], T), lo);
    return {lo, min(hi - lo, max_new), hi - lo};
}

__global__ __launch_bounds__(TB) void tree_tables_kernel(const TreeTablesArgs a) {
    __shared__ uint32_t bits[N_MAX][WORDS + 1];
    __shared__ int up[N_MAX], depth[N_MAX];
    const int tid = threadIdx.x;
    auto none = [&](int t) {   // a row without a place in any tree
        a.positions[t] = 0;
        for (int w = 0; w < a.words; ++w) a.mask[(size_t)t * a.words + w] = 0;
    };
    if ((int)blockIdx.x >= a.n_requests) {   // rows behind the last request's
        const int64_t t = (int64_t)((int)blockIdx.x - a.n_requests) * TB + tid;
        const int end = a.n_requests > 0 ? max(min(a.q_offsets[a.n_requests], a.n_tokens), 0) : 0;
        if (t >= end && t < a.n_tokens) none((int)t);
        return;
    }
    const Rows r = rows_of(a.q_offsets, blockIdx.x, a.n_tokens, a.max_new);
    for (int i = r.n + tid; i < r.all; i += TB) none(r.first + i);
    uint32_t own[WORDS];
    int p = -1, d = 0;
    if (tid < r.n) {
        p = a.parents[r.first + tid];
        if (p < 0 || p >= tid) p = -1;
    }
#pragma unroll
    for (int w = 0; w < WORDS; ++w) bits[tid][w] = own[w] = tid >> 5 == w ? 1u << (tid & 31) : 0u;
    depth[tid] = d = p >= 0 ? 1 : 0;
    up[tid] = p;
    while (__syncthreads_or(p >= 0)) {
        uint32_t more[WORDS];
        int q = -1, e = 0;
        if (p >= 0) {
            q = up[p];
            e = depth[p];
#pragma unroll
            for (int w = 0; w < WORDS; ++w) more[w] = bits[p][w];
        }
        __syncthreads();
        if (p >= 0) {
#pragma unroll
            for (int w = 0; w < WORDS; ++w) bits[tid][w] = own[w] |= more[w];
            depth[tid] = d += e;
            up[tid] = p = q;
        }
    }
    if (tid >= r.n) return;
    const int64_t at = (int64_t)max(a.cached_len[blockIdx.x], 0) + d;
    a.positions[r.first + tid] = (int32_t)min(at, (int64_t)INT32_MAX);
    uint32_t* row = a.mask + (size_t)(r.first + tid) * a.words;
#pragma unroll
    for (int w = 0; w < WORDS; ++w)
        if (w < a.words) row[w] = own[w];
}

// A request's rows in a wave's registers.
constexpr int PER = N_MAX / 64;
struct WalkRows {
    Rows r;
    int given, parent[PER], token[PER], choice[PER];
};
__device__ __forceinline__ WalkRows walk_rows(const TreeKeepArgs& a, int b, int lane) {
    WalkRows w;
    w.r = rows_of(a.q_offsets, b, a.n_tokens, a.max_new);
    w.given = a.n_given != nullptr ? max(1, min(a.n_given[b], w.r.n)) : 1;
    if (w.r.n == 0) return w;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int i = 64 * k + lane, t = w.r.first + min(i, w.r.n - 1);
        w.parent[k] = i < w.r.n ? a.parents[t] : -1;
        w.token[k] = a.tokens[t];
        w.choice[k] = a.choice[t];
    }
    return w;
}
// The walk; put(i, row): the i-th row that stays (a lane's, or lane 0's).
struct Walked { int kept, next; };
template <typename Put>
__device__ __forceinline__ Walked walk(const WalkRows& w, int lane, Put put) {
    if (w.r.n == 0) return {0, -1};
    for (int i = lane; i < w.given; i += 64) put(i, i);
    int at = __builtin_amdgcn_readfirstlane(w.given - 1), kept = at + 1, after = 0;
    while (true) {
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (at >> 6 == k) after = __builtin_amdgcn_readlane(w.choice[k], at & 63);
        int next = -1;
#pragma unroll
        for (int k = PER - 1; k >= 0; --k) {
            const uint64_t hit = __ballot(w.parent[k] == at && w.token[k] == after && 64 * k + lane > at);
            if (hit != 0) next = 64 * k + __builtin_ctzll(hit);
        }
        if (next < 0) break;
        at = next;
        if (lane == 0) put(kept, at);
        ++kept;
    }
    return {kept, after};
}
// One wave per request.
__global__ __launch_bounds__(64) void tree_walk_kernel(const TreeKeepArgs a) {
    const int b = blockIdx.x, lane = threadIdx.x;
    const WalkRows w = walk_rows(a, b, lane);
    const Walked got = walk(w, lane, [&](int i, int row) { a.path[w.r.first + i] = row; });
    for (int i = got.kept + lane; i < w.r.all; i += 64) a.path[w.r.first + i] = -1;
    if (lane == 0) { a.kept_len[b] = got.kept; a.next_token[b] = got.next; }
}

// Pages of a request that the step's rows reached and the kept ones do not: blocks lo .. hi - 1.
struct Blocks { int lo, hi; };
__device__ __forceinline__ Blocks empty_blocks(const TreeKeepArgs& a, int b, int kept) {
    const Rows r = rows_of(a.q_offsets, b, a.n_tokens, a.max_new);
    const uint32_t c = (uint32_t)max(a.cached_len[b], 0), P = (uint32_t)a.page_rows, W = (uint32_t)a.max_blocks;
    const uint32_t stays = c + (uint32_t)kept, was = c + (uint32_t)r.all;   // (below 2^32: 2^31 - 1 + 2^30)
    return {(int)min(stays / P + (stays % P != 0), W), (int)min(was / P + (was % P != 0), W)};
}

// One workgroup: pages back to the free list, in the order of the requests and their positions.  ONE: in the launch that walks too; it walks all trees by itself.
constexpr int ONE_MAX = 16;   // requests of such a call, at most
template <bool ONE>
__device__ __forceinline__ void give_pages_back(const TreeKeepArgs& a) {
    __shared__ int wave_sum[TB / 64], kept[ONE_MAX];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if constexpr (ONE) {
        constexpr int EACH = ONE_MAX / (TB / 64);
        WalkRows w[EACH];   // (one trip to memory for all)
#pragma unroll
        for (int i = 0; i < EACH; ++i) w[i] = walk_rows(a, min(wave + TB / 64 * i, a.n_requests - 1), lane);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int n = walk(w[i], lane, [](int, int) {}).kept;
            if (lane == 0) kept[wave + TB / 64 * i] = n;
        }
        __syncthreads();
    }
    const int end = max(0, min(*a.free_end, a.n_free));
    Blocks blocks{0, 0};   // of request b0 + tid
    int mine = 0;          // pages of it that go back
    auto look = [&](int b0) {
        const int b = b0 + tid;
        blocks = b < a.n_requests ? empty_blocks(a, b, ONE ? kept[b] : a.kept_len[b]) : Blocks{0, 0};
        mine = 0;
        for (int j = blocks.lo; j < blocks.hi; ++j) mine += (uint32_t)a.block_table[(size_t)b * a.max_blocks + j] < (uint32_t)a.n_pages;
    };
    int total = 0;
    for (int b0 = 0; b0 < a.n_requests; b0 += TB) {
        look(b0);
        total += mine;
    }
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    if (lane == 0) wave_sum[wave] = total;
    __syncthreads();
    total = 0;
#pragma unroll
    for (int w = 0; w < TB / 64; ++w) total += wave_sum[w];
    const int start = max(0, end - total);
    __syncthreads();
    int64_t to = (int64_t)end - total;   // of the next page
    for (int b0 = 0; b0 < a.n_requests; b0 += TB) {
        if (a.n_requests > TB) look(b0);   // (else it stands from above)
        int s = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(s, d);
            if (lane >= d) s += v;
        }
        if (lane == 63) wave_sum[wave] = s;
        __syncthreads();
        int before = s - mine, all = 0;
#pragma unroll
        for (int w = 0; w < TB / 64; ++w) {
            if (w < wave) before += wave_sum[w];
            all += wave_sum[w];
        }
        int64_t at = to + before;
        for (int j = blocks.lo; j < blocks.hi; ++j) {
            const int p = a.block_table[(size_t)(b0 + tid) * a.max_blocks + j];
            if ((uint32_t)p >= (uint32_t)a.n_pages) continue;
            if (at >= 0) a.free_pages[at] = p;   // (below 0: a list that is shorter than what it has given)
            ++at;
        }
        to += all;
        __syncthreads();
    }
    if (tid == 0) *a.free_start = start;
}

// blockIdx.x = layer x requests + request; the last workgroup sees to the pages.  ONE: every workgroup walks its request's tree again, those of the first layer write down what stays.
template <bool ONE>
__global__ __launch_bounds__(TB) void tree_move_kernel(const TreeKeepArgs a) {
    if (blockIdx.x == gridDim.x - 1) {
        if (a.free_end != nullptr) give_pages_back<ONE>(a);
        return;
    }
    __shared__ int place[N_MAX], from[N_MAX], path[ONE ? N_MAX : 1];   // slots of the request's rows; of the rows that stay
    __shared__ int first_moved;
    __shared__ Walked walked;
    const int b = blockIdx.x % a.n_requests, layer = blockIdx.x / a.n_requests, tid = threadIdx.x;
    const Rows r = rows_of(a.q_offsets, b, a.n_tokens, a.max_new);
    if (tid < r.n && a.n_layers > 0) {
        const int64_t position = (int64_t)max(a.cached_len[b], 0) + tid, block = position / a.page_rows;
        const int page = block < a.max_blocks ? a.block_table[(size_t)b * a.max_blocks + block] : -1;
        place[tid] = (uint32_t)page < (uint32_t)a.n_pages ? (int)(page * (int64_t)a.page_rows + position % a.page_rows) : -1;
    }
    if constexpr (ONE) {
        if (tid < 64) {
            const Walked got = walk(walk_rows(a, b, tid), tid, [&](int i, int row) { path[i] = row; });
            if (tid == 0) walked = got;
        }
        __syncthreads();
        if (layer == 0) {
            for (int i = tid; i < r.all; i += TB) a.path[r.first + i] = i < walked.kept ? path[i] : -1;
            if (tid == 0) { a.kept_len[b] = walked.kept; a.next_token[b] = walked.next; }
            if (a.n_layers == 0) return;
        }
    }
    const int kept = ONE ? walked.kept : a.kept_len[b];
    if (tid == 0) first_moved = kept;
    __syncthreads();
    if (tid < kept) {
        const int row = ONE ? path[tid] : a.path[r.first + tid];
        if (row != tid) atomicMin(&first_moved, tid);   // (rows stay in place up to the first that does not)
        from[tid] = place[row];
    }
    __syncthreads();
    u32x4 *k = (u32x4*)a.k_pages[layer], *v = (u32x4*)a.v_pages[layer];
    const int rv = a.row_vectors;
    constexpr int AHEAD = 4;   // rows in flight
    for (int e = tid; e < 2 * rv; e += TB) {
        u32x4* p = e < rv ? k + e : v + (e - rv);
        for (int i0 = first_moved; i0 < kept; i0 += AHEAD) {
            u32x4 x[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i < kept && from[i0 + i] >= 0) x[i] = p[(size_t)from[i0 + i] * rv];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i < kept && from[i0 + i] >= 0 && place[i0 + i] >= 0) p[(size_t)place[i0 + i] * rv] = x[i];
        }
    }
}

}  // namespace

hipError_t launch_tree_tables(const TreeTablesArgs& a, hipStream_t st) {
    const int64_t blocks = a.n_requests + ((int64_t)a.n_tokens + TB - 1) / TB;
    if (a.n_tokens == 0) return hipSuccess;
    tree_tables_kernel<<<dim3((unsigned)blocks), dim3(TB), 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_tree_keep(const TreeKeepArgs& a, hipStream_t st) {
    // One launch where few trees are to be walked for the pages: a workgroup's waves walk 4 of 16 each.
    if (a.n_requests > 0 && a.n_requests <= ONE_MAX) {
        tree_move_kernel<true><<<dim3((unsigned)(a.n_requests * std::max(a.n_layers, 1) + 1)), dim3(TB), 0, st>>>(a);
        return hipGetLastError();
    }
    if (a.n_requests > 0) tree_walk_kernel<<<dim3((unsigned)a.n_requests), dim3(64), 0, st>>>(a);
    if (a.n_layers > 0 || a.free_end != nullptr)
        tree_move_kernel<false><<<dim3((unsigned)((int64_t)a.n_requests * a.n_layers + 1)), dim3(TB), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace fr
