// What a serving step does to a paged cache around its attention: tables from the requests' lengths, and the new rows into their pages.
//
// Tables.  off[b] = min(T, sum of new_len below b); request b takes its pages first_b = ceil(c_b / P) .. last_b - 1, last_b = ceil((c_b + n_b) / P),
// n_b = off[b + 1] - off[b], from the free list behind those of the requests before it; row t of request b is position c_b + t - off[b].  A launch
// of one kernel is all there is to it: every workgroup scans the lengths of all requests itself (32 KB at most, in the caches) rather than
// wait for a pass that does, then every thread finds the request of its row, and of its page, by bisection in LDS.  The pages of a row are looked up
// in the free list, not in the table that other threads are writing.  Latency: 4.4 us for 64 requests of a row each, 5.3 for 256 that bring 13 668; a launch of nothing is 4.
//
// Append.  One wave per row: its lanes form the row's (cos, sin) pairs in fp64, rounded once, while the row's vectors are on their way, and then take
// vectors v and v + NV / 2 of a head together, which are a pair's two halves in the half-split layout, so that q may be rotated in place.
// Streaming: bound by memory for long prompts, by the chain positions -> angle -> store for a decoding step.
// 16896 rows of 32 / 8 heads 79 us = 5.25 TB/s read and written (a device copy of 1 GiB 5.09); 64 rows 3.8 us, 2640 rows of 16 / 8 heads of 64 5.7.
#include "k_rotate.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr int TB = 256;            // threads of the tables kernel
constexpr int PER = 4;             // requests per thread and round of its scans

struct TablesLds {
    uint32_t off[FR_PAGED_MAX_REQUESTS + 1];    // first row of each request
    uint32_t page[FR_PAGED_MAX_REQUESTS + 1];   // pages taken by the requests before it
    uint32_t wave_sum[TB / 64];
};

// Exclusive sum over the workgroup's threads, sums capped at `most` (no 32-bit overflow: most < 2^31); `total` = the sum of all.
__device__ __forceinline__ uint32_t scan_exclusive(uint32_t v, uint32_t most, uint32_t* wave_sum, uint32_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t s = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t t = __shfl_up(s, d);
        if (lane >= d) s = min(most, s + t);
    }
    if (lane == 63) wave_sum[wave] = s;
    uint32_t before = __shfl_up(s, 1);
    if (lane == 0) before = 0;
    __syncthreads();
    uint32_t all = 0, mine = 0;
#pragma unroll
    for (int w = 0; w < TB / 64; ++w) {
        if (w == wave) mine = all;
        all = min(most, all + wave_sum[w]);
    }
    __syncthreads();   // (wave_sum is free again)
    *total = all;
    return min(most, mine + before);
}

// The last b of 0 .. n - 1 with first[b] <= i; first ascends, first[0] = 0.
__device__ __forceinline__ int request_of(const uint32_t* first, int n, uint32_t i) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= i) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__global__ __launch_bounds__(TB) void page_tables_kernel(const PageTablesArgs a) {
    __shared__ TablesLds sm;
    const uint32_t T = (uint32_t)a.n_tokens, P = (uint32_t)a.page_rows, W = (uint32_t)a.max_blocks;
    const int B = a.n_requests, tid = threadIdx.x;
    const int64_t start = a.free_start != nullptr ? (int64_t)*a.free_start : 0;
    uint32_t rows = 0, pages = 0;
    for (int b0 = 0; b0 < B; b0 += TB * PER) {
        uint32_t n[PER], c[PER], s = 0, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = b0 + PER * tid + i;
            n[i] = b < B ? min((uint32_t)max(a.new_len[b], 0), T) : 0u;
            c[i] = b < B ? (uint32_t)max(a.cached_len[b], 0) : 0u;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) s = min(T, s + n[i]);
        uint32_t at = min(T, rows + scan_exclusive(s, T, sm.wave_sum, &total));
        rows = min(T, rows + total);
        uint32_t taken[PER], p = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = b0 + PER * tid + i;
            const uint32_t end = min(T, at + n[i]);
            if (b < B) sm.off[b] = at;
            // (c + n < 2^32: 2^31 - 1 + 2^30)
            const uint32_t first = c[i] / P + (c[i] % P != 0), seen = c[i] + (end - at), last = seen / P + (seen % P != 0);
            taken[i] = b < B && end > at ? min(last, W) - min(first, W) : 0u;
            p += taken[i];
            at = end;
        }
        uint32_t q = pages + scan_exclusive(p, 0x7FFFFFFFu, sm.wave_sum, &total);
        pages += total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int b = b0 + PER * tid + i;
            if (b < B) sm.page[b] = q;
            q += taken[i];
        }
    }
    if (tid == 0) { sm.off[B] = rows; sm.page[B] = pages; }
    __syncthreads();
    const int64_t i = (int64_t)blockIdx.x * TB + tid;
    if (i == 0 && a.pages_needed != nullptr) *a.pages_needed = (int32_t)pages;
    if (i <= B) a.q_offsets[i] = (int32_t)sm.off[i];
    auto free_page = [&](int64_t k) {   // the k-th page of this call
        const int64_t at = start + k;
        return at >= 0 && at < a.n_free ? a.free_pages[at] : -1;
    };
    if (i < pages) {
        const int b = request_of(sm.page, B, (uint32_t)i);
        const uint32_t c = (uint32_t)max(a.cached_len[b], 0);
        const uint32_t j = c / P + (c % P != 0) + ((uint32_t)i - sm.page[b]);
        a.block_table[(size_t)b * W + j] = free_page(i);
    }
    if (i < T) {
        int32_t position = 0, slot = -1;
        if (i < rows) {
            const int b = request_of(sm.off, B, (uint32_t)i);
            const uint32_t c = (uint32_t)max(a.cached_len[b], 0), at = c + ((uint32_t)i - sm.off[b]), block = at / P;
            const uint32_t first = c / P + (c % P != 0);
            position = (int32_t)at;
            if (block < W) {
                const int32_t page = block < first ? a.block_table[(size_t)b * W + block] : free_page((int64_t)sm.page[b] + (block - first));
                const int64_t row = (int64_t)page * P + at % P;
                if (page >= 0 && row <= INT32_MAX) slot = (int32_t)row;
            }
        }
        a.positions[i] = position;
        a.slots[i] = slot;
    }
}

// grid: blockDim / 64 rows per workgroup, one per wave.
template <typename T, int D, int LAYOUT>
__global__ __launch_bounds__(256) void paged_append_kernel(const PagedAppendArgs a) {
    constexpr int N = 16 / sizeof(T), NV = D / N, HV = NV / 2;   // elements of a vector, vectors of a head, pairs of them
    constexpr int HEADS = 64 / HV;                               // heads that a wave takes at once
    constexpr int AHEAD = 6;
    __shared__ float2 rot[4][D / 2];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int t = blockIdx.x * (blockDim.x >> 6) + wave;
    if (t >= a.n_tokens) return;
    const int v = lane % HV, h0 = lane / HV, skip = a.q != nullptr ? 0 : a.Hq;
    const int n_heads = a.Hq + 2 * a.Hkv - skip;
    const int64_t slot = a.slots[t];
    const bool in_cache = slot >= 0 && slot < a.n_rows;
    const T *q = (const T*)a.q, *k = (const T*)a.k, *val = (const T*)a.v;
    auto source = [&](int h) -> const T* {   // head h of the row: query heads, key heads, value heads
        if (h < a.Hq) return q + ((size_t)t * a.Hq + h) * D;
        if (h < a.Hq + a.Hkv) return k + ((size_t)t * a.Hkv + (h - a.Hq)) * D;
        return val + ((size_t)t * a.Hkv + (h - a.Hq - a.Hkv)) * D;
    };
    rot_u32x4 x[AHEAD][2];
    auto load = [&](int i0) {   // past the end: the last head, not stored (a branch would wait for each load)
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const T* s = source(skip + min(i0 + h0 + HEADS * u, n_heads - 1));
            x[u][0] = *reinterpret_cast<const rot_u32x4*>(s + N * v);
            x[u][1] = *reinterpret_cast<const rot_u32x4*>(s + N * (v + HV));
        }
    };
    load(0);
    const bool rotate = a.positions != nullptr;
    float2 lo[N], hi[N];   // rotations of the lane's two vectors (interleaved: N / 2 each)
    if (rotate) {
        const int p = lane & (D / 2 - 1);
        rot[wave][p] = chunk_rotation(a.positions[t], a.theta[p]);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");   // the wave's writes precede its reads
        __builtin_amdgcn_wave_barrier();
        constexpr int M = LAYOUT == FR_ROPE_INTERLEAVED ? N / 2 : N;
#pragma unroll
        for (int e = 0; e < M; ++e) {
            lo[e] = rot[wave][M * v + e];
            if (LAYOUT == FR_ROPE_INTERLEAVED) hi[e] = rot[wave][M * (v + HV) + e];
        }
    }
    for (int i0 = 0; i0 < n_heads; i0 += AHEAD * HEADS) {
        if (i0 > 0) load(i0);
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int i = i0 + h0 + HEADS * u, h = skip + i;
            if (i >= n_heads) continue;
            rot_u32x4 y0 = x[u][0], y1 = x[u][1];
            if (rotate && h < a.Hq + a.Hkv) {
                y0 = rotate_vector<T, LAYOUT>(x[u][0], x[u][1], lo, true);
                y1 = rotate_vector<T, LAYOUT>(x[u][1], x[u][0], LAYOUT == FR_ROPE_INTERLEAVED ? hi : lo, false);
            }
            T* dst;
            if (h < a.Hq) {
                dst = (T*)a.q_out + ((size_t)t * a.Hq + h) * D;
            } else {
                if (!in_cache) continue;
                const bool key = h < a.Hq + a.Hkv;
                dst = (T*)(key ? a.k_pages : a.v_pages) + ((size_t)slot * a.Hkv + (h - a.Hq - (key ? 0 : a.Hkv))) * D;
            }
            *reinterpret_cast<rot_u32x4*>(dst + N * v) = y0;
            *reinterpret_cast<rot_u32x4*>(dst + N * (v + HV)) = y1;
        }
    }
}

template <typename T, int D>
hipError_t append(const Shape& s, const PagedAppendArgs& a, int n_cu, hipStream_t st) {
    // One row per workgroup while that leaves at most two per compute unit, else four.
    const int rows = a.n_tokens <= 2 * n_cu ? 1 : 4;
    const dim3 grid((unsigned)((a.n_tokens + rows - 1) / rows)), block(64 * rows);
    if (s.rope_layout == FR_ROPE_INTERLEAVED)
        paged_append_kernel<T, D, FR_ROPE_INTERLEAVED><<<grid, block, 0, st>>>(a);
    else
        paged_append_kernel<T, D, FR_ROPE_HALF><<<grid, block, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_page_tables(const PageTablesArgs& a, hipStream_t st) {
    // a thread per row, per page that may be taken (every request ends at most one that is not full), per request and one more
    const int64_t items = std::max<int64_t>(a.n_tokens, (int64_t)a.n_tokens / a.page_rows + a.n_requests) + 1;
    page_tables_kernel<<<dim3((unsigned)((items + TB - 1) / TB)), dim3(TB), 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_paged_append(const Shape& s, const PagedAppendArgs& a, int n_cu, hipStream_t st) {
    if (a.n_tokens == 0) return hipSuccess;
    if (s.dtype == FR_BF16) return s.d == 128 ? append<__bf16, 128>(s, a, n_cu, st) : append<__bf16, 64>(s, a, n_cu, st);
    return s.d == 128 ? append<float, 128>(s, a, n_cu, st) : append<float, 64>(s, a, n_cu, st);
}

}  // namespace fr
