// What the attention kernels over a paged cache share: their arguments, how the work of a launch is dealt out, and how pieces of an item are joined.
#pragma once

#include "fr_internal.hpp"

namespace fr {

// Arguments of the kernels.  A launch takes the requests with cols_lo < rows x G <= cols_hi query columns.
// route: whether requests with more than `few` columns go through the tiled kernel is for the kernels to find out (paged_route); if they do, those with fewer go with
// them where `together` says so.
struct PagedArgs {
    const void* q;
    const int32_t *q_offsets, *cached_len, *block_table;
    const void *k_pages, *v_pages;
    void* out;
    float* lse;
    float* partials;
    int B, T, max_new, n_pages, P, W, cap;   // cap = W P: positions that the table has room for
    int Hq, Hkv, G, cols_lo, cols_hi;
    int route, few, together;
    int n_wg;                // workgroups per KV head that the work is dealt to
    uint32_t g_magic;        // ceil(2^32 / G): c / G = mulhi(c, g_magic) for c < 2^26
    uint32_t p_magic, p_shift;   // j / P = mulhi(2 j, p_magic) >> p_shift for j < 2^30
    float scale_log2e;
};

// A request as a launch sees it.
struct PagedRequest {
    int first, n;     // its first row and how many count
    int cached;
};
__device__ __forceinline__ PagedRequest paged_request(const PagedArgs& a, int b) {
    const int lo = max(min(a.q_offsets[b], a.T), 0), hi = max(min(a.q_offsets[b + 1], a.T), lo);
    PagedRequest r;
    r.first = lo;
    r.n = min(hi - lo, a.max_new);
    r.cached = a.cached_len[b];
    const int64_t cols = (int64_t)r.n * a.G;
    if (cols <= a.cols_lo || (a.cols_hi < INT32_MAX && cols > a.cols_hi)) r.n = 0;
    return r;
}
__device__ __forceinline__ int paged_position(const PagedArgs& a, const PagedRequest& r, int i) {   // of its row i; -1: sees nothing
    return (int)max((int64_t)-1, min((int64_t)r.cached + i, (int64_t)a.cap - 1));
}
__device__ __forceinline__ int paged_token(const PagedArgs& a, int col) { return a.G > 1 ? (int)__umulhi((uint32_t)col, a.g_magic) : col; }
__device__ __forceinline__ int paged_block(const PagedArgs& a, int j) { return (int)(__umulhi(2u * (uint32_t)j, a.p_magic) >> a.p_shift); }

// Over the first n lanes of the wave (lanes 0 .. n - 1 hold the result; the others hold nothing of use): a batch of few requests takes few steps.
__device__ __forceinline__ int64_t wave_sum64(int64_t v, int n) {
    for (int d = 1; d < n; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ int64_t wave_scan64(int64_t v, int n) {   // inclusive
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < n; d <<= 1) {
        const int64_t t = __shfl_up(v, d);
        if (lane >= d) v += t;
    }
    return v;
}
__device__ __forceinline__ int64_t uniform64(int64_t v) {
    const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
    return (int64_t)(((uint64_t)hi << 32) | lo);
}

// blockIdx.x = workgroup of the KV head x Hkv + KV head: blocks go to the eight dies in turn, so that with 8 KV heads each die's cache serves one of them.
__device__ __forceinline__ int paged_head(const PagedArgs& a) { return blockIdx.x % a.Hkv; }
__device__ __forceinline__ int paged_workgroup(const PagedArgs& a) { return blockIdx.x / a.Hkv; }
inline unsigned paged_grid(int64_t workgroups, int Hkv) { return (unsigned)(workgroups * Hkv); }

// Do the requests with many columns go through the tiled kernel?  It takes 34 us for the shortest call and 1.5 us for 256 columns x 64 keys on a
// compute unit, the streaming kernel 11 us and twice the time per column, and it reads the keys again for every 32 columns, from the die's cache as
// long as they fit about twice.  us tiled : streaming, rows behind positions (columns x keys of all KV heads); 32 / 8 heads: 128 behind 1000 (5 M) 58 : 23, 512 behind 4000 (74 M) 103 : 68,
// 512 behind 14336 (243 M) 167 : 196, 1024 from nothing (34 M) 63 : 42, 2048 (134 M) 90 : 112; 64 / 8 heads: 512 behind 4000 (148 M) 128 : 126, 128 behind 14336 (118 M) 98 : 110;
// sixteen times 40 behind 3000: 32 / 8 heads (62 M, 25 MB per KV head) 107 : 168, head_dim 64 (31 M, 12 MB) 59 : 41.
// Few keys make short items, which the tiled kernel takes whole, one for a workgroup: 30 us and 1.5 for 64 of its keys.  From nothing, 64 / 8 heads, 768 rows (38 M) 56 : 47, 900 (52 M) 59 : 72, 1024 (67 M)
// 63 : 70, 1200 (92 M) 84 : 105; 600 behind 500 (42 M) 64 : 64, 512 behind 1000 (50 M) 70 : 51; 28 / 4 heads, 1200 (40 M) 65 : 57, 1500 (63 M) 73 : 75.
constexpr int64_t PAGED_PAIRS_NEAR = 100000000, PAGED_PAIRS_FAR = 35000000;   // columns x keys; the keys of a KV head in PAGED_NEAR_BYTES, or more
constexpr int64_t PAGED_PAIRS_SHORT = 24000000, PAGED_PAIRS_KEY = 29000;   // and near keys that are few: this, and this for each of them
constexpr int64_t PAGED_NEAR_BYTES = 8 << 20;
__device__ __forceinline__ bool paged_route(const PagedArgs& a, int row_bytes) {
    const int lane = threadIdx.x & 63;
    int64_t pairs = 0, keys = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        int64_t p = 0, k = 0;
        if (b0 + lane < a.B) {
            const int b = b0 + lane, lo = max(min(a.q_offsets[b], a.T), 0), hi = max(min(a.q_offsets[b + 1], a.T), lo);
            const int64_t cols = (int64_t)min(hi - lo, a.max_new) * a.G;
            if (cols > a.few) {
                k = max((int64_t)0, min((int64_t)a.cached_len[b] + (hi - lo), (int64_t)a.cap));
                p = cols * k >> 10;   // (in thousands: no sum passes 64 bits)
            }
        }
        pairs += uniform64(wave_sum64(p, min(64, a.B - b0)));
        keys += uniform64(wave_sum64(k, min(64, a.B - b0)));
    }
    return pairs * a.Hkv > (keys * row_bytes <= PAGED_NEAR_BYTES ? min(PAGED_PAIRS_NEAR, PAGED_PAIRS_SHORT + PAGED_PAIRS_KEY * keys) : PAGED_PAIRS_FAR) >> 10;
}

// How a launch's work is dealt out.  The work of a KV head is one line of units: requests in order, of each its column tiles, of each its units of keys.
// Workgroup w of n takes units floor(w U / n) .. floor((w + 1) U / n) - 1 of it, wherever they begin and end, so every workgroup has the same
// share whatever the lengths are, and the host need not know them.  n is at most U (paged_sharers): none of them goes without.  An item (column tile) that falls to several
// workgroups leaves a partial result per piece: in slot 2 w of a workgroup whose piece begins behind the item's start, in 2 w + 1 of the one that has its start but not its
// end.  The one with the start also leaves a PagedCut, which is all that the joining pass has to read to find its work.  A query column is read by the workgroups of its item
// alone, and its output is stored when they have read it: out may be q.
struct alignas(16) PagedCut {   // of a workgroup and KV head; in front of the partial results
    int pieces;      // of the item that it has the start but not the end of: its own and those of the workgroups behind it; 0: there is no such item
    int first_row;   // of the request
    int col0, cols;  // the item's first query column, and how many the request has
};
__device__ __forceinline__ PagedCut* paged_cuts(const PagedArgs& a) { return reinterpret_cast<PagedCut*>(a.partials); }
__device__ __forceinline__ float* paged_slot(const PagedArgs& a, int w, int g, int which, int floats) {
    return a.partials + (size_t)a.n_wg * a.Hkv * (sizeof(PagedCut) / 4) + (((size_t)w * a.Hkv + g) * 2 + which) * floats;
}
struct PagedLine {
    int64_t total;    // U
    int64_t start;    // of the unit that was looked for: first unit of its request
    int b;            // and the request
};
// cost(b) = units of request b (0: none).  Every wave does this by itself.  find(total) = the unit to look for, or -1.
template <typename Cost, typename Find>
__device__ __forceinline__ PagedLine paged_line(int B, Cost cost, Find find) {
    const int lane = threadIdx.x & 63;
    PagedLine r{0, 0, -1};
    int64_t mine = 0;
    for (int b0 = 0; b0 < B; b0 += 64) {
        mine = b0 + lane < B ? cost(b0 + lane) : 0;
        r.total += uniform64(wave_sum64(mine, min(64, B - b0)));
    }
    const int64_t u = find(r.total);
    if (u < 0 || u >= r.total) return r;
    for (int b0 = 0; b0 < B; b0 += 64) {
        if (B > 64) mine = b0 + lane < B ? cost(b0 + lane) : 0;
        const int64_t upto = r.start + wave_scan64(mine, min(64, B - b0));
        const uint64_t beyond = __ballot(upto > u);
        if (beyond != 0) {
            const int l = __builtin_ctzll(beyond);
            r.b = b0 + l;
            const int64_t end = uniform64(__shfl(upto, l)), own = uniform64(__shfl(mine, l));
            r.start = end - own;
            return r;
        }
        r.start = uniform64(__shfl(upto, 63));
    }
    return r;
}
__device__ __forceinline__ int paged_sharers(const PagedArgs& a, int64_t total) { return (int)min((int64_t)a.n_wg, total); }
// floor(x / d), x >= 0, d > 0: by a product in fp64 and a step or two (a division of 64-bit integers is over a hundred instructions; eight of them were 4 us in front of
// a piece's first load).
__device__ __forceinline__ int64_t paged_div(int64_t x, int64_t d) {
    int64_t q = (int64_t)((double)x * (1.0 / (double)d));
    while (q * d > x) --q;
    while ((q + 1) * d <= x) ++q;
    return q;
}
__device__ __forceinline__ int64_t paged_first_unit(int64_t w, int64_t total, int n) { return paged_div(w * total, n); }
__device__ __forceinline__ int paged_owner(int64_t u, int64_t total, int n) { return (int)paged_div((u + 1) * n - 1, total); }   // the workgroup that has unit u

// ---- matrix-core helpers ------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
constexpr float PAGED_NO_MAX = -3.402823466e38f;   // exponent reference of a column that has seen nothing: below every finite logit times the scale (0.18 at most)
constexpr float PAGED_RAISE = 8.f;         // a column's reference goes up when a logit is this far (base 2) above it: weights stay below 2^8
// References of this size (base 2) and more: the reference is a rounded product (logit x scale), and a multiply-add that subtracts it sees the product before its rounding, up to half a
// step of the reference away, which is a factor of 2 in the weights at 2^24, and from 2^31 on infinity, or 0 for the largest logit itself.  There the products are rounded first.
constexpr float PAGED_FAR = 16777216.f;

// Sum and maximum over the four lanes that hold the same column (lanes x, x + 16, x + 32, x + 48).
__device__ __forceinline__ float paged_column_sum(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float paged_column_max(float v) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Is what a word holds (two bf16 numbers, or one of fp32) not finite, and the word with 0 in the place of such a number.
template <typename T>
__device__ __forceinline__ bool paged_not_finite(uint32_t w) { return (sizeof(T) == 2 && (w & 0x00007F80u) == 0x00007F80u) || (w & 0x7F800000u) == 0x7F800000u; }
template <typename T>
__device__ __forceinline__ uint32_t paged_finite_or_zero(uint32_t w) {
    if (sizeof(T) == 2 && (w & 0x00007F80u) == 0x00007F80u) w &= 0xFFFF0000u;
    if ((w & 0x7F800000u) == 0x7F800000u) w &= sizeof(T) == 2 ? 0x0000FFFFu : 0u;
    return w;
}

// ---- copies global -> LDS without registers; completion: the issuing wave's vmcnt, in order of issue ------
__device__ __forceinline__ uint32_t paged_lds(const void* p) {
    return __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) const unsigned char*)p);
}
__device__ __forceinline__ void paged_copy16(const void* src, uint32_t lds) {   // lane i's 16 bytes to lds + 16 i
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
__device__ __forceinline__ void paged_copy4(const void* src, uint32_t lds) {    // lane i's 4 bytes to lds + 4 i
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" : : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
// The same from a base that the wave shares.
__device__ __forceinline__ void paged_copy16(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
__device__ __forceinline__ void paged_copy4(const void* base, uint32_t off, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(off), "s"(base), "s"(__builtin_amdgcn_readfirstlane(lds)) : "memory");
}
__device__ __forceinline__ const unsigned char* paged_uniform(const unsigned char* p) {   // in scalar registers, whatever the compiler makes of it
    return reinterpret_cast<const unsigned char*>((uintptr_t)uniform64((int64_t)(uintptr_t)p));
}
template <int N>
__device__ __forceinline__ void paged_wait_but() {   // until all but the wave's last N copies have landed
    static_assert(N < 64, "the counter's six bits, in two fields");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | N >> 4 << 14);
    asm volatile("" ::: "memory");
}

size_t paged_stream_partials_bytes(const Shape& s, int n_cu);
hipError_t launch_paged_stream(const Shape& s, const PagedArgs& a, int n_cu, hipStream_t st);

size_t paged_tile_partials_bytes(const Shape& s, int n_cu);
hipError_t launch_paged_tile(const Shape& s, const PagedArgs& a, int n_cu, hipStream_t st);

__device__ __forceinline__ void paged_lds_barrier() {   // a workgroup's barrier for LDS alone: __syncthreads() also waits for stores to memory
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// ---- joining pieces -----------------------------------------------------------------------------------
// A piece's slot: [column][D + 2] fp32: exponent reference (base 2), sum of weights, weighted values.
template <int D>
constexpr int paged_part_floats() { return D + 2; }

}  // namespace fr
