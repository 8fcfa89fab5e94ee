// Attention of chunks of new tokens over a paged cache.  Row i of request b is the token at position p = cached_len[b] + i and sees the
// keys at positions 0 .. p, key j in row j % P of page block_table[b][j / P].
//
// One workgroup per (row, KV head), four query heads at a time: a group of lanes per key row, 16 bytes each, an online softmax per lane group,
// merged through LDS at the end.
#include "k_paged.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr float NEG_BIG = -1.0e30f;
constexpr int GC = 4;

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_rows_kernel(const PagedArgs a) {
    constexpr int N = 16 / sizeof(T), LPK = D / N, KPW = 64 / LPK;
    __shared__ float mo[4][GC][D], mm[4][GC], ml[4][GC];
    const int t = blockIdx.x, g = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane % LPK, r = lane / LPK;
    int b = -1, first = 0;
    for (int i = 0; i < a.B; ++i) {
        const PagedRequest r = paged_request(a, i);
        if (t >= r.first && t < r.first + r.n) { b = i; first = r.first; break; }
    }
    if (b < 0) return;
    const int seen = paged_position(a, paged_request(a, b), t - first) + 1;   // keys 0 .. seen - 1
    for (int h0 = 0; h0 < a.G; h0 += GC) {
        float q[GC][N], o[GC][N], m[GC], l[GC];
#pragma unroll
        for (int i = 0; i < GC; ++i) {
            const T* p = (const T*)a.q + ((size_t)t * a.Hq + g * a.G + min(h0 + i, a.G - 1)) * D + c * N;
            m[i] = NEG_BIG; l[i] = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) { q[i][e] = Elem<T>::to_f32(p[e]); o[i][e] = 0.f; }
        }
        for (int j0 = 0; j0 < seen; j0 += 4 * KPW) {
            const int j = j0 + wave * KPW + r;
            const int page = j < seen ? a.block_table[(size_t)b * a.W + paged_block(a, j)] : -1;
            const bool ok = page >= 0 && page < a.n_pages;
            const size_t at = ok ? (((size_t)page * a.P + (j - paged_block(a, j) * a.P)) * a.Hkv + g) * D + c * N : 0;
            float kf[N], vf[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                kf[e] = ok ? Elem<T>::to_f32(((const T*)a.k_pages)[at + e]) : 0.f;
                vf[e] = ok ? Elem<T>::to_f32(((const T*)a.v_pages)[at + e]) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < GC; ++i) {
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) s = __builtin_fmaf(q[i][e], kf[e], s);
                for (int d = 1; d < LPK; d <<= 1) s += __shfl_xor(s, d);
                s = ok ? s * a.scale_log2e : -INFINITY;
                const float mn = fmaxf(m[i], s), alpha = __builtin_amdgcn_exp2f(m[i] - mn), p = __builtin_amdgcn_exp2f(s - mn);
                m[i] = mn;
                l[i] = l[i] * alpha + p;
#pragma unroll
                for (int e = 0; e < N; ++e) o[i][e] = __builtin_fmaf(p, vf[e], o[i][e] * alpha);
            }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < GC; ++i) {
            float mt = m[i];
            for (int d = LPK; d < 64; d <<= 1) mt = fmaxf(mt, __shfl_xor(mt, d));
            const float f = __builtin_amdgcn_exp2f(m[i] - mt);
            float lt = l[i] * f;
            for (int d = LPK; d < 64; d <<= 1) lt += __shfl_xor(lt, d);
            if (lane == 0) { mm[wave][i] = mt; ml[wave][i] = lt; }
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float x = o[i][e] * f;
                for (int d = LPK; d < 64; d <<= 1) x += __shfl_xor(x, d);
                if (r == 0) mo[wave][i][c * N + e] = x;
            }
        }
        __syncthreads();
        for (int idx = tid; idx < GC * D; idx += 256) {
            const int i = idx / D, e = idx % D;
            if (h0 + i >= a.G) continue;
            float mt = NEG_BIG, lt = 0.f, x = 0.f;
            for (int w = 0; w < 4; ++w) mt = fmaxf(mt, mm[w][i]);
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(mm[w][i] - mt);
                lt += ml[w][i] * f;
                x += mo[w][i][e] * f;
            }
            const size_t row = (size_t)t * a.Hq + g * a.G + h0 + i;
            ((T*)a.out)[row * D + e] = Elem<T>::from_f32(lt > 0.f ? x / lt : 0.f);
            if (e == 0 && a.lse != nullptr) a.lse[row] = lt > 0.f ? (mt + __builtin_amdgcn_logf(lt)) * 0.6931471805599453f : -INFINITY;
        }
    }
}

template <typename T, int D>
hipError_t launch_rows(const PagedArgs& a, hipStream_t st) {
    paged_rows_kernel<T, D><<<dim3((unsigned)a.T, (unsigned)a.Hkv), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(const Shape& s, const PagedAttnArgs& args, float* partials, int n_cu, hipStream_t st) {
    if (args.n_tokens == 0 || args.n_requests == 0 || args.max_new == 0) return hipSuccess;
    PagedArgs a{};
    a.q = args.q; a.q_offsets = args.q_offsets; a.cached_len = args.cached_len; a.block_table = args.block_table;
    a.k_pages = args.k_pages; a.v_pages = args.v_pages; a.out = args.out; a.lse = args.lse; a.partials = partials;
    a.B = args.n_requests; a.T = args.n_tokens; a.max_new = args.max_new;
    a.n_pages = args.n_pages; a.P = args.page_rows; a.W = args.max_blocks;
    a.cap = args.n_pages > 0 ? args.max_blocks * args.page_rows : 0;   // (a cache without pages shows nothing)
    a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
    a.g_magic = (uint32_t)((((uint64_t)1 << 32) + s.G - 1) / s.G);
    while (((int64_t)1 << a.p_shift) < a.P) ++a.p_shift;
    a.p_magic = (uint32_t)(2 * ((((uint64_t)1 << (30 + a.p_shift)) + a.P - 1) / a.P));
    a.scale_log2e = (1.0f / sqrtf((float)s.d)) * 1.4426950408889634f;
    if (s.dtype != FR_BF16) {
        a.cols_hi = INT32_MAX;
        return s.d == 128 ? launch_rows<float, 128>(a, st) : launch_rows<float, 64>(a, st);
    }
    // requests with few columns, and the others (a few of the former beside others: with them, two launches less)
    const int few = std::max(64, s.G);
    const bool others = (int64_t)args.max_new * s.G > few;
    a.cols_lo = 0;
    a.cols_hi = few;
    if (!others || args.n_requests > 8) {
        hipError_t e = launch_paged_stream(s, a, n_cu, st);
        if (e != hipSuccess || !others) return e;
        a.cols_lo = few;
    }
    a.cols_hi = INT32_MAX;
    return launch_paged_tile(s, a, n_cu, st);
}

size_t paged_attn_partials_bytes(const Shape& s, int n_cu) { return s.dtype == FR_BF16 ? std::max(paged_stream_partials_bytes(s, n_cu), paged_tile_partials_bytes(s, n_cu)) : 0; }

}  // namespace fr
