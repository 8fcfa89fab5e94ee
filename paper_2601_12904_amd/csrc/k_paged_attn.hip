// Attention of chunks of new tokens over a paged cache.  Row i of request b is the token at position p = cached_len[b] + i and sees the
// keys at positions 0 .. p, key j in row j % P of page block_table[b][j / P].
//
// One workgroup per (row, KV head), four query heads at a time: a group of lanes per key row, 16 bytes each, an online softmax per lane group,
// merged through LDS at the end.
#include "fr_internal.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr float NEG_BIG = -1.0e30f;
constexpr int GC = 4;

template <typename T, int D>
__global__ __launch_bounds__(256) void paged_rows_kernel(const PagedAttnArgs a) {
    constexpr int N = 16 / sizeof(T), LPK = D / N, KPW = 64 / LPK;
    __shared__ float mo[4][GC][D], mm[4][GC], ml[4][GC];
    const int t = blockIdx.x, g = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, c = lane % LPK, r = lane / LPK;
    int b = -1, first = 0;
    for (int i = 0; i < a.n_requests; ++i) {
        const int lo = max(a.q_offsets[i], 0), hi = min(a.q_offsets[i + 1], a.n_tokens);
        if (t >= lo && t < hi) { b = i; first = lo; break; }
    }
    if (b < 0 || t - first >= a.max_new) return;
    const int64_t cap = (int64_t)a.max_blocks * a.page_rows;
    const int seen = (int)min((int64_t)a.cached_len[b] + (t - first) + 1, cap);   // keys 0 .. seen - 1
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
            const int page = j < seen ? a.block_table[(size_t)b * a.max_blocks + j / a.page_rows] : -1;
            const bool ok = page >= 0 && page < a.n_pages;
            const size_t at = ok ? (((size_t)page * a.page_rows + j % a.page_rows) * a.Hkv + g) * D + c * N : 0;
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
hipError_t launch(const PagedAttnArgs& a, hipStream_t st) {
    paged_rows_kernel<T, D><<<dim3((unsigned)a.n_tokens, (unsigned)a.Hkv), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(const Shape& s, const PagedAttnArgs& args, hipStream_t st) {
    if (args.n_tokens == 0 || args.n_requests == 0 || args.max_new == 0) return hipSuccess;
    PagedAttnArgs a = args;
    a.Hq = s.Hq; a.Hkv = s.Hkv; a.G = s.G;
    a.scale_log2e = (1.0f / sqrtf((float)s.d)) * 1.4426950408889634f;
    if (s.dtype == FR_BF16) return s.d == 128 ? launch<__bf16, 128>(a, st) : launch<__bf16, 64>(a, st);
    return s.d == 128 ? launch<float, 128>(a, st) : launch<float, 64>(a, st);
}

}  // namespace fr
