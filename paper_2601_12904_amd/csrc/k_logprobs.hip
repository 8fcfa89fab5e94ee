// Log probabilities of given tokens, entropies and the likeliest tokens from rows of logits.  With x = scale * logit, m the row's largest x and t = x - m:
//
//   S = sum e^t,  W = sum e^t t,  lse = m + ln S,  log p = t - ln S,  entropy = -sum p log p = ln S - W / S   (both terms are at least 0: nothing cancels)
//
// Every logit is read once: a row's threads each hold (m, S, W) of the vectors that they have seen, scaled when m grows, and add up at the end.
//
// The n largest.  A thread also keeps the largest value of its vectors and the first vector that holds it.  Ordered by (value, lower index), the n-th best of these is a bound
// that n elements reach, and an element that is better than it lies in one of the n best threads: their vectors are read once more (n in TB of the row), what
// reaches the bound (about n elements) goes to a list in LDS and finds its rank by counting.  All of a thread's vectors are looked at only where its second best one reaches the bound, which
// it has kept too: else its best vector is enough (the 16 bytes of a vector come as a line of 128; 4096 rows of 128256, 20 alternatives, 242 us otherwise).  A list that runs over, in rows that no model makes, is replaced by n
// passes over the row.  The n best threads are found the same way: n / 4 rounds of a maximum in each of the four waves leave some 2 n of them to be counted (counting all 256 against one
// another took 4 us, twice in a call of few rows).
//
// One alternative, as in greedy steps, needs no list: the largest of the threads' keys, whose holder looks at one vector again (8 rows 6.8 us, 64 rows 10.6; while both were there, the list of one took 3.3 us longer).
//
// Few rows: each row in parts, joined by a second launch in a fixed order.
//
// Bound by memory: 4096 rows of 128256 in bf16 with 5 alternatives 195 us, 5.4 TB/s (reads alone; a copy's rate is 5.1).  Vector instructions are issued in 88 % of the cycles then: an
// exponential, two multiply-adds and the maxima per element.  8 rows of 128256, us by the number of alternatives, 0, 1, 5, 20, 32: 5.8, 6.8, 10.9, 13.1, 18; latency of two launches and of finding the best.
#include "fr_internal.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr int TB = 256, CAP = 1024;   // threads; candidates
constexpr int MAX_TOP = FR_LOGPROBS_MAX_TOP;
static_assert(MAX_TOP * MAX_TOP <= CAP, "the lists of MAX_TOP parts");
constexpr float LOW = -1e30f;         // in the place of a difference of -inf: 0 times it is 0

typedef unsigned long long u64;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

// Values in their order as whole numbers, then lower indexes first; 0: no element.  A NaN counts as -inf, -0 as 0.
__device__ __forceinline__ u64 key_of(float x, uint32_t index) {
    const uint32_t u = __float_as_uint(x != x ? -INFINITY : x + 0.f);
    return (u64)(u ^ ((u >> 31) != 0 ? 0xFFFFFFFFu : 0x80000000u)) << 32 | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float value_of(u64 key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u ^ ((u >> 31) != 0 ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ int index_of(u64 key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

struct Sums {   // of some of a row's elements, relative to the largest of them (base 2)
    float m, s, w;
    __device__ __forceinline__ static float ref(float m) { return m == -INFINITY ? 0.f : m; }   // (nothing but -inf: weights of 0)
    __device__ __forceinline__ void raise(float to, float c) {
        const float d = fmaxf((m - ref(to)) * c, LOW), f = __builtin_amdgcn_exp2f(d);
        w = f * (w + s * d);
        s *= f;
        m = to;
    }
};

struct Lds {
    u64 key[TB + 4];
    u64 candidate[CAP + 4];
    u64 top[MAX_TOP];
    int best_at[TB];
    float second[TB];
    u64 wave_key[TB / 64];
    Sums part[TB / 64];
    int chosen[MAX_TOP];
    u64 bound;
    int n_keys, n;
};

// Over the wave's lanes, all of them active, from lane to lane without LDS (through it sums and maxima took 1300 cycles of a part's 12000, twice as much of what joins them): `with` of a value and of
// what comes from 1, 2, 4, 8 lanes to the left within 16, then from the last lane of 16 to the next 16, and of 32 to the next 32; `none` where nothing comes.  In the last lane; uniform.
template <typename With>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, uint32_t none, With with) {
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x111, 0xF, 0xF, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x112, 0xF, 0xF, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x114, 0xF, 0xF, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x118, 0xF, 0xF, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x142, 0xA, 0xF, false));
    v = with(v, __builtin_amdgcn_update_dpp(none, v, 0x143, 0xC, 0xF, false));
    return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ float wave_sum(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ float wave_max(float v) {
    return __uint_as_float(wave_reduce(__float_as_uint(v), __float_as_uint(-INFINITY), [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    return wave_reduce(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ u64 wave_max(u64 key) {
    const uint32_t hi = (uint32_t)(key >> 32), lo = (uint32_t)key, top = wave_max(hi);
    const uint64_t lanes = __ballot(hi == top);
    const uint32_t low = (lanes & (lanes - 1)) == 0 ? __builtin_amdgcn_readlane(lo, __builtin_ctzll(lanes)) : wave_max(hi == top ? lo : 0u);
    return (u64)top << 32 | low;
}

// Over the workgroup, in a fixed order; every thread has the result.
__device__ __forceinline__ Sums all_sums(Sums a, float c, Lds& sm) {
    a.raise(wave_max(a.m), c);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    if ((threadIdx.x & 63) == 0) sm.part[threadIdx.x >> 6] = a;
    __syncthreads();
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < TB / 64; ++w) top = fmaxf(top, sm.part[w].m);
    Sums r{top, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < TB / 64; ++w) {
        Sums p = sm.part[w];
        p.raise(top, c);
        r.s += p.s;
        r.w += p.w;
    }
    return r;
}

// The largest key of the workgroup; every thread has the result.
__device__ __forceinline__ u64 largest(u64 key, Lds& sm) {
    key = wave_max(key);
    if ((threadIdx.x & 63) == 0) sm.wave_key[threadIdx.x >> 6] = key;
    __syncthreads();
    u64 r = sm.wave_key[0];
#pragma unroll
    for (int w = 1; w < TB / 64; ++w) r = max(r, sm.wave_key[w]);
    return r;
}
// Bits of the numbers below n (a list of n lists is walked without divisions).
__device__ __forceinline__ int bits_below(int n) { return n <= 1 ? 0 : 32 - __builtin_clz(n - 1); }
// How many of list[0 .. count - 1] are above `mine`; zeros stand behind them up to a multiple of four.
__device__ __forceinline__ int rank_in(const u64* list, int count, u64 mine) {
    int rank = 0;
    for (int i = 0; i < count; i += 4) rank += (list[i] > mine) + (list[i + 1] > mine) + (list[i + 2] > mine) + (list[i + 3] > mine);
    return rank;
}

// The first n_keys threads have a key (none of them twice), the others 0.  Leaves the n-th best of them as sm.bound (0 if there are fewer), and who has the best n as sm.chosen, best
// first; returns how many are chosen.
__device__ __forceinline__ int choose(u64 key, int n, int n_keys, Lds& sm) {
    const int tid = threadIdx.x, wave = tid >> 6, full = n_keys / 64;   // waves that have 64
    if (tid == 0) { sm.bound = 0; sm.n_keys = 0; sm.n = 0; }
    if (wave < full) {   // the best ceil(n / full) of the wave, one by one: n in all, and the least of them bounds the n-th best of all
        u64 left = key, top = 0;
        for (int i = 0; i < n; i += full) {
            top = wave_max(left);
            if (left == top) left = 0;
        }
        if ((tid & 63) == 0) sm.wave_key[wave] = top;
    }
    __syncthreads();
    u64 low = full > 0 ? ~(u64)0 : 0;
    for (int w = 0; w < full; ++w) low = min(low, sm.wave_key[w]);
    const bool some = key != 0 && key >= low;
    const uint64_t lanes = __ballot(some);
    int at = 0;
    if ((tid & 63) == 0 && lanes != 0) at = atomicAdd(&sm.n_keys, __popcll(lanes));
    at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
    if (some) sm.key[at] = key;
    __syncthreads();
    const int count = sm.n_keys;
    if (tid < 4) sm.key[count + tid] = 0;
    __syncthreads();
    if (some) {
        const int rank = rank_in(sm.key, count, key);
        if (rank < n) sm.chosen[rank] = tid;
        if (rank == n - 1) sm.bound = key;
    }
    __syncthreads();
    return min(n, n_keys);
}
// The best n of the candidates, best first; 0 behind them.
__device__ __forceinline__ void rank_candidates(int count, int n, Lds& sm) {
    const int tid = threadIdx.x;
    if (tid < MAX_TOP) sm.top[tid] = 0;
    if (tid < 4) sm.candidate[count + tid] = 0;
    __syncthreads();
    for (int j = tid; j < count; j += TB) {
        const u64 mine = sm.candidate[j];
        const int rank = rank_in(sm.candidate, count, mine);
        if (rank < n) sm.top[rank] = mine;
    }
    __syncthreads();
}

// The logit of the row's token, which thread 64 fetches before it is needed.
struct TokenLogit { bool inside; float x; };
template <typename T>
__device__ __forceinline__ TokenLogit token_logit(const TokenLogprobsArgs& a, int64_t t) {
    if (threadIdx.x != 64 || a.logprobs == nullptr) return {false, 0.f};
    const int token = a.tokens[t];
    const bool inside = (uint32_t)token < (uint32_t)a.n_vocab;
    return {inside, inside ? Elem<T>::to_f32(((const T*)a.logits)[t * a.row_stride + token]) : 0.f};
}
// A row's outputs, from its sums and its best elements (sm.top).
template <typename T>
__device__ __forceinline__ void answer(const TokenLogprobsArgs& a, int64_t t, const Sums& r, const TokenLogit& of_token, const Lds& sm) {
    const int tid = threadIdx.x;
    const bool none = r.m == -INFINITY && r.s == 0.f;
    const float ln_s = logf(r.s);
    auto logprob = [&](float x) { return none ? -INFINITY : (x - r.m) * a.scale - ln_s; };
    if (tid < a.n_top) {
        const u64 key = sm.top[tid];
        if (a.top_ids != nullptr) a.top_ids[t * a.n_top + tid] = key != 0 ? index_of(key) : -1;
        if (a.top_logprobs != nullptr) a.top_logprobs[t * a.n_top + tid] = key != 0 ? logprob(value_of(key)) : -INFINITY;
    }
    if (tid == 0) {
        if (a.lse != nullptr) a.lse[t] = none ? -INFINITY : r.m * a.scale + ln_s;
        if (a.entropy != nullptr) a.entropy[t] = none ? 0.f : ln_s - r.w / r.s * 0.6931471805599453f;
    }
    if (tid == 64 && a.logprobs != nullptr) a.logprobs[t] = of_token.inside ? logprob(of_token.x) : -INFINITY;
}

// Results of a part, in memory: m, s, w, one unused, then its best elements.
__device__ __forceinline__ float* part_of(float* partials, int64_t t, int part, int parts, int n_top) { return partials + (t * parts + part) * (4 + 2 * n_top); }

// blockIdx.x = row x parts + part.  SEVERAL: more than one alternative is asked for.
template <typename T, bool SEVERAL>
__global__ __launch_bounds__(TB) void token_logprobs_kernel(const TokenLogprobsArgs a, float* partials, int parts) {
    constexpr int N = 16 / sizeof(T), U = 4;   // elements of a vector; vectors of a thread in flight
    struct alignas(16) V { T v[N]; };
    __shared__ Lds sm;
    const int tid = threadIdx.x;
    const int64_t t = blockIdx.x / parts;
    const int part = blockIdx.x % parts;
    // The row as vectors of 16 bytes, from the one that holds its first element on: shift elements of that belong to the row before.
    const int64_t start = t * a.row_stride;
    const int shift = (int)(start % N), vocab = a.n_vocab;
    const T* row = (const T*)a.logits + start;
    const V* vectors = reinterpret_cast<const V*>(row - shift);
    const int first = shift > 0 ? 1 : 0, full = max(0, (int)(((int64_t)shift + vocab) / N) - first);   // vectors that lie in the row as a whole
    const int head = shift > 0 ? min(vocab, N - shift) : 0, tail0 = max((int64_t)head, (int64_t)N * (first + full) - shift), tail = max(0, vocab - tail0);
    const int n_edge = part == 0 ? head + tail : 0;                 // elements of the others, one to a thread
    const int edge = tid < head ? tid : tail0 + tid - head;
    const int some = full / parts, more = full - some * parts;      // vectors of a part; the first parts have one more
    const int lo = first + some * part + min(part, more), hi = lo + some + (part < more ? 1 : 0);
    const float c = fminf(a.scale * 1.4426950408889634f, 3.4e38f);

    Sums r{-INFINITY, 0.f, 0.f};
    if (tid < n_edge) {
        const float x = Elem<T>::to_f32(row[edge]);
        r.m = fmaxf(r.m, x);
        r.s = __builtin_amdgcn_exp2f((x - Sums::ref(r.m)) * c);
    }
    float best = -INFINITY, second = -INFINITY;   // the largest values of the thread's vectors, and the first vector that has the largest
    int best_at = lo + tid;
    auto take = [&](const V (&x)[U], int v0) {
        float f[U][N], top = r.m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float m = -INFINITY;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                f[u][e] = Elem<T>::to_f32(x[u].v[e]);
                m = fmaxf(m, f[u][e]);
            }
            second = __builtin_amdgcn_fmed3f(m, best, second);
            if (m > best) { best = m; best_at = v0 + TB * u; }
            top = fmaxf(top, m);
        }
        r.raise(top, c);
        const float ref = Sums::ref(top);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s = 0.f, w = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float d = (f[u][e] - ref) * c, p = __builtin_amdgcn_exp2f(d);
                s += p;
                w = __builtin_fmaf(p, fmaxf(d, LOW), w);
            }
            r.s += s;
            r.w += w;
        }
    };
    int v = lo + tid;
    for (; v + TB * (U - 1) < hi; v += TB * U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = vectors[v + TB * u];
        take(x, v);
    }
    if (v < hi) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int e = 0; e < N; ++e) x[u].v[e] = Elem<T>::from_f32(-INFINITY);
            if (v + TB * u < hi) x[u] = vectors[v + TB * u];
        }
        take(x, v);
    }
    r = all_sums(r, c, sm);
    const int n = a.n_top;
    if (!SEVERAL && n == 1) {   // only the likeliest: who has it looks at its vector once more
        const u64 mine = lo + tid < hi ? key_of(best, (uint32_t)(best_at * (int64_t)N - shift)) : 0, at_edge = tid < n_edge ? key_of(Elem<T>::to_f32(row[edge]), (uint32_t)edge) : 0;
        const u64 first_of = largest(max(mine, at_edge), sm);
        if (first_of == at_edge && at_edge != 0) sm.top[0] = at_edge;
        if (first_of == mine && mine != 0) {
            const V x = vectors[best_at];
            u64 top = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) top = max(top, key_of(Elem<T>::to_f32(x.v[e]), (uint32_t)(best_at * (int64_t)N - shift) + e));
            sm.top[0] = top;
        }
        __syncthreads();
    }
    if constexpr (SEVERAL) {
        const int n_keys = min(TB, hi - lo);
        sm.best_at[tid] = best_at;
        sm.second[tid] = second;
        const int n_chosen = choose(lo + tid < hi ? key_of(best, (uint32_t)(best_at * (int64_t)N - shift)) : 0, n, n_keys, sm);
        // (the index in the bound is that of the best thread's vector's first element: its last one will do)
        const u64 bound = sm.bound == 0 ? 0 : sm.bound - (N - 1);
        const float least = bound == 0 ? -INFINITY : value_of(bound);
        auto offer = [&](u64 key) {
            if (key < bound) return;
            const int at = atomicAdd(&sm.n, 1);
            if (at < CAP) sm.candidate[at] = key;
        };
        const int each = (hi - lo + TB - 1) / TB, shift_n = bits_below(n_chosen);   // vectors of a thread, at most
        for (int i = tid; i >> shift_n < each; i += TB) {
            const int rank = i & ((1 << shift_n) - 1);
            if (rank >= n_chosen) continue;
            const int who = sm.chosen[rank], at = lo + who + TB * (i >> shift_n);
            if (at >= hi || (at != sm.best_at[who] && sm.second[who] < least)) continue;
            const V x = vectors[at];
            const uint32_t index = (uint32_t)(at * (int64_t)N - shift);
#pragma unroll
            for (int e = 0; e < N; ++e) offer(key_of(Elem<T>::to_f32(x.v[e]), index + e));
        }
        if (tid < n_edge) offer(key_of(Elem<T>::to_f32(row[edge]), (uint32_t)edge));
        __syncthreads();
        const int count = sm.n;
        if (count <= CAP) {
            rank_candidates(count, n, sm);
        } else {
            u64 last = ~(u64)0;
            for (int i = 0; i < n; ++i) {   // the best one below the last
                u64 next = 0;
                auto see = [&](u64 key) { next = key < last && key > next ? key : next; };
                for (int at = lo + tid; at < hi; at += TB) {
                    const V x = vectors[at];
#pragma unroll
                    for (int e = 0; e < N; ++e) see(key_of(Elem<T>::to_f32(x.v[e]), (uint32_t)(at * (int64_t)N - shift) + e));
                }
                if (tid < n_edge) see(key_of(Elem<T>::to_f32(row[edge]), (uint32_t)edge));
                for (int d = 1; d < 64; d <<= 1) next = max(next, (u64)__shfl_xor(next, d));
                __syncthreads();
                if ((tid & 63) == 0) sm.wave_key[tid >> 6] = next;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < TB / 64; ++w) next = max(next, sm.wave_key[w]);
                if (tid == 0) sm.top[i] = next;
                last = next;
            }
            __syncthreads();
        }
    }
    if (parts == 1) {
        answer<T>(a, t, r, token_logit<T>(a, t), sm);
        return;
    }
    float* to = part_of(partials, t, part, parts, n);
    if (tid == 0) { to[0] = r.m; to[1] = r.s; to[2] = r.w; }
    if (tid < n) reinterpret_cast<u64*>(to + 4)[tid] = sm.top[tid];
}

// blockIdx.x = row; parts <= TB.  A part's best elements stand in their order, so its first is what a thread's largest was above.
template <typename T>
__global__ __launch_bounds__(TB) void token_logprobs_join_kernel(const TokenLogprobsArgs a, float* partials, int parts) {
    __shared__ Lds sm;
    const int tid = threadIdx.x, n = a.n_top;
    const int64_t t = blockIdx.x;
    const float c = fminf(a.scale * 1.4426950408889634f, 3.4e38f);
    const TokenLogit of_token = token_logit<T>(a, t);
    Sums r{-INFINITY, 0.f, 0.f};
    u64 key = 0;
    if (tid < parts) {
        const float* p = part_of(partials, t, tid, parts, n);
        r = Sums{p[0], p[1], p[2]};
        if (n > 0) key = reinterpret_cast<const u64*>(p + 4)[0];
    }
    r = all_sums(r, c, sm);
    if (n == 1) {
        key = largest(key, sm);
        if (tid == 0) sm.top[0] = key;   // (its own reader)
    } else if (n > 0) {
        const int n_chosen = choose(key, n, parts, sm);
        u64 bound = sm.bound;
        auto best_of = [&](int part, int i) { return reinterpret_cast<const u64*>(part_of(partials, t, part, parts, n) + 4)[i]; };
        // Another bound: the best ceil(n / depth) parts have depth elements each above the least of their depth-th ones.
        const int depth = max(n >= 16 ? 4 : n >= 4 ? 2 : 1, (n + n_chosen - 1) / n_chosen), lists = (n + depth - 1) / depth;
        if (tid < 64) {
            u64 least = tid < lists ? best_of(sm.chosen[tid], depth - 1) : ~(u64)0;
            for (int d = 1; d < 32; d <<= 1) least = min(least, (u64)__shfl_xor(least, d));
            if (tid == 0) sm.wave_key[0] = least;
        }
        __syncthreads();
        bound = max(bound, sm.wave_key[0]);
        const int shift_n = bits_below(n);
        for (int i = tid; i >> shift_n < n_chosen; i += TB) {
            if ((i & ((1 << shift_n) - 1)) >= n) continue;
            const u64 k = best_of(sm.chosen[i >> shift_n], i & ((1 << shift_n) - 1));
            if (k != 0 && k >= bound) sm.candidate[atomicAdd(&sm.n, 1)] = k;   // (n x n of them at most)
        }
        __syncthreads();
        rank_candidates(sm.n, n, sm);
    }
    answer<T>(a, t, r, of_token, sm);
}

template <typename T>
hipError_t launch(const TokenLogprobsArgs& a, float* partials, int n_cu, hipStream_t st) {
    constexpr int N = 16 / sizeof(T);
    // Parts of a row: until there are four workgroups per compute unit, none of fewer than two vectors for each thread.
    int parts = 1;
    if (a.n_tokens < 2 * n_cu) parts = (int)std::max<int64_t>(1, std::min<int64_t>({4 * n_cu / (int64_t)a.n_tokens, a.n_vocab / (2 * N * TB), TB}));
    const dim3 grid((unsigned)((int64_t)a.n_tokens * parts));
    if (a.n_top > 1) token_logprobs_kernel<T, true><<<grid, dim3(TB), 0, st>>>(a, partials, parts);
    else token_logprobs_kernel<T, false><<<grid, dim3(TB), 0, st>>>(a, partials, parts);
    if (parts > 1) token_logprobs_join_kernel<T><<<dim3((unsigned)a.n_tokens), dim3(TB), 0, st>>>(a, partials, parts);
    return hipGetLastError();
}

}  // namespace

size_t token_logprobs_partials_bytes(int n_cu) { return (size_t)4 * n_cu * (4 + 2 * MAX_TOP) * sizeof(float); }

hipError_t launch_token_logprobs(const TokenLogprobsArgs& a, float* partials, int n_cu, hipStream_t st) {
    if (a.n_tokens == 0) return hipSuccess;
    return a.dtype == FR_BF16 ? launch<__bf16>(a, partials, n_cu, st) : launch<float>(a, partials, n_cu, st);
}

}  // namespace fr
