// Attention over a paged cache: bf16 requests with few query columns (decoding, drafted tokens), and all requests in fp32; head_dim 64 or 128.
//
// Every byte of K and V is used for a handful of columns, so the rate of memory is the bound.  One workgroup = one KV head x 16 NC query columns
// ((row, query head) pairs, the heads of the group fastest); its four waves deal the blocks of 32 keys among themselves, each with accumulators of its own
// that are merged through LDS at the end of a piece: nothing in the loop waits for another wave.  The line of work is dealt out in equal shares
// (k_paged.hpp): units of 128 keys of a column tile, as many for a tile of a prompt's first rows as for its last.  (Tiles by what they see would balance the load, but cuts most items of a
// prompt, which costs more: 512 rows from nothing, 32 / 8 heads, 31 us for 20, 1024 rows 77 for 41.)
//
// Measured, kernel alone: 64 rows behind 571 - 15757 positions (0.99 GB), 32 / 8 heads, 185 us = 5.4 TB/s; 32 times 2 - 8 rows behind 324 - 4902, 16 / 8 heads of 64 (0.14 GB), 31 us = 4.6 TB/s; one row behind
// 4096 (17 MB) 10 us: the chain lengths -> table -> keys -> values -> merge; 254 rows in fp32, 4 heads of 64, 11 us.  The joining pass 3.9 - 7.9 us, of which a launch of nothing is 4.
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16 (fp32: v_mfma_f32_16x16x4_f32), keys on the register dimension of S^T and columns on lanes: the accumulators of two 16-key
// blocks are, after conversion, the B operand of the second product.  Row m of value product md is dim D / 16 m + md, so that a lane needs 16 (8)
// neighbouring bytes of each of its eight value rows and transposes them itself with byte permutes.  Weights go into the second product as bf16 (half a
// step, 2^-8, of each; their sum is taken in fp32 before), as the output does; in fp32 nothing is rounded to fewer bits.  A step of the fp32 instruction takes
// four dims, or four keys: with 16 bytes per lane, element e of quarter kg is dim 16 j + 4 kg + e of step (j, e) in both operands, and the accumulator
// of key 4 kg + e is as it stands the operand of step e of the second product.
//
// A wave copies a block global -> LDS (no registers, no wait) while it works on the one before.  The page numbers of a block's keys come the same way
// one block earlier, so that the copies of a wave are the only thing its memory counter counts, and every page size goes the same way.
//
// Softmax.  A column's exponent reference goes up, and its sums are scaled, only when a logit is 8 (base 2) or more above it.  A wave one of whose references
// is PAGED_FAR or more rounds the scaled logits before it takes the reference from them.
//
// What a column does not see stays out of it by hand, as a weight of 0 does not take a NaN or an infinity out of a product: keys behind the tile's last
// row repeat that one, and values that are not finite leave a block that only some columns see whole and reach those columns when the loop is over.
#include "k_paged.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr int W = 4;              // waves per workgroup
constexpr int UNIT = 32 * W;      // keys of a unit of work: a block for every wave

template <typename T, int D, int NC>
struct StreamLds {
    static constexpr int TILE = 32 * D * (int)sizeof(T);   // bytes of a block of 32 keys or values
    static constexpr int C = 16 * NC;
    int32_t page[W][2][64];                   // page numbers of the keys of a wave's next blocks
    union {
        struct { unsigned char k[W][TILE], v[W][TILE]; };
        struct {
            float o[W][C][D + 4];
            float m[C][W], l[C][W];
        };
    };
};
// Workgroups that are resident on a compute unit: as many as its LDS and registers hold.
template <typename T, int D, int NC>
constexpr int RESIDENT = sizeof(T) * D <= 128 ? (NC == 1 ? 4 : 3) : sizeof(T) * D <= 256 ? 2 : 1;

// Units of a request: column tiles x units of keys.
template <int C>
__device__ __forceinline__ int64_t stream_cost(const PagedArgs& a, int b, int* n_ct = nullptr, int* n_units = nullptr, PagedRequest* req = nullptr) {
    const PagedRequest r = paged_request(a, b);
    if (req) *req = r;
    if (r.n == 0) return 0;
    const int ct = (int)(((int64_t)r.n * a.G + C - 1) / C), units = max(paged_position(a, r, r.n - 1), 0) / UNIT + 1;
    if (n_ct) { *n_ct = ct; *n_units = units; }
    return (int64_t)ct * units;
}

template <typename T, int D, int NC, bool ALIGNED>
struct StreamPiece {
    static constexpr bool F32 = sizeof(T) == 4;
    static constexpr int N = 16 / sizeof(T), NJ = D / 16;         // elements of a 16-byte vector; dims per lane of a value row
    static constexpr int NK = D / (4 * N), VW = NJ * (int)sizeof(T) / 4;   // vectors of a lane's key (and query) row, words of its values
    static constexpr int RV = D / N, COPIES = 32 * RV / 64;       // vectors of a row; copies of 1 KB of a block
    static constexpr int C = 16 * NC;
    using Lds = StreamLds<T, D, NC>;
    typedef __attribute__((ext_vector_type(VW))) uint32_t VVec;

    // One piece: units [r0, r1) of column tile ct of request b.  whole: it is all of the item, the outputs are stored; else the partial result goes to `part`.
    static __device__ __forceinline__ void run(const PagedArgs& a, Lds& sm, const PagedRequest& rq, int b, int ct, int g, int r0, int r1, bool whole, float* part) {
        const int tid = threadIdx.x, lane = tid & 63, x = lane & 15, kg = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int G = a.G, cols = rq.n * G, col0 = C * ct, token0 = col0 / G, head0 = col0 - token0 * G;
        const T* q_rows = (const T*)a.q;
        auto token_of = [&](int cl) { return token0 + paged_token(a, head0 + cl); };   // row, within the request, of column cl of the tile
        auto out_row = [&](int cl) {   // (row, head) of a column, counted over all heads
            const int i = paged_token(a, head0 + cl);
            return (size_t)(rq.first + token0 + i) * a.Hq + g * G + (head0 + cl - i * G);
        };
        const int last_col = min(C, cols - col0) - 1;
        u32x4 qf[NC][NK];   // B operand of S^T = K Q^T
        int pos[NC];
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {   // columns past the end: a copy of the last
            const int cl = min(16 * nb + x, last_col);
            const T* p = q_rows + out_row(cl) * D + N * kg;
            pos[nb] = paged_position(a, rq, token_of(cl));
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) qf[nb][ks] = *reinterpret_cast<const u32x4*>(p + 4 * N * ks);
        }
        const int p_first = paged_position(a, rq, token0);                     // keys up to here are visible to every column
        const int p_last = paged_position(a, rq, token_of(last_col));
        const int n_blocks = min((p_last + 32) / 32, W * r1);                                     // (none for a tile that sees nothing)
        f32x4 o[NJ][NC];   // O^T: row m of product md is dim NJ m + md
        float m[NC], l[NC];
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            m[nb] = PAGED_NO_MAX;
            l[nb] = 0.f;
#pragma unroll
            for (int md = 0; md < NJ; ++md) o[md][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int32_t* table = a.block_table + (size_t)b * a.W;
        const uint32_t row_bytes = (uint32_t)(a.Hkv * D * (int)sizeof(T));
        const unsigned char *k_base = (const unsigned char*)a.k_pages + (size_t)g * D * sizeof(T), *v_base = (const unsigned char*)a.v_pages + (size_t)g * D * sizeof(T);
        // A copy brings 64 / RV rows, RV lanes side by side to a row; copy i the rows COPIES q + i of the lanes' groups q, so that a lane's sources are
        // neighbours.  Vector c of key row r sits in place c ^ swz(r), so that the 16 rows of a fragment read meet in no bank.
        auto swz = [](int r) { return RV >= 16 ? r & 15 : (r & 3) | (r >> 1 & 4); };
        auto row_at = [](int r) { return 1024 * (r % COPIES) + 16 * RV * (r / COPIES); };
        const uint32_t k_lds = paged_lds(sm.k[wave]), v_lds = paged_lds(sm.v[wave]), page_lds = paged_lds(sm.page[wave]);
        const int qg = lane / RV, vec = lane % RV;
        const uint32_t k_place = 16 * (vec ^ swz(COPIES * qg)), v_place = 16 * vec;   // swz(COPIES q + i) = swz(COPIES q) ^ swz(i)
        auto is_page = [&](int p) { return (uint32_t)p < (uint32_t)a.n_pages; };
        auto copy_pages = [&](int blk, int ring) {   // of keys 32 blk .. 32 blk + 31 (twice)
            paged_copy4(table + paged_block(a, min(32 * blk + (lane & 31), p_last)), page_lds + 256 * ring);
        };
        uint32_t row[COPIES];   // cache rows of the lane's keys of the block on its way
        bool holes_next = false;
        auto find_rows = [&](int blk, int ring) {
            const int j0 = 32 * blk + COPIES * qg;
            bool hole = false;
            if constexpr (ALIGNED) {   // pages are whole multiples of the lane's COPIES rows
                const int page = sm.page[wave][ring][COPIES * qg], jc = min(j0, p_last), in = j0 - jc, base = jc - paged_block(a, jc) * a.P;
                hole = !is_page(page);
                const uint32_t at = (uint32_t)(hole ? 0 : page) * (uint32_t)a.P + (uint32_t)base;
                const int most = p_last - jc;
#pragma unroll
                for (int i = 0; i < COPIES; ++i) row[i] = at + (uint32_t)min(in + i, most);
            } else {
#pragma unroll
                for (int i = 0; i < COPIES; ++i) {
                    const int page = sm.page[wave][ring][COPIES * qg + i], j = min(j0 + i, p_last);
                    const bool none = !is_page(page);
                    hole = hole || none;
                    row[i] = (uint32_t)(none ? 0 : page) * (uint32_t)a.P + (uint32_t)(j - paged_block(a, j) * a.P);
                }
            }
            holes_next = __any(hole);
        };
        auto copy_k = [&] {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) paged_copy16(k_base + (size_t)row[i] * row_bytes + (k_place ^ (swz(i) * 16u)), k_lds + 1024 * i);
        };
        auto copy_v = [&] {
#pragma unroll
            for (int i = 0; i < COPIES; ++i) paged_copy16(v_base + (size_t)row[i] * row_bytes + v_place, v_lds + 1024 * i);
        };
        bool apart = false, far = false;   // far: some column's reference has reached PAGED_FAR
        int blk = W * r0 + wave;
        if (blk < n_blocks) {
            const int last = n_blocks - 1;   // (past the last block: that one again, nobody uses it; the counts of the waits stay the same)
            paged_wait_but<0>();   // (nothing that the compiler counts is in flight from here on)
            copy_pages(blk, 0);
            copy_pages(min(blk + W, last), 1);
            paged_wait_but<1>();
            find_rows(blk, 0);
            copy_k();
            copy_v();
            int ring = 1;   // of the next block's pages
#pragma unroll 1
            for (; blk < n_blocks; blk += W) {
                const bool holes = holes_next;
                f32x4 s[2][NC];
                paged_wait_but<COPIES>();   // this block's keys, and the next one's pages
                {
                    u32x4 kf[2][NK];   // keys 32 blk + 16 bb + x: elements 4 N ks + N kg ..
#pragma unroll
                    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
                        for (int bb = 0; bb < 2; ++bb)
                            kf[bb][ks] = *reinterpret_cast<const u32x4*>(sm.k[wave] + row_at(16 * bb + x) + 16 * ((4 * ks + kg) ^ swz(x)));
#pragma unroll
                    for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                        for (int nb = 0; nb < NC; ++nb) s[bb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int ks = 0; ks < NK; ++ks)
#pragma unroll
                        for (int e = 0; e < (F32 ? 4 : 1); ++e)
#pragma unroll
                            for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                                for (int nb = 0; nb < NC; ++nb) {
                                    if constexpr (F32)
                                        s[bb][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kf[bb][ks][e]), __uint_as_float(qf[nb][ks][e]), s[bb][nb], 0, 0, 0);
                                    else
                                        s[bb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[bb][ks]), __builtin_bit_cast(bf16x8, qf[nb][ks]),
                                                                                            s[bb][nb], 0, 0, 0);
                                }
                }
                int hole_of[2] = {0, 0};   // bit v: key 16 bb + 4 kg + v of this block has no page
                if (__builtin_expect(holes, 0)) {
#pragma unroll
                    for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                        for (int v = 0; v < 4; ++v) hole_of[bb] |= is_page(sm.page[wave][ring ^ 1][16 * bb + 4 * kg + v]) ? 0 : 1 << v;
                }
                __builtin_amdgcn_sched_barrier(0);
                find_rows(min(blk + W, last), ring);
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // (this block's pages and keys have been read)
                copy_k();
                copy_pages(min(blk + 2 * W, last), ring ^ 1);
                ring ^= 1;
                const bool partial = 32 * blk + 31 > p_first || holes;   // not every column sees all of these keys
                if (partial) {
#pragma unroll
                    for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb)
                                if (32 * blk + 16 * bb + 4 * kg + v > pos[nb] || (hole_of[bb] >> v & 1)) s[bb][nb][v] = -INFINITY;
                }
                float top[NC];
                bool raise = false;
#pragma unroll
                for (int nb = 0; nb < NC; ++nb) {
                    float t = s[0][nb][0];
#pragma unroll
                    for (int v = 1; v < 8; ++v) t = fmaxf(t, s[v / 4][nb][v % 4]);
                    top[nb] = paged_column_max(t) * a.scale_log2e;
                    raise = raise || top[nb] > m[nb] + PAGED_RAISE;
                }
                if (__any(raise)) {
#pragma unroll
                    for (int nb = 0; nb < NC; ++nb) {
                        const float up = fmaxf(m[nb], top[nb]), down = __builtin_amdgcn_exp2f(m[nb] - up);
                        m[nb] = up;
                        l[nb] *= down;
#pragma unroll
                        for (int md = 0; md < NJ; ++md) o[md][nb] *= down;
                        far = far || __any(fabsf(up) >= PAGED_FAR && up != PAGED_NO_MAX);
                    }
                }
                const float scale = far ? 1.f : a.scale_log2e;
                if (__builtin_expect(far, 0)) {
#pragma clang fp contract(off)
#pragma unroll
                    for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                        for (int nb = 0; nb < NC; ++nb)
#pragma unroll
                            for (int v = 0; v < 4; ++v) s[bb][nb][v] *= a.scale_log2e;
                }
                u32x4 p[NC];   // bf16: weights as the B operand of the second product: slot 4 bb + v of quarter kg is key 16 bb + 4 kg + v
#pragma unroll
                for (int nb = 0; nb < NC; ++nb)
#pragma unroll
                    for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                        for (int v = 0; v < 4; v += 2) {
                            const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[bb][nb][v], scale, -m[nb]));
                            const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[bb][nb][v + 1], scale, -m[nb]));
                            l[nb] += p0 + p1;
                            if constexpr (F32) {
                                s[bb][nb][v] = p0;
                                s[bb][nb][v + 1] = p1;
                            } else {
                                bf16x2 t;
                                t[0] = (__bf16)p0;
                                t[1] = (__bf16)p1;
                                p[nb][2 * bb + v / 2] = __builtin_bit_cast(uint32_t, t);
                            }
                        }
                paged_wait_but<COPIES + 1>();   // this block's values
                VVec vf[8];   // values of keys 32 blk + 16 (i / 4) + 4 kg + i % 4, dims NJ x ..
#pragma unroll
                for (int i = 0; i < 8; ++i) vf[i] = *reinterpret_cast<const VVec*>(sm.v[wave] + row_at(16 * (i >> 2) + 4 * kg + (i & 3)) + (int)sizeof(T) * NJ * x);
                if (partial) {
                    bool bad = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int e = 0; e < VW; ++e) bad = bad || paged_not_finite<T>(vf[i][e]);
                    if (__builtin_expect(__any(bad), 0)) {   // values that are not finite: not into the product
                        apart = true;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
#pragma unroll
                            for (int e = 0; e < VW; ++e) vf[i][e] = paged_finite_or_zero<T>(vf[i][e]);
                    }
                }
#pragma unroll
                for (int md = 0; md < NJ; ++md) {
                    if constexpr (F32) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb)
                                o[md][nb] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[i][md]), s[i / 4][nb][i % 4], o[md][nb], 0, 0, 0);
                    } else {
                        u32x4 vt;   // dim NJ x + md of the eight keys
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            vt[j] = __builtin_amdgcn_perm(vf[2 * j + 1][md / 2], vf[2 * j][md / 2], md % 2 == 0 ? 0x05040100u : 0x07060302u);
#pragma unroll
                        for (int nb = 0; nb < NC; ++nb)
                            o[md][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt), __builtin_bit_cast(bf16x8, p[nb]), o[md][nb], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
                asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // (the values have been read)
                copy_v();
            }
            paged_wait_but<0>();
        }
        if (__builtin_expect(apart, 0)) {   // the values that were left out reach the columns that see them
#pragma unroll 1
            for (int at = W * r0 + wave; at < n_blocks; at += W)
#pragma unroll 1
                for (int t = 0; t < 32; ++t) {
                    const int j = 32 * at + t;
                    if (j > p_last) break;
                    const int blk0 = 32 * at, page_block = paged_block(a, j), page = table[page_block];
                    if (!is_page(page)) continue;
                    // (only what the loop left out: blocks that some column does not see whole)
                    bool partial = blk0 + 31 > p_first;
                    if (!partial) {
                        for (int i = 0; i < 32; ++i) partial = partial || !is_page(table[paged_block(a, blk0 + i)]);
                    }
                    if (!partial) continue;
                    const T* key = (const T*)(v_base + ((size_t)page * a.P + (j - page_block * a.P)) * row_bytes);
#pragma unroll
                    for (int v = 0; v < 4; ++v)
#pragma unroll
                        for (int md = 0; md < NJ; ++md) {
                            const float w = Elem<T>::to_f32(key[NJ * (4 * kg + v) + md]);
                            const float add = (__float_as_uint(w) & 0x7F800000u) == 0x7F800000u ? w : 0.f;
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb) o[md][nb][v] += j <= pos[nb] ? add : 0.f;
                        }
                }
        }
        paged_lds_barrier();   // everyone is done with the copies
        // ---- merge the waves ---------------------------------------------------------------------------------------------
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            const float sum = paged_column_sum(l[nb]);
            if (kg == 0) { sm.m[16 * nb + x][wave] = m[nb]; sm.l[16 * nb + x][wave] = sum; }
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int h = 0; h < NJ / 4; ++h)
                    *reinterpret_cast<f32x4*>(&sm.o[wave][16 * nb + x][NJ * (4 * kg + v) + 4 * h]) =
                        f32x4{o[4 * h][nb][v], o[4 * h + 1][nb][v], o[4 * h + 2][nb][v], o[4 * h + 3][nb][v]};
        }
        paged_lds_barrier();
        constexpr int NV = D / 8;
        for (int i = tid; i < C * NV; i += 64 * W) {
            const int c = i / NV, v8 = i % NV;
            if (c > last_col) break;
            float mw[W], lsum = 0.f, top = PAGED_NO_MAX;
#pragma unroll
            for (int w = 0; w < W; ++w) { mw[w] = sm.m[c][w]; top = fmaxf(top, mw[w]); }
            f32x4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float f = __builtin_amdgcn_exp2f(mw[w] - top);   // (a wave that saw nothing: 0, beside one that did)
                lsum = __builtin_fmaf(sm.l[c][w], f, lsum);
                lo += *reinterpret_cast<const f32x4*>(&sm.o[w][c][8 * v8]) * f;
                hi += *reinterpret_cast<const f32x4*>(&sm.o[w][c][8 * v8 + 4]) * f;
            }
            if (!whole) {
                float* dst = part + c * paged_part_floats<D>();
                if (v8 == 0) { dst[0] = top; dst[1] = lsum; }
#pragma unroll
                for (int e = 0; e < 4; ++e) { dst[2 + 8 * v8 + e] = lo[e]; dst[6 + 8 * v8 + e] = hi[e]; }
                continue;
            }
            const bool none = lsum == 0.f;   // it saw nothing (the largest weight of one that did is at least 2^-8)
            const float inv_l = none ? 0.f : 1.0f / lsum;
            const size_t oc = out_row(c);
            T* dst = (T*)a.out + oc * D + 8 * v8;
            struct alignas(16) { T v[8]; } y;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                y.v[e] = Elem<T>::from_f32(lo[e] * inv_l);
                y.v[4 + e] = Elem<T>::from_f32(hi[e] * inv_l);
            }
#pragma unroll
            for (int h = 0; h < (F32 ? 2 : 1); ++h) reinterpret_cast<u32x4*>(dst)[h] = reinterpret_cast<const u32x4*>(&y)[h];
            if (v8 == 0 && a.lse != nullptr) a.lse[oc] = none ? -INFINITY : (top + __builtin_amdgcn_logf(lsum)) * 0.6931471805599453f;
        }
        paged_lds_barrier();   // (the next piece's copies overwrite what was merged)
    }
};

template <typename T, int D, int NC, bool ALIGNED>
__global__ __launch_bounds__(64 * W, (RESIDENT<T, D, NC>)) void paged_stream_kernel(const PagedArgs args) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    PagedArgs a = args;
    if (a.route) {   // all requests, those with few columns, or none
        a.cols_lo = 0;
        a.cols_hi = !paged_route(a, D * (int)sizeof(T) * 2) ? INT32_MAX : a.together ? 0 : a.few;
    }
    auto& sm = *reinterpret_cast<StreamLds<T, D, NC>*>(smem_raw);
    constexpr int C = 16 * NC;
    const int g = paged_head(a), w = paged_workgroup(a);
    int64_t u = 0, end = 0;
    const PagedLine line = paged_line(a.B, [&](int b) { return stream_cost<C>(a, b); }, [&](int64_t total) {
        const int n = paged_sharers(a, total);
        if (w >= n) return (int64_t)-1;
        u = paged_first_unit(w, total, n);
        end = paged_first_unit(w + 1, total, n);
        return u;
    });
    PagedCut cut{0, 0, 0, 0};
    int64_t start = line.start;   // of the request's units
    for (int b = line.b; b >= 0 && u < end && b < a.B; ++b) {
        int n_ct, units;
        PagedRequest rq;
        const int64_t cost = stream_cost<C>(a, b, &n_ct, &units, &rq);
        if (cost == 0) continue;
        while (u < end && u < start + cost) {
            const int64_t in = u - start;
            const int ct = (int)paged_div(in, units), r0 = (int)(in - (int64_t)ct * units);
            const int r1 = (int)min((int64_t)units, r0 + (end - u));
            const bool whole = r0 == 0 && r1 == units;
            float* part = paged_slot(a, w, g, r0 > 0 ? 0 : 1, C * paged_part_floats<D>());
            if (r0 == 0 && r1 < units) cut = PagedCut{paged_owner(u + units - 1, line.total, paged_sharers(a, line.total)) - w + 1, rq.first, C * ct, rq.n * a.G};
            StreamPiece<T, D, NC, ALIGNED>::run(a, sm, rq, b, ct, g, r0, r1, whole, part);
            u += r1 - r0;
        }
        start += cost;
    }
    if (threadIdx.x == 0) paged_cuts(a)[(size_t)w * a.Hkv + g] = cut;
}

// Joins the pieces of the items that fell to several workgroups, in their order: blockIdx.x = workgroup x Hkv + KV head, whose cut it sees to.  One wave per column
// (blockIdx.y: four of them), all of a column's pieces in one trip to memory or a few: four at a time of an item of up to four, as most are (16 in any case: the loads
// of pieces that are not there made the pass 12.9 us instead of 7.9 for a chunk of 777 rows x 28 heads), else 16.  (A join by the last workgroup of an item to arrive, by a counter, needs no
// second launch, but its loads and stores go past the caches of the dies: one row behind 4096 18.4 us for the whole call, 16.4 this way.)
template <typename T, int D, int NC, int AHEAD>
__device__ __forceinline__ void join_column(const PagedArgs& a, const PagedCut& cut, int c, int g, int w0) {
    constexpr int C = 16 * NC, PF = paged_part_floats<D>(), EPT = D / 64;
    typedef __attribute__((ext_vector_type(EPT))) float Own;   // a lane's dims
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    const int n = cut.pieces, lane = threadIdx.x & 63;
    float top = PAGED_NO_MAX, l = 0.f;
    Own o = {};
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        f32x2 ml[AHEAD];
        Own po[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {   // (past the end: the last piece, which does not count)
            const int i = min(i0 + k, n - 1);
            const float* p = paged_slot(a, w0 + i, g, i == 0 ? 1 : 0, C * PF) + c * PF;
            ml[k] = *reinterpret_cast<const f32x2*>(p);
            po[k] = *reinterpret_cast<const Own*>(p + 2 + EPT * lane);
        }
        float up = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) up = i0 + k < n ? fmaxf(up, ml[k][0]) : up;
        const float f = __builtin_amdgcn_exp2f(top - up);
        top = up;
        l *= f;
        o *= f;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= n) continue;
            const float w = __builtin_amdgcn_exp2f(ml[k][0] - top);
            l += ml[k][1] * w;
            o += po[k] * w;
        }
    }
    const int col = cut.col0 + c, i = col / a.G;
    const size_t oc = (size_t)(cut.first_row + i) * a.Hq + g * a.G + (col - i * a.G);
    const bool none = l == 0.f;
    const float inv_l = none ? 0.f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < EPT; ++e) ((T*)a.out)[oc * D + EPT * lane + e] = Elem<T>::from_f32(o[e] * inv_l);
    if (lane == 0 && a.lse != nullptr) a.lse[oc] = none ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <typename T, int D, int NC>
__global__ __launch_bounds__(256) void paged_stream_join_kernel(const PagedArgs a) {
    const int g = blockIdx.x % a.Hkv, w0 = blockIdx.x / a.Hkv;
    const PagedCut cut = paged_cuts(a)[blockIdx.x];
    if (cut.pieces == 0) return;
    const int c = 4 * blockIdx.y + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (c >= min(16 * NC, cut.cols - cut.col0)) return;   // (wave-uniform)
    if (cut.pieces <= 4)
        join_column<T, D, NC, 4>(a, cut, c, g, w0);
    else
        join_column<T, D, NC, 16>(a, cut, c, g, w0);
}

template <typename T, int D, int NC, bool ALIGNED>
hipError_t launch(const PagedArgs& a, int cols, hipStream_t st) {
    using Lds = StreamLds<T, D, NC>;
    static_assert(RESIDENT<T, D, NC> * sizeof(Lds) <= 160 * 1024, "LDS of a compute unit");
    // Raises the kernel's dynamic LDS limit, once per process.
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_stream_kernel<T, D, NC, ALIGNED>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Lds));
    if (once != hipSuccess) return once;
    paged_stream_kernel<T, D, NC, ALIGNED><<<dim3(paged_grid(a.n_wg, a.Hkv)), dim3(64 * W), sizeof(Lds), st>>>(a);
    if (a.n_wg > 1 && a.cap > UNIT)   // (else every item is one unit, and none is cut)
        paged_stream_join_kernel<T, D, NC><<<dim3((unsigned)((a.n_wg - 1) * a.Hkv), (unsigned)((cols + 3) / 4)), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

template <typename T, int D, int NC>
hipError_t launch(const PagedArgs& a, int cols, hipStream_t st) {
    return a.P % StreamPiece<T, D, NC, true>::COPIES == 0 ? launch<T, D, NC, true>(a, cols, st) : launch<T, D, NC, false>(a, cols, st);
}

template <typename T, int D>
hipError_t launch(const PagedArgs& args, int n_cu, hipStream_t st) {
    PagedArgs a = args;
    const int64_t most = std::min<int64_t>((int64_t)a.max_new * a.G, a.cols_hi);   // columns of a request
    a.n_wg = std::max(1, (most <= 16 ? RESIDENT<T, D, 1> : RESIDENT<T, D, 2>) * n_cu / a.Hkv);
    return most <= 16 ? launch<T, D, 1>(a, (int)most, st) : launch<T, D, 2>(a, (int)std::min<int64_t>(most, 32), st);
}

// Columns of all workgroups' pieces on a compute unit, the larger of the two tilings'.
template <typename T, int D>
constexpr int COLUMNS = std::max(16 * RESIDENT<T, D, 1>, 32 * RESIDENT<T, D, 2>);
int columns(const Shape& s) {
    if (s.dtype == FR_BF16) return s.d == 128 ? COLUMNS<__bf16, 128> : COLUMNS<__bf16, 64>;
    return s.d == 128 ? COLUMNS<float, 128> : COLUMNS<float, 64>;
}

}  // namespace

size_t paged_stream_partials_bytes(const Shape& s, int n_cu) {
    // (one workgroup per KV head, where there are more of those than workgroups: nothing is cut)
    return (size_t)columns(s) * n_cu * 2 * (s.d + 2) * sizeof(float) + (size_t)std::max(4 * n_cu, s.Hkv) * sizeof(PagedCut);
}

hipError_t launch_paged_stream(const Shape& s, const PagedArgs& a, int n_cu, hipStream_t st) {
    if (s.dtype == FR_BF16) return s.d == 128 ? launch<__bf16, 128>(a, n_cu, st) : launch<__bf16, 64>(a, n_cu, st);
    return s.d == 128 ? launch<float, 128>(a, n_cu, st) : launch<float, 64>(a, n_cu, st);
}

}  // namespace fr
