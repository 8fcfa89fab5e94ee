// Attention of a step with trees over a paged cache: bf16 requests with more than a few query columns (some ten to a few hundred drafted tokens' heads), head_dim 64 or 128.
//
// K and V of a request are read once for 256 columns ((row, query head) pairs, the heads of the group fastest): up to there memory is the bound, beyond the matrix
// instructions.  One workgroup of eight waves to a compute unit; a step is 64 keys, of which every wave brings 8 rows global -> LDS (no registers), three steps ahead of
// the one that all work on (96 KB on their way; one step of 128 keys ahead, 64 KB, left a quarter of the memory's rate unused), and a barrier a step is all that they wait for
// one another.  A wave has 32 columns, and all keys of a step where the tile has more than 128 columns, else half of them; the halves' sums meet through LDS at the end of a
// piece.  Work is dealt out as one line of units (steps of a column tile, by what they cost) in equal shares, cut items are joined by a second launch (k_paged.hpp).
//
// S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, keys on the register dimension of S^T and columns on lanes: the accumulators of two 16-key blocks
// are, after conversion, the B operand of the second product.  V^T is read by ds_read_b64_tr_b16, which transposes 4 keys x 16 dims on the way.  Weights go into the second
// product as bf16, as that takes no other type at this rate (half a step, 2^-8, of each; their sum is taken in fp32 before); the output is rounded once.  The root mean square of what is off is 0.0022 of
// the output's for 0.0017 by the output's rounding alone.
//
// Softmax.  Weights are taken with the reference that a column has, before anything is known of the block's logits: the loop holds no maximum.  Where a lane's weights of a step (16, or 8)
// add up to more than 2^8 (the first that a column sees are infinite), the references go up to the largest logits, the sums are scaled and the weights taken again from the
// logits, which are still there.  A wave one of whose references is PAGED_FAR or more rounds the scaled logits before it takes the
// reference from them.
//
// 32 trees of 8 - 64 rows behind 500 - 16900 positions, 32 / 8 heads of 128 (694 MB): 178 us, 3.9 TB/s, joining included; one tree of 24 rows behind 4096 (17 MB): 19.7 us, of which two launches are 8 and the way
// to the first key (lengths -> share -> page -> row) 4; 8 trees of 65 - 255 rows, 28 / 4 heads (30 GFLOP): 70.8 us, 0.43 PFLOP/s.  There a step of 64 keys by 256 columns takes 4700 cycles, of which
// the matrix instructions are 2050 and the vector instructions some 2000 (half of them exponentials): the two waves of a SIMD do the same at the same time, and each of the eight reads all of K and V from LDS for its
// 32 columns.  Setting them apart was slower, us of the same call:
// waves 4 - 7 a phase behind 82; two groups that take turns at the matrix pipe, a barrier between, 79 (64 keys a turn: 2000 cycles for 1024 of products, the others wait) and 81 - 84 (32 keys, what the products read
// fetched beside the exponentials: 700 for 512, but 1200 for the exponentials); two blocks interleaved in one wave 81 (registers spilled).
//
// What a column does not see stays out of it by hand, as a weight of 0 does not take a NaN or an infinity out of a product: keys behind the request's last
// row repeat that one, and values that are not finite leave a block that only some columns see whole and reach those columns when the loop is over.
#include "k_paged.hpp"

#include <algorithm>
#include <type_traits>

namespace fr {

namespace {

constexpr int W = 8, NC = 2, CW = 16 * NC, C = CW * W;   // waves; blocks of 16 columns of a wave; columns of a wave and of a tile
constexpr int KT = 64, RW = KT / W;                      // keys of a step; rows of it that a wave brings
constexpr int RING = 4;                                  // steps in LDS
constexpr int HALF_COST = 3, FULL_COST = 5;              // units of a step of a tile of up to 128 columns, and of more
constexpr int MIN_UNITS = 12;                            // a share smaller than this costs more to write and read as partial results than it saves
static_assert(MIN_UNITS >= FULL_COST, "a step begins in every share");
constexpr int WORDS = FR_TREE_MAX_ROWS / 32;
constexpr float RAISE_SUM = 256.f;                       // a lane's weights of a block: none of them is above 2^8, so sums of them and of values have that much less room than fp32

template <int D>
struct TreeLds {
    static constexpr int TILE = KT * 2 * D, MD = D / 16;
    union {
        struct { unsigned char k[RING][TILE], v[RING][TILE]; };
        struct {   // what two waves, each with a half of the keys, hand over to one another: the sums of one of their blocks of columns
            f32x4 o[W][MD][64];
            float2 ml[W][64];
        };
    };
    uint32_t mask[C][WORDS + 1];   // of the rows that the tile's columns belong to
    int32_t page[W][RING][64];     // page numbers of the rows that a wave is to bring
    int hole[RING][W];             // bit r: row r of the wave's has no page
};

// A piece's slot: [block of 16 columns][D / 16][lane] of four fp32 accumulators, then [column] (exponent reference, base 2, and sum of weights).
template <int D>
constexpr int PART = C * (D + 2);

// A request's tiles, all but the last of 256 columns, and its steps; the line of work has them one after the other.  A step is done by the workgroup that has its first unit.
struct TreeTiles {
    PagedRequest rq;
    int n, steps, last_cost;
    __device__ __forceinline__ int64_t units() const { return rq.n == 0 ? 0 : (int64_t)steps * ((int64_t)(n - 1) * FULL_COST + last_cost); }
};
__device__ __forceinline__ TreeTiles tree_tiles(const PagedArgs& a, int b) {
    TreeTiles t;
    t.rq = paged_tree_request(a, b);
    const int cols = t.rq.n * a.G;   // (below 2^18: 256 rows, 1024 heads)
    t.n = (cols + C - 1) / C;
    t.last_cost = cols - (t.n - 1) * C > C / 2 ? FULL_COST : HALF_COST;
    t.steps = max(paged_position(a, t.rq, t.rq.n - 1), 0) / KT + 1;
    return t;
}
__device__ __forceinline__ int tree_sharers(const PagedArgs& a, int64_t total) { return (int)max((int64_t)1, min((int64_t)a.n_wg, total / MIN_UNITS)); }

template <int D, bool ALIGNED>
struct TreePiece {
    static constexpr int MD = D / 16, NK = D / 32;                // 16-dim blocks of the output; 16-byte vectors of a lane's key (and query) row
    static constexpr int RV = D / 8, COPIES = RW * RV / 64;       // vectors of a row; copies of 1 KB of a wave's rows
    using Lds = TreeLds<D>;
    typedef short __attribute__((ext_vector_type(4))) i16x4;

    // One piece: blocks [r0, r1) of column tile ct of request b.  whole: it is all of the item, the outputs are stored; else the partial result goes to `part`.
    static __device__ __forceinline__ void run(const PagedArgs& a, Lds& sm, const PagedRequest& rq, int b, int ct, int g, int r0, int r1, bool whole, float* part) {
        const int lane = threadIdx.x & 63, x = lane & 15, kg = lane >> 4;
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
        const int G = a.G, cols = rq.n * G, col0 = C * ct, token0 = col0 / G, head0 = col0 - token0 * G;
        auto out_row = [&](int cl) {   // (row, head) of a column, counted over all heads
            const int i = paged_token(a, head0 + cl);
            return (size_t)(rq.first + token0 + i) * a.Hq + g * G + (head0 + cl - i * G);
        };
        const int last_col = min(C, cols - col0) - 1;
        const bool halves = last_col < C / 2;                    // the waves are two groups, each with a half of the keys
        const int half = halves ? wave / (W / 2) : 0, wave0 = CW * (halves ? wave % (W / 2) : wave);   // the wave's first column
        const bool active = wave0 <= last_col;
        u32x4 qf[NC][NK];   // B operand of S^T = K Q^T
        int token[NC];      // the column's row, of those of the tile
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {   // columns past the end: a copy of the last
            const int cl = min(wave0 + 16 * nb + x, last_col);
            const __bf16* p = (const __bf16*)a.q + out_row(cl) * D + 8 * kg;
            token[nb] = paged_token(a, head0 + cl);
#pragma unroll
            for (int ks = 0; ks < NK; ++ks) qf[nb][ks] = *reinterpret_cast<const u32x4*>(p + 32 * ks);
        }
        const int p_first = paged_position(a, rq, -1);            // keys up to here are visible to every column
        const int p_last = paged_position(a, rq, rq.n - 1);       // none beyond to any
        const int end = min((p_last + KT) / KT, r1);              // (none for a request that sees nothing)
        auto visible32 = [&](int nb, int j0) { return paged_visible(sm.mask[token[nb]], a.words, j0 - rq.cached, p_last + 1 - rq.cached); };   // keys j0 .. j0 + 31 to block nb's column
        f32x4 o[MD][NC];   // O^T: row m of product md is dim 16 md + m
        float m[NC], l[NC];
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            m[nb] = PAGED_NO_MAX;
            l[nb] = 0.f;
#pragma unroll
            for (int md = 0; md < MD; ++md) o[md][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int32_t* table = a.block_table + (size_t)b * a.W;
        const uint32_t row_bytes = (uint32_t)(a.Hkv * D * 2);
        const unsigned char *k_base = (const unsigned char*)a.k_pages + (size_t)g * D * 2, *v_base = (const unsigned char*)a.v_pages + (size_t)g * D * 2;
        // A copy brings 64 / RV rows, RV lanes side by side to a row; copy i the rows COPIES q + i of the lanes' groups q, so that a lane's sources are
        // neighbours.  Vector c of row r sits in place c ^ swz(r), so that no two lanes that are served at once meet in a bank: of a key fragment these are rows 0 .. 3 and 12 .. 15 of one quarter
        // of the lanes with rows 4 .. 11 of the next, of a transposing read 32 bytes each of 8 consecutive rows.  (Counted: none; with (r & 7) << 1 | r >> 3 three of ten active cycles were conflicts.)
        auto swz = [](int r) { return (RV >= 16 ? (r & 7) ^ (r >> 3 & 1) << 2 : (r >> 1 & 3) ^ (r >> 3 & 1) << 1) << 1 | (r >> 3 & 1); };
        auto row_at = [](int r) { return COPIES * 1024 * (r / RW) + 1024 * (r % COPIES) + 16 * RV * (r % RW / COPIES); };
        const uint32_t page_lds = paged_lds(sm.page[wave]);
        const int qg = lane / RV, vec = lane % RV;
        const uint32_t place = 16 * (vec ^ swz(RW * wave + COPIES * qg));   // (the row of copy i: exclusive or with swz(i))
        auto is_page = [&](int p) { return (uint32_t)p < (uint32_t)a.n_pages; };
        auto copy_pages = [&](int step) {   // of the wave's rows of a step (eight times over)
            paged_copy4(table + paged_block(a, min(KT * step + RW * wave + (lane & (RW - 1)), p_last)), page_lds + 256 * (step % RING));
        };
        auto copy_rows = [&](int step) {    // the wave's rows of a step
            const int j0 = KT * step + RW * wave + COPIES * qg, buf = step % RING;
            uint32_t row[COPIES];
            int holes = 0;
            if constexpr (ALIGNED) {   // pages are whole multiples of the lane's COPIES rows
                const int page = sm.page[wave][buf][COPIES * qg], jc = min(j0, p_last), in = j0 - jc, base = jc - paged_block(a, jc) * a.P;
                const bool none = !is_page(page);
                const uint32_t at = (uint32_t)(none ? 0 : page) * (uint32_t)a.P + (uint32_t)base;
                const int most = p_last - jc;
#pragma unroll
                for (int i = 0; i < COPIES; ++i) row[i] = at + (uint32_t)min(in + i, most);
                holes = none ? (1 << COPIES) - 1 : 0;
            } else {
#pragma unroll
                for (int i = 0; i < COPIES; ++i) {
                    const int page = sm.page[wave][buf][COPIES * qg + i], j = min(j0 + i, p_last);
                    const bool none = !is_page(page);
                    row[i] = (uint32_t)(none ? 0 : page) * (uint32_t)a.P + (uint32_t)(j - paged_block(a, j) * a.P);
                    holes |= none ? 1 << i : 0;
                }
            }
            const uint32_t k_lds = paged_lds(sm.k[buf]) + COPIES * 1024 * wave, v_lds = paged_lds(sm.v[buf]) + COPIES * 1024 * wave;
#pragma unroll
            for (int i = 0; i < COPIES; ++i) paged_copy16(k_base + (size_t)row[i] * row_bytes + (place ^ (swz(i) * 16u)), k_lds + 1024 * i);
#pragma unroll
            for (int i = 0; i < COPIES; ++i) paged_copy16(v_base + (size_t)row[i] * row_bytes + (place ^ (swz(i) * 16u)), v_lds + 1024 * i);
            int all = 0;
            if (__builtin_expect(__any(holes != 0), 0)) {
#pragma unroll
                for (int q = 0; q < 64 / RV; ++q) all |= __builtin_amdgcn_readlane(holes, q * RV) << (COPIES * q);
            }
            if (lane == 0) sm.hole[buf][wave] = all;
        };
        bool apart = false, far = false;   // far: some column's reference has reached PAGED_FAR
        if (r0 < end) {
            const int last = end - 1;
            const int y = 4 * kg + (x >> 2);   // the lane's key, of 16, in a transposing read
            const uint32_t k_lane = row_at(x) + 16 * (kg ^ swz(x)), v_lane = row_at(y) + 16 * ((x >> 1 & 1) ^ swz(y)) + 8 * (x & 1);
            copy_pages(r0);
            copy_pages(r0 + 1);
            copy_pages(r0 + 2);             // (past the last step: its last rows')
            if (KT * end - 1 > p_first) {   // the step's own rows are among the keys
                const int rows = paged_token(a, head0 + last_col) + 1;
                for (int i = threadIdx.x; i < rows * a.words; i += 64 * W) sm.mask[i / a.words][i % a.words] = a.mask[(size_t)(rq.first + token0) * a.words + i];
            }
            paged_wait_but<0>();            // (nothing that the compiler counts is in flight from here on)
            auto bring = [&](int step) {    // the rows of a step, and the page numbers of three steps further on
                if (step <= last) copy_rows(step);
                copy_pages(step + 3);
            };
#pragma unroll 1
            for (int step = r0; step < r0 + 3; ++step) bring(step);
            // A step's work; NB: its blocks of 16 keys, from `key0` on, that are the wave's.
            auto work = [&](int step, int key0, auto blocks) __attribute__((always_inline)) {
                constexpr int NB = decltype(blocks)::value;
                const int buf = step % RING, j0 = KT * step + key0;
                const unsigned char* kt = sm.k[buf] + row_at(key0);
                const uint32_t vt = paged_lds(sm.v[buf]) + row_at(key0) + v_lane;
                int hole[2 * NB], any_hole = 0;   // (8 rows of a wave each)
#pragma unroll
                for (int i = 0; i < 2 * NB; ++i) any_hole |= hole[i] = sm.hole[buf][key0 / RW + i];
                f32x4 s[NB][NC];
#pragma unroll
                for (int k0 = 0; k0 < NK; k0 += 8 / NB) {   // eight fragments on their way at once: two waves of a SIMD do not hide the LDS's latency
                    u32x4 kf[8 / NB][NB];   // keys j0 + 16 bb + x: elements 32 ks + 8 kg ..
#pragma unroll
                    for (int ks = k0; ks < k0 + 8 / NB && ks < NK; ++ks)
#pragma unroll
                        for (int bb = 0; bb < NB; ++bb) kf[ks - k0][bb] = *reinterpret_cast<const u32x4*>(kt + row_at(16 * bb) + (k_lane ^ (64 * ks)));
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int ks = k0; ks < k0 + 8 / NB && ks < NK; ++ks)
#pragma unroll
                        for (int bb = 0; bb < NB; ++bb)
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb)
                                s[bb][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[ks - k0][bb]), __builtin_bit_cast(bf16x8, qf[nb][ks]),
                                                                                    ks == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[bb][nb], 0, 0, 0);
                }
                any_hole = __builtin_amdgcn_readfirstlane(any_hole);
                const bool partial = j0 + 16 * NB - 1 > p_first || any_hole != 0;   // not every column sees all of these keys
                if (partial) {
#pragma unroll
                    for (int nb = 0; nb < NC; ++nb)
#pragma unroll
                        for (int h = 0; h < NB / 2; ++h) {
                            const uint32_t seen = (visible32(nb, j0 + 32 * h) & ~((uint32_t)hole[4 * h] | (uint32_t)hole[4 * h + 1] << 8 | (uint32_t)hole[4 * h + 2] << 16 | (uint32_t)hole[4 * h + 3] << 24)) >> 4 * kg;
#pragma unroll
                            for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                                for (int v = 0; v < 4; ++v)
                                    if ((seen >> (16 * bb + v) & 1) == 0) s[2 * h + bb][nb][v] = -INFINITY;
                        }
                }
                float scale = a.scale_log2e;
                auto scale_first = [&] {
#pragma clang fp contract(off)
#pragma unroll
                    for (int bb = 0; bb < NB; ++bb)
#pragma unroll
                        for (int nb = 0; nb < NC; ++nb)
#pragma unroll
                            for (int v = 0; v < 4; ++v) s[bb][nb][v] *= scale;
                    scale = 1.f;
                };
                if (__builtin_expect(far, 0)) scale_first();
                u32x4 p[NB / 2][NC];   // weights as the B operand of the second product: slot 4 bb + v of quarter kg is key 32 h + 16 bb + 4 kg + v
                float sum[NC];
#pragma unroll 1
                for (int go = 0; go < 2; ++go) {
                    bool high = false;
#pragma unroll
                    for (int nb = 0; nb < NC; ++nb) {
                        sum[nb] = 0.f;
#pragma unroll
                        for (int bb = 0; bb < NB; ++bb)
#pragma unroll
                            for (int v = 0; v < 4; v += 2) {
                                const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[bb][nb][v], scale, -m[nb]));
                                const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[bb][nb][v + 1], scale, -m[nb]));
                                sum[nb] += p0 + p1;
                                bf16x2 t;
                                t[0] = (__bf16)p0;
                                t[1] = (__bf16)p1;
                                p[bb / 2][nb][2 * (bb % 2) + v / 2] = __builtin_bit_cast(uint32_t, t);
                            }
                        high = high || sum[nb] > RAISE_SUM;
                    }
                    if (__builtin_expect(!__any(high), 1)) break;
                    bool now_far = false;
#pragma unroll
                    for (int nb = 0; nb < NC; ++nb) {
                        float t = s[0][nb][0];
#pragma unroll
                        for (int v = 1; v < 4 * NB; ++v) t = fmaxf(t, s[v / 4][nb][v % 4]);
                        const float up = fmaxf(m[nb], paged_column_max(t) * scale), down = __builtin_amdgcn_exp2f(m[nb] - up);
                        m[nb] = up;
                        l[nb] *= down;
#pragma unroll
                        for (int md = 0; md < MD; ++md) o[md][nb] *= down;
                        now_far = now_far || (fabsf(up) >= PAGED_FAR && up != PAGED_NO_MAX);
                    }
                    if (__builtin_expect(!far && __any(now_far), 0)) {
                        far = true;
                        scale_first();
                    }
                }
#pragma unroll
                for (int nb = 0; nb < NC; ++nb) l[nb] += sum[nb];
#pragma unroll
                for (int h = 0; h < NB / 2; ++h) {
                    bf16x8 vf[MD];   // dim 16 md + x of keys j0 + 32 h + 16 (i / 4) + 4 kg + i % 4
#pragma unroll
                    for (int md = 0; md < MD; ++md) {
                        const auto at = [&](int bb) { return reinterpret_cast<__attribute__((address_space(3))) i16x4*>((uintptr_t)((vt ^ (32u * md)) + row_at(32 * h + 16 * bb))); };
                        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(0)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at(1));
                        vf[md] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                    if (partial) {
                        uint32_t noted = 0;
#pragma unroll
                        for (int md = 0; md < MD; ++md)
#pragma unroll
                            for (int e = 0; e < 4; ++e) paged_note<__bf16>(noted, __builtin_bit_cast(u32x4, vf[md])[e]);
                        if (__builtin_expect(__any(paged_not_finite(noted)), 0)) {   // values that are not finite: not into the product
                            apart = true;
#pragma unroll
                            for (int md = 0; md < MD; ++md) {
                                u32x4 w = __builtin_bit_cast(u32x4, vf[md]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) w[e] = paged_finite_or_zero<__bf16>(w[e]);
                                vf[md] = __builtin_bit_cast(bf16x8, w);
                            }
                        }
                    }
#pragma unroll
                    for (int md = 0; md < MD; ++md)
#pragma unroll
                        for (int nb = 0; nb < NC; ++nb)
                            o[md][nb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf[md], __builtin_bit_cast(bf16x8, p[h][nb]), o[md][nb], 0, 0, 0);
                }
            };
            constexpr int ISSUED = 2 * COPIES + 1;   // copies of a step
            auto steps = [&](int key0, auto blocks) __attribute__((always_inline)) {
#pragma unroll 1
                for (int step = r0; step < end; ++step) {
                    // the wave's rows of this step, and the page numbers of the third one from here; not what was issued behind them
                    if (step + 2 <= last) paged_wait_but<2 * ISSUED>();
                    else if (step + 1 <= last) paged_wait_but<ISSUED + 1>();
                    else paged_wait_but<2>();
                    paged_lds_barrier();    // everybody's; and everybody is done with the step before
                    // (half of the waves, one on each SIMD, bring their rows before they work, the others behind it)
                    if (!active || wave < W / 2) bring(step + 3);
                    if (active) work(step, key0, blocks);
                    if (active && wave >= W / 2) bring(step + 3);
                }
            };
            if (halves) steps(half * (KT / 2), std::integral_constant<int, 2>{});
            else steps(0, std::integral_constant<int, 4>{});
            paged_wait_but<0>();
        }
        if (__builtin_expect(apart, 0)) {   // the values that were left out reach the columns that see them
#pragma unroll 1
            for (int step = r0; step < end; ++step) {
                // (only what the loop left out: blocks that some column does not see whole)
                const int keys = halves ? KT / 2 : KT, j0 = KT * step + half * keys;
                bool partial = j0 + keys - 1 > p_first;
                if (!partial) {
                    for (int i = 0; i < keys; ++i) partial = partial || !is_page(table[paged_block(a, j0 + i)]);
                }
                if (!partial) continue;
#pragma unroll 1
                for (int j = j0; j < j0 + keys && j <= p_last; ++j) {
                    const int page_block = paged_block(a, j), page = table[page_block];
                    if (!is_page(page)) continue;
                    const __bf16* value = (const __bf16*)(v_base + ((size_t)page * a.P + (j - page_block * a.P)) * row_bytes);
                    bool seen[NC];
#pragma unroll
                    for (int nb = 0; nb < NC; ++nb) seen[nb] = (visible32(nb, j) & 1) != 0;
#pragma unroll
                    for (int v = 0; v < 4; ++v)
#pragma unroll
                        for (int md = 0; md < MD; ++md) {
                            const float w = (float)value[16 * md + 4 * kg + v];
                            const float add = (__float_as_uint(w) & 0x7F800000u) == 0x7F800000u ? w : 0.f;
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb) o[md][nb][v] += seen[nb] ? add : 0.f;
                        }
                }
            }
        }
        // ---- the two halves of the keys ------------------------------------------------------------------------------------
        float sum[NC];
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) sum[nb] = paged_column_sum(l[nb]);
        paged_lds_barrier();   // everybody is done with the keys and values
        if (halves) {
            static_assert(NC == 2, "a block for each half");
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                if (!active || nb == half) continue;
                sm.ml[wave][lane] = make_float2(m[nb], sum[nb]);
#pragma unroll
                for (int md = 0; md < MD; ++md) sm.o[wave][md][lane] = o[md][nb];
            }
            paged_lds_barrier();
            const int from = wave ^ (W / 2);
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                if (!active || nb != half) continue;
                const float2 other = sm.ml[from][lane];
                const float up = fmaxf(m[nb], other.x), f0 = __builtin_amdgcn_exp2f(m[nb] - up), f1 = __builtin_amdgcn_exp2f(other.x - up);   // (one that saw nothing: 0, beside one that did)
                m[nb] = up;
                sum[nb] = sum[nb] * f0 + other.y * f1;
#pragma unroll
                for (int md = 0; md < MD; ++md) o[md][nb] = o[md][nb] * f0 + sm.o[from][md][lane] * f1;
            }
        }
        // ---- out with them ---------------------------------------------------------------------------------------------------
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            const int c = wave0 + 16 * nb + x;
            if (c - x > last_col || (halves && nb != half)) continue;   // (wave-uniform)
            if (!whole) {
                const int cb = wave0 / 16 + nb;   // block of 16 columns of the tile
#pragma unroll
                for (int md = 0; md < MD; ++md) reinterpret_cast<f32x4*>(part)[(cb * MD + md) * 64 + lane] = o[md][nb];
                if (kg == 0) reinterpret_cast<float2*>(part + C * D)[c] = make_float2(m[nb], sum[nb]);
                continue;
            }
            if (c > last_col) continue;
            const bool none = sum[nb] == 0.f;   // it saw nothing (one that did has had a weight of about 1 when its reference was last raised)
            const float inv_l = none ? 0.f : 1.0f / sum[nb];
            const size_t oc = out_row(c);
            __bf16* dst = (__bf16*)a.out + oc * D;
#pragma unroll
            for (int md = 0; md < MD; ++md) {
                struct alignas(8) { __bf16 e[4]; } y;
#pragma unroll
                for (int v = 0; v < 4; ++v) y.e[v] = (__bf16)(o[md][nb][v] * inv_l);
                *reinterpret_cast<decltype(y)*>(dst + 16 * md + 4 * kg) = y;
            }
            if (kg == 0 && a.lse != nullptr) a.lse[oc] = none ? -INFINITY : (m[nb] + __builtin_amdgcn_logf(sum[nb])) * 0.6931471805599453f;
        }
        paged_lds_barrier();   // (the next piece's copies overwrite what was handed over, and its masks these)
    }
};

template <int D, bool ALIGNED>
__global__ __launch_bounds__(64 * W) void paged_tree_kernel(const PagedArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    auto& sm = *reinterpret_cast<TreeLds<D>*>(smem_raw);
    const int g = paged_head(a), w = paged_workgroup(a);
    int64_t u = 0, end = 0;
    const PagedLine line = paged_line(a.B, [&](int b) { return tree_tiles(a, b).units(); }, [&](int64_t total) {
        const int n = tree_sharers(a, total);
        if (w >= n || total == 0) return (int64_t)-1;
        u = paged_first_unit(w, total, n);
        end = paged_first_unit(w + 1, total, n);
        return u;
    });
    PagedCut cut{0, 0, 0, 0};
    int64_t start = line.start;   // of the request's units
    for (int b = line.b; b >= 0 && u < end && b < a.B; ++b) {
        const TreeTiles t = tree_tiles(a, b);
        const int64_t units = t.units();
        while (u < end && u < start + units) {
            const int64_t in = u - start, full = (int64_t)t.steps * FULL_COST;
            const int ct = t.n == 1 ? 0 : (int)min(paged_div(in, full), (int64_t)t.n - 1), cost = ct < t.n - 1 ? FULL_COST : t.last_cost;
            const int at = (int)(in - ct * full), upto = (int)min((int64_t)t.steps * cost, at + (end - u));   // units of the tile: below 2^27 (2^24 steps)
            auto steps_before = [&](int unit) { return cost == FULL_COST ? (unit + FULL_COST - 1) / FULL_COST : (unit + HALF_COST - 1) / HALF_COST; };
            const int r0 = steps_before(at), r1 = steps_before(upto);
            const bool whole = r0 == 0 && r1 == t.steps;
            float* part = paged_slot(a, w, g, r0 > 0 ? 0 : 1, PART<D>);
            if (r0 == 0 && !whole)
                cut = PagedCut{paged_owner(u - at + (int64_t)(t.steps - 1) * cost, line.total, tree_sharers(a, line.total)) - w + 1, t.rq.first, C * ct, t.rq.n * a.G};
            if (r0 < r1) TreePiece<D, ALIGNED>::run(a, sm, t.rq, b, ct, g, r0, r1, whole, part);
            u += upto - at;
        }
        start += units;
    }
    if (threadIdx.x == 0) paged_cuts(a)[(size_t)w * a.Hkv + g] = cut;
}

// Joins the pieces of the items that fell to several workgroups, in their order: blockIdx.x = workgroup x Hkv + KV head, whose cut it sees to; blockIdx.y: a block of 16
// columns.  A lane holds the accumulators that it would in the kernel above, a wave a quarter of the value products; eight pieces in one trip to memory.
template <int D>
__global__ __launch_bounds__(256) void paged_tree_join_kernel(const PagedArgs a) {
    constexpr int MD = D / 16, MW = MD / 4, AHEAD = 8;
    const int g = blockIdx.x % a.Hkv, w0 = blockIdx.x / a.Hkv;
    const PagedCut cut = paged_cuts(a)[blockIdx.x];
    const int n = cut.pieces, cb = blockIdx.y, cols = min(C, cut.cols - cut.col0);
    if (n == 0 || 16 * cb >= cols) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, x = lane & 15, kg = lane >> 4;
    float top = PAGED_NO_MAX, l = 0.f;
    f32x4 o[MW] = {};
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        float2 ml[AHEAD];
        f32x4 po[AHEAD][MW];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {   // (past the end: the last piece, which does not count)
            const int i = min(i0 + k, n - 1);
            const float* p = paged_slot(a, w0 + i, g, i == 0 ? 1 : 0, PART<D>);
            ml[k] = reinterpret_cast<const float2*>(p + C * D)[16 * cb + x];
#pragma unroll
            for (int md = 0; md < MW; ++md) po[k][md] = reinterpret_cast<const f32x4*>(p)[(cb * MD + MW * wave + md) * 64 + lane];
        }
        float up = top;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) up = i0 + k < n ? fmaxf(up, ml[k].x) : up;
        const float f = __builtin_amdgcn_exp2f(top - up);
        top = up;
        l *= f;
#pragma unroll
        for (int md = 0; md < MW; ++md) o[md] *= f;
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= n) continue;
            const float w = __builtin_amdgcn_exp2f(ml[k].x - top);
            l += ml[k].y * w;
#pragma unroll
            for (int md = 0; md < MW; ++md) o[md] += po[k][md] * w;
        }
    }
    const int c = 16 * cb + x;
    if (c >= cols) return;
    const int col = cut.col0 + c, i = paged_token(a, col);
    const size_t oc = (size_t)(cut.first_row + i) * a.Hq + g * a.G + (col - i * a.G);
    const bool none = l == 0.f;
    const float inv_l = none ? 0.f : 1.0f / l;
#pragma unroll
    for (int md = 0; md < MW; ++md) {
        struct alignas(8) { __bf16 e[4]; } y;
#pragma unroll
        for (int v = 0; v < 4; ++v) y.e[v] = (__bf16)(o[md][v] * inv_l);
        *reinterpret_cast<decltype(y)*>((__bf16*)a.out + oc * D + 16 * (MW * wave + md) + 4 * kg) = y;
    }
    if (wave == 0 && kg == 0 && a.lse != nullptr) a.lse[oc] = none ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, bool ALIGNED>
hipError_t launch(const PagedArgs& a, int cols, hipStream_t st) {
    using Lds = TreeLds<D>;
    static_assert(sizeof(Lds) <= 160 * 1024, "LDS of a compute unit");
    // Raises the kernel's dynamic LDS limit, once per process.
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_tree_kernel<D, ALIGNED>), hipFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Lds));
    if (once != hipSuccess) return once;
    paged_tree_kernel<D, ALIGNED><<<dim3(paged_grid(a.n_wg, a.Hkv)), dim3(64 * W), sizeof(Lds), st>>>(a);
    if (a.n_wg > 1 && a.cap > KT)   // (else every item is one unit, and none is cut)
        paged_tree_join_kernel<D><<<dim3((unsigned)((a.n_wg - 1) * a.Hkv), (unsigned)((cols + 15) / 16)), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const PagedArgs& args, int n_cu, hipStream_t st) {
    PagedArgs a = args;
    a.n_wg = std::max(1, n_cu / a.Hkv);
    const int cols = (int)std::min<int64_t>((int64_t)a.max_new * a.G, C);
    if constexpr (TreePiece<D, true>::COPIES > 1) {
        if (a.P % TreePiece<D, true>::COPIES != 0) return launch<D, false>(a, cols, st);
    }
    return launch<D, true>(a, cols, st);
}

}  // namespace

size_t paged_tree_partials_bytes(const Shape& s, int n_cu) {
    // (one workgroup per KV head, where there are more of those than workgroups: nothing is cut)
    return (size_t)n_cu * 2 * C * (s.d + 2) * sizeof(float) + (size_t)std::max(n_cu, s.Hkv) * sizeof(PagedCut);
}

hipError_t launch_paged_tree(const Shape& s, const PagedArgs& a, int n_cu, hipStream_t st) { return s.d == 128 ? launch<128>(a, n_cu, st) : launch<64>(a, n_cu, st); }

}  // namespace fr
