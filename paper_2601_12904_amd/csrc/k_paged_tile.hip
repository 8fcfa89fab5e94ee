// Attention over a paged cache, requests with many query columns (chunks of prompts, whole prompts): bf16, head_dim 64 or 128.
//
// One workgroup owns one KV head and a tile of 256 query columns ((row, query head) pairs, the heads of the group fastest) in four row groups of 64; eight
// waves, two per row group and per SIMD, of which the first takes keys 0..31 of every tile of 64 keys and the second keys 32..63, each with output
// accumulators of its own, which are added up at the end.  S^T = K Q^T and O^T = V^T P^T with v_mfma_f32_16x16x32_bf16, keys on the register
// dimension of S^T, columns on lanes: the accumulators of two 16-key blocks are, after conversion, the B operand of the second product.
//
// Keys and values come straight from the pages, global -> LDS without registers: a wave brings eight consecutive rows of each tile, so in pages of a multiple of
// eight rows their address is the same for the whole wave (scalar registers), and one table entry per wave and tile, itself copied to LDS two tiles
// ahead, is all the look-up there is.  Rows lie in LDS as they do in memory, the 16-byte vectors of row r permuted by an exclusive or with r (the lanes ask for them
// in that order), so that the rows of a fragment lie in different banks: K by 16-byte reads, V^T by ds_read_b64_tr_b16, which
// transposes 4 keys x 16 dims on the way.  (Counted: a quarter of the LDS's active cycles are still conflicts, 260 of 1105 per tile; the loop over packed images has 6 of 665.)  So no pass packs or transposes anything in front: a chunk of 2048 rows behind 14336 would read, write and read
// again 67 MB for it.
//
// A wave alternates between a matrix phase (O += its half of tile kt - 1, logits of its half of tile kt) and a softmax phase; the two waves of a SIMD do so in turn,
// so that the vector work of one runs beside the matrix instructions of the other:
//   waves 0..3   barrier kt | matrix (kt - 1, kt) | copies kt | softmax kt
//   waves 4..7   barrier kt | softmax kt - 1 | copies kt | matrix (kt - 1, kt)
// (copies of all waves at once, behind the barrier, hold the softmax up: 1000 cycles for five of them each, 440 apart).
//
// Softmax.  exp(x - m) / sum exp(x - m) does not depend on m, and fp32 and bf16 leave about 2^127 of room, so a column's exponent reference is the maximum over its
// visible ones of the request's keys 0..31, in every piece of its item, and the loop holds no maximum, no comparison and no rescaling (which would
// spill registers).  Where the sums show that a later logit passed it by more than that, or where it is PAGED_FAR or more, the piece is done again with the largest logit of its own
// keys, found in a pass over them that forms nothing but logits.  Weights go into the second product as bf16 (half a step, 2^-8, of each; their sum is
// taken in fp32 before), as the output does.
//
// Bound by how well the loop feeds the matrix pipes: of 3450 cycles of a compute unit per tile of 64 keys (2048 rows behind 14336, everything counted; 3680 for 16896 from nothing) 2048 are matrix
// instructions of each SIMD, 59 and 56 %.  2048 rows behind 14336 (32 / 8 heads, head_dim 128) 441 us = 1.17 PFLOP/s, 16896 from nothing 2020 us = 1.16; this library's prefill over a cache
// of its own, which packs tile images first and then takes V by 16-byte reads and one of four query steps from LDS, does the same product in 1750 us with the packing, pipes busy 71 %.  An item takes
// 17 us beside its tiles: plan, queries and page numbers 9, first copies and references 3, exchange and output 5.
//
// What a column does not see stays out of it by hand, as a weight of 0 does not take a NaN or an infinity out of a product: keys behind the tile's last row
// repeat that one; a value that is not finite and that some column does not see makes that one's sums NaN, and in the second go the wave that brought a
// row of such a tile takes values that are not finite out of LDS; they reach the columns that see them when the loop is over.
#include "k_paged.hpp"

#include <algorithm>

namespace fr {

namespace {

constexpr int WAVES = 8, RG = 4, KT = 64, NC = 4;   // waves; row groups; keys of a tile; blocks of 16 columns of a row group
constexpr int C = 64 * RG;                          // columns of a tile
constexpr int RW = KT / WAVES;                      // rows of a tile that a wave brings
constexpr int TILE0 = 8;                            // ring slot of tile 0's page numbers; the others: tile % 8
constexpr int ITEM_KEYS = 512;                      // what a piece costs beside its keys, in keys, a tile of 64 being 1.5 us: 12 of the 17 us above (the plan comes once for a workgroup)
constexpr int MIN_SHARE = 1024;                     // a share smaller than this costs more to write and read as partial results than it saves

typedef short __attribute__((ext_vector_type(4))) i16x4;
typedef const bf16x8 __attribute__((address_space(3)))* lds_b128;

template <int D>
struct __attribute__((aligned(16))) TileLds {
    static constexpr int ROW = 2 * D, TILE = KT * ROW;
    static constexpr int NK = D / 32, MD = D / 16;            // matrix steps over the dims of a logit, 16-dim blocks of the output
    static constexpr int QR = 2, QL = NK - QR;                // matrix steps whose query fragments stay in registers; those that come from LDS
    unsigned char k[3][TILE], v[3][TILE];                     // rings
    unsigned char q[QL > 0 ? RG * QL * NC * 1024 : 16];
    int pos[RG][64];                                          // positions of the columns (masked tiles)
    int page[WAVES][9][64];                                   // page numbers of the rows that a wave is to bring, per tile
    unsigned char hole[8][8];                                 // per tile and wave: bit r = its row r has no page (EXACT)
    float ref[WAVES][64];                                     // the waves' largest logits (EXACT)
    int apart;
};
template <int D>
constexpr int EXCHANGE_WAVE = D / 32 * NC * 1024 + 1024;      // half of a wave's accumulators, and its sums
template <int D>
constexpr size_t references_at() {   // behind everything: the columns' exponent references (registers would spill)
    constexpr size_t a = sizeof(TileLds<D>), b = (size_t)WAVES * EXCHANGE_WAVE<D>, c = (size_t)RG * 64 * (D + 8) * 2;
    return a > b ? (a > c ? a : c) : (b > c ? b : c);
}
template <int D>
constexpr size_t tile_lds_bytes() { return references_at<D>() + C * sizeof(float) + 2 * WAVES * sizeof(int); }   // and the waves' answers to two questions

// ---- how the work is dealt out --------------------------------------------------------------------------
// The cost of a column tile in keys: what its last row sees, about (the line of work only has to be the same for everybody), and what every item takes.
struct TileCosts {
    int64_t base;   // tile t: base + (t + 1) step
    int step, n_ct;
    __device__ __forceinline__ int64_t tile(int t) const { return base + (int64_t)(t + 1) * step; }
    __device__ __forceinline__ int64_t before(int t) const { return t * base + (int64_t)step * ((int64_t)t * (t + 1) / 2); }   // of tiles 0 .. t - 1
    __device__ __forceinline__ int tile_at(int64_t v) const {   // the tile that unit v falls into
        const double s = (double)step, h = (double)base + 0.5 * s;
        int t = (int)((__builtin_sqrt(h * h + 2.0 * s * (double)v) - h) / s);
        t = max(0, min(t, n_ct - 1));
        while (t > 0 && before(t) > v) --t;
        while (t + 1 < n_ct && before(t + 1) <= v) ++t;
        return t;
    }
};
__device__ __forceinline__ TileCosts tile_costs(const PagedArgs& a, const PagedRequest& r) {
    TileCosts c;
    c.base = (int64_t)max(0, min(r.cached, a.cap)) + KT + ITEM_KEYS;
    c.step = (C + a.G - 1) / a.G;
    c.n_ct = (int)(((int64_t)r.n * a.G + C - 1) / C);
    return c;
}

struct TilePlan {
    bool whole;         // a workgroup per item; else equal shares of the line of work
    int64_t total;      // units of the line
    int sharers;        // workgroups that share it
    int b;              // the request that holds what was looked for, -1: none
    int64_t start;      // its first unit (whole: its first item)
};
// Both ways of dealing: whole items, longest of a request first, which walk the keys of a KV head side by side and share them in the caches; or equal shares.
// Whole where its estimated end (the longest item; the average load and one of the shortest, where there are several items for each workgroup) is no later than that of
// equal shares, which read keys at different places (an eighth) and join pieces (three items' own cost).  us whole : in shares, 32 / 8 heads, rows behind
// positions: 2048 behind 14336 455 : 469, 1024 361 : 267, 512 344 : 178, 64 333 : 76; 2048 behind 4000 197 : 237, 512 137 : 115; 300 behind 1000 66 : 86; from nothing
// 512 49 : 80, 4096 182 : 259, 8192 544 : 713; 2300 behind 4000 280 : 254, 2400 behind 14000 736 : 569; 16 times 40 behind 3000 126 : 117, behind 100 61 : 115.
__device__ __forceinline__ TilePlan tile_plan(const PagedArgs& a, int64_t item, int w) {
    const int lane = threadIdx.x & 63;
    int64_t total = 0, items = 0, cost = 0, most = 0, least = INT64_MAX;
    int n_ct = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        cost = 0;
        n_ct = 0;
        if (b0 + lane < a.B) {
            const PagedRequest r = paged_request(a, b0 + lane);
            if (r.n > 0) {
                const TileCosts c = tile_costs(a, r);
                n_ct = c.n_ct;
                cost = c.before(n_ct);
                most = max(most, c.tile(n_ct - 1));
                least = min(least, c.tile(0));
            }
        }
        const int lanes = min(64, a.B - b0);
        total += uniform64(wave_sum64(cost, lanes));
        items += uniform64(wave_sum64(n_ct, lanes));
    }
    for (int d = 1; d < min(64, a.B); d <<= 1) {
        most = max(most, (int64_t)__shfl_xor(most, d));
        least = min(least, (int64_t)__shfl_xor(least, d));
    }
    most = uniform64(most);
    least = uniform64(least);
    TilePlan p{false, total, 1, -1, 0};
    if (total == 0) return p;
    const int n = p.sharers = (int)max((int64_t)1, min((int64_t)a.n_wg, paged_div(total, MIN_SHARE)));
    const int64_t share = paged_div(total, n);
    const int64_t in_items = items <= n ? most : max(most, share + least);
    p.whole = in_items <= share + (share >> 3) + 3 * ITEM_KEYS;
    const int64_t u = p.whole ? item : paged_first_unit(w, total, n);
    if (p.whole ? u >= items : w >= n) return p;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        if (a.B > 64) {
            cost = 0;
            n_ct = 0;
            if (b0 + lane < a.B) {
                const PagedRequest r = paged_request(a, b0 + lane);
                if (r.n > 0) {
                    const TileCosts c = tile_costs(a, r);
                    n_ct = c.n_ct;
                    cost = c.before(n_ct);
                }
            }
        }
        const int64_t mine = p.whole ? n_ct : cost, upto = p.start + wave_scan64(mine, min(64, a.B - b0));
        const uint64_t beyond = __ballot(upto > u);
        if (beyond != 0) {
            const int l = __builtin_ctzll(beyond);
            p.b = b0 + l;
            p.start = uniform64(__shfl(upto, l)) - uniform64(__shfl(mine, l));
            return p;
        }
        p.start = uniform64(__shfl(upto, 63));
    }
    return p;
}

__device__ __forceinline__ f32x4 mfma(const bf16x8& a, const bf16x8& b, const f32x4& c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// A barrier (for LDS), and whether any thread says v; uniform in the compiler's eyes too (what lies behind a divergent branch keeps its registers through the other side).
__device__ __forceinline__ bool any_of_workgroup(bool v, int* answers) {
    const bool any = __any(v);
    if ((threadIdx.x & 63) == 0) answers[threadIdx.x >> 6] = any ? 1 : 0;
    paged_lds_barrier();
    int all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all |= answers[w];
    return __builtin_amdgcn_readfirstlane(all) != 0;
}

// A column tile of a request, and what a lane knows of its columns.
template <int D>
struct TileItem {
    int first_row;                 // the request's first row
    int g, col0, head0, token0;    // first column; its head within the group and its row within the request
    int cols, p_first, p_last;     // columns of the request; keys up to p_first are visible to every column, none beyond p_last to any
    __device__ __forceinline__ void init(const PagedArgs& a, const PagedRequest& r, int t, int g_) {
        g = g_;
        first_row = r.first;
        cols = r.n * a.G;
        col0 = C * t;
        token0 = col0 / a.G;
        head0 = col0 - token0 * a.G;
        p_first = paged_position(a, r, token0);
        p_last = paged_position(a, r, min((int64_t)col0 + C, (int64_t)cols) == cols ? r.n - 1 : (col0 + C - 1) / a.G);
    }
    // column cl of the tile (past the end: the request's last): row within the request and head within the group
    __device__ __forceinline__ void column(const PagedArgs& a, int cl, int* token, int* head) const {
        const int c = head0 + min(cl, cols - 1 - col0), i = paged_token(a, c);
        *token = token0 + i;
        *head = c - i * a.G;
    }
    __device__ __forceinline__ size_t out_row(const PagedArgs& a, int cl) const {
        int token, head;
        column(a, cl, &token, &head);
        return (size_t)(first_row + token) * a.Hq + g * a.G + head;
    }
};

// One matrix phase: O^T += V^T P^T for the wave's half of one tile, S^T = K Q^T for its half of another.  tv, tk: LDS addresses of the lane's first fragments.
// Fragments are requested PF steps of four matrix instructions ahead.
// m: the columns' references, for the softmax phase behind it.
template <int D, bool PV>
__device__ __forceinline__ void matrix_phase(uint32_t tv, uint32_t tk, const bf16x8 (&qf)[NC][TileLds<D>::QR], uint32_t q_lds, const u32x4 (&p)[NC],
                                             f32x4 (&o)[D / 16][NC], f32x4 (&s)[2][NC], uint32_t ref_lds, f32x4& m) {
    using L = TileLds<D>;
    constexpr int NK = L::NK, MD = L::MD, PF = 5, QR = L::QR, FIRST = PV ? 0 : MD, STEPS = MD + 2 * NK, BLOCK = 16 * L::ROW;
    auto dims = [](int j) { return QR < NK ? (j & 1 ? j / 2 : QR + j / 2) : j; };   // order of the dims: LDS, registers, LDS, registers
    bf16x8 fr[PF + 1], qb[2][NC];
    const lds_b128 q_frag = reinterpret_cast<lds_b128>((uintptr_t)q_lds);
    auto frag = [&](int i) -> bf16x8 {
        if (i < MD) {
            const auto at = reinterpret_cast<__attribute__((address_space(3))) i16x4*>((uintptr_t)(tv ^ (32u * i)));
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(at + BLOCK / 8);
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        return reinterpret_cast<lds_b128>((uintptr_t)(tk ^ (64u * dims((i - MD) / 2))))[(i & 1) * BLOCK / 16];
    };
    auto load_q = [&](int j) {   // query fragments of the j-th step of the dims, if they are in LDS
        const int ks = dims(j);
        if (ks < QR) return 0;
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) qb[j & 1][nb] = q_frag[((ks - QR) * NC + nb) * 64];
        return NC;
    };
    int reads[STEPS] = {};   // LDS reads issued in front of step i's products
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int i = FIRST; i < FIRST + PF; ++i) fr[i % (PF + 1)] = frag(i);
    if (!PV) reads[FIRST] += load_q(0);
#pragma unroll
    for (int i = FIRST; i < STEPS; ++i) {
        if (i + PF < STEPS) {
            fr[(i + PF) % (PF + 1)] = frag(i + PF);
            reads[i] += i + PF < MD ? 2 : 1;
        }
        if (PV && i == MD - 2) reads[i] += load_q(0);   // two steps ahead
        if (i >= MD && (i - MD) % 2 == 0 && (i - MD) / 2 + 1 < NK) reads[i] += load_q((i - MD) / 2 + 1);
        if (PV && i == STEPS - 3) {
            m = *reinterpret_cast<const f32x4 __attribute__((address_space(3)))*>((uintptr_t)ref_lds);
            ++reads[i];
        }
        const bf16x8 f = fr[i % (PF + 1)];
        if (i < MD) {
#pragma unroll
            for (int c = 0; c < NC; ++c) {   // (back and forth: neighbours in time share an operand, which saves power)
                const int nb = i & 1 ? NC - 1 - c : c;
                o[i][nb] = mfma(f, __builtin_bit_cast(bf16x8, p[nb]), o[i][nb]);
            }
        } else {
            const int j = (i - MD) / 2, ks = dims(j), b = i & 1;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                const int nb = b ? NC - 1 - c : c;
                s[b][nb] = mfma(f, ks < QR ? qf[nb][ks < QR ? ks : 0] : qb[j & 1][nb], j == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[b][nb]);
            }
        }
    }
    __builtin_amdgcn_sched_group_barrier(0x100, PV ? 2 * PF : PF, 0);
#pragma unroll
    for (int i = FIRST; i < STEPS; ++i) {
        if (reads[i] == 1) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        if (reads[i] == 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        if (reads[i] == NC) __builtin_amdgcn_sched_group_barrier(0x100, NC, 0);
        if (reads[i] == NC + 1) __builtin_amdgcn_sched_group_barrier(0x100, NC + 1, 0);
        if (reads[i] == NC + 2) __builtin_amdgcn_sched_group_barrier(0x100, NC + 2, 0);
        __builtin_amdgcn_sched_group_barrier(0x008, NC, 0);
    }
    __builtin_amdgcn_s_setprio(0);
    __builtin_amdgcn_sched_barrier(0);
}

// Key tiles [kb, ke) of an item.  whole: they are all it has, the outputs are stored; else the partial result goes to `part`: [C][2] references and sums,
// then [C][D] weighted values.
// EXACT = false: returns false where the sums overflowed the reference or are NaN, where the reference is far from 0, or where keys 0..31 have none; what it stored is worth nothing then, and the caller does
// the piece again with EXACT = true.
template <int D, bool ALIGNED, bool EXACT>
__device__ __forceinline__ bool process_piece(const PagedArgs& a, const PagedRequest& rq, int b, int t, int g, int kb, int ke, bool whole, float* part,
                                              unsigned char* smem_raw) {
    using L = TileLds<D>;
    constexpr int NK = L::NK, MD = L::MD, QR = L::QR, QL = L::QL, ROW = L::ROW, TILE = L::TILE;
    constexpr int RV = D / 8, RC = 64 / RV, COPIES = RW / RC;   // vectors of a row; rows of a copy; copies of a wave, of a tile's keys or values
    L& sm = *reinterpret_cast<L*>(smem_raw);
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));   // (opaque: what is formed from it again later need not be kept meanwhile)
    const int lane = tid & 63, x = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), group = wave & 3, second = wave >> 2;
    TileItem<D> it;
    it.init(a, rq, t, g);
    const int p_last = it.p_last;
    const bool empty = kb >= ke;   // nothing to see, or no tile of a small item falls to this piece
    if (empty && !whole) {
        if (tid < C) { part[2 * tid] = PAGED_NO_MAX; part[2 * tid + 1] = 0.f; }
        return true;
    }
    const uint32_t k_base = paged_lds(sm.k[0]), v_base = paged_lds(sm.v[0]);
    const uint32_t q_lds = paged_lds(sm.q) + group * (QL * NC * 1024) + lane * 16u;
    bf16x8 qf[NC][QR], ql[2][QL > 0 ? QL : 1];
#pragma unroll
    for (int nb = 0; nb < NC; ++nb) {
        const __bf16* p = (const __bf16*)a.q + it.out_row(a, 64 * group + 16 * nb + x) * D + 8 * kg;
#pragma unroll
        for (int ks = 0; ks < QR; ++ks) qf[nb][ks] = *reinterpret_cast<const bf16x8*>(p + 32 * ks);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {   // the two waves of a row group bring two column blocks' each to LDS
        const __bf16* p = (const __bf16*)a.q + it.out_row(a, 64 * group + 16 * (2 * second + i) + x) * D + 8 * kg;
#pragma unroll
        for (int ks = 0; ks < QL; ++ks) ql[i][ks] = *reinterpret_cast<const bf16x8*>(p + 32 * (QR + ks));
    }
    auto store_q = [&] {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int ks = 0; ks < QL; ++ks)
                *reinterpret_cast<bf16x8 __attribute__((address_space(3)))*>((uintptr_t)(q_lds + (ks * NC + 2 * second + i) * 1024)) = ql[i][ks];
    };
    if (!second) {
        int token, head;
        it.column(a, 64 * group + lane, &token, &head);
        sm.pos[group][lane] = paged_position(a, rq, token);
    }
    if (tid == 0) sm.apart = 0;

    // ---- copies --------------------------------------------------------------------------------------------
    const int32_t* table = a.block_table + (size_t)b * a.W;
    const uint32_t row_bytes = (uint32_t)(a.Hkv * D * 2);
    const unsigned char *k_pages = (const unsigned char*)a.k_pages + (size_t)g * ROW, *v_pages = (const unsigned char*)a.v_pages + (size_t)g * ROW;
    const uint64_t page_bytes = (uint64_t)(uint32_t)a.P * row_bytes;
    const uint32_t page_lds = paged_lds(sm.page[wave]);
    auto is_page = [&](int p) { return (uint32_t)p < (uint32_t)a.n_pages; };
    const int last = max(ke - 1, 0);   // (past the piece's last tile the copies repeat that one: the counts of the waits stay the same, and nobody reads them)
    auto copy_pages = [&](int kt, int slot) {    // page numbers of the wave's rows of tile kt (aligned pages: one, in every lane)
        const int j = KT * min(kt, last) + RW * wave;
        if constexpr (ALIGNED)
            paged_copy4(paged_uniform((const unsigned char*)(table + paged_block(a, min(j, p_last)))), 0u, page_lds + 256 * slot);
        else
            paged_copy4(table + paged_block(a, min(j + (lane & (RW - 1)), p_last)), page_lds + 256 * slot);
    };
    // Where the wave's rows of a tile are.  Aligned pages: the first one, the same for all lanes, and how many rows there are behind it up to the last visible
    // one (those behind that repeat it); else the row of each copy's lane.
    struct Rows {
        uint64_t at;
        int most;
        uint32_t row[ALIGNED ? 1 : COPIES];
    };
    // Place of vector v of row r: v ^ swz(r).  The 16 rows of a K fragment meet in no bank, and neither do the 32-byte pieces that a transposing read
    // takes from 8 consecutive rows.
    auto swz = [](int r) { return D == 128 ? (r & 7) << 1 | (r >> 3 & 1) : (r >> 1 & 3) << 1 | (r >> 3 & 1); };
    const int lr = lane / RV, lv = lane % RV;   // row of the lane within a copy, place of its vector
    auto lane_vec = [&](int c) { return 16u * (uint32_t)(lv ^ swz(RW * wave + RC * c + lr)); };
    const uint32_t lane_off = (uint32_t)lr * row_bytes + lane_vec(0);   // (copy 1: rows RC .. of the eight, whose vectors are permuted by 8 more)
    static_assert(COPIES == 1 || (COPIES == 2 && RC == 4), "swz(r + 4) = swz(r) ^ 8");
    auto find_rows = [&](int kt, int slot) {
        Rows r;
        const int j0 = KT * min(kt, last) + RW * wave;
        int holes;
        if constexpr (ALIGNED) {
            const int page = __builtin_amdgcn_readfirstlane(sm.page[wave][slot][0]), jc = min(j0, p_last);
            holes = !EXACT || is_page(page) ? 0 : (1 << RW) - 1;   // (else the piece has none)
            r.at = (uint64_t)(uint32_t)(holes ? 0 : page) * page_bytes + (uint64_t)(uint32_t)(jc - paged_block(a, jc) * a.P) * row_bytes;
            r.most = j0 > p_last ? 0 : p_last - jc;
        } else {
            const int mine = sm.page[wave][slot][lane & (RW - 1)];
            holes = (int)(__ballot(!is_page(mine)) & ((1 << RW) - 1));
#pragma unroll
            for (int c = 0; c < COPIES; ++c) {
                const int i = RC * c + lr, page = sm.page[wave][slot][i], j = min(j0 + i, p_last);
                r.row[c] = (uint32_t)(is_page(page) ? page : 0) * (uint32_t)a.P + (uint32_t)(j - paged_block(a, j) * a.P);
            }
        }
        if (EXACT && lane == 0) sm.hole[slot & 7][wave] = (unsigned char)holes;
        return r;
    };
    auto copy_rows = [&](const Rows& r, const unsigned char* pages, uint32_t lds) {
        if constexpr (ALIGNED) {
            const unsigned char* src = pages + r.at;
            const uint32_t to = lds + RW * wave * ROW;
            if (__builtin_expect(r.most >= RW - 1, 1)) {
                paged_copy16(src, lane_off, to);
                if constexpr (COPIES == 2) paged_copy16(src + RC * row_bytes, lane_off ^ 128u, to + 1024);
            } else {
#pragma unroll
                for (int c = 0; c < COPIES; ++c) paged_copy16(src, (uint32_t)min(RC * c + lr, r.most) * row_bytes + lane_vec(c), to + 1024 * c);
            }
        } else {
#pragma unroll
            for (int c = 0; c < COPIES; ++c) paged_copy16(pages + (size_t)r.row[c] * row_bytes + lane_vec(c), lds + (RW * wave + RC * c) * ROW);
        }
    };
    f32x4 o[MD][NC], s[2][NC];
    u32x4 p[NC];
    float l[NC];
    float* refs = reinterpret_cast<float*>(smem_raw + references_at<D>()) + 64 * group + 4 * x;   // of the lane's four columns
    const uint32_t ref_lds = paged_lds(smem_raw + references_at<D>()) + 256 * group + 16 * x;
    int* answers = reinterpret_cast<int*>(smem_raw + references_at<D>() + C * sizeof(float));
    f32x4 m;
    const int n_plain = (it.p_first + 1) / KT;   // leading tiles whose keys are visible to every column
    if (!empty) {
        const uint32_t tk0 = k_base + x * ROW + 16 * (kg ^ swz(x)), tk = tk0 + 32 * second * ROW;
        const int y = 4 * kg + (x >> 2);        // the lane's key of a transposing read
        const uint32_t tv = v_base + 32 * second * ROW + y * ROW + 16 * ((x >> 1 & 1) ^ swz(y)) + 8 * (x & 1);
        int c0, c1, c2;     // ring slots (their bytes) of tiles kt, kt + 1, kt + 2
        Rows next;          // of the tile whose values are to be copied next
        auto copy_first = [&](bool values) {   // K tiles kb and kb + 1 and V tile kb
            const Rows r0 = find_rows(kb, kb & 7);
            copy_rows(r0, k_pages, k_base);
            if (values) copy_rows(r0, v_pages, v_base);
            next = find_rows(kb + 1, (kb + 1) & 7);
            copy_rows(next, k_pages, k_base + TILE);
            c0 = 0; c1 = TILE; c2 = 2 * TILE;
        };
        auto prime = [&](bool values) {   // the same with the page numbers, up to those of tile kb + 4, in front
            paged_wait_but<0>();   // (nothing that the compiler counts is in flight from here on)
#pragma unroll
            for (int i = 0; i < 5; ++i) copy_pages(kb + i, (kb + i) & 7);
            paged_wait_but<3>();
            copy_first(values);
        };
        auto mask = [&](int kt, uint32_t hole) {   // hole: bits of the wave's 32 keys
            int ln = lane;
            asm volatile("" : "+v"(ln));
            const int quarter = ln >> 4, key0 = KT * kt + 32 * second + 4 * quarter;
            const uint32_t mine = hole >> (4 * quarter);   // bits 16 bb + v
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                const int pos = sm.pos[group][16 * nb + (ln & 15)];
#pragma unroll
                for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        if (key0 + 16 * bb + v > pos || (mine >> (16 * bb + v) & 1)) s[bb][nb][v] = -INFINITY;
                __builtin_amdgcn_sched_barrier(0);   // (block by block: the results of all comparisons at once take registers that the loop needs)
            }
        };
        auto holes_of = [&](int kt, uint32_t* mine) {   // does the tile have any, and which of the wave's 32 keys
            const uint64_t hole = *reinterpret_cast<const uint64_t*>(sm.hole[kt & 7]);
            const uint32_t lo = __builtin_amdgcn_readfirstlane((int)(uint32_t)hole), hi = __builtin_amdgcn_readfirstlane((int)(hole >> 32));
            *mine = second ? hi : lo;
            return (lo | hi) != 0;
        };
        auto plain_barrier = [] {   // without the fences of __syncthreads(): the waits are explicit
            asm volatile("" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        if constexpr (EXACT) {   // the maximum of its logits over the piece's visible keys
            f32x4 top = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            store_q();
            prime(false);
            paged_wait_but<0>();
            __syncthreads();
            for (int kt = kb; kt < ke; ++kt) {   // K tiles kt and kt + 1 are in ring slots, kt + 2 follows
                const Rows after = find_rows(kt + 2, (kt + 2) & 7);
                copy_rows(after, k_pages, k_base + c2);
                copy_pages(kt + 5, (kt + 5) & 7);
                matrix_phase<D, false>(0, tk + c0, qf, q_lds, p, o, s, ref_lds, m);
                uint32_t hole;
                if (holes_of(kt, &hole) || kt >= n_plain) mask(kt, hole);
#pragma unroll
                for (int nb = 0; nb < NC; ++nb)
#pragma unroll
                    for (int v = 0; v < 4; ++v) top[nb] = fmaxf(top[nb], fmaxf(s[0][nb][v], s[1][nb][v]));
                paged_wait_but<COPIES + 1>();          // all but the newest tile
                __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0): the wave's own reads and writes
                plain_barrier();
                const int c = c0;
                c0 = c1; c1 = c2; c2 = c;
            }
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                top[nb] = paged_column_max(top[nb]);
                if (kg == 0) sm.ref[wave][16 * nb + x] = top[nb];
            }
            paged_wait_but<0>();
            __syncthreads();
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                const float t = fmaxf(top[nb], sm.ref[wave ^ 4][16 * nb + x]);
                if (!second && kg == 0) refs[nb] = fmaxf(t * a.scale_log2e, PAGED_NO_MAX);
            }
            prime(true);
#pragma unroll
            for (int i = 0; i < TILE / (64 * WAVES * 16); ++i)
                *reinterpret_cast<u32x4*>(sm.v[2] + (i * 64 * WAVES + tid) * 16) = u32x4{0u, 0u, 0u, 0u};
            paged_wait_but<0>();
            __syncthreads();
        } else {   // the maximum over the visible ones of keys 0..31
            // (positions without a page, in tile 0 or in the piece: EXACT sees to them)
            copy_pages(0, TILE0);
#pragma unroll
            for (int i = 0; i < 5; ++i) copy_pages(kb + i, (kb + i) & 7);
            bool none = tid <= min(KT - 1, p_last) && !is_page(table[paged_block(a, min(tid, p_last))]);
            for (int i = paged_block(a, KT * kb) + tid; i <= paged_block(a, min(KT * ke - 1, p_last)); i += 64 * WAVES) none = none || !is_page(table[i]);
            store_q();
#pragma unroll
            for (int i = 0; i < TILE / (64 * WAVES * 16); ++i)   // V ring slot 2 holds zeros for the matrix phase in front
                *reinterpret_cast<u32x4*>(sm.v[2] + (i * 64 * WAVES + tid) * 16) = u32x4{0u, 0u, 0u, 0u};
            paged_wait_but<0>();   // (nothing that the compiler counts is in flight from here on)
            if (any_of_workgroup(none, answers)) return false;
            copy_rows(find_rows(0, TILE0), k_pages, k_base + 2 * TILE);
            copy_first(true);
            paged_wait_but<0>();
            paged_lds_barrier();
            matrix_phase<D, false>(0, tk0 + 2 * TILE, qf, q_lds, p, o, s, ref_lds, m);
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                const int pos = sm.pos[group][16 * nb + x];
                float t = -INFINITY;
#pragma unroll
                for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                    for (int v = 0; v < 4; ++v) t = fmaxf(t, 16 * bb + 4 * kg + v <= pos ? s[bb][nb][v] : -INFINITY);
                t = fmaxf(paged_column_max(t) * a.scale_log2e, PAGED_NO_MAX);
                if (!second && kg == 0) refs[nb] = t;
            }
            paged_lds_barrier();   // (K ring slot 2 is free)
        }
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            l[nb] = 0.f;
            p[nb] = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
            for (int md = 0; md < MD; ++md) o[md][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        // ---- tile loop -------------------------------------------------------------------------------------
        // Barrier kt says that K tile kt and V tile kt - 1 have landed and that nobody reads K tile kt - 1 and V tile kt - 2 any more; the copies
        // behind it refill those slots: K tile kt + 2 and V tile kt + 1; and the page numbers of tile kt + 5.
        int vp = 2 * TILE;                      // ring slot of V tile kt - 1
        Rows after = find_rows(kb + 2, (kb + 2) & 7);   // of tile kt + 2, found during the softmax phase in front of copies(kt)
        auto copies = [&](int kt) {
            copy_rows(after, k_pages, k_base + c2);
            copy_rows(next, v_pages, v_base + c1);
            copy_pages(kt + 5, (kt + 5) & 7);
            next = after;
        };
        // Values of tile kt (ring slot `slot`), this wave's rows, that are not finite: out of LDS.
        auto scrub = [&](int kt, int slot) {
            if (kt < n_plain && sm.hole[kt & 7][wave] == 0) return;   // (its own entry)
            bool found = false;
#pragma unroll 1
            for (int i = lane * 16; i < RW * ROW; i += 1024) {
                unsigned char* at = sm.v[0] + slot + RW * wave * ROW + i;
                u32x4 w = *reinterpret_cast<const u32x4*>(at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t kept = paged_finite_or_zero<__bf16>(w[e]);
                    found = found || kept != w[e];
                    w[e] = kept;
                }
                *reinterpret_cast<u32x4*>(at) = w;
            }
            if (__any(found) && lane == 0) sm.apart = 1;
        };
        auto barrier = [&](int kt) {
            __builtin_amdgcn_sched_barrier(0);
            paged_wait_but<2 * COPIES + 1>();      // all but the newest tile's copies
            if constexpr (EXACT) scrub(kt, c0);
            __builtin_amdgcn_s_waitcnt(0xc07f);    // lgkmcnt(0): the wave's own reads and writes
            plain_barrier();
            vp = c0;
            c0 = c1; c1 = c2; c2 = vp;
            __builtin_amdgcn_sched_barrier(0);
        };
        auto above = [&](float logit, float reference) {   // logit x scale - reference (EXACT: of the rounded product, PAGED_FAR)
#pragma clang fp contract(off)
            return EXACT ? logit * a.scale_log2e - reference : __builtin_fmaf(logit, a.scale_log2e, -reference);
        };
        auto softmax = [&](int kt, int ahead) {   // and the rows of tile `ahead`, which the copies behind it, or the next ones, do not bring yet
            const Rows found = find_rows(ahead, ahead & 7);
            uint32_t hole = 0;
            bool any_hole = false;
            if constexpr (EXACT) any_hole = holes_of(kt, &hole);
            if (__builtin_expect(kt >= n_plain || any_hole, 0)) mask(kt, hole);
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                float s0, s1;
#pragma unroll
                for (int bb = 0; bb < 2; ++bb)
#pragma unroll
                    for (int v = 0; v < 4; v += 2) {
                        const float p0 = __builtin_amdgcn_exp2f(above(s[bb][nb][v], m[nb]));
                        const float p1 = __builtin_amdgcn_exp2f(above(s[bb][nb][v + 1], m[nb]));
                        s0 = bb == 0 && v == 0 ? p0 : s0 + p0;
                        s1 = bb == 0 && v == 0 ? p1 : s1 + p1;
                        bf16x2 w;
                        w[0] = (__bf16)p0;
                        w[1] = (__bf16)p1;
                        p[nb][2 * bb + v / 2] = __builtin_bit_cast(uint32_t, w);
                    }
                l[nb] += s0 + s1;
            }
            __builtin_amdgcn_sched_barrier(0);
            return found;
        };
        if (!second) {
            for (int kt = kb;; ++kt) {
                matrix_phase<D, true>(tv + vp, tk + c0, qf, q_lds, p, o, s, ref_lds, m);
                if (kt == ke) break;
                copies(kt);
                after = softmax(kt, kt + 3);
                barrier(kt);
            }
        } else {
            copies(kb);
            after = find_rows(kb + 3, (kb + 3) & 7);
            for (int kt = kb;; ++kt) {
                matrix_phase<D, true>(tv + vp, tk + c0, qf, q_lds, p, o, s, ref_lds, m);
                if (kt == ke) break;
                barrier(kt);
                const Rows found = softmax(kt, kt + 4);
                copies(kt + 1);
                after = found;
            }
        }
        paged_wait_but<0>();
    } else {
        if (tid < C) reinterpret_cast<float*>(smem_raw + references_at<D>())[tid] = PAGED_NO_MAX;
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            l[nb] = 0.f;
#pragma unroll
            for (int md = 0; md < MD; ++md) o[md][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }

    // ---- the two waves of a row group add up: each keeps half of the dims ------------------------------------------
    paged_lds_barrier();   // (also: everyone is done with the rings)
    bool apart = false;
    if constexpr (EXACT) {
        apart = sm.apart != 0;
        paged_lds_barrier();
    }
    constexpr int MH = MD / 2;
    f32x4 oh[MH][NC];
    const int md0 = second * MH;
    {
        unsigned char* mine = smem_raw + (size_t)wave * EXCHANGE_WAVE<D> + lane * 16;
        const unsigned char* other = smem_raw + (size_t)(wave ^ 4) * EXCHANGE_WAVE<D> + lane * 16;
        if (second) {
#pragma unroll
            for (int md = 0; md < MH; ++md)
#pragma unroll
                for (int nb = 0; nb < NC; ++nb) {
                    *reinterpret_cast<f32x4*>(mine + (md * NC + nb) * 1024) = o[md][nb];
                    oh[md][nb] = o[MH + md][nb];
                }
        } else {
#pragma unroll
            for (int md = 0; md < MH; ++md)
#pragma unroll
                for (int nb = 0; nb < NC; ++nb) {
                    *reinterpret_cast<f32x4*>(mine + (md * NC + nb) * 1024) = o[MH + md][nb];
                    oh[md][nb] = o[md][nb];
                }
        }
        *reinterpret_cast<f32x4*>(mine + MH * NC * 1024) = f32x4{l[0], l[1], l[2], l[3]};
        paged_lds_barrier();
#pragma unroll
        for (int md = 0; md < MH; ++md)
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                const f32x4 w = *reinterpret_cast<const f32x4*>(other + (md * NC + nb) * 1024);
#pragma unroll
                for (int e = 0; e < 4; ++e) oh[md][nb][e] += w[e];
            }
        const f32x4 l2 = *reinterpret_cast<const f32x4*>(other + MH * NC * 1024);
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) l[nb] = paged_column_sum(l[nb] + l2[nb]);
    }
    if constexpr (EXACT) {
        if (apart) {   // the values that were left out reach the columns that see them
            int pos[NC];
#pragma unroll
            for (int nb = 0; nb < NC; ++nb) {
                int token, head;
                it.column(a, 64 * group + 16 * nb + x, &token, &head);
                pos[nb] = paged_position(a, rq, token);
            }
#pragma unroll 1
            for (int j0 = KT * kb; j0 <= p_last && j0 < KT * ke; j0 += RW) {
                bool left = j0 / KT >= n_plain;
                for (int i = 0; i < RW && !left; ++i) left = !is_page(table[paged_block(a, j0 + i)]);
                if (!left) continue;
#pragma unroll 1
                for (int j = j0; j < j0 + RW && j <= p_last; ++j) {
                    const int block = paged_block(a, j), page = table[block];
                    if (!is_page(page)) continue;
                    const uint16_t* key = (const uint16_t*)(v_pages + ((size_t)page * a.P + (j - block * a.P)) * row_bytes);
#pragma unroll
                    for (int md = 0; md < MH; ++md)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const uint32_t w = key[16 * (md0 + md) + 4 * kg + v];
                            const float add = (w & 0x7F80u) == 0x7F80u ? __uint_as_float(w << 16) : 0.f;
#pragma unroll
                            for (int nb = 0; nb < NC; ++nb) oh[md][nb][v] += j <= pos[nb] ? add : 0.f;
                        }
                }
            }
        }
    }
    // With a fixed reference a runaway logit shows up as inf or NaN in the sums.  The sums of a part stay so far below that many of them add up.
    bool bad = false;
    if constexpr (!EXACT) {
        const float limit = whole ? INFINITY : 0x1p100f;
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            float check = l[nb];
#pragma unroll
            for (int md = 0; md < MH; ++md)
#pragma unroll
                for (int v = 0; v < 4; ++v) check += fabsf(oh[md][nb][v]);
            const float ref = refs[nb];
            bad = bad || !(check < limit) || (fabsf(ref) >= PAGED_FAR && ref != PAGED_NO_MAX);
        }
        if (any_of_workgroup(bad, answers + WAVES)) return false;   // (also: the exchange has been read)
    } else {
        paged_lds_barrier();
    }
    if (!whole) {
#pragma unroll
        for (int nb = 0; nb < NC; ++nb) {
            const int c = 64 * group + 16 * nb + x;
            if (!second && kg == 0) { part[2 * c] = refs[nb]; part[2 * c + 1] = l[nb]; }
#pragma unroll
            for (int md = 0; md < MH; ++md) *reinterpret_cast<f32x4*>(part + 2 * C + c * D + 16 * (md0 + md) + 4 * kg) = oh[md][nb];
        }
        return true;
    }
    // ---- normalise, transpose through LDS and store 16 bytes per lane ---------------------------------------------
    constexpr int PITCH = D + 8, NV = D / 8;
    __bf16* ob = reinterpret_cast<__bf16*>(smem_raw) + group * 64 * PITCH;   // [64 columns][d]
#pragma unroll
    for (int nb = 0; nb < NC; ++nb) {
        const bool none = l[nb] == 0.f;   // it saw nothing
        const float inv_l = none ? 0.f : 1.0f / l[nb];
        typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
        for (int md = 0; md < MH; ++md) {
            bf16x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = (__bf16)(oh[md][nb][e] * inv_l);
            *reinterpret_cast<bf16x4*>(&ob[(16 * nb + x) * PITCH + 16 * (md0 + md) + 4 * kg]) = w;
        }
        const int cl = 64 * group + 16 * nb + x;
        if (!second && kg == 0 && a.lse != nullptr && it.col0 + cl < it.cols)
            a.lse[it.out_row(a, cl)] = none ? -INFINITY : (refs[nb] + __builtin_amdgcn_logf(l[nb])) * 0.6931471805599453f;
    }
    paged_lds_barrier();   // (the rows of a group come from both of its waves)
#pragma unroll
    for (int i = 0; i < NV / 2; ++i) {
        const int c = (64 / NV) * (i + second * (NV / 2)) + lane / NV, v = lane % NV;
        if (it.col0 + 64 * group + c < it.cols)
            *reinterpret_cast<u32x4*>((__bf16*)a.out + it.out_row(a, 64 * group + c) * D + 8 * v) = *reinterpret_cast<const u32x4*>(&ob[c * PITCH + 8 * v]);
    }
    paged_lds_barrier();   // (the next piece's copies overwrite what was staged)
    return true;
}

template <int D, bool ALIGNED>
__global__ __launch_bounds__(64 * WAVES) void paged_tile_kernel(const PagedArgs args) {
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    PagedArgs a = args;
    if (a.route) {   // the requests with many columns, all, or none
        a.cols_hi = INT32_MAX;
        a.cols_lo = !paged_route(a, D * 4) ? INT32_MAX : a.together ? 0 : a.few;
    }
    const int g = paged_head(a), w = paged_workgroup(a);
    const TilePlan plan = tile_plan(a, w, w);
    PagedCut cut{0, 0, 0, 0};
    int64_t u = plan.whole ? 0 : paged_first_unit(w, plan.total, plan.sharers), start = plan.start;
    const int64_t end = plan.whole ? 0 : paged_first_unit(w + 1, plan.total, plan.sharers);
    for (int b = plan.b; b >= 0 && b < a.B;) {
        const PagedRequest rq = paged_request(a, b);
        const TileCosts c = tile_costs(a, rq);
        const int64_t all = rq.n > 0 ? c.before(c.n_ct) : 0;
        if (!plan.whole && u >= start + all) {
            start += all;
            ++b;
            continue;
        }
        const int t = plan.whole ? c.n_ct - 1 - (int)(w - start) : c.tile_at(u - start);
        const int i = (int64_t)C * (t + 1) >= (int64_t)rq.n * a.G ? rq.n - 1 : (C * (t + 1) - 1) / a.G;   // the tile's last row
        const int n = (paged_position(a, rq, i) + KT) / KT;                                              // its key tiles
        const int64_t cost = c.tile(t), x0 = plan.whole ? 0 : u - start - c.before(t), x1 = plan.whole ? cost : min(cost, x0 + (end - u));
        const int kb = x0 == 0 ? 0 : (int)paged_div(x0 * n, cost), ke = x1 == cost ? n : (int)paged_div(x1 * n, cost);
        float* part = paged_slot(a, w, g, x0 > 0 ? 0 : 1, C * paged_part_floats<D>());
        if (x0 == 0 && x1 < cost) cut = PagedCut{paged_owner(u + cost - 1, plan.total, plan.sharers) - w + 1, rq.first, C * t, rq.n * a.G};
        const bool whole = x0 == 0 && x1 == cost;
        if (!process_piece<D, ALIGNED, false>(a, rq, b, t, g, kb, ke, whole, part, smem_raw))
            process_piece<D, ALIGNED, true>(a, rq, b, t, g, kb, ke, whole, part, smem_raw);
        u += x1 - x0;
        if (plan.whole || u >= end) break;
    }
    if (threadIdx.x == 0 && w < a.n_wg) paged_cuts(a)[(size_t)w * a.Hkv + g] = cut;
}

// Joins the pieces of the items that fell to several workgroups, in their order: blockIdx.x = workgroup x Hkv + KV head, whose cut it sees to.  blockIdx.y: 16 columns,
// 16 threads each.
template <int D>
__global__ __launch_bounds__(256) void paged_tile_join_kernel(const PagedArgs a) {
    const int g = blockIdx.x % a.Hkv, w0 = blockIdx.x / a.Hkv;
    const PagedCut cut = paged_cuts(a)[blockIdx.x];
    const int n = cut.pieces;
    if (n == 0) return;
    constexpr int NV = D / 64, AHEAD = 8;   // vectors of a thread; pieces in flight
    const int cl = 16 * blockIdx.y + threadIdx.x / 16, e0 = 4 * (threadIdx.x % 16);
    if (cut.col0 + cl >= cut.cols) return;
    float top = PAGED_NO_MAX, l = 0.f;
    f32x4 o[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) o[k] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        float pm[AHEAD], pl[AHEAD];
        f32x4 po[AHEAD][NV];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {   // (past the end: the last piece, which does not count)
            const int i = min(i0 + k, n - 1);
            const float* part = paged_slot(a, w0 + i, g, i == 0 ? 1 : 0, C * paged_part_floats<D>());
            pm[k] = part[2 * cl];
            pl[k] = part[2 * cl + 1];
#pragma unroll
            for (int v = 0; v < NV; ++v) po[k][v] = *reinterpret_cast<const f32x4*>(part + 2 * C + cl * D + 64 * v + e0);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= n || pl[k] == 0.f) continue;   // (a piece that saw nothing of this column: its values may be anything)
            const float up = fmaxf(top, pm[k]), f = __builtin_amdgcn_exp2f(top - up), w = __builtin_amdgcn_exp2f(pm[k] - up);
            top = up;
            l = l * f + pl[k] * w;
#pragma unroll
            for (int v = 0; v < NV; ++v) o[v] = o[v] * f + po[k][v] * w;
        }
    }
    const bool none = l == 0.f;
    const float inv_l = none ? 0.f : 1.0f / l;
    const int col = cut.col0 + cl, i = col / a.G;
    const size_t oc = (size_t)(cut.first_row + i) * a.Hq + g * a.G + (col - i * a.G);
    typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        bf16x4 y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[v][e] * inv_l);
        *reinterpret_cast<bf16x4*>((__bf16*)a.out + oc * D + 64 * v + e0) = y;
    }
    if (e0 == 0 && a.lse != nullptr) a.lse[oc] = none ? -INFINITY : (top + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
}

template <int D, bool ALIGNED>
hipError_t launch(const PagedArgs& a, hipStream_t st) {
    static_assert(tile_lds_bytes<D>() <= 160 * 1024, "LDS of a compute unit");
    // Raises the kernel's dynamic LDS limit, once per process.
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void*>(&paged_tile_kernel<D, ALIGNED>),
                                                       hipFuncAttributeMaxDynamicSharedMemorySize, (int)tile_lds_bytes<D>());
    if (once != hipSuccess) return once;
    // no more items than this: full tiles of all rows, and one that is not full per request
    const int64_t rows = std::min<int64_t>(a.T, (int64_t)a.B * a.max_new);
    const int64_t items = rows * a.G / C + std::min<int64_t>(a.B, rows * a.G / ((int64_t)a.cols_lo + 1));
    const int64_t grid = std::max<int64_t>(a.n_wg, items);
    paged_tile_kernel<D, ALIGNED><<<dim3(paged_grid(grid, a.Hkv)), dim3(64 * WAVES), tile_lds_bytes<D>(), st>>>(a);
    if (a.n_wg > 1) paged_tile_join_kernel<D><<<dim3((unsigned)((a.n_wg - 1) * a.Hkv), C / 16), dim3(256), 0, st>>>(a);
    return hipGetLastError();
}

int tile_workgroups(int Hkv, int n_cu) { return std::max(1, n_cu / Hkv); }   // per KV head

}  // namespace

size_t paged_tile_partials_bytes(const Shape& s, int n_cu) {
    const int n = tile_workgroups(s.Hkv, n_cu);   // (one: nothing is cut)
    return (size_t)n * s.Hkv * ((n > 1 ? 2 * C * (s.d + 2) * sizeof(float) : 0) + sizeof(PagedCut));
}

hipError_t launch_paged_tile(const Shape& s, const PagedArgs& args, int n_cu, hipStream_t st) {
    PagedArgs a = args;
    a.n_wg = tile_workgroups(s.Hkv, n_cu);
    if (s.d == 128) return a.P % RW == 0 ? launch<128, true>(a, st) : launch<128, false>(a, st);
    return a.P % RW == 0 ? launch<64, true>(a, st) : launch<64, false>(a, st);
}

}  // namespace fr
