// Attention of chunks of new tokens over a paged cache: row i of request b is the token at position p = cached_len[b] + i and sees the keys at
// positions 0 .. p, key j in row j % P of page block_table[b][j / P].
//
//   out = sum_{j <= p} w_j v_j / sum_j w_j,  w_j = exp(q . k_j / sqrt(d) - m),  lse = m + log sum_j w_j
//
// Which kernels a call takes.  The lengths are on the device; the host knows the number of requests and rows and a bound on the rows of one.  A request with few query columns
// (rows x heads of a group) is bound by the bytes of its keys and values: k_paged_stream.hip; one with many by the matrix instructions: k_paged_tile.hip, whose
// tile of 256 columns takes 1.5 us per 64 keys however few of them there are.  Where the total decides and the host's bounds do not (a table has room for more than
// its requests hold), both are launched and find out which of them works (paged_route); the other one's launch and its joining pass take 9.5 us.
//
// A step with trees (masks): the same with "see" by the rows' masks among the request's own rows; requests with many columns by k_paged_tree.hip.
#include "k_paged.hpp"

#include <algorithm>

namespace fr {

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
    a.mask = args.mask; a.words = args.mask_words;
    if (a.mask != nullptr) {
        // A step with trees.  k_paged_tree.hip reads the keys once for 256 columns and takes 12 - 20 us for the shortest call, the streaming kernel once for 32 and 7 - 14 us.  us
        // streaming : tree, requests x rows behind positions (columns of a request; columns x keys of all KV heads); 32 / 8 heads of 128: 1 x 16 behind 4000 (64; 2.1 M) 23 : 20,
        // 1 x 64 behind 1000 (256; 2.2 M) 21 : 22, 16 x 24 behind 100 (96; 1.5 M) 16 : 24, 16 x 24 behind 1000 (12.6 M) 47 : 30, 16 x 40 behind 16000 (160; 328 M) 934 : 277, and with up to 32 columns
        // 4 x 8 behind 4000 26 : 25, 16 x 8 behind 16000 207 : 204, 48 x 4 behind 1000 55 : 55; 16 / 8 heads of 64: 4 x 24 behind 16000 (48; 25 M) 43 : 42, 4 x 40 behind 1000 (80; 2.7 M) 19 : 21, 16 x 40 behind
        // 1000 (80; 10.6 M) 25 : 24, 48 x 40 behind 4000 (80; 124 M) 242 : 111.
        // Where the rule errs: of 375 calls (1 - 48 requests of one length, 2 - 128 rows behind 100 - 16000, those two and 28 / 4 heads of 128, tables as wide as the lengths) 14 take over 10 % longer than the other
        // kernel would.  Many rows behind few keys or few columns behind many should stream: 4 x 128 behind 100 18 : 34, 16 x 64 behind 100 29 : 37, 1 x 128 behind 1000 23 : 29, 1 x 64 behind 4000 26 : 30, 28 / 4 heads 4 x 8
        // behind 4000 22 : 28, 4 x 16 26 : 32, 1 x 16 behind 16000 27 : 33; long ones of head_dim 64 should not: 16 x 24 behind 16000 155 : 121, 48 x 24 behind 4000 116 : 102.  And it counts the room of
        // the table, as the host does not know the lengths: with room for 131072 positions 69 of the 375 do, 59 of them behind 100 or 1000 (16 x 24 behind 100 16 : 24, 28 / 4 heads 16 : 31).
        a.cols_hi = INT32_MAX;
        const double pairs = (double)std::min<int64_t>(a.T, (int64_t)a.B * a.max_new) * s.Hq * a.cap;   // at most
        const bool many = (int64_t)a.max_new * s.G > (s.d == 128 ? 32 : 64) && pairs > (s.d == 128 ? 2.5e6 : 10e6);
        const bool tiled = args.kernel == FR_PAGED_KERNEL_AUTO ? many : args.kernel == FR_PAGED_KERNEL_TILED;
        return s.dtype == FR_BF16 && tiled ? launch_paged_tree(s, a, n_cu, st) : launch_paged_stream(s, a, n_cu, st);
    }
    if (s.dtype != FR_BF16 || args.kernel == FR_PAGED_KERNEL_STREAM) {
        a.cols_hi = INT32_MAX;
        return launch_paged_stream(s, a, n_cu, st);
    }
    // Requests with few columns, and the others.  Where there are others, up to a quarter as many requests x KV heads as compute units go with them, which saves two launches: us
    // apart : together, one request of 777 rows behind 4000 and n of one row behind 2000 - 8000; 32 / 8 heads n = 4 150 : 138, 8 153 : 145, 16 202 : 193, 32 269 : 303, 63 373 : 532;
    // 28 / 4 heads n = 8 142 : 125, 16 154 : 143, 32 200 : 206; 16 / 8 heads, head_dim 64, n = 4 71 : 65, 8 80 : 80, 16 92 : 103; behind 100 - 1000 rows
    // of 32 / 8 heads n = 4 138 : 126, 8 135 : 144, 16 144 : 155.
    a.few = std::max(64, s.G);
    a.cols_hi = INT32_MAX;
    if (args.kernel == FR_PAGED_KERNEL_TILED) return launch_paged_tile(s, a, n_cu, st);
    const int64_t rows = std::min<int64_t>(a.T, (int64_t)a.B * a.max_new);
    // columns x keys of all KV heads (paged_route).  No more than what the table has room for
    const double most = (double)rows * s.Hq * a.cap;
    if ((int64_t)args.max_new * s.G <= a.few || most <= (double)PAGED_PAIRS_FAR) return launch_paged_stream(s, a, n_cu, st);
    // and no less than the chunks themselves, the rows spread evenly (the sum of squares is least then) and those of requests with few columns taken off: if every row of the call is
    // some request's.  A captured call has rows for the longest step it is replayed for, so there the lengths decide.
    const double few_rows = (double)a.few / s.G;
    const double least = args.captured || a.max_new > a.cap ? 0. : ((double)rows * rows / a.B - few_rows * few_rows * a.B) * s.Hq;
    a.together = (int64_t)(args.n_requests - 1) * s.Hkv <= n_cu / 4;
    a.route = least <= std::min((double)PAGED_PAIRS_NEAR, PAGED_PAIRS_SHORT + (double)PAGED_PAIRS_KEY * a.B * a.cap);
    if (a.route || !a.together) {
        if (!a.route) a.cols_hi = a.few;
        hipError_t e = launch_paged_stream(s, a, n_cu, st);
        if (e != hipSuccess) return e;
        a.cols_hi = INT32_MAX;
    }
    a.cols_lo = a.together ? 0 : a.few;
    return launch_paged_tile(s, a, n_cu, st);
}

size_t paged_attn_partials_bytes(const Shape& s, int n_cu) {
    const size_t stream = paged_stream_partials_bytes(s, n_cu);
    return s.dtype == FR_BF16 ? std::max({stream, paged_tile_partials_bytes(s, n_cu), paged_tree_partials_bytes(s, n_cu)}) : stream;
}

}  // namespace fr
