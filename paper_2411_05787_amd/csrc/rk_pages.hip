// rk_page_scores and rk_page_select: which pages of a cache a token reads.
#include "rk_pages.h"

namespace rk {

typedef short s16x2 __attribute__((ext_vector_type(2)));

// ---- bounds of the scores ----
// For a query q and a page whose keys lie between k_min and k_max in every dim,
//     sum_d max(q_d k_min_d, q_d k_max_d) = sum_d max(q_d, 0) k_max_d + min(q_d, 0) k_min_d,
// two products of q's non-negative and negative parts: 256 products of bf16 to a page and query on the matrix cores.  A wavefront holds 16
// pages (v_mfma_f32_16x16x32_bf16, columns) and goes over the tokens four at a time, four heads of each (rows): lane (n, g) gets page n's sums for four heads of token g, so that the
// heads of a group meet in one lane.
struct ScoreParams {
    const uint16_t* q; int64_t q_b, q_t;
    const uint16_t *k_min, *k_max;
    const int32_t *table, *seq_lens, *new_lens;
    int32_t width, shift, n_pages, n_new, Hq, Hkv, G, agg, chunk, chunks, page_blocks;
    float scale;
    float* scores; int64_t s_stride;
    const int32_t* pred; int32_t pred_val;
};

// 64 pages to a wavefront, all of whose bounds are requested at once.  TOKENS: the workgroup's wavefronts have the same pages, by way of LDS, and every fourth four
// tokens, so that a bound is requested once in whole rows and a query is read and its signs parted once for 64 pages; it also makes four times the
// workgroups.  Otherwise they have pages of their own and all tokens, which leaves the barrier out and asks for four times as much before the first wait.
// 32 heads over 8, TOKENS against the other: one token, 1 sequence of 1024 pages 4.0 and 7.1 us, 4 sequences 5.1 and 7.6, 8 sequences 10.2 and 9.3, 16
// sequences 16.5 and 14.3 (67.1 MB of bounds: 4.7 TB/s of scattered rows of 256 bytes); 16 tokens of 16 sequences 20.3 and 18.9, 32 of 8 15.2 and 17.2, 128 of 16 63.7 and
// 64.6, 256 of 16 111 and 118; 1000 tokens of 28 heads over 4, 313 pages 11.9 and 20.4.
constexpr int kScoreBlocks = 4;               // of 16 pages
template <bool TOKENS, int AGG>
__global__ __launch_bounds__(256, 2)
void page_score_kernel(const ScoreParams p) {
    constexpr int P = kScoreBlocks;
    const uint32_t part = blockIdx.x / (uint32_t)p.Hkv, part_b = part / (uint32_t)p.page_blocks;
    const int g = (int)(blockIdx.x - part * (uint32_t)p.Hkv), lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, gr = lane >> 4;
    const int block = (int)(part - part_b * (uint32_t)p.page_blocks), b = (int)(part_b / (uint32_t)p.chunks), t_first = (int)(part_b - b * (uint32_t)p.chunks) * p.chunk;
    const int most = (int)min((int64_t)p.width, p.s_stride);      // pages that are looked at
    const int j0 = TOKENS ? block * 16 * P : (block * 4 + w) * 16 * P;
    int page[P];                              // (requested before the sequence's length is known)
#pragma unroll
    for (int x = 0; x < P; ++x) page[x] = p.table[(int64_t)b * p.width + min(j0 + 16 * x + n, p.width - 1)];
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const int raw = p.seq_lens[b], n_tok = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    const int64_t start = (int64_t)raw - n_tok;
    const int t_end = min(t_first + p.chunk, n_tok);
    // pages that token i sees
    auto pages_of = [&](int i) { return (int)min(((start + i) >> p.shift) + 1, (int64_t)most); };
    if (t_first >= t_end || start + t_end - 1 < 0) return;
    const int some = pages_of(t_end - 1);     // that any of the tokens sees
    if (j0 >= some) return;
    bf16x8 hi[P][4], lo[P][4];
    if constexpr (TOKENS) {                   // by way of LDS: each bound is requested once, a row by 16 lanes
        constexpr int kRow = kD * 2 + 16;     // (16 rows of an operand fall on different banks)
        __shared__ __attribute__((aligned(16))) unsigned char sBounds[2][16 * P * kRow];
        const int seg = (threadIdx.x & 15) * 16, row0 = threadIdx.x >> 4;
        u32x4 u[2][P];
#pragma unroll
        for (int x = 0; x < P; ++x) {         // row 16 x + row0 is page j0 + 16 x + row0
            const int j = j0 + 16 * x + row0, pg = p.table[(int64_t)b * p.width + min(j, p.width - 1)];
            const int64_t at = ((int64_t)((uint32_t)pg < (uint32_t)p.n_pages && j < some ? pg : 0) * p.Hkv + g) * (kD * 2) + seg;
            u[0][x] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p.k_max) + at);
            u[1][x] = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(p.k_min) + at);
        }
#pragma unroll
        for (int x = 0; x < P; ++x)
#pragma unroll
            for (int y = 0; y < 2; ++y) *reinterpret_cast<u32x4*>(&sBounds[y][(16 * x + row0) * kRow + seg]) = u[y][x];
        __syncthreads();
#pragma unroll
        for (int x = 0; x < P; ++x)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                hi[x][s] = *reinterpret_cast<const bf16x8*>(&sBounds[0][(16 * x + n) * kRow + 64 * s + 16 * gr]);
                lo[x][s] = *reinterpret_cast<const bf16x8*>(&sBounds[1][(16 * x + n) * kRow + 64 * s + 16 * gr]);
            }
    } else {
#pragma unroll
        for (int x = 0; x < P; ++x) {
            const bool there = (uint32_t)page[x] < (uint32_t)p.n_pages && j0 + 16 * x + n < some;
            const int64_t at = ((int64_t)(there ? page[x] : 0) * p.Hkv + g) * kD + 8 * gr;
            if (x > 0 && j0 + 16 * x >= some) {       // (none of the block's pages is there)
#pragma unroll
                for (int s = 0; s < 4; ++s) hi[x][s] = lo[x][s] = bf16x8{};
                continue;
            }
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                hi[x][s] = *reinterpret_cast<const bf16x8*>(p.k_max + at + 32 * s);
                lo[x][s] = *reinterpret_cast<const bf16x8*>(p.k_min + at + 32 * s);
            }
        }
    }
    const uint16_t* q0 = p.q + (int64_t)b * p.q_b + (int64_t)(g * p.G) * kD + 8 * gr;
    u32x4 q[4];
    auto ask = [&](int t0, int h0) {
        const uint16_t* qr = q0 + (int64_t)min(t0 + (n >> 2), t_end - 1) * p.q_t + (int64_t)min(h0 + (n & 3), p.G - 1) * kD;
#pragma unroll
        for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const u32x4*>(qr + 32 * s);
    };
    constexpr int step = TOKENS ? 16 : 4;
    const int t_mine = t_first + (TOKENS ? 4 * w : 0), heads = AGG == RK_AGG_FIRST ? 1 : p.G;
    if (t_mine < t_end) ask(t_mine, 0);
    for (int t0 = t_mine; t0 < t_end; t0 += step) {
        const int i = t0 + gr;
        float best[P];
#pragma unroll
        for (int x = 0; x < P; ++x) best[x] = AGG == RK_AGG_MAX ? -INFINITY : 0.f;
        for (int h0 = 0; h0 < heads; h0 += 4) {
            u32x4 up[4], down[4];
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t word = q[s][e];
                    const s16x2 signs = __builtin_bit_cast(s16x2, word) >> 15;        // (a half in full where it is set)
                    const uint32_t negative = __builtin_bit_cast(uint32_t, signs);
                    down[s][e] = word & negative;
                    up[s][e] = word & ~negative;
                }
            const bool more = h0 + 4 < heads;
            ask(more ? t0 : min(t0 + step, t_end - 1), more ? h0 + 4 : 0);       // (the next one's, beside the products)
            f32x4 acc[P];
#pragma unroll
            for (int x = 0; x < P; ++x) acc[x] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
#pragma unroll
                for (int x = 0; x < P; ++x) acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up[s]), hi[x][s], acc[x], 0, 0, 0);
#pragma unroll
                for (int x = 0; x < P; ++x) acc[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down[s]), lo[x][s], acc[x], 0, 0, 0);
            }
            // (heads beyond the group repeat its last one: once more for a maximum, nothing for a sum)
#pragma unroll
            for (int x = 0; x < P; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float one = acc[x][y] * p.scale;
                    if constexpr (AGG == RK_AGG_MAX) best[x] = __builtin_elementwise_maximum(best[x], one);      // (no number stays none)
                    else if constexpr (AGG == RK_AGG_MEAN) { if (h0 + y < p.G) best[x] += one; }
                    else if (y == 0) best[x] = one;
                }
        }
        if (i >= t_end || start + i < 0) continue;
        const int seen = pages_of(i);
        float* to = p.scores + (((int64_t)b * p.n_new + i) * p.Hkv + g) * p.s_stride + j0 + n;
#pragma unroll
        for (int x = 0; x < P; ++x) {
            if constexpr (AGG == RK_AGG_MEAN) best[x] /= (float)p.G;
            if ((uint32_t)page[x] >= (uint32_t)p.n_pages) best[x] = -INFINITY;
            if (j0 + 16 * x + n < seen) to[16 * x] = best[x];
        }
    }
    // Pages that tokens see behind the table's last one, whose rows do not exist (mostly none): whoever has that page says so.
    if (p.s_stride <= most || j0 + 16 * P < most || (start + t_end - 1) >> p.shift < most) return;
    for (int t0 = t_mine; t0 < t_end; t0 += step) {
        const int i = t0 + gr;
        if (i >= t_end || start + i < 0) continue;
        float* to = p.scores + (((int64_t)b * p.n_new + i) * p.Hkv + g) * p.s_stride;
        const int all = (int)min(((start + i) >> p.shift) + 1, p.s_stride);
        for (int j = most + n; j < all; j += 16) to[j] = -INFINITY;
    }
}
using ScoreKernel = void (*)(const ScoreParams);
template <bool TOKENS> static ScoreKernel score_kernel(int agg) {
    return agg == RK_AGG_MAX ? page_score_kernel<TOKENS, RK_AGG_MAX> : agg == RK_AGG_MEAN ? page_score_kernel<TOKENS, RK_AGG_MEAN> : page_score_kernel<TOKENS, RK_AGG_FIRST>;
}

// ---- the pages with the largest ----
// W wavefronts to a row of up to 64 W R scores, which stay in registers, R to a lane; bound by its chain of instructions.  The threshold is built bit by bit
// from the top: the largest T with k keys or more at or above it, and as soon as there are k exactly the pages are found (mostly after a third of the 32
// steps).  One wavefront needs no exchange for its counts, four have a quarter of the compares each: 128 rows of 313 scores 4.7 us with one, 6.4 with four, of 600 6.4
// and 6.4, of 1000 9.3 and 6.8; where the rows fill the chip the exchange only costs: 1024 rows of 1000 scores 10.1 and 9.7 us, 2048 rows 10.8 and 13.9, 16384
// rows 36 and 73.  So one up to 640 scores, four beyond that for up to 1024 rows, and for any beyond 1024 scores.  R only follows the width
// (with 16 to a lane and 8: 128 rows of 2000 scores 11.8 and 8.8 us, 16384 rows of 1100 156 and 93).  Rows of more scores than 16384 go to the long form.
constexpr int kSelectThreads = 256, kSelectMost = 16 * 16 * 64;
struct SelectParams {
    const float* scores; int64_t s_stride;
    const int32_t *seq_lens, *new_lens;
    int32_t shift, n_new, Hkv, k, keep_first, keep_last;
    int32_t* idx;
    const int32_t* pred; int32_t pred_val;
};

// A row: its token's pages n and its own one, how many are wanted of them, its scores and results.  wanted < 0: there is no such token.
struct SelectRow { int n, last, wanted; const float* scores; int32_t* idx; };
__device__ __forceinline__ SelectRow select_row(const SelectParams& p, int row) {
    const int bt = (int)((uint32_t)row / (uint32_t)p.Hkv), b = bt / p.n_new, i = bt - b * p.n_new;
    SelectRow x{0, 0, -1, p.scores + (int64_t)row * p.s_stride, p.idx + (int64_t)row * p.k};
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return x;
    const int n_tok = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    if (i >= n_tok) return x;
    const int64_t pos = (int64_t)p.seq_lens[b] - n_tok + i;
    x.last = pos < 0 ? -1 : (int)(pos >> p.shift);
    x.n = (int)min((int64_t)x.last + 1, p.s_stride);
    x.wanted = min(p.k, x.n);
    return x;
}
// (what is kept in any case, and what is no number, counts as +infinity; one zero; above 0 in any case)
__device__ __forceinline__ uint32_t select_key(const SelectParams& p, const SelectRow& x, int j, float s) {
    return j < p.keep_first || j > x.last - p.keep_last || !(s <= INFINITY) ? key_of(INFINITY) : key_of(s + 0.f);
}

template <int W, int R>
__global__ __launch_bounds__(W * 64)
void page_select_kernel(const SelectParams p) {
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // (the whole row of scores, requested before its token's pages are known)
    float s[R];
    const float* scores = p.scores + (int64_t)blockIdx.x * p.s_stride;
#pragma unroll
    for (int r = 0; r < R; ++r) s[r] = scores[min((w * R + r) * 64 + lane, (int)p.s_stride - 1)];
    __builtin_amdgcn_sched_barrier(0);
    const SelectRow row = select_row(p, (int)blockIdx.x);
    if (row.wanted < 0) return;
    const int n = row.n, k = row.wanted;
    for (int x = k + tid; x < p.k; x += W * 64) row.idx[x] = -1;
    if (k == n) {
        for (int x = tid; x < n; x += W * 64) row.idx[x] = x;
        return;
    }
    uint32_t x[R];
#pragma unroll
    for (int r = 0; r < R; ++r) { const int j = (w * R + r) * 64 + lane; x[r] = j < n ? select_key(p, row, j, s[r]) : 0u; }
    // (few scores to a lane and an exchange: of three thresholds at once, two bits for one exchange.  One bit at a time and two: 128 rows of 1000 scores 6.8 and 6.6 us,
    // 512 rows 7.9 and 8.0, 1024 rows 9.15 and 9.8; of 4000, 16 to a lane, 11.6 and 13.9)
    constexpr int kBits = W > 1 && R <= 4 ? 2 : 1, N = (1 << kBits) - 1;
    struct Counts { int c[N]; };
    __shared__ __attribute__((aligned(16))) int sCount[2][W][4];
    __shared__ int sBase[W][2];
    int turn = 0;
    // keys of the row at or above v, v + step, ..
    auto count = [&](uint32_t v, uint32_t step) {
        Counts n{};
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int r = 0; r < R; ++r) n.c[i] += __popcll(__ballot(x[r] >= v + i * step));
        if constexpr (W > 1) {
            if (lane < N) sCount[turn][w][lane] = lane == 0 ? n.c[0] : lane == 1 ? n.c[N / 2] : n.c[N - 1];
            lds_barrier();
            n = Counts{};
#pragma unroll
            for (int y = 0; y < W; ++y)
#pragma unroll
                for (int i = 0; i < N; ++i) n.c[i] += sCount[turn][y][i];
            turn ^= 1;                        // (the next count's words: these may still be read)
#pragma unroll
            for (int i = 0; i < N; ++i) n.c[i] = __builtin_amdgcn_readfirstlane(n.c[i]);
        }
        return n;
    };
    uint32_t at = 0;
    int above = -1;                           // keys above `at`, where some that equal it stay out
    bool exact = false;
    for (int bit = 32 - kBits; bit >= 0 && !exact; bit -= kBits) {
        const uint32_t step = 1u << bit, from = at;
        const Counts n = count(from + step, step);
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (n.c[i] >= k) { at = from + (i + 1) * step; exact = n.c[i] == k; }
    }
    if (!exact) above = at == 0xffffffffu ? 0 : count(at + 1, 0).c[0];
    const int left = exact ? 0 : k - above;   // of the keys that equal `at`
    int done = 0, ties = 0;
    if constexpr (W > 1) {
        int a = 0, t = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            a += __popcll(__ballot(exact ? x[r] >= at : x[r] > at));
            t += __popcll(__ballot(!exact && x[r] == at));
        }
        if (lane == 0) { sBase[w][0] = a; sBase[w][1] = t; }
        lds_barrier();
        for (int y = 0; y < w; ++y) { done += sBase[y][0]; ties += sBase[y][1]; }
        done = __builtin_amdgcn_readfirstlane(done);
        ties = __builtin_amdgcn_readfirstlane(ties);
    }
    const unsigned long long below = (1ull << lane) - 1ull;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool in = exact ? x[r] >= at : x[r] > at, tie = !exact && x[r] == at;
        const unsigned long long am = __ballot(in), tm = __ballot(tie);
        const int t = ties + __popcll(tm & below);
        if (in || (tie && t < left)) row.idx[done + __popcll(am & below) + min(t, left)] = (w * R + r) * 64 + lane;
        done += __popcll(am); ties += __popcll(tm);
    }
}

// The long form: a workgroup to a row, which is read again for every eight bits of the threshold.
__global__ __launch_bounds__(kSelectThreads)
void page_select_long_kernel(const SelectParams p) {
    const SelectRow row = select_row(p, (int)blockIdx.x);
    if (row.wanted < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = row.n, k = row.wanted;
    for (int x = k + tid; x < p.k; x += kSelectThreads) row.idx[x] = -1;
    if (k == n) {
        for (int x = tid; x < n; x += kSelectThreads) row.idx[x] = x;
        return;
    }
    auto key = [&](int j) { return select_key(p, row, j, row.scores[j]); };
    __shared__ uint32_t hist[256];
    __shared__ uint32_t sPrefix;
    __shared__ int sLeft, sCount[kSelectThreads / 64][2];
    uint32_t prefix = 0;
    int left = k;                             // of the keys that begin with the prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += kSelectThreads) {
            const uint32_t x = key(j);
            if (shift == 24 || x >> (shift + 8) == prefix) atomicAdd(&hist[x >> shift & 255u], 1u);
        }
        __syncthreads();
        if (w == 0) {                         // lane x: digits 255 - 4 x down to 252 - 4 x
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) { c[e] = hist[255 - 4 * lane - e]; sum += c[e]; }
            uint32_t before = wave_inclusive_scan(sum) - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if ((int)before < left && left <= (int)(before + c[e])) { sPrefix = prefix << 8 | (uint32_t)(255 - 4 * lane - e); sLeft = left - (int)before; }
                before += c[e];
            }
        }
        __syncthreads();
        prefix = sPrefix; left = sLeft;
    }
    int done = 0, ties = 0;
    for (int j0 = 0; j0 < n; j0 += kSelectThreads) {
        const int j = j0 + tid;
        const uint32_t x = j < n ? key(j) : 0u;
        const bool above = j < n && x > prefix, tie = j < n && x == prefix;
        const unsigned long long am = __ballot(above), tm = __ballot(tie), below = (1ull << lane) - 1ull;
        if (lane == 0) { sCount[w][0] = __popcll(am); sCount[w][1] = __popcll(tm); }
        __syncthreads();
        int a = done, t = ties;
        for (int y = 0; y < kSelectThreads / 64; ++y) {
            if (y < w) { a += sCount[y][0]; t += sCount[y][1]; }
            done += sCount[y][0]; ties += sCount[y][1];
        }
        a += __popcll(am & below); t += __popcll(tm & below);
        if (above || (tie && t < left)) row.idx[a + min(t, left)] = j;
        __syncthreads();
    }
}

}  // namespace rk

using namespace rk;

extern "C" int rk_page_scores(const rk_geom* geom, const void* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_new, const rk_pages* pages,
                              const int32_t* table, int32_t table_width, const int32_t* seq_lens, const int32_t* new_lens, int32_t agg,
                              float* scores, int64_t s_stride, const int32_t* pred, int32_t pred_val, void* stream) {
    int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!q || !seq_lens || !scores || n_new <= 0 || s_stride <= 0 || !aligned16(q) || ((uintptr_t)scores & 3u)) return RK_ERR_INVALID_ARG;
    if (q_stride_b < 0 || q_stride_t < 0 || q_stride_b % 8 != 0 || q_stride_t % 8 != 0) return RK_ERR_INVALID_ARG;
    if ((agg != RK_AGG_MAX && agg != RK_AGG_MEAN && agg != RK_AGG_FIRST) || n_new > 1 << 30) return RK_ERR_UNSUPPORTED;      // (tokens are counted past the last in 32 bits)
    if ((rc = check_pages(pages, false, true)) != RK_OK || (rc = check_table(pages, table, table_width)) != RK_OK) return rc;
    ScoreParams p{};
    p.q = (const uint16_t*)q; p.q_b = q_stride_b; p.q_t = q_stride_t;
    p.k_min = (const uint16_t*)pages->k_min; p.k_max = (const uint16_t*)pages->k_max;
    p.table = table; p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.width = table_width; p.shift = page_shift(pages->page); p.n_pages = pages->n_pages;
    p.n_new = n_new; p.Hq = geom->n_q_heads; p.Hkv = geom->n_kv_heads; p.G = p.Hq / p.Hkv; p.agg = agg;
    p.scale = geom->scale; p.scores = scores; p.s_stride = s_stride;
    p.pred = pred; p.pred_val = pred_val;
    const int64_t most = table_width < s_stride ? table_width : s_stride;
    const int64_t pairs = (int64_t)p.Hkv * geom->batch;
    // (few tokens, and pages that fill the chip 256 to a workgroup: a wavefront's own; otherwise 64 to a workgroup: see the kernel)
    const bool tokens = n_new > 16 || pairs * ((most + 255) / 256) < kComputeUnits;
    const int per = tokens ? 64 : 256;
    p.page_blocks = (int)((most + per - 1) / per);
    const int64_t wgs = p.page_blocks * pairs;
    const int unit = tokens ? 16 : 4;           // tokens of a workgroup's round
    int64_t chunks = 2 * kComputeUnits / wgs;
    if (chunks > (n_new + unit - 1) / unit) chunks = (n_new + unit - 1) / unit;
    if (chunks < 1) chunks = 1;
    p.chunk = (int)(((n_new + chunks - 1) / chunks + unit - 1) / unit * unit);
    p.chunks = (int)((n_new + p.chunk - 1) / p.chunk);
    const int64_t total = (int64_t)p.page_blocks * p.chunks * geom->batch * p.Hkv;
    if (!fits_launch(total, 256)) return RK_ERR_UNSUPPORTED;
    auto kernel = tokens ? score_kernel<true>(agg) : score_kernel<false>(agg);
    hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(256), 0, (hipStream_t)stream, p);
    return launch_status();
}

extern "C" int rk_page_select(const rk_geom* geom, const float* scores, int64_t s_stride, int32_t n_new, int32_t page, const int32_t* seq_lens,
                              const int32_t* new_lens, int32_t k, int32_t keep_first, int32_t keep_last, int32_t* idx,
                              const int32_t* pred, int32_t pred_val, void* stream) {
    const int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!scores || !seq_lens || !idx || n_new <= 0 || s_stride <= 0 || k <= 0 || keep_first < 0 || keep_last < 0) return RK_ERR_INVALID_ARG;
    if (((uintptr_t)scores & 3u) || ((uintptr_t)idx & 3u)) return RK_ERR_INVALID_ARG;
    if (page != 16 && page != 32 && page != 64 && page != 128) return RK_ERR_UNSUPPORTED;
    if ((int64_t)k * page > INT32_MAX - 2 * kMaxChunks * kMinChunk) return RK_ERR_UNSUPPORTED;      // (more than any sequence has, as for rk_sparse_attn)
    const int64_t rows = (int64_t)geom->batch * n_new * geom->n_kv_heads;
    SelectParams p{};
    p.scores = scores; p.s_stride = s_stride; p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.shift = page_shift(page); p.n_new = n_new; p.Hkv = geom->n_kv_heads; p.k = k; p.keep_first = keep_first; p.keep_last = keep_last;
    p.idx = idx; p.pred = pred; p.pred_val = pred_val;
    const int64_t n = s_stride;
    const bool four = n > 4096 ? false : n > 1024 || (n > 640 && rows <= 4 * kComputeUnits);
    auto kernel = n <= 192 ? page_select_kernel<1, 3> : n <= 384 ? page_select_kernel<1, 6> : n <= 640 ? page_select_kernel<1, 10>
                  : n <= 1024 ? (four ? page_select_kernel<4, 4> : page_select_kernel<1, 16>) : n <= 2048 ? page_select_kernel<4, 8> : n <= 4096 ? page_select_kernel<4, 16>
                  : n <= kSelectMost ? page_select_kernel<16, 16> : page_select_long_kernel;
    const int threads = four || n > kSelectMost ? 256 : n <= 1024 ? 64 : 1024;
    if (!fits_launch(rows, threads)) return RK_ERR_UNSUPPORTED;
    hipLaunchKernelGGL(kernel, dim3((unsigned)rows), dim3(threads), 0, (hipStream_t)stream, p);
    return launch_status();
}
