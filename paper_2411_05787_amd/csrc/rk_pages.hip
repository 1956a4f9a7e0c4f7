// rk_page_scores and rk_page_select: which pages of a cache a token reads.
#include "rk_pages.h"

namespace rk {

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
    int32_t width, shift, n_pages, n_new, Hq, Hkv, G, agg, chunk, page_blocks;
    float scale;
    float* scores; int64_t s_stride;
    const int32_t* pred; int32_t pred_val;
};

__global__ __launch_bounds__(256)
void page_score_kernel(const ScoreParams p) {
    const int g = blockIdx.y, b = blockIdx.z, lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, gr = lane >> 4;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const int block = (int)(blockIdx.x % (uint32_t)p.page_blocks), t_first = (int)(blockIdx.x / (uint32_t)p.page_blocks) * p.chunk;
    const int raw = p.seq_lens[b], n_tok = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    const int64_t start = (int64_t)raw - n_tok;
    const int t_end = min(t_first + p.chunk, n_tok), j0 = block * 64 + w * 16;
    const int most = (int)min((int64_t)p.width, p.s_stride);      // pages that are looked at
    // pages that token i sees
    auto pages_of = [&](int i) { return (int)min(((start + i) >> p.shift) + 1, (int64_t)most); };
    if (t_first >= t_end || start + t_end - 1 < 0 || j0 >= pages_of(t_end - 1)) return;
    const int j = j0 + n, page = j < most ? p.table[(int64_t)b * p.width + j] : -1;
    const bool there = (uint32_t)page < (uint32_t)p.n_pages;
    const int64_t at = ((int64_t)(there ? page : 0) * p.Hkv + g) * kD + 8 * gr;
    bf16x8 hi[4], lo[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        hi[s] = *reinterpret_cast<const bf16x8*>(p.k_max + at + 32 * s);
        lo[s] = *reinterpret_cast<const bf16x8*>(p.k_min + at + 32 * s);
    }
    for (int t0 = t_first; t0 < t_end; t0 += 4) {
        const int i = t0 + gr;
        float best = -INFINITY;
        bool none = false;
        for (int h0 = 0; h0 < p.G; h0 += 4) {
            const uint16_t* qr = p.q + (int64_t)b * p.q_b + (int64_t)min(t0 + (n >> 2), t_end - 1) * p.q_t + (int64_t)(g * p.G + min(h0 + (n & 3), p.G - 1)) * kD + 8 * gr;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const u32x4 x = *reinterpret_cast<const u32x4*>(qr + 32 * s);
                u32x4 up, down;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t negative = ((x[e] & 0x80008000u) >> 15) * 0xffffu;      // the halves whose sign is set, in full
                    down[e] = x[e] & negative;
                    up[e] = x[e] & ~negative;
                }
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, up), hi[s], acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, down), lo[s], acc, 0, 0, 0);
            }
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (h0 + x < p.G) {
                    const float one = acc[x] * p.scale;
                    best = aggregate(best, one, h0 + x, p.agg);
                    none = none || (one != one && (h0 + x == 0 || p.agg != RK_AGG_FIRST));      // (a maximum would pass over it)
                }
        }
        if (none) best = __uint_as_float(0x7fc00000u);
        if (p.agg == RK_AGG_MEAN) best /= (float)p.G;
        if (i < t_end && start + i >= 0 && j < pages_of(i)) p.scores[(((int64_t)b * p.n_new + i) * p.Hkv + g) * p.s_stride + j] = there ? best : -INFINITY;
    }
}

// ---- the pages with the largest ----
// A workgroup to a row: the k-th largest key digit by digit, then the pages above it and the first of those that equal it, in their order.
constexpr int kSelectThreads = 256;
struct SelectParams {
    const float* scores; int64_t s_stride;
    const int32_t *seq_lens, *new_lens;
    int32_t shift, n_new, Hkv, k, keep_first, keep_last;
    int32_t* idx;
    const int32_t* pred; int32_t pred_val;
};

__global__ __launch_bounds__(kSelectThreads)
void page_select_kernel(const SelectParams p) {
    const int g = (int)(blockIdx.x % (uint32_t)p.Hkv), bt = (int)(blockIdx.x / (uint32_t)p.Hkv), b = bt / p.n_new, i = bt - b * p.n_new;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const int n_tok = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    if (i >= n_tok) return;
    const int64_t pos = (int64_t)p.seq_lens[b] - n_tok + i;
    const int last = pos < 0 ? -1 : (int)(pos >> p.shift), n = (int)min((int64_t)last + 1, p.s_stride), k = min(p.k, n);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const float* row = p.scores + ((int64_t)bt * p.Hkv + g) * p.s_stride;
    int32_t* out = p.idx + ((int64_t)bt * p.Hkv + g) * p.k;
    for (int x = k + tid; x < p.k; x += kSelectThreads) out[x] = -1;
    if (k == n) {
        for (int x = tid; x < n; x += kSelectThreads) out[x] = x;
        return;
    }
    // (what is kept in any case, and what is no number, counts as +infinity; one zero)
    auto key = [&](int j) {
        const float x = row[j];
        return j < p.keep_first || j > last - p.keep_last || !(x <= INFINITY) ? key_of(INFINITY) : key_of(x + 0.f);
    };
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
        if (above || (tie && t < left)) out[a + min(t, left)] = j;
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
    if (agg != RK_AGG_MAX && agg != RK_AGG_MEAN && agg != RK_AGG_FIRST) return RK_ERR_UNSUPPORTED;
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
    p.page_blocks = (int)((most + 63) / 64);
    const int64_t wgs = (int64_t)p.page_blocks * p.Hkv * geom->batch;
    int64_t chunks = 4 * kComputeUnits / wgs;
    if (chunks > (n_new + 3) / 4) chunks = (n_new + 3) / 4;
    if (chunks < 1) chunks = 1;
    p.chunk = (int)(((n_new + chunks - 1) / chunks + 3) / 4 * 4);
    chunks = (n_new + p.chunk - 1) / p.chunk;
    hipLaunchKernelGGL(page_score_kernel, dim3((unsigned)(p.page_blocks * chunks), p.Hkv, geom->batch), dim3(256), 0, (hipStream_t)stream, p);
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
    const int64_t rows = (int64_t)geom->batch * n_new * geom->n_kv_heads;
    if (rows > INT32_MAX / 2) return RK_ERR_UNSUPPORTED;
    SelectParams p{};
    p.scores = scores; p.s_stride = s_stride; p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.shift = page_shift(page); p.n_new = n_new; p.Hkv = geom->n_kv_heads; p.k = k; p.keep_first = keep_first; p.keep_last = keep_last;
    p.idx = idx; p.pred = pred; p.pred_val = pred_val;
    hipLaunchKernelGGL(page_select_kernel, dim3((unsigned)rows), dim3(kSelectThreads), 0, (hipStream_t)stream, p);
    return launch_status();
}
