// rk_prompt_attn: attention of the new tokens of each sequence over the bf16 cache that holds them (kernels and their shapes: rk_prompt.h).
#include "rk_prompt.h"

namespace rk {

// Joins the parts of a row, sum_s 2^(m_s - m) (l_s, o_s): a wavefront each.  8 sequences of one token, 32 heads: 4.2 us, a launch and three
// dependent reads.
__global__ __launch_bounds__(256)
void prompt_merge_kernel(const PromptParams p) {
    const int g = blockIdx.y, b = blockIdx.z, w = threadIdx.x >> 6, lane = threadIdx.x & 63, row = blockIdx.x * 4 + w;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    __shared__ float sW[4][kMaxSplits];
    const Tokens tok = tokens_of(p, b);
    if (row >= tok.n * p.G) return;
    const int64_t bg = (int64_t)b * p.Hkv + g;
    const int rows = p.n_new * p.G, parts = p.cols ? p.parts[2 * bg + 1] : p.parts[bg * p.row_tiles + row / kPromptRows];
    if (!p.cols && parts == 1) return;
    // part s of this row is at + s * step
    const int64_t at = p.cols ? ((int64_t)g * p.splits * p.batch + p.parts[2 * bg]) * rows + row : (bg * rows + row) * p.splits;
    const int step = p.cols ? rows : 1;
    float m[kMaxSplits / 64], l[kMaxSplits / 64], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 64; ++i) {
        const int s = lane + 64 * i;
        const float2 ml = s < parts ? *reinterpret_cast<const float2*>(p.part_ml + (at + (int64_t)s * step) * 2) : make_float2(-INFINITY, 0.f);
        m[i] = ml.x; l[i] = ml.y;
        top = fmaxf(top, ml.x);
    }
    top = wave_max(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < kMaxSplits / 64; ++i) {
        const float a = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top);
        sum = fmaf(a, l[i], sum);
        sW[w][lane + 64 * i] = a;
    }
    sum = wave_sum(sum);
    wave_lds_sync();
    const float2* from = reinterpret_cast<const float2*>(p.part_o + at * kD) + lane;
    float o0 = 0.f, o1 = 0.f;
    for (int s = 0; s < parts; s += 8) {
        float2 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = from[(int64_t)min(s + i, parts - 1) * step * (kD / 2)];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = s + i < parts ? sW[w][s + i] : 0.f;
            if (a != 0.f) { o0 = fmaf(a, v[i].x, o0); o1 = fmaf(a, v[i].y, o1); }      // (a part without rows left nothing)
        }
    }
    const int i = (uint32_t)row / (uint32_t)p.G;
    const int64_t to = ((int64_t)b * p.n_new + i) * p.Hq + g * p.G + (row - i * p.G);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    reinterpret_cast<uint32_t*>(p.out + to * kD)[lane] = pack_bf16(o0 * inv, o1 * inv);
    if (lane == 0 && p.lse != nullptr) p.lse[to] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
}

static int cap_form(const rk_prompt_scores* s) { return !s || s->cap == 0.f ? kNoCap : s->cap <= kNearCapMost ? kNearCap : kFarCap; }
using PromptKernel = void (*)(const PromptParams);
template <int W> static PromptKernel prompt_cols_form(const rk_prompt_scores* s, bool slope) {
    switch (cap_form(s)) {
        case kNearCap: return slope ? prompt_cols_kernel<W, kNearCap, true> : prompt_cols_kernel<W, kNearCap, false>;
        case kFarCap: return slope ? prompt_cols_kernel<W, kFarCap, true> : prompt_cols_kernel<W, kFarCap, false>;
        default: return slope ? prompt_cols_kernel<W, kNoCap, true> : prompt_cols_kernel<W, kNoCap, false>;
    }
}
static PromptKernel prompt_tile_form(const rk_prompt_scores* s, bool slope) {
    switch (cap_form(s)) {
        case kNearCap: return slope ? prompt_tile_kernel<1, kNearCap, true> : prompt_tile_kernel<1, kNearCap, false>;
        case kFarCap: return slope ? prompt_tile_kernel<1, kFarCap, true> : prompt_tile_kernel<1, kFarCap, false>;
        default: return slope ? prompt_tile_kernel<1, kNoCap, true> : prompt_tile_kernel<1, kNoCap, false>;
    }
}

}  // namespace rk

using namespace rk;

extern "C" size_t rk_prompt_workspace_bytes(const rk_geom* geom, int32_t n_new, int32_t max_len) {
    if (check_geom(geom) != RK_OK || n_new <= 0 || max_len <= 0) return 0;
    return align_up(((size_t)prompt_partials(geom, n_new, max_len) * (kD + 2) + kPromptTarget) * sizeof(float), 256);
}

extern "C" int rk_prompt_attn(const rk_geom* geom, const void* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_new, rk_kv cache,
                              const int32_t* seq_lens, const int32_t* new_lens, int32_t max_len, const rk_prompt_scores* scores,
                              void* out, float* lse, const int32_t* pred, int32_t pred_val,
                              void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!q || !out || !seq_lens || n_new <= 0 || max_len <= 0 || !aligned16(q) || !aligned16(out)) return RK_ERR_INVALID_ARG;
    if (q_stride_b < 0 || q_stride_t < 0 || q_stride_b % 8 != 0 || q_stride_t % 8 != 0) return RK_ERR_INVALID_ARG;
    if (scores && !(scores->cap >= 0.f && isfinite(scores->cap))) return RK_ERR_INVALID_ARG;
    if ((rc = check_kv(cache)) != RK_OK) return rc;
    const int G = geom->n_q_heads / geom->n_kv_heads;
    const int64_t pairs = (int64_t)geom->batch * geom->n_kv_heads;
    if ((int64_t)n_new * G > INT32_MAX - 128) return RK_ERR_UNSUPPORTED;
    // (a scale of 0 goes with the slopes: masked products would be 0 times infinity in a weight's exponent)
    const bool cap = scores && scores->cap > 0.f, slope = (scores && scores->slopes) || (geom->scale == 0.f && !cap);
    const PromptPlan plan = prompt_plan(geom, n_new, max_len, !cap && !slope);
    if (pairs * plan.row_tiles * plan.splits > INT32_MAX / 2) return RK_ERR_UNSUPPORTED;
    PromptParams p{};
    p.q = (const uint16_t*)q; p.q_b = q_stride_b; p.q_t = q_stride_t;
    p.k = (const uint16_t*)cache.k; p.v = (const uint16_t*)cache.v; p.s_b = cache.stride_b; p.s_h = cache.stride_h; p.cap_rows = (int32_t)cache.capacity;
    p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.n_new = n_new; p.max_len = max_len; p.Hq = geom->n_q_heads; p.Hkv = geom->n_kv_heads; p.G = G; p.batch = geom->batch;
    p.scale = geom->scale;
    if (scores) { p.cap = scores->cap; p.slopes = scores->slopes; p.first = scores->first; p.end = scores->end; }
    p.out = (uint16_t*)out; p.lse = lse;
    p.pred = pred; p.pred_val = pred_val;
    p.splits = plan.splits; p.row_tiles = plan.row_tiles; p.split_tiles = plan.split_tiles;
    if (plan.splits > 1) {
        const size_t rows = (size_t)pairs * n_new * G * plan.splits;
        const size_t counts = (size_t)pairs * (plan.cols ? 2 : plan.row_tiles);
        if (!workspace || ((uintptr_t)workspace & 255u) != 0 || workspace_bytes < (rows * (kD + 2) + counts) * sizeof(float)) return RK_ERR_WORKSPACE;
        p.part_o = (float*)workspace;
        p.part_ml = p.part_o + rows * kD;
        p.parts = (int32_t*)(p.part_ml + rows * 2);
        p.cols = plan.cols ? 1 : 0;
        p.ragged = plan.cols ? ragged_batch_of(geom) : 0;
    }
    hipStream_t st = (hipStream_t)stream;
    if (plan.cols) {
        auto kernel = plan.alone ? prompt_cols_form<kColAlone>(scores, slope) : prompt_cols_form<kColWaves>(scores, slope);
        hipLaunchKernelGGL(kernel, dim3(plan.splits, geom->n_kv_heads, geom->batch), dim3((plan.alone ? kColAlone : kColWaves) * 64), 0, st, p);
    } else {
        auto kernel = plan.wide ? prompt_tile_kernel<2, kNoCap, false> : prompt_tile_form(scores, slope);
        const int64_t total = pairs * plan.row_tiles * plan.splits;
        // (Where all workgroups are there at once, two to a compute unit, the second ones come in the opposite order: the longest beside the
        // shortest.  8000 tokens of 8 heads 173 -> 165 us, 2048 of 32 over 8 53.0 -> 51.0, three capped chunks 70.3 -> 69.0.)
        p.first_round = !plan.wide && total <= 2 * kComputeUnits ? (int)((kComputeUnits + pairs - 1) / pairs) : INT32_MAX;
        hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(256), 0, st, p);
    }
    if ((rc = launch_status()) != RK_OK || plan.splits == 1) return rc;
    hipLaunchKernelGGL(prompt_merge_kernel, dim3((unsigned)((n_new * G + 3) / 4), geom->n_kv_heads, geom->batch), dim3(256), 0, st, p);
    return launch_status();
}
