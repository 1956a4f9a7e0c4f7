// rk_paged_attn, rk_prefix_attn and rk_sparse_attn: attention of new tokens over a cache in pages.
//
// The kernels of rk_prompt.h over rows that a table leads to, and for up to 16 rows (a decode step's token, drafted ones, one token over its chosen
// pages) the streaming one below.  A prefix that all sequences share is read once: the queries of all of them are the rows of one
// call over it (kRowsShared), each sequence's own rows behind it are another's, and the two leave partial results that one launch joins.
#include "rk_prompt.h"
#include "rk_pages.h"

namespace rk {

// ---- up to 16 rows in all ----
// prompt_cols_kernel over units of 16 rows: each is a buffer of its own inside its page.  A wavefront looks its next 64 tiles up at once, a lane each, and
// takes the page numbers from the lanes: no wait for a number of the table stands before a request.
template <int W, int CAP, bool SLOPE, int ROWS>
__global__ __launch_bounds__(W * 64, W == kColWaves ? 2 : 1)
void paged_cols_kernel(const PromptParams p) {
    constexpr bool CHOSEN = ROWS == kRowsChosen, SHARED = ROWS == kRowsShared;
    int b, g, split, slot, parts = p.splits, token = 0;
    if constexpr (CHOSEN) {                   // (KV heads fastest: those of all tokens that share rows meet in few caches)
        g = (int)(blockIdx.x % (uint32_t)p.Hkv);
        const int rest = (int)(blockIdx.x / (uint32_t)p.Hkv), bt = rest / p.splits;
        split = rest - bt * p.splits;
        b = bt / p.n_new; token = bt - b * p.n_new;
        slot = (bt * p.Hkv + g) * p.splits + split;
    } else {
        g = blockIdx.y; b = SHARED ? 0 : (int)blockIdx.z; split = blockIdx.x;
        slot = (int)(blockIdx.z * gridDim.x + blockIdx.x);
        if (!SHARED && p.ragged != 0) {
            AttnParams a;
            a.ragged_batch = p.ragged; a.nch = p.splits; a.share_cap = kMaxSplits; a.cap2 = p.cap_rows; a.max_rows2 = p.max_len;
            const RaggedSlot r = ragged_slot<false>(a, p.seq_lens, slot);
            if (r.b < 0) return;
            b = r.b; split = r.c; parts = r.nchunks;
        }
    }
    if (!SHARED && p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const Tokens tok = SHARED ? Tokens{} : tokens_of(p, b);
    const int n_rows = SHARED ? p.rows : CHOSEN ? (token < tok.n ? p.G : 0) : tok.n * p.G;
    if (n_rows == 0) return;
    const int64_t bg = SHARED ? g : (int64_t)b * p.Hkv + g;
    const bool partial = p.splits > 1 || p.joined != 0;
    if (!CHOSEN && partial && split == 0 && threadIdx.x == 0) { p.parts[2 * bg] = slot; p.parts[2 * bg + 1] = parts; }
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, gr = lane >> 4;
    bool real = col < n_rows;
    const int r0 = (CHOSEN ? token * p.G : 0) + min(col, n_rows - 1);
    const Query me = SHARED ? shared_query(p, g, r0, real) : paged_query<ROWS>(p, tok, b, g, r0);
    const bool some = real && me.lo < me.hi;
    const int seen = wave_min(some ? me.lo : INT32_MAX), hi = wave_max_i(some ? me.hi : INT32_MIN);
    const int in_lo = wave_max_i(real ? me.lo : INT32_MIN), in_hi = wave_min(real ? me.hi : INT32_MAX);
    const int lo = seen & -kTileRows;
    const int tiles = hi <= seen ? 0 : CHOSEN ? (int)((((int64_t)p.n_idx << p.shift) + kTileRows - 1) / kTileRows) : (int)(((int64_t)hi - lo + kTileRows - 1) / kTileRows);

    bf16x8 q[4];
    const uint16_t* qr = p.q + (int64_t)me.b * p.q_b + (int64_t)me.token * p.q_t + (int64_t)me.head * kD;
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const bf16x8*>(qr + operand_dim<false>(s, gr));
    __builtin_amdgcn_sched_barrier(0);
    const ScoreForm form = score_form<CAP>(p, 1.f);       // (natural units, as the columns' running state has them)
    const float slope = SLOPE && p.slopes != nullptr ? p.slopes[me.head] : 0.f;
    const uint16_t* k = p.k + (int64_t)g * p.s_h;
    const uint16_t* v = p.v + (int64_t)g * p.s_h;
    const int32_t* table = p.table + (SHARED ? 0 : (int64_t)b * p.width);
    const int32_t* idx = CHOSEN ? p.idx + (((int64_t)b * p.n_new + token) * p.Hkv + g) * p.n_idx : nullptr;
    const int step = parts * W, in_page = (1 << p.shift) - 1;

    // this lane's of the wavefront's next 64 tiles: each unit's page (-1: none) and first row
    int page[2], first[2];
    auto look = [&](int t) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int64_t at = ((int64_t)t + (int64_t)lane * step) * kTileRows + 16 * c + (CHOSEN ? 0 : lo);
            int64_t j = at >> p.shift;
            bool there;
            if constexpr (CHOSEN) {
                const int x = j < p.n_idx ? idx[j] : -1;
                there = (uint32_t)x < (uint32_t)p.width;
                j = there ? x : 0;
                first[c] = ((int)j << p.shift) + ((int)at & in_page);
                there = there && first[c] < hi && first[c] + 16 > seen;      // (what the token sees nothing of is not read)
            } else {
                there = at < hi;
                first[c] = there ? (int)at : 0;
                j = there ? j : 0;
            }
            const int x = there ? table[j] : -1;
            page[c] = (uint32_t)x < (uint32_t)p.n_pages ? x : -1;
        }
        asm volatile("" : "+v"(page[0]), "+v"(page[1]));      // (here before the loop goes on: see request_keys)
    };
    // A tile: its units' first rows, how many rows of each there are (0: none), and where they are in elements from the head's first page.
    struct Tile { int row[2], rows[2]; int64_t at[2]; };
    auto tile_at = [&](int n) {
        Tile x;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int pg = __builtin_amdgcn_readlane(page[c], n);
            x.row[c] = __builtin_amdgcn_readlane(first[c], n);
            int rows = min(hi - x.row[c], 16);
            asm("" : "+s"(rows));
            x.rows[c] = pg < 0 ? 0 : max(rows, 0);
            x.at[c] = pg < 0 ? 0 : (int64_t)pg * p.s_p + (int64_t)(x.row[c] & in_page) * kD;
        }
        return x;
    };
    auto buffer = [&](const uint16_t* base, const Tile& x, int c) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(base + x.at[c]), 0, x.rows[c] * (kD * 2), 0x00020000);
    };
    TileRows<kBf16> rows;
    auto ask_keys = [&](const Tile& x) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const __amdgpu_buffer_rsrc_t r = buffer(k, x, c);
#pragma unroll
            for (int s = 0; s < 4; ++s) rows.k[c][s] = __builtin_amdgcn_raw_buffer_load_b128(r, col * (kD * 2) + operand_dim<false>(s, gr) * 2, 0, kStreamAux);
        }
    };
    auto ask_values = [&](const Tile& x) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const __amdgpu_buffer_rsrc_t r = buffer(v, x, c);
#pragma unroll
            for (int e = 0; e < 4; ++e) rows.v[4 * c + e] = __builtin_amdgcn_raw_buffer_load_b128(r, (4 * gr + e) * (kD * 2) + 16 * col, 0, kStreamAux);
        }
    };

    ColState st;
    st.clear();
    int t = split * W + w, n = 0;
    Tile now{};
    if (t < tiles) {
        look(t);
        now = tile_at(0);
        ask_keys(now);
        ask_values(now);
    }
    queries_here(q);
    for (; t < tiles; t += step) {
        float s[2][4];
        tile_scores<kBf16>(rows, q, s);
        if (++n == 64) { look(t + step); n = 0; }
        const Tile next = tile_at(n);         // (past the last tile: nothing)
        ask_keys(next);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = fmaf(bend<CAP>(s[x][i], form), form.a, form.b);
                if constexpr (SLOPE) s[x][i] = fmaf(-slope, fabsf((float)(me.pos - now.row[x] - 4 * gr) - (float)i), s[x][i]);
            }
        bool masked = false;
#pragma unroll
        for (int x = 0; x < 2; ++x) masked = masked || now.rows[x] < 16 || now.row[x] < in_lo || now.row[x] + 16 > in_hi;
        auto sees = [&](int x, int j) { return now.rows[x] != 0 && j >= me.lo && j < me.hi; };
        if (masked) {
            asm volatile("" ::: "memory");    // (a branch: most tiles have nothing to mask)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = sees(x, now.row[x] + 4 * gr + i) ? s[x][i] : -INFINITY;
        }
        tile_softmax(st, s);
        bf16x8 ph, pl;
        weight_operands(s, ph, pl);
        bool bad = false;
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bad = bad || has_non_finite(rows.v[e]);
            if (bad) {
#pragma unroll
                for (int e = 0; e < 8; ++e) drop_non_finite(rows.v[e]);
            }
        }
        tile_output<kBf16>(rows, st, ph, pl);
        if (__any(bad)) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
                for (int i = 0; i < now.rows[x]; ++i) {
                    if (!sees(x, now.row[x] + i)) continue;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u32x4 u = *reinterpret_cast<const u32x4*>(v + now.at[x] + (int64_t)i * kD + 8 * (4 * gr + r));
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            st.o[2 * e][r] += only_non_finite(bf16_lo(u[e]));
                            st.o[2 * e + 1][r] += only_non_finite(bf16_hi(u[e]));
                        }
                    }
                }
        }
        ask_values(next);
        now = next;
    }

    __shared__ __attribute__((aligned(16))) ColMergeLds<W, 16> lds;
    __shared__ float sInv[16];
    if (partial) {
        // (columns of one pair and part side by side)
        const int64_t at = CHOSEN ? (int64_t)slot * p.G : ((int64_t)g * p.splits * (SHARED ? 1 : p.batch) + slot) * (SHARED ? p.rows : p.n_new * p.G);
        merge_columns(lds, st, n_rows,
                      [&](int x, int d, float o0, float o1, float) {
                          *reinterpret_cast<float2*>(p.part_o + (at + x) * kD + d) = make_float2(o0, o1);
                      },
                      [&](int x, float m, float l) {
                          *reinterpret_cast<float2*>(p.part_ml + (at + x) * 2) = make_float2(m * kLog2e, l);
                      });
        return;
    }
    if constexpr (SHARED) return;             // (never: the shared rows' results are joined)
    auto out_row = [&](int x) { const int i = x / p.G; return ((int64_t)b * p.n_new + token + i) * p.Hq + g * p.G + (x - i * p.G); };
    float* o = &lds.o[0][0][0];
    merge_columns(lds, st, n_rows,
                  [&](int x, int d, float o0, float o1, float) { o[x * kD + d] = o0; o[x * kD + d + 1] = o1; },
                  [&](int x, float m, float l) {
                      sInv[x] = l == 0.f ? 0.f : 1.f / l;
                      if (p.lse != nullptr) p.lse[out_row(x)] = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l) * (1.f / kLog2e);
                  });
    __syncthreads();
    for (int x = threadIdx.x; x < n_rows * (kD / 2); x += W * 64) {
        const int r = x / (kD / 2), d = 2 * (x % (kD / 2));
        *reinterpret_cast<uint32_t*>(p.out + out_row(r) * kD + d) = pack_bf16(o[r * kD + d] * sInv[r], o[r * kD + d + 1] * sInv[r]);
    }
}

// Where the partial results of a row are: numbers at, at + step, .. of them.
struct PartSource { const float *o, *ml; const int32_t* parts; int32_t rows_of, cols, splits, row_tiles, rows, batch; };
struct PartRow { int64_t at; int step, n; };
__device__ __forceinline__ PartRow part_row(const PartSource& s, const PromptParams& p, int b, int g, int row) {
    const int per = p.n_new * p.G;
    if (s.rows_of == kRowsChosen) {
        const int i = (uint32_t)row / (uint32_t)p.G;
        return {(((int64_t)b * p.n_new + i) * p.Hkv + g) * s.splits * p.G + (row - i * p.G), p.G, s.splits};
    }
    const bool shared = s.rows_of == kRowsShared;
    const int64_t pair = shared ? g : (int64_t)b * p.Hkv + g;
    const int r = shared ? b * per + row : row;
    if (s.cols) return {((int64_t)g * s.splits * (shared ? 1 : p.batch) + s.parts[2 * pair]) * s.rows + r, s.rows, s.parts[2 * pair + 1]};
    return {(pair * s.rows + r) * s.splits, 1, s.parts[pair * s.row_tiles + r / kPromptRows]};
}

// Joins the parts of a row, sum_s 2^(m_s - m) (l_s, o_s): a wavefront each.  SOURCES = 2: those over the shared rows, then those over the sequence's own.
template <int SOURCES>
__global__ __launch_bounds__(256)
void paged_merge_kernel(const PromptParams p, const PartSource s0, const PartSource s1) {
    constexpr int N = SOURCES * kMaxSplits;
    const int g = blockIdx.y, b = blockIdx.z, w = threadIdx.x >> 6, lane = threadIdx.x & 63, row = blockIdx.x * 4 + w;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    __shared__ float sW[4][N];
    const Tokens tok = tokens_of(p, b);
    if (row >= tok.n * p.G) return;
    const PartRow r0 = part_row(s0, p, b, g, row);
    PartRow r1{0, 0, 0};
    if constexpr (SOURCES == 2) r1 = part_row(s1, p, b, g, row);
    if (SOURCES == 1 && p.joined == 0 && !s0.cols && s0.rows_of == kRowsPaged && r0.n == 1) return;      // (the output is there already)
    float m[N / 64], l[N / 64], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) {
        const int s = lane + 64 * i;
        float2 ml = make_float2(-INFINITY, 0.f);
        if (s < r0.n) ml = *reinterpret_cast<const float2*>(s0.ml + (r0.at + (int64_t)s * r0.step) * 2);
        else if (SOURCES == 2 && s - r0.n < r1.n) ml = *reinterpret_cast<const float2*>(s1.ml + (r1.at + (int64_t)(s - r0.n) * r1.step) * 2);
        m[i] = ml.x; l[i] = ml.y;
        top = fmaxf(top, ml.x);
    }
    top = wave_max(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) {
        const float a = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top);
        sum = fmaf(a, l[i], sum);
        sW[w][lane + 64 * i] = a;
    }
    sum = wave_sum(sum);
    wave_lds_sync();
    float o0 = 0.f, o1 = 0.f;
    auto add = [&](const float* from_o, const PartRow& r, int w0) {
        const float2* from = reinterpret_cast<const float2*>(from_o + r.at * kD) + lane;
        for (int s = 0; s < r.n; s += 8) {
            float2 v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = from[(int64_t)min(s + i, r.n - 1) * r.step * (kD / 2)];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = s + i < r.n ? sW[w][w0 + s + i] : 0.f;
                if (a != 0.f) { o0 = fmaf(a, v[i].x, o0); o1 = fmaf(a, v[i].y, o1); }      // (a part without rows left nothing)
            }
        }
    };
    add(s0.o, r0, 0);
    if constexpr (SOURCES == 2) add(s1.o, r1, r0.n);
    const int i = (uint32_t)row / (uint32_t)p.G;
    const int64_t to = ((int64_t)b * p.n_new + i) * p.Hq + g * p.G + (row - i * p.G);
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    reinterpret_cast<uint32_t*>(p.out + to * kD)[lane] = pack_bf16(o0 * inv, o1 * inv);
    if (lane == 0 && p.lse != nullptr) p.lse[to] = sum == 0.f ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
}

// ---- host side ----
static int cap_of(const rk_prompt_scores* s) { return !s || s->cap == 0.f ? kNoCap : s->cap <= kNearCapMost ? kNearCap : kFarCap; }
using PagedKernel = void (*)(const PromptParams);
template <int W, int ROWS> static PagedKernel cols_form(int cap, bool slope) {
    switch (cap) {
        case kNearCap: return slope ? paged_cols_kernel<W, kNearCap, true, ROWS> : paged_cols_kernel<W, kNearCap, false, ROWS>;
        case kFarCap: return slope ? paged_cols_kernel<W, kFarCap, true, ROWS> : paged_cols_kernel<W, kFarCap, false, ROWS>;
        default: return slope ? paged_cols_kernel<W, kNoCap, true, ROWS> : paged_cols_kernel<W, kNoCap, false, ROWS>;
    }
}
template <int ROWS> static PagedKernel tile_form(int cap, bool slope) {
    switch (cap) {
        case kNearCap: return slope ? prompt_tile_kernel<1, kNearCap, true, ROWS> : prompt_tile_kernel<1, kNearCap, false, ROWS>;
        case kFarCap: return slope ? prompt_tile_kernel<1, kFarCap, true, ROWS> : prompt_tile_kernel<1, kFarCap, false, ROWS>;
        default: return slope ? prompt_tile_kernel<1, kNoCap, true, ROWS> : prompt_tile_kernel<1, kNoCap, false, ROWS>;
    }
}

// Rows of partial results that a launch over `pairs` of `rows` rows each and up to max_len cache rows can leave: it splits them only where it has at
// most kPromptTarget workgroups of at most kPromptRows rows each.
static int64_t paged_partials(int64_t pairs, int64_t rows, int64_t max_len) {
    const int64_t most = (int64_t)kPromptTarget * kPromptRows + pairs * rows, all = pairs * rows * ((max_len + kMinChunk - 1) / kMinChunk);
    return all < most ? all : most;
}
static int64_t paged_counts(int64_t pairs, int64_t rows) { return pairs * (rows / kPromptRows + 2); }
static size_t paged_scratch(int64_t pairs, int64_t rows, int64_t max_len) {
    return align_up(((size_t)paged_partials(pairs, rows, max_len) * (kD + 2) + paged_counts(pairs, rows)) * sizeof(float), 256);
}

// What all three calls ask of their arguments.
static int check_paged(const rk_geom* geom, const void* q, int64_t q_b, int64_t q_t, int32_t n_new, const rk_pages* pages, const int32_t* table, int32_t width,
                       const int32_t* seq_lens, const rk_prompt_scores* scores, const void* out) {
    int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!q || !out || !seq_lens || n_new <= 0 || !aligned16(q) || !aligned16(out)) return RK_ERR_INVALID_ARG;
    if (q_b < 0 || q_t < 0 || q_b % 8 != 0 || q_t % 8 != 0) return RK_ERR_INVALID_ARG;
    if (scores && !(scores->cap >= 0.f && isfinite(scores->cap))) return RK_ERR_INVALID_ARG;
    if ((rc = check_pages(pages, true, false)) != RK_OK || (rc = check_table(pages, table, width)) != RK_OK) return rc;
    return (int64_t)n_new * (geom->n_q_heads / geom->n_kv_heads) > INT32_MAX - 128 ? RK_ERR_UNSUPPORTED : RK_OK;
}
static PromptParams paged_params(const rk_geom* geom, const void* q, int64_t q_b, int64_t q_t, int32_t n_new, const rk_pages* pages, const int32_t* table,
                                 int32_t width, const int32_t* seq_lens, const int32_t* new_lens, const rk_prompt_scores* scores, void* out, float* lse,
                                 const int32_t* pred, int32_t pred_val) {
    PromptParams p{};
    p.q = (const uint16_t*)q; p.q_b = q_b; p.q_t = q_t;
    p.k = (const uint16_t*)pages->k; p.v = (const uint16_t*)pages->v; p.s_h = pages->stride_h; p.s_p = pages->stride_p;
    p.table = table; p.width = width; p.n_pages = pages->n_pages; p.shift = page_shift(pages->page);
    p.cap_rows = width * pages->page; p.max_len = p.cap_rows;
    p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.n_new = n_new; p.Hq = geom->n_q_heads; p.Hkv = geom->n_kv_heads; p.G = p.Hq / p.Hkv; p.batch = geom->batch;
    p.scale = geom->scale;
    if (scores) { p.cap = scores->cap; p.slopes = scores->slopes; p.first = scores->first; p.end = scores->end; }
    p.out = (uint16_t*)out; p.lse = lse;
    p.pred = pred; p.pred_val = pred_val;
    p.first_round = INT32_MAX;
    return p;
}
// The partial results' place in [scratch, scratch + bytes): false if they do not fit.
static bool place_parts(PromptParams& p, const PromptPlan& plan, int64_t pairs, int64_t rows, char* scratch, size_t bytes) {
    const size_t n = (size_t)pairs * rows * plan.splits, counts = (size_t)pairs * (plan.cols ? 2 : plan.row_tiles);
    if (!scratch || ((uintptr_t)scratch & 255u) != 0 || bytes < (n * (kD + 2) + counts) * sizeof(float)) return false;
    p.part_o = (float*)scratch;
    p.part_ml = p.part_o + n * kD;
    p.parts = (int32_t*)(p.part_ml + n * 2);
    p.cols = plan.cols ? 1 : 0;
    return true;
}
static PartSource source_of(const PromptParams& p, int rows_of, int rows) {
    return {p.part_o, p.part_ml, p.parts, rows_of, p.cols, p.splits, p.row_tiles, rows, p.batch};
}
static void set_plan(PromptParams& p, const PromptPlan& plan) { p.splits = plan.splits; p.row_tiles = plan.row_tiles; p.split_tiles = plan.split_tiles; }
template <int ROWS>
static int launch_rows(PromptParams& p, const PromptPlan& plan, int64_t pairs, int cap, bool slope, hipStream_t st) {
    if (plan.cols) {
        auto kernel = plan.alone && ROWS == kRowsPaged ? cols_form<kColAlone, kRowsPaged>(cap, slope) : cols_form<kColWaves, ROWS>(cap, slope);
        hipLaunchKernelGGL(kernel, dim3(plan.splits, p.Hkv, ROWS == kRowsShared ? 1 : p.batch), dim3((plan.alone && ROWS == kRowsPaged ? kColAlone : kColWaves) * 64), 0, st, p);
    } else {
        auto kernel = plan.wide && ROWS == kRowsPaged ? prompt_tile_kernel<2, kNoCap, false, kRowsPaged> : tile_form<ROWS>(cap, slope);
        const int64_t total = pairs * plan.row_tiles * plan.splits;
        // (the second workgroup of a compute unit in the opposite order: see rk_prompt_attn)
        p.first_round = !plan.wide && total <= 2 * kComputeUnits ? (int)((kComputeUnits + pairs - 1) / pairs) : INT32_MAX;
        hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(256), 0, st, p);
    }
    return launch_status();
}
static dim3 merge_grid(const PromptParams& p) { return dim3((unsigned)((p.n_new * p.G + 3) / 4), p.Hkv, p.batch); }

}  // namespace rk

using namespace rk;

extern "C" int rk_paged_attn(const rk_geom* geom, const void* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_new, const rk_pages* pages,
                             const int32_t* table, int32_t table_width, const int32_t* seq_lens, const int32_t* new_lens, int32_t max_len,
                             const rk_prompt_scores* scores, void* out, float* lse, const int32_t* pred, int32_t pred_val,
                             void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_paged(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, scores, out);
    if (rc != RK_OK) return rc;
    if (max_len <= 0) return RK_ERR_INVALID_ARG;
    PromptParams p = paged_params(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, new_lens, scores, out, lse, pred, pred_val);
    if (max_len < p.max_len) p.max_len = max_len;
    const int cap = cap_of(scores);
    const bool slope = (scores && scores->slopes) || (geom->scale == 0.f && cap == kNoCap);
    const int64_t pairs = (int64_t)p.batch * p.Hkv, rows = (int64_t)n_new * p.G;
    const PromptPlan plan = prompt_plan(geom, n_new, p.max_len, cap == kNoCap && !slope);
    if (pairs * plan.row_tiles * plan.splits > INT32_MAX / 2) return RK_ERR_UNSUPPORTED;
    set_plan(p, plan);
    if (plan.splits > 1) {
        if (!place_parts(p, plan, pairs, rows, (char*)workspace, workspace_bytes)) return RK_ERR_WORKSPACE;
        p.ragged = plan.cols ? ragged_batch_of(geom) : 0;
    }
    hipStream_t st = (hipStream_t)stream;
    if ((rc = launch_rows<kRowsPaged>(p, plan, pairs, cap, slope, st)) != RK_OK || plan.splits == 1) return rc;
    const PartSource s = source_of(p, kRowsPaged, (int)rows);
    hipLaunchKernelGGL(paged_merge_kernel<1>, merge_grid(p), dim3(256), 0, st, p, s, s);
    return launch_status();
}

extern "C" size_t rk_prefix_workspace_bytes(const rk_geom* geom, int32_t n_new, int32_t max_prefix, int32_t max_own) {
    if (check_geom(geom) != RK_OK || n_new <= 0 || max_prefix <= 0 || max_own <= 0) return 0;
    const int64_t rows = (int64_t)n_new * (geom->n_q_heads / geom->n_kv_heads);
    return paged_scratch(geom->n_kv_heads, rows * geom->batch, max_prefix) + paged_scratch((int64_t)geom->batch * geom->n_kv_heads, rows, max_own);
}

extern "C" int rk_prefix_attn(const rk_geom* geom, const void* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_new, const rk_pages* pages,
                              const int32_t* prefix_table, int32_t prefix_width, const int32_t* prefix_len, int32_t max_prefix,
                              const int32_t* table, int32_t table_width, const int32_t* seq_lens, const int32_t* new_lens, int32_t max_own,
                              const rk_prompt_scores* scores, void* out, float* lse, const int32_t* pred, int32_t pred_val,
                              void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_paged(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, scores, out);
    if (rc != RK_OK) return rc;
    if ((rc = check_table(pages, prefix_table, prefix_width)) != RK_OK) return rc;
    if (!prefix_len || max_prefix <= 0 || max_own <= 0) return RK_ERR_INVALID_ARG;
    PromptParams own = paged_params(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, new_lens, scores, out, lse, pred, pred_val);
    const int64_t rows = (int64_t)n_new * own.G, pairs = (int64_t)own.batch * own.Hkv, all_rows = rows * own.batch;
    if (all_rows > INT32_MAX - 128) return RK_ERR_UNSUPPORTED;
    own.bound = prefix_len;
    own.most_shared = (int32_t)((int64_t)prefix_width * pages->page < max_prefix ? prefix_width * pages->page : max_prefix);
    own.most_own = max_own < own.cap_rows ? max_own : own.cap_rows;
    if ((int64_t)own.most_shared + own.most_own > INT32_MAX - 2 * kMaxChunks * kMinChunk) return RK_ERR_UNSUPPORTED;
    own.joined = 1;
    PromptParams all = own;
    all.table = prefix_table; all.width = prefix_width;
    all.cap_rows = all.max_len = INT32_MAX - 2 * kMaxChunks * kMinChunk;      // (what a token sees of the prefix ends at *prefix_len)
    all.rows = (int32_t)all_rows;
    const int cap = cap_of(scores);
    const bool slope = (scores && scores->slopes) || (geom->scale == 0.f && cap == kNoCap);
    PromptPlan plan_all = prompt_plan_of(own.Hkv, all_rows, own.most_shared, false, false);
    PromptPlan plan_own = prompt_plan_of(pairs, rows, own.most_own, false, false);
    plan_all.alone = plan_own.alone = false;
    if (pairs * plan_own.row_tiles * plan_own.splits > INT32_MAX / 2 || own.Hkv * (int64_t)plan_all.row_tiles * plan_all.splits > INT32_MAX / 2) return RK_ERR_UNSUPPORTED;
    set_plan(all, plan_all);
    set_plan(own, plan_own);
    const size_t first = paged_scratch(own.Hkv, all_rows, own.most_shared);
    if (workspace_bytes < first || !place_parts(all, plan_all, own.Hkv, all_rows, (char*)workspace, first) ||
        !place_parts(own, plan_own, pairs, rows, (char*)workspace + first, workspace_bytes - first)) return RK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    if ((rc = launch_rows<kRowsShared>(all, plan_all, own.Hkv, cap, slope, st)) != RK_OK) return rc;
    if ((rc = launch_rows<kRowsPaged>(own, plan_own, pairs, cap, slope, st)) != RK_OK) return rc;
    hipLaunchKernelGGL(paged_merge_kernel<2>, merge_grid(own), dim3(256), 0, st, own, source_of(all, kRowsShared, (int)all_rows), source_of(own, kRowsPaged, (int)rows));
    return launch_status();
}

extern "C" size_t rk_sparse_workspace_bytes(const rk_geom* geom, int32_t n_new, int32_t k, int32_t page) {
    if (check_geom(geom) != RK_OK || n_new <= 0 || k <= 0 || (page != 16 && page != 32 && page != 64 && page != 128)) return 0;
    return paged_scratch((int64_t)geom->batch * n_new * geom->n_kv_heads, geom->n_q_heads / geom->n_kv_heads, (int64_t)k * page);
}

extern "C" int rk_sparse_attn(const rk_geom* geom, const void* q, int64_t q_stride_b, int64_t q_stride_t, int32_t n_new, const rk_pages* pages,
                              const int32_t* table, int32_t table_width, const int32_t* idx, int32_t k,
                              const int32_t* seq_lens, const int32_t* new_lens, const rk_prompt_scores* scores, void* out, float* lse,
                              const int32_t* pred, int32_t pred_val, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_paged(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, scores, out);
    if (rc != RK_OK) return rc;
    if (!idx || ((uintptr_t)idx & 3u) || k <= 0) return RK_ERR_INVALID_ARG;
    const int64_t chosen = (int64_t)k * pages->page;
    if (chosen > INT32_MAX - 2 * kMaxChunks * kMinChunk) return RK_ERR_UNSUPPORTED;
    PromptParams p = paged_params(geom, q, q_stride_b, q_stride_t, n_new, pages, table, table_width, seq_lens, new_lens, scores, out, lse, pred, pred_val);
    p.idx = idx; p.n_idx = k;
    const int cap = cap_of(scores);
    const bool slope = (scores && scores->slopes) || (geom->scale == 0.f && cap == kNoCap);
    const int64_t pairs = (int64_t)p.batch * n_new * p.Hkv;
    PromptPlan plan = prompt_plan_of(pairs, p.G, chosen, false, false);
    plan.alone = false;
    if (pairs * plan.splits > INT32_MAX / 2) return RK_ERR_UNSUPPORTED;
    set_plan(p, plan);
    if (plan.splits > 1 && !place_parts(p, plan, pairs, p.G, (char*)workspace, workspace_bytes)) return RK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    hipLaunchKernelGGL((cols_form<kColWaves, kRowsChosen>(cap, slope)), dim3((unsigned)(pairs * plan.splits)), dim3(kColWaves * 64), 0, st, p);
    if ((rc = launch_status()) != RK_OK || plan.splits == 1) return rc;
    const PartSource s = source_of(p, kRowsChosen, p.G);
    hipLaunchKernelGGL(paged_merge_kernel<1>, merge_grid(p), dim3(256), 0, st, p, s, s);
    return launch_status();
}
