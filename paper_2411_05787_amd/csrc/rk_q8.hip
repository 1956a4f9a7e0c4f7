// rk_full_attn_q8 and rk_gather_small_kv_q8: the full step and the refresh over a cache of 8 bits.
//
// The step streams 256 bytes of a KV head's row instead of 512 and is bound by that: what the matrix cores and the conversions take
// fits behind it.  The scale of a block of rows multiplies its scores (K) and its weights (V), never the rows.  Split, work shares of
// ragged batches and the layout of the partial results are those of the step over the bf16 cache (rk_attn_common.h).
#include "rk_cols.h"

namespace rk {

// Four weights of a row, which starts at any multiple of four bytes: memory takes them as one access all the same.  Those that a second
// launch reads are streamed: stores that the caches keep cost 131072 rows 64.9 us instead of 60.9 (45 without weights at all).  Where the workgroup that wrote
// them reads them, the caches keep them: 64 sequences of 4000 rows 131.1 -> 128.0, of 1000 41.1 -> 39.9.
typedef float Floats4 __attribute__((ext_vector_type(4), aligned(4)));
struct Q8Rows { const uint8_t *k, *v; const float *ks, *vs; const uint16_t *kt, *vt; int64_t s_b; int32_t s_h, blocks, shift; };

// Workgroups per (sequence, KV head): with the scores returned as the step over the bf16 cache has it, without them one to a compute unit, as
// no stores come between the requests.  us by workgroups in all (256 / 512 / 768 / 1024), 32 heads over 8, e4m3: with weights 32777 rows 21.6 /
// 21.6 / 22.3 / 24.0, 65536 36.4 / 35.7 / 36.2 / 34.2, 131072 70.4 / 68.5 / 67.3 / 60.8, without 65536 26.9 / 27.0 / 28.7 / 28.8, 4 sequences of
// 32768 45.6 / 47.1 / 47.6 / 48.2, 16 ragged ones of up to 16384, 28 over 4, int8 37.8 / 35.6 / 36.1 / 38.6.
static int q8_split_workgroups(const rk_geom* g, int32_t max_len, bool weights) {
    return split_workgroups(max_len, (int64_t)g->batch * g->n_kv_heads, kMaxChunks, weights ? emit_split_target(g, max_len) : kComputeUnits);
}

// One workgroup of kAlone wavefronts to a (sequence, KV head), and no launch behind it: where the pairs fill the chip once or twice and no sharing by
// length is there to lose, or the sequences are so short that a second launch costs more than the rows.  us, e4m3, 32 heads over 8 unless said
// (split / alone): without weights 4 sequences of 500 rows 9.1 / 8.4, of 1000 9.3 / 11.6, 16 of 500 12.5 / 9.6, of 1000 14.6 / 13.6, of 1500 17.3 / 17.5, 32
// of 500 16.5 / 10.0, of 2000 30.5 / 24.7, 64 of 1000 34.9 / 28.9, of 4000 92 / 85, one of 500 8.1 / 8.3, but 100 of 1000 49.8 / 52.5; with weights, which
// the workgroup goes over once more, 32 of 500 19.6 / 13.2, 64 of 4000 139 / 128, 66 of 1000, 28 heads over 4, 47.4 / 36.4, of 4000 87 / 108.
constexpr int kAlone = 16;
static bool q8_alone(const rk_geom* g, int32_t max_len, bool weights) {
    const int64_t pairs = (int64_t)g->batch * g->n_kv_heads;
    if (pairs < 32 || pairs > 2 * kComputeUnits) return false;
    return max_len <= (pairs > 64 ? 8 * pairs : 512) || (!weights && pairs >= kComputeUnits && ragged_batch_of(g) == 0);
}

// log-sum-exp as hi + lo, of a maximum and a sum (no rows: -inf; a NaN among the sums: NaN).
__device__ __forceinline__ float2 lse_of(float m, double l) {
    if (l == 0.0) return make_float2(-INFINITY, 0.f);
    const double x = (double)m + log(l);
    const float hi = (float)x;
    return make_float2(hi, (float)(x - (double)hi));
}

// Tiles of a sequence of len rows (of which the call looks at the first n): those of whole blocks, then those of the tail. ALONE: one workgroup of
// W wavefronts has all rows, and does what the launch behind would. 32777 rows, with weights: 15.5 us (4.6 TB/s with what it writes); 131072: 50.4
// us (5.7 TB/s); a tile's requests are ahead by one tile, more does not help (measured before the scores were streamed: 131072 rows
// 65.0 -> 64.5 in all, 32777 21.0 -> 22.8).
template <int FORMAT, bool EMIT, int W, bool ALONE>
__global__ __launch_bounds__(W * 64, ALONE ? 1 : 2)
void q8_attn_kernel(const AttnParams p, const Q8Rows c8) {
    const int g = blockIdx.y;
    int b = blockIdx.z, c = blockIdx.x, nchunks = 1;
    if (!ALONE && p.ragged_batch != 0) {
        const RaggedSlot slot = ragged_slot<false>(p, p.seq_lens, (int)(blockIdx.z * gridDim.x + blockIdx.x));
        if (slot.b < 0) return;
        b = slot.b; c = slot.c; nchunks = slot.nchunks;
    }
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const int len = __builtin_amdgcn_readfirstlane(min(max(p.seq_lens[b], 0), p.cap2)), n = min(len, p.max_rows2);
    if (!ALONE && p.ragged_batch == 0) {
        nchunks = active_workgroups(n, p.nch);
        if (c >= nchunks) return;
    }
    const int G = p.Hq / p.Hkv;
    const int64_t bg = (int64_t)b * p.Hkv + g;
    if (!ALONE && p.ragged_batch != 0 && c == 0 && threadIdx.x == 0) store_chunks(p.counters, bg, nchunks);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, gr = lane >> 4;
    const int full = len >> c8.shift << c8.shift, main_rows = min(n, full);
    const int main_tiles = (main_rows + kTileRows - 1) / kTileRows, tiles = main_tiles + (n - main_rows + kTileRows - 1) / kTileRows;
    const uint8_t* k = c8.k + b * c8.s_b + (int64_t)g * c8.s_h;
    const uint8_t* v = c8.v + b * c8.s_b + (int64_t)g * c8.s_h;
    const float* ks = c8.ks + bg * c8.blocks;
    const float* vs = c8.vs + bg * c8.blocks;

    bf16x8 q[4];                              // (columns beyond the group repeat its last head: they are never looked at)
    const uint16_t* qr = p.q + ((int64_t)b * p.Hq + g * G + min(col, G - 1)) * kD;
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const bf16x8*>(qr + operand_dim<true>(s, gr));
    __builtin_amdgcn_sched_barrier(0);

    ColState st;
    st.clear();
    // (where scores are returned: this lane's row of them, and where it has 16 bytes of a whole tile's line of 128)
    float* wline = EMIT ? p.weights + ((int64_t)b * p.Hq + g * G + (col >= G ? min(col - G, G - 1) : col)) * p.w_stride + (col >= G ? 16 : 0) : nullptr;
    float* wrow = EMIT ? p.weights + ((int64_t)b * p.Hq + g * G + min(col, G - 1)) * p.w_stride : nullptr;
    // scores of rows first .. first + 31, the first `rows` of which exist
    auto finish_scores = [&](float (&s)[2][4], int first, int rows, float k0, float k1) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
#pragma unroll
            for (int i = 0; i < 4; ++i) s[x][i] *= x ? k1 : k0;
        }
        if (EMIT && rows >= kTileRows) {      // (the same for the whole wavefront)
            // the second block's scores to the lanes behind the group's: whole lines of 128 bytes leave in one store
            const int from = (lane & 48) + (col >= G ? col - G : col);
            Floats4 v;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float up = __int_as_float(__builtin_amdgcn_ds_bpermute(from * 4, __float_as_int(s[1][i])));
                v[i] = col < G ? s[0][i] : up;
            }
            if (col < 2 * G) {
                Floats4* to = reinterpret_cast<Floats4*>(wline + first + 4 * gr);
                if constexpr (ALONE) *to = v;
                else __builtin_nontemporal_store(v, to);
            }
        } else if (EMIT && col < G) {
            float* to = wrow + first + 4 * gr;
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) if (16 * x + 4 * gr + i < rows) to[16 * x + i] = s[x][i];
        }
        if (rows < kTileRows) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = 16 * x + 4 * gr + i < rows ? s[x][i] : -INFINITY;
        }
        tile_softmax(st, s);
    };
    const int t0 = c * W + w, step = nchunks * W;
    TileRows<FORMAT> rows;
    // the scales of a tile's two blocks of 16 rows, requested with its rows
    struct Scales { float k0, k1, v0, v1; };
    auto request_scales = [&](int t) {
        const int x = min(t * kTileRows, main_rows - 1) >> c8.shift, y = min(t * kTileRows + 16, main_rows - 1) >> c8.shift;
        typedef const __attribute__((address_space(4))) float* Scalar;      // (nothing writes them meanwhile: scalar loads)
        return Scales{((Scalar)ks)[x], ((Scalar)ks)[y], ((Scalar)vs)[x], ((Scalar)vs)[y]};
    };
    Scales sc{};
    int t = t0;
    if (t < main_tiles) {
        request_keys<FORMAT, true>(rows, k, t * kTileRows, main_rows - t * kTileRows);
        request_values<FORMAT>(rows, v, t * kTileRows, main_rows - t * kTileRows);
        sc = request_scales(t);
    }
    queries_here(q);
    // The next tile's rows are requested as soon as the registers of this one's are consumed, past the last tile as well (nothing then): a
    // request that is not always made would leave the compiler to wait for all that are in flight.
    for (; t < main_tiles; t += step) {
        const int first = t * kTileRows;
        float s[2][4];
        tile_scores<FORMAT>(rows, q, s);
        const int next = (t + step) * kTileRows;      // (no more than 2 kMaxChunks * kMinChunk beyond the rows there are: see check_kv8)
        request_keys<FORMAT, true>(rows, k, next, main_rows - next);
        const Scales now = sc;
        sc = request_scales(t + step);
        finish_scores(s, first, main_rows - first, now.k0 * p.scale, now.k1 * p.scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[0][i] *= now.v0; s[1][i] *= now.v1; }      // (rows that are not there: 0, and the last row's scale)
        bf16x8 hi, lo;
        weight_operands(s, hi, lo);
        tile_output<FORMAT>(rows, st, hi, lo);
        request_values<FORMAT>(rows, v, next, main_rows - next);
    }
    for (; t < tiles; t += step) {            // the block that is not full: bf16
        const int at = (t - main_tiles) * kTileRows, left = n - main_rows - at;
        const uint16_t* kt = c8.kt + (bg << c8.shift) * kD;
        const uint16_t* vt = c8.vt + (bg << c8.shift) * kD;
        TileRows<kBf16> x;
        request_keys<kBf16, true>(x, kt, at, left);
        request_values<kBf16>(x, vt, at, left);
        float s[2][4];
        tile_scores<kBf16>(x, q, s);
        finish_scores(s, main_rows + at, left, p.scale, p.scale);
        bf16x8 hi, lo;
        weight_operands(s, hi, lo);
        tile_output<kBf16>(x, st, hi, lo);
    }

    __shared__ __attribute__((aligned(16))) ColMergeLds<W, RK_MAX_GROUP> lds;
    if constexpr (ALONE) {
        __shared__ float2 sLse[RK_MAX_GROUP];
        const int64_t head0 = (int64_t)b * p.Hq + g * G;
        merge_columns(lds, st, G,
                      [&](int x, int d, float o0, float o1, float l) {
                          const float inv = l == 0.f ? 0.f : 1.f / l;
                          uint16_t* out = p.out + (head0 + x) * kD + d;
                          out[0] = f32_to_bf16(o0 * inv);      // (out is 2-byte aligned)
                          out[1] = f32_to_bf16(o1 * inv);
                      },
                      [&](int x, float m, float l) {
                          sLse[x] = lse_of(m, (double)l);
                          if (p.lse != nullptr) p.lse[head0 + x] = sLse[x].x;
                      });
        if constexpr (EMIT) {
            __syncthreads();                  // (this workgroup's scores are written)
            float* first = p.weights + head0 * p.w_stride;
            auto normalise = [&](int j) {      // four positions of all heads, requested together
                float v[RK_MAX_GROUP][4];
#pragma unroll
                for (int x = 0; x < RK_MAX_GROUP; ++x) {
                    if (x >= G) break;
#pragma unroll
                    for (int u = 0; u < 4; ++u) if (j + u * (W * 64) < n) v[x][u] = first[x * p.w_stride + j + u * (W * 64)];
                }
#pragma unroll
                for (int x = 0; x < RK_MAX_GROUP; ++x) {
                    if (x >= G) break;
                    const float nl = -sLse[x].x, ll = sLse[x].y;
#pragma unroll
                    for (int u = 0; u < 4; ++u) if (j + u * (W * 64) < n) first[x * p.w_stride + j + u * (W * 64)] = weight_of(v[x][u], nl, ll);
                }
            };
            for (int j = threadIdx.x; j < n; j += 4 * W * 64) normalise(j);
        }
        return;
    }
    float* po = p.part_o + (bg * p.max_chunks + c) * G * kD;
    float* ml = p.part_ml + (bg * kMaxChunks + c) * G * 2;
    merge_columns(lds, st, G,
                  [&](int x, int d, float o0, float o1, float) { *reinterpret_cast<float2*>(po + x * kD + d) = make_float2(o0, o1); },
                  [&](int x, float m, float l) { *reinterpret_cast<float2*>(ml + 2 * x) = make_float2(m, l); });
}

// The launch behind it (5.1 us at 32777 rows, 10.2 at 131072, where it moves 33.5 MB).  Workgroups x < G: the output of query head x of the group,
// four wavefronts with every fourth partial result each.  The others: kWeightTile positions of all G heads, raw scores -> weights in place,
// requested before the log-sum-exps that they wait for are worked out, by a wavefront each.  Every wavefront that needs a head's statistics reduces
// them by itself, without a barrier.
constexpr int kWeightTile = 1024, kOutRound = 16;
struct HeadStats { float M; double L; };
// a[i]: what partial result lane + 64 i weighs.
__device__ __forceinline__ HeadStats head_stats(const AttnParams& p, int G, int64_t bg, int gi, int nchunks, float (&a)[kMaxChunks / 64]) {
    const float* ml = p.part_ml + (bg * kMaxChunks * G + gi) * 2;
    const int lane = threadIdx.x & 63;
    float2 t[kMaxChunks / 64];
#pragma unroll
    for (int i = 0; i < kMaxChunks / 64; ++i)
        t[i] = lane + 64 * i < nchunks ? *reinterpret_cast<const float2*>(ml + (int64_t)(lane + 64 * i) * G * 2) : make_float2(-INFINITY, 0.f);
    float m = fmaxf(fmaxf(t[0].x, t[1].x), fmaxf(t[2].x, t[3].x));
    m = wave_max(m);
    double l = 0.0;
#pragma unroll
    for (int i = 0; i < kMaxChunks / 64; ++i) {
        a[i] = t[i].x == -INFINITY ? 0.f : fast_exp2((t[i].x - m) * kLog2e);
        l += (double)a[i] * (double)t[i].y;
    }
    return {m, wave_sum(l)};
}
static_assert(kMaxChunks == 256, "statistics in four registers to a lane");

__global__ __launch_bounds__(256)
void q8_finish_kernel(const AttnParams p) {
    const int x = blockIdx.x, g = blockIdx.y, b = blockIdx.z, G = p.Hq / p.Hkv;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const int len = clamped_len(p.seq_lens[b], p.cap2, p.max_rows2), j0 = (x - G) * kWeightTile;
    if (x >= G && j0 >= len) return;
    const int64_t bg = (int64_t)b * p.Hkv + g;
    const int nchunks = p.ragged_batch != 0 ? stored_chunks(p.counters, bg) : active_workgroups(len, p.nch);
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int64_t head0 = (int64_t)b * p.Hq + g * G;
    if (x >= G) {
        __shared__ float2 sLse[RK_MAX_GROUP];
        float* rows = p.weights + head0 * p.w_stride + j0;
        const int n = len - j0;
        float v[RK_MAX_GROUP][4];
        const bool vec = n >= kWeightTile;
#pragma unroll
        for (int gi = 0; gi < RK_MAX_GROUP; ++gi) {
            if (gi >= G) break;
            const float* row = rows + gi * p.w_stride;
            if (vec) {
                const Floats4 f = __builtin_nontemporal_load(reinterpret_cast<const Floats4*>(row + 4 * tid));
#pragma unroll
                for (int i = 0; i < 4; ++i) v[gi][i] = f[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) v[gi][i] = tid + 256 * i < n ? row[tid + 256 * i] : 0.f;
            }
        }
        for (int gi = w; gi < G; gi += 4) {
            float a[kMaxChunks / 64];
            const HeadStats hs = head_stats(p, G, bg, gi, nchunks, a);
            const float2 lse = lse_of(hs.M, hs.L);
            if (lane == 0) sLse[gi] = lse;
        }
        __syncthreads();
#pragma unroll
        for (int gi = 0; gi < RK_MAX_GROUP; ++gi) {
            if (gi >= G) break;
            float* row = rows + gi * p.w_stride;
            const float nl = -sLse[gi].x, ll = sLse[gi].y;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[gi][i] = weight_of(v[gi][i], nl, ll);
            if (vec) {
                __builtin_nontemporal_store(Floats4{v[gi][0], v[gi][1], v[gi][2], v[gi][3]}, reinterpret_cast<Floats4*>(row + 4 * tid));
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) if (tid + 256 * i < n) row[tid + 256 * i] = v[gi][i];
            }
        }
        return;
    }
    __shared__ float sW[4][kMaxChunks];
    __shared__ float2 sOut[4][64];
    const float2* po = reinterpret_cast<const float2*>(p.part_o + (bg * p.max_chunks * G + x) * kD) + lane;
    float2 v[kOutRound];
    auto request = [&](int c0) {
#pragma unroll
        for (int u = 0; u < kOutRound; ++u) v[u] = po[(int64_t)min(c0 + 4 * u, nchunks - 1) * G * (kD / 2)];
    };
    request(w);
    float a[kMaxChunks / 64];
    const HeadStats st = head_stats(p, G, bg, x, nchunks, a);
#pragma unroll
    for (int i = 0; i < kMaxChunks / 64; ++i) sW[w][lane + 64 * i] = a[i];
    wave_lds_sync();
    float o0 = 0.f, o1 = 0.f;
    for (int c0 = w; c0 < nchunks; c0 += 4 * kOutRound) {
        if (c0 != w) request(c0);
#pragma unroll
        for (int u = 0; u < kOutRound; ++u) {
            const float wc = c0 + 4 * u < nchunks ? sW[w][c0 + 4 * u] : 0.f;
            o0 = fmaf(wc, v[u].x, o0); o1 = fmaf(wc, v[u].y, o1);
        }
    }
    sOut[w][lane] = make_float2(o0, o1);
    __syncthreads();
    if (w != 0) return;
    const float inv = st.L == 0.0 ? 0.f : 1.f / (float)st.L;
    uint16_t* out = p.out + (head0 + x) * kD + 2 * lane;
    out[0] = f32_to_bf16((sOut[0][lane].x + sOut[1][lane].x + sOut[2][lane].x + sOut[3][lane].x) * inv);      // (out is 2-byte aligned)
    out[1] = f32_to_bf16((sOut[0][lane].y + sOut[1][lane].y + sOut[2][lane].y + sOut[3][lane].y) * inv);
    if (lane == 0 && p.lse != nullptr) p.lse[head0 + x] = lse_of(st.M, st.L).x;
}

// rk_gather_small_kv out of a cache of 8 bits: 16 lanes to a row.  Bound by its reads of 128 bytes out of all of the cache: 16 sequences, 101 MB,
// 21.7 us (4.7 TB/s); 2048 rows 4.2 us, a launch and two dependent reads.
constexpr int kGatherRows8 = 16;
template <int FORMAT>
__global__ __launch_bounds__(256)
void gather_q8_kernel(const rk_kv8 c8, uint16_t* __restrict__ sk, uint16_t* __restrict__ sv, int64_t ss_b, int64_t ss_h,
                      const int32_t* __restrict__ idx, int32_t k, int32_t Hkv, const int32_t* __restrict__ seq_lens,
                      int32_t* __restrict__ tail_start, const int32_t* pred, int32_t pred_val) {
    const int g = blockIdx.y, b = blockIdx.z;
    if (pred != nullptr && pred[b] != pred_val) return;
    const int raw = seq_lens[b];
    if (tail_start != nullptr && blockIdx.x == 0 && g == 0 && threadIdx.x == 0) tail_start[b] = raw;
    const int i = blockIdx.x * kGatherRows8 + (threadIdx.x >> 4);
    if (i >= k) return;
    const int64_t bg = (int64_t)b * Hkv + g;
    const int j = idx[bg * k + i], len = (int)min((int64_t)max(raw, 0), c8.capacity), full = len / c8.block * c8.block;
    if (j < 0 || j >= len) return;
    const int seg = (threadIdx.x & 15) * 8;
    const int64_t to = (int64_t)b * ss_b + (int64_t)g * ss_h + (int64_t)i * kD + seg;
    u32x4 row[2];
    if (j >= full) {
        const int64_t at = (bg * c8.block + (j - full)) * kD + seg;
        row[0] = *reinterpret_cast<const u32x4*>((const uint16_t*)c8.k_tail + at);
        row[1] = *reinterpret_cast<const u32x4*>((const uint16_t*)c8.v_tail + at);
    } else {
        const int64_t at = (int64_t)b * c8.stride_b + (int64_t)g * c8.stride_h + (int64_t)j * kD + seg;
        const int64_t block = bg * (c8.capacity / c8.block) + j / c8.block;
        const uint2 w[2] = {*reinterpret_cast<const uint2*>((const uint8_t*)c8.k + at), *reinterpret_cast<const uint2*>((const uint8_t*)c8.v + at)};
        const float scale[2] = {c8.k_scale[block], c8.v_scale[block]};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            // (a value of the format has at most 8 bits: its product with a power of two is a bf16, with another scale it is rounded)
            const uint32_t v[4] = {pair_of<FORMAT, false>(w[x].x), pair_of<FORMAT, true>(w[x].x), pair_of<FORMAT, false>(w[x].y), pair_of<FORMAT, true>(w[x].y)};
#pragma unroll
            for (int e = 0; e < 4; ++e) row[x][e] = pack_bf16(bf16_lo(v[e]) * scale[x], bf16_hi(v[e]) * scale[x]);
        }
    }
    *reinterpret_cast<u32x4*>(sk + to) = row[0];
    *reinterpret_cast<u32x4*>(sv + to) = row[1];
}

}  // namespace rk

using namespace rk;

extern "C" int rk_full_attn_q8(const rk_geom* geom, const void* q, const rk_kv8* full, const int32_t* seq_lens, int32_t max_len,
                               void* out, float* weights, int64_t w_stride, float* lse, const int32_t* pred, int32_t pred_val,
                               void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!q || !out || !seq_lens || max_len <= 0 || !aligned16(q) || ((uintptr_t)out & 1u)) return RK_ERR_INVALID_ARG;
    if ((rc = check_kv8(full)) != RK_OK) return rc;
    if (weights && (w_stride < max_len || ((uintptr_t)weights & 3u))) return RK_ERR_INVALID_ARG;
    Workspace ws;
    if ((rc = check_workspace(geom, max_len, 0, workspace, workspace_bytes, &ws)) != RK_OK) return rc;
    AttnParams p{};
    p.q = (const uint16_t*)q;
    p.seq_lens = seq_lens; p.max_rows2 = max_len; p.cap2 = (int32_t)full->capacity;
    p.nch = q8_split_workgroups(geom, max_len, weights != nullptr);
    p.Hq = geom->n_q_heads; p.Hkv = geom->n_kv_heads;
    p.scale = geom->scale;
    p.out = (uint16_t*)out;
    p.weights = weights; p.w_stride = w_stride;
    p.lse = lse;
    p.pred = pred; p.pred_val = pred_val;
    p.counters = ws.counters; p.part_ml = ws.part_ml; p.part_o = ws.part_o; p.max_chunks = ws.max_chunks;
    p.ragged_batch = ragged_batch_of(geom); p.share_cap = kMaxChunks;
    const Q8Rows rows{(const uint8_t*)full->k, (const uint8_t*)full->v, full->k_scale, full->v_scale, (const uint16_t*)full->k_tail,
                      (const uint16_t*)full->v_tail, full->stride_b, (int32_t)full->stride_h, (int32_t)(full->capacity / full->block),
                      full->block == 16 ? 4 : full->block == 32 ? 5 : full->block == 64 ? 6 : 7};
    const dim3 grid(p.nch, geom->n_kv_heads, geom->batch);
    const bool e4m3 = full->format == RK_Q8_E4M3;
    if (q8_alone(geom, max_len, weights != nullptr)) {
        auto kernel = e4m3 ? (weights ? q8_attn_kernel<RK_Q8_E4M3, true, kAlone, true> : q8_attn_kernel<RK_Q8_E4M3, false, kAlone, true>)
                           : (weights ? q8_attn_kernel<RK_Q8_INT8, true, kAlone, true> : q8_attn_kernel<RK_Q8_INT8, false, kAlone, true>);
        hipLaunchKernelGGL(kernel, dim3(1, geom->n_kv_heads, geom->batch), dim3(kAlone * 64), 0, (hipStream_t)stream, p, rows);
        return launch_status();
    }
    auto kernel = e4m3 ? (weights ? q8_attn_kernel<RK_Q8_E4M3, true, kColWaves, false> : q8_attn_kernel<RK_Q8_E4M3, false, kColWaves, false>)
                       : (weights ? q8_attn_kernel<RK_Q8_INT8, true, kColWaves, false> : q8_attn_kernel<RK_Q8_INT8, false, kColWaves, false>);
    hipLaunchKernelGGL(kernel, grid, dim3(kColWaves * 64), 0, (hipStream_t)stream, p, rows);
    if ((rc = launch_status()) != RK_OK) return rc;
    const int tiles = weights ? (max_len + kWeightTile - 1) / kWeightTile : 0;
    hipLaunchKernelGGL(q8_finish_kernel, dim3(geom->n_q_heads / geom->n_kv_heads + tiles, geom->n_kv_heads, geom->batch), dim3(256), 0, (hipStream_t)stream, p);
    return launch_status();
}

extern "C" int rk_gather_small_kv_q8(const rk_geom* geom, const rk_kv8* full, const int32_t* idx, int32_t k, rk_kv small,
                                     const int32_t* seq_lens, int32_t* tail_start, const int32_t* pred, int32_t pred_val, void* stream) {
    int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!idx || k <= 0 || !seq_lens) return RK_ERR_INVALID_ARG;
    if ((rc = check_kv8(full)) != RK_OK) return rc;
    if ((rc = check_kv(small)) != RK_OK) return rc;
    if (small.capacity < k) return RK_ERR_INVALID_ARG;
    auto kernel = full->format == RK_Q8_E4M3 ? gather_q8_kernel<RK_Q8_E4M3> : gather_q8_kernel<RK_Q8_INT8>;
    hipLaunchKernelGGL(kernel, dim3((k + kGatherRows8 - 1) / kGatherRows8, geom->n_kv_heads, geom->batch), dim3(256), 0, (hipStream_t)stream,
                       *full, (uint16_t*)small.k, (uint16_t*)small.v, small.stride_b, small.stride_h, idx, k, geom->n_kv_heads, seq_lens,
                       tail_start, pred, pred_val);
    return launch_status();
}
