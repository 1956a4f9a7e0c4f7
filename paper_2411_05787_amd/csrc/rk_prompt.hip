// rk_prompt_attn: attention of the new tokens of each sequence over the bf16 cache that holds them.
//
// The query heads of a group and the new tokens are one axis, row = token * G + head, so a tile of rows shares every K and V row that it
// reads among the group's heads too.  Two kernels:
//   prompt_tile_kernel  128 rows to a workgroup, 64 cache rows at a time through LDS, everything on the matrix cores:
//                       bound by those and by the softmax between the two products;
//   prompt_cols_kernel  up to 16 rows in all (a decode step's token, a few drafted ones): the cache streams past once, bound by memory
//                       (rk_cols.h).
// A row r sees cache rows lo <= j < hi.  Tiles that no row of a workgroup sees are never read; only those that a bound runs through are masked.
// Where there are few rows the cache rows are split over workgroups, and prompt_merge_kernel joins their (maximum, sum, output).
#include "rk_cols.h"

namespace rk {

struct PromptParams {
    const uint16_t* q; int64_t q_b, q_t;
    const uint16_t *k, *v; int64_t s_b, s_h; int32_t cap_rows;
    const int32_t *seq_lens, *new_lens;
    int32_t n_new, max_len, Hq, Hkv, G, batch;
    float scale, cap;
    const float* slopes; const int32_t *first, *end;
    uint16_t* out; float* lse;
    const int32_t* pred; int32_t pred_val;
    int32_t splits, row_tiles, split_tiles;   // at most `splits` parts to a row tile, of no fewer than split_tiles tiles of cache rows
    // partial results, [..][128] and their (maximum in units of ln 2, sum): of row tiles [batch * Hkv][n_new * G][splits], of columns
    // [Hkv][splits * batch][n_new * G]
    float *part_o, *part_ml;
    int32_t* parts;                           // of row tiles [batch * Hkv][row_tiles]: how many (1: the output is there already); of columns
                                              // [batch * Hkv][2]: the first one's number and how many
    int32_t cols, ragged;                     // ragged != 0 (= batch): the columns' workgroups are shared out by length
};

typedef float f32x16 __attribute__((ext_vector_type(16)));

// New tokens of sequence b and the cache row of the first.
struct Tokens { int n, len; int64_t start; };
__device__ __forceinline__ Tokens tokens_of(const PromptParams& p, int b) {
    const int raw = p.seq_lens[b], n = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    return {n, min(max(raw, 0), min(p.cap_rows, p.max_len)), (int64_t)raw - n};
}
// What row `row` of (sequence b, KV head g) is: its token, head, position and range.
struct Query { int token, head, pos, lo, hi; };
__device__ __forceinline__ Query query_of(const PromptParams& p, const Tokens& t, int b, int g, int row) {
    Query x;
    x.token = (uint32_t)row / (uint32_t)p.G;
    x.head = g * p.G + row - x.token * p.G;
    const int64_t pos = t.start + x.token;
    x.pos = (int)pos;
    const int64_t at = (int64_t)b * p.n_new + x.token;
    x.lo = max(p.first != nullptr ? p.first[at] : 0, 0);
    x.hi = (int)min((int64_t)t.len, p.end != nullptr ? (int64_t)p.end[at] : pos + 1);
    return x;
}

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = min(v, __shfl_xor(v, o));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_max_i(int v) { return ~wave_min(~v); }

// Raw product x -> score = a * bend(x) + b, in units of ln 2 or 1 / `unit` of that.  Without a cap bend(x) = x; with one, cap tanh(y / cap) =
// 2 cap / (1 + e^(-2 y / cap)) - cap, right at both ends and off by 2^-22 of the cap between: one exponential and one reciprocal, and the
// product and sum around them become part of the multiply-add ahead of the weight's exponential.
struct ScoreForm { float a, b, inner; };
template <bool CAP>
__device__ __forceinline__ ScoreForm score_form(const PromptParams& p, float unit) {
    if constexpr (CAP) return {2.f * p.cap * unit, -p.cap * unit, p.scale / p.cap * (-2.f * kLog2e)};
    return {p.scale * unit, 0.f, 0.f};
}
template <bool CAP>
__device__ __forceinline__ float bend(float x, const ScoreForm& f) {
    if constexpr (CAP) return __builtin_amdgcn_rcpf(fast_exp2(x * f.inner) + 1.f);
    return x;
}

// Infinities and NaN of V in a tile of which a row sees a part.  A weight of 0 times one of them would be NaN in rows that do not see it, so such
// tiles are multiplied with zeros in their place, and the rows that see one get it added afterwards, read from memory once more.
__device__ __forceinline__ bool has_non_finite(u32x4 v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad = bad || (v[i] & 0x7f80u) == 0x7f80u || (v[i] & 0x7f800000u) == 0x7f800000u;
    return bad;
}
__device__ __forceinline__ void drop_non_finite(u32x4& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
    }
}
__device__ __forceinline__ float only_non_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? v : 0.f; }

// ---- 128 rows to a workgroup ----
constexpr int kPromptRows = 128, kPromptTile = 64;
constexpr int kMaxSplits = 256;

// SLOPE: scores are worked out one by one, not in the weights' exponents.
template <bool CAP, bool SLOPE>
__global__ __launch_bounds__(256, 2)
void prompt_tile_kernel(const PromptParams p) {
    // Consecutive workgroups go round the 8 dies, and the (sequence, KV head) pairs run fastest: a die sees few pairs (one, where there are 8; the same
    // head of every sequence), whose rows its L2 keeps, and of each sequence as many row tiles as any other die.  The last tokens', which see most, come first.
    const int pairs = p.Hkv * p.batch, bg = (int)(blockIdx.x % (uint32_t)pairs), rest = (int)(blockIdx.x / (uint32_t)pairs);
    const int tile = p.row_tiles - 1 - rest / p.splits, split = rest % p.splits;
    const int b = bg / p.Hkv, g = bg - b * p.Hkv;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const Tokens tok = tokens_of(p, b);
    const int n_rows = tok.n * p.G;
    if (tile * kPromptRows >= n_rows) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int row = tile * kPromptRows + w * 32 + n;
    const bool real = row < n_rows;
    const Query me = query_of(p, tok, b, g, min(row, n_rows - 1));

    // two tiles of K and V: one is worked on while the next is written
    constexpr int kHalf = kPromptTile * kD * 2;
    __shared__ __attribute__((aligned(16))) unsigned char sK[2 * kHalf], sV[2 * kHalf];
    __shared__ int sLo[4], sHi[4], sInLo[4], sInHi[4], sBad[2];

    // ranges: of the wavefront's rows together, and what all of them see
    const bool some = real && me.lo < me.hi;
    const int w_lo = wave_min(some ? me.lo : INT32_MAX), w_hi = wave_max_i(some ? me.hi : INT32_MIN);
    const int in_lo = wave_max_i(real ? me.lo : INT32_MIN), in_hi = wave_min(real ? me.hi : INT32_MAX);
    if (lane == 0) { sLo[w] = w_lo; sHi[w] = w_hi; sInLo[w] = in_lo; sInHi[w] = in_hi; }
    if (tid == 0) sBad[0] = sBad[1] = -1;

    bf16x8 q[8];
    const uint16_t* qr = p.q + (int64_t)b * p.q_b + (int64_t)me.token * p.q_t + (int64_t)me.head * kD;
#pragma unroll
    for (int s = 0; s < 8; ++s) q[s] = *reinterpret_cast<const bf16x8*>(qr + 16 * s + 8 * h);
    ScoreForm form = score_form<CAP>(p, kLog2e);
    if (!SLOPE && form.a < 0.f) {             // raw products are compared below: their order has to be the scores'
        form.a = -form.a;
#pragma unroll
        for (int s = 0; s < 8; ++s) q[s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[s]) ^ 0x80008000u);
    }
    const float slope2 = SLOPE && p.slopes != nullptr ? p.slopes[me.head] * kLog2e : 0.f;
    __syncthreads();
    const int lo = __builtin_amdgcn_readfirstlane(min(min(sLo[0], sLo[1]), min(sLo[2], sLo[3])));
    const int hi = __builtin_amdgcn_readfirstlane(max(max(sHi[0], sHi[1]), max(sHi[2], sHi[3])));
    const int all_lo = max(max(sInLo[0], sInLo[1]), max(sInLo[2], sInLo[3])), all_hi = min(min(sInHi[0], sInHi[1]), min(sInHi[2], sInHi[3]));
    const int tiles = hi > lo ? (int)(((int64_t)hi - lo + kPromptTile - 1) / kPromptTile) : 0;
    const int parts = max(1, min(p.splits, (int)((uint32_t)(tiles + p.split_tiles - 1) / (uint32_t)p.split_tiles)));
    if (split >= parts) return;
    if (split == 0 && tid == 0 && p.splits > 1) p.parts[bg * p.row_tiles + tile] = parts;
    // (scalars, and known as such: the buffers of the tiles hang on them)
    const int t0 = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * split / parts));
    const int t1 = __builtin_amdgcn_readfirstlane((int)((int64_t)tiles * (split + 1) / parts));

    float m = -INFINITY, l = 0.f;
    f32x16 o[4];
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;

    // staging: thread -> chunk of 16 bytes c of rows r16 + 16 i.  K: chunk c of row r lies at c ^ (r & 15); V: at c ^ 2 (r & 7), so that the
    // transposing reads of four rows of 16 dims fall on different banks.
    const int c = tid & 15, r16 = tid >> 4;
    const uint16_t* k_rows = p.k + (int64_t)b * p.s_b + (int64_t)g * p.s_h;
    const uint16_t* v_rows = p.v + (int64_t)b * p.s_b + (int64_t)g * p.s_h;
    u32x4 kr[4], vr[4];
    // (a tile is a buffer of its own: rows past `hi` read as zeros, which no row sees)
    auto request = [&](int t) {
        const int at = lo + t * kPromptTile, bytes = min(hi - at, kPromptTile) * (kD * 2);
        const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(k_rows) + (int64_t)at * kD, 0, bytes, 0x00020000);
        const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(v_rows) + (int64_t)at * kD, 0, bytes, 0x00020000);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kr[i] = __builtin_amdgcn_raw_buffer_load_b128(rk, tid * 16, i * 4096, 0);
            vr[i] = __builtin_amdgcn_raw_buffer_load_b128(rv, tid * 16, i * 4096, 0);
        }
    };
    const int k_to = r16 * 256 + ((c ^ r16) << 4), v_to = r16 * 256 + ((c ^ (2 * (r16 & 7))) << 4);
    const int k_from = n * 256 + ((h ^ (n & 15)) << 4);              // ^ 32 s for operand s; + 8192 for the second block of 32 rows
    const int i16 = lane & 15, q4 = (lane >> 4) & 1;
    const int v_from = (4 * h + (i16 >> 2)) * 256 + (((2 * q4 + ((i16 & 3) >> 1)) ^ (2 * (4 * h + (i16 >> 2)))) << 4) + (i16 & 1) * 8;

    auto write = [&](int t) {                 // the requested tile, number t, to its half of the LDS
        const int j0 = lo + t * kPromptTile, half = (t & 1) * kHalf;
        if (j0 < all_lo || j0 + kPromptTile > all_hi) {
            if (has_non_finite(vr[0]) || has_non_finite(vr[1]) || has_non_finite(vr[2]) || has_non_finite(vr[3])) {
                sBad[t & 1] = t;
#pragma unroll
                for (int i = 0; i < 4; ++i) drop_non_finite(vr[i]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            *reinterpret_cast<u32x4*>(sK + half + k_to + i * 4096) = kr[i];
            *reinterpret_cast<u32x4*>(sV + half + v_to + i * 4096) = vr[i];
        }
    };
    auto work = [&](int t) {
        const int j0 = lo + t * kPromptTile, half = (t & 1) * kHalf;
        if (j0 >= w_hi || j0 + kPromptTile <= w_lo) return;
        const bool masked = j0 < in_lo || j0 + kPromptTile > in_hi;
        // ---- S^T: rows j0 + 32 x + 8 (r / 4) + 4 h + r % 4 of column n ----
        f32x16 s[2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[x][r] = 0.f;
        // (kAhead operands are read, and waited for, ahead of an unbroken run of products)
        auto key = [&](int i) { return *reinterpret_cast<const bf16x8*>(sK + half + (k_from ^ (i >> 1 << 5)) + (i & 1) * 8192); };
        constexpr int kAhead = 6;
        bf16x8 a[16];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) a[i] = key(i);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[i], q[i >> 1], s[i & 1], 0, 0, 0);
            if (i + kAhead < 16) a[i + kAhead] = key(i + kAhead);
        }
#pragma unroll
        for (int i = 0; i < 16 - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
        __builtin_amdgcn_sched_barrier(0);
        auto row_of = [&](int x, int r) { return j0 + 32 * x + 8 * (r >> 2) + 4 * h + (r & 3); };
        if constexpr (CAP || SLOPE) {
            const float far0 = (float)(me.pos - j0 - 4 * h);       // (distances beyond 2^24 to 2^-24 of themselves)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[x][r] = bend<CAP>(s[x][r], form);
                    if constexpr (SLOPE) s[x][r] = fmaf(-slope2, fabsf(far0 - (float)(32 * x + 8 * (r >> 2) + (r & 3))), fmaf(s[x][r], form.a, form.b));
                }
        }
        if (masked) {
            asm volatile("" ::: "memory");    // (a branch: most tiles have nothing to mask)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int r = 0; r < 16; ++r) { const int j = row_of(x, r); s[x][r] = j >= me.lo && j < me.hi ? s[x][r] : -INFINITY; }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int r = 0; r < 16; r += 2) mx = fmaxf(fmaxf(s[x][r], s[x][r + 1]), mx);
        if constexpr (!SLOPE) mx = fmaf(mx, form.a, form.b);
        mx = max_xor32(mx);
        // The maximum that weights are taken against follows the true one only when that has grown by more than 8: weights stay below 2^8, and the output
        // is rescaled a few times in all.
        if (__any(mx > m + 8.f)) {
            const float to = fmaxf(m, mx), a = to == -INFINITY ? 1.f : fast_exp2(m - to);
            m = to;
            l *= a;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= a;
        }
        __builtin_amdgcn_s_setprio(1);        // (two wavefronts to a SIMD: the one here goes first, the other's products fill in; 558 -> 542 us)
        const float ref = m == -INFINITY ? 0.f : m, from = form.b - ref;
        // ---- weights, and O^T += V^T P^T, 16 rows at a time: slot e of half h is row 8 (e / 4) + 4 h + e % 4 of them ----
        auto value = [&](int y, int d) {
            const unsigned char* at = sV + half + (v_from ^ (d << 6)) + y * 4096;
            const v4s v0 = lds_read_tr16(reinterpret_cast<const uint16_t*>(at)), v1 = lds_read_tr16(reinterpret_cast<const uint16_t*>(at + 2048));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        };
        float part[4];
        auto weights = [&](int y) {
            u32x4 u;
            part[y] = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float s0 = s[y >> 1][8 * (y & 1) + 2 * e], s1 = s[y >> 1][8 * (y & 1) + 2 * e + 1];
                const float a = fast_exp2(SLOPE ? s0 - ref : fmaf(s0, form.a, from)), bb = fast_exp2(SLOPE ? s1 - ref : fmaf(s1, form.a, from));
                part[y] += a + bb;
                u[e] = pack_bf16(a, bb);              // (8 bits a weight: its rounding is as large as the output's own and not common to the rows)
            }
            return __builtin_bit_cast(bf16x8, u);
        };
        bf16x8 v[2][4], pw[2];
#pragma unroll
        for (int d = 0; d < 4; ++d) v[0][d] = value(0, d);
        pw[0] = weights(0);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            __builtin_amdgcn_sched_barrier(0);
            if (y < 3) {
#pragma unroll
                for (int d = 0; d < 4; ++d) v[(y + 1) & 1][d] = value(y + 1, d);
                pw[(y + 1) & 1] = weights(y + 1);
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[y & 1][d], pw[y & 1], o[d], 0, 0, 0);
            if (y < 3) {                      // a matrix instruction, then what fits beside it: transposing reads and the next 16 rows' weights
                __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x402, 9, 0);
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        l += (part[0] + part[1]) + (part[2] + part[3]);
        if (sBad[t & 1] == t) {
            const uint16_t* from = p.v + (int64_t)b * p.s_b + (int64_t)g * p.s_h + 4 * h;
            for (int j = max(j0, me.lo); j < j0 + kPromptTile && j < me.hi; ++j) {
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const uint2 x = *reinterpret_cast<const uint2*>(from + (int64_t)j * kD + 32 * d + 8 * r);
                        o[d][4 * r] += only_non_finite(bf16_lo(x.x)); o[d][4 * r + 1] += only_non_finite(bf16_hi(x.x));
                        o[d][4 * r + 2] += only_non_finite(bf16_lo(x.y)); o[d][4 * r + 3] += only_non_finite(bf16_hi(x.y));
                    }
            }
        }
    };
    // (the queries are here before the loop begins: see queries_here)
#pragma unroll
    for (int s = 0; s < 8; ++s) {
        u32x4 x = __builtin_bit_cast(u32x4, q[s]);
        asm volatile("" : "+v"(x));
        q[s] = __builtin_bit_cast(bf16x8, x);
    }
    if (t0 < t1) {
        request(t0);
        write(t0);
        if (t0 + 1 < t1) request(t0 + 1);
        __syncthreads();
    }
    for (int t = t0; t < t1; ++t) {
        work(t);
        if (t + 1 < t1) write(t + 1);
        if (t + 2 < t1) request(t + 2);
        lds_barrier();
    }
    // ---- lane (n, h) has dims 32 d + 8 (r / 4) + 4 h + r % 4 of row n ----
    l = sum_xor32(l);
    if (!real) return;
    if (parts > 1) {
        const int64_t at = ((int64_t)bg * p.n_new * p.G + row) * p.splits + split;
        if (h == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(m, l);
        float* to = p.part_o + at * kD + 4 * h;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<float4*>(to + 32 * d + 8 * r) = make_float4(o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]);
        return;
    }
    const int64_t at = ((int64_t)b * p.n_new + me.token) * p.Hq + me.head;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (h == 0 && p.lse != nullptr) p.lse[at] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (1.f / kLog2e);
    uint16_t* to = p.out + at * kD + 4 * h;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r)
            *reinterpret_cast<uint2*>(to + 32 * d + 8 * r) =
                make_uint2(pack_bf16(o[d][4 * r] * inv, o[d][4 * r + 1] * inv), pack_bf16(o[d][4 * r + 2] * inv, o[d][4 * r + 3] * inv));
}

// ---- up to 16 rows in all ----
template <bool CAP, bool SLOPE>
__global__ __launch_bounds__(kColWaves * 64, 2)
void prompt_cols_kernel(const PromptParams p) {
    const int g = blockIdx.y, slot = (int)(blockIdx.z * gridDim.x + blockIdx.x);
    int b = blockIdx.z, split = blockIdx.x, parts = p.splits;
    if (p.ragged != 0) {                      // (sequences by their lengths: what the ranges leave of them is not known here)
        AttnParams a;
        a.ragged_batch = p.ragged; a.nch = p.splits; a.share_cap = kMaxSplits; a.cap2 = p.cap_rows; a.max_rows2 = p.max_len;
        const RaggedSlot r = ragged_slot<false>(a, p.seq_lens, slot);
        if (r.b < 0) return;
        b = r.b; split = r.c; parts = r.nchunks;
    }
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const Tokens tok = tokens_of(p, b);
    const int n_rows = tok.n * p.G;
    if (n_rows == 0) return;
    const int64_t bg = (int64_t)b * p.Hkv + g;
    if (p.splits > 1 && split == 0 && threadIdx.x == 0) { p.parts[2 * bg] = slot; p.parts[2 * bg + 1] = parts; }
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, gr = lane >> 4;
    const bool real = col < n_rows;
    const Query me = query_of(p, tok, b, g, min(col, n_rows - 1));
    const bool some = real && me.lo < me.hi;
    const int lo = wave_min(some ? me.lo : INT32_MAX), hi = wave_max_i(some ? me.hi : INT32_MIN);
    const int in_lo = wave_max_i(real ? me.lo : INT32_MIN), in_hi = wave_min(real ? me.hi : INT32_MAX);
    const int tiles = hi > lo ? (int)(((int64_t)hi - lo + kTileRows - 1) / kTileRows) : 0;

    bf16x8 q[4];
    const uint16_t* qr = p.q + (int64_t)b * p.q_b + (int64_t)me.token * p.q_t + (int64_t)me.head * kD;
#pragma unroll
    for (int s = 0; s < 4; ++s) q[s] = *reinterpret_cast<const bf16x8*>(qr + operand_dim<false>(s, gr));
    __builtin_amdgcn_sched_barrier(0);
    const ScoreForm form = score_form<CAP>(p, 1.f);       // (natural units, as the columns' running state has them)
    const float slope = SLOPE && p.slopes != nullptr ? p.slopes[me.head] : 0.f;
    const uint16_t* k = p.k + (int64_t)b * p.s_b + (int64_t)g * p.s_h;
    const uint16_t* v = p.v + (int64_t)b * p.s_b + (int64_t)g * p.s_h;

    ColState st;
    st.clear();
    TileRows<kBf16> rows;
    const int step = parts * kColWaves;
    int t = split * kColWaves + w;
    auto first_of = [&](int x) { return lo + x * kTileRows; };        // (past the rows there are by a round at most: see check_kv)
    if (t < tiles) {
        request_keys<kBf16, false>(rows, k, first_of(t), hi - first_of(t));
        request_values<kBf16>(rows, v, first_of(t), hi - first_of(t));
    }
    queries_here(q);
    for (; t < tiles; t += step) {
        const int j0 = first_of(t);
        float s[2][4];
        tile_scores<kBf16>(rows, q, s);
        request_keys<kBf16, false>(rows, k, first_of(t + step), hi - first_of(t + step));       // (past the last tile: nothing)
        const bool masked = j0 < in_lo || (int64_t)j0 + kTileRows > in_hi;
        auto sees = [&](int j) { return j >= me.lo && j < me.hi; };
        const float far0 = (float)(me.pos - j0 - 4 * gr);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = fmaf(bend<CAP>(s[x][i], form), form.a, form.b);
                if constexpr (SLOPE) s[x][i] = fmaf(-slope, fabsf(far0 - (float)(16 * x + i)), s[x][i]);
            }
        if (masked) {
            asm volatile("" ::: "memory");    // (a branch: most tiles have nothing to mask)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = sees(j0 + 16 * x + 4 * gr + i) ? s[x][i] : -INFINITY;
        }
        tile_softmax(st, s);
        bf16x8 ph, pl;
        weight_operands(s, ph, pl);
        // (one token: all columns have one range, and rows outside it were never read)
        bool bad = false;
        if (masked && tok.n > 1) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bad = bad || has_non_finite(rows.v[e]);
            if (bad) {
#pragma unroll
                for (int e = 0; e < 8; ++e) drop_non_finite(rows.v[e]);
            }
        }
        tile_output<kBf16>(rows, st, ph, pl);
        if (__any(bad)) {
            for (int j = max(j0, me.lo); j < j0 + kTileRows && j < me.hi; ++j) {
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const u32x4 x = *reinterpret_cast<const u32x4*>(v + (int64_t)j * kD + 8 * (4 * gr + r));
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        st.o[2 * i][r] += only_non_finite(bf16_lo(x[i]));
                        st.o[2 * i + 1][r] += only_non_finite(bf16_hi(x[i]));
                    }
                }
            }
        }
        request_values<kBf16>(rows, v, first_of(t + step), hi - first_of(t + step));
    }

    __shared__ __attribute__((aligned(16))) ColMergeLds lds;
    __shared__ float sInv[16];
    if (p.splits > 1) {
        const int64_t at = ((int64_t)g * p.splits * p.batch + slot) * p.n_new * p.G;
        merge_columns(lds, st, n_rows,
                      [&](int x, int d, float o0, float o1) {
                          *reinterpret_cast<float2*>(p.part_o + (at + x) * kD + d) = make_float2(o0, o1);
                      },
                      [&](int x, float m, float l) {
                          *reinterpret_cast<float2*>(p.part_ml + (at + x) * 2) = make_float2(m * kLog2e, l);
                      });
        return;
    }
    // (the statistics of a column come with its first pair of dims: they are worked out once more for the others)
    auto out_row = [&](int x) { const int i = x / p.G; return ((int64_t)b * p.n_new + i) * p.Hq + g * p.G + (x - i * p.G); };
    float* o = &lds.o[0][0][0];
    merge_columns(lds, st, n_rows,
                  [&](int x, int d, float o0, float o1) { o[x * kD + d] = o0; o[x * kD + d + 1] = o1; },
                  [&](int x, float m, float l) {
                      sInv[x] = l == 0.f ? 0.f : 1.f / l;
                      if (p.lse != nullptr) p.lse[out_row(x)] = l == 0.f ? -INFINITY : m + __builtin_amdgcn_logf(l) * (1.f / kLog2e);
                  });
    __syncthreads();
    for (int x = threadIdx.x; x < n_rows * (kD / 2); x += kColWaves * 64) {
        const int r = x / (kD / 2), d = 2 * (x % (kD / 2));
        *reinterpret_cast<uint32_t*>(p.out + out_row(r) * kD + d) = pack_bf16(o[r * kD + d] * sInv[r], o[r * kD + d + 1] * sInv[r]);
    }
}

// Joins the parts of a row: a wavefront each.
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

// Which kernel, and over how many workgroups at most the cache rows of one row tile are split: so that the launch has up to kPromptTarget workgroups (two to
// a compute unit).  Columns: none with fewer than a round of 128 rows.  Row tiles: a part no shorter than split_tiles tiles of 64 rows, which
// the kernel sees to, as only it knows the ranges: 32, or 16 where there are few row tiles.  us, 32 heads over 8 (parts: most to a row tile):
//   128 tokens behind 32640: 1 part 740, 2: 378, 4: 197, 8: 108, 16: 84, 32: 101;  300 behind 7892: 1: 190, 2: 107, 4: 69, 6: 77;
//   512 behind 32256: 1: 742, 4: 285;  8 behind 32760, parts of 32 tiles: 47, 16: 32, 8: 33, 4: 43;  whole prompts of 600: 1: 20.0, 2: 26.4,
//   of 2048: 1: 59, 2: 77 (there the partial results cost more than the even spread gains).
constexpr int kPromptTarget = 2 * kComputeUnits;
struct PromptPlan { bool cols; int row_tiles, splits, split_tiles; };
static PromptPlan prompt_plan(const rk_geom* g, int64_t n_new, int64_t max_len) {
    const int64_t pairs = (int64_t)g->batch * g->n_kv_heads, rows = n_new * (g->n_q_heads / g->n_kv_heads);
    PromptPlan f{rows <= 16, 1, 1, 1};
    int64_t most = (max_len + kMinChunk - 1) / kMinChunk;
    if (!f.cols) {
        f.row_tiles = (int)((rows + kPromptRows - 1) / kPromptRows);
        f.split_tiles = pairs * f.row_tiles < 64 ? 16 : 32;
        most = (max_len + f.split_tiles * kPromptTile - 1) / (f.split_tiles * kPromptTile);
    }
    int64_t s = kPromptTarget / (pairs * f.row_tiles);
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    f.splits = (int)(s < 1 ? 1 : s);
    return f;
}
// Rows of partial results that any call of up to n_new tokens and max_len rows can need: a launch that splits has at most
// kPromptTarget workgroups of at most kPromptRows rows each.
static int64_t prompt_partials(const rk_geom* g, int64_t n_new, int64_t max_len) {
    const int64_t pairs = (int64_t)g->batch * g->n_kv_heads, rows = n_new * (g->n_q_heads / g->n_kv_heads);
    const int64_t most = (int64_t)kPromptTarget * kPromptRows, all = pairs * rows * ((max_len + kMinChunk - 1) / kMinChunk);
    return pairs > kPromptTarget / 2 ? 0 : all < most ? all : most;
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
    if ((int64_t)n_new * G > INT32_MAX - kPromptRows) return RK_ERR_UNSUPPORTED;
    const PromptPlan plan = prompt_plan(geom, n_new, max_len);
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
    // (a scale of 0 goes with the slopes: masked products would be 0 times infinity in a weight's exponent)
    const bool cap = p.cap > 0.f, slope = p.slopes != nullptr || (p.scale == 0.f && !cap);
    hipStream_t st = (hipStream_t)stream;
    if (plan.cols) {
        auto kernel = cap ? (slope ? prompt_cols_kernel<true, true> : prompt_cols_kernel<true, false>)
                          : (slope ? prompt_cols_kernel<false, true> : prompt_cols_kernel<false, false>);
        hipLaunchKernelGGL(kernel, dim3(plan.splits, geom->n_kv_heads, geom->batch), dim3(kColWaves * 64), 0, st, p);
    } else {
        auto kernel = cap ? (slope ? prompt_tile_kernel<true, true> : prompt_tile_kernel<true, false>)
                          : (slope ? prompt_tile_kernel<false, true> : prompt_tile_kernel<false, false>);
        const int64_t total = pairs * plan.row_tiles * plan.splits;
        hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(256), 0, st, p);
    }
    if ((rc = launch_status()) != RK_OK || plan.splits == 1) return rc;
    hipLaunchKernelGGL(prompt_merge_kernel, dim3((unsigned)((n_new * G + 3) / 4), geom->n_kv_heads, geom->batch), dim3(256), 0, st, p);
    return launch_status();
}
