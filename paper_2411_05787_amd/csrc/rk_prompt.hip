// rk_prompt_attn: attention of the new tokens of each sequence over the bf16 cache that holds them.
//
// The query heads of a group and the new tokens are one axis, row = token * G + head, so a tile of rows shares every K and V row that it
// reads among the group's heads too.  Two kernels:
//   prompt_tile_kernel  128 or 256 rows to a workgroup, the cache rows through LDS, everything on the matrix cores: bound by those, by the
//                       softmax between the two products and, in long calls, by the power that both draw;
//   prompt_cols_kernel  up to 16 rows in all (a decode step's token, a few drafted ones): the cache streams past once, bound by memory
//                       (rk_cols.h).
// A row r sees cache rows lo <= j < hi.  Tiles that no row of a workgroup sees are never read; only those that a bound runs through are masked.
// Where there are few rows the cache rows are split over workgroups, and prompt_merge_kernel joins their (maximum, sum, output).
#include "rk_cols.h"

#include <cfloat>
#include <type_traits>

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
    int32_t first_round;                      // workgroups of a (sequence, KV head) in the launch's order, of which the others' order is turned around
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
    x.pos = (int)max(pos, (int64_t)INT32_MIN);
    const int64_t at = (int64_t)b * p.n_new + x.token;
    x.lo = max(p.first != nullptr ? p.first[at] : 0, 0);
    // (a negative length less its tokens is below 32 bits: bounded before it is narrowed)
    x.hi = (int)max(min((int64_t)t.len, p.end != nullptr ? (int64_t)p.end[at] : pos + 1), (int64_t)0);
    return x;
}

__device__ __forceinline__ int wave_min(int v) {
    auto moved = [](int x, auto how) { return __float_as_int(dpp_move_f<decltype(how)::value>(__int_as_float(x))); };
    v = min(v, moved(v, std::integral_constant<int, kDppXor1>{}));
    v = min(v, moved(v, std::integral_constant<int, kDppXor2>{}));
    v = min(v, moved(v, std::integral_constant<int, kDppRor4>{}));
    v = min(v, moved(v, std::integral_constant<int, kDppRor8>{}));
    const LanePair a = rows_xor16(v);
    const LanePair b = halves_xor32(min(a.a, a.b));
    return __builtin_amdgcn_readfirstlane(min(b.a, b.b));
}
__device__ __forceinline__ int wave_max_i(int v) { return ~wave_min(~v); }

// Raw product x -> score = a * bend(x) + b, in units of ln 2 or 1 / `unit` of that.  CAP says how bend caps:
//   kNoCap    bend(x) = x.
//   kNearCap  y = scale * x, cap tanh(y / cap) = 2 cap / (1 + e^(-2 y / cap)) - cap: one exponential and one reciprocal, and the product and sum around
//             them become part of the multiply-add ahead of the weight's exponential.  A difference of numbers of the cap's size: right at both ends and
//             off by 2^-22 of the cap between, 2^-15 for the largest cap that takes it (kNearCapMost).
//   kFarCap   any cap, to 2^-19 of the score: y (1 - z^2 / 3 + 2 z^4 / 15 - 17 z^6 / 315 + 62 z^8 / 2835), z = y / cap, where |z| < 1/4 (what the series
//             leaves out is below 2^-26 there), and as above beyond, where tanh is no smaller than 0.24.  Three capped chunks 93.4 us, kNearCap 69.1.
constexpr int kNoCap = 0, kNearCap = 1, kFarCap = 2;
constexpr float kNearCapMost = 128.f;
struct ScoreForm { float a, b, inner, per, cap; };
template <int CAP>
__device__ __forceinline__ ScoreForm score_form(const PromptParams& p, float unit) {
    // (kept finite below caps of 1e-38 or so: a product of 0 stays 0)
    if constexpr (CAP == kNearCap) return {2.f * p.cap * unit, -p.cap * unit, fminf(fmaxf(p.scale / p.cap * (-2.f * kLog2e), -FLT_MAX), FLT_MAX), 0.f, 0.f};
    if constexpr (CAP == kFarCap) return {unit, 0.f, p.scale, 1.f / p.cap, p.cap};
    return {p.scale * unit, 0.f, 0.f, 0.f, 0.f};
}
template <int CAP>
__device__ __forceinline__ float bend(float x, const ScoreForm& f) {
    if constexpr (CAP == kNearCap) return __builtin_amdgcn_rcpf(fast_exp2(x * f.inner) + 1.f);
    if constexpr (CAP == kFarCap) {
        const float y = x * f.inner, z = y * f.per, zz = z * z;
        const float near = y * fmaf(zz, fmaf(zz, fmaf(zz, fmaf(zz, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), 1.f);
        const float far = f.cap * fmaf(2.f, __builtin_amdgcn_rcpf(fast_exp2(z * (-2.f * kLog2e)) + 1.f), -1.f);
        return fabsf(z) < 0.25f ? near : far;
    }
    return x;
}

// Infinities and NaN of V in a tile of which a row sees a part.  A weight of 0 times one of them would be NaN in rows that do not see it, so such
// tiles are multiplied with zeros in their place, and the rows that see one get it added afterwards, read from memory once more.
__device__ __forceinline__ bool has_non_finite(u32x4 v) {
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad |= (uint32_t)((v[i] & 0x7f80u) == 0x7f80u) | (uint32_t)((v[i] & 0x7f800000u) == 0x7f800000u);
    return bad != 0;
}
__device__ __forceinline__ void drop_non_finite(u32x4& v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if ((v[i] & 0x7f80u) == 0x7f80u) v[i] &= 0xffff0000u;
        if ((v[i] & 0x7f800000u) == 0x7f800000u) v[i] &= 0xffffu;
    }
}
__device__ __forceinline__ float only_non_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) == 0x7f800000u ? v : 0.f; }

// ---- 128 or 256 rows to a workgroup ----
//   S^T = K Q^T   v_mfma_f32_32x32x16_bf16: lane (n, h) = (lane % 32, lane / 32) gets column (row of the tile) n, cache rows 8 (r / 4) + 4 h + r % 4 of a
//                 block of 32;
//   O^T += V^T P^T  the contraction slots are numbered as S^T left the rows in the lanes, so P goes from the softmax to the matrix cores without
//                 leaving its lane; V is turned around by the transposing reads of LDS.
// A wavefront takes 32 QB rows and works a block at a time, in stages of 16 QB slots: while the products of the block ahead (S^T) and of the one
// behind (O^T) are on the matrix cores, it makes weights of the scores between them, a matrix instruction and about five others to a slot.  K and V
// come through LDS, whose rows are padded so that no two lanes of a read's phase meet in a bank: rings of 4 QB blocks, a barrier to QB stages. 8192
// tokens, 32 heads over 8, QB = 2: 480-490 us, 1120-1145 TFLOP/s (a library matrix product of 8192^3 beside it 1390; with zeros for data, which
// draw less power, 1320 and 1800).  Three capped chunks, QB = 1: 69 us, 480 TFLOP/s.  8192 tokens with a
// bias or a cap of 50, QB = 1 too: 662 us, 507 plain beside them.  Without stages, two tiles of 64 rows in LDS and a barrier a
// tile: 554 and 76 us. Instructions count: one wavefront on a SIMD issues one every five cycles or so (QB = 2: 218 to a stage, 32 of them
// products).
constexpr int kPromptRows = 128, kPromptTile = 64, kMaxSplits = 256;      // (cache rows are split over workgroups in tiles of two blocks)
constexpr int kBlockRows = 32;
constexpr int kKRow = kD * 2 + 16, kVRow = kD * 2 + 64;     // bytes from row to row in LDS: the reads of a phase fall on different banks
constexpr int kKBlock = kBlockRows * kKRow, kVBlock = kBlockRows * kVRow;

template <int QB, int CAP, bool SLOPE>
__global__ __launch_bounds__(256, QB == 1 ? 2 : 1)
void prompt_tile_kernel(const PromptParams p) {
    constexpr int kRows = kPromptRows * QB, kSlots = 16 * QB, kRing = 4 * QB, kAheadK = 2 + QB, kAheadV = QB;
    // Consecutive workgroups go round the 8 dies, and the (sequence, KV head) pairs run fastest: a die sees few pairs (one, where there are 8; the
    // same head of every sequence), whose rows its L2 keeps, and of each sequence as many row tiles as any other die.  The last tokens', which see
    // most, come first.
    const int pairs = p.Hkv * p.batch, bg = (int)(blockIdx.x % (uint32_t)pairs);
    int rest = (int)(blockIdx.x / (uint32_t)pairs);
    if (rest >= p.first_round) rest = p.row_tiles * p.splits - 1 - (rest - p.first_round);
    const int tile = p.row_tiles - 1 - rest / p.splits, split = rest % p.splits;
    const int b = bg / p.Hkv, g = bg - b * p.Hkv;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    const Tokens tok = tokens_of(p, b);
    const int n_rows = tok.n * p.G;
    if (tile * kRows >= n_rows) return;
    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, h = lane >> 5;
    const int row0 = tile * kRows + w * 32 * QB + n;
    bool real[QB];
    Query me[QB];
#pragma unroll
    for (int x = 0; x < QB; ++x) { real[x] = row0 + 32 * x < n_rows; me[x] = query_of(p, tok, b, g, min(row0 + 32 * x, n_rows - 1)); }

    __shared__ __attribute__((aligned(16))) unsigned char sK[kRing * kKBlock], sV[kRing * kVBlock];
    __shared__ int sLo[4], sHi[4], sInLo[4], sInHi[4], sBad;

    int w_lo = INT32_MAX, w_hi = INT32_MIN, in_lo = INT32_MIN, in_hi = INT32_MAX;
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        if (!real[x]) continue;
        if (me[x].lo < me[x].hi) { w_lo = min(w_lo, me[x].lo); w_hi = max(w_hi, me[x].hi); }
        in_lo = max(in_lo, me[x].lo); in_hi = min(in_hi, me[x].hi);
    }
    w_lo = wave_min(w_lo); w_hi = wave_max_i(w_hi); in_lo = wave_max_i(in_lo); in_hi = wave_min(in_hi);
    if (lane == 0) { sLo[w] = w_lo; sHi[w] = w_hi; sInLo[w] = in_lo; sInHi[w] = in_hi; }
    if (tid == 0) sBad = 0;

    bf16x8 q[QB][8];
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        const uint16_t* qr = p.q + (int64_t)b * p.q_b + (int64_t)me[x].token * p.q_t + (int64_t)me[x].head * kD;
#pragma unroll
        for (int s = 0; s < 8; ++s) q[x][s] = *reinterpret_cast<const bf16x8*>(qr + 16 * s + 8 * h);
    }
    ScoreForm form = score_form<CAP>(p, kLog2e);
    if (!SLOPE && form.a < 0.f) {             // raw products are compared below: their order has to be the scores'
        form.a = -form.a;
#pragma unroll
        for (int x = 0; x < QB; ++x)
#pragma unroll
            for (int s = 0; s < 8; ++s) q[x][s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[x][s]) ^ 0x80008000u);
    }
    float slope2[QB];
    if constexpr (SLOPE) {
#pragma unroll
        for (int x = 0; x < QB; ++x) slope2[x] = p.slopes != nullptr ? p.slopes[me[x].head] * kLog2e : 0.f;
    }
    __syncthreads();
    const int lo = __builtin_amdgcn_readfirstlane(min(min(sLo[0], sLo[1]), min(sLo[2], sLo[3])));
    const int hi = __builtin_amdgcn_readfirstlane(max(max(sHi[0], sHi[1]), max(sHi[2], sHi[3])));
    const int all_lo = __builtin_amdgcn_readfirstlane(max(max(sInLo[0], sInLo[1]), max(sInLo[2], sInLo[3])));
    const int all_hi = __builtin_amdgcn_readfirstlane(min(min(sInHi[0], sInHi[1]), min(sInHi[2], sInHi[3])));
    const int tiles = hi > lo ? (int)(((int64_t)hi - lo + kPromptTile - 1) / kPromptTile) : 0;
    const int parts = max(1, min(p.splits, (int)((uint32_t)(tiles + p.split_tiles - 1) / (uint32_t)p.split_tiles)));
    if (split >= parts) return;
    if (split == 0 && tid == 0 && p.splits > 1) p.parts[bg * p.row_tiles + tile] = parts;
    // (scalars, and known as such: the buffers of the tiles hang on them)
    const int each = tiles / parts, rest_tiles = tiles - each * parts;
    const int t0 = __builtin_amdgcn_readfirstlane(each * split + rest_tiles * split / parts);
    const int t1 = __builtin_amdgcn_readfirstlane(each * (split + 1) + rest_tiles * (split + 1) / parts);
    const int b0 = 2 * t0, b1 = 2 * t1, end = min(hi, lo + b1 * kBlockRows);       // blocks
    // the blocks whose stage has nothing to mask and nothing to clean: safe .. safe + n_safe - 1
    const int safe = (int)(((int64_t)all_lo - lo + kBlockRows - 1) >> 5), n_safe = max((int)(((int64_t)all_hi - lo) >> 5) - kAheadV - safe, 0);
    float m[QB], l[QB], from[QB], limit[QB], alpha[QB];
    f32x16 o[QB][4];
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        m[x] = limit[x] = -INFINITY; l[x] = from[x] = 0.f; alpha[x] = 1.f;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[x][d][r] = 0.f;
    }

    // staging: thread -> chunk of 16 bytes tid % 16 of rows tid / 16 and tid / 16 + 16
    const uint16_t* k_rows = p.k + (int64_t)b * p.s_b + (int64_t)g * p.s_h;
    const uint16_t* v_rows = p.v + (int64_t)b * p.s_b + (int64_t)g * p.s_h;
    struct Staged { u32x4 r[2]; };
    // (a block is a buffer of its own: rows that no stage sees read as zeros, without traffic)
    auto bytes_of = [&](int i) {
        int have = min(end - (lo + i * kBlockRows), kBlockRows);
        asm("" : "+s"(have));
        return max(have, 0) * (kD * 2);
    };
    auto buffer = [&](const uint16_t* rows, int bytes) { return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(rows), 0, bytes, 0x00020000); };
    auto request = [&](const uint16_t* rows, int i) {
        const __amdgpu_buffer_rsrc_t rsrc = buffer(rows + (int64_t)(lo + i * kBlockRows) * kD, bytes_of(i));
        return Staged{__builtin_amdgcn_raw_buffer_load_b128(rsrc, tid * 16, 0, 0), __builtin_amdgcn_raw_buffer_load_b128(rsrc, tid * 16, 4096, 0)};
    };
    const int k_slot = (tid >> 4) * kKRow + (tid & 15) * 16, v_slot = (tid >> 4) * kVRow + (tid & 15) * 16;
    auto write_k = [&](const Staged& s, int at, int c) { *reinterpret_cast<u32x4*>(sK + at + k_slot + c * 16 * kKRow) = s.r[c]; };
    auto write_v = [&](const Staged& s, int at, int c) { *reinterpret_cast<u32x4*>(sV + at + v_slot + c * 16 * kVRow) = s.r[c]; };
    auto outside = [&](int i) { const int j0 = lo + i * kBlockRows; return j0 < all_lo || j0 + kBlockRows > all_hi; };
    auto clean = [&](Staged& v, int i) {      // V's block i, where a row sees a part of it only
        if (!outside(i)) return;
        if (has_non_finite(v.r[0]) || has_non_finite(v.r[1])) {
            sBad = 1;
            drop_non_finite(v.r[0]);
            drop_non_finite(v.r[1]);
        }
    };

    const int k_from = n * kKRow + h * 16;
    const int i16 = lane & 15, q4 = (lane >> 4) & 1;
    const int v_from = (4 * h + (i16 >> 2)) * kVRow + (2 * q4 + ((i16 & 3) >> 1)) * 16 + (i16 & 1) * 8;
    auto key = [&](int at, int s) { return *reinterpret_cast<const bf16x8*>(sK + at + k_from + s * 32); };
    auto value = [&](int at, int y, int d) {
        const unsigned char* from = sV + at + v_from + y * 16 * kVRow + d * 64;
        const v4s v0 = lds_read_tr16(reinterpret_cast<const uint16_t*>(from)), v1 = lds_read_tr16(reinterpret_cast<const uint16_t*>(from + 8 * kVRow));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
    };

    // What a stage hands on to the next one, that of block i: its raw products (with CAP or SLOPE what has been made of them), this lane's largest
    // of them, and the first operands of block i + 1's keys.
    struct Ahead { f32x16 s[QB]; float top[QB]; bf16x8 k[4]; };
    struct Weights { u32x4 p[QB][2]; };
    auto score = [&](Ahead& a, int x, int r, float far0) {
        if constexpr (CAP != kNoCap) a.s[x][r] = bend<CAP>(a.s[x][r], form);
        if constexpr (SLOPE) a.s[x][r] = fmaf(-slope2[x], fabsf(far0 - (float)(8 * (r >> 2) + (r & 3))), fmaf(a.s[x][r], form.a, form.b));
    };
    auto largest = [&](Ahead& a, int x, int r) {      // of elements up to r + 1, r from 0 in steps of 2
        a.top[x] = fmaxf(fmaxf(a.s[x][r], a.s[x][r + 1]), r == 0 ? -INFINITY : a.top[x]);
    };
    auto mask = [&](Ahead& a, int i) {
        const int j0 = lo + 32 * i;
        if (j0 >= in_lo && j0 + 32 <= in_hi) return;
#pragma unroll
        for (int x = 0; x < QB; ++x) {
#pragma unroll
            for (int r = 0; r < 16; ++r) { const int j = j0 + 8 * (r >> 2) + 4 * h + (r & 3); a.s[x][r] = j >= me[x].lo && j < me[x].hi ? a.s[x][r] : -INFINITY; }
#pragma unroll
            for (int r = 0; r < 16; r += 2) largest(a, x, r);
        }
    };
    // The maximum that weights are taken against follows the true one only when that has grown by more than 8: weights stay below 2^8, the output
    // is rescaled a few times in all (at the stage's end, when the weights made before have gone into it), and blocks that change nothing cost one
    // comparison.
    auto follow = [&](Ahead& a) {
        const bool grew = __any(a.top[0] > limit[0] || (QB > 1 && a.top[QB - 1] > limit[QB - 1]));
        if (grew) {
            asm volatile("" ::: "memory");
#pragma unroll
            for (int x = 0; x < QB; ++x) {
                const float mx = max_xor32(SLOPE ? a.top[x] : fmaf(a.top[x], form.a, form.b)), to = mx > m[x] + 8.f ? mx : m[x];
                alpha[x] = to == -INFINITY ? 1.f : fast_exp2(m[x] - to);
                m[x] = to;
                from[x] = (SLOPE ? 0.f : form.b) - (to == -INFINITY ? 0.f : to);
                limit[x] = SLOPE ? to + 8.f : (to + 8.f - form.b) / form.a;
                l[x] *= alpha[x];
            }
        }
        return grew;
    };
    auto prime = [&](Ahead& a, int i, int k_at, int k_next) {
#pragma unroll
        for (int x = 0; x < QB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) a.s[x][r] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bf16x8 k = key(k_at, e);
#pragma unroll
            for (int x = 0; x < QB; ++x) a.s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[x][e], a.s[x], 0, 0, 0);
        }
#pragma unroll
        for (int x = 0; x < QB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) { score(a, x, r, (float)(me[x].pos - (lo + 32 * i) - 4 * h)); if (r & 1) largest(a, x, r - 1); }
#pragma unroll
        for (int e = 0; e < 4; ++e) a.k[e] = key(k_next, e);
    };
    auto drain = [&](const Weights& pw, int v_at) {
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const bf16x8 v = value(v_at, y, d);
#pragma unroll
                for (int x = 0; x < QB; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, __builtin_bit_cast(bf16x8, pw.p[x][y]), o[x][d], 0, 0, 0);
            }
    };
    // Block i's stage, in slots of one matrix instruction and what fits beside it: products of block i + 1 (keys at k_at) in the first half, those
    // of block i - 1's weights (values at v_at) in the other, block i's weights all along or, where scores take work of their own, in the first
    // half, and that and the next maximum in the second.  Keys of block i + 2 are at k_next.  Beside it keys of block i + kAheadK are written to
    // k_to and values of block i + kAheadV to v_to, those of the blocks behind them requested.
    Staged kr, vr;
    const uint16_t *k_next_rows = k_rows, *v_next_rows = v_rows;      // of the blocks that are requested next
    auto wait_lds = [](auto n) { __builtin_amdgcn_s_waitcnt(0xc07f | decltype(n)::value << 8); };
    auto stage = [&](Ahead& now, Ahead& ahead, const Weights& behind, Weights& made, int i, int& v_bytes, int k_at, int k_next, int k_to, int v_at, int v_to, bool fenced, bool fence) {
        constexpr int kPer = CAP != kNoCap || SLOPE ? 2 : 1, kHalf = kSlots / 2, kTail = kHalf + 2;
        if ((uint32_t)(i - safe) >= (uint32_t)n_safe) {
            asm volatile("" ::: "memory");    // (a branch: most blocks have nothing of it)
            mask(now, i);
            clean(vr, i + kAheadV);
        }
        const bool grew = follow(now);
        const int k_bytes = bytes_of(i + kAheadK + 1);
        const __amdgpu_buffer_rsrc_t k_in = buffer(k_next_rows, k_bytes), v_in = buffer(v_next_rows, v_bytes);
        v_bytes = k_bytes;                    // (of V that block is requested two stages later)
        k_next_rows += kBlockRows * kD; v_next_rows += kBlockRows * kD;
        bf16x8 kk[8], vv[8];
        float part[QB], wt[16 * QB], far0[QB];
        if constexpr (SLOPE) {
#pragma unroll
            for (int x = 0; x < QB; ++x) far0[x] = (float)(me[x].pos - (lo + 32 * i + 32) - 4 * h);      // (distances beyond 2^24 to 2^-24 of themselves)
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) kk[e] = now.k[e];
#pragma unroll
        for (int x = 0; x < QB; ++x)
#pragma unroll
            for (int r = 0; r < 16; ++r) ahead.s[x][r] = 0.f;
        auto exponent = [&](int e) { const float v = now.s[e >> 4][e & 15]; wt[e] = SLOPE ? v + from[e >> 4] : fmaf(v, form.a, from[e >> 4]); };
        auto add = [&](int e) { const float t = wt[e] + wt[e + 1]; part[e >> 4] = e % 16 == 0 ? t : part[e >> 4] + t; };
        auto pack = [&](int e) {              // (8 bits a weight: its rounding is as large as the output's own and not common to the rows)
            made.p[e >> 4][(e & 15) >> 3][(e & 7) >> 1] = pack_bf16(wt[e], wt[e + 1]);
        };
#pragma unroll
        for (int e = 0; e < kPer; ++e) exponent(e);
#pragma unroll
        for (int k = 0; k < kSlots; ++k) {
            __builtin_amdgcn_sched_barrier(0);
            const int x = k % QB;
            if constexpr (QB > 1) {           // (one wavefront to a SIMD: one wait for several operands)
                if (k == 0 && !fenced) wait_lds(std::integral_constant<int, 0>{});
                if (k == 4 * QB) wait_lds(std::integral_constant<int, 4>{});
                if (k == kHalf) wait_lds(std::integral_constant<int, 4>{});
                if (k == kHalf + 4 * QB) wait_lds(std::integral_constant<int, 0>{});
                if (k == kHalf) __builtin_amdgcn_s_waitcnt(0xf70);      // (vmcnt 0: all that the last stage requested, before the first of it is written)
            }
            if (k < kHalf) {
                ahead.s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk[k / QB], q[x][k / QB], ahead.s[x], 0, 0, 0);
            } else {
                const int j = (k - kHalf) / QB;       // (16 rows, then the other 16)
                o[x][j & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vv[j], __builtin_bit_cast(bf16x8, behind.p[x][j >> 2]), o[x][j & 3], 0, 0, 0);
            }
            if (k < 4) kk[4 + k] = key(k_at, 4 + k);
            constexpr int kFirstV = QB == 1 ? 3 : 5;
            if (k >= kFirstV && k < kFirstV + 8 * QB && (k - kFirstV) % QB == 0) { const int j = (k - kFirstV) / QB; vv[j] = value(v_at, j >> 2, j & 3); }
            if (k >= kSlots - 4 * QB && (k % QB) == 0) { const int j = (k - (kSlots - 4 * QB)) / QB; ahead.k[j] = key(k_next, j); }
            if (k >= kHalf && k < kHalf + 4) { if (k - kHalf < 2) write_k(kr, k_to, k - kHalf); else write_v(vr, v_to, k - kHalf - 2); }
            if (k >= kHalf + 4 && k < kHalf + 6) kr.r[k - kHalf - 4] = __builtin_amdgcn_raw_buffer_load_b128(k_in, tid * 16, (k - kHalf - 4) * 4096, 0);
            if (k >= kHalf + 6 && k < kHalf + 8) vr.r[k - kHalf - 6] = __builtin_amdgcn_raw_buffer_load_b128(v_in, tid * 16, (k - kHalf - 6) * 4096, 0);
#pragma unroll
            for (int e = kPer * k; e < kPer * (k + 1) && e < 16 * QB; ++e) {
                wt[e] = fast_exp2(wt[e]);
                if (e + kPer < 16 * QB) exponent(e + kPer);
                if (e >= 2 && e % 2 == 0 && kPer == 1) add(e - 2);
                if (e >= 3 && e % 2 == 1) { if (kPer == 2) add(e - 3); pack(e - 3); }
            }
            if (k >= kTail) {
                if constexpr (CAP != kNoCap || SLOPE) {
#pragma unroll
                    for (int e = (k - kTail) * 16 * QB / (kSlots - kTail); e < (k - kTail + 1) * 16 * QB / (kSlots - kTail); ++e) {
                        score(ahead, e >> 4, e & 15, far0[e >> 4]);
                        if (e & 1) largest(ahead, e >> 4, (e & 15) - 1);
                    }
                } else {
#pragma unroll
                    for (int e = (k - kTail) * 8 * QB / (kSlots - kTail); e < (k - kTail + 1) * 8 * QB / (kSlots - kTail); ++e) largest(ahead, e % QB, 2 * (e / QB));
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        add(16 * QB - 2); pack(16 * QB - 2);
#pragma unroll
        for (int x = 0; x < QB; ++x) {
            l[x] += part[x];
            asm volatile("" : "+v"(made.p[x][0]), "+v"(made.p[x][1]), "+v"(l[x]), "+v"(ahead.top[x]));      // (made here, and not where they are needed)
        }
        if (grew) {
#pragma unroll
            for (int x = 0; x < QB; ++x)
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[x][d][r] *= alpha[x];
        }
        if (fence) lds_barrier();
    };

    // (the queries are here before the loop begins: see queries_here)
#pragma unroll
    for (int x = 0; x < QB; ++x)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            u32x4 u = __builtin_bit_cast(u32x4, q[x][e]);
            if constexpr (QB == 1) asm volatile("" : "+v"(u));
            else asm volatile("" : "+a"(u));
            q[x][e] = __builtin_bit_cast(bf16x8, u);
        }
    if (b0 < b1) {
        // tiles of two blocks in LDS
        constexpr int kKTile = 2 * kKBlock, kVTile = 2 * kVBlock, kTiles = kRing / 2;
        int kt[kTiles], vt[kTiles];           // of the block's own tile, the next one, ..
#pragma unroll
        for (int c = 0; c < kTiles; ++c) { kt[c] = c * kKTile; vt[c] = c * kVTile; }
        Staged ks[kAheadK], vs[kAheadV];
#pragma unroll
        for (int c = 0; c < kAheadK; ++c) ks[c] = request(k_rows, b0 + c);
#pragma unroll
        for (int c = 0; c < kAheadV; ++c) vs[c] = request(v_rows, b0 + c);
        for (int x = tid; x < kVBlock / 16; x += 256) *reinterpret_cast<u32x4*>(sV + (kRing - 1) * kVBlock + 16 * x) = u32x4{0u, 0u, 0u, 0u};      // (nothing lies behind the first block)
#pragma unroll
        for (int c = 0; c < kAheadK; ++c) { write_k(ks[c], c * kKBlock, 0); write_k(ks[c], c * kKBlock, 1); }
#pragma unroll
        for (int c = 0; c < kAheadV; ++c) { clean(vs[c], b0 + c); write_v(vs[c], c * kVBlock, 0); write_v(vs[c], c * kVBlock, 1); }
        kr = request(k_rows, b0 + kAheadK);
        vr = request(v_rows, b0 + kAheadV);
        int v_even = bytes_of(b0 + kAheadV + 1), v_odd = bytes_of(b0 + kAheadV + 2);
        k_next_rows += (int64_t)(lo + (b0 + kAheadK + 1) * kBlockRows) * kD; v_next_rows += (int64_t)(lo + (b0 + kAheadV + 1) * kBlockRows) * kD;
        __syncthreads();
        Ahead even, odd;
        Weights pe, po{};
        prime(even, b0, 0, kKBlock);
        for (int i = b0; i < b1; i += 2) {
            constexpr int last = kTiles - 1;
            if constexpr (QB == 1) {
                stage(even, odd, po, pe, i, v_even, kt[0] + kKBlock, kt[1], kt[1] + kKBlock, vt[last] + kVBlock, vt[0] + kVBlock, true, true);
                stage(odd, even, pe, po, i + 1, v_odd, kt[1], kt[1] + kKBlock, kt[0], vt[0], vt[1], true, true);
            } else {
                stage(even, odd, po, pe, i, v_even, kt[0] + kKBlock, kt[1], kt[2 % kTiles], vt[last] + kVBlock, vt[1], true, false);
                stage(odd, even, pe, po, i + 1, v_odd, kt[1], kt[1] + kKBlock, kt[2 % kTiles] + kKBlock, vt[0], vt[1] + kVBlock, false, true);
            }
            const int k0 = kt[0], v0 = vt[0];
#pragma unroll
            for (int c = 0; c < last; ++c) { kt[c] = kt[c + 1]; vt[c] = vt[c + 1]; }
            kt[last] = k0; vt[last] = v0;
        }
        drain(po, vt[kTiles - 1] + kVBlock);
        if (sBad != 0) {
#pragma unroll 1
            for (int i = b0; i < b1; ++i) {
                if (!outside(i)) continue;
                const int j0 = lo + i * kBlockRows;
#pragma unroll
                for (int x = 0; x < QB; ++x)
                    for (int j = max(j0, me[x].lo); j < j0 + kBlockRows && j < me[x].hi; ++j) {
#pragma unroll
                        for (int d = 0; d < 4; ++d)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint2 u = *reinterpret_cast<const uint2*>(v_rows + 4 * h + (int64_t)j * kD + 32 * d + 8 * e);
                                o[x][d][4 * e] += only_non_finite(bf16_lo(u.x)); o[x][d][4 * e + 1] += only_non_finite(bf16_hi(u.x));
                                o[x][d][4 * e + 2] += only_non_finite(bf16_lo(u.y)); o[x][d][4 * e + 3] += only_non_finite(bf16_hi(u.y));
                            }
                    }
            }
        }
    }
    // ---- lane (n, h) has dims 32 d + 8 (r / 4) + 4 h + r % 4 of rows n + 32 x ----
#pragma unroll
    for (int x = 0; x < QB; ++x) {
        const float sum = sum_xor32(l[x]);
        if (!real[x]) continue;
        if (parts > 1) {
            const int64_t at = ((int64_t)bg * p.n_new * p.G + row0 + 32 * x) * p.splits + split;
            if (h == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = make_float2(m[x], sum);
            float* to = p.part_o + at * kD + 4 * h;
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    *reinterpret_cast<float4*>(to + 32 * d + 8 * r) = make_float4(o[x][d][4 * r], o[x][d][4 * r + 1], o[x][d][4 * r + 2], o[x][d][4 * r + 3]);
            continue;
        }
        const int token = (uint32_t)(row0 + 32 * x) / (uint32_t)p.G;
        const int64_t at = ((int64_t)b * p.n_new + token) * p.Hq + g * p.G + (row0 + 32 * x - token * p.G);
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        if (h == 0 && p.lse != nullptr) p.lse[at] = sum == 0.f ? -INFINITY : (m[x] + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
        uint16_t* to = p.out + at * kD + 4 * h;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                *reinterpret_cast<uint2*>(to + 32 * d + 8 * r) =
                    make_uint2(pack_bf16(o[x][d][4 * r] * inv, o[x][d][4 * r + 1] * inv), pack_bf16(o[x][d][4 * r + 2] * inv, o[x][d][4 * r + 3] * inv));
    }
}

// ---- up to 16 rows in all ----
// The tile of rk_cols.h; bound by memory: 8 sequences of up to 16384 rows, 356 MB, 63.6 us with the launch that joins the parts (5.6 TB/s), 32 of
// 4000 rows alone 77 (6.8 TB/s). (W = kColAlone wavefronts where a workgroup has all rows of a (sequence, KV head))
constexpr int kColAlone = 8;
template <int W, int CAP, bool SLOPE>
__global__ __launch_bounds__(W * 64, W == kColWaves ? 2 : 1)
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
    const int step = parts * W;
    int t = split * W + w;
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

    __shared__ __attribute__((aligned(16))) ColMergeLds<W, 16> lds;
    __shared__ float sInv[16];
    if (p.splits > 1) {
        const int64_t at = ((int64_t)g * p.splits * p.batch + slot) * p.n_new * p.G;
        merge_columns(lds, st, n_rows,
                      [&](int x, int d, float o0, float o1, float) {
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

// Which kernel, and over how many workgroups at most the cache rows of one row tile are split. 64 rows to a wavefront where two rounds of such
// workgroups or more come together, nothing capped and no bias: those are long enough for the card to lower its clock with the power it draws, and
// half the reads from LDS then count for more than a second wavefront on the SIMD (us, 64 rows / 32: 8192 tokens of 32 heads over 8 480 / 514, and
// 416 / 387 with zeros for data, where the clock stays; 4096 tokens 133 / 147, 3000 84.4 / 83.5, 2048 59.0 / 46.9; 4 prompts of 1024 52.3 / 51.9;
// three capped chunks 132 / 70). Columns: no part with fewer than a round of 128 rows, two workgroups to a compute unit; or a larger workgroup
// alone with all rows and no second launch, where the pairs nearly fill the chip or the sequences are short (us, one token, split / alone: 16
// sequences of 500 rows 13.5 / 11.4, of 1000 19.1 / 18.8, of up to 1000 15.9 / 17.5, 32 of 500 19.0 / 13.2, of 1000 27.6 / 23.0, 64 of 1000, 28 heads over 4, 29.7 / 23.1, 4
// of 1000 9.9 / 13.8; 64 of 2000, 32 heads over 8, which four wavefronts take alone: 76.3 / 79.3).  Row tiles: one workgroup to a compute unit, two
// where that leaves parts of more than 32 tiles of cache rows; no part shorter than split_tiles tiles, which the kernel sees to, as only it knows
// the ranges.  us, 32 heads over 8, by workgroups in all (256 / 512): 8 tokens behind 32752 33.7 / 35.0, 64 behind 16320 34.8 / 38.3, 128 behind
// 8064 34.4 / 37.4, 128 behind 32640 99 / 91, 300 behind 7892 64 / 61, 512 behind 32256 348 / 287; by the shortest part (4 / 8 / 16 tiles): 8
// tokens behind 992 12.9 / 17.0 / 22.0, 8 behind 4088 14.8 / 18.2 / 26.4, whole prompts of 400 19.1 / 13.9 / 14.0.
constexpr int kPromptTarget = 2 * kComputeUnits;
struct PromptPlan { bool cols, wide, alone; int row_tiles, splits, split_tiles; };
static PromptPlan prompt_plan(const rk_geom* g, int64_t n_new, int64_t max_len, bool plain) {
    const int64_t pairs = (int64_t)g->batch * g->n_kv_heads, rows = n_new * (g->n_q_heads / g->n_kv_heads);
    PromptPlan f{rows <= 16, plain && pairs * ((rows + 2 * kPromptRows - 1) / (2 * kPromptRows)) >= 2 * kComputeUnits, false, 1, 1, 1};
    int64_t s = kPromptTarget / pairs, most = (max_len + kMinChunk - 1) / kMinChunk;
    if (!f.cols) {
        const int tile = f.wide ? 2 * kPromptRows : kPromptRows;
        f.row_tiles = (int)((rows + tile - 1) / tile);
        const int64_t wgs = pairs * f.row_tiles, tiles = (max_len + kPromptTile - 1) / kPromptTile;
        s = kComputeUnits / wgs;
        f.split_tiles = wgs <= 32 ? 4 : 8;
        if (tiles > 32 * (s < 1 ? 1 : s)) { s = f.wide ? 1 : kPromptTarget / wgs; f.split_tiles = 16; }
        most = (tiles + f.split_tiles - 1) / f.split_tiles;
    }
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    f.splits = (int)(s < 1 ? 1 : s);
    f.alone = f.cols && pairs >= 64 && pairs < kPromptTarget && (max_len <= (pairs >= kComputeUnits ? 8 * pairs : 512) || (pairs >= kComputeUnits && ragged_batch_of(g) == 0));
    if (f.alone) f.splits = 1;
    return f;
}
// Rows of partial results that any call of up to n_new tokens and max_len rows can need: a launch that splits has at most
// kPromptTarget workgroups of at most kPromptRows rows each.
static int64_t prompt_partials(const rk_geom* g, int64_t n_new, int64_t max_len) {
    const int64_t pairs = (int64_t)g->batch * g->n_kv_heads, rows = n_new * (g->n_q_heads / g->n_kv_heads);
    const int64_t most = (int64_t)kPromptTarget * kPromptRows, all = pairs * rows * ((max_len + kMinChunk - 1) / kMinChunk);
    return pairs > kPromptTarget / 2 ? 0 : all < most ? all : most;
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
