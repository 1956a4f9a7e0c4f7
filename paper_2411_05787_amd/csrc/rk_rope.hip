// Rotary positions of new tokens, and their rows into the full cache: rk_rope_table, rk_rope_append, rk_rope_append_q8,
// rk_rope_append_paged.
//
// A pass reads every new row once and writes it once; there is nothing to reuse but a token's cosines and sines, which all of its
// heads share.  Eight lanes take a row of 256 bytes, two chunks of eight dims each: in the half layout the two halves of eight pairs, in the
// interleaved one any.  So a pair never leaves its lane, a turn needs no exchange, and q_out may be q.
#include "rk_q8.h"
#include "rk_pages.h"

namespace rk {

struct RopeParams {
    const uint16_t *q, *k, *v;
    int64_t q_b, q_t, k_b, k_t, v_b, v_t;
    const float* rope;                        // the table of cosines and sines; NULL: nothing is turned
    int32_t max_pos, rot, interleaved;
    const int32_t* positions; const int32_t* seq_lens; const int32_t* new_lens;
    int32_t n_new, Hq, Hkv;
    uint16_t* q_out;
    uint16_t *ck, *cv; int64_t c_b, c_h; int32_t capacity;       // the bf16 cache
    rk_kv8 c8;                                                   // the one of 8 bits
    const int32_t* pred; int32_t pred_val;
    int32_t rows_per_token;                   // that token_row takes
    int32_t block_wgs;                        // 8 bits and pages with bounds: workgroups ahead of those that take rows
    rk_pages pages;                           // the one in pages
    const int32_t* table; int32_t width, shift;
};
enum CacheOf { kInRows, kIn8Bits, kInPages, kInBoundedPages };      // where the new rows go; the last: keys by append_page

// Products and sums are rounded one by one: what is quantised later must not depend on which of them a compiler fuses.
__device__ __forceinline__ void turn_pair(float& a, float& b, float c, float s) {
#pragma clang fp contract(off)
    const float x = a * c, y = b * s, z = b * c, w = a * s;
    a = x - y;
    b = z + w;
}

// What lane c of the eight has of a row: the dims where its two chunks start, 64 or rot / 2 apart, so that the eight lanes' chunks lie side by
// side.  Half layout: lo and hi are the halves of eight pairs, or both are not turned.  Interleaved: each is four pairs, or is not turned.
struct LaneDims { int lo, hi; bool turn_lo, turn_hi; };
__device__ __forceinline__ LaneDims lane_dims(int c, const RopeParams& p) {
    const int pairs = p.rot >> 4;             // lanes whose chunks are turned in the half layout
    if (p.interleaved) return {c * 8, 64 + c * 8, c * 8 < p.rot, 64 + c * 8 < p.rot};
    if (c < pairs) return {c * 8, (p.rot >> 1) + c * 8, true, true};
    return {(c + pairs) * 8, 64 + c * 8, false, false};
}
// Cosines and sines of a lane's eight pairs: pairs lo .. lo + 7 of the half layout, lo / 2 .. + 3 and hi / 2 .. + 3 of the interleaved one.
struct Turn { float c[8], s[8]; };
__device__ __forceinline__ void load_turn(Turn& t, const RopeParams& p, int pos, const LaneDims& d) {
    const bool known = (uint32_t)pos < (uint32_t)p.max_pos;
    const float* row = p.rope + (int64_t)(known ? pos : 0) * p.rot;
    const int a = p.interleaved ? d.lo >> 1 : d.lo, b = p.interleaved ? d.hi >> 1 : d.lo + 4;
    float4 x[4] = {};
    if (d.turn_lo) { x[0] = *reinterpret_cast<const float4*>(row + a); x[2] = *reinterpret_cast<const float4*>(row + (p.rot >> 1) + a); }
    if (d.turn_hi) { x[1] = *reinterpret_cast<const float4*>(row + b); x[3] = *reinterpret_cast<const float4*>(row + (p.rot >> 1) + b); }
    const float nan = __uint_as_float(0x7fc00000u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        t.c[4 * i] = x[i].x; t.c[4 * i + 1] = x[i].y; t.c[4 * i + 2] = x[i].z; t.c[4 * i + 3] = x[i].w;
        t.s[4 * i] = x[2 + i].x; t.s[4 * i + 1] = x[2 + i].y; t.s[4 * i + 2] = x[2 + i].z; t.s[4 * i + 3] = x[2 + i].w;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) { t.c[i] = known ? t.c[i] : nan; t.s[i] = known ? t.s[i] : nan; }
}
__device__ __forceinline__ void turn_chunks(u32x4& lo, u32x4& hi, const Turn& t, const LaneDims& d, bool interleaved) {
    float a[8], b[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[2 * i] = bf16_lo(lo[i]); a[2 * i + 1] = bf16_hi(lo[i]);
        b[2 * i] = bf16_lo(hi[i]); b[2 * i + 1] = bf16_hi(hi[i]);
    }
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            turn_pair(a[2 * i], a[2 * i + 1], t.c[i], t.s[i]);
            turn_pair(b[2 * i], b[2 * i + 1], t.c[4 + i], t.s[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) turn_pair(a[i], b[i], t.c[i], t.s[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (d.turn_lo) lo[i] = pack_bf16(a[2 * i], a[2 * i + 1]);
        if (d.turn_hi) hi[i] = pack_bf16(b[2 * i], b[2 * i + 1]);
    }
}

// New tokens of a sequence, and the cache row of the first of them (it may lie outside the cache).
struct NewTokens { int n; int64_t start; };
__device__ __forceinline__ NewTokens new_tokens(const RopeParams& p, int b) {
    const int n = p.new_lens != nullptr ? min(max(p.new_lens[b], 0), p.n_new) : p.n_new;
    return {n, (int64_t)p.seq_lens[b] - n};
}
__device__ __forceinline__ int position_of(const RopeParams& p, int b, int i, int64_t start) {
    return p.positions != nullptr ? p.positions[(int64_t)b * p.n_new + i] : (int)min(max(start + i, (int64_t)-1), (int64_t)INT32_MAX);
}

// Eight lanes, one row of a token: q heads (turned, to q_out), then with the bf16 cache k heads (turned) and v heads (copied).  Sharing a
// token's cosines and sines among several rows of a lane saves reads that hit in L2 and costs registers and coalescing: 8192 tokens of 48
// heads take 39.1 us with one row to eight lanes (204 MB, 5.2 TB/s, the rate of a plain copy), 44.9 with two or four, 47.4 with eight; one
// token 2.8, 3.4 and (four) 4.2.
template <CacheOf C>
__device__ __forceinline__ void token_row(const RopeParams& p, int b, uint32_t team) {
    const int i = (int)(team / (uint32_t)p.rows_per_token), r = (int)(team - (uint32_t)i * (uint32_t)p.rows_per_token);
    const NewTokens nt = new_tokens(p, b);
    if (i >= nt.n) return;
    const int n_q = p.q != nullptr ? p.Hq : 0;
    const int64_t at = nt.start + i;
    const LaneDims d = lane_dims(threadIdx.x & 7, p);
    const uint16_t* from;
    uint16_t* to;
    if (r < n_q) {
        from = p.q + (int64_t)b * p.q_b + (int64_t)i * p.q_t + (int64_t)r * kD;
        to = p.q_out + (((int64_t)b * p.n_new + i) * p.Hq + r) * kD;
    } else {
        if (C == kIn8Bits || at < 0 || at >= p.capacity) return;
        const bool key = C != kInBoundedPages && r < n_q + p.Hkv;
        const int g = r - n_q - (key || C == kInBoundedPages ? 0 : p.Hkv);
        from = (key ? p.k + (int64_t)b * p.k_b + (int64_t)i * p.k_t : p.v + (int64_t)b * p.v_b + (int64_t)i * p.v_t) + (int64_t)g * kD;
        if constexpr (C == kInPages || C == kInBoundedPages) {
            const int page = p.table[(int64_t)b * p.width + (at >> p.shift)];
            if ((uint32_t)page >= (uint32_t)p.pages.n_pages) return;
            to = (uint16_t*)(key ? p.pages.k : p.pages.v) + (int64_t)page * p.pages.stride_p + (int64_t)g * p.pages.stride_h + (at & ((1 << p.shift) - 1)) * kD;
        } else {
            to = (key ? p.ck : p.cv) + (int64_t)b * p.c_b + (int64_t)g * p.c_h + at * kD;
        }
    }
    u32x4 lo = *reinterpret_cast<const u32x4*>(from + d.lo), hi = *reinterpret_cast<const u32x4*>(from + d.hi);
    if (p.rope != nullptr && r < n_q + (C == kInBoundedPages ? 0 : p.Hkv)) {
        Turn t;
        load_turn(t, p, position_of(p, b, i, nt.start), d);
        turn_chunks(lo, hi, t, d, p.interleaved != 0);
    }
    *reinterpret_cast<u32x4*>(to + d.lo) = lo;
    *reinterpret_cast<u32x4*>(to + d.hi) = hi;
}

// ---- blocks of the cache of 8 bits ----
// Largest magnitude of the bf16 in a dword, as bits (an infinity or a NaN: 0x7f80 or more).
__device__ __forceinline__ uint32_t top_bits(uint32_t x) { return max(x & 0x7fffu, (x >> 16) & 0x7fffu); }

// The smallest power of two, at least 2^-126, with a <= M * scale, a > 0 given by its bf16 bits: M = 1.75 * 2^8 (e4m3) or
// 1.984375 * 2^6 (int8), so the exponent of a less that of M, and one more where a's mantissa is the larger one.
__device__ __forceinline__ int scale_exponent(uint32_t a, int format) {
    const int e = (int)(a >> 7) - 127;               // (subnormal: -126 is the answer in any case)
    const uint32_t m = a & 0x7fu;
    const int over = format == RK_Q8_E4M3 ? (m > 0x60u) : (m > 0x7eu);
    return max(e - (format == RK_Q8_E4M3 ? 8 : 6) + over, -126);
}

// Eight bf16 -> eight values of the format.  x * inv is exact, or beside a largest value near the end of the range below 2^-126, and rounds to 0 either way.
template <int FORMAT>
__device__ __forceinline__ uint2 quantise8(const u32x4 x, float inv) {
    uint32_t o[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float f0 = bf16_lo(x[2 * h]) * inv, f1 = bf16_hi(x[2 * h]) * inv, f2 = bf16_lo(x[2 * h + 1]) * inv, f3 = bf16_hi(x[2 * h + 1]) * inv;
        if (FORMAT == RK_Q8_E4M3) {
            int u = __builtin_amdgcn_cvt_pk_fp8_f32(f0, f1, 0, false);
            o[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f2, f3, u, true);
        } else {
            const int i0 = (int)rintf(f0), i1 = (int)rintf(f1), i2 = (int)rintf(f2), i3 = (int)rintf(f3);
            o[h] = (uint32_t)(i0 & 0xff) | (uint32_t)(i1 & 0xff) << 8 | (uint32_t)(i2 & 0xff) << 16 | (uint32_t)(i3 & 0xff) << 24;
        }
    }
    return make_uint2(o[0], o[1]);
}

// Ragged prompts of up to 2048 tokens, 186 MB, 42.5 us (4.4 TB/s); one token of each of 64 sequences 3.7 us.
// One workgroup: block number start / block + x of one (sequence, KV head), keys or values.  PASSES times 32 rows by eight lanes each, all
// rows held in registers until their largest magnitude is known.  The first block's workgroup also has the rows that stay in the
// tail when they belong to a later block: it has read the tail's old rows by then.
template <int FORMAT, int PASSES>
__device__ __forceinline__ void append_block(const RopeParams& p, int b, int x, int g, bool values) {
    const NewTokens nt = new_tokens(p, b);
    if (nt.n == 0) return;
    const int blk = p.c8.block;
    const int64_t start = max(nt.start, (int64_t)0), end = min((int64_t)p.seq_lens[b], p.c8.capacity);
    if (end <= start) return;
    const int64_t first = start / blk, last = (end - 1) / blk, number = first + x;
    const bool partial = end % blk != 0;      // (the capacity is whole blocks: the last block is full otherwise)
    if (number > last || (number == last && partial && x != 0)) return;
    const int c = threadIdx.x & 7, slot0 = threadIdx.x >> 3;
    const LaneDims d = lane_dims(c, p);
    uint16_t* tail = (uint16_t*)(values ? p.c8.v_tail : p.c8.k_tail) + ((int64_t)b * p.Hkv + g) * blk * kD;
    auto new_row = [&](int64_t r, u32x4& lo, u32x4& hi) {
        const int i = (int)(r - nt.start);
        const uint16_t* from = values ? p.v + (int64_t)b * p.v_b + (int64_t)i * p.v_t : p.k + (int64_t)b * p.k_b + (int64_t)i * p.k_t;
        from += (int64_t)g * kD;
        lo = *reinterpret_cast<const u32x4*>(from + d.lo);
        hi = *reinterpret_cast<const u32x4*>(from + d.hi);
        if (!values && p.rope != nullptr) {
            Turn t;
            load_turn(t, p, position_of(p, b, i, nt.start), d);
            turn_chunks(lo, hi, t, d, p.interleaved != 0);
        }
    };
    auto rows_to_tail = [&](int64_t block_first) {       // the new rows of the last block
        for (int s = slot0; s < blk; s += 32) {
            const int64_t r = block_first + s;
            if (r < start || r >= end) continue;
            u32x4 lo, hi;
            new_row(r, lo, hi);
            *reinterpret_cast<u32x4*>(tail + (int64_t)s * kD + d.lo) = lo;
            *reinterpret_cast<u32x4*>(tail + (int64_t)s * kD + d.hi) = hi;
        }
    };
    if (number == last && partial) { rows_to_tail(number * blk); return; }
    u32x4 lo[PASSES], hi[PASSES];
    uint32_t top = 0;
#pragma unroll
    for (int y = 0; y < PASSES; ++y) {
        const int s = slot0 + 32 * y;
        lo[y] = hi[y] = u32x4{0u, 0u, 0u, 0u};
        if (s >= blk) continue;
        const int64_t r = number * blk + s;
        if (r < start) {
            lo[y] = *reinterpret_cast<const u32x4*>(tail + (int64_t)s * kD + d.lo);
            hi[y] = *reinterpret_cast<const u32x4*>(tail + (int64_t)s * kD + d.hi);
        } else {
            new_row(r, lo[y], hi[y]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) top = max(top, max(top_bits(lo[y][e]), top_bits(hi[y][e])));
    }
    __shared__ uint32_t sTop[4];
    top = (uint32_t)wave_max((float)top);
    if ((threadIdx.x & 63) == 0) sTop[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(sTop[0], sTop[1]), max(sTop[2], sTop[3]));
    const bool finite = top < 0x7f80u;
    const int e = top != 0 && finite ? scale_exponent(top, FORMAT) : 0;
    const float inv = finite ? __uint_as_float((uint32_t)(127 - e) << 23) : 0.f;      // 2^-e: e is -126 .. 122
    if (threadIdx.x == 0) {
        float* scales = (values ? p.c8.v_scale : p.c8.k_scale) + ((int64_t)b * p.Hkv + g) * (p.c8.capacity / blk);
        scales[number] = finite ? __uint_as_float((uint32_t)(127 + e) << 23) : __uint_as_float(0x7fc00000u);
    }
    uint8_t* to = (uint8_t*)(values ? p.c8.v : p.c8.k) + (int64_t)b * p.c8.stride_b + (int64_t)g * p.c8.stride_h;
#pragma unroll
    for (int y = 0; y < PASSES; ++y) {
        const int s = slot0 + 32 * y;
        if (s >= blk) continue;
        uint8_t* row = to + (number * blk + s) * kD;
        *reinterpret_cast<uint2*>(row + d.lo) = finite ? quantise8<FORMAT>(lo[y], inv) : make_uint2(0u, 0u);
        *reinterpret_cast<uint2*>(row + d.hi) = finite ? quantise8<FORMAT>(hi[y], inv) : make_uint2(0u, 0u);
    }
    if (x == 0 && partial && last != number) rows_to_tail(last * blk);       // (behind the barrier: the old rows have been read)
}

__global__ __launch_bounds__(256) void rope_append_kernel(const RopeParams p) {
    const int b = blockIdx.y;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    token_row<kInRows>(p, b, blockIdx.x * 32 + (threadIdx.x >> 3));
}

template <int FORMAT, int PASSES>
__global__ __launch_bounds__(256) void rope_append_q8_kernel(const RopeParams p) {
    const int b = blockIdx.y;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    if ((int)blockIdx.x < p.block_wgs) {
        const int kv = blockIdx.x % (2 * p.Hkv);
        append_block<FORMAT, PASSES>(p, b, blockIdx.x / (2 * p.Hkv), kv >> 1, (kv & 1) != 0);
        return;
    }
    token_row<kIn8Bits>(p, b, (blockIdx.x - (uint32_t)p.block_wgs) * 32 + (threadIdx.x >> 3));
}

// ---- pages with bounds of their keys ----
// Two bf16 as signed 16-bit numbers in their order, -NaN < -infinity .. -0 < +0 .. +infinity < NaN, and back.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ s16x2 in_order(uint32_t x) { return __builtin_bit_cast(s16x2, x ^ ((x & 0x80008000u) >> 15) * 0x7fffu); }
__device__ __forceinline__ uint32_t out_of_order(s16x2 v) { const uint32_t x = __builtin_bit_cast(uint32_t, v); return x ^ ((x & 0x80008000u) >> 15) * 0x7fffu; }

// One workgroup: page number start / page + x of one (sequence, KV head).  Its new keys are turned and written, and the bounds are taken of all rows
// that the page holds then: so they depend on the rows alone, also where a sequence has been shortened and continued.  (The rows that were there are
// read for it: half a page on average.)
__device__ __forceinline__ void append_page(const RopeParams& p, int b, int x, int g) {
    const NewTokens nt = new_tokens(p, b);
    if (nt.n == 0) return;
    const int64_t start = max(nt.start, (int64_t)0), end = min((int64_t)p.seq_lens[b], (int64_t)p.capacity);
    const int64_t number = (start >> p.shift) + x;
    if (end <= start || number > (end - 1) >> p.shift) return;
    const int page = p.table[(int64_t)b * p.width + number];
    if ((uint32_t)page >= (uint32_t)p.pages.n_pages) return;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const LaneDims d = lane_dims(tid & 7, p);
    uint16_t* keys = (uint16_t*)p.pages.k + (int64_t)page * p.pages.stride_p + (int64_t)g * p.pages.stride_h;
    const int rows = (int)min(end - (number << p.shift), (int64_t)1 << p.shift);
    s16x2 least[8], most[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { least[e] = s16x2{32767, 32767}; most[e] = s16x2{-32768, -32768}; }
    for (int s = tid >> 3; s < rows; s += 32) {
        const int64_t r = (number << p.shift) + s;
        uint16_t* at = keys + (int64_t)s * kD;
        u32x4 lo, hi;
        if (r < start) {
            lo = *reinterpret_cast<const u32x4*>(at + d.lo);
            hi = *reinterpret_cast<const u32x4*>(at + d.hi);
        } else {
            const int i = (int)(r - nt.start);
            const uint16_t* from = p.k + (int64_t)b * p.k_b + (int64_t)i * p.k_t + (int64_t)g * kD;
            lo = *reinterpret_cast<const u32x4*>(from + d.lo);
            hi = *reinterpret_cast<const u32x4*>(from + d.hi);
            if (p.rope != nullptr) {
                Turn t;
                load_turn(t, p, position_of(p, b, i, nt.start), d);
                turn_chunks(lo, hi, t, d, p.interleaved != 0);
            }
            *reinterpret_cast<u32x4*>(at + d.lo) = lo;
            *reinterpret_cast<u32x4*>(at + d.hi) = hi;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const s16x2 v = in_order(e < 4 ? lo[e] : hi[e - 4]);
            least[e] = __builtin_elementwise_min(least[e], v);
            most[e] = __builtin_elementwise_max(most[e], v);
        }
    }
    // over the rows of the wavefront (lanes 8 apart), then over the wavefronts
    __shared__ uint32_t sLeast[4][8][8], sMost[4][8][8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        auto both = [&](auto&& pick, s16x2 v) {
            const uint32_t x = __builtin_bit_cast(uint32_t, v);
            v = pick(v, __builtin_bit_cast(s16x2, (uint32_t)dpp_move<kDppRor8>((int)x)));
            LanePair r = rows_xor16(__builtin_bit_cast(int, v));
            v = pick(__builtin_bit_cast(s16x2, r.a), __builtin_bit_cast(s16x2, r.b));
            r = halves_xor32(__builtin_bit_cast(int, v));
            return pick(__builtin_bit_cast(s16x2, r.a), __builtin_bit_cast(s16x2, r.b));
        };
        least[e] = both([](s16x2 a, s16x2 c) { return __builtin_elementwise_min(a, c); }, least[e]);
        most[e] = both([](s16x2 a, s16x2 c) { return __builtin_elementwise_max(a, c); }, most[e]);
        if (lane < 8) { sLeast[w][lane][e] = __builtin_bit_cast(uint32_t, least[e]); sMost[w][lane][e] = __builtin_bit_cast(uint32_t, most[e]); }
    }
    __syncthreads();
    if (tid < 64) {                           // lane 8 c + e: dword e of lane c's dims
        const int c = tid >> 3, e = tid & 7;
        const LaneDims dc = lane_dims(c, p);
        s16x2 lo = __builtin_bit_cast(s16x2, sLeast[0][c][e]), hi = __builtin_bit_cast(s16x2, sMost[0][c][e]);
#pragma unroll
        for (int y = 1; y < 4; ++y) {
            lo = __builtin_elementwise_min(lo, __builtin_bit_cast(s16x2, sLeast[y][c][e]));
            hi = __builtin_elementwise_max(hi, __builtin_bit_cast(s16x2, sMost[y][c][e]));
        }
        const int64_t to = ((int64_t)page * p.Hkv + g) * kD + (e < 4 ? dc.lo + 2 * e : dc.hi + 2 * (e - 4));
        *reinterpret_cast<uint32_t*>((uint16_t*)p.pages.k_min + to) = out_of_order(lo);
        *reinterpret_cast<uint32_t*>((uint16_t*)p.pages.k_max + to) = out_of_order(hi);
    }
}

template <bool BOUNDS>
__global__ __launch_bounds__(256) void rope_append_paged_kernel(const RopeParams p) {
    const int b = blockIdx.y;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    if (BOUNDS && (int)blockIdx.x < p.block_wgs) {
        append_page(p, b, blockIdx.x / p.Hkv, blockIdx.x % p.Hkv);
        return;
    }
    token_row<BOUNDS ? kInBoundedPages : kInPages>(p, b, (blockIdx.x - (uint32_t)p.block_wgs) * 32 + (threadIdx.x >> 3));
}

// One workgroup per position.
__global__ __launch_bounds__(64) void rope_table_kernel(float* table, int32_t rot, rk_rope_scaling s) {
    const int i = threadIdx.x, half = rot >> 1;
    if (i >= half) return;
    double f = pow(s.base, -2.0 * i / rot);
    if (s.original_len > 0.0) {
        const double turns = s.original_len * f / 6.283185307179586476925286766559;
        double keep = (turns - s.low_turns) / (s.high_turns - s.low_turns);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        f = keep * f + (1.0 - keep) * (f / s.factor);
    } else {
        f /= s.factor;
    }
    const double a = (double)blockIdx.x * f;
    float* row = table + (int64_t)blockIdx.x * rot;
    row[i] = (float)(s.amplitude * cos(a));
    row[half + i] = (float)(s.amplitude * sin(a));
}

static int check_rope(const rk_geom* geom, const rk_new_rows* rows, const rk_rope* rope, const int32_t* seq_lens, void* q_out) {
    const int rc = check_geom(geom);
    if (rc != RK_OK) return rc;
    if (!rows || !rows->k || !rows->v || !seq_lens || rows->n_new <= 0) return RK_ERR_INVALID_ARG;
    if ((rows->q != nullptr) != (q_out != nullptr) || (rows->q && !rope)) return RK_ERR_INVALID_ARG;
    if (!aligned16(rows->q) || !aligned16(rows->k) || !aligned16(rows->v) || !aligned16(q_out)) return RK_ERR_INVALID_ARG;
    for (const int64_t s : {rows->q_stride_b, rows->q_stride_t, rows->k_stride_b, rows->k_stride_t, rows->v_stride_b, rows->v_stride_t})
        if (s < 0 || s % 8 != 0) return RK_ERR_INVALID_ARG;
    if (rope) {
        if (!rope->table || !aligned16(rope->table) || rope->max_pos <= 0) return RK_ERR_INVALID_ARG;
        if (rope->rot_dim <= 0 || rope->rot_dim > kD || rope->rot_dim % 16 != 0) return RK_ERR_UNSUPPORTED;
    }
    return RK_OK;
}

// In place a row has to be written where it was read: elsewhere it would be another token's.
static bool turned_over_others(const rk_geom* g, const rk_new_rows* rows, const void* q_out) {
    const int64_t token = (int64_t)g->n_q_heads * kD;
    return rows->q && rows->q == q_out && ((rows->n_new > 1 && rows->q_stride_t != token) || (g->batch > 1 && rows->q_stride_b != rows->n_new * token));
}

static RopeParams rope_params(const rk_geom* geom, const rk_new_rows* rows, const rk_rope* rope, const int32_t* positions,
                              const int32_t* seq_lens, const int32_t* new_lens, void* q_out, const int32_t* pred, int32_t pred_val) {
    RopeParams p{};
    p.q = (const uint16_t*)rows->q; p.k = (const uint16_t*)rows->k; p.v = (const uint16_t*)rows->v;
    p.q_b = rows->q_stride_b; p.q_t = rows->q_stride_t; p.k_b = rows->k_stride_b; p.k_t = rows->k_stride_t;
    p.v_b = rows->v_stride_b; p.v_t = rows->v_stride_t;
    if (rope) { p.rope = rope->table; p.max_pos = rope->max_pos; p.rot = rope->rot_dim; p.interleaved = rope->interleaved; }
    p.positions = positions; p.seq_lens = seq_lens; p.new_lens = new_lens;
    p.n_new = rows->n_new; p.Hq = geom->n_q_heads; p.Hkv = geom->n_kv_heads;
    p.q_out = (uint16_t*)q_out;
    p.pred = pred; p.pred_val = pred_val;
    return p;
}

}  // namespace rk

using namespace rk;

extern "C" int rk_rope_table(float* table, int32_t max_pos, int32_t rot_dim, const rk_rope_scaling* scaling, void* stream) {
    if (!table || !aligned16(table) || max_pos <= 0 || !scaling) return RK_ERR_INVALID_ARG;
    if (rot_dim <= 0 || rot_dim > kD || rot_dim % 16 != 0) return RK_ERR_UNSUPPORTED;
    if (!(scaling->base > 0.0) || !(scaling->factor > 0.0) || !isfinite(scaling->amplitude)) return RK_ERR_INVALID_ARG;
    if (scaling->original_len > 0.0 && !(scaling->low_turns < scaling->high_turns)) return RK_ERR_INVALID_ARG;
    hipLaunchKernelGGL(rope_table_kernel, dim3(max_pos), dim3(64), 0, (hipStream_t)stream, table, rot_dim, *scaling);
    return launch_status();
}

extern "C" int rk_rope_append(const rk_geom* geom, const rk_new_rows* rows, const rk_rope* rope, const int32_t* positions,
                              rk_kv cache, const int32_t* seq_lens, const int32_t* new_lens, void* q_out,
                              const int32_t* pred, int32_t pred_val, void* stream) {
    int rc = check_rope(geom, rows, rope, seq_lens, q_out);
    if (rc != RK_OK) return rc;
    if ((rc = check_kv(cache)) != RK_OK) return rc;
    RopeParams p = rope_params(geom, rows, rope, positions, seq_lens, new_lens, q_out, pred, pred_val);
    p.ck = (uint16_t*)cache.k; p.cv = (uint16_t*)cache.v; p.c_b = cache.stride_b; p.c_h = cache.stride_h; p.capacity = (int32_t)cache.capacity;
    p.rows_per_token = (rows->q ? p.Hq : 0) + 2 * p.Hkv;
    const int64_t wgs = ((int64_t)p.n_new * p.rows_per_token + 31) / 32;
    if (wgs * 32 > INT32_MAX) return RK_ERR_UNSUPPORTED;
    if (turned_over_others(geom, rows, q_out)) return RK_ERR_INVALID_ARG;
    hipLaunchKernelGGL(rope_append_kernel, dim3((unsigned)wgs, geom->batch), dim3(256), 0, (hipStream_t)stream, p);
    return launch_status();
}

extern "C" int rk_rope_append_q8(const rk_geom* geom, const rk_new_rows* rows, const rk_rope* rope, const int32_t* positions,
                                 const rk_kv8* cache, const int32_t* seq_lens, const int32_t* new_lens, void* q_out,
                                 const int32_t* pred, int32_t pred_val, void* stream) {
    int rc = check_rope(geom, rows, rope, seq_lens, q_out);
    if (rc != RK_OK) return rc;
    if ((rc = check_kv8(cache)) != RK_OK) return rc;
    RopeParams p = rope_params(geom, rows, rope, positions, seq_lens, new_lens, q_out, pred, pred_val);
    p.c8 = *cache;
    p.rows_per_token = rows->q ? p.Hq : 0;
    const int64_t blocks = ((int64_t)p.n_new + p.c8.block - 2) / p.c8.block + 1;       // that n_new rows can touch
    const int64_t block_wgs = blocks * 2 * p.Hkv, q_wgs = ((int64_t)p.n_new * p.rows_per_token + 31) / 32;
    if (block_wgs + q_wgs * 32 > INT32_MAX) return RK_ERR_UNSUPPORTED;
    if (turned_over_others(geom, rows, q_out)) return RK_ERR_INVALID_ARG;
    p.block_wgs = (int32_t)block_wgs;
    const bool e4m3 = cache->format == RK_Q8_E4M3;
    auto kernel = cache->block == 128 ? (e4m3 ? rope_append_q8_kernel<RK_Q8_E4M3, 4> : rope_append_q8_kernel<RK_Q8_INT8, 4>)
                  : cache->block == 64 ? (e4m3 ? rope_append_q8_kernel<RK_Q8_E4M3, 2> : rope_append_q8_kernel<RK_Q8_INT8, 2>)
                                       : (e4m3 ? rope_append_q8_kernel<RK_Q8_E4M3, 1> : rope_append_q8_kernel<RK_Q8_INT8, 1>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(block_wgs + q_wgs), geom->batch), dim3(256), 0, (hipStream_t)stream, p);
    return launch_status();
}

extern "C" int rk_rope_append_paged(const rk_geom* geom, const rk_new_rows* rows, const rk_rope* rope, const int32_t* positions,
                                    const rk_pages* pages, const int32_t* table, int32_t table_width, const int32_t* seq_lens, const int32_t* new_lens,
                                    void* q_out, const int32_t* pred, int32_t pred_val, void* stream) {
    int rc = check_rope(geom, rows, rope, seq_lens, q_out);
    if (rc != RK_OK) return rc;
    if ((rc = check_pages(pages, true, false)) != RK_OK || (rc = check_table(pages, table, table_width)) != RK_OK) return rc;
    RopeParams p = rope_params(geom, rows, rope, positions, seq_lens, new_lens, q_out, pred, pred_val);
    p.pages = *pages;
    p.table = table; p.width = table_width; p.shift = page_shift(pages->page);
    p.capacity = table_width * pages->page;
    const bool bounds = pages->k_min != nullptr;
    p.rows_per_token = (rows->q ? p.Hq : 0) + (bounds ? 1 : 2) * p.Hkv;
    const int64_t touched = ((int64_t)p.n_new + pages->page - 2) / pages->page + 1;       // pages that n_new rows can touch
    const int64_t page_wgs = bounds ? touched * p.Hkv : 0, row_wgs = ((int64_t)p.n_new * p.rows_per_token + 31) / 32;
    if (!fits_launch(page_wgs + row_wgs, 256)) return RK_ERR_UNSUPPORTED;
    if (turned_over_others(geom, rows, q_out)) return RK_ERR_INVALID_ARG;
    p.block_wgs = (int32_t)page_wgs;
    auto kernel = bounds ? rope_append_paged_kernel<true> : rope_append_paged_kernel<false>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(page_wgs + row_wgs), geom->batch), dim3(256), 0, (hipStream_t)stream, p);
    return launch_status();
}
