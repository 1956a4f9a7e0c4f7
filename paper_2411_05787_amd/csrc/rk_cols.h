// Attention of a few query columns of one KV head over rows that stream past once: the tile of 32 rows that the step over the
// cache of 8 bits (rk_q8.hip) and the prompt attention of few tokens (rk_prompt.hip) share.
//
// A wavefront takes 32 rows (two blocks of 16) and up to 16 columns:
//   S^T = K Q^T   v_mfma_f32_16x16x32_bf16: lane (n, g) = (lane % 16, lane / 16) holds row n of each block of K, and gets column n, rows
//                 4 g .. 4 g + 3 of each block;
//   O^T += V^T P^T  the contraction slots are numbered the way S^T left the rows in the lanes (slot 8 g + e is row 4 g + e of block e / 4), so P
//                 goes from the softmax to the matrix cores without leaving its lane.  V's rows come as they lie in memory, eight dims
//                 to a lane (dims 8 n ..), and the lane's 8 x 8 piece is turned around in registers: v_perm_b32 puts two rows'
//                 values of a dim side by side.  For 8 bits that is one permutation per four values and one conversion per two; LDS is
//                 not used and no wavefront waits for another until the end.
// P is handed over as two bf16 operands hi + lo (about 17 bits): memory sets the time, not the matrix cores.
#pragma once

#include "rk_q8.h"

namespace rk {

constexpr int kBf16 = 2;                      // beside RK_Q8_E4M3 and RK_Q8_INT8
constexpr int kColWaves = 4;

// The dims of a row that a lane's four operands of S^T hold: where they start.  8-bit rows are read 16 dims at a time.
template <bool BYTES> __device__ __forceinline__ int operand_dim(int s, int g) {
    return BYTES ? 64 * (s >> 1) + 16 * g + 8 * (s & 1) : 32 * s + 8 * g;
}

template <int FORMAT> struct TileRows {       // bf16
    u32x4 k[2][4], v[8];
};
template <> struct TileRows<RK_Q8_E4M3> { u32x4 k[2][2]; uint2 v[8]; };
template <> struct TileRows<RK_Q8_INT8> { u32x4 k[2][2]; uint2 v[8]; };

// Row of the tile that slot e of lane group g of the second product is.
__device__ __forceinline__ int slot_row(int e, int g) { return (e >> 2) * 16 + 4 * g + (e & 3); }

// Requests the rows at..at + 31 of k, v (base pointers of the (sequence, KV head), the same in the whole wavefront), of which `left` exist (any
// number, also none): the tile is a buffer of its own, so that a lane's place in it is worked out once for all tiles and rows past the end read as
// zeros without traffic. All are streamed: see load_rows16.
constexpr int kStreamAux = 2;                 // cache-policy operand of buffer loads: nt
template <int FORMAT>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_buffer(const void* base, int at, int left) {
    constexpr int row = FORMAT == kBf16 ? kD * 2 : kD;
    int rows = min(left, kTileRows);
    asm("" : "+s"(rows));                     // (scalar minimum and maximum, one after the other)
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>((const uint8_t*)base + (int64_t)at * row), 0, max(rows, 0) * row, 0x00020000);
}
template <int FORMAT, bool BYTES>
__device__ __forceinline__ void request_keys(TileRows<FORMAT>& t, const void* k, int at, int left) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const __amdgpu_buffer_rsrc_t r = tile_buffer<FORMAT>(k, at, left);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        if constexpr (FORMAT == kBf16) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                t.k[x][s] = __builtin_amdgcn_raw_buffer_load_b128(r, (16 * x + n) * (kD * 2) + operand_dim<BYTES>(s, g) * 2, 0, kStreamAux);
        } else {
#pragma unroll
            for (int s = 0; s < 2; ++s) t.k[x][s] = __builtin_amdgcn_raw_buffer_load_b128(r, (16 * x + n) * kD + 64 * s + 16 * g, 0, kStreamAux);
        }
    }
}
template <int FORMAT>
__device__ __forceinline__ void request_values(TileRows<FORMAT>& t, const void* v, int at, int left) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const __amdgpu_buffer_rsrc_t r = tile_buffer<FORMAT>(v, at, left);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        if constexpr (FORMAT == kBf16) {
            t.v[e] = __builtin_amdgcn_raw_buffer_load_b128(r, slot_row(e, g) * (kD * 2) + 16 * n, 0, kStreamAux);
        } else {
            const auto x = __builtin_amdgcn_raw_buffer_load_b64(r, slot_row(e, g) * kD + 8 * n, 0, kStreamAux);
            t.v[e] = make_uint2(x[0], x[1]);
        }
    }
}

// The two values in the low (HIGH: upper) half of w, as a pair of bf16 (every value of either format is one).
template <int FORMAT, bool HIGH>
__device__ __forceinline__ uint32_t pair_of(uint32_t w) {
    if constexpr (FORMAT == RK_Q8_E4M3) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, HIGH));
    else return HIGH ? pack_bf16((float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)) : pack_bf16((float)(int8_t)w, (float)(int8_t)(w >> 8));
}

// Operand s of block x of S^T.
template <int FORMAT>
__device__ __forceinline__ bf16x8 key_operand(const TileRows<FORMAT>& t, int x, int s) {
    if constexpr (FORMAT == kBf16) {
        return __builtin_bit_cast(bf16x8, t.k[x][s]);
    } else {
        const uint32_t a = t.k[x][s >> 1][2 * (s & 1)], b = t.k[x][s >> 1][2 * (s & 1) + 1];
        const u32x4 o = {pair_of<FORMAT, false>(a), pair_of<FORMAT, true>(a), pair_of<FORMAT, false>(b), pair_of<FORMAT, true>(b)};
        return __builtin_bit_cast(bf16x8, o);
    }
}

// Operands 4 h .. 4 h + 3 of the second product: operand i holds dim 8 n + i of the lane's eight rows.
template <int FORMAT>
__device__ __forceinline__ void value_operands(const TileRows<FORMAT>& t, int h, u32x4 (&o)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {             // rows 2 j and 2 j + 1
        if constexpr (FORMAT == kBf16) {
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const uint32_t a = t.v[2 * j][2 * h + d], b = t.v[2 * j + 1][2 * h + d];
                o[2 * d][j] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                o[2 * d + 1][j] = __builtin_amdgcn_perm(b, a, 0x07060302u);
            }
        } else {
            const uint32_t a = h ? t.v[2 * j].y : t.v[2 * j].x, b = h ? t.v[2 * j + 1].y : t.v[2 * j + 1].x;
            const uint32_t w0 = __builtin_amdgcn_perm(b, a, 0x05010400u), w1 = __builtin_amdgcn_perm(b, a, 0x07030602u);
            o[0][j] = pair_of<FORMAT, false>(w0); o[1][j] = pair_of<FORMAT, true>(w0);
            o[2][j] = pair_of<FORMAT, false>(w1); o[3][j] = pair_of<FORMAT, true>(w1);
        }
    }
}

// The queries' operands are here once this returns.  Called behind the first tile's requests: left to itself the compiler finds them still on their
// way where the loop begins, and every round of the loop then waits for all that is in flight (with tiles as buffers 18.4 -> 16.8 us for 32777 rows
// of 8 bits).
__device__ __forceinline__ void queries_here(bf16x8 (&q)[4]) {
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        u32x4 x = __builtin_bit_cast(u32x4, q[s]);
        asm volatile("" : "+v"(x));
        q[s] = __builtin_bit_cast(bf16x8, x);
    }
}

// Running state of a wavefront's column n: maximum (the same in the four lane groups), this lane's share of the sum, and 32 dims of the
// output: o[i][r] is dim 8 (4 g + r) + i.
struct ColState {
    float m, l;
    f32x4 o[8];
    __device__ __forceinline__ void clear() {
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
};

template <int FORMAT>
__device__ __forceinline__ void tile_scores(const TileRows<FORMAT>& t, const bf16x8 (&q)[4], float (&s)[2][4]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < 4; ++k) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key_operand<FORMAT>(t, x, k), q[k], acc, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[x][i] = acc[i];
    }
}

// Scores (natural units, -inf where hidden) -> weights against the running maximum, which grows where it has to.
__device__ __forceinline__ void tile_softmax(ColState& st, float (&s)[2][4]) {
    float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    mx = max_xor32(max_xor16(mx));
    if (__any(mx > st.m)) {
        const float m = fmaxf(st.m, mx);
        const float alpha = m == -INFINITY ? 1.f : fast_exp2((st.m - m) * kLog2e);      // (the first rows: 0 times nothing)
        st.m = m;
        st.l *= alpha;
#pragma unroll
        for (int i = 0; i < 8; ++i) st.o[i] *= alpha;
    }
    const float ref = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { s[x][i] = fast_exp2((s[x][i] - ref) * kLog2e); st.l += s[x][i]; }
    }
}

// Weights, each times its row's scale -> the two operands hi + lo.
__device__ __forceinline__ void weight_operands(const float (&p)[2][4], bf16x8& hi, bf16x8& lo) {
    u32x4 h, l;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float a = p[x][2 * i], b = p[x][2 * i + 1];
            h[2 * x + i] = pack_bf16(a, b);
            l[2 * x + i] = pack_bf16(a - bf16_lo(h[2 * x + i]), b - bf16_hi(h[2 * x + i]));
        }
    }
    hi = __builtin_bit_cast(bf16x8, h);
    lo = __builtin_bit_cast(bf16x8, l);
}

template <int FORMAT>
__device__ __forceinline__ void tile_output(const TileRows<FORMAT>& t, ColState& st, bf16x8 hi, bf16x8 lo) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        u32x4 o[4];
        value_operands<FORMAT>(t, h, o);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, o[i]);
            st.o[4 * h + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, hi, st.o[4 * h + i], 0, 0, 0);
            st.o[4 * h + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, lo, st.o[4 * h + i], 0, 0, 0);
        }
    }
}

// The workgroup's columns < ncols <= C merged over its W wavefronts: calls put(column, dim, o0, o1, L) for the pairs of dims (the unnormalised
// output against the common maximum, and its sum) and stat(column, m, l).
template <int W, int C> struct ColMergeLds { float m[W][16], l[W][16]; float o[W][C][kD]; };
template <int W, int C, class Put, class Stat>
__device__ __forceinline__ void merge_columns(ColMergeLds<W, C>& lds, ColState& st, int ncols, Put&& put, Stat&& stat) {
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, n = lane & 15, g = lane >> 4;
    const float l = sum_xor32(sum_xor16(st.l));
    if (g == 0) { lds.m[w][n] = st.m; lds.l[w][n] = l; }
    if (n < ncols) {
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float4* to = reinterpret_cast<float4*>(&lds.o[w][n][8 * (4 * g + r)]);
            to[0] = make_float4(st.o[0][r], st.o[1][r], st.o[2][r], st.o[3][r]);
            to[1] = make_float4(st.o[4][r], st.o[5][r], st.o[6][r], st.o[7][r]);
        }
    }
    __syncthreads();
    for (int x = tid; x < ncols * (kD / 2); x += W * 64) {
        const int c = x / (kD / 2), d = 2 * (x % (kD / 2));
        float M = lds.m[0][c];
#pragma unroll
        for (int i = 1; i < W; ++i) M = fmaxf(M, lds.m[i][c]);
        float L = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float a = lds.m[i][c] == -INFINITY ? 0.f : fast_exp2((lds.m[i][c] - M) * kLog2e);
            const float2 v = *reinterpret_cast<const float2*>(&lds.o[i][c][d]);
            // (a wavefront without rows has nothing; NaN statistics stay NaN)
            L = fmaf(a, lds.l[i][c], L); o0 = fmaf(a, v.x, o0); o1 = fmaf(a, v.y, o1);
        }
        put(c, d, o0, o1, L);
        if (d == 0) stat(c, M, L);
    }
}

}  // namespace rk
