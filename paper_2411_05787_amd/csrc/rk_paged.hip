// rk_paged_attn, rk_prefix_attn and rk_sparse_attn: attention of new tokens over a cache in pages.
//
// The kernels of rk_prompt.h over rows that a table leads to, and for up to 16 rows (a decode step's token, drafted ones, one token over its chosen
// pages) the streaming one below.  A prefix that all sequences share is read once: the queries of all of them are the rows of one
// call over it (kRowsShared), each sequence's own rows behind it are another's, and the two leave partial results that one launch joins.
#include "rk_prompt.h"
#include "rk_pages.h"

namespace rk {

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

// ---- up to 16 rows in all ----
// prompt_cols_kernel over units of 16 rows: each is a buffer of its own inside its page.  A wavefront looks its next 64 tiles up at once, a lane each, and
// takes the page numbers from the lanes: no wait for a number of the table stands before a request.  SUB: pairs side by side in a workgroup, W wavefronts and a
// room each; all of its wavefronts come to one barrier, also those that have nothing to do (there: x0 < 0).
// The running maximum is in units of ln 2 and follows the true one only when that has grown by more than 8 (see prompt_tile).  A chosen token's rows are no more
// than 8: the upper eight columns repeat them, and hold the weights' low parts beside the high ones of the lower, so that one matrix instruction takes both; and as
// tokens share rows, which come out of the L2 then, its keys are read in whole rows and turned into the operand's layout by way of LDS: straight into it, every 16
// lanes of a request touch 16 lines (500 tokens of 28 heads over 4, 32 pages of 64 rows each: 163 us so, 126 in whole rows).
// kRowsChosenOnce: few tokens to a page, whose rows pass the caches by as streamed ones do elsewhere.  16 sequences of 32 heads over 8, 64 of 1024 pages of 32 rows for each token, once
// and kept: 1 token 28.0 and 31.8 us, 4 tokens 81 and 87, 8 tokens 152 and 149, 16 tokens 279 and 233; the 500 tokens 198 and 110.
// The form without a cap or bias has room for three wavefronts to a SIMD without spilling (124 -> 120 us).
// What is left there is what the L2s miss: 2.1 GB are asked for, 0.8 GB come from behind them, at 6.5 TB/s.
constexpr int kTurnRow = kD * 2 + 16, kTurn = kTileRows * kTurnRow;      // (rows of LDS: 16 of an operand fall on different banks)
template <int W, int ROWS> constexpr int cols_lds() {
    constexpr int merge = (int)sizeof(ColMergeLds<W, 16>), turn = ROWS == kRowsChosen || ROWS == kRowsChosenOnce ? W * kTurn : 0;
    return merge > turn ? merge : turn;
}
template <int W, int CAP, bool SLOPE, int ROWS, int SUB = 1>
__device__ __forceinline__ void paged_cols(const PromptParams& p, const int x0, const int y0, const int z0, unsigned char* room) {
    auto leave = [&]() { if constexpr (SUB > 1) __syncthreads(); };
    if (SUB > 1 && x0 < 0) { leave(); return; }
    constexpr bool CHOSEN = ROWS == kRowsChosen || ROWS == kRowsChosenOnce, SHARED = ROWS == kRowsShared;
    int b, g, split, slot, parts = p.splits, token = 0;
    if constexpr (CHOSEN) {                   // (KV heads fastest: those of all tokens that share rows meet in few caches)
        g = (int)((uint32_t)x0 % (uint32_t)p.Hkv);
        const int rest = (int)((uint32_t)x0 / (uint32_t)p.Hkv), bt = rest / p.splits;
        split = rest - bt * p.splits;
        b = bt / p.n_new; token = bt - b * p.n_new;
        slot = (bt * p.Hkv + g) * p.splits + split;
    } else {
        g = y0; b = SHARED ? 0 : z0; split = x0;
        slot = z0 * p.splits + x0;
        if (!SHARED && p.ragged != 0) {
            AttnParams a;
            a.ragged_batch = p.ragged; a.nch = p.splits; a.share_cap = kMaxSplits; a.cap2 = p.cap_rows; a.max_rows2 = p.max_len;
            const RaggedSlot r = ragged_slot<false>(a, p.seq_lens, slot);
            if (r.b < 0) return;
            b = r.b; split = r.c; parts = r.nchunks;
        }
    }
    if (!SHARED && p.pred != nullptr && p.pred[b] != p.pred_val) { leave(); return; }
    const Tokens tok = SHARED ? Tokens{} : tokens_of(p, b);
    const int n_rows = SHARED ? p.rows : CHOSEN ? (token < tok.n ? p.G : 0) : tok.n * p.G;
    if (n_rows == 0) { leave(); return; }
    const int tid = SUB > 1 ? threadIdx.x % (W * 64) : threadIdx.x;
    const int64_t bg = SHARED ? g : (int64_t)b * p.Hkv + g;
    const bool partial = p.splits > 1 || p.joined != 0;
    if (!CHOSEN && partial && split == 0 && tid == 0) { p.parts[2 * bg] = slot; p.parts[2 * bg + 1] = parts; }
    const int lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 15, gr = lane >> 4;
    const int mine = CHOSEN ? col & 7 : col;
    bool real = mine < n_rows;
    const int r0 = (CHOSEN ? token * p.G : 0) + min(mine, n_rows - 1);
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
    ScoreForm form = score_form<CAP>(p, kLog2e);
    if (!SLOPE && form.a < 0.f) {             // raw products are compared below: their order has to be the scores'
        form.a = -form.a;
#pragma unroll
        for (int s = 0; s < 4; ++s) q[s] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[s]) ^ 0x80008000u);
    }
    const float slope = SLOPE && p.slopes != nullptr ? p.slopes[me.head] * kLog2e : 0.f;
    const uint16_t* k = p.k + (int64_t)g * p.s_h;
    const uint16_t* v = p.v + (int64_t)g * p.s_h;
    const int32_t* table = p.table + (SHARED ? 0 : (int64_t)b * p.width);
    const int32_t* idx = CHOSEN ? p.idx + (((int64_t)b * p.n_new + token) * p.Hkv + g) * p.n_idx : nullptr;
    const int step = parts * W, in_page = (1 << p.shift) - 1;

    // this lane's of the wavefront's next 64 tiles: each unit's first row, and where it is in bytes from the head's first page (the highest bit: there is none)
    int first[2];
    uint32_t at_lo[2], at_hi[2];
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
            const int page = there ? table[j] : -1;
            there = (uint32_t)page < (uint32_t)p.n_pages;
            const uint64_t where = there ? (uint64_t)page * (uint64_t)(p.s_p * 2) + (uint32_t)((first[c] & in_page) * (kD * 2)) : 0;
            at_lo[c] = (uint32_t)where;
            at_hi[c] = (uint32_t)(where >> 32) | (there ? 0u : 0x80000000u);
        }
        // (here before the loop goes on: a request that may be in flight or not would be waited for with all others)
        asm volatile("" : "+v"(at_lo[0]), "+v"(at_hi[0]), "+v"(at_lo[1]), "+v"(at_hi[1]));
    };
    // A tile: its units' first rows, how many rows of each there are (0: none), and where they are in bytes from the head's first page.
    struct Tile { int row[2], rows[2]; int64_t at[2]; };
    auto tile_at = [&](int n) {
        Tile x;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const uint32_t hi32 = __builtin_amdgcn_readlane(at_hi[c], n);
            x.row[c] = __builtin_amdgcn_readlane(first[c], n);
            int rows = min(hi - x.row[c], 16);
            asm("" : "+s"(rows));
            rows = max(rows, 0) & ~((int)hi32 >> 31);
            asm("" : "+s"(rows));             // (no branch)
            x.rows[c] = rows;
            x.at[c] = (int64_t)((uint64_t)(hi32 & 0x7fffffffu) << 32 | (uint32_t)__builtin_amdgcn_readlane(at_lo[c], n));
        }
        return x;
    };
    auto buffer = [&](const uint16_t* base, const Tile& x, int c) {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(reinterpret_cast<const uint8_t*>(base) + x.at[c]), 0, x.rows[c] * (kD * 2), 0x00020000);
    };
    constexpr int kAux = ROWS == kRowsChosen ? 0 : kStreamAux;
    TileRows<kBf16> rows;
    auto ask_keys = [&](const Tile& x) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const __amdgpu_buffer_rsrc_t r = buffer(k, x, c);
#pragma unroll
            for (int s = 0; s < 4; ++s) rows.k[c][s] = CHOSEN ? __builtin_amdgcn_raw_buffer_load_b128(r, (4 * gr + s) * (kD * 2) + 16 * col, 0, kAux) : __builtin_amdgcn_raw_buffer_load_b128(r, col * (kD * 2) + operand_dim<false>(s, gr) * 2, 0, kAux);
        }
    };
    auto ask_values = [&](const Tile& x) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const __amdgpu_buffer_rsrc_t r = buffer(v, x, c);
#pragma unroll
            for (int e = 0; e < 4; ++e) rows.v[4 * c + e] = __builtin_amdgcn_raw_buffer_load_b128(r, (4 * gr + e) * (kD * 2) + 16 * col, 0, kAux);
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
        if constexpr (CHOSEN) {
            unsigned char* turn = room + w * kTurn;
#pragma unroll
            for (int e = 0; e < 8; ++e) *reinterpret_cast<u32x4*>(turn + (16 * (e >> 2) + 4 * gr + (e & 3)) * kTurnRow + 16 * col) = rows.k[e >> 2][e & 3];
            wave_lds_sync();
#pragma unroll
            for (int e = 0; e < 8; ++e) rows.k[e >> 2][e & 3] = *reinterpret_cast<const u32x4*>(turn + (16 * (e >> 2) + col) * kTurnRow + 64 * (e & 3) + 16 * gr);
            wave_lds_sync();
        }
        tile_scores<kBf16>(rows, q, s);
        if (++n == 64) { look(t + step); n = 0; }
        const Tile next = tile_at(n);         // (past the last tile: nothing)
        ask_keys(next);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                s[x][i] = bend<CAP>(s[x][i], form);
                if constexpr (SLOPE) s[x][i] = fmaf(-slope, fabsf((float)(me.pos - now.row[x] - 4 * gr) - (float)i), fmaf(s[x][i], form.a, form.b));
            }
        // (one sign of them all, and no branch for each)
        const int inside = min(min(now.rows[0], now.rows[1]) - 16, min(min(now.row[0], now.row[1]) - in_lo, in_hi - 16 - max(now.row[0], now.row[1])));
        const bool masked = inside < 0;
        auto sees = [&](int x, int j) { return now.rows[x] != 0 && j >= me.lo && j < me.hi; };
        if (masked) {
            asm volatile("" ::: "memory");    // (a branch: most tiles have nothing to mask)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[x][i] = sees(x, now.row[x] + 4 * gr + i) ? s[x][i] : -INFINITY;
        }
        float mx = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        mx = max_xor32(max_xor16(mx));
        if constexpr (!SLOPE) mx = fmaf(mx, form.a, form.b);
        if (__any(mx > st.m + 8.f)) {
            const float to = mx > st.m + 8.f ? mx : st.m, alpha = to == -INFINITY ? 1.f : fast_exp2(st.m - to);
            st.m = to;
            st.l *= alpha;
#pragma unroll
            for (int i = 0; i < 8; ++i) st.o[i] *= alpha;
        }
        const float from = (SLOPE ? 0.f : form.b) - (st.m == -INFINITY ? 0.f : st.m);
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) { s[x][i] = fast_exp2(SLOPE ? s[x][i] + from : fmaf(s[x][i], form.a, from)); st.l += s[x][i]; }
        bf16x8 ph, pl;
        weight_operands(s, ph, pl);
        if constexpr (CHOSEN) {
            const u32x4 h = __builtin_bit_cast(u32x4, ph), l = __builtin_bit_cast(u32x4, pl);
            u32x4 both;
#pragma unroll
            for (int e = 0; e < 4; ++e) both[e] = col < 8 ? h[e] : l[e];
            ph = __builtin_bit_cast(bf16x8, both);
        }
        bool bad = false;
        if (masked) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bad = bad || has_non_finite(rows.v[e]);
            if (bad) {
#pragma unroll
                for (int e = 0; e < 8; ++e) drop_non_finite(rows.v[e]);
            }
        }
        if constexpr (CHOSEN) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 o[4];
                value_operands<kBf16>(rows, h, o);
#pragma unroll
                for (int i = 0; i < 4; ++i) st.o[4 * h + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, o[i]), ph, st.o[4 * h + i], 0, 0, 0);
            }
        } else {
            tile_output<kBf16>(rows, st, ph, pl);
        }
        if (__any(bad)) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
                for (int i = 0; i < now.rows[x]; ++i) {
                    if (!sees(x, now.row[x] + i) || (CHOSEN && col >= 8)) continue;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const u32x4 u = *reinterpret_cast<const u32x4*>(reinterpret_cast<const uint8_t*>(v) + now.at[x] + (int64_t)i * (kD * 2) + 16 * (4 * gr + r));
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

    if constexpr (CHOSEN) {                   // the low parts' products to the high ones'
        __syncthreads();                      // (other wavefronts' keys are in the room still)
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) st.o[i][r] += dpp_move_f<kDppRor8>(st.o[i][r]);
    }
    ColMergeLds<W, 16>& lds = *reinterpret_cast<ColMergeLds<W, 16>*>(room);
    if (partial) {
        // (columns of one pair and part side by side)
        const int64_t at = CHOSEN ? (int64_t)slot * p.G : ((int64_t)g * p.splits * (SHARED ? 1 : p.batch) + slot) * (SHARED ? p.rows : p.n_new * p.G);
        merge_columns(lds, st, n_rows,
                      [&](int x, int d, float o0, float o1, float) {
                          *reinterpret_cast<float2*>(p.part_o + (at + x) * kD + d) = make_float2(o0, o1);
                      },
                      [&](int x, float m, float l) {
                          *reinterpret_cast<float2*>(p.part_ml + (at + x) * 2) = make_float2(m, l);
                      }, tid, 1.f);
        return;
    }
    if constexpr (SHARED || SUB > 1) return;  // (never: those results are joined)
    auto out_row = [&](int x) { const int i = x / p.G; return ((int64_t)b * p.n_new + token + i) * p.Hq + g * p.G + (x - i * p.G); };
    float* o = &lds.o[0][0][0];
    __shared__ float sInv[16];
    merge_columns(lds, st, n_rows,
                  [&](int x, int d, float o0, float o1, float) { o[x * kD + d] = o0; o[x * kD + d + 1] = o1; },
                  [&](int x, float m, float l) {
                      sInv[x] = l == 0.f ? 0.f : 1.f / l;
                      if (p.lse != nullptr) p.lse[out_row(x)] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * (1.f / kLog2e);
                  }, tid, 1.f);
    __syncthreads();
    for (int x = threadIdx.x; x < n_rows * (kD / 2); x += W * 64) {
        const int r = x / (kD / 2), d = 2 * (x % (kD / 2));
        *reinterpret_cast<uint32_t*>(p.out + out_row(r) * kD + d) = pack_bf16(o[r * kD + d] * sInv[r], o[r * kD + d + 1] * sInv[r]);
    }
}

template <int W, int CAP, bool SLOPE, int ROWS>
__global__ __launch_bounds__(W * 64, (ROWS == kRowsChosen || ROWS == kRowsChosenOnce) && CAP == kNoCap && !SLOPE ? 3 : W == kColWaves ? 2 : 1)
void paged_cols_kernel(const PromptParams p) {
    __shared__ __attribute__((aligned(16))) unsigned char room[cols_lds<W, ROWS>()];
    paged_cols<W, CAP, SLOPE, ROWS>(p, (int)blockIdx.x, (int)blockIdx.y, (int)blockIdx.z, room);
}

// ---- a shared prefix ----
// The first `shared_wgs` workgroups go over the shared rows for the queries of all sequences, the others over each sequence's own: in one launch, as both wait more
// than they work (one token of 64 sequences of 32 heads over 8 behind 8192 rows, 200-1000 rows of their own: 51 us in two launches, 41 in one).  The matrix
// cores are busy for 4.3 of its 32 us, and for 7.6 of 36 with five tokens of 6 sequences of 28 heads over 4 behind 32777 rows, the vector units for 6 and 8.
// The shared part, with a row or two of the sequences' own: behind 8192, 16384, 32768, 65536 rows 22.6, 33.0, 56.4, 104.7 us (the drafted tokens
// 17.7, 21.9, 34.4, 52.4), that is about 12 and 0.65-0.75 for each stage of 32 rows in 256 workgroups.  With one wavefront to a SIMD and requests two stages
// ahead that is waiting; for which of the reads has not been measured.
// Weights: where all query rows of a KV head together are more than 16, those over the shared rows meet V as bf16, 2^-8 (prompt_tile, half the matrix instructions of two
// parts), also where a sequence's own rows are columns, whose weights keep 2^-17 there: errors against 64 bits 0.0023 and 0.0017 of the outputs, the
// latter all by their own rounding.
// Both leave partial results.  OWN: wavefronts to a pair where a sequence's own are columns, 0: row tiles.  Two, and two pairs to a
// workgroup, where one workgroup to a pair would be more than the chip has room for beside the shared ones (there: 33.7 -> 31.1 us).
template <int CAP, bool SLOPE, bool ALL_COLS, int OWN>
__global__ __launch_bounds__(256, 2)
void prefix_kernel(const PromptParams all, const PromptParams own, const int32_t shared_wgs, const int32_t own_parts) {
    constexpr int kCols = (int)sizeof(ColMergeLds<kColWaves, 16>), kRoom = ALL_COLS ? kCols : tile_lds(1);
    static_assert(kRoom >= kCols && 2 * sizeof(ColMergeLds<2, 16>) <= (size_t)kRoom, "room");
    __shared__ __attribute__((aligned(16))) unsigned char room[kRoom];
    if ((int)blockIdx.x < shared_wgs) {
        if constexpr (ALL_COLS) paged_cols<kColWaves, CAP, SLOPE, kRowsShared>(all, (int)(blockIdx.x % (uint32_t)all.splits), (int)(blockIdx.x / (uint32_t)all.splits), 0, room);
        else prompt_tile<1, CAP, SLOPE, kRowsShared>(all, blockIdx.x, room);
        return;
    }
    const int x = (int)blockIdx.x - shared_wgs;
    if constexpr (OWN != 0) {
        constexpr int SUB = kColWaves / OWN;
        const int sub = SUB == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / (OWN * 64)), y = SUB * x + sub;
        const int rest = y / own.splits, b = rest / own.Hkv;
        paged_cols<OWN, CAP, SLOPE, kRowsPaged, SUB>(own, y < own_parts ? y - rest * own.splits : -1, rest - b * own.Hkv, b, room + sub * sizeof(ColMergeLds<OWN, 16>));
    } else {
        prompt_tile<1, CAP, SLOPE, kRowsPaged>(own, (uint32_t)x, room);
    }
}

// Joins the parts of a row, sum_s 2^(m_s - m) (l_s, o_s).   SOURCES = 2: those over the shared rows, then those over the sequence's own.
// TEAM wavefronts to a row: one, or where there are more than 16 parts four, of which each adds every fourth.  One token of 32 heads over 8, one sequence of
// 32768 rows (the call, one and four): 31.9 and 27.3 us, behind a prefix of 8192 rows 26.7 and 18.2; where rows are many it is equal (64 sequences behind 8192 rows, 7.2
// and 7.4 us, half of it the launch and the rest the partial results' 17 MB).
template <int SOURCES, int TEAM>
__global__ __launch_bounds__(256)
void paged_merge_kernel(const PromptParams p, const PartSource s0, const PartSource s1) {
    constexpr int N = SOURCES * kMaxSplits, kRound = 8;
    const int g = blockIdx.y, b = blockIdx.z, w = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int row = TEAM == 1 ? blockIdx.x * 4 + w : blockIdx.x, mine = TEAM == 1 ? 0 : w;
    if (p.pred != nullptr && p.pred[b] != p.pred_val) return;
    __shared__ float sW[4][N];
    // (requested with the sequence's length: of a row that there is not, any numbers, which nothing is made of)
    const int safe_row = min(row, p.n_new * p.G - 1);
    const PartRow r0 = part_row(s0, p, b, g, safe_row);
    PartRow r1{0, 0, 0};
    if constexpr (SOURCES == 2) r1 = part_row(s1, p, b, g, safe_row);
    asm volatile("" :: "s"(__builtin_amdgcn_readfirstlane(r0.n)), "s"(__builtin_amdgcn_readfirstlane(r1.n)));
    const Tokens tok = tokens_of(p, b);
    if (row >= tok.n * p.G) return;
    if (SOURCES == 1 && p.joined == 0 && !s0.cols && s0.rows_of == kRowsPaged && r0.n == 1) return;      // (the output is there already)
    // what a lane takes of both sources' statistics, and the first outputs, requested together
    const int n = r0.n + r1.n;
    float m[N / 64], l[N / 64], top = -INFINITY;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) {
        m[i] = -INFINITY; l[i] = 0.f;
        if (64 * i >= n) continue;            // (the same for the whole wavefront)
        const int s = min(lane + 64 * i, n - 1);
        const bool second = SOURCES == 2 && s >= r0.n;
        const float2 ml = *reinterpret_cast<const float2*>(second ? s1.ml + (r1.at + (int64_t)(s - r0.n) * r1.step) * 2 : s0.ml + (r0.at + (int64_t)s * r0.step) * 2);
        m[i] = lane + 64 * i < n ? ml.x : -INFINITY; l[i] = ml.y;
    }
    const float2* from0 = reinterpret_cast<const float2*>(s0.o + r0.at * kD) + lane;
    const float2* from1 = SOURCES == 2 ? reinterpret_cast<const float2*>(s1.o + r1.at * kD) + lane : nullptr;
    float2 v[kRound];
    auto request = [&](int s) {
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const int x = min(s + TEAM * i, n - 1);
            v[i] = SOURCES == 2 && x >= r0.n ? from1[(int64_t)(x - r0.n) * r1.step * (kD / 2)] : from0[(int64_t)x * r0.step * (kD / 2)];
        }
    };
    request(mine);
#pragma unroll
    for (int i = 0; i < N / 64; ++i) top = fmaxf(top, m[i]);
    top = wave_max(top);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < N / 64; ++i) {
        if (64 * i >= n) continue;
        const float a = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - top);
        sum = fmaf(a, l[i], sum);
        sW[w][lane + 64 * i] = a;
    }
    sum = wave_sum(sum);
    wave_lds_sync();
    float o0 = 0.f, o1 = 0.f;
    for (int s = mine; s < n; s += TEAM * kRound) {
        if (s != mine) request(s);
#pragma unroll
        for (int i = 0; i < kRound; ++i) {
            const float a = s + TEAM * i < n ? sW[w][s + TEAM * i] : 0.f;
            if (a != 0.f) { o0 = fmaf(a, v[i].x, o0); o1 = fmaf(a, v[i].y, o1); }      // (a part without rows left nothing)
        }
    }
    if constexpr (TEAM > 1) {
        __shared__ float2 sO[TEAM][64];
        sO[w][lane] = make_float2(o0, o1);
        __syncthreads();
        if (w != 0) return;
        o0 = o1 = 0.f;
#pragma unroll
        for (int y = 0; y < TEAM; ++y) { o0 += sO[y][lane].x; o1 += sO[y][lane].y; }
    }
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
static PagedKernel tile_form(int cap, bool slope) {
    constexpr int ROWS = kRowsPaged;
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
// rk_prompt_attn's launches, over pages.
static int launch_paged(PromptParams& p, const PromptPlan& plan, int64_t pairs, int cap, bool slope, hipStream_t st) {
    if (plan.cols) {
        auto kernel = plan.alone ? cols_form<kColAlone, kRowsPaged>(cap, slope) : cols_form<kColWaves, kRowsPaged>(cap, slope);
        hipLaunchKernelGGL(kernel, dim3(plan.splits, p.Hkv, p.batch), dim3((plan.alone ? kColAlone : kColWaves) * 64), 0, st, p);
    } else {
        auto kernel = plan.wide ? prompt_tile_kernel<2, kNoCap, false, kRowsPaged> : tile_form(cap, slope);
        const int64_t total = pairs * plan.row_tiles * plan.splits;
        // (the second workgroup of a compute unit in the opposite order: see rk_prompt_attn)
        p.first_round = !plan.wide && total <= 2 * kComputeUnits ? (int)((kComputeUnits + pairs - 1) / pairs) : INT32_MAX;
        hipLaunchKernelGGL(kernel, dim3((unsigned)total), dim3(256), 0, st, p);
    }
    return launch_status();
}
using PrefixKernel = void (*)(const PromptParams, const PromptParams, const int32_t, const int32_t);
template <bool ALL_COLS, int OWN_COLS> static PrefixKernel prefix_form(int cap, bool slope) {
    switch (cap) {
        case kNearCap: return slope ? prefix_kernel<kNearCap, true, ALL_COLS, OWN_COLS> : prefix_kernel<kNearCap, false, ALL_COLS, OWN_COLS>;
        case kFarCap: return slope ? prefix_kernel<kFarCap, true, ALL_COLS, OWN_COLS> : prefix_kernel<kFarCap, false, ALL_COLS, OWN_COLS>;
        default: return slope ? prefix_kernel<kNoCap, true, ALL_COLS, OWN_COLS> : prefix_kernel<kNoCap, false, ALL_COLS, OWN_COLS>;
    }
}
// What is launched, and how many of the sequences' own (pair, part)s a workgroup takes: all columns (a sequence has no more rows than the batch), columns of a
// sequence, or neither.  Two pairs to a workgroup only where a form of that kind is: the grid goes by what is returned here.
struct PrefixLaunch { PrefixKernel kernel; int per_wg; };
static PrefixLaunch prefix_launch(const PromptPlan& all, const PromptPlan& own, int64_t wgs_own, int cap, bool slope) {
    if (all.cols) return {prefix_form<true, kColWaves>(cap, slope), 1};
    if (!own.cols) return {prefix_form<false, 0>(cap, slope), 1};
    if (own.splits == 1 && wgs_own > kComputeUnits) return {prefix_form<false, 2>(cap, slope), 2};
    return {prefix_form<false, kColWaves>(cap, slope), 1};
}
// The workgroups over the shared rows: one to a compute unit, beside those over the sequences' own (one token of 64 sequences behind 8192 rows: 33.8 us, with
// two to a compute unit, which both wait for the matrix cores and leave twice the partial results, 44.0).
static PromptPlan shared_plan(int64_t pairs, int64_t rows, int64_t max_len) {
    PromptPlan f = prompt_plan_of(pairs, rows, max_len, false, false);
    f.alone = false;
    if (f.cols) return f;
    f.split_tiles = 4;
    int64_t s = kComputeUnits / (pairs * f.row_tiles);
    const int64_t most = (max_len + f.split_tiles * kPromptTile - 1) / (f.split_tiles * kPromptTile);
    if (s > most) s = most;
    if (s > kMaxSplits) s = kMaxSplits;
    f.splits = (int)(s < 1 ? 1 : s);
    return f;
}
template <int SOURCES>
static int launch_merge(const PromptParams& p, const PartSource& s0, const PartSource& s1, hipStream_t st) {
    const int rows = p.n_new * p.G, parts = s0.splits + (SOURCES == 2 ? s1.splits : 0);
    if (parts > 16) hipLaunchKernelGGL((paged_merge_kernel<SOURCES, 4>), dim3((unsigned)rows, p.Hkv, p.batch), dim3(256), 0, st, p, s0, s1);
    else hipLaunchKernelGGL((paged_merge_kernel<SOURCES, 1>), dim3((unsigned)((rows + 3) / 4), p.Hkv, p.batch), dim3(256), 0, st, p, s0, s1);
    return launch_status();
}

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
    if (!plan.cols && !fits_launch(pairs * plan.row_tiles * plan.splits, 256)) return RK_ERR_UNSUPPORTED;      // (a launch that splits, and so the join, is small)
    set_plan(p, plan);
    if (plan.splits > 1) {
        if (!place_parts(p, plan, pairs, rows, (char*)workspace, workspace_bytes)) return RK_ERR_WORKSPACE;
        p.ragged = plan.cols ? ragged_batch_of(geom) : 0;
    }
    hipStream_t st = (hipStream_t)stream;
    if ((rc = launch_paged(p, plan, pairs, cap, slope, st)) != RK_OK || plan.splits == 1) return rc;
    const PartSource s = source_of(p, kRowsPaged, (int)rows);
    return launch_merge<1>(p, s, s, st);
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
    const PromptPlan plan_all = shared_plan(own.Hkv, all_rows, own.most_shared);
    PromptPlan plan_own = prompt_plan_of(pairs, rows, own.most_own, false, false);
    plan_own.alone = false;
    const int64_t wgs_all = (int64_t)own.Hkv * plan_all.row_tiles * plan_all.splits, wgs_own = pairs * plan_own.row_tiles * plan_own.splits;
    if (!fits_launch(wgs_all + wgs_own, 256) || !fits_launch(rows, 256)) return RK_ERR_UNSUPPORTED;      // (the join: up to a workgroup to a row of a pair)
    set_plan(all, plan_all);
    set_plan(own, plan_own);
    const size_t first = paged_scratch(own.Hkv, all_rows, own.most_shared);
    if (workspace_bytes < first || !place_parts(all, plan_all, own.Hkv, all_rows, (char*)workspace, first) ||
        !place_parts(own, plan_own, pairs, rows, (char*)workspace + first, workspace_bytes - first)) return RK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const PrefixLaunch f = prefix_launch(plan_all, plan_own, wgs_own, cap, slope);
    hipLaunchKernelGGL(f.kernel, dim3((unsigned)(wgs_all + (wgs_own + f.per_wg - 1) / f.per_wg)), dim3(256), 0, st, all, own, (int32_t)wgs_all, (int32_t)wgs_own);
    if ((rc = launch_status()) != RK_OK) return rc;
    return launch_merge<2>(own, source_of(all, kRowsShared, (int)all_rows), source_of(own, kRowsPaged, (int)rows), st);
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
    if (!fits_launch(pairs * plan.splits, 256)) return RK_ERR_UNSUPPORTED;       // (a launch that splits, and so the join, is small)
    set_plan(p, plan);
    if (plan.splits > 1 && !place_parts(p, plan, pairs, p.G, (char*)workspace, workspace_bytes)) return RK_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    // (whether tokens meet in a page, for all that is known here: half a token to a page of the table or more.  The pages that there are are the device's to know:
    // where the table is far wider than those, tokens that do meet are taken for such that do not)
    const bool often = n_new > 1 && 2 * (int64_t)n_new * k >= table_width;
    auto kernel = often ? cols_form<kColWaves, kRowsChosen>(cap, slope) : cols_form<kColWaves, kRowsChosenOnce>(cap, slope);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(pairs * plan.splits)), dim3(kColWaves * 64), 0, st, p);
    if ((rc = launch_status()) != RK_OK || plan.splits == 1) return rc;
    const PartSource s = source_of(p, kRowsChosen, p.G);
    return launch_merge<1>(p, s, s, st);
}
