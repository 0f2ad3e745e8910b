// kv_attend_few.cuh -- attention over a cache of 8 or 4 bits for few query rows a sequence and head (single
// tokens, a few proposed ones), the joining of split sequences, and the choice of kernels.  kBits: 8 (mp_kv_attend,
// instances in kv_attend.cu) or 4 (mp_kv_four_attend, kv4_attend.cu).
//
// A work unit is one granule (32 tokens) of one cache head under one tile of 8 * NT
// query rows (rows = tokens x heads of a group, which share the cached head).
// k_kv_attend_few: the units of all sequences, tiles and heads lie on one line that is cut
// evenly among the warps of the grid, so ragged batches and single long contexts keep every
// SM at the memory alike; a warp walks its stretch with bulk copies into a ring of
// its own, no warp waiting for another.  A (sequence, tile, head) that one warp holds
// whole is written at once; the others leave (sum, reference, weighted values) and
// k_kv_join adds them up.  k_kv_attend_short: a CTA a (sequence, head) for short contexts.
//
// Per granule: scores S^T = K Q^T and O^T += V^T P^T on warp-level matrix products
// in f16, rows of the stored tiles as the left operand, so that 8 query rows cost one
// product column block and no query row is padding for a group of 8.  Stored bytes
// become f16 exactly.  With x_j = scale * q.k_j * log2(e) * key scale + log2(value
// scale), w_j = 2^(x_j - M) <= 1 under the running maximum M, the output is
// sum w_j byte_j / sum (w_j / value scale): the value scale costs nothing per element
// and products stay within f16's range.  Sums are f32, where weights below 2^-126 are lost: a context's
// value scales may be 2^100 apart.  w is rounded to f16: 11 bits down to 2^-28 of the largest, none below 2^-38.
//
// Measured (32 heads over 8 of 128): 64 ragged contexts of up to 8,191 tokens 97 us, 5.5
// TB/s of the 6.8 that a copy reaches; two of 262,144 tokens 173 us, 6.0 TB/s; one of 512 6.6
// us of GPU time.  Long contexts are bound by memory; the rest is the ramp (lengths, table,
// queries, first bytes: four trips one after another) and the joining launch, about 12 us.
//
// 4 bits.  A code times its scale is exact in f16, so both products take the values themselves: w_j = 2^(x_j - M), no value
// scale in the sum (they take sixteenths, which cost one shift a word less).  The reference M stays until a score passes it by
// 2^5 (kFewGrow), which one vote a granule says; w has 11 bits down to 2^-24 of it.  A granule is 4.4 KB where it is 8.2 KB of 8 bits, and takes as many products and more
// operations on codes: about 580 instructions, of which 136 pick codes out of words, 128 scale them and 32 are products.
// Measured: the 64 contexts 80 us (3.6 TB/s; 64 us without any operation on the bytes), the two long ones 119 us (4.7 TB/s;
// 99).  What grows with the granules does so at 5.7 TB/s, 84% of a copy: 64 contexts of one length take 22 us (GPU time) and 50 for
// each 4,096 tokens of all of them; ragged ones of the same bytes 7 more.  The growing part goes by the number of instructions,
// at 0.6 a clock and scheduler: the work alone, without loads, takes 118 us of the long ones' 127 (GPU time with the timing), 93
// without the 128 operations that scale codes, 122 with integer ones in their place.  Dropped: 64 tokens a step, 8 and 16
// warps, four granules ahead (89 and 128 us for 85 and 126), bulk copies for the ring (93 and 130).
#pragma once

#include <algorithm>
#include <cmath>

#include "kv_attend.cuh"

namespace mp {
namespace {

// Warps of a CTA, and granules that the ring of each holds (192 KB at most in all). Registers bound the warps, an even
// share for the four schedulers: 12 of D = 128 with 16 rows spill (64 ragged contexts 127 -> 153 us, 10 160; D = 64 with 16 rows
// over 8 bits keeps 8 bytes a thread in memory), 12 instead of 16 of D = 64 with 8 rows take 66 for 60 us. 8 with 3 granules for
// 12 with 2: 164 for 170 us over two of 262,144 tokens, but 103 for 97 over 64 ragged ones; 3 granules for 2 never paid otherwise
// (130 for 127).
constexpr int few_warps(int d, int nt) { return d == 128 ? (nt == 1 ? 12 : 8) : (nt == 1 ? 16 : 12); }
constexpr int kFewStages = 2;
constexpr int short_warps(int nt) { return nt == 1 ? 16 : 8; }
constexpr int kLeastUnits = 4;  // of 4 bits, that a warp takes where there are more
constexpr int kFewRows = 16;  // most rows of a sequence and head
// k_kv_join with a warp a row has 48 registers and keeps 16 bytes a thread in memory (D = 128, 8 bits) or 8 (D = 64), or has 64 and
// keeps none (D = 128, 4 bits); with 8 warps a row it has 63 or 64 and keeps none.
constexpr int kJoinThreads = 256;

template <int kRows>
__device__ __forceinline__ int seq_tiles(const AttendArgs& a, const SeqView& s) {
    return (int)(((int64_t)s.n * a.group + kRows - 1) / kRows);
}
template <int kRows>
__device__ __forceinline__ int64_t seq_units(const AttendArgs& a, int b) {
    const SeqView s = load_seq(a.bt, b, false);
    if (s.st != MP_OK || !seq_is_few(a, s)) return 0;
    int lo, hi;
    seq_granules(a, s, lo, hi);
    return (int64_t)(hi - lo) * a.c.n_heads * seq_tiles<kRows>(a, s);
}

// A position on the line of units.
struct Cursor {
    int b, lo, hi, g;    // sequence, its granules, the granule
    int col, in_block;   // g as a column of the table and a granule of its block
    int slots, slot;     // tiles x heads, tile * heads + head
    int tile, head;
    int64_t row;         // first row of the token arrays
    int n, len;          // the call's tokens, tokens held
    __device__ __forceinline__ void at(const AttendArgs& a, int gran) {
        const int per = a.c.block_tokens / kGranule;
        g = gran, col = gran / per, in_block = gran - col * per;
    }
    __device__ __forceinline__ void seek(const AttendArgs& a, int lo_, int hi_, int slots_, int64_t unit) {
        lo = lo_, hi = hi_, slots = slots_;
        slot = (int)quotient(unit, hi - lo);
        tile = slot / a.c.n_heads, head = slot - tile * a.c.n_heads;
        at(a, lo + (int)(unit - (int64_t)slot * (hi - lo)));
    }
};
template <int kRows>
__device__ __forceinline__ bool enter(const AttendArgs& a, Cursor& c, int64_t unit) {
    const SeqView s = load_seq(a.bt, c.b, false);
    if (s.st != MP_OK || !seq_is_few(a, s)) return false;
    int lo, hi;
    seq_granules(a, s, lo, hi);
    const int slots = a.c.n_heads * seq_tiles<kRows>(a, s);
    if (hi <= lo || slots == 0) return false;
    c.row = s.lo, c.n = s.n, c.len = s.len;
    c.seek(a, lo, hi, slots, unit);
    return true;
}
template <int kRows>
__device__ __forceinline__ void next(const AttendArgs& a, Cursor& c) {
    if (++c.g < c.hi) {
        if (++c.in_block == a.c.block_tokens / kGranule) c.in_block = 0, ++c.col;
        return;
    }
    if (++c.slot < c.slots) {
        if (++c.head == a.c.n_heads) c.head = 0, ++c.tile;
        return c.at(a, c.lo);
    }
    do ++c.b;
    while (c.b < a.bt.n_seqs && !enter<kRows>(a, c, 0));
}
__device__ __forceinline__ int page_of(const AttendArgs& a, const Cursor& c) {
    const int p = __ldg(a.bt.table + (int64_t)c.b * a.bt.max_blocks + c.col);
    return (uint32_t)p < (uint32_t)a.c.n_blocks ? p : 0;  // k_kv_join reports it; nothing outside the pool is read
}

__device__ __forceinline__ void mma(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// A warp's sums for one tile of 8 * NT query rows of a sequence and cache head.
template <typename T, int D, int NT, int kBits>
struct Tile {
    uint32_t qf[NT][D / 16][2];        // Q^T: 4 values of row 8 nt + g a lane and chunk, in the order of the keys' codes
    float unit[NT][2];                 // of score columns 2t, 2t + 1: scale * log2(e) over the row's power of two
    float top[NT][2], sum[NT][2];      // running maximum of x, this lane's part of the sum
    float o[NT][D / 16][4];
    int see_lo[NT][2], see_hi[NT][2];  // positions that the column's row sees
    int last;                          // stored bytes from this position on mean nothing
    // 4 bits: positions that every row sees; the columns' own positions (kNoEnd: all that is held is seen, or no one reads
    // the column); weights are 2^((score - mark) * unit + lift) -- the difference first, so that they stay in their range
    // however large scores are -- and a score above limit moves the mark
    int all_lo, all_hi, held, window, pos[NT][2];
    float mark[NT][2], limit[NT][2];
    static constexpr int kNoEnd = 1 << 30;

    // rows: of the sequence and head, at least 1; row: the sequence's first in the token arrays
    __device__ __forceinline__ void begin(const AttendArgs& a, int64_t row, int rows, int len, int n, int head, int tile) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
        last = all_lo = 0, all_hi = held = len, window = a.window;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = tile * 8 * NT + nt * 8 + g, there = min(r, rows - 1);
            // 8 bits: 4 consecutive values of each 16; 4 bits: D / 4 consecutive ones
            constexpr int kStep = kBits == 8 ? 16 : 4;
            const T* p = static_cast<const T*>(a.q.data) + (row + there / a.group) * a.q.token_stride +
                         (head * a.group + there % a.group) * a.q.head_stride + t * (kBits == 8 ? 4 : D / 4);
            // all loads at once: a branch in between would have each wait for the one before
            Pack<T, 4> raw[D / 16];
            if (a.wide_q) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) raw[i] = *reinterpret_cast<const Pack<T, 4>*>(p + i * kStep);
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) raw[i].x[k] = p[i * kStep + k];
            }
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) most = fmaxf(most, fabsf(to_f32(raw[i].x[k])));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
            const float f = row_factor(most);
            if constexpr (kBits == 8) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    qf[nt][i][0] = pack_f16(to_f32(raw[i].x[0]) * f, to_f32(raw[i].x[1]) * f);
                    qf[nt][i][1] = pack_f16(to_f32(raw[i].x[2]) * f, to_f32(raw[i].x[3]) * f);
                }
            } else {
                // a word of codes is pairs of values i and i + 4
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k)
                        qf[nt][i][k] = pack_f16(to_f32(raw[i & ~1].x[i % 2 * 2 + k]) * f, to_f32(raw[i | 1].x[i % 2 * 2 + k]) * f);
            }
            const float mine = row_unit(a.scale, f);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                unit[nt][k] = __shfl_sync(~0u, mine, (2 * t + k) * 4);
                const int col = tile * 8 * NT + nt * 8 + 2 * t + k;
                const int at = len - n + col / a.group;
                // columns past the last row repeat it and see all that is held: no one reads them
                see_hi[nt][k] = col < rows && a.causal ? min(len, at + 1) : len;
                see_lo[nt][k] = col < rows && a.window > 0 ? at - a.window + 1 : 0;
                pos[nt][k] = col < rows && a.causal ? at : kNoEnd;
                last = max(last, see_hi[nt][k]);
                all_lo = max(all_lo, see_lo[nt][k]), all_hi = min(all_hi, see_hi[nt][k]);
                top[nt][k] = limit[nt][k] = -INFINITY, sum[nt][k] = mark[nt][k] = 0.f;
                if (kBits == 4) unit[nt][k] = fmaxf(unit[nt][k] * kSixteenth, 0x1p-126f);  // not 0: what is not seen stays -inf
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
        }
        last = __reduce_max_sync(~0u, last);
        if (kBits == 4) all_lo = __reduce_max_sync(~0u, all_lo), all_hi = __reduce_min_sync(~0u, all_hi);
    }

    // The granule at position base: its keys kb and values vb as stored, and their scales as stored.
    __device__ __forceinline__ void add8(const uint8_t* kb, const uint8_t* vb, float ks, float stored_vs, int base) {
        float s[NT][2][4] = {};
        scores8(kb, s);
        const float vs = value_scale(stored_vs);
        uint32_t p[NT][2][2];
        weigh(s, ks, log2f(vs), __fdiv_rn(1.f, vs), base, p);
        values8(vb, stored_vs < kLeastValueScale ? 0 : last, base, p);
    }
    // ... of 4 bits, whose scales lie with the codes.
    __device__ __forceinline__ void add4(const uint8_t* kb, const uint8_t* vb, int base) {
        float s[NT][2][4] = {};
        scores4(kb, s);
        uint32_t p[NT][2][2];
        weigh4(s, base, p);
        values4(vb, base, p);
    }

    // Of the 32 tokens, product row r of 16 is token token_of(r): of 8 bits the order in which a lane's 4 stored value
    // bytes meet the second product.
    static __device__ __forceinline__ int token_of(int g, int h) { return kBits == 8 ? 4 * (g / 2) + g % 2 + 2 * h : g + 8 * h; }
    // Value of the output that row g + 8 h of product i is.
    static __device__ __forceinline__ int value_of(int i, int g, int h) { return kBits == 8 ? i * 16 + g + 8 * h : g * (D / 8) + 2 * i + h; }

    __device__ __forceinline__ void scores8(const uint8_t* kb, float (&s)[NT][2][4]) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int tok = token_of(g, 0);
            const uint8_t* row = kb + (m * 2 + tok / 8) * (D * 8) + tok % 8 * 16 + t * 4;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                uint32_t a0, a1, a2, a3;
                e4m3_to_f16(*reinterpret_cast<const uint32_t*>(row + i * 128), a0, a2);
                e4m3_to_f16(*reinterpret_cast<const uint32_t*>(row + i * 128 + 32), a1, a3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) mma(s[nt][m], a0, a1, a2, a3, qf[nt][i][0], qf[nt][i][1]);
            }
        }
    }
    // A lane has D / 4 consecutive values of its four tokens, of one group's scale; the two products of 16 tokens take turns.
    __device__ __forceinline__ void scores4(const uint8_t* kb, float (&s)[NT][2][4]) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
        const uint32_t scales = *reinterpret_cast<const uint32_t*>(kb + 16 * D + key4_scale<D>(g, t * (D / 4)));
        Pack<uint32_t, D / 32> w[4];
        Sixteenths x[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            w[r] = *reinterpret_cast<const Pack<uint32_t, D / 32>*>(kb + key4_byte<D>(r * 8 + g, t * (D / 4)));
            x[r] = sixteenths_of((scales >> (8 * r) & 0xff) * 0x00800080u);
        }
#pragma unroll
        for (int j = 0; j < D / 32; ++j)
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                uint32_t a[2][4];
                codes_to_sixteenths(w[2 * m].x[j], x[2 * m], a[0]), codes_to_sixteenths(w[2 * m + 1].x[j], x[2 * m + 1], a[1]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma(s[nt][m], a[0][0], a[1][0], a[0][1], a[1][1], qf[nt][2 * j][0], qf[nt][2 * j][1]);
                    mma(s[nt][m], a[0][2], a[1][2], a[0][3], a[1][3], qf[nt][2 * j + 1][0], qf[nt][2 * j + 1][1]);
                }
            }
    }

    // Scores become weights p of the second product; lv, iv: log2 and inverse of the values' scale.
    __device__ __forceinline__ void weigh(float (&s)[NT][2][4], float ks, float lv, float iv, int base, uint32_t (&p)[NT][2][2]) {
        const int lane = threadIdx.x % 32, g = lane / 4;
        bool moved = false;
        float fade[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float unit_k = unit[nt][k] * ks;
                float most = -INFINITY;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int j = base + m * 16 + token_of(g, h);
                        const bool seen = j < see_hi[nt][k] && j >= see_lo[nt][k];
                        float& x = s[nt][m][2 * h + k];
                        x = seen ? fmaf(x, unit_k, lv) : -INFINITY;
                        most = fmaxf(most, x);
                    }
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 4));
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 8));
                most = fmaxf(most, __shfl_xor_sync(~0u, most, 16));
                const float now = fmaxf(top[nt][k], most);
                const float ref = now == -INFINITY ? 0.f : now - kLift;
                fade[nt][k] = exp2_approx(top[nt][k] - kLift - ref);
                moved |= now != top[nt][k];
                top[nt][k] = now;
                float part = 0.f;
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float& x = s[nt][m][2 * h + k];
                        x = exp2_approx(x - ref);
                        part += x;
                    }
                sum[nt][k] = fmaf(part, iv, sum[nt][k] * fade[nt][k]);
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                p[nt][m][0] = transposed(pack_f16(s[nt][m][0], s[nt][m][1]));
                p[nt][m][1] = transposed(pack_f16(s[nt][m][2], s[nt][m][3]));
            }
        }
        if (__any_sync(~0u, moved)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[nt][i][k] *= fade[nt][k % 2];
        }
    }

    // ... of 4 bits: no scales are left, and a reference stays until a score passes it by 2^kFewGrow, which weights have
    // room for: one vote a granule in the place of a maximum over lanes.
    __device__ __forceinline__ void weigh4(float (&s)[NT][2][4], int base, uint32_t (&p)[NT][2][2]) {
        const int lane = threadIdx.x % 32, g = lane / 4;
        if (base < all_lo || base + kGranule > all_hi) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = base + i / 2 * 16 + token_of(g, i % 2), before = pos[nt][k] - j;
                        if (j >= held || before < 0 || (window > 0 && before >= window)) s[nt][i / 2][i % 2 * 2 + k] = -INFINITY;
                    }
        }
        float most[NT][2];
        bool over = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                most[nt][k] = fmaxf(fmaxf(s[nt][0][k], s[nt][0][2 + k]), fmaxf(s[nt][1][k], s[nt][1][2 + k]));
                over |= most[nt][k] > limit[nt][k];
            }
        if (__any_sync(~0u, over)) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float x = most[nt][k];
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 4));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 8));
                    x = fmaxf(x, __shfl_xor_sync(~0u, x, 16));
                    if (x > limit[nt][k]) {
                        const float fade = limit[nt][k] == -INFINITY ? 0.f : exp2_approx((mark[nt][k] - x) * unit[nt][k]);
                        // kFewGrow / unit and the sum rounded down: where scores are large a step of 32 bits is several powers
                        // of two of weight (with a division that rounds down 64 ragged contexts took 88 us for 86, 4 tokens
                        // over them 126 for 122)
                        mark[nt][k] = x, limit[nt][k] = __fadd_rd(x, rcp_approx(unit[nt][k]) * (kFewGrow * (1.f - 0x1p-20f)));
                        sum[nt][k] *= fade;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) o[nt][i][k] *= fade, o[nt][i][2 + k] *= fade;
                    }
                }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                float part[2] = {};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float& x = s[nt][i / 2][i % 2 * 2 + k];
                    x = exp2_approx(fmaf(x - mark[nt][k], unit[nt][k], lift_of(4)));
                    part[i % 2] += x;
                }
                sum[nt][k] += part[0] + part[1];
            }
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                p[nt][m][0] = transposed(pack_f16(s[nt][m][0], s[nt][m][1]));
                p[nt][m][1] = transposed(pack_f16(s[nt][m][2], s[nt][m][3]));
            }
        }
    }

    // Values from position `meant` on are zeros.
    __device__ __forceinline__ void values8(const uint8_t* vb, int meant, int base, const uint32_t (&p)[NT][2][2]) {
        const int lane = threadIdx.x % 32, t = lane % 4;
        if (base + kGranule <= meant) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint8_t* at = vb + i * 512 + h * 128 + lane * 4;
                    uint32_t a0, a1, a2, a3;
                    e4m3_to_f16(*reinterpret_cast<const uint32_t*>(at), a0, a2);
                    e4m3_to_f16(*reinterpret_cast<const uint32_t*>(at + 256), a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(o[nt][i], a0, a1, a2, a3, p[nt][h][0], p[nt][h][1]);
                }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int left = meant - (base + h * 16 + t * 4);  // of this lane's 4 tokens
                const uint32_t keep = left >= 4 ? ~0u : left <= 0 ? 0u : (1u << (8 * left)) - 1;
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                    const uint8_t* at = vb + i * 512 + h * 128 + lane * 4;
                    uint32_t a0, a1, a2, a3;
                    e4m3_to_f16(*reinterpret_cast<const uint32_t*>(at) & keep, a0, a2);
                    e4m3_to_f16(*reinterpret_cast<const uint32_t*>(at + 256) & keep, a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma(o[nt][i], a0, a1, a2, a3, p[nt][h][0], p[nt][h][1]);
                }
            }
        }
    }
    // A lane has D / 8 consecutive values of two neighbouring tokens of each 8: a pair of codes in a word is one value of
    // both.  Tokens from position `last` on count as zeros, whatever their codes and scales are.
    __device__ __forceinline__ void values4(const uint8_t* vb, int base, const uint32_t (&p)[NT][2][2]) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
        const uint2 scales = *reinterpret_cast<const uint2*>(vb + 16 * D + value4_scale<D>(2 * t, g * (D / 8)));
        const bool edge = base + kGranule > last;
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            Pack<uint32_t, D / 32> w[2];
            Sixteenths x[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                w[r] = *reinterpret_cast<const Pack<uint32_t, D / 32>*>(vb + (2 * m + r) * 4 * D + lane * (D / 8));
                uint32_t s2 = __byte_perm(m ? scales.y : scales.x, 0, r ? 0x4342 : 0x4140) << 7;
                if (edge) {
                    const int left = last - (base + m * 16 + r * 8 + 2 * t);
                    s2 &= left >= 2 ? ~0u : left == 1 ? 0xffffu : 0u;
                }
                x[r] = sixteenths_of(s2);
            }
#pragma unroll
            for (int j = 0; j < D / 32; ++j) {
                uint32_t a[2][4];
                codes_to_sixteenths(w[0].x[j], x[0], a[0]), codes_to_sixteenths(w[1].x[j], x[1], a[1]);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    mma(o[nt][2 * j], a[0][0], a[0][1], a[1][0], a[1][1], p[nt][m][0], p[nt][m][1]);
                    mma(o[nt][2 * j + 1], a[0][2], a[0][3], a[1][2], a[1][3], p[nt][m][0], p[nt][m][1]);
                }
            }
        }
    }

    // The reference of a column's weights, which are 2^lift_of(kBits) there.
    __device__ __forceinline__ float reference(int nt, int k) const {
        return kBits == 8 ? top[nt][k] : limit[nt][k] == -INFINITY ? -INFINITY : mark[nt][k] * unit[nt][k];
    }

    // This lane's part of a column's sum becomes the column's.
    __device__ __forceinline__ float total(int nt, int k) const {
        float l = sum[nt][k];
        l += __shfl_xor_sync(~0u, l, 4);
        l += __shfl_xor_sync(~0u, l, 8);
        l += __shfl_xor_sync(~0u, l, 16);
        return l;
    }
};

// Copies a granule's keys and values (of kBytes each) into shared memory, 16 bytes a lane and step.
template <int kBytes>
struct GranuleCopy {
    static constexpr int kSteps = kBytes / 512, kRest = kBytes % 512;  // the rest of both in one step
    static_assert(kRest <= 256, "a lane has one of the rest");
    const uint8_t *k, *v, *rest;  // this lane's of the pools' first granule
    int rest_to;
    __device__ __forceinline__ explicit GranuleCopy(const mp_kv_cache& c) {
        const int lane = threadIdx.x % 32;
        const bool values = lane >= kRest / 16;
        const int o = kSteps * 512 + (lane - (values ? kRest / 16 : 0)) * 16;
        k = c.k + lane * 16, v = c.v + lane * 16, rest = (values ? c.v : c.k) + o, rest_to = (values ? kBytes : 0) + o;
    }
    // to: shared address of the stage; at: the granule's place in either pool
    __device__ __forceinline__ void operator()(uint32_t to, int64_t at) const {
        const int lane = threadIdx.x % 32;
        const uint32_t mine = to + lane * 16;
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + i * 512), "l"(k + at + i * 512) : "memory");
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + kBytes + i * 512), "l"(v + at + i * 512) : "memory");
        }
        if (lane < kRest / 8) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to + rest_to), "l"(rest + at) : "memory");
    }
};

template <typename T, int D, int NT, int kBits>
__global__ void __launch_bounds__(few_warps(D, NT) * 32, 1) k_kv_attend_few(AttendArgs a, FewWork work) {
    constexpr int kFewWarps = few_warps(D, NT);
    constexpr int kRows = 8 * NT;
    constexpr int kBytes = granule_bytes(kBits, D);  // of either array
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ int64_t strip_base[kFewWarps * 32 + 1];
    __shared__ int64_t warp_sum[kFewWarps];
    __shared__ __align__(8) uint64_t bars[kFewWarps * kFewStages];
    __shared__ int pages[kFewWarps * kFewStages];
    const int tid = threadIdx.x, lane = tid % 32, wid = tid / 32;
    const int g = lane / 4, t = lane % 4;

    after_previous();
    let_next_begin();
    // every CTA lays the line out for itself: thread i sums a strip of sequences
    const int strip = (a.bt.n_seqs + kFewWarps * 32 - 1) / (kFewWarps * 32);
    {
        int64_t mine = 0;
        for (int i = 0; i < strip; ++i) {
            const int b = tid * strip + i;
            if (b < a.bt.n_seqs) mine += seq_units<kRows>(a, b);
        }
        int64_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += x;
        }
        if (lane == 31) warp_sum[wid] = sum;
        if (tid < kFewWarps * kFewStages) mbar_init(&bars[tid], 1);
        fence_mbar_init();
        __syncthreads();
        for (int w = 0; w < wid; ++w) sum += warp_sum[w];
        strip_base[tid] = sum - mine;
        if (tid == kFewWarps * 32 - 1) strip_base[kFewWarps * 32] = sum;
        __syncthreads();
        if (blockIdx.x == gridDim.x - 1) {  // the one with the shortest part
            int64_t at = sum - mine;
            for (int i = 0; i < strip; ++i) {
                const int b = tid * strip + i;
                if (b < a.bt.n_seqs) {
                    work.base[b] = at;
                    at += strip == 1 ? mine : seq_units<kRows>(a, b);
                    if (b == a.bt.n_seqs - 1) work.base[b + 1] = at;
                }
            }
        }
    }
    const int warps = gridDim.x * kFewWarps;
    const int64_t total = strip_base[kFewWarps * 32];
    // of 4 bits at least so many that what is left to add up is worth it (one context of 8,000 tokens 22 us with 1, 18 with 4, 20
    // with 6; four of 4,000 22, 20 and 20)
    const int64_t per_warp = max(quotient(total + warps - 1, warps), kBits == 8 ? (int64_t)0 : min(total, (int64_t)kLeastUnits));
    // consecutive warps of the line are on different SMs: short lines reach them all
    const int w = wid * gridDim.x + blockIdx.x;
    if (w == 0 && lane == 0) work.base[a.bt.n_seqs + 1] = per_warp;
    const int64_t u0 = min(total, w * per_warp), u1 = min(total, u0 + per_warp);
    if (lane == 0) work.gave_up[w] = 0;
    if (u0 >= u1) return;

    Cursor cur;
    {
        // the strip that holds u0 (the last whose base is not past it), then the sequence
        int lo = 0, hi = kFewWarps * 32;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (strip_base[mid] <= u0) lo = mid;
            else hi = mid;
        }
        int64_t at = strip_base[lo];
        cur.b = lo * strip;
        while (strip > 1) {
            const int64_t n = seq_units<kRows>(a, cur.b);
            if (u0 < at + n) break;
            at += n, ++cur.b;
        }
        enter<kRows>(a, cur, u0 - at);
    }
    uint8_t* ring = dyn + wid * kFewStages * 2 * kBytes;
    uint64_t* bar = bars + wid * kFewStages;
    int* ring_page = pages + wid * kFewStages;

    Cursor ahead = cur;
    int64_t issued = u0;
    int page_ahead = page_of(a, ahead);
    const GranuleCopy<kBytes> copy(a.c);  // of 4 bits
    const uint32_t first_stage = smem_addr(ring), last_stage = first_stage + (kFewStages - 1) * 2 * kBytes;
    uint32_t next_stage = first_stage;
    int to_come = (int)(u1 - u0);
    auto issue = [&]() {  // the next unit's bytes into its stage
        if constexpr (kBits == 4) {  // (these copies end by themselves: there is no wait to give up)
            if (to_come > 0) {
                copy(next_stage, block_byte<kBits>(a.c, page_ahead, ahead.head) + ahead.in_block * kBytes);
                next_stage = next_stage == last_stage ? first_stage : next_stage + 2 * kBytes;
                if (--to_come > 0) {
                    next<kRows>(a, ahead);
                    page_ahead = page_of(a, ahead);
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return;
        }
        if (issued >= u1) return;
        const int st = (int)((issued - u0) % kFewStages);
        const int64_t at = block_byte<kBits>(a.c, page_ahead, ahead.head) + ahead.in_block * kBytes;
        if (lane == 0) {
            ring_page[st] = page_ahead;
            mbar_expect(&bar[st], 2 * kBytes);
            if (!test_held(a, issued)) {
                bulk_load(ring + st * 2 * kBytes, a.c.k + at, kBytes, &bar[st]);
                bulk_load(ring + st * 2 * kBytes + kBytes, a.c.v + at, kBytes, &bar[st]);
            }
        }
        if (++issued < u1) {
            next<kRows>(a, ahead);
            page_ahead = page_of(a, ahead);
        }
    };
#pragma unroll
    for (int i = 0; i < kFewStages; ++i) issue();
    __syncwarp();

    Tile<T, D, NT, kBits> x;
    bool up = false;
    int done = 0;  // units

    for (int left = (int)(u1 - u0); left > 0 && !up;) {
        // one (sequence, tile, head) or what this warp has of it
        const int head = cur.head, tile = cur.tile;
        const int rows = cur.n * a.group, units = min(cur.hi - cur.g, left);
        const bool whole = units == cur.hi - cur.lo;
        const bool first = done == 0;
        left -= units;
        x.begin(a, cur.row, rows, cur.len, cur.n, head, tile);
        if constexpr (kBits == 4) {
#pragma unroll 1
            for (int i = 0; i < units; ++i, ++done, ++cur.g) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 1) : "memory");
                __syncwarp();
                const uint8_t* kv = ring + done % kFewStages * (2 * kBytes);
                x.add4(kv, kv + kBytes, cur.g * kGranule);
                __syncwarp();
                issue();
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < units; ++i, ++done, ++cur.g) {
                const int st = done % kFewStages;
                if (!__all_sync(~0u, mbar_wait(&bar[st], (uint32_t)(done / kFewStages & 1)))) {
                    up = true;
                    break;
                }
                const int64_t sc = (int64_t)ring_page[st] * a.c.n_heads + head;
                const float ks = __ldg(a.c.k_scale + sc), vs = __ldg(a.c.v_scale + sc);
                x.add8(ring + st * 2 * kBytes, ring + st * 2 * kBytes + kBytes, ks, vs, cur.g * kGranule);
                __syncwarp();
                issue();
            }
        }
        if (up) break;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float l = x.total(nt, k);
                const int in_tile = nt * 8 + 2 * t + k, r = tile * kRows + in_tile;
                const float m = x.reference(nt, k);
                if (whole) {
                    if (r < rows) {
                        const int64_t tok = cur.row + r / a.group;
                        const int qh = head * a.group + r % a.group;
                        T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
                        const float inv = l == 0.f ? 0.f : __fdiv_rn(kBits == 8 ? 1.f : kSixteenth, l);
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            dst[x.value_of(i, g, 0)] = from_f32<T>(x.o[nt][i][k] * inv);
                            dst[x.value_of(i, g, 1)] = from_f32<T>(x.o[nt][i][2 + k] * inv);
                        }
                        if (a.lse != nullptr && g == 0)
                            a.lse[tok * a.q.n_heads + qh] = log_sum(m, lift_of(kBits), l);
                    }
                } else {
                    // a warp leaves at most two parts: of what began before it or with it, and of
                    // what it begins and does not end
                    float* part = work.part + ((int64_t)2 * w + (first ? 0 : 1)) * (kRows * (D + 2));
                    float* dst = part + in_tile * D;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        dst[x.value_of(i, g, 0)] = x.o[nt][i][k];
                        dst[x.value_of(i, g, 1)] = x.o[nt][i][2 + k];
                    }
                    if (g == 0) {
                        part[kRows * D + 2 * in_tile] = m;
                        part[kRows * D + 2 * in_tile + 1] = l;
                    }
                }
            }
        --cur.g;
        if (left > 0) next<kRows>(a, cur);  // (a new slot or sequence: it sets col and in_block, which no one read here)
    }
    if (up) {
        if (lane == 0) work.gave_up[w] = 1;
        // leave no copy in flight behind
        for (int64_t u = max(u0 + done, issued - kFewStages); u < issued; ++u)
            mbar_wait(&bar[(u - u0) % kFewStages], (uint32_t)((u - u0) / kFewStages & 1));
    }
}

// Short contexts in small batches: one CTA a (sequence, tile, head), whose warps take its granules in turn and
// add their sums up in shared memory, so that there is no second launch and no workspace.
constexpr int short_bytes(int bits, int d, int nt) {  // a warp's granules, and its sums in their place
    return std::max(2 * granule_bytes(bits, d), 8 * nt * d * (int)sizeof(float));
}
template <typename T, int D, int NT, int kBits>
__global__ void __launch_bounds__(short_warps(NT) * 32, 1) k_kv_attend_short(AttendArgs a) {
    constexpr int kRows = 8 * NT, kBytes = granule_bytes(kBits, D), kWarps = short_warps(NT), kMine = short_bytes(kBits, D, NT);
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ float ref[kWarps][kRows], weight[kWarps][kRows];
    const int lane = threadIdx.x % 32, wid = threadIdx.x / 32, g = lane / 4, t = lane % 4;
    after_previous();
    let_next_begin();
    const int b = blockIdx.x / a.c.n_heads, head = blockIdx.x % a.c.n_heads;
    const SeqView s = load_seq(a.bt, b, false);
    int lo, hi;
    seq_granules(a, s, lo, hi);
    const int rows = s.n * a.group, per = a.c.block_tokens / kGranule;
    const int32_t* table = a.bt.table + (int64_t)b * a.bt.max_blocks;
    if (head == 0) {  // this CTA has the sequence's status
        bool ok = s.st == MP_OK;
        if (ok && hi > lo)
            for (int col = lo / per + threadIdx.x; col <= (hi - 1) / per; col += kWarps * 32) {
                const int p = __ldg(table + col);
                ok &= p >= 0 && p < a.c.n_blocks;
            }
        ok = !__syncthreads_or(!ok);
        if (threadIdx.x == 0) a.status[b] = ok ? MP_OK : MP_EINVAL;
    }
    if (s.st != MP_OK) return;
    uint8_t* const mine = dyn + wid * kMine;
    Tile<T, D, NT, kBits> x;
    for (int tile = 0; tile * kRows < rows; ++tile) {
        for (int gran = lo + wid; gran < hi; gran += kWarps) {
            int page = __ldg(table + gran / per);
            if (page < 0 || page >= a.c.n_blocks) page = 0;  // reported above
            const int64_t at = block_byte<kBits>(a.c, page, head) + (int64_t)(gran % per) * kBytes;
#pragma unroll
            for (int i = 0; i < (kBytes + 511) / 512; ++i) {
                const int o = (i * 32 + lane) * 16;
                if (kBytes % 512 && o >= kBytes) break;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(mine + o)), "l"(a.c.k + at + o) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(mine + kBytes + o)), "l"(a.c.v + at + o)
                             : "memory");
            }
            float ks = 1.f, vs = 1.f;
            if constexpr (kBits == 8) {
                const int64_t sc = (int64_t)page * a.c.n_heads + head;
                ks = __ldg(a.c.k_scale + sc), vs = __ldg(a.c.v_scale + sc);
            }
            if (gran == lo + wid) x.begin(a, s.lo, rows, s.len, s.n, head, tile);
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            if constexpr (kBits == 8) {
                x.add8(mine, mine + kBytes, ks, vs, gran * kGranule);
            } else {
                x.add4(mine, mine + kBytes, gran * kGranule);
            }
            __syncwarp();
        }
        const bool any = lo + wid < hi;
        float* const acc = reinterpret_cast<float*>(mine);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = nt * 8 + 2 * t + k;
                const float l = any ? x.total(nt, k) : 0.f;
                if (any) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        acc[r * D + x.value_of(i, g, 0)] = x.o[nt][i][k];
                        acc[r * D + x.value_of(i, g, 1)] = x.o[nt][i][2 + k];
                    }
                }
                if (g == 0) ref[wid][r] = any ? x.reference(nt, k) : -INFINITY, weight[wid][r] = l;
            }
        __syncthreads();
        for (int i = threadIdx.x; i < kRows * (D / 2); i += kWarps * 32) {
            const int in_tile = i / (D / 2), d = i % (D / 2) * 2, r = tile * kRows + in_tile;
            if (r >= rows) break;
            float top = -INFINITY, sum = 0.f, o0 = 0.f, o1 = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) top = fmaxf(top, ref[w][in_tile]);
            const float from = top == -INFINITY ? 0.f : top;
#pragma unroll 4
            for (int w = 0; w < kWarps; ++w) {
                if (lo + w >= hi) break;
                const float f = exp2_approx(ref[w][in_tile] - from);
                const float2 y = *reinterpret_cast<const float2*>(dyn + w * kMine + (in_tile * D + d) * sizeof(float));
                sum += weight[w][in_tile] * f, o0 += y.x * f, o1 += y.y * f;
            }
            const float inv = sum == 0.f ? 0.f : __fdiv_rn(kBits == 8 ? 1.f : kSixteenth, sum);
            const int64_t tok = s.lo + r / a.group;
            const int qh = head * a.group + r % a.group;
            T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride + d;
            const float y[2] = {o0 * inv, o1 * inv};
            store_values<T, 2>(dst, a.wide_out, y);
            if (d == 0 && a.lse != nullptr)
                a.lse[tok * a.q.n_heads + qh] = log_sum(top, lift_of(kBits), sum);
        }
        __syncthreads();
    }
}

// Rows of a sequence and head that k_kv_attend_few may have.
__host__ __device__ __forceinline__ int join_rows(const AttendArgs& a) {
    const int64_t rows = (int64_t)a.bt.max_tokens * a.group;
    return (int)(rows < 1 ? 1 : rows > a.few_rows ? a.few_rows : rows);
}

constexpr int kJoinCols = 16;  // of D, a CTA's share of a pair of tiles
struct JoinPlan {
    int cuts, checks, row_ctas;  // CTAs: of k_kv_attend_many's cuts, of the sequences' status, of k_kv_attend_few's rows
};

// Adds up the 16 columns y of the (sequence, pair, head) in which CTA w of k_kv_attend_many began, if w is the first to
// begin inside it: a thread a row.
template <typename T, int D>
__device__ void join_cut(const AttendArgs& a, const ManyWork& work, int w, int y) {
    const ManyStart st = work.starts[w];
    if (!st.there || st.into <= kExtra) return;  // (it began with the pair's first unit)
    const int64_t us = w * st.per - st.into;     // the pair and head on the line
    const int begun = (int)quotient(us + kExtra, st.per), last = (int)quotient(us + kExtra + st.cnt - 1, st.per);
    if (w != begun + 1) return;  // another CTA cut it before
    const SeqView s = load_seq(a.bt, st.b, false);
    const int in_pair = threadIdx.x, r = st.tile * kPair + in_pair;
    if (r >= s.n * a.group) return;
    float top = -INFINITY, sum = 0.f, o[kJoinCols] = {};
#pragma unroll 1
    for (int v = begun; v <= last; ++v) {
        const float* part = work.part + ((int64_t)2 * v + (v * st.per >= us ? 0 : 1)) * (kPair * (D + 2)) + in_pair;
        float x[kJoinCols];
        const float m = part[D * kPair], l = part[(D + 1) * kPair];
#pragma unroll
        for (int j = 0; j < kJoinCols; ++j) x[j] = part[(y * kJoinCols + j) * kPair];
        const float now = fmaxf(top, m), ref = now == -INFINITY ? 0.f : now;
        const float f = exp2_approx(top - ref), g = exp2_approx(m - ref);
        sum = sum * f + l * g;
#pragma unroll
        for (int j = 0; j < kJoinCols; ++j) o[j] = o[j] * f + x[j] * g;
        top = now;
    }
    const int64_t tok = s.lo + r / a.group;
    const int qh = st.head * a.group + r % a.group;
    const float inv = sum == 0.f ? 0.f : __fdiv_rn(1.f, sum);
    T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride + y * kJoinCols;
#pragma unroll
    for (int j = 0; j < kJoinCols; ++j) o[j] *= inv;
    store_values<T, 8>(dst, a.wide_out, o);
    store_values<T, 8>(dst + 8, a.wide_out, o + 8);
    if (y == 0 && a.lse != nullptr)
        a.lse[tok * a.q.n_heads + qh] = log_sum(top, kManyLift, sum);
}

// A sequence's status, and its rows that see nothing (no kernel has units of theirs).
template <typename T, int D>
__device__ void check_seq(const AttendArgs& a, const FewWork& few, bool late, int b) {
    const SeqView s = load_seq(a.bt, b, false);
    int lo, hi;
    seq_granules(a, s, lo, hi);
    bool ok = s.st == MP_OK;
    if (ok && hi > lo) {
        const int per = a.c.block_tokens / kGranule;
        for (int col = lo / per + threadIdx.x; col <= (hi - 1) / per; col += kJoinThreads) {
            const int p = __ldg(a.bt.table + (int64_t)b * a.bt.max_blocks + col);
            ok &= p >= 0 && p < a.c.n_blocks;
        }
    }
    if (ok && few.base != nullptr && seq_is_few(a, s)) {
        const int64_t from = few.base[b], past = few.base[b + 1], per = few.base[a.bt.n_seqs + 1];
        if (past > from)
            for (int64_t w = quotient(from, per) + threadIdx.x; w <= quotient(past - 1, per); w += kJoinThreads)
                late |= few.gave_up[w] != 0;
    }
    ok = !__syncthreads_or(!ok);
    late = __syncthreads_or(late);
    if (threadIdx.x == 0) a.status[b] = !ok ? MP_EINVAL : late ? MP_ETIMEOUT : MP_OK;
    // queries before the first position, or of an empty sequence
    const int blind = s.st != MP_OK ? 0 : s.len == 0 ? s.n : a.causal ? min(s.n, max(s.n - s.len, 0)) : 0;
    for (int64_t i = threadIdx.x; i < (int64_t)blind * a.q.n_heads * (D / 2); i += kJoinThreads) {
        const int64_t tok = s.lo + i / (D / 2) / a.q.n_heads;
        const int qh = (int)(i / (D / 2) % a.q.n_heads), d = (int)(i % (D / 2)) * 2;
        T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride + d;
        dst[0] = dst[1] = from_f32<T>(0.f);
        if (d == 0 && a.lse != nullptr) a.lse[tok * a.q.n_heads + qh] = -INFINITY;
    }
}

// kPer warps a query row add up what several warps of k_kv_attend_few had of it.
template <typename T, int D, int NT, int kPer, int kBits>
__device__ void join_row(const AttendArgs& a, const FewWork& work, int64_t u, bool there) {
    constexpr int kRows = 8 * NT, kCols = D / 32, kAhead = kPer == 1 ? 4 : 8;
    __shared__ float acc[kJoinThreads / 32][D + 2];
    const int lane = threadIdx.x % 32, wid = threadIdx.x / 32;
    const int head = (int)(u % a.c.n_heads), rows_max = join_rows(a);
    const int r = (int)(u / a.c.n_heads % rows_max), b = (int)(u / a.c.n_heads / rows_max);
    SeqView s = {};
    int lo = 0, hi = 0;
    int64_t from = 0, per = 1;
    if (there) {
        s = load_seq(a.bt, b, false);
        from = work.base[b], per = work.base[a.bt.n_seqs + 1];
        seq_granules(a, s, lo, hi);
        there = s.st == MP_OK && seq_is_few(a, s) && r < s.n * a.group && hi > lo;
    }
    const int tile = r / kRows, in_tile = r % kRows, cnt = hi - lo;
    const int64_t us = from + ((int64_t)tile * a.c.n_heads + head) * cnt;
    const int64_t w0 = there ? quotient(us, per) : 0, w1 = there ? quotient(us + cnt - 1, per) : 0;
    there = there && w0 != w1;  // else one warp had it all
    float top = -INFINITY, l = 0.f, o[kCols] = {};
    if (there) {
        auto part_of = [&](int64_t w) { return work.part + (2 * w + (w * per >= us ? 0 : 1)) * (kRows * (D + 2)); };
        // the largest reference first, so that the sums do not depend on one another
        for (int64_t w = w0 + lane; w <= w1; w += 32) top = fmaxf(top, part_of(w)[kRows * D + 2 * in_tile]);
#pragma unroll
        for (int k = 16; k > 0; k >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, k));
        const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll kAhead
        for (int64_t w = w0 + wid % kPer; w <= w1; w += kPer) {
            const float* part = part_of(w);
            const float f = exp2_approx(part[kRows * D + 2 * in_tile] - ref);
            l += part[kRows * D + 2 * in_tile + 1] * f;
            const Pack<float, kCols> x = *reinterpret_cast<const Pack<float, kCols>*>(part + in_tile * D + lane * kCols);
#pragma unroll
            for (int i = 0; i < kCols; ++i) o[i] += x.x[i] * f;
        }
    }
    if (kPer > 1) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[wid][lane * kCols + i] = o[i];
        if (lane == 0) acc[wid][D] = l;
        __syncthreads();
        if (wid > 0 || !there) return;
        l = 0.f;
#pragma unroll
        for (int i = 0; i < kCols; ++i) o[i] = 0.f;
#pragma unroll
        for (int v = 0; v < kPer; ++v) {
            l += acc[v][D];
#pragma unroll
            for (int i = 0; i < kCols; ++i) o[i] += acc[v][lane * kCols + i];
        }
    }
    if (!there) return;
    const int64_t tok = s.lo + r / a.group;
    const int qh = head * a.group + r % a.group;
    T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
    const float inv = l == 0.f ? 0.f : __fdiv_rn(kBits == 8 ? 1.f : kSixteenth, l);
#pragma unroll
    for (int i = 0; i < kCols; ++i) o[i] *= inv;
    store_values<T, kCols>(dst + lane * kCols, a.wide_out, o);
    if (a.lse != nullptr && lane == 0)
        a.lse[tok * a.q.n_heads + qh] = log_sum(top, lift_of(kBits), l);
}

// After both kernels: what more than one CTA or warp had of a row, and the sequences' status.  kPer: warps a row.
template <typename T, int D, int NT, int kPer, int kBits>
__global__ void __launch_bounds__(kJoinThreads) k_kv_join(AttendArgs a, FewWork few, ManyWork many, JoinPlan plan) {
    after_previous();
    let_next_begin();
    int cta = blockIdx.x;
    if (cta < plan.cuts) return join_cut<T, D>(a, many, cta / (D / kJoinCols), cta % (D / kJoinCols));
    cta -= plan.cuts;
    if (cta < plan.checks) {
        bool late = false;
        if (many.part != nullptr)
            for (int i = threadIdx.x; i < kManyCtas; i += kJoinThreads) late |= many.gave_up[i] != 0;
        for (int b = cta; b < a.bt.n_seqs; b += plan.checks) check_seq<T, D>(a, few, late, b);
        return;
    }
    cta -= plan.checks;
    constexpr int kRowsCta = kJoinThreads / 32 / kPer;
    const int64_t rows = (int64_t)a.bt.n_seqs * join_rows(a) * a.c.n_heads;
    for (int64_t u = (int64_t)cta * kRowsCta; u < rows; u += (int64_t)plan.row_ctas * kRowsCta) {
        const int64_t mine = u + threadIdx.x / 32 / kPer;
        join_row<T, D, NT, kPer, kBits>(a, few, mine < rows ? mine : 0, mine < rows);
    }
}

// Sequences of few rows in a batch that also has many: k_kv_attend_many takes them at about 2.5 TB/s of cache bytes, which
// up to this size costs less than the other kernel with its joining where most sequences have many rows (8 heads of 128,
// GPU time without and with it: 16 x 1,000 tokens 31 and 45 us, 8 x 4,000 96 and 145, 3 x 4,000-16,384 157 and 161; 16 of up
// to 8,000, 8 with pieces of 512 and 8 with single tokens, 315 and 331).  Where one piece of 512 comes with single
// tokens, both kernels are the faster way from well below: 16 singles of up to 2,000 (41 MB held) 57 and 57, 32 of up to
// 4,000 (145 MB) 116 and 94, 63 of up to 2,000 (162 MB) 130 and 87; past the line 63 of up to 4,000 (294 MB) 189 and 122, 255 of
// up to 8,000 (2.2 GB) 1,019 and 490.  The line goes by what the host knows, the number of sequences times the bound of
// their lengths; a generous bound leads to both kernels.  Of 4 bits the first kernel reads half of the bytes, and the second
// takes as long: 16 singles of up to 2,000 with a piece of 512 (37 MB) 64 us without the first and 70 with it, 32 of up to 4,000 (143
// MB) 115 and 91, 8 pieces of 512 and 8 singles over up to 8,000 (139 MB) 471 and 470.
constexpr int64_t small_cache(int bits) { return bits == 8 ? 256 << 20 : 64 << 20; }
// Which kernels a batch needs, by its host scalars: sequences of at most kFewRows rows are
// bound by the cache's bytes, which k_kv_attend_few streams; above it the products count.
// A batch whose sequences all have max_tokens has no sequence for the first.
// Few rows of short contexts in batches that fill the GPU at most twice over go to k_kv_attend_short (8 heads, the GPU's
// time of a call: 1 x 512 tokens 6.6 us against 9.4, 8 x 1,024 8.8 against 11.7, 38 x 2,048 32.6 against 37.2; but
// 1 x 4,096 19.3 against 14.7, and 128 x 512, four times the SMs, 48.6 against 35.4).  Of 4 bits the same lines hold: 1 x 512 7
// against 11, 8 x 1,024 9 against 15, 38 x 2,048 27 against 38, but 2 x 4,000 21 against 17.
constexpr int32_t kShortLen = 2048;
constexpr int64_t kShortCtas = 2 * kSms;
struct Route {
    bool few, many, brief;
};
template <int kBits>
Route route(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t group, int32_t window) {
    // An empty pool has no block that could stand in for a bad table entry's: k_kv_join alone says which sequences are
    // wrong (all that see a position) and writes the rows that see nothing.
    if (c.n_blocks == 0) return {false, false, false};
    if ((int64_t)bt.max_tokens * group <= kFewRows) {
        const int32_t span = window > 0 ? std::min(bt.max_len, window + bt.max_tokens) : bt.max_len;
        const bool brief = span <= kShortLen && (int64_t)bt.n_seqs * c.n_heads <= kShortCtas;
        return {!brief, false, brief};
    }
    const int64_t bytes = (int64_t)bt.n_seqs * bt.max_len * c.n_heads * granule_bytes(kBits, c.head_dim) / (kGranule / 2);
    return {bt.n_tokens != (int64_t)bt.n_seqs * bt.max_tokens && bytes > small_cache(kBits), true, false};
}

struct Layout {
    size_t base, gave_up, part, starts, many_gave_up, many_part, bytes;
};
// (The scratch is asked for before the window is known: a window can only leave it unused.)
template <int kBits>
Layout layout(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t group) {
    Layout l = {};
    const Route r = route<kBits>(c, bt, group, 0);
    const size_t warps8 = few_warps(c.head_dim, 1), warps16 = few_warps(c.head_dim, 2);
    auto take = [&](size_t bytes) {
        const size_t at = l.bytes;
        l.bytes += align_up(bytes);
        return at;
    };
    if (r.few) {
        l.base = take(sizeof(int64_t) * ((size_t)bt.n_seqs + 2));
        l.gave_up = take(sizeof(int32_t) * kFewCtas * std::max(warps8, warps16));
        l.part = take(sizeof(float) * 2 * kFewCtas * std::max(8 * warps8, 16 * warps16) * (size_t)(c.head_dim + 2));
    }
    if (r.many) {
        l.starts = take(sizeof(ManyStart) * kManyCtas);
        l.many_gave_up = take(sizeof(int32_t) * kManyCtas);
        l.many_part = take(kv_many_part_bytes(c));
    }
    return l;
}

template <typename T, int D, int NT, int kBits>
cudaError_t short_as(const AttendArgs& a, cudaStream_t stream) {
    constexpr size_t smem = (size_t)short_warps(NT) * short_bytes(kBits, D, NT);
    cudaError_t e = set_smem_limit((const void*)k_kv_attend_short<T, D, NT, kBits>, smem);
    if (e != cudaSuccess) return e;
    return launch_close(k_kv_attend_short<T, D, NT, kBits>, a.bt.n_seqs * a.c.n_heads, short_warps(NT) * 32, smem, stream, a);
}

template <typename T, int D, int NT, int kBits>
cudaError_t attend_as(const AttendArgs& a, const FewWork& few, const ManyWork& many, cudaStream_t stream) {
    cudaError_t e;
    JoinPlan plan = {};
    plan.checks = std::min(a.bt.n_seqs, 1024);
    int64_t rows = 0;
    if (few.base != nullptr) {
        constexpr size_t smem = (size_t)few_warps(D, NT) * kFewStages * 2 * granule_bytes(kBits, D);
        e = set_smem_limit((const void*)k_kv_attend_few<T, D, NT, kBits>, smem);
        if (e == cudaSuccess)
            e = launch_close(k_kv_attend_few<T, D, NT, kBits>, kFewCtas, few_warps(D, NT) * 32, smem, stream, a, few);
        if (e != cudaSuccess) return e;
        rows = (int64_t)a.bt.n_seqs * join_rows(a) * a.c.n_heads;
    }
    if (many.part != nullptr) {
        e = kBits == 8 ? launch_kv_many(a, many, stream) : launch_kv4_many(a, many, stream);
        if (e != cudaSuccess) return e;
        plan.cuts = kManyCtas * (D / kJoinCols);
    }
    // rows that are cut into many parts have a CTA each, whose warps share the parts (64 rows of 76 parts: 18 -> 5 us), the
    // others a warp (2,048 rows of two or three: 12 -> 7 us)
    constexpr int kWarps = kJoinThreads / 32;
    const int64_t parts = kFewCtas * few_warps(D, NT) / ((int64_t)a.bt.n_seqs * a.c.n_heads);
    if (rows <= 8 * kFewCtas || parts > 12) {
        plan.row_ctas = (int)std::min<int64_t>(rows, 1 << 20);
        return launch_close(k_kv_join<T, D, NT, kWarps, kBits>, plan.cuts + plan.checks + plan.row_ctas, kJoinThreads, 0, stream, a,
                            few, many, plan);
    }
    plan.row_ctas = (int)std::min<int64_t>((rows + kWarps - 1) / kWarps, 1 << 20);
    return launch_close(k_kv_join<T, D, NT, 1, kBits>, plan.cuts + plan.checks + plan.row_ctas, kJoinThreads, 0, stream, a, few, many,
                        plan);
}
template <typename T, int D, int kBits>
cudaError_t attend_rows(const AttendArgs& a, bool brief, const FewWork& few, const ManyWork& many, cudaStream_t stream) {
    if (brief)
        return join_rows(a) <= 8 ? short_as<T, D, 1, kBits>(a, stream) : short_as<T, D, 2, kBits>(a, stream);
    return join_rows(a) <= 8 ? attend_as<T, D, 1, kBits>(a, few, many, stream) : attend_as<T, D, 2, kBits>(a, few, many, stream);
}

template <int kBits>
size_t attend_workspace_bytes(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t n_q_heads) {
    return bt.n_seqs == 0 ? 0 : layout<kBits>(c, bt, n_q_heads / c.n_heads).bytes;
}

// hold: a unit that a test build holds back (-1: none).
template <int kBits>
cudaError_t launch_attend(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& q, float scale, int32_t causal,
                          int32_t window, const mp_tokens& out, float* lse, int32_t* status, void* workspace, int64_t hold,
                          cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    const int32_t group = q.n_heads / c.n_heads;
    const Layout l = layout<kBits>(c, bt, group);
    if (window >= bt.max_len) window = 0;  // reaches back to every start
    const Route r = route<kBits>(c, bt, group, window);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    AttendArgs a;
    a.c = c, a.bt = bt, a.q = q, a.out = out, a.lse = lse, a.status = status;
    a.scale = scale, a.causal = causal, a.window = window;
    a.group = group;
    a.few_rows = r.few || r.brief ? kFewRows : -1;
    a.wide_q = rows_aligned(q), a.wide_out = rows_aligned(out);
#ifdef MP_TEST_HOOKS
    a.hold = hold;
#endif
    FewWork few = {};
    ManyWork many = {};
    if (r.few) {
        few.base = reinterpret_cast<int64_t*>(ws + l.base);
        few.gave_up = reinterpret_cast<int32_t*>(ws + l.gave_up);
        few.part = reinterpret_cast<float*>(ws + l.part);
    }
    if (r.many) {
        many.starts = reinterpret_cast<ManyStart*>(ws + l.starts);
        many.gave_up = reinterpret_cast<int32_t*>(ws + l.many_gave_up);
        many.part = reinterpret_cast<float*>(ws + l.many_part);
    }
    if (q.dtype == MP_F16)
        return c.head_dim == 64 ? attend_rows<__half, 64, kBits>(a, r.brief, few, many, stream)
                                : attend_rows<__half, 128, kBits>(a, r.brief, few, many, stream);
    return c.head_dim == 64 ? attend_rows<__nv_bfloat16, 64, kBits>(a, r.brief, few, many, stream)
                            : attend_rows<__nv_bfloat16, 128, kBits>(a, r.brief, few, many, stream);
}

}  // namespace
}  // namespace mp
