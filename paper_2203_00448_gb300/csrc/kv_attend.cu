// kv_attend.cu -- mp_kv_attend for few query rows a sequence and head (single
// tokens, a few proposed ones), the joining of split sequences, and the choice of kernels.
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
#include <algorithm>
#include <cmath>

#include "kv_attend.cuh"

namespace mp {
namespace {

// Warps of a CTA, and granules that the ring of each holds (192 KB at most in all). Registers bound the warps, an even
// share for the four schedulers: 12 of D = 128 with 16 rows spill (64 ragged contexts 127 -> 153 us, 10 160), 12 instead of
// 16 of D = 64 with 8 rows take 66 for 60 us. 8 with 3 granules for 12 with 2: 164 for 170 us over two of 262,144 tokens,
// but 103 for 97 over 64 ragged ones; 3 granules for 2 never paid otherwise (130 for 127).
constexpr int few_warps(int d, int nt) { return d == 128 ? (nt == 1 ? 12 : 8) : (nt == 1 ? 16 : 12); }
constexpr int kFewStages = 2;
constexpr int short_warps(int nt) { return nt == 1 ? 16 : 8; }
constexpr int kFewRows = 16;  // most rows of a sequence and head
constexpr int kJoinThreads = 256;  // k_kv_join of D = 128 keeps 16 bytes a thread in memory for it (48 registers), of 64 8 bytes

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
    int slots, slot;     // tiles x heads, tile * heads + head
    int64_t row;         // first row of the token arrays
    int n, len;          // the call's tokens, tokens held
    __device__ __forceinline__ void seek(int lo_, int hi_, int slots_, int64_t unit) {
        lo = lo_, hi = hi_, slots = slots_;
        slot = (int)quotient(unit, hi - lo);
        g = lo + (int)(unit - (int64_t)slot * (hi - lo));
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
    c.seek(lo, hi, slots, unit);
    return true;
}
template <int kRows>
__device__ __forceinline__ void next(const AttendArgs& a, Cursor& c) {
    if (++c.g < c.hi) return;
    c.g = c.lo;
    if (++c.slot < c.slots) return;
    do ++c.b;
    while (c.b < a.bt.n_seqs && !enter<kRows>(a, c, 0));
}
__device__ __forceinline__ int page_of(const AttendArgs& a, const Cursor& c) {
    const int p = __ldg(a.bt.table + (int64_t)c.b * a.bt.max_blocks + c.g / (a.c.block_tokens / kGranule));
    return p >= 0 && p < a.c.n_blocks ? p : 0;  // k_kv_join reports it; nothing outside the pool is read
}

__device__ __forceinline__ void mma(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                    uint32_t b1) {
    asm volatile(
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
template <typename T, int D, int NT>
struct Tile {
    uint32_t qf[NT][D / 16][2];        // Q^T: 4 consecutive values of row 8 nt + g a lane and chunk
    float unit[NT][2];                 // of score columns 2t, 2t + 1: scale * log2(e) over the row's power of two
    float top[NT][2], sum[NT][2];      // running maximum of x, this lane's part of the sum
    float o[NT][D / 16][4];
    int see_lo[NT][2], see_hi[NT][2];  // positions that the column's row sees
    int last;                          // stored bytes from this position on mean nothing

    // rows: of the sequence and head, at least 1; row: the sequence's first in the token arrays
    __device__ __forceinline__ void begin(const AttendArgs& a, int64_t row, int rows, int len, int n, int head, int tile) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
        last = 0;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = tile * 8 * NT + nt * 8 + g, there = min(r, rows - 1);
            const T* p = static_cast<const T*>(a.q.data) + (row + there / a.group) * a.q.token_stride +
                         (head * a.group + there % a.group) * a.q.head_stride + t * 4;
            // all loads at once: a branch in between would have each wait for the one before
            Pack<T, 4> raw[D / 16];
            if (a.wide_q) {
#pragma unroll
                for (int i = 0; i < D / 16; ++i) raw[i] = *reinterpret_cast<const Pack<T, 4>*>(p + i * 16);
            } else {
#pragma unroll
                for (int i = 0; i < D / 16; ++i)
#pragma unroll
                    for (int k = 0; k < 4; ++k) raw[i].x[k] = p[i * 16 + k];
            }
            float most = 0.f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) most = fmaxf(most, fabsf(to_f32(raw[i].x[k])));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
            most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
            const float f = row_factor(most);
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                qf[nt][i][0] = pack_f16(to_f32(raw[i].x[0]) * f, to_f32(raw[i].x[1]) * f);
                qf[nt][i][1] = pack_f16(to_f32(raw[i].x[2]) * f, to_f32(raw[i].x[3]) * f);
            }
            const float mine = __fdiv_rn(a.scale * 1.4426950408889634f, f);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                unit[nt][k] = __shfl_sync(~0u, mine, (2 * t + k) * 4);
                const int col = tile * 8 * NT + nt * 8 + 2 * t + k;
                const int pos = len - n + col / a.group;
                // columns past the last row repeat it and see all that is held: no one reads them
                see_hi[nt][k] = col < rows && a.causal ? min(len, pos + 1) : len;
                see_lo[nt][k] = col < rows && a.window > 0 ? pos - a.window + 1 : 0;
                last = max(last, see_hi[nt][k]);
                top[nt][k] = -INFINITY, sum[nt][k] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < D / 16; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
        }
        last = __reduce_max_sync(~0u, last);
    }

    // The granule at position base: its keys kb and values vb as stored, and their scales as stored.
    __device__ __forceinline__ void add(const uint8_t* kb, const uint8_t* vb, float ks, float stored_vs, int base) {
        const int lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
        // scores: product row r of 16 is token 4 (r % 8 / 2) + r % 2 + 2 (r / 8), the order in which a
        // lane's 4 stored value bytes meet the second product
        float s[NT][2][4] = {};
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const int tok = 4 * (g / 2) + g % 2;
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
        const float vs = value_scale(stored_vs), lv = log2f(vs), iv = __fdiv_rn(1.f, vs);
        uint32_t p[NT][2][2];
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
                        const int j = base + m * 16 + 4 * (g / 2) + g % 2 + 2 * h;
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
        const int meant = stored_vs < kLeastValueScale ? 0 : last;  // values from this position on are zeros
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

    // This lane's part of a column's sum becomes the column's.
    __device__ __forceinline__ float total(int nt, int k) const {
        float l = sum[nt][k];
        l += __shfl_xor_sync(~0u, l, 4);
        l += __shfl_xor_sync(~0u, l, 8);
        l += __shfl_xor_sync(~0u, l, 16);
        return l;
    }
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(few_warps(D, NT) * 32, 1) k_kv_attend_few(AttendArgs a, FewWork work) {
    constexpr int kFewWarps = few_warps(D, NT);
    constexpr int kRows = 8 * NT;
    constexpr int kBytes = kGranule * D;  // of either array
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
    const int64_t per_warp = quotient(total + warps - 1, warps);
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
    auto issue = [&]() {  // the next unit's bytes into its stage
        if (issued >= u1) return;
        const int st = (int)((issued - u0) % kFewStages);
        const int64_t at = block_byte(a.c, page_ahead, ahead.slot % a.c.n_heads) +
                           (int64_t)(ahead.g % (a.c.block_tokens / kGranule)) * kBytes;
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

    Tile<T, D, NT> x;
    bool up = false;
    int done = 0;  // units

    for (int left = (int)(u1 - u0); left > 0 && !up;) {
        // one (sequence, tile, head) or what this warp has of it
        const int head = cur.slot % a.c.n_heads, tile = cur.slot / a.c.n_heads;
        const int rows = cur.n * a.group, units = min(cur.hi - cur.g, left);
        const bool whole = units == cur.hi - cur.lo;
        const bool first = done == 0;
        left -= units;
        x.begin(a, cur.row, rows, cur.len, cur.n, head, tile);
#pragma unroll 1
        for (int i = 0; i < units; ++i, ++done, ++cur.g) {
            const int st = done % kFewStages;
            if (!__all_sync(~0u, mbar_wait(&bar[st], (uint32_t)(done / kFewStages & 1)))) {
                up = true;
                break;
            }
            const int64_t sc = (int64_t)ring_page[st] * a.c.n_heads + head;
            const float ks = __ldg(a.c.k_scale + sc), vs = __ldg(a.c.v_scale + sc);
            x.add(ring + st * 2 * kBytes, ring + st * 2 * kBytes + kBytes, ks, vs, cur.g * kGranule);
            __syncwarp();
            issue();
        }
        if (up) break;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float l = x.total(nt, k);
                const int in_tile = nt * 8 + 2 * t + k, r = tile * kRows + in_tile;
                const float m = x.top[nt][k];
                if (whole) {
                    if (r < rows) {
                        const int64_t tok = cur.row + r / a.group;
                        const int qh = head * a.group + r % a.group;
                        T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
                        const float inv = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) {
                            dst[i * 16 + g] = from_f32<T>(x.o[nt][i][k] * inv);
                            dst[i * 16 + g + 8] = from_f32<T>(x.o[nt][i][2 + k] * inv);
                        }
                        if (a.lse != nullptr && g == 0)
                            a.lse[tok * a.q.n_heads + qh] = log_sum(m, kLift, l);
                    }
                } else {
                    // a warp leaves at most two parts: of what began before it or with it, and of
                    // what it begins and does not end
                    float* part = work.part + ((int64_t)2 * w + (first ? 0 : 1)) * (kRows * (D + 2));
                    float* dst = part + in_tile * D;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        dst[i * 16 + g] = x.o[nt][i][k];
                        dst[i * 16 + g + 8] = x.o[nt][i][2 + k];
                    }
                    if (g == 0) {
                        part[kRows * D + 2 * in_tile] = m;
                        part[kRows * D + 2 * in_tile + 1] = l;
                    }
                }
            }
        --cur.g;
        if (left > 0) next<kRows>(a, cur);
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
template <typename T, int D, int NT>
__global__ void __launch_bounds__(short_warps(NT) * 32, 1) k_kv_attend_short(AttendArgs a) {
    constexpr int kRows = 8 * NT, kBytes = kGranule * D, kWarps = short_warps(NT);
    static_assert(kRows * D * sizeof(float) <= 2 * kBytes, "a warp's sums fit where its granules were");
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
    uint8_t* const mine = dyn + wid * 2 * kBytes;
    Tile<T, D, NT> x;
    for (int tile = 0; tile * kRows < rows; ++tile) {
        for (int gran = lo + wid; gran < hi; gran += kWarps) {
            int page = __ldg(table + gran / per);
            if (page < 0 || page >= a.c.n_blocks) page = 0;  // reported above
            const int64_t at = block_byte(a.c, page, head) + (int64_t)(gran % per) * kBytes;
#pragma unroll
            for (int i = 0; i < kBytes / 512; ++i) {
                const int o = (i * 32 + lane) * 16;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(mine + o)), "l"(a.c.k + at + o) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(mine + kBytes + o)), "l"(a.c.v + at + o)
                             : "memory");
            }
            const int64_t sc = (int64_t)page * a.c.n_heads + head;
            const float ks = __ldg(a.c.k_scale + sc), vs = __ldg(a.c.v_scale + sc);
            if (gran == lo + wid) x.begin(a, s.lo, rows, s.len, s.n, head, tile);
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            x.add(mine, mine + kBytes, ks, vs, gran * kGranule);
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
                        acc[r * D + i * 16 + g] = x.o[nt][i][k];
                        acc[r * D + i * 16 + g + 8] = x.o[nt][i][2 + k];
                    }
                }
                if (g == 0) ref[wid][r] = any ? x.top[nt][k] : -INFINITY, weight[wid][r] = l;
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
                const float2 y = *reinterpret_cast<const float2*>(dyn + w * 2 * kBytes + (in_tile * D + d) * sizeof(float));
                sum += weight[w][in_tile] * f, o0 += y.x * f, o1 += y.y * f;
            }
            const float inv = sum == 0.f ? 0.f : __fdiv_rn(1.f, sum);
            const int64_t tok = s.lo + r / a.group;
            const int qh = head * a.group + r % a.group;
            T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride + d;
            const float y[2] = {o0 * inv, o1 * inv};
            store_values<T, 2>(dst, a.wide_out, y);
            if (d == 0 && a.lse != nullptr)
                a.lse[tok * a.q.n_heads + qh] = log_sum(top, kLift, sum);
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
template <typename T, int D, int NT, int kPer>
__device__ void join_row(const AttendArgs& a, const FewWork& work, int64_t u, bool there) {
    constexpr int kRows = 8 * NT, kCols = D / 32, kAhead = 4;
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
    const float inv = l == 0.f ? 0.f : __fdiv_rn(1.f, l);
#pragma unroll
    for (int i = 0; i < kCols; ++i) o[i] *= inv;
    store_values<T, kCols>(dst + lane * kCols, a.wide_out, o);
    if (a.lse != nullptr && lane == 0)
        a.lse[tok * a.q.n_heads + qh] = log_sum(top, kLift, l);
}

// After both kernels: what more than one CTA or warp had of a row, and the sequences' status.  kPer: warps a row.
template <typename T, int D, int NT, int kPer>
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
        join_row<T, D, NT, kPer>(a, few, mine < rows ? mine : 0, mine < rows);
    }
}

// Sequences of few rows in a batch that also has many: k_kv_attend_many takes them at about 2.5 TB/s of cache bytes, which
// up to this size costs less than the other kernel with its joining where most sequences have many rows (8 heads of 128,
// GPU time without and with it: 16 x 1,000 tokens 31 and 45 us, 8 x 4,000 96 and 145, 3 x 4,000-16,384 157 and 161; 16 of up
// to 8,000, 8 with pieces of 512 and 8 with single tokens, 315 and 331).  Where one piece of 512 comes with single
// tokens, both kernels are the faster way from well below: 16 singles of up to 2,000 (41 MB held) 57 and 57, 32 of up to
// 4,000 (145 MB) 116 and 94, 63 of up to 2,000 (162 MB) 130 and 87; past the line 63 of up to 4,000 (294 MB) 189 and 122, 255 of
// up to 8,000 (2.2 GB) 1,019 and 490.  The line goes by what the host knows, the number of sequences times the bound of
// their lengths; a generous bound leads to both kernels.
constexpr int64_t kSmallCache = 256 << 20;
// Which kernels a batch needs, by its host scalars: sequences of at most kFewRows rows are
// bound by the cache's bytes, which k_kv_attend_few streams; above it the products count.
// A batch whose sequences all have max_tokens has no sequence for the first.
// Few rows of short contexts in batches that fill the GPU at most twice over go to k_kv_attend_short (8 heads, the GPU's
// time of a call: 1 x 512 tokens 6.6 us against 9.4, 8 x 1,024 8.8 against 11.7, 38 x 2,048 32.6 against 37.2; but
// 1 x 4,096 19.3 against 14.7, and 128 x 512, four times the SMs, 48.6 against 35.4).
constexpr int32_t kShortLen = 2048;
constexpr int64_t kShortCtas = 2 * kSms;
struct Route {
    bool few, many, brief;
};
Route route(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t group, int32_t window) {
    // An empty pool has no block that could stand in for a bad table entry's: k_kv_join alone says which sequences are
    // wrong (all that see a position) and writes the rows that see nothing.
    if (c.n_blocks == 0) return {false, false, false};
    if ((int64_t)bt.max_tokens * group <= kFewRows) {
        const int32_t span = window > 0 ? std::min(bt.max_len, window + bt.max_tokens) : bt.max_len;
        const bool brief = span <= kShortLen && (int64_t)bt.n_seqs * c.n_heads <= kShortCtas;
        return {!brief, false, brief};
    }
    const int64_t bytes = (int64_t)bt.n_seqs * bt.max_len * c.n_heads * c.head_dim * 2;
    return {bt.n_tokens != (int64_t)bt.n_seqs * bt.max_tokens && bytes > kSmallCache, true, false};
}

struct Layout {
    size_t base, gave_up, part, starts, many_gave_up, many_part, bytes;
};
// (The scratch is asked for before the window is known: a window can only leave it unused.)
Layout layout(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t group) {
    Layout l = {};
    const Route r = route(c, bt, group, 0);
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

template <typename T, int D, int NT>
cudaError_t short_as(const AttendArgs& a, cudaStream_t stream) {
    constexpr size_t smem = (size_t)short_warps(NT) * 2 * kGranule * D;
    cudaError_t e = set_smem_limit((const void*)k_kv_attend_short<T, D, NT>, smem);
    if (e != cudaSuccess) return e;
    return launch_close(k_kv_attend_short<T, D, NT>, a.bt.n_seqs * a.c.n_heads, short_warps(NT) * 32, smem, stream, a);
}

template <typename T, int D, int NT>
cudaError_t attend_as(const AttendArgs& a, const FewWork& few, const ManyWork& many, cudaStream_t stream) {
    cudaError_t e;
    JoinPlan plan = {};
    plan.checks = std::min(a.bt.n_seqs, 1024);
    int64_t rows = 0;
    if (few.base != nullptr) {
        constexpr size_t smem = (size_t)few_warps(D, NT) * kFewStages * 2 * kGranule * D;
        e = set_smem_limit((const void*)k_kv_attend_few<T, D, NT>, smem);
        if (e == cudaSuccess)
            e = launch_close(k_kv_attend_few<T, D, NT>, kFewCtas, few_warps(D, NT) * 32, smem, stream, a, few);
        if (e != cudaSuccess) return e;
        rows = (int64_t)a.bt.n_seqs * join_rows(a) * a.c.n_heads;
    }
    if (many.part != nullptr) {
        e = launch_kv_many(a, many, stream);
        if (e != cudaSuccess) return e;
        plan.cuts = kManyCtas * (D / kJoinCols);
    }
    // rows that are cut into many parts have a CTA each, whose warps share the parts (64 rows of 76 parts: 18 -> 5 us), the
    // others a warp (2,048 rows of two or three: 12 -> 7 us)
    constexpr int kWarps = kJoinThreads / 32;
    const int64_t parts = kFewCtas * few_warps(D, NT) / ((int64_t)a.bt.n_seqs * a.c.n_heads);
    if (rows <= 8 * kFewCtas || parts > 12) {
        plan.row_ctas = (int)std::min<int64_t>(rows, 1 << 20);
        return launch_close(k_kv_join<T, D, NT, kWarps>, plan.cuts + plan.checks + plan.row_ctas, kJoinThreads, 0, stream, a,
                            few, many, plan);
    }
    plan.row_ctas = (int)std::min<int64_t>((rows + kWarps - 1) / kWarps, 1 << 20);
    return launch_close(k_kv_join<T, D, NT, 1>, plan.cuts + plan.checks + plan.row_ctas, kJoinThreads, 0, stream, a, few, many,
                        plan);
}
template <typename T, int D>
cudaError_t attend_rows(const AttendArgs& a, bool brief, const FewWork& few, const ManyWork& many, cudaStream_t stream) {
    if (brief)
        return join_rows(a) <= 8 ? short_as<T, D, 1>(a, stream) : short_as<T, D, 2>(a, stream);
    return join_rows(a) <= 8 ? attend_as<T, D, 1>(a, few, many, stream) : attend_as<T, D, 2>(a, few, many, stream);
}

}  // namespace

size_t kv_attend_workspace_bytes(const mp_kv_cache& c, const mp_kv_batch& bt, int32_t n_q_heads) {
    return bt.n_seqs == 0 ? 0 : layout(c, bt, n_q_heads / c.n_heads).bytes;
}

#ifdef MP_TEST_HOOKS
static int64_t g_test_kv_hold = -1;
#endif

cudaError_t launch_kv_attend(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& q, float scale,
                             int32_t causal, int32_t window, const mp_tokens& out, float* lse, int32_t* status,
                             void* workspace, cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    const int32_t group = q.n_heads / c.n_heads;
    const Layout l = layout(c, bt, group);
    if (window >= bt.max_len) window = 0;  // reaches back to every start
    const Route r = route(c, bt, group, window);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    AttendArgs a;
    a.c = c, a.bt = bt, a.q = q, a.out = out, a.lse = lse, a.status = status;
    a.scale = scale, a.causal = causal, a.window = window;
    a.group = group;
    a.few_rows = r.few || r.brief ? kFewRows : -1;
    a.wide_q = rows_aligned(q), a.wide_out = rows_aligned(out);
#ifdef MP_TEST_HOOKS
    a.hold = g_test_kv_hold;
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
        return c.head_dim == 64 ? attend_rows<__half, 64>(a, r.brief, few, many, stream)
                                : attend_rows<__half, 128>(a, r.brief, few, many, stream);
    return c.head_dim == 64 ? attend_rows<__nv_bfloat16, 64>(a, r.brief, few, many, stream)
                            : attend_rows<__nv_bfloat16, 128>(a, r.brief, few, many, stream);
}

}  // namespace mp

#ifdef MP_TEST_HOOKS
// Test builds only: later mp_kv_attend calls of this process hold the unit back (-1: none).
extern "C" __attribute__((visibility("default"))) void mp_test_kv_hold(int64_t unit) { mp::g_test_kv_hold = unit; }
#endif
