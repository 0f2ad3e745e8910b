// kv_attend_many.cu -- mp_kv_attend for sequences with many query rows (prompts, pieces
// of prompts): both products on the fifth-generation tensor cores.
//
// Rows are tokens x heads of a group, so a tile of 128 rows shares the cached head
// whatever the group.  A CTA works on two such tiles: while one's scores become weights
// (a thread a row), the tensor cores work for the other.  Warps 0-3 and 4-7: softmax of
// tile 0 and 1; warps 8-11 turn the stored bytes of 128 tokens into f16 operands in
// shared memory (exact; two hardware conversions for 4 bytes, 8 thread operations a
// clock less than a third of what the products leave free); one thread of warp 12 issues
// every product.  Scores (128 x 128 f32) and sums (128 x D f32) of both tiles fill the
// 512 columns of tensor memory; weights go back as f16 over the scores they came from
// and are the left operand of the second product from there.  The softmax is that of the
// kernel for few rows (the value scale in the exponent), but a row's sums are rescaled
// only when its maximum has grown by 2^8.
//
// (sequence, row tile pair, head, 128 tokens) units lie on a line that is cut evenly
// among 152 CTAs, so that causal rows, ragged prompts and a short piece over a long
// context all end together; what a CTA does not hold whole is added up by
// k_kv_join_many.
#include <algorithm>
#include <cmath>

#include "kv_attend.cuh"

namespace mp {
namespace {

constexpr int kRows = 128;      // of one tile
constexpr int kPair = 2 * kRows;
constexpr int kTokens = 128;    // of a unit
constexpr int kGrans = kTokens / kGranule;
constexpr int kStages = 2;      // of keys and of values
constexpr int kScaleRing = 4;
constexpr int kThreads = 13 * 32;
constexpr int kStrips = 1024;
constexpr float kManyLift = 7.f;  // weights are at most 2^(8 + 7)
constexpr float kGrow = 8.f;

__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t lead, uint32_t stride) {
    // K-major tiles of 8 rows x 16 bytes: lead = bytes between neighbours along K, stride = along M or N
    return (uint64_t)((addr >> 4) & 0x3fff) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 | 1ull << 46;
}
constexpr uint32_t product_of(int m, int n) {  // f16 x f16 -> f32, both K-major
    return 1u << 4 | (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t what, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(what), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t what, bool add) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(what), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar))
                 : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ void ld32(uint32_t addr, float* x) {
    uint32_t* r = reinterpret_cast<uint32_t*>(x);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}
__device__ __forceinline__ void st32(uint32_t addr, const float* x) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(x);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
        "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]),
        "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
        "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(addr));
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr));
}

// A stretch of the line inside one (sequence, pair of row tiles, head).
struct Stretch {
    int b, tile, head;
    int cnt, k;              // units of the whole, the first of this stretch
    int first_gran, grans;   // granules that the pair's rows see
    int rows;                // of the sequence and head
    int len, start;          // tokens held; position of the call's first
    int64_t row;             // its first row of the token arrays
};

__device__ __forceinline__ int pairs_of(const ManyArgs& a, const SeqView& s) {
    if (s.st != MP_OK || (a.few_rows > 0 && (int64_t)s.n * a.group <= a.few_rows)) return 0;
    return (s.n * a.group + kPair - 1) / kPair;
}
__device__ __forceinline__ void pair_grans(const ManyArgs& a, const SeqView& s, int tile, int& lo, int& n) {
    const int start = s.len - s.n, rows = s.n * a.group;
    const int p0 = start + tile * kPair / a.group, p1 = start + (min(rows, (tile + 1) * kPair) - 1) / a.group;
    const int past = a.causal ? min(s.len, max(p1 + 1, 0)) : s.len;
    lo = a.window > 0 ? max(0, p0 - a.window + 1) / kGranule : 0;
    n = max(0, (past + kGranule - 1) / kGranule - lo);
}
__device__ __forceinline__ int pair_units(const ManyArgs& a, const SeqView& s, int tile) {
    int lo, n;
    pair_grans(a, s, tile, lo, n);
    return (n + kGrans - 1) / kGrans;
}
// Units of a sequence; a warp's lanes take its pairs in turn.
__device__ __forceinline__ int64_t seq_units_warp(const ManyArgs& a, int b, int lane) {
    const SeqView s = load_seq(a.bt, b, false);
    const int pairs = pairs_of(a, s);
    int64_t n = 0;
    for (int i = lane; i < pairs; i += 32) n += pair_units(a, s, i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(~0u, n, o);
    return n * a.c.n_heads;
}
__device__ __forceinline__ void fill(const ManyArgs& a, const SeqView& s, Stretch& x) {
    pair_grans(a, s, x.tile, x.first_gran, x.grans);
    x.cnt = (x.grans + kGrans - 1) / kGrans;
    x.rows = s.n * a.group;
    x.len = s.len, x.start = s.len - s.n, x.row = s.lo;
}
// The stretch that follows on the line (there is one: the caller has units left).
__device__ __forceinline__ void advance(const ManyArgs& a, Stretch& x) {
    x.k = 0;
    if (++x.head < a.c.n_heads) return;
    x.head = 0;
    ++x.tile;
    for (;;) {
        const SeqView s = load_seq(a.bt, x.b, false);
        const int pairs = pairs_of(a, s);
        for (; x.tile < pairs; ++x.tile)
            if (pair_units(a, s, x.tile) > 0) {
                fill(a, s, x);
                return;
            }
        ++x.b, x.tile = 0;
        if (x.b >= a.bt.n_seqs) return;
    }
}
__device__ __forceinline__ int granule_page(const ManyArgs& a, int b, int gran) {
    const int p = __ldg(a.bt.table + (int64_t)b * a.bt.max_blocks + gran / (a.c.block_tokens / kGranule));
    return p >= 0 && p < a.c.n_blocks ? p : 0;  // k_kv_join_many reports it
}

template <int D>
struct Smem {
    uint8_t q[2][kRows * D * 2];
    uint8_t k[kStages][kTokens * D * 2];
    uint8_t v[kStages][kTokens * D * 2];
    int64_t strip[kStrips];
    float scales[kScaleRing][3][kGrans];  // key scale, log2 of the value scale, 1 / value scale
    uint64_t q_full[2], s_full[2], p_full[2], o_done[2], k_full[kStages], k_empty[kStages], v_full[kStages],
        v_empty[kStages], drained;
    Stretch first;
    int64_t total;
    uint32_t tmem;
    int gave_up;
};

// Waits until the phase ends; false if some wait of the CTA has given up.
__device__ __forceinline__ bool await(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (!mbar_try(bar, parity)) {
        if (*gave_up) return false;
        if (clock64() - t0 > kKvSpinCycles) {
            *gave_up = 1;
            return false;
        }
    }
    return true;
}

// ... by all lanes of a warp, with one answer for all.
__device__ __forceinline__ bool await_warp(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
    return __all_sync(~0u, await(bar, parity, gave_up));
}

constexpr uint32_t kScoreCol = 0, kSumCol = 256;  // of tile 0; tile 1 has + 128 and + D

template <typename T, int D>
__device__ void convert_role(const ManyArgs& a, Smem<D>& m, Stretch x, int64_t left) {
    constexpr int kLoads = kTokens * D / 16 / 128;       // 16-byte loads a thread, of either array
    constexpr int kPerGran = kGranule * D / 16 / 128;    // ... of which a granule is this many, 1 or 2
    const int tid = threadIdx.x - 256;
    uint4 kr[kLoads], vr[kLoads];
    int64_t at[kGrans];
    int it = 0, tail = 0;
    // the granules of the unit at hand: where they are, -1 past the last
    auto locate = [&]() {
#pragma unroll
        for (int i = 0; i < kGrans; ++i) {
            const int g = x.k * kGrans + i;
            at[i] = -1;
            if (g < x.grans) {
                const int gran = x.first_gran + g, page = granule_page(a, x.b, gran);
                at[i] = block_byte(a.c, page, x.head) +
                        (int64_t)(gran % (a.c.block_tokens / kGranule)) * (kGranule * D);
            }
        }
        tail = x.len - (x.first_gran + x.k * kGrans) * kGranule;  // tokens of the unit that are held
    };
    auto load = [&](const uint8_t* pool, uint4* r) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            r[i] = at[i / kPerGran] < 0 ? make_uint4(0, 0, 0, 0)
                                        : __ldg(reinterpret_cast<const uint4*>(pool + at[i / kPerGran]) +
                                                (i % kPerGran) * 128 + tid);
    };
    auto widen = [](const uint4& w, uint4& lo, uint4& hi) {
        e4m3_to_f16(w.x, lo.x, lo.y), e4m3_to_f16(w.y, lo.z, lo.w);
        e4m3_to_f16(w.z, hi.x, hi.y), e4m3_to_f16(w.w, hi.z, hi.w);
    };
    if (left > 0) {
        locate();
        load(a.c.k, kr);
    }
    while (left > 0) {
        const int st = it % kStages;
        const uint32_t empty = (it / kStages & 1) ^ 1;
        load(a.c.v, vr);
        float ks = 0.f, vs = 1.f;
        if (tid < kGrans && x.k * kGrans + tid < x.grans) {
            const int64_t sc =
                (int64_t)granule_page(a, x.b, x.first_gran + x.k * kGrans + tid) * a.c.n_heads + x.head;
            ks = __ldg(a.c.k_scale + sc), vs = value_scale(__ldg(a.c.v_scale + sc));
        }
        if (!await_warp(&m.k_empty[st], empty, &m.gave_up)) return;
        if (tid < kGrans) {
            // the slot's last readers are done: this stage's last scores were issued after sums that had
            // waited for the weights of the unit that had the slot
            float(*sc)[kGrans] = m.scales[it % kScaleRing];
            sc[0][tid] = ks, sc[1][tid] = log2f(vs), sc[2][tid] = __fdiv_rn(1.f, vs);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            // stored tiles [token / 8][D / 16][8][16] become f16 tiles [token / 8][D / 8][8][8]
            const int q = i * 128 + tid;
            uint4 lo, hi;
            widen(kr[i], lo, hi);
            uint4* dst = reinterpret_cast<uint4*>(m.k[st]) + (q / 8) * 16 + q % 8;
            dst[0] = lo, dst[8] = hi;
        }
        fence_smem();
        mbar_arrive(&m.k_full[st]);
        const int had = tail;
        const bool more = left > 1;
        if (more) {
            if (++x.k == x.cnt) advance(a, x);
            locate();
            load(a.c.k, kr);
        }
        if (!await_warp(&m.v_empty[st], empty, &m.gave_up)) return;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            // stored tiles [granule][D / 8][2][8][16] become [granule][D / 8][4][8][8]
            const int q = i * 128 + tid;
            uint4 w = vr[i], lo, hi;
            const int t0 = i / kPerGran * kGranule + (q / 8 % 2) * 16;
            if (had < t0 + 16) {  // bytes behind the last token mean nothing, NaN among them
                uint32_t* p = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = had - t0 - 4 * j;
                    p[j] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                }
            }
            widen(w, lo, hi);
            uint4* dst = reinterpret_cast<uint4*>(m.v[st]) + (q / 8) * 16 + q % 8;
            dst[0] = lo, dst[8] = hi;
        }
        fence_smem();
        mbar_arrive(&m.v_full[st]);
        ++it, --left;
    }
}

template <int D>
__device__ void product_role(const ManyArgs& a, Smem<D>& m, Stretch x, int64_t left) {
    constexpr uint32_t kScores = product_of(kRows, kTokens), kSums = product_of(kRows, D);
    const uint32_t tm = m.tmem;
    int it = 0, n[2] = {0, 0}, seg[2] = {0, 0};  // units, units of either tile, stretches of either tile
    auto scores = [&](int i, int st) {
        const uint32_t q = smem_addr(m.q[i]), k = smem_addr(m.k[st]);
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
            mma_ss(tm + kScoreCol + i * 128, operand(q + s * 256, 128, D * 16), operand(k + s * 256, 128, D * 16), kScores,
                   s > 0);
        commit(&m.s_full[i]);
    };
    auto sums = [&](int i, int st, bool add) {
        const uint32_t v = smem_addr(m.v[st]);
#pragma unroll
        for (int s = 0; s < kTokens / 16; ++s)
            mma_ts(tm + kSumCol + i * D, tm + kScoreCol + i * 128 + s * 8,
                   operand(v + (s / 2) * (kGranule * D * 2) + (s % 2) * 256, 128, 512), kSums, add || s > 0);
        commit(&m.o_done[i]);
    };
    // the first unit's scores
    {
        const int tiles = x.rows - x.tile * kPair > kRows ? 2 : 1;
        if (!await(&m.k_full[0], 0, &m.gave_up)) return;
        for (int i = 0; i < tiles; ++i) {
            if (!await(&m.q_full[i], seg[i]++ & 1, &m.gave_up)) return;
            fence_after();
            scores(i, 0);
        }
        commit(&m.k_empty[0]);
    }
    while (left > 0) {
        const int tiles = x.rows - x.tile * kPair > kRows ? 2 : 1;
        const bool add = n[0] > 0 && x.k > 0 && it > 0;
        Stretch y = x;
        bool fresh = false;
        if (left > 1 && ++y.k == y.cnt) {
            advance(a, y);
            fresh = true;
        }
        const int next_tiles = left > 1 ? (y.rows - y.tile * kPair > kRows ? 2 : 1) : 0;
        const int st = it % kStages, nst = (it + 1) % kStages;
        if (!await(&m.v_full[st], it / kStages & 1, &m.gave_up)) return;
        for (int i = 0; i < 2; ++i) {
            if (i < tiles) {
                if (!await(&m.p_full[i], n[i] & 1, &m.gave_up)) return;
                fence_after();
                sums(i, st, add);
                if (i == tiles - 1) commit(&m.v_empty[st]);
                ++n[i];
            }
            if (i < next_tiles) {
                if (i == 0 && !await(&m.k_full[nst], (it + 1) / kStages & 1, &m.gave_up)) return;
                if (fresh && !await(&m.q_full[i], seg[i]++ & 1, &m.gave_up)) return;
                // its scores overwrite the weights that the product before reads: products of different
                // sums are not ordered among themselves
                if (n[i] > 0 && !await(&m.o_done[i], (n[i] - 1) & 1, &m.gave_up)) return;
                fence_after();
                scores(i, nst);
                if (i == next_tiles - 1) commit(&m.k_empty[nst]);
            }
        }
        x = y;
        ++it, --left;
    }
}

template <typename T, int D>
__device__ void softmax_role(const ManyArgs& a, Smem<D>& m, Stretch x, int64_t left, int w) {
    const int tile = threadIdx.x / 128, tid = threadIdx.x % 128, warp = tid / 32;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t sc = m.tmem + lanes + kScoreCol + tile * 128, su = m.tmem + lanes + kSumCol + tile * D;
    int it = 0, n = 0;  // units of the CTA, of this tile
    float unit = 0.f, next_unit = 0.f;
    // a row of the tile into shared memory as f16, scaled; returns what scores are to be multiplied by
    auto load_q = [&](const Stretch& y) {
        const int r = y.tile * kPair + tile * kRows + tid;
        const bool there = r < y.rows;
        const T* p = static_cast<const T*>(a.q.data) + (y.row + r / a.group) * a.q.token_stride +
                     (y.head * a.group + r % a.group) * a.q.head_stride;
        float most = 0.f;
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
            float v[8];
            if (there) {
                load_values<T, 8>(p + i * 8, a.wide_q, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(v[j]));
            }
        }
        const float f = row_factor(most);
#pragma unroll 4
        for (int i = 0; i < D / 8; ++i) {
            float v[8] = {};
            if (there) load_values<T, 8>(p + i * 8, a.wide_q, v);
            uint4 o;
            o.x = pack_f16(v[0] * f, v[1] * f), o.y = pack_f16(v[2] * f, v[3] * f);
            o.z = pack_f16(v[4] * f, v[5] * f), o.w = pack_f16(v[6] * f, v[7] * f);
            reinterpret_cast<uint4*>(m.q[tile])[((tid / 8) * (D / 8) + i) * 8 + tid % 8] = o;
        }
        fence_smem();
        mbar_arrive(&m.q_full[tile]);
        return __fdiv_rn(a.scale * 1.4426950408889634f, f);
    };
    auto active = [&](const Stretch& y) { return tile == 0 || y.rows - y.tile * kPair > kRows; };

    if (active(x)) next_unit = load_q(x);
    const int64_t whole_line = left;
    while (left > 0) {
        const int units = (int)min((int64_t)(x.cnt - x.k), left);  // of this stretch
        const bool mine = active(x);
        if (!mine) {
            it += units, left -= units;
            if (left > 0) {
                advance(a, x);
                if (active(x)) next_unit = load_q(x);
            }
            continue;
        }
        unit = next_unit;
        const int r = x.tile * kPair + tile * kRows + tid;
        const int pos = x.start + r / a.group;
        const int see_hi = r >= x.rows ? 0 : a.causal ? min(x.len, max(pos + 1, 0)) : x.len;
        const int see_lo = a.window > 0 ? pos - a.window + 1 : 0;
        float top = -INFINITY, sum = 0.f;
        for (int u = 0; u < units; ++u, ++it, ++n) {
            const int base = (x.first_gran + (x.k + u) * kGrans) * kGranule;
            if (!await_warp(&m.s_full[tile], n & 1, &m.gave_up)) return;
            fence_after();
            const float(*scale)[kGrans] = m.scales[it % kScaleRing];
            const bool edge = __any_sync(~0u, base + kTokens > see_hi || base < see_lo);
            float most = -INFINITY;
            float s[32];
#pragma unroll
            for (int c = 0; c < kGrans; ++c) {
                ld32(sc + c * 32, s);
                wait_ld();
                float big = -INFINITY;
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int t = base + c * 32 + j;
                        if (t < see_hi && t >= see_lo) big = fmaxf(big, s[j]);
                    }
                    if (big > -INFINITY) most = fmaxf(most, fmaf(big, unit * scale[0][c], scale[1][c]));
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) big = fmaxf(big, s[j]);
                    most = fmaxf(most, fmaf(big, unit * scale[0][c], scale[1][c]));
                }
            }
            const bool grows = most > top + kGrow || (top == -INFINITY && most > -INFINITY);
            if (__any_sync(~0u, grows)) {
                const float now = grows ? most : top;
                const float fade = top == -INFINITY ? 0.f : exp2_approx(top - now);
                top = now;
                sum *= fade;
                if (u > 0) {
                    if (!await_warp(&m.o_done[tile], (n - 1) & 1, &m.gave_up)) return;
                    fence_after();
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        ld32(su + c * 32, s);
                        wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) s[j] *= fade;
                        st32(su + c * 32, s);
                    }
                }
            }
            const float ref = top == -INFINITY ? 0.f : top - kManyLift;
#pragma unroll
            for (int c = 0; c < kGrans; ++c) {
                ld32(sc + c * 32, s);
                wait_ld();
                const float mul = unit * scale[0][c], off = scale[1][c] - ref;
                float part = 0.f;
                uint32_t p[16];
                if (edge) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int t = base + c * 32 + j;
                        s[j] = t < see_hi && t >= see_lo ? exp2_approx(fmaf(s[j], mul, off)) : 0.f;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) s[j] = exp2_approx(fmaf(s[j], mul, off));
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    part += s[2 * j] + s[2 * j + 1];
                    p[j] = pack_f16(s[2 * j], s[2 * j + 1]);
                }
                sum = fmaf(part, scale[2][c], sum);
                st16(sc + c * 16, p);
            }
            wait_st();
            fence_before();
            mbar_arrive(&m.p_full[tile]);
        }
        // the next stretch's queries go in before this one's sums come out
        const Stretch done = x;
        left -= units;
        if (left > 0) {
            advance(a, x);
            if (active(x)) next_unit = load_q(x);
        }
        if (!await_warp(&m.o_done[tile], (n - 1) & 1, &m.gave_up)) return;
        fence_after();
        const bool whole = done.k == 0 && units == done.cnt;
        const bool first = whole_line - left - units == 0;  // of the CTA's stretches
        const int64_t tok = done.row + r / a.group;
        const int qh = done.head * a.group + r % a.group;
        T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
        const float inv = sum == 0.f ? 0.f : __fdiv_rn(1.f, sum);
        // stretches that are not whole: at most the CTA's first and its last
        float* part = a.part + ((int64_t)2 * w + (first ? 0 : 1)) * (kPair * (D + 2));
        const int pr = tile * kRows + tid;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            float o[32];
            ld32(su + c * 32, o);
            wait_ld();
            if (whole) {
                if (r < done.rows) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) o[j] *= inv;
#pragma unroll
                    for (int j = 0; j < 4; ++j) store_values<T, 8>(dst + c * 32 + j * 8, a.wide_out, o + j * 8);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) part[(c * 32 + j) * kPair + pr] = o[j];
            }
        }
        if (whole) {
            if (r < done.rows && a.lse != nullptr)
                a.lse[tok * a.q.n_heads + qh] = top == -INFINITY ? -INFINITY : (top - kManyLift + log2f(sum)) * 0.6931471805599453f;
        } else {
            part[D * kPair + pr] = top;
            part[(D + 1) * kPair + pr] = sum;
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) k_kv_attend_many(ManyArgs a) {
    extern __shared__ __align__(1024) uint8_t dyn[];
    Smem<D>& m = *reinterpret_cast<Smem<D>*>(dyn);
    const int tid = threadIdx.x, lane = tid % 32, wid = tid / 32;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&m.q_full[i], kRows), mbar_init(&m.s_full[i], 1);
            mbar_init(&m.p_full[i], kRows), mbar_init(&m.o_done[i], 1);
        }
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&m.k_full[i], 128), mbar_init(&m.k_empty[i], 1);
            mbar_init(&m.v_full[i], 128), mbar_init(&m.v_empty[i], 1);
        }
        mbar_init(&m.drained, 1);
        m.gave_up = 0;
        fence_mbar_init();
    }
    if (wid == 12) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&m.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    // the line: strips of sequences, a warp a strip
    const int strip = (a.bt.n_seqs + kStrips - 1) / kStrips;
    for (int i = wid; i < kStrips; i += kThreads / 32) {
        int64_t n = 0;
        for (int b = i * strip; b < min((i + 1) * strip, a.bt.n_seqs); ++b) n += seq_units_warp(a, b, lane);
        if (lane == 0) m.strip[i] = n;
    }
    __syncthreads();
    if (wid == 0) {
        // totals before each run of 32 strips, then the strip, sequence and pair of this CTA's first unit
        int64_t mine = 0;
        for (int i = 0; i < kStrips / 32; ++i) mine += m.strip[lane * (kStrips / 32) + i];
        int64_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += y;
        }
        const int64_t total = __shfl_sync(~0u, sum, 31), per = (total + gridDim.x - 1) / gridDim.x;
        const int64_t u0 = min(total, blockIdx.x * per);
        Stretch x = {};
        if (u0 < total) {
            const int run = __popc(__ballot_sync(~0u, sum <= u0));
            int64_t at = __shfl_sync(~0u, sum - mine, run);
            int i = run * (kStrips / 32);
            while (at + m.strip[i] <= u0) at += m.strip[i++];
            int b = i * strip;
            for (;; ++b) {
                const int64_t n = seq_units_warp(a, b, lane);
                if (u0 < at + n) break;
                at += n;
            }
            const SeqView s = load_seq(a.bt, b, false);
            const int pairs = pairs_of(a, s);
            for (int t0 = 0;; t0 += 32) {
                const int64_t n = t0 + lane < pairs ? (int64_t)pair_units(a, s, t0 + lane) * a.c.n_heads : 0;
                int64_t up = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t y = __shfl_up_sync(~0u, up, o);
                    if (lane >= o) up += y;
                }
                const int skip = __popc(__ballot_sync(~0u, at + up <= u0));
                if (skip < 32) {
                    at += __shfl_sync(~0u, up - n, skip);
                    x.b = b, x.tile = t0 + skip;
                    break;
                }
                at += __shfl_sync(~0u, up, 31);
            }
            fill(a, s, x);
            x.head = (int)((u0 - at) / x.cnt);
            x.k = (int)((u0 - at) % x.cnt);
        }
        if (lane == 0) {
            m.first = x, m.total = total;
            ManyStart st = {x.b, x.tile, x.head, x.cnt, x.k, u0 < total, per};
            a.starts[blockIdx.x] = st;
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    const int64_t per = (m.total + gridDim.x - 1) / gridDim.x;
    const int64_t u0 = min(m.total, blockIdx.x * per), left = min(m.total, u0 + per) - u0;
    if (left > 0) {
        if (wid < 8) softmax_role<T, D>(a, m, m.first, left, blockIdx.x);
        else if (wid < 12) convert_role<T, D>(a, m, m.first, left);
        else if (lane == 0) {
            product_role<D>(a, m, m.first, left);
            commit(&m.drained);  // nothing may be in flight when tensor memory goes
            mbar_wait(&m.drained, 0);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (wid == 12) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(m.tmem));
    }
    if (tid == 0) a.gave_up[blockIdx.x] = m.gave_up;
}

constexpr int kJoinCols = 16;  // of D, a CTA of 256 rows

// CTA (w, y): adds up the 16 columns y of the stretch in which CTA w of the line began,
// if w is the first to begin inside it; the last CTAs write what sees nothing and the
// sequences' status.
template <typename T, int D>
__global__ void __launch_bounds__(kPair) k_kv_join_many(ManyArgs a) {
    const int tid = threadIdx.x;
    const int cuts = a.ctas * (D / kJoinCols);
    if (blockIdx.x < cuts) {
        const int w = blockIdx.x / (D / kJoinCols), y = blockIdx.x % (D / kJoinCols);
        const ManyStart st = a.starts[w];
        if (!st.there || st.k == 0) return;
        const int64_t us = w * st.per - st.k;  // the stretch's first unit
        if (us < (w - 1) * st.per) return;
        const int last = (int)((us + st.cnt - 1) / st.per);
        const SeqView s = load_seq(a.bt, st.b, false);
        const int r = st.tile * kPair + tid;
        if (r >= s.n * a.group) return;
        float top = -INFINITY, sum = 0.f, o[kJoinCols] = {};
        for (int v = w - 1; v <= last; ++v) {
            const float* part = a.part + ((int64_t)2 * v + (v * st.per >= us ? 0 : 1)) * (kPair * (D + 2));
            const float m = part[D * kPair + tid], l = part[(D + 1) * kPair + tid];
            const float now = fmaxf(top, m), ref = now == -INFINITY ? 0.f : now;
            const float f = exp2_approx(top - ref), g = exp2_approx(m - ref);
            sum = sum * f + l * g;
#pragma unroll
            for (int j = 0; j < kJoinCols; ++j) o[j] = o[j] * f + part[(y * kJoinCols + j) * kPair + tid] * g;
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
            a.lse[tok * a.q.n_heads + qh] = top == -INFINITY ? -INFINITY : (top - kManyLift + log2f(sum)) * 0.6931471805599453f;
        return;
    }
    bool late = false;
    for (int i = tid; i < a.ctas; i += kPair) late |= a.gave_up[i] != 0;
    late = __syncthreads_or(late);
    for (int b = blockIdx.x - cuts; b < a.bt.n_seqs; b += gridDim.x - cuts) {
        const SeqView s = load_seq(a.bt, b, false);
        const int pairs = pairs_of(a, s);
        if (pairs == 0 && a.few_rows > 0) continue;  // the other kernel's
        bool ok = s.st == MP_OK;
        int lo = INT32_MAX, hi = 0;
        for (int t = 0; t < pairs; ++t) {
            int g, n;
            pair_grans(a, s, t, g, n);
            if (n > 0) {
                lo = min(lo, g), hi = max(hi, g + n);
                continue;
            }
            for (int i = tid; i < kPair * a.c.n_heads; i += kPair) {
                const int r = t * kPair + i % kPair, head = i / kPair;
                if (r >= s.n * a.group) continue;
                const int64_t tok = s.lo + r / a.group;
                const int qh = head * a.group + r % a.group;
                T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
                for (int d = 0; d < D; ++d) dst[d] = from_f32<T>(0.f);
                if (a.lse != nullptr) a.lse[tok * a.q.n_heads + qh] = -INFINITY;
            }
        }
        if (hi > 0) {
            const int in = a.c.block_tokens / kGranule;
            for (int col = lo / in + tid; col <= (hi - 1) / in; col += kPair) {
                const int p = __ldg(a.bt.table + (int64_t)b * a.bt.max_blocks + col);
                ok &= p >= 0 && p < a.c.n_blocks;
            }
        }
        ok = !__syncthreads_or(!ok);
        if (tid == 0) a.status[b] = !ok ? MP_EINVAL : late ? MP_ETIMEOUT : MP_OK;
    }
}

template <typename T, int D>
cudaError_t many_as(const ManyArgs& a, cudaStream_t stream) {
    cudaError_t e = set_smem_limit((const void*)k_kv_attend_many<T, D>, sizeof(Smem<D>) + 16);
    if (e != cudaSuccess) return e;
    k_kv_attend_many<T, D><<<a.ctas, kThreads, sizeof(Smem<D>), stream>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    const int cuts = a.ctas * (D / kJoinCols);
    k_kv_join_many<T, D><<<cuts + std::min(a.bt.n_seqs, 1024), kPair, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace

size_t kv_many_part_bytes(const mp_kv_cache& c) {
    return sizeof(float) * 2 * kManyCtas * kPair * (size_t)(c.head_dim + 2);
}

cudaError_t launch_kv_many(const ManyArgs& a, cudaStream_t stream) {
    if (a.q.dtype == MP_F16) return a.c.head_dim == 64 ? many_as<__half, 64>(a, stream) : many_as<__half, 128>(a, stream);
    return a.c.head_dim == 64 ? many_as<__nv_bfloat16, 64>(a, stream) : many_as<__nv_bfloat16, 128>(a, stream);
}

}  // namespace mp
