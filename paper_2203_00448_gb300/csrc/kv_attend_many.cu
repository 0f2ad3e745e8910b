// kv_attend_many.cu -- mp_kv_attend for sequences with many query rows (prompts, pieces
// of prompts): both products on the fifth-generation tensor cores.
//
// Rows are tokens x heads of a group, so a tile of 128 rows shares the cached head
// whatever the group.  A CTA works on two such tiles against the same 128 tokens (a unit),
// or, where there is one tile only, on two units in turn, whose sums are added up at the end.
// Warps 0-3 and 4-7, a thread a row: softmax of tile 0 and 1.  Warps 8-11: stored bytes
// become f16 operands in shared memory, exactly, two hardware conversions for 4 bytes
// (59 thread operations a clock and SM; spreading bytes with integer operations: 16).
// Warps 12 and 13: the products of tile 0 and 1.  Warp 14: the work list.  Scores (128 x 128
// f32) and sums (128 x D f32) of both tiles fill the 512 columns of tensor memory; weights
// go back as f16 over the scores they came from and are the left operand of the second
// product from there, so that the next scores wait for it to end.
//
// x_j = scale * q.k_j * log2(e) * key scale + log2(value scale) as in kv_attend.cu; a row's
// sums are rescaled only when its maximum has grown by 2^8, which weights as f16 (at most
// 2^15 here, down to 2^-24) leave room for.
//
// (sequence, pair of row tiles, head, unit) lie on a line that is cut evenly among 152 CTAs,
// so that causal rows, ragged prompts and a short piece over a long context all end
// together; a pair's beginning and end count as 3 units (a prompt of 8,000 tokens with 1: 671
// us, 2: 547, 3: 466, 5: 468).  What a CTA does not hold whole is added up by
// k_kv_join.
//
// Measured: 8,000 tokens, 32 heads over 8 of 128: 465 us, 1,128 TFLOP/s counted causally; 64
// tokens over 60,000 each for 8 sequences: 396 us, 1,270 TFLOP/s (cuBLAS bf16: 1,887); 8 tokens
// over 64 ragged contexts of up to 8,191: 208 us, 5 to 8 over four of 60,000: 185 (251 and 217 with one
// tile at work, before waits read the clock only where a first try fails, which took 1 to 2% off); the two ways of working
// cost prompts 1 to 2%.  A unit of both tiles takes
// 3,900 cycles where its 32 products take 2,080 on their own: the converting warps are busy or
// wait for loads through most of it, both tiles' products and both tiles' exponentials tend to
// come together, and products, operands and loads share one shared-memory pipe (about 70% busy).
// Dropped after measuring: the tiles taking turns at the exponentials, a quarter of the
// exponentials as polynomials, scores of 64 tokens in columns of their own, which the next
// scores need not wait for (466 -> 487 us: narrower products read the queries twice as often), two
// threads a row (1,038 -> 1,059), prefetches of the units to come into L2 (480 for 465), table entries
// and scales fetched by a warp of their own (473 for 464).
#include <algorithm>
#include <cmath>

#include "kv_attend.cuh"

namespace mp {
namespace {

constexpr int kRows = 128;      // of one tile
static_assert(kPair == 2 * kRows, "a pair of tiles");
constexpr int kTokens = 128;    // of a unit
constexpr int kGrans = kTokens / kGranule;
constexpr int kStages = 2;      // of keys and of values
constexpr int kScaleRing = 4;
constexpr int kLineRing = 4;
constexpr int kSoftmaxWarps = 8;
constexpr int kLineReaders = kSoftmaxWarps + 4 + 2;  // warps that read a stretch
constexpr int kThreads = 16 * 32;
// Registers a thread after the roles part: 256 x 176 + 128 x 112 + 128 x 48 = 512 x 128, the launch's.
// (D = 128 keeps 14 bytes a thread in memory all the same; 64 none.)
constexpr int kSoftmaxRegs = 176, kConvertRegs = 112, kProductRegs = 48;
constexpr int kUnitCycles = 1 << 16;  // a unit takes less by far
constexpr int kStrips = 1024;
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
// True in one lane of a whole warp, always the same one.
__device__ __forceinline__ bool elected() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
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

// n columns of this warp's 32 lanes of tensor memory, from and to registers.
__device__ __forceinline__ void ld32(uint32_t addr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(addr));
}
__device__ __forceinline__ void st16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(addr));
}
__device__ __forceinline__ void ld16(uint32_t addr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr));
}
__device__ __forceinline__ float max3(float x, float y, float z) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ void fma2(float& x, float& y, float m, float o) {  // x, y = x m + o, y m + o
    asm("{\n\t.reg .b64 v, w, z;\n\tmov.b64 v, {%0, %1};\n\tmov.b64 w, {%2, %2};\n\tmov.b64 z, {%3, %3};\n\t"
        "fma.rn.f32x2 v, v, w, z;\n\tmov.b64 {%0, %1}, v;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(m), "f"(o));
}
__device__ __forceinline__ void add2(float& x, float& y, float u, float v) {  // x, y = x + u, y + v
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%0, %1};\n\tmov.b64 q, {%2, %3};\n\tadd.rn.f32x2 p, p, q;\n\t"
        "mov.b64 {%0, %1}, p;\n\t}"
        : "+f"(x), "+f"(y)
        : "f"(u), "f"(v));
}
template <int kRegs>
__device__ __forceinline__ void more_regs() {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegs));
}
template <int kRegs>
__device__ __forceinline__ void fewer_regs() {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegs));
}

// A stretch of the line inside one (sequence, pair of row tiles, head).
struct Stretch {
    int b, tile, head;
    int cnt, k;              // units of the whole, the first of this stretch
    int units;               // of this stretch; 0: the CTA has no more
    int tiles;               // 1 or 2 of the pair have rows; 1: both work on these, tile i on the units i, i + 2, ..
    int first;               // of its CTA
    int first_gran, grans;   // granules that the pair's rows see
    int rows;                // of the sequence and head
    int len, start;          // tokens held; position of the call's first
    int64_t row;             // its first row of the token arrays
};

__device__ __forceinline__ int pairs_of(const AttendArgs& a, const SeqView& s) {
    if (s.st != MP_OK || seq_is_few(a, s)) return 0;
    return (s.n * a.group + kPair - 1) / kPair;
}
__device__ __forceinline__ void pair_grans(const AttendArgs& a, const SeqView& s, int tile, int& lo, int& n) {
    const int start = s.len - s.n, rows = s.n * a.group;
    const int p0 = start + tile * kPair / a.group, p1 = start + (min(rows, (tile + 1) * kPair) - 1) / a.group;
    const int past = a.causal ? min(s.len, max(p1 + 1, 0)) : s.len;
    lo = a.window > 0 ? max(0, p0 - a.window + 1) / kGranule : 0;
    n = max(0, (past + kGranule - 1) / kGranule - lo);
}
__device__ __forceinline__ int units_of(int grans) { return (grans + kGrans - 1) / kGrans; }
// Length on the line: its units and what beginning and ending a pair costs beside them.
__device__ __forceinline__ int pair_length(const AttendArgs& a, const SeqView& s, int tile) {
    int lo, n;
    pair_grans(a, s, tile, lo, n);
    return n > 0 ? units_of(n) + kExtra : 0;
}
// Length of a sequence; a warp's lanes take its pairs in turn.
__device__ __forceinline__ int64_t seq_length(const AttendArgs& a, int b, int lane) {
    const SeqView s = load_seq(a.bt, b, false);
    const int pairs = pairs_of(a, s);
    int64_t n = 0;
    for (int i = lane; i < pairs; i += 32) n += pair_length(a, s, i);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(~0u, n, o);
    return n * a.c.n_heads;
}
__device__ __forceinline__ void fill(const AttendArgs& a, const SeqView& s, Stretch& x) {
    pair_grans(a, s, x.tile, x.first_gran, x.grans);
    x.cnt = units_of(x.grans);
    x.rows = s.n * a.group;
    x.tiles = x.rows - x.tile * kPair > kRows ? 2 : 1;
    x.len = s.len, x.start = s.len - s.n, x.row = s.lo;
}
// The next pair or head on the line; false at its end.
__device__ __forceinline__ bool advance(const AttendArgs& a, Stretch& x) {
    if (++x.head < a.c.n_heads) return true;
    x.head = 0;
    ++x.tile;
    SeqView s;
    s.lo = x.row, s.len = x.len, s.n = x.len - x.start, s.st = MP_OK;
    for (;;) {
        const int pairs = pairs_of(a, s);
        for (; x.tile < pairs; ++x.tile) {
            fill(a, s, x);
            if (x.cnt > 0) return true;
        }
        ++x.b, x.tile = 0;
        if (x.b >= a.bt.n_seqs) return false;
        s = load_seq(a.bt, x.b, false);
    }
}

// 8 values of 16 bits from and to memory that is aligned to one.
template <typename T>
__device__ __forceinline__ uint4 load_narrow(const T* p) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint16_t* e = reinterpret_cast<const uint16_t*>(p) + 2 * i;
        w[i] = (uint32_t)e[0] | (uint32_t)e[1] << 16;
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <typename T>
__device__ __forceinline__ void store_narrow(T* p, uint4 v) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint16_t* e = reinterpret_cast<uint16_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) e[2 * i] = (uint16_t)w[i], e[2 * i + 1] = (uint16_t)(w[i] >> 16);
}

template <int D>
struct Smem {
    uint8_t q[2][kRows * D * 2];
    uint8_t k[kStages][kTokens * D * 2];
    uint8_t v[kStages][kTokens * D * 2];
    int64_t strip[kStrips];
    float scales[kScaleRing][3][kGrans];  // key scale, log2 of the value scale, 1 / value scale
    float tops[2][kRows], sums[2][kRows];  // of rows that both tiles worked on
    uint64_t posted, added;                // ... are there; ... have been added up
    uint64_t q_full[2], s_full[2], p_full[2], o_done[2], k_full[kStages], k_empty[kStages], v_full[kStages],
        v_empty[kStages], drained, line_full[kLineRing], line_empty[kLineRing],
        scales_full[kScaleRing];
    Stretch line[kLineRing];  // the CTA's stretches as line_role lays them out
    Stretch first;
    int64_t length;  // of the CTA's part of the line
    int into;        // where in its first pair and head it begins, on the line
    uint32_t tmem;
    int gave_up;
};

// Waits until the phase ends; false if some wait of the CTA has given up, which one does after kKvSpinCycles (by the
// clock: a try may take thousands of cycles).
__device__ __forceinline__ bool await(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
    static_assert(kKvSpinCycles < 1ll << 32, "the clock's low word tells");
    if (mbar_try(bar, parity)) return true;
    const uint32_t t0 = clock();
    while (!mbar_try(bar, parity))
        if (*gave_up || (uint32_t)clock() - t0 > (uint32_t)kKvSpinCycles) {
            *gave_up = 1;
            return false;
        }
    return true;
}
// ... by all lanes of a warp, with one answer for all.
__device__ __forceinline__ bool await_warp(uint64_t* bar, uint32_t parity, volatile int* gave_up) {
    return __all_sync(~0u, await(bar, parity, gave_up));
}

// ... for as long as a stretch of that many units may take.
__device__ __forceinline__ bool await_stretch(uint64_t* bar, uint32_t parity, int units, volatile int* gave_up) {
    const long long t0 = clock64();
    while (!mbar_try(bar, parity)) {
        if (*gave_up) return false;
        if (clock64() - t0 > kKvSpinCycles + (long long)units * kUnitCycles) {
            *gave_up = 1;
            return false;
        }
        __nanosleep(100);
    }
    return true;
}

constexpr uint32_t kScoreCol = 0, kSumCol = 256;  // of tile 0; tile 1 has + 128 and + D

// One thread walks the CTA's part of the line ahead of the roles.
template <int D>
__device__ void line_role(const AttendArgs& a, Smem<D>& m) {
    Stretch x = m.first;
    int64_t left = m.length;
    int into = m.into, longest = 0;
    x.first = 1;
#pragma unroll 1
    for (int seg = 0;; ++seg) {
        // units come last on a pair's part of the line
        x.units = 0;
        while (left > 0) {
            const int span = (int)min((int64_t)(x.cnt + kExtra - into), left);
            x.k = max(0, into - kExtra);
            x.units = max(0, into + span - kExtra) - x.k;
            left -= span;
            if (x.units > 0) break;
        }
        if (!await_stretch(&m.line_empty[seg % kLineRing], (seg / kLineRing & 1) ^ 1, longest, &m.gave_up)) return;
        longest = max(longest, x.units);
        m.line[seg % kLineRing] = x;
        mbar_arrive(&m.line_full[seg % kLineRing]);
        if (x.units == 0) return;
        x.first = into = 0;
        if (left > 0 && !advance(a, x)) left = 0;
    }
}
template <int D>
__device__ __forceinline__ void release(Smem<D>& m, int seg) {
    __syncwarp();
    if (threadIdx.x % 32 == 0) mbar_arrive(&m.line_empty[seg % kLineRing]);
}

template <typename T, int D>
__device__ void convert_role(const AttendArgs& a, Smem<D>& m) {
    constexpr int kLoads = kTokens * D / 16 / 128;     // 16-byte loads a thread, of either array
    constexpr int kPerGran = kGranule * D / 16 / 128;  // ... of which a granule is this many, 1 or 2
    const int tid = threadIdx.x - kSoftmaxWarps * 32;
    uint4 kr[kLoads], vr[kLoads];
    const int lane = tid % 32, mine = lane % kGrans, per = a.c.block_tokens / kGranule;
    int64_t at[kGrans];  // the granules of the unit at hand: where they are, -1 past the last
    int seg = 0, u = 0, had = 0;
    float ks = 0.f, vs = 1.f;
    // a unit's table entries are read a unit ahead, a granule a lane
    int page = 0, in_page = 0, head = 0, next_had = 0;
    bool more = true, there = false;  // that unit is one; it has this granule
    auto look_up = [&]() {
        if (u == 0 && !await_warp(&m.line_full[seg % kLineRing], seg / kLineRing & 1, &m.gave_up)) return false;
        const Stretch& x = m.line[seg % kLineRing];
        more = x.units > 0;
        if (!more) return true;
        const int g = (x.k + u) * kGrans + mine, gran = x.first_gran + g, col = gran / per;
        in_page = gran - col * per, head = x.head, there = g < x.grans;
        if (there) page = __ldg(a.bt.table + (int64_t)x.b * a.bt.max_blocks + col);  // looked at a unit later
        next_had = x.len - (gran - mine) * kGranule;  // tokens of the unit that are held
        if (++u == x.units) {
            release(m, seg);
            ++seg, u = 0;
        }
        return true;
    };
    auto locate = [&]() {
        int64_t here = -1;
        ks = 0.f, vs = 1.f;
        if (there) {
            if (page < 0 || page >= a.c.n_blocks) page = 0;  // k_kv_join reports it
            here = block_byte(a.c, page, head) + in_page * (kGranule * D);
            const int64_t sc = (int64_t)page * a.c.n_heads + head;
            ks = __ldg(a.c.k_scale + sc), vs = __ldg(a.c.v_scale + sc);
        }
#pragma unroll
        for (int i = 0; i < kGrans; ++i) at[i] = __shfl_sync(~0u, here, i);
        had = next_had;
    };
    auto load = [&](const uint8_t* pool, uint4* r) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            r[i] = at[i / kPerGran] < 0 ? make_uint4(0, 0, 0, 0)
                                        : __ldg(reinterpret_cast<const uint4*>(pool + at[i / kPerGran]) +
                                                (i % kPerGran) * 128 + tid);
    };
    auto widen = [](const uint4& w, uint4* dst) {
        uint4 lo, hi;
        e4m3_to_f16(w.x, lo.x, lo.y), e4m3_to_f16(w.y, lo.z, lo.w);
        e4m3_to_f16(w.z, hi.x, hi.y), e4m3_to_f16(w.w, hi.z, hi.w);
        dst[0] = lo, dst[8] = hi;
    };
    if (!look_up() || !more) return;
    locate();
    load(a.c.k, kr);
    if (!look_up()) return;
#pragma unroll 1
    for (int it = 0;; ++it) {
        const int st = it % kStages, held = had;
        const uint32_t nothing = __ballot_sync(~0u, vs < kLeastValueScale);  // bit g: granule g's values count as zeros
        const uint32_t empty = (it / kStages & 1) ^ 1;
        load(a.c.v, vr);
        if (!await_warp(&m.k_empty[st], empty, &m.gave_up)) return;
        if (tid < kGrans) {
            // the slot's last readers are done: this stage's last scores were issued after sums that had
            // waited for the weights of the unit that had the slot
            float(*sc)[kGrans] = m.scales[it % kScaleRing];
            const float s = value_scale(vs);
            sc[0][tid] = ks, sc[1][tid] = log2f(s), sc[2][tid] = __fdiv_rn(1.f, s);
        }
        __syncwarp();
        if (tid == 0) mbar_arrive(&m.scales_full[it % kScaleRing]);
        // stored tiles [token / 8][D / 16][8][16] become f16 tiles [token / 8][D / 8][8][8]
        uint4* to = reinterpret_cast<uint4*>(m.k[st]) + (tid / 8) * 16 + tid % 8;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) widen(kr[i], to + i * 256);
        fence_smem();
        if (!(blockIdx.x == 0 && tid == 0 && test_held(a, it))) mbar_arrive(&m.k_full[st]);
        const bool again = more;
        if (again) {
            locate();
            load(a.c.k, kr);
            if (!look_up()) return;
        }
        if (!await_warp(&m.v_empty[st], empty, &m.gave_up)) return;
        // stored tiles [granule][D / 8][2][8][16] become [granule][D / 8][4][8][8]
        to = reinterpret_cast<uint4*>(m.v[st]) + (tid / 8) * 16 + tid % 8;
        if (held < kTokens || nothing) {  // bytes behind the last token mean nothing, NaN among them
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                const int left_here = nothing >> (i / kPerGran) & 1 ? 0 : held - (i / kPerGran * kGranule + (tid / 8 % 2) * 16);
                uint32_t* p = reinterpret_cast<uint32_t*>(&vr[i]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int n = left_here - 4 * j;
                    p[j] &= n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1;
                }
            }
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) widen(vr[i], to + i * 256);
        fence_smem();
        mbar_arrive(&m.v_full[st]);
        if (!again) return;
    }
}

// One warp a tile, a lane of which issues: sums of a unit as its weights come, then the
// next unit's scores over them.
template <int D>
__device__ void product_role(Smem<D>& m, int tile) {
    constexpr uint32_t kScores = product_of(kRows, kTokens), kSums = product_of(kRows, D);
    constexpr uint32_t kStep = kTokens * D * 2 >> 4;  // between stages and between tiles, in descriptors
    const uint32_t sc = __shfl_sync(~0u, m.tmem, 0) + kScoreCol + tile * 128;
    const uint32_t su = __shfl_sync(~0u, m.tmem, 0) + kSumCol + tile * D;
    const uint64_t q = operand(smem_addr(m.q[tile]), 128, D * 16);
    const uint64_t k0 = operand(smem_addr(m.k[0]), 128, D * 16), v0 = operand(smem_addr(m.v[0]), 128, 512);
    uint32_t it = 0, mine = 0, asked = 0;  // units of the CTA; units and stretches of this tile
    int seg = 0;
#pragma unroll 1
    for (;;) {
        if (!await_warp(&m.line_full[seg % kLineRing], seg / kLineRing & 1, &m.gave_up)) return;
        const int units = m.line[seg % kLineRing].units;
        const int turns = m.line[seg % kLineRing].tiles == 1, begin = turns ? tile : 0;  // its first unit
        release(m, seg++);
        if (units == 0) return;
        if (begin < units && !await_warp(&m.q_full[tile], asked++ & 1, &m.gave_up)) return;
#pragma unroll 1
        for (int u = 0; u < units; ++u, ++it) {
            const uint32_t st = it & 1, round = it >> 1 & 1;
            if (!await_warp(&m.k_full[st], round, &m.gave_up)) return;
            if (turns & (u ^ tile)) {
                // the other tile's unit: this one gives its part of the stages back as they fill
                if (elected()) mbar_arrive(&m.k_empty[st]);
                if (!await_warp(&m.v_full[st], round, &m.gave_up)) return;
                if (elected()) mbar_arrive(&m.v_empty[st]);
                continue;
            }
            // scores overwrite the weights that the product before reads: products of different sums are not
            // ordered among themselves
            if (mine > 0 && !await_warp(&m.o_done[tile], (mine - 1) & 1, &m.gave_up)) return;
            fence_after();
            if (elected()) {
                const uint64_t k = k0 + st * kStep;
#pragma unroll
                for (int s = 0; s < D / 16; ++s) mma_ss(sc, q + s * 16, k + s * 16, kScores, s > 0);
                commit(&m.s_full[tile]);
                commit(&m.k_empty[st]);
            }
            __syncwarp();
            if (!await_warp(&m.v_full[st], round, &m.gave_up)) return;
            if (!await_warp(&m.p_full[tile], mine & 1, &m.gave_up)) return;
            fence_after();
            if (elected()) {
                const uint64_t v = v0 + st * kStep;
#pragma unroll
                for (int s = 0; s < kTokens / 16; ++s)
                    mma_ts(su, sc + s * 8, v + (s / 2) * (kGranule * D * 2 >> 4) + (s % 2) * 16, kSums,
                           u > begin || s > 0);
                commit(&m.o_done[tile]);
                commit(&m.v_empty[st]);
            }
            __syncwarp();
            ++mine;
        }
    }
}

// 4 warps a tile, a thread a row.
template <typename T, int D>
__device__ void softmax_role(const AttendArgs& a, const ManyWork& work, Smem<D>& m) {
    const int tile = threadIdx.x / 128, in_tile = threadIdx.x % 128, warp = in_tile / 32, lane = threadIdx.x % 32;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16;
    const uint32_t sc = m.tmem + lanes + kScoreCol + tile * 128, su = m.tmem + lanes + kSumCol + tile * D;
    uint32_t it = 0, n = 0, shared = 0;  // units of the CTA, of this tile; stretches that both tiles summed
    float top = -INFINITY, sum = 0.f;
    bool pending = false;
#pragma unroll 1
    for (int seg = 0;; ++seg) {
        // a stretch's queries go in before the sums of the one before it come out
        if (!await_warp(&m.line_full[seg % kLineRing], seg / kLineRing & 1, &m.gave_up)) return;
        const Stretch& x = m.line[seg % kLineRing];
        const Stretch& done = m.line[(seg + kLineRing - 1) % kLineRing];
        const int units = x.units;
        const bool turns = x.tiles == 1;  // the tiles take the units in turn
        const int begin = turns ? tile : 0, first_row = x.tile * kPair + (turns ? 0 : tile * kRows);
        const bool mine = begin < units;
        float unit = 0.f;  // what the row's scores are to be multiplied by
        if (mine) {
            // as they are into their places, 8 rows x 4 chunks of 16 bytes a step; then a thread its row
            uint4* const q = reinterpret_cast<uint4*>(m.q[tile]);
#pragma unroll 1
            for (int g = 0; g < 4; ++g) {
                const int at = warp * 32 + g * 8 + lane / 4, row = first_row + at;
                const T* p = static_cast<const T*>(a.q.data) + (x.row + row / a.group) * a.q.token_stride +
                             (x.head * a.group + row % a.group) * a.q.head_stride + lane % 4 * 8;
                uint4* to = q + (at / 8 * (D / 8) + lane % 4) * 8 + at % 8;
                if (row >= x.rows) {
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) to[i * 32] = make_uint4(0, 0, 0, 0);
                } else if (a.wide_q) {
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(to + i * 32)), "l"(p + i * 32)
                                     : "memory");
                } else {
#pragma unroll 1
                    for (int i = 0; i < D / 32; ++i) to[i * 32] = load_narrow(p + i * 32);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            __syncwarp();
            uint4* const row = q + in_tile / 8 * D + in_tile % 8;
            float most = 0.f;
#pragma unroll 2
            for (int i = 0; i < D / 8; ++i) {
                const uint4 v = row[i * 8];
                const T* e = reinterpret_cast<const T*>(&v);
#pragma unroll
                for (int j = 0; j < 8; j += 2) most = max3(most, fabsf(to_f32(e[j])), fabsf(to_f32(e[j + 1])));
            }
            const float f = row_factor(most);
            unit = __fdiv_rn(a.scale * 1.4426950408889634f, f);
#pragma unroll 2
            for (int i = 0; i < D / 8; ++i) {
                const uint4 v = row[i * 8];
                const T* e = reinterpret_cast<const T*>(&v);
                uint4 o;
                o.x = pack_f16(to_f32(e[0]) * f, to_f32(e[1]) * f), o.y = pack_f16(to_f32(e[2]) * f, to_f32(e[3]) * f);
                o.z = pack_f16(to_f32(e[4]) * f, to_f32(e[5]) * f), o.w = pack_f16(to_f32(e[6]) * f, to_f32(e[7]) * f);
                row[i * 8] = o;
            }
            fence_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&m.q_full[tile]);
        }
        if (pending) {
            if (!await_warp(&m.o_done[tile], (n - 1) & 1, &m.gave_up)) return;
            fence_after();
            const bool whole = done.units == done.cnt;
            const bool both = done.tiles == 1 && done.units > 1;
            const int at = done.tiles == 1 ? in_tile : threadIdx.x, dr = done.tile * kPair + at;
            const int64_t tok = done.row + dr / a.group;
            const int qh = done.head * a.group + dr % a.group;
            float f = 1.f, g = 0.f;  // of tile 0's and tile 1's sums
            if (both) {
                // both tiles have sums of the same rows, in the same lanes of tensor memory: each adds up half of the columns
                m.tops[tile][in_tile] = top, m.sums[tile][in_tile] = sum;
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.posted);
                if (!await_warp(&m.posted, shared & 1, &m.gave_up)) return;
                fence_after();
                const float t0 = m.tops[0][in_tile], t1 = m.tops[1][in_tile];
                top = fmaxf(t0, t1);
                const float ref = top == -INFINITY ? 0.f : top;
                f = exp2_approx(t0 - ref), g = exp2_approx(t1 - ref);
                sum = m.sums[0][in_tile] * f + m.sums[1][in_tile] * g;
            }
            const float inv = sum == 0.f ? 0.f : __fdiv_rn(1.f, sum);
            // stretches that are not whole: at most the CTA's first and its last
            float* part = work.part + ((int64_t)2 * blockIdx.x + (done.first ? 0 : 1)) * (kPair * (D + 2)) + at;
            T* dst = static_cast<T*>(a.out.data) + tok * a.out.token_stride + qh * a.out.head_stride;
#pragma unroll 1
            for (int c = both ? tile * (D / 64) : 0; c < (both ? (tile + 1) * (D / 64) : D / 32); ++c) {
                uint32_t o[32];
                ld32((both ? m.tmem + lanes + kSumCol : su) + c * 32, o);
                wait_ld();
                if (both) {
                    uint32_t o1[32];
                    ld32(m.tmem + lanes + kSumCol + D + c * 32, o1);
                    wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        o[j] = __float_as_uint(__uint_as_float(o[j]) * f + __uint_as_float(o1[j]) * g);
                }
                if (whole) {
                    if (dr < done.rows) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(o[j]) * inv;
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            Pack<T, 8> o8;
#pragma unroll
                            for (int i = 0; i < 8; ++i) o8.x[i] = from_f32<T>(v[j * 8 + i]);
                            const uint4 w4 = *reinterpret_cast<const uint4*>(&o8);
                            if (a.wide_out) reinterpret_cast<uint4*>(dst + c * 32)[j] = w4;
                            else store_narrow(dst + c * 32 + j * 8, w4);
                        }
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 32; ++j) part[(c * 32 + j) * kPair] = __uint_as_float(o[j]);
                }
            }
            if (both && tile == 1) {
            } else if (!whole) {
                part[D * kPair] = top;
                part[(D + 1) * kPair] = sum;
            } else if (dr < done.rows && a.lse != nullptr) {
                a.lse[tok * a.q.n_heads + qh] = log_sum(top, kManyLift, sum);
            }
            if (both) {
                // neither tile's next sums go over these before both have read them
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.added);
                if (!await_warp(&m.added, shared++ & 1, &m.gave_up)) return;
                fence_after();
            }
            pending = false;
        }
        if (seg > 0) release(m, seg - 1);
        if (units == 0) return;
        if (mine) {
            const int r = first_row + in_tile;
            // units from one of the tile's to its next; read again where it is needed, for registers are short
            auto step = [&]() { return 3 - *(const volatile int*)&x.tiles; };
            const int pos = x.start + r / a.group;
            const int first_token = (x.first_gran + (x.k + begin) * kGrans) * kGranule;
            // seen: [lo, hi) counted from the unit's first score
            int hi = (r >= x.rows ? 0 : a.causal ? min(x.len, max(pos + 1, 0)) : x.len) - first_token;
            int lo = (a.window > 0 ? pos - a.window + 1 : 0) - first_token;
            top = -INFINITY, sum = 0.f;
#pragma unroll 1
            for (int u = begin; u < x.units; ++n) {
                const float(*scale)[kGrans] = m.scales[(it + u) % kScaleRing];
                // a tile that sat stretches out is ahead of the ring, where an old phase looks like the one to come:
                // its first scores say that the unit is at hand
                const bool opening = u < step();
                if (opening && !await_warp(&m.s_full[tile], n & 1, &m.gave_up)) return;
                if (!await_warp(&m.scales_full[(it + u) % kScaleRing], (it + u) / kScaleRing & 1, &m.gave_up)) return;
                const bool edge = __any_sync(~0u, hi < kTokens || lo > 0);
                float mul[kGrans], add[kGrans], inverse[kGrans];
#pragma unroll
                for (int c = 0; c < kGrans; ++c) {
                    mul[c] = fmaxf(unit * scale[0][c], 0x1p-126f);  // not 0: what is not seen stays -inf
                    add[c] = scale[1][c], inverse[c] = scale[2][c];
                }
                if (!opening && !await_warp(&m.s_full[tile], n & 1, &m.gave_up)) return;
                fence_after();
                uint32_t raw[kTokens];
                float* s = reinterpret_cast<float*>(raw);
#pragma unroll
                for (int c = 0; c < kGrans; ++c) ld32(sc + c * 32, raw + c * 32);
                wait_ld();
                if (edge) {
#pragma unroll
                    for (int c = 0; c < kGrans; ++c) {
                        const int h = hi - c * 32, l = lo - c * 32;
                        const uint32_t seen = (h >= 32 ? ~0u : h <= 0 ? 0u : (1u << h) - 1) &
                                              (l <= 0 ? ~0u : l >= 32 ? 0u : ~0u << l);
                        if (__any_sync(~0u, seen != ~0u)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(seen >> j & 1)) s[c * 32 + j] = -INFINITY;
                        }
                    }
                }
                float most = -INFINITY;
#pragma unroll
                for (int c = 0; c < kGrans; ++c) {
                    float b0 = max3(s[c * 32], s[c * 32 + 1], s[c * 32 + 2]);
                    float b1 = max3(s[c * 32 + 3], s[c * 32 + 4], s[c * 32 + 5]);
#pragma unroll
                    for (int j = 6; j < 30; j += 4) {
                        b0 = max3(b0, s[c * 32 + j], s[c * 32 + j + 1]);
                        b1 = max3(b1, s[c * 32 + j + 2], s[c * 32 + j + 3]);
                    }
                    b0 = max3(b0, s[c * 32 + 30], s[c * 32 + 31]);
                    most = fmaxf(most, fmaf(fmaxf(b0, b1), mul[c], add[c]));
                }
                const bool grows = most > top + kGrow;
                const float now = grows ? most : top;
                const float fade = top == -INFINITY ? 0.f : exp2_approx(top - now);
                const float ref = now == -INFINITY ? 0.f : now - kManyLift;
                sum *= fade;
                top = now;
#pragma unroll
                for (int c = 0; c < kGrans; ++c) {
                    const float off = add[c] - ref;
                    float p0 = 0.f, p1 = 0.f, p2 = 0.f, p3 = 0.f;
                    uint32_t p[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float &e0 = s[c * 32 + 2 * j], &e1 = s[c * 32 + 2 * j + 1];
                        fma2(e0, e1, mul[c], off);
                        e0 = exp2_approx(e0), e1 = exp2_approx(e1);
                        if (j % 2 == 0) add2(p0, p1, e0, e1);
                        else add2(p2, p3, e0, e1);
                        p[j] = pack_f16(e0, e1);
                    }
                    sum = fmaf((p0 + p1) + (p2 + p3), inverse[c], sum);
                    // over scores that have been read: 16 columns for 32
                    st16(sc + c * 16, p);
                }
                if (__any_sync(~0u, grows) && u >= step()) {
                    if (!await_warp(&m.o_done[tile], (n - 1) & 1, &m.gave_up)) return;
                    fence_after();
#pragma unroll 1
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        ld16(su + c * 16, o);
                        wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * fade);
                        st16(su + c * 16, o);
                    }
                }
                wait_st();
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&m.p_full[tile]);
                const int next = step();
                u += next, hi -= next * kTokens, lo -= next * kTokens;
            }
            pending = true;
        }
        it += units;
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 1) k_kv_attend_many(AttendArgs a, ManyWork work) {
    extern __shared__ __align__(1024) uint8_t dyn[];
    Smem<D>& m = *reinterpret_cast<Smem<D>*>(dyn);
    const int tid = threadIdx.x, lane = tid % 32, wid = tid / 32;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&m.q_full[i], kSoftmaxWarps / 2), mbar_init(&m.s_full[i], 1);
            mbar_init(&m.p_full[i], kSoftmaxWarps / 2), mbar_init(&m.o_done[i], 1);
        }
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&m.k_full[i], 128), mbar_init(&m.k_empty[i], 2);
            mbar_init(&m.v_full[i], 128), mbar_init(&m.v_empty[i], 2);
        }
        for (int i = 0; i < kScaleRing; ++i) mbar_init(&m.scales_full[i], 1);
        for (int i = 0; i < kLineRing; ++i) mbar_init(&m.line_full[i], 1), mbar_init(&m.line_empty[i], kLineReaders);
        mbar_init(&m.drained, 2), mbar_init(&m.posted, kSoftmaxWarps), mbar_init(&m.added, kSoftmaxWarps);
        m.gave_up = 0;
        fence_mbar_init();
    }
    if (wid == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&m.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    after_previous();
    let_next_begin();
    // the line: strips of sequences, a warp a strip
    const int strip = (a.bt.n_seqs + kStrips - 1) / kStrips, strips = (a.bt.n_seqs + strip - 1) / strip;
#pragma unroll 1
    for (int i = wid; i < strips; i += kThreads / 32) {
        int64_t n = 0;
#pragma unroll 1
        for (int b = i * strip; b < min((i + 1) * strip, a.bt.n_seqs); ++b) n += seq_length(a, b, lane);
        if (lane == 0) m.strip[i] = n;
    }
    __syncthreads();
    if (wid == 0) {
        // the strip, the sequence and the pair in which this CTA's part begins
        const int each = (strips + 31) / 32;
        int64_t mine = 0;
#pragma unroll 1
        for (int i = lane * each; i < min((lane + 1) * each, strips); ++i) mine += m.strip[i];
        int64_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += y;
        }
        const int64_t total = __shfl_sync(~0u, sum, 31);
        const int64_t per = total < INT32_MAX ? ((uint32_t)total + gridDim.x - 1) / gridDim.x
                                              : (total + gridDim.x - 1) / gridDim.x;
        const int64_t u0 = min(total, blockIdx.x * per);
        Stretch x = {};
        int into = 0;
        if (u0 < total) {
            const int run = __popc(__ballot_sync(~0u, sum <= u0));
            int64_t at = __shfl_sync(~0u, sum - mine, run);
            int i = run * each;
#pragma unroll 1
            while (at + m.strip[i] <= u0) at += m.strip[i++];
            int b = i * strip;
#pragma unroll 1
            while (strip > 1) {
                const int64_t n = seq_length(a, b, lane);
                if (u0 < at + n) break;
                at += n, ++b;
            }
            const SeqView s = load_seq(a.bt, b, false);
            const int pairs = pairs_of(a, s);
#pragma unroll 1
            for (int t0 = 0;; t0 += 32) {
                const int64_t n = t0 + lane < pairs ? (int64_t)pair_length(a, s, t0 + lane) * a.c.n_heads : 0;
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
            x.head = (int)((uint32_t)(u0 - at) / (uint32_t)(x.cnt + kExtra));
            into = (int)((uint32_t)(u0 - at) % (uint32_t)(x.cnt + kExtra));
        }
        if (lane == 0) {
            m.first = x, m.length = min(total, u0 + per) - u0, m.into = into;
            const ManyStart st = {x.b, x.tile, x.head, x.cnt, into, u0 < total, per};
            work.starts[blockIdx.x] = st;
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (wid < kSoftmaxWarps) {
        more_regs<kSoftmaxRegs>();
        softmax_role<T, D>(a, work, m);
        wait_st();  // a tile that gave up may have weights on their way, and tensor memory goes below
    } else if (wid < kSoftmaxWarps + 4) {
        fewer_regs<kConvertRegs>();
        convert_role<T, D>(a, m);
    } else {
        fewer_regs<kProductRegs>();
        const int role = wid - kSoftmaxWarps - 4;
        if (role < 2) {
            product_role<D>(m, role);
            __syncwarp();
            if (elected()) commit(&m.drained);  // nothing may be in flight when tensor memory goes
            __syncwarp();
            mbar_wait(&m.drained, 0);
        } else if (role == 2 && lane == 0) {
            line_role<D>(a, m);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (wid == 0) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(m.tmem));
    }
    if (tid == 0) work.gave_up[blockIdx.x] = m.gave_up;
}

template <typename T, int D>
cudaError_t many_as(const AttendArgs& a, const ManyWork& w, cudaStream_t stream) {
    cudaError_t e = set_smem_limit((const void*)k_kv_attend_many<T, D>, sizeof(Smem<D>));
    if (e != cudaSuccess) return e;
    return launch_close(k_kv_attend_many<T, D>, kManyCtas, kThreads, sizeof(Smem<D>), stream, a, w);
}

}  // namespace

size_t kv_many_part_bytes(const mp_kv_cache& c) {
    return sizeof(float) * 2 * kManyCtas * kPair * (size_t)(c.head_dim + 2);
}

cudaError_t launch_kv_many(const AttendArgs& a, const ManyWork& w, cudaStream_t stream) {
    if (a.q.dtype == MP_F16)
        return a.c.head_dim == 64 ? many_as<__half, 64>(a, w, stream) : many_as<__half, 128>(a, w, stream);
    return a.c.head_dim == 64 ? many_as<__nv_bfloat16, 64>(a, w, stream) : many_as<__nv_bfloat16, 128>(a, w, stream);
}

}  // namespace mp
