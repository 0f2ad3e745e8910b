// kv_attend.cuh -- what the attention kernels over the caches share: barriers
// with bounded waits, bulk copies, and the scaling that both products use.
#pragma once

#include "kv.cuh"

namespace mp {

#ifdef MP_TEST_SPIN_CYCLES
constexpr long long kKvSpinCycles = MP_TEST_SPIN_CYCLES;
#else
constexpr long long kKvSpinCycles = 1ll << 31;  // about a second; a longer wait is a fault
#endif

// Weights are kept as 2^kLift times their value under the running maximum: as f16 they have
// all 11 bits down to 2^-28 of the largest, one less for each power of two below, none under 2^-38.
constexpr float kLift = 14.f;
// k_kv_attend_few over 4 bits keeps its reference until a score passes it by 2^5, so weights are 2^10 times theirs: 11 bits
// down to 2^-24 of the reference.
constexpr float kFewGrow = 5.f;
constexpr float lift_of(int bits) { return bits == 8 ? kLift : 10.f; }

__device__ __forceinline__ uint32_t smem_addr(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void mbar_init(uint64_t* bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_addr(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void fence_mbar_init() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_expect(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_addr(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_addr(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// Waits for the phase of that parity to end; false if it has not after kKvSpinCycles.
__device__ __forceinline__ bool mbar_wait(uint64_t* bar, uint32_t parity) {
    if (mbar_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (clock64() - t0 < kKvSpinCycles)
        if (mbar_try(bar, parity)) return true;
    return false;
}
// bytes (a multiple of 16, both addresses on 16-byte boundaries) into shared memory.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
                     smem_addr(dst)),
                 "l"(src), "r"(bytes), "r"(smem_addr(bar))
                 : "memory");
}

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 1 / x to 2^-23 of itself
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// lo in the low half
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// The power of two that brings a query row's largest magnitude to [2^14, 2^15), so
// that every bf16 and f16 row is an f16 row without loss (elements below 2^-28 of the
// largest aside).  1 for rows of zeros, infinities or NaN.
__device__ __forceinline__ float row_factor(float most) {
    const int e = (int)(__float_as_uint(most) >> 23);
    if (most == 0.f || e >= 255) return 1.f;
    return __uint_as_float((uint32_t)min(268 - e, 254) << 23);
}

// What a row's products with keys are multiplied by, as powers of two.  Finite, so that products of 0 stay 0 under the largest
// scales; where the bound is met, other scores over 4 bits are of 2^77 and more anyway.
__device__ __forceinline__ float row_unit(float scale, float factor) {
    return fminf(__fdiv_rn(scale * 1.4426950408889634f, factor), 0x1p122f);
}

// The scale of a block of values as the kernels use it: they divide by it and take its logarithm.  Sums of weights over
// scales stay finite: 2^28 tokens of weight 2^15 over 2^-84 make 2^127.  A smaller scale, 0 among them, counts as 0: its
// bytes are taken as zeros.
constexpr float kLeastValueScale = 0x1p-84f;
__device__ __forceinline__ float value_scale(float s) { return fmaxf(s, kLeastValueScale); }

// A row's log-sum from its reference top, at which weights are 2^lift, and their sum.  No weight at all: the row saw
// nothing; where no score was a number, neither is the sum.
__device__ __forceinline__ float log_sum(float top, float lift, float sum) {
    return sum == 0.f ? -INFINITY : (top - lift + log2f(sum)) * 0.6931471805599453f;
}

// What both kernels and the joining need of a call.
struct AttendArgs {
    mp_kv_cache c;
    mp_kv_batch bt;
    mp_tokens q, out;
    float* lse;
    int32_t* status;
    float scale;
    int32_t causal, window;
    int32_t group;     // query heads a cache head
    int32_t few_rows;  // sequences of at most this many rows (tokens x group) are k_kv_attend_few's, the others k_kv_attend_many's
    bool wide_q, wide_out;
#ifdef MP_TEST_HOOKS
    int64_t hold;  // a unit whose bytes never come, so that waits run out (-1: none)
#endif
};
// Test builds (MP_TEST_HOOKS) can hold a unit back: k_kv_attend_few's by its place on the line, k_kv_attend_many's by its
// number in the first CTA.
#ifdef MP_TEST_HOOKS
__device__ __forceinline__ bool test_held(const AttendArgs& a, int64_t unit) { return unit == a.hold; }
#else
__device__ __forceinline__ bool test_held(const AttendArgs&, int64_t) { return false; }
#endif
__device__ __forceinline__ bool seq_is_few(const AttendArgs& a, const SeqView& s) {
    return (int64_t)s.n * a.group <= a.few_rows;
}
// Granules [lo, hi) that the call's tokens of a sequence see.
__device__ __forceinline__ void seq_granules(const AttendArgs& a, const SeqView& s, int& lo, int& hi) {
    const int start = s.len - s.n;
    lo = a.window > 0 ? max(0, start - a.window + 1) / kGranule : 0;
    hi = s.n > 0 ? (s.len + kGranule - 1) / kGranule : lo;
}

// k_kv_attend_few: warps share the line of units; what is left to add up.
constexpr int kFewCtas = kSms;  // one an SM: its rings take most of the shared memory
struct FewWork {
    int64_t* base;     // [n_seqs + 1] first unit of each sequence, then units a warp
    float* part;       // [2 * warps][rows * (D + 2)]
    int32_t* gave_up;  // [warps]
};

// k_kv_attend_many: pairs of tiles of 128 rows, units of 128 tokens; where on the line a CTA began.
constexpr int kManyCtas = kSms;
constexpr int kPair = 256;
constexpr int kExtra = 3;           // units that a stretch costs beside its own: queries in, sums out
constexpr float kManyLift = 7.f;    // weights are at most 2^(8 + 7), and have 11 bits down to 2^-21 of their reference
struct ManyStart {
    int32_t b, tile, head, cnt, into;  // cnt: units of that (sequence, pair of tiles, head)
    int32_t there;
    int64_t per;  // length of a CTA's part
};
struct ManyWork {
    float* part;  // [2 * ctas][(D + 2) * 256]
    ManyStart* starts;
    int32_t* gave_up;  // [ctas]
};

// x / y for both below 2^63, mostly below 2^32: a 64-bit division takes a hundred instructions.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
    return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

// A kernel's launch may begin while the one before it in the stream ends; it touches memory after this.
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_begin() { asm volatile("griddepcontrol.launch_dependents;"); }
template <typename... K, typename... A>
inline cudaError_t launch_close(void (*kernel)(K...), int grid, int threads, size_t smem, cudaStream_t stream, A... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

size_t kv_many_part_bytes(const mp_kv_cache& c);
cudaError_t launch_kv_many(const AttendArgs& a, const ManyWork& w, cudaStream_t stream);   // over 8 bits
cudaError_t launch_kv4_many(const AttendArgs& a, const ManyWork& w, cudaStream_t stream);  // over 4

}  // namespace mp
