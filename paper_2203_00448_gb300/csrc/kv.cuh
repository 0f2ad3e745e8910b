// kv.cuh -- what the key/value cache kernels share (sm_103a): the stored layout,
// the sequences' checks and e4m3 conversions.
#pragma once

#include <cstdint>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "launch.h"
#include "memplan.h"

namespace mp {

// Both arrays are stored in granules of 32 tokens of 32 * D bytes: a block is
// whole granules, so kernels walk granules whatever the block size.
constexpr int kGranule = 32;

// GB300's SMs.  Grids that scratch is laid out for take this number, for the size of scratch is asked for without a
// device; a device with fewer runs the same CTAs in turn.
constexpr int kSms = 152;

// Byte of key (t, d) and of value (t, d) inside one block and head.
template <int D>
__device__ __forceinline__ int key_byte(int t, int d) {
    return ((t >> 3) * (D / 16) + (d >> 4)) * 128 + (t & 7) * 16 + (d & 15);
}
template <int D>
__device__ __forceinline__ int value_byte(int t, int d) {
    return (t >> 5) * 32 * D + (d >> 3) * 256 + ((t >> 4) & 1) * 128 + (d & 7) * 16 + (t & 15);
}

// Bytes of a granule of either array: 32 D values of 8 bits, or of 4 bits and D scales of 8 behind them.
__host__ __device__ constexpr int granule_bytes(int bits, int d) { return bits == 8 ? kGranule * d : 17 * d; }

// First byte of a block and head in either pool (64 bits: pools pass 4 GB).
template <int kBits = 8>
__device__ __forceinline__ int64_t block_byte(const mp_kv_cache& c, int page, int head) {
    return ((int64_t)page * c.n_heads + head) * ((int64_t)(c.block_tokens / kGranule) * granule_bytes(kBits, c.head_dim));
}

// 4 bits: byte of key and value (t, d) inside a granule (d even or odd: its low or high half), and byte of their scale
// behind the codes.  A key's codes lie in a row; a warp's lanes find the D / 8 values of two neighbouring tokens that they
// multiply in one piece, and their scales in one word.
template <int D>
__device__ __forceinline__ int key4_byte(int t, int d) {
    return t * (D / 2) + d / 2;
}
template <int D>
__device__ __forceinline__ int value4_byte(int t, int d) {
    return ((t / 8 * 8 + d / (D / 8)) * 4 + t % 8 / 2) * (D / 8) + d % (D / 8) / 4 * 4 + t % 2 * 2 + d % 4 / 2;
}
template <int D>
__device__ __forceinline__ int key4_scale(int t, int d) {
    return t % 8 * (D / 8) + d / 32 * 4 + t / 8;
}
template <int D>
__device__ __forceinline__ int value4_scale(int t, int d) {
    return (d / 32 * 4 + t / 2 % 4) * 8 + t / 8 * 2 + t % 2;
}

// The 4-bit pool as the attention kernels take it.
inline mp_kv_cache as_pool(const mp_kv4_cache& c) {
    return {c.n_blocks, c.block_tokens, c.n_heads, c.head_dim, c.k, c.v, nullptr, nullptr};
}

// Scales (s, s') of a pair of codes as f16, and what is to be added to s times 16 + u and 256 + u so that s (u - 8) comes
// out.  s has 4 significant bits and is at most 240: 24 s and 264 s are f16 values, and so is every s (u - 8); the fused
// product and sum rounds nothing.
struct Steps {
    uint32_t s, off16, off256;
};
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t x, uint32_t y, uint32_t z) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(y), "r"(z));
    return r;
}
__device__ __forceinline__ Steps steps_of(uint32_t s) {
    return {s, mul_f16x2(s, 0xce00ce00u), mul_f16x2(s, 0xdc20dc20u)};  // -24, -264
}
// x & mask | bits in one operation (written with & and | it became two, for both constants would be immediate ones: 774
// instructions a granule of k_kv_attend_few for 646).
__device__ __forceinline__ uint32_t masked_or(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(x), "r"(mask), "r"(bits));
    return r;
}
// 8 codes of a word as f16 pairs of codes i and i + 4, by the well-known way of widening small whole numbers, their bits placed in the
// fraction under a fixed exponent: a code that is moved to bits 6-9 under the exponent of 16 is 16 +
// u, at bits 2-5 under that of 256 it is 256 + u, so that 10 operations make 8 values.
__device__ __forceinline__ void codes_to_f16(uint32_t w, const Steps& s, uint32_t* pairs) {
    const uint32_t lo = w << 2, hi = w >> 6;
    pairs[0] = fma_f16x2(masked_or(lo, 0x003c003cu, 0x5c005c00u), s.s, s.off256);
    pairs[1] = fma_f16x2(masked_or(lo, 0x03c003c0u, 0x4c004c00u), s.s, s.off16);
    pairs[2] = fma_f16x2(masked_or(hi, 0x003c003cu, 0x5c005c00u), s.s, s.off256);
    pairs[3] = fma_f16x2(masked_or(hi, 0x03c003c0u, 0x4c004c00u), s.s, s.off16);
}

// The same, a sixteenth of each value: then 72 and 1,032 times a sixteenth of the scale are f16 values too (129 times 4 bits
// are 11), so that codes may stay at bits 0-3 under the exponent of 1,024 and at bits 4-7 under that of 64, and one shift
// serves a word (two of 262,144 tokens 127.3 -> 126.3 us, 4 tokens over 64 ragged contexts 125 -> 122).
struct Sixteenths {
    uint32_t s, off64, off1024;
};
constexpr float kSixteenth = 16.f;  // what products with them are to be multiplied by
__device__ __forceinline__ Sixteenths sixteenths_of(uint32_t s) {
    return {mul_f16x2(s, 0x2c002c00u), mul_f16x2(s, 0xc480c480u), mul_f16x2(s, 0xd408d408u)};  // 1/16, -4.5, -64.5
}
__device__ __forceinline__ void codes_to_sixteenths(uint32_t w, const Sixteenths& s, uint32_t* pairs) {
    const uint32_t hi = w >> 8;
    pairs[0] = fma_f16x2(masked_or(w, 0x000f000fu, 0x64006400u), s.s, s.off1024);
    pairs[1] = fma_f16x2(masked_or(w, 0x00f000f0u, 0x54005400u), s.s, s.off64);
    pairs[2] = fma_f16x2(masked_or(hi, 0x000f000fu, 0x64006400u), s.s, s.off1024);
    pairs[3] = fma_f16x2(masked_or(hi, 0x00f000f0u, 0x54005400u), s.s, s.off64);
}

struct SeqView {
    int64_t lo;   // first row of the token arrays
    int32_t n;    // the call's tokens
    int32_t len;  // tokens held
    int32_t st;   // MP_OK or MP_EINVAL
};

__device__ __forceinline__ SeqView load_seq(const mp_kv_batch& bt, int b, bool stored) {
    SeqView v;
    const int64_t lo = __ldg(bt.token_ptr + b), hi = __ldg(bt.token_ptr + b + 1);
    v.len = __ldg(bt.lens + b);
    v.lo = lo;
    v.n = 0;
    v.st = MP_EINVAL;
    if (lo < 0 || hi < lo || hi > bt.n_tokens || hi - lo > bt.max_tokens || v.len < 0 || v.len > bt.max_len) return v;
    if (stored && hi - lo > v.len) return v;
    v.n = (int32_t)(hi - lo);
    v.st = MP_OK;
    return v;
}

// 4 e4m3 bytes as two f16 pairs (exact).
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}"
        : "=r"(lo), "=r"(hi)
        : "r"(w));
}
__device__ __forceinline__ void e4m3_to_f32(uint32_t w, float* x) {
    uint32_t lo, hi;
    e4m3_to_f16(w, lo, hi);
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
}
// 4 values as e4m3 bytes: to nearest even, saturating.
__device__ __forceinline__ uint32_t f32_to_e4m3(const float* x) {
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
        "mov.b32 %0, {l, h};\n\t}"
        : "=r"(r)
        : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]));
    return r;
}

template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ float to_f32<__half>(__half x) {
    return __half2float(x);
}
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) {
    return __bfloat162float(x);
}
template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) {
    return x;
}
template <>
__device__ __forceinline__ __half from_f32<__half>(float x) {
    return __float2half_rn(x);
}
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) {
    return __float2bfloat16_rn(x);
}

// N consecutive values from memory that is aligned to them all (wide) or only
// to one.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
    T x[N];
};
template <typename T, int N>
__device__ __forceinline__ void load_values(const T* p, bool wide, float* x) {
    if (wide) {
        const Pack<T, N> v = *reinterpret_cast<const Pack<T, N>*>(p);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = to_f32(v.x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = to_f32(p[i]);
    }
}
template <typename T, int N>
__device__ __forceinline__ void store_values(T* p, bool wide, const float* x) {
    if (wide) {
        Pack<T, N> v;
#pragma unroll
        for (int i = 0; i < N; ++i) v.x[i] = from_f32<T>(x[i]);
        *reinterpret_cast<Pack<T, N>*>(p) = v;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = from_f32<T>(x[i]);
    }
}

// Whether every row of t starts on a 16-byte boundary.
inline bool rows_aligned(const mp_tokens& t) {
    const int64_t size = t.dtype == MP_F32 ? 4 : 2;
    return reinterpret_cast<uintptr_t>(t.data) % 16 == 0 && t.token_stride * size % 16 == 0 &&
           t.head_stride * size % 16 == 0;
}

}  // namespace mp
