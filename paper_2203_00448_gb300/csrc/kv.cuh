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

// First byte of a block and head in either pool (64 bits: pools pass 4 GB).
__device__ __forceinline__ int64_t block_byte(const mp_kv_cache& c, int page, int head) {
    return ((int64_t)page * c.n_heads + head) * ((int64_t)c.block_tokens * c.head_dim);
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
