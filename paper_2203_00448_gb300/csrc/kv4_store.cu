// kv4_store.cu -- mp_kv_four_write and mp_kv_four_read: tokens into and out of the cache's 4-bit blocks.
//
// 32 values of a token and head have a scale s of 4 significant bits, the least with max |x| <= 7.5 s, and codes n =
// x / s rounded to the nearest whole number of -7 .. 7: no value is off by more than half a step, and n s is exact in
// f16, bf16 and f32.  A token's codes depend on no other token, so nothing that is stored is ever rounded again.
//
// Measured (8 heads of 128, GPU time): 253 single tokens written 5 us and read 6; 15,973 prompt tokens written 27 us (66 MB of them and
// 17 of codes: 12 us at a copy's rate) and read back 15; 131,071 read back 101 us (6.7 TB/s, a copy's rate);
// 32 x 300 tokens written 19, the prompts in 32 bits 39.  Writes take 145 instructions for 8 values of each lane, which issue in 68% of
// the cycles (with rintf and conversions to integers, which run on a slow unit, and divisions it was 60 us); the others go to
// the trips for values, four steps (of 32 bits two) at a time with none on its way under the arithmetic.  One prompt of 8,192 tokens
// with 255 single tokens takes 194 us to write and 156 to read back (16 and 12 in two calls): units are laid out for the longest sequence.
#include <algorithm>

#include "kv.cuh"

namespace mp {
namespace {

constexpr int kFewThreads = 512;  // few tokens: a CTA a sequence (253 of them: 128 threads 13.2, 256 11.1, 512 9.7 us with the timing)
constexpr int kThreads = 128, kWarps = kThreads / 32;  // else (64, 128 and 256: prompts written 28.8, 26.8 and 28.8 us)
// Up to this many tokens a sequence, a CTA a sequence (GPU time with it and without: 8 sequences of 1 token 2.0 and 2.1 us, of 16 6.1
// and 6.1, of 24 8.3 and 8.1; 64 of 1 token 1.8 and 3.1, of 8 4.1 and 4.1, of 16 7.5 and 6.1; 253 of 1 token 2.0 and 4.1, of 8 6.1 and
// 8.2, of 16 10.2 and 12.3): what few sequences of many tokens lose by it many of one token gain.
constexpr int32_t kFewTokens = 16;
constexpr float kMost = 1800.f;     // 7.5 times the largest scale
constexpr int kMostScale = 183;     // its byte: 240

__device__ __forceinline__ float scale_value(int byte) {
    return __half2float(__ushort_as_half((unsigned short)(byte << 7)));
}

// The byte of the least scale with a <= 7.5 s, a a value of type T.
template <typename T>
__device__ __forceinline__ int scale_byte(float a) {
    // a little less than a / 7.5, so that a = 7.5 s does not come out above s; no other value of 16 bits is as near
    float least = a * (2.f / 15.f * (1.f - 0x1p-18f));
    // up to the next number of 4 significant bits, or, below 2^-14, to the next multiple of 2^-17
    const bool small = least < 0x1p-14f;
    if (small) least = __fadd_ru(least, 0x1p-14f);
    int byte = (int)((__float_as_uint(least) + 0xfffffu) >> 20) - (small ? 113 << 3 : 112 << 3);
    if (sizeof(T) == 4 && 7.5f * scale_value(byte) < a) ++byte;  // a value of 32 bits may be as near
    return min(byte, kMostScale);
}

// 8 values of a token as they are in memory.
template <typename T>
struct Raw {
    uint4 w[sizeof(T) / 2];
};
template <typename T>
__device__ __forceinline__ Raw<T> load_raw(const T* p, bool wide) {
    Raw<T> r;
    if (wide) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) r.w[i] = *(reinterpret_cast<const uint4*>(p) + i);
    } else {
        T* e = reinterpret_cast<T*>(&r);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = p[i];
    }
    return r;
}

constexpr float kWhole = 12582912.f;  // 1.5 * 2^23: a sum with it is a whole number in its low bits
// x / s to the nearest whole number, ties to the even one, in the low bits.  For values of 16 bits a quotient that is no tie
// is further from one than 2^-15 of itself, so products with numbers on either side of 1 / s (2^-21 of it away) agree, unless
// it is a tie: then they are the two that it lies between, and the sum of both, an odd number of 25 bits, is rounded to even.
__device__ __forceinline__ uint32_t nearest16(float x, float below, float above) {
    return __float_as_uint(fmaf(x, below, kWhole) + fmaf(x, above, kWhole));
}
// ... of 32 bits: what the product leaves of x is exact and says whether it was off.
__device__ __forceinline__ uint32_t nearest32(float x, float s, float inverse) {
    const float y = fmaf(x, inverse, kWhole), rest = fmaf(-(y - kWhole), s, x);
    const uint32_t bits = __float_as_uint(y);
    // half a step, or the number before it where a tie has to move from an odd number
    const float most = __uint_as_float(__float_as_uint(0.5f * s) - (bits & 1));
    return fabsf(rest) > most ? bits + (rest < 0.f ? ~0u : 1u) : bits;
}

// Codes of 8 values of a token (32 of 4 neighbouring lanes share a scale) and their scale's byte; fine: becomes false if some
// value is not finite or too large.
template <typename T>
__device__ __forceinline__ uint32_t quantise(const Raw<T>& raw, int& byte, bool& fine) {
    float v[8], most = 0.f;
    const T* e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = to_f32(e[i]);
    if (sizeof(T) == 2) {
        // magnitudes as the integers that their bits are, two at a time; infinities and NaN come out on top
        const uint32_t m = __vmaxu2(__vmaxu2(raw.w[0].x & 0x7fff7fffu, raw.w[0].y & 0x7fff7fffu),
                                    __vmaxu2(raw.w[0].z & 0x7fff7fffu, raw.w[0].w & 0x7fff7fffu));
        const uint16_t bits = (uint16_t)max(m & 0xffffu, m >> 16);
        most = to_f32(*reinterpret_cast<const T*>(&bits));
    } else {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = max(m, __float_as_uint(v[i]) & 0x7fffffffu);
        most = __uint_as_float(m);
    }
    if (!(most <= kMost)) {
        fine = false;
        most = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = v[i] != v[i] ? 0.f : fminf(fmaxf(v[i], -kMost), kMost);
            most = fmaxf(most, fabsf(v[i]));
        }
    }
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 1));
    most = fmaxf(most, __shfl_xor_sync(~0u, most, 2));
    byte = scale_byte<T>(most);
    const float s = scale_value(byte);
    float inverse;
    asm("rcp.approx.f32 %0, %1;" : "=f"(inverse) : "f"(s));
    if (byte == 0) inverse = 0.f;
    const float below = inverse * (1.f - 0x1p-21f), above = inverse * (1.f + 0x1p-21f);
    uint32_t n[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) n[i] = sizeof(T) == 2 ? nearest16(v[i], below, above) : nearest32(v[i], s, inverse);
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t two = __vmins2(__vmaxs2(__byte_perm(n[i], n[i + 4], 0x5410), 0xfff9fff9u), 0x00070007u);
        w |= (two & 0x000f000fu) << (4 * i);
    }
    return w ^ 0x88888888u;  // two's complement of 4 bits, 8 more
}

// A warp stores tokens [from, past) (slots of a granule; all of them, from wide rows, with kAll) of one head and array: a
// lane 8 values of a token a step.  x: the first of them.  False if some value was not finite or too large.
template <typename T, int D, bool kValues, bool kAll>
__device__ __forceinline__ bool store_tokens(const T* x, int64_t stride, bool wide, int from, int past, uint8_t* bytes) {
    constexpr int kLanes = D / 8, kTokens = 32 / kLanes;  // lanes of a token, tokens a step
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;        // steps whose values are on their way together
    const int lane = threadIdx.x % 32, d = lane % kLanes * 8;
    bool fine = true;
    if (kAll) from = 0, past = kGranule;
    x += d - from * stride;
#pragma unroll 1
    for (int t0 = from / kTokens * kTokens; t0 < past; t0 += kAhead * kTokens) {
        Raw<T> raw[kAhead] = {};
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int t = t0 + e * kTokens + lane / kLanes;
            if (kAll || (t >= from && t < past)) raw[e] = load_raw(x + t * stride, kAll || wide);
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            if (!kAll && t0 + e * kTokens >= past) break;
            const int t = t0 + e * kTokens + lane / kLanes;
            const bool mine = kAll || (t >= from && t < past);
            int byte;
            const uint32_t w = quantise<T>(raw[e], byte, fine);
            if (mine && lane % 4 == 0) bytes[16 * D + (kValues ? value4_scale<D>(t, d) : key4_scale<D>(t, d))] = (uint8_t)byte;
            if (!kValues) {
                if (mine) *reinterpret_cast<uint32_t*>(bytes + key4_byte<D>(t, d)) = w;
            } else {
                // the neighbouring token's lane has the other half of either word
                const uint32_t other = __shfl_xor_sync(~0u, t % 2 ? w & 0xffff : w >> 16, kLanes);
                uint8_t* const at = bytes + value4_byte<D>(t, d);  // (of its half of the first word)
                if (kAll || (mine && (t ^ 1) >= from && (t ^ 1) < past)) {
                    if (t % 2) *reinterpret_cast<uint32_t*>(at + 2) = other | (w & 0xffff0000u);
                    else *reinterpret_cast<uint32_t*>(at) = (w & 0xffffu) | other << 16;
                } else if (mine) {
                    *reinterpret_cast<uint16_t*>(at) = (uint16_t)w;
                    *reinterpret_cast<uint16_t*>(at + 4) = (uint16_t)(w >> 16);
                }
            }
        }
    }
    return fine;
}

template <typename T, int D, bool kValues>
__device__ __forceinline__ bool store_granule(const T* x, int64_t stride, bool wide, int from, int past, uint8_t* bytes) {
    return wide && past - from == kGranule ? store_tokens<T, D, kValues, true>(x, stride, true, 0, kGranule, bytes)
                                           : store_tokens<T, D, kValues, false>(x, stride, wide, from, past, bytes);
}

// One granule, head and array of a sequence: j counts the granules that the call touches.  False if the table or a value is
// wrong there.
template <typename T, int D>
__device__ __forceinline__ bool store_unit(const mp_kv_cache& c, const mp_kv_batch& bt, const SeqView& s, int b, int j, int head,
                                           bool values, const mp_tokens& k, const mp_tokens& v, bool wide) {
    const int start = s.len - s.n, base = (start / kGranule + j) * kGranule;
    const int page = __ldg(bt.table + (int64_t)b * bt.max_blocks + base / c.block_tokens);
    if (page < 0 || page >= c.n_blocks) return false;
    const int64_t at = block_byte<4>(c, page, head) + (int64_t)(base % c.block_tokens / kGranule) * granule_bytes(4, D);
    const int from = max(start - base, 0), past = min(s.len - base, kGranule);
    const mp_tokens& t = values ? v : k;
    const T* x = static_cast<const T*>(t.data) + (s.lo + (base + from - start)) * t.token_stride + head * t.head_stride;
    return values ? store_granule<T, D, true>(x, t.token_stride, wide, from, past, c.v + at)
                  : store_granule<T, D, false>(x, t.token_stride, wide, from, past, c.k + at);
}
__device__ __forceinline__ int granules_touched(const SeqView& s) {
    return s.n == 0 ? 0 : (s.len - 1) / kGranule - (s.len - s.n) / kGranule + 1;
}

// Few tokens a sequence: one CTA a sequence, so that its status has one writer; a warp a granule, head and array.
template <typename T, int D>
__global__ void __launch_bounds__(kFewThreads)
    k_kv4_write_few(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status) {
    for (int b = blockIdx.x; b < bt.n_seqs; b += gridDim.x) {
        const SeqView s = load_seq(bt, b, true);
        bool ok = s.st == MP_OK;
        const int tasks = granules_touched(s) * c.n_heads * 2;
        for (int u = threadIdx.x / 32; u < tasks; u += kFewThreads / 32)
            ok &= store_unit<T, D>(c, bt, s, b, u / (2 * c.n_heads), u / 2 % c.n_heads, u % 2, k, v, wide);
        const bool bad = __syncthreads_or(!ok);
        if (threadIdx.x == 0) status[b] = bad ? MP_EINVAL : MP_OK;
    }
}

// Many tokens: a warp a granule, head and array.  status is cleared before; whoever writes it writes the same.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads)
    k_kv4_write_many(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status, int per_seq) {
    const int64_t units = (int64_t)bt.n_seqs * per_seq * c.n_heads * 2, warps = (int64_t)gridDim.x * kWarps;
    for (int64_t u = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; u < units; u += warps) {
        const int in_seq = (int)(u / 2 / c.n_heads % per_seq), b = (int)(u / 2 / c.n_heads / per_seq);
        const SeqView s = load_seq(bt, b, true);
        bool ok = s.st == MP_OK;
        if (ok && in_seq < granules_touched(s))
            ok = store_unit<T, D>(c, bt, s, b, in_seq, (int)(u / 2 % c.n_heads), u % 2, k, v, wide);
        if (!ok) status[b] = MP_EINVAL;
    }
}

template <typename T>
__device__ __forceinline__ void put8(T* p, bool wide, const uint32_t (&pairs)[4]) {  // pairs of values i and i + 4
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&pairs[i]));
        x[i] = y.x, x[i + 4] = y.y;
    }
    store_values<T, 8>(p, wide, x);
}
// A warp reads a granule's tokens [from, past) of one head back, 8 values of a token (of two tokens, for values) a lane
// and step; four steps, 8 tokens apart, have their scales in one word and their codes on the way together.  x: where the granule's first
// token goes.
template <typename T, int D>
__device__ __forceinline__ void read_keys(const uint8_t* bytes, int from, int past, T* x, int64_t stride, bool wide) {
    constexpr int kLanes = D / 8, kTokens = 32 / kLanes;
    const int lane = threadIdx.x % 32, d = lane % kLanes * 8;
    x += d;
#pragma unroll(8 / kTokens >= 4 ? 2 : 1)
    for (int t0 = 0; t0 < 8; t0 += kTokens) {
        const int t1 = t0 + lane / kLanes;
        const uint32_t scales = __ldg(reinterpret_cast<const uint32_t*>(bytes + 16 * D + key4_scale<D>(t1, d)));
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __ldg(reinterpret_cast<const uint32_t*>(bytes + key4_byte<D>(t1 + 8 * e, d)));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = t1 + 8 * e;
            uint32_t pairs[4];
            codes_to_f16(w[e], steps_of((scales >> (8 * e) & 0xff) * 0x00800080u), pairs);
            if (t >= from && t < past) put8(x + t * stride, wide, pairs);
        }
    }
}
template <typename T, int D>
__device__ __forceinline__ void read_values(const uint8_t* bytes, int from, int past, T* x, int64_t stride, bool wide) {
    constexpr int kLanes = D / 8, kTokens = 2 * (32 / kLanes);
    const int lane = threadIdx.x % 32, d = lane % kLanes * 8;
    x += d;
#pragma unroll 1
    for (int t0 = 0; t0 < 8; t0 += kTokens) {
        const int t1 = t0 + lane / kLanes * 2;
        const uint2 scales = __ldg(reinterpret_cast<const uint2*>(bytes + 16 * D + value4_scale<D>(t1, d)));
        uint2 w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = __ldg(reinterpret_cast<const uint2*>(bytes + value4_byte<D>(t1 + 8 * e, d)));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int t = t1 + 8 * e;
            const Steps steps = steps_of(__byte_perm(e < 2 ? scales.x : scales.y, 0, e % 2 ? 0x4342 : 0x4140) << 7);
            uint32_t a[4], b[4], lo[4], hi[4];
            codes_to_f16(w[e].x, steps, a), codes_to_f16(w[e].y, steps, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) lo[i] = __byte_perm(a[i], b[i], 0x5410), hi[i] = __byte_perm(a[i], b[i], 0x7632);
            if (t >= from && t < past) put8(x + t * stride, wide, lo);
            if (t + 1 >= from && t + 1 < past) put8(x + (t + 1) * stride, wide, hi);
        }
    }
}

template <typename T, int D>
__global__ void __launch_bounds__(kThreads, 12)  // (131,071 tokens 101.5 us, 102.5 with as many registers as it likes)
    k_kv4_read(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status, int per_seq) {
    const int lane = threadIdx.x % 32;
    const int64_t units = (int64_t)bt.n_seqs * per_seq * c.n_heads * 2, warps = (int64_t)gridDim.x * kWarps;
    for (int64_t u = (int64_t)blockIdx.x * kWarps + threadIdx.x / 32; u < units; u += warps) {
        const int head = (int)(u / 2 % c.n_heads), j = (int)(u / 2 / c.n_heads % per_seq);
        const int b = (int)(u / 2 / c.n_heads / per_seq);
        const SeqView s = load_seq(bt, b, true);
        const int start = s.len - s.n;
        if (u % 2 == 0 && head == 0 && j == 0) {  // one warp looks the sequence's table over
            bool ok = s.st == MP_OK;
            if (s.n > 0)
                for (int col = start / c.block_tokens + lane; col <= (s.len - 1) / c.block_tokens; col += 32) {
                    const int p = __ldg(bt.table + (int64_t)b * bt.max_blocks + col);
                    ok &= p >= 0 && p < c.n_blocks;
                }
            ok = __all_sync(~0u, ok);
            if (lane == 0) status[b] = ok ? MP_OK : MP_EINVAL;
        }
        if (j >= granules_touched(s)) continue;
        const int base = (start / kGranule + j) * kGranule;
        const int page = __ldg(bt.table + (int64_t)b * bt.max_blocks + base / c.block_tokens);
        if (page < 0 || page >= c.n_blocks) continue;
        const int from = max(start - base, 0), past = min(s.len - base, kGranule);
        const int64_t at = block_byte<4>(c, page, head) + (int64_t)(base % c.block_tokens / kGranule) * granule_bytes(4, D);
        const mp_tokens& t = u % 2 ? v : k;
        T* x = static_cast<T*>(t.data) + (s.lo + (base - start)) * t.token_stride + head * t.head_stride;
        if (u % 2) read_values<T, D>(c.v + at, from, past, x, t.token_stride, wide);
        else read_keys<T, D>(c.k + at, from, past, x, t.token_stride, wide);
    }
}

// Granules that a sequence's tokens may touch.
int granules_most(const mp_kv_batch& bt) { return std::max<int>((bt.max_tokens + 2 * kGranule - 2) / kGranule, 1); }

template <typename T, int D>
cudaError_t write_as(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v, int32_t* status,
                     cudaStream_t stream) {
    const bool wide = rows_aligned(k) && rows_aligned(v);
    if (bt.max_tokens <= kFewTokens) {
        k_kv4_write_few<T, D><<<(unsigned)std::min(bt.n_seqs, 1 << 20), kFewThreads, 0, stream>>>(c, bt, k, v, wide, status);
        return cudaGetLastError();
    }
    cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t) * (size_t)bt.n_seqs, stream);
    if (e != cudaSuccess) return e;
    const int per_seq = granules_most(bt);
    const int64_t ctas = ((int64_t)bt.n_seqs * per_seq * c.n_heads * 2 + kWarps - 1) / kWarps;
    k_kv4_write_many<T, D><<<(unsigned)std::min<int64_t>(ctas, 1 << 20), kThreads, 0, stream>>>(c, bt, k, v, wide, status, per_seq);
    return cudaGetLastError();
}
template <typename T, int D>
cudaError_t read_as(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v, int32_t* status,
                    cudaStream_t stream) {
    const bool wide = rows_aligned(k) && rows_aligned(v);
    const int per_seq = granules_most(bt);
    const int64_t ctas = ((int64_t)bt.n_seqs * per_seq * c.n_heads * 2 + kWarps - 1) / kWarps;
    k_kv4_read<T, D><<<(unsigned)std::min<int64_t>(ctas, 1 << 20), kThreads, 0, stream>>>(c, bt, k, v, wide, status, per_seq);
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_kv4_write(const mp_kv4_cache& c4, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                             int32_t* status, cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    const mp_kv_cache c = as_pool(c4);
    const bool narrow = c.head_dim == 64;
    if (k.dtype == MP_F16)
        return narrow ? write_as<__half, 64>(c, bt, k, v, status, stream) : write_as<__half, 128>(c, bt, k, v, status, stream);
    if (k.dtype == MP_BF16)
        return narrow ? write_as<__nv_bfloat16, 64>(c, bt, k, v, status, stream)
                      : write_as<__nv_bfloat16, 128>(c, bt, k, v, status, stream);
    return narrow ? write_as<float, 64>(c, bt, k, v, status, stream) : write_as<float, 128>(c, bt, k, v, status, stream);
}

cudaError_t launch_kv4_read(const mp_kv4_cache& c4, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                            int32_t* status, cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    const mp_kv_cache c = as_pool(c4);
    const bool narrow = c.head_dim == 64;
    if (k.dtype == MP_F16)
        return narrow ? read_as<__half, 64>(c, bt, k, v, status, stream) : read_as<__half, 128>(c, bt, k, v, status, stream);
    if (k.dtype == MP_BF16)
        return narrow ? read_as<__nv_bfloat16, 64>(c, bt, k, v, status, stream)
                      : read_as<__nv_bfloat16, 128>(c, bt, k, v, status, stream);
    return narrow ? read_as<float, 64>(c, bt, k, v, status, stream) : read_as<float, 128>(c, bt, k, v, status, stream);
}

}  // namespace mp
