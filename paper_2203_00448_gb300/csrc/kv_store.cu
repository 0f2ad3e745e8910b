// kv_store.cu -- mp_kv_write and mp_kv_read: tokens into and out of the cache's
// 8-bit blocks.
//
// A block and head is stored under one scale s = 2^e, the least power of two with
// max |x| <= 448 s (448 is the largest e4m3 value).  Dividing by it is exact, so a
// stored value carries the one rounding to e4m3's 4 significant bits, whatever the
// scale; when a later token makes the scale grow, earlier bytes are rounded again,
// which loses bits only among subnormals.
//
// Measured (8 heads of 128): a step of 253 single tokens 4.9 us of GPU time, bound by
// three trips to memory one after another (lengths, table, values and scale); 15,973
// prompt tokens 27 us (98 MB, 14.4 us at the rate of a copy), bound by instructions
// (two thirds of the issue slots while CTAs run) and the uneven last CTAs; 131,071 tokens
// read back 126 us, 94% of a copy's rate.  The same prompts in 32 bits 46 us (164 MB, 24 us at a copy's rate), bound alike;
// 8 ragged reads of up to 512 tokens (16 heads of 64, 32 bits) 9.0 us, where each warp takes the trips to its keys and
// to its values one after the other.
#include <algorithm>

#include "kv.cuh"

namespace mp {
namespace {

constexpr int kWriteWarps = 16;          // few tokens: one CTA a sequence, a warp a block, head and array
// ... up to this many tokens a sequence.  GPU time of this kernel and of the other (a clear of the status and a launch; 8
// heads of 128, bf16): 8 sequences of 1 token 3.7 and 8.2 us, of 4 7.0 and 8.2, of 8 10.1 and 8.2, of 16 16.5 and 8.2; 253
// of 1 5.1 and 12.4, of 4 10.9 and 16.4, of 8 18.9 and 19.0, of 16 35.5 and 27.2.  They meet at 5 to 8 tokens; the line
// is higher than that, and 9 to 16 proposed tokens pay for it.
constexpr int32_t kWriteFewTokens = 16;
constexpr int kWriteThreads = 128;
// CTAs below which a CTA takes fewer heads.  With 1, 4, 12, 24 and 48 an SM (f16, 8 heads of 128): 18,800 prompt tokens of 9
// sequences 48.9, 29.5, 28.9, 28.9 and 28.8 us, 32 x 300 tokens 41.3, 22.4, 18.5, 18.5 and 18.5, 64 x 2,000 145, 145, 145, 136
// and 134, 1 x 4,000 14.3, 10.8, 12.3, 11.7 and 10.7.
constexpr int kWriteCtas = kSms * 12;
constexpr int kReadThreads = 256;

// Magnitudes are compared as the integers that their bits are (without the sign): one operation a value or a pair,
// and infinities and NaN come out above everything finite.
template <typename T>
constexpr uint32_t kInfBits = 0x7f800000u;
template <>
constexpr uint32_t kInfBits<__half> = 0x7c00u;
template <>
constexpr uint32_t kInfBits<__nv_bfloat16> = 0x7f80u;
template <typename T>
__device__ __forceinline__ float value_of(uint32_t bits) {
    if (sizeof(T) == 4) return __uint_as_float(bits);
    const uint16_t h = (uint16_t)bits;
    return to_f32(*reinterpret_cast<const T*>(&h));
}
// The largest magnitude of the values in a word (4-byte types: one, else two) joins top (two halves for two).
template <typename T>
__device__ __forceinline__ uint32_t join_word(uint32_t top, uint32_t w) {
    return sizeof(T) == 4 ? max(top, w & 0x7fffffffu) : __vmaxu2(top, w & 0x7fff7fffu);
}
// ... only finite ones.
template <typename T>
__device__ __forceinline__ uint32_t join_finite(uint32_t top, uint32_t w) {
    if (sizeof(T) == 4) return (w & 0x7fffffffu) < kInfBits<T> ? max(top, w & 0x7fffffffu) : top;
    const uint32_t lo = w & 0x7fffu, hi = w & 0x7fff0000u;
    if (lo < kInfBits<T>) top = __vmaxu2(top, lo);
    if (hi < kInfBits<T> << 16) top = __vmaxu2(top, hi);
    return top;
}
template <typename T>
__device__ __forceinline__ uint32_t join_end(uint32_t top) {
    return sizeof(T) == 4 ? top : max(top & 0xffffu, top >> 16);
}
// The largest of all threads' integers, over a warp (kGroup 32) or a CTA (0).
template <int kGroup>
__device__ __forceinline__ uint32_t group_max(uint32_t x, uint32_t* smem) {
    x = __reduce_max_sync(~0u, x);
    if (kGroup == 0) {
        __syncthreads();  // smem's last use
        if (threadIdx.x % 32 == 0) smem[threadIdx.x / 32] = x;
        __syncthreads();
        x = smem[threadIdx.x % (kWriteThreads / 32)];
        x = __reduce_max_sync(~0u, x);
    }
    return x;
}
// The values in a word, times the inverse of the scale; kOdd: some value of the block is not finite (NaN is stored as 0).
template <typename T, bool kOdd>
__device__ __forceinline__ void scaled(uint32_t w, float inverse, float* y) {
    if (sizeof(T) == 4) {
        y[0] = __uint_as_float(w);
    } else {
        const uint16_t lo = (uint16_t)w, hi = (uint16_t)(w >> 16);
        y[0] = to_f32(*reinterpret_cast<const T*>(&lo)), y[1] = to_f32(*reinterpret_cast<const T*>(&hi));
    }
#pragma unroll
    for (int i = 0; i < 4 / (int)sizeof(T); ++i) {
        if (kOdd) y[i] = y[i] == y[i] ? y[i] : 0.f;
        y[i] *= inverse;
    }
}

// 2^e with the least e in [-60, 120] such that a <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ float scale_of(float a) {
    const uint32_t u = __float_as_uint(a);
    int e = (int)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);
    e = min(max(e, -60), 120);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// 4 stored bytes under another scale (ratio: the old one over the new one).
__device__ __forceinline__ uint32_t rescale(uint32_t w, float ratio) {
    float x[4];
    e4m3_to_f32(w, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= ratio;
    return f32_to_e4m3(x);
}

// The earlier tokens (slots below first) of one block and head under a larger scale; kGroup threads.
template <int D, bool kValues>
__device__ __noinline__ void rescale_block(uint8_t* bytes, int first, float ratio, int rank, int group) {
    uint32_t* const word = reinterpret_cast<uint32_t*>(bytes);
    const int words = (first + kGranule - 1) / kGranule * kGranule * D / 4;
    for (int i = rank; i < words; i += group) {
        const int byte = i * 4;
        if (!kValues) {
            if (byte / 128 / (D / 16) * 8 + byte % 128 / 16 < first) word[i] = rescale(word[i], ratio);
        } else {
            const int t = byte / (32 * D) * 32 + byte / 128 % 2 * 16 + byte % 16, n = first - t;
            if (n <= 0) continue;
            const uint32_t keep = n >= 4 ? ~0u : (1u << (8 * n)) - 1, had = word[i];
            word[i] = (rescale(had, ratio) & keep) | (had & ~keep);
        }
    }
}

// What the tokens of a block and head are stored under, given the largest new magnitude; earlier tokens are brought
// under it too.  Every thread of the group calls it, after top is known to all; returns the scale's inverse.
template <int D, bool kValues, int kGroup>
__device__ __forceinline__ float settle(float top, float old, int first, uint8_t* bytes, float* scale_at, int rank) {
    const float scale = fmaxf(scale_of(top), old);
    if (first > 0 && scale > old) {
        rescale_block<D, kValues>(bytes, first, __fdiv_rn(old, scale), rank, kGroup == 32 ? 32 : blockDim.x);
        // a new token's bytes may share words with earlier ones
        if (kGroup == 32) __syncwarp();
        else __syncthreads();
    }
    if (rank == 0 && !(first > 0 && scale == old)) *scale_at = scale;
    return __fdiv_rn(1.f, scale);
}

// Where a block, head and array of the call lies.
struct Place {
    const void* x;  // its first new token's values
    int64_t stride;
    int first, n;  // slots [first, first + n)
    uint8_t* bytes;
    float* scale;
};
// j counts the blocks that the call touches; false if the table is wrong there.
template <typename T>
__device__ __forceinline__ bool find(const mp_kv_cache& c, const mp_kv_batch& bt, const SeqView& s, int b, int j, int head,
                                     bool values, const mp_tokens& k, const mp_tokens& v, Place& p) {
    const int start = s.len - s.n, col = start / c.block_tokens + j, base = col * c.block_tokens;
    const int page = __ldg(bt.table + (int64_t)b * bt.max_blocks + col);
    if (page < 0 || page >= c.n_blocks) return false;
    p.first = max(start - base, 0), p.n = min(s.len - base, c.block_tokens) - p.first;
    const mp_tokens& t = values ? v : k;
    p.stride = t.token_stride;
    p.x = static_cast<const T*>(t.data) + (s.lo + (base + p.first - start)) * t.token_stride + head * t.head_stride;
    const int64_t at = block_byte(c, page, head), sc = (int64_t)page * c.n_heads + head;
    p.bytes = (values ? c.v : c.k) + at, p.scale = (values ? c.v_scale : c.k_scale) + sc;
    return true;
}

__device__ __forceinline__ int blocks_touched(const mp_kv_cache& c, const SeqView& s) {
    return s.n == 0 ? 0 : (s.len - 1) / c.block_tokens - (s.len - s.n) / c.block_tokens + 1;
}

// A lane's D / 32 values of a token as words.
template <typename T, int D>
__device__ __forceinline__ void read_lane(const T* at, bool wide, uint32_t* w) {
    constexpr int kWords = D / 32 * sizeof(T) / 4;
    if (wide) {
        const Pack<uint32_t, kWords> v = *reinterpret_cast<const Pack<uint32_t, kWords>*>(at);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = v.x[i];
    } else if (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint32_t*>(at)[i];
    } else {
        const uint16_t* h = reinterpret_cast<const uint16_t*>(at);
#pragma unroll
        for (int i = 0; i < kWords; ++i) w[i] = (uint32_t)h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
    }
}

// A warp stores n tokens one after another, a lane D / 32 values of each.
template <typename T, int D, bool kValues>
__device__ __forceinline__ bool store_few(const Place& p, bool wide, int lane) {
    constexpr int kPer = D / 32, kWords = kPer * sizeof(T) / 4, kIn = 4 / sizeof(T);
    const T* x = static_cast<const T*>(p.x) + lane * kPer;
    const float old = p.first > 0 ? *p.scale : 0.f;
    uint32_t w[kWords], top = 0;
    for (int i = 0; i < p.n; ++i) {
        read_lane<T, D>(x + i * p.stride, wide, w);
#pragma unroll
        for (int k = 0; k < kWords; ++k) top = join_word<T>(top, w[k]);
    }
    top = group_max<32>(join_end<T>(top), nullptr);
    const bool odd = top >= kInfBits<T>;
    if (odd) {
        top = 0;
        for (int i = 0; i < p.n; ++i) {
            read_lane<T, D>(x + i * p.stride, wide, w);
            for (int k = 0; k < kWords; ++k) top = join_finite<T>(top, w[k]);
        }
        top = group_max<32>(join_end<T>(top), nullptr);
    }
    const float inverse = settle<D, kValues, 32>(value_of<T>(top), old, p.first, p.bytes, p.scale, lane);
    for (int i = 0; i < p.n; ++i) {
        if (p.n > 1) read_lane<T, D>(x + i * p.stride, wide, w);
        float v[4] = {};
#pragma unroll
        for (int k = 0; k < kWords; ++k) scaled<T, true>(w[k], inverse, v + k * kIn);
        const uint32_t out = f32_to_e4m3(v);
        const int t = p.first + i, d = lane * kPer;
        if (!kValues) {
            uint8_t* at = p.bytes + key_byte<D>(t, d);
            if (kPer == 4) *reinterpret_cast<uint32_t*>(at) = out;
            else *reinterpret_cast<uint16_t*>(at) = (uint16_t)out;
        } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) p.bytes[value_byte<D>(t, d + k)] = (uint8_t)(out >> (8 * k));
        }
    }
    return !odd;
}

// Few tokens a sequence: one CTA a sequence, so that its status has one writer; a warp a block, head and array.  (16 warps
// leave 64 registers a thread: 24 bytes are kept in memory for values of 32 bits, 8 for others of D = 128.)
template <typename T, int D>
__global__ void __launch_bounds__(kWriteWarps * 32)
    k_kv_write_few(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status) {
    for (int b = blockIdx.x; b < bt.n_seqs; b += gridDim.x) {
        const SeqView s = load_seq(bt, b, true);
        const int tasks = blocks_touched(c, s) * c.n_heads * 2;
        bool ok = s.st == MP_OK;
        for (int u = threadIdx.x / 32; u < tasks; u += kWriteWarps) {
            Place p;
            if (!find<T>(c, bt, s, b, u / (2 * c.n_heads), u / 2 % c.n_heads, u % 2, k, v, p)) ok = false;
            else if (u % 2) ok &= store_few<T, D, true>(p, wide, threadIdx.x % 32);
            else ok &= store_few<T, D, false>(p, wide, threadIdx.x % 32);
        }
        const bool bad = __syncthreads_or(!ok);
        if (threadIdx.x == 0) status[b] = bad ? MP_EINVAL : MP_OK;
    }
}

// A unit's values [tokens][D] at x into its block: keys, 16 values of a token a step.
template <typename T, int D, bool kOdd>
__device__ __forceinline__ void store_keys(const uint4* x, const Place& p, float inverse, int rank) {
    constexpr int kIn = 16 / sizeof(T), kFour = 16 / kIn;  // values in 16 bytes, and 16 bytes in 16 values
    for (int i = rank; i < p.n * (D / 16); i += kWriteThreads) {
        float y[16];
#pragma unroll
        for (int e = 0; e < kFour; ++e) {
            const uint4 w = x[i * kFour + e];
            scaled<T, kOdd>(w.x, inverse, y + e * kIn), scaled<T, kOdd>(w.y, inverse, y + e * kIn + kIn / 4);
            scaled<T, kOdd>(w.z, inverse, y + e * kIn + kIn / 2), scaled<T, kOdd>(w.w, inverse, y + e * kIn + kIn / 4 * 3);
        }
        *reinterpret_cast<uint4*>(p.bytes + key_byte<D>(p.first + i / (D / 16), i % (D / 16) * 16)) =
            make_uint4(f32_to_e4m3(y), f32_to_e4m3(y + 4), f32_to_e4m3(y + 8), f32_to_e4m3(y + 12));
    }
}
// ... values, 16 tokens of 2 neighbouring ones a step: lanes along the values to read, 16 bytes a lane to store.
template <typename T, int D, bool kOdd>
__device__ __forceinline__ void store_columns(const uint4* x, const Place& p, float inverse, int rank) {
    const int past = p.first + p.n, from = p.first / 16;
    for (int i = rank; i < ((past + 15) / 16 - from) * (D / 2); i += kWriteThreads) {
        const int t0 = (from + i / (D / 2)) * 16, d = i % (D / 2) * 2;
        const T* col = reinterpret_cast<const T*>(x) + (t0 - p.first) * D + d;
        uint8_t* at = p.bytes + value_byte<D>(t0, d);
        auto pair = [&](int t, float& y0, float& y1) {
            const uint32_t* w = reinterpret_cast<const uint32_t*>(col + t * D);
            float y[2];
            scaled<T, kOdd>(w[0], inverse, y);
            if (sizeof(T) == 4) scaled<T, kOdd>(w[1], inverse, y + 1);
            y0 = y[0], y1 = y[1];
        };
        if (t0 >= p.first && t0 + 16 <= past) {
            uint32_t out[2][4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float y[2][4];
#pragma unroll
                for (int f = 0; f < 4; ++f) pair(4 * e + f, y[0][f], y[1][f]);
                out[0][e] = f32_to_e4m3(y[0]), out[1][e] = f32_to_e4m3(y[1]);
            }
            *reinterpret_cast<uint4*>(at) = make_uint4(out[0][0], out[0][1], out[0][2], out[0][3]);
            *reinterpret_cast<uint4*>(at + 16) = make_uint4(out[1][0], out[1][1], out[1][2], out[1][3]);
        } else {  // an end of the new tokens: byte by byte
#pragma unroll 1
            for (int t = max(p.first - t0, 0); t < min(past - t0, 16); ++t) {
                float y[4] = {};
                pair(t, y[0], y[1]);
                const uint32_t w = f32_to_e4m3(y);
                at[t] = (uint8_t)w, at[16 + t] = (uint8_t)(w >> 8);
            }
        }
    }
}

// Many tokens: a CTA a block and `heads` of its heads, keys and values one after another, each read once into shared
// memory.  Many small CTAs an SM hide each other's trips to memory better than two stages of one do (31 against 27 us for
// 15,973 tokens of 8 heads of 128).  status is cleared before.
template <typename T, int D>
__global__ void __launch_bounds__(kWriteThreads)
    k_kv_write_many(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status, int per_seq,
                    int heads) {
    extern __shared__ __align__(16) uint8_t dyn[];
    __shared__ uint32_t smem[kWriteThreads / 32];
    const int rank = threadIdx.x, groups = (c.n_heads + heads - 1) / heads;
    const int64_t work = (int64_t)bt.n_seqs * per_seq * groups;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int h0 = (int)(w % groups) * heads, j = (int)(w / groups % per_seq), b = (int)(w / groups / per_seq);
        const SeqView s = load_seq(bt, b, true);
        bool ok = s.st == MP_OK;
        const int units = j < blocks_touched(c, s) ? 2 * min(heads, c.n_heads - h0) : 0;
        Place p;
        if (!ok || (units > 0 && !find<T>(c, bt, s, b, j, h0, false, k, v, p))) {
            status[b] = MP_EINVAL;  // whoever writes it writes the same
            continue;
        }
        constexpr int kIn = 16 / sizeof(T);  // values in 16 bytes
        const int step = kWriteThreads / (D / kIn), t_in = rank / (D / kIn), d_in = rank % (D / kIn) * kIn;
        for (int u = 0; u < units; ++u) {
            find<T>(c, bt, s, b, j, h0 + u / 2, u % 2, k, v, p);
            {
                T* to = reinterpret_cast<T*>(dyn) + rank * kIn;
                const T* at = static_cast<const T*>(p.x) + t_in * p.stride + d_in;
                for (int t = t_in; t < p.n; t += step, at += step * p.stride, to += kWriteThreads * kIn) {
                    if (wide) {
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(
                                         (uint32_t)__cvta_generic_to_shared(to)),
                                     "l"(at)
                                     : "memory");
                    } else {
#pragma unroll
                        for (int e = 0; e < kIn; ++e) to[e] = at[e];
                    }
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
            }
            const float old = p.first > 0 ? *p.scale : 0.f;
            __syncthreads();
            const uint4* x = reinterpret_cast<const uint4*>(dyn);
            const int chunks = p.n * (D / kIn);  // of 16 bytes
            uint32_t top = 0;
            for (int i = rank; i < chunks; i += kWriteThreads) {
                const uint4 w = x[i];
                top = join_word<T>(join_word<T>(top, w.x), w.y);
                top = join_word<T>(join_word<T>(top, w.z), w.w);
            }
            top = group_max<0>(join_end<T>(top), smem);
            const bool odd = top >= kInfBits<T>;
            if (odd) {
                ok = false;
                top = 0;
                for (int i = rank; i < chunks; i += kWriteThreads) {
                    const uint4 w = x[i];
                    top = join_finite<T>(join_finite<T>(top, w.x), w.y);
                    top = join_finite<T>(join_finite<T>(top, w.z), w.w);
                }
                top = group_max<0>(join_end<T>(top), smem);
            }
            if (u % 2 == 0) {
                const float inverse = settle<D, false, 0>(value_of<T>(top), old, p.first, p.bytes, p.scale, rank);
                if (odd) store_keys<T, D, true>(x, p, inverse, rank);
                else store_keys<T, D, false>(x, p, inverse, rank);
            } else {
                const float inverse = settle<D, true, 0>(value_of<T>(top), old, p.first, p.bytes, p.scale, rank);
                if (odd) store_columns<T, D, true>(x, p, inverse, rank);
                else store_columns<T, D, false>(x, p, inverse, rank);
            }
            __syncthreads();  // the next unit's values may come
        }
        if (!ok) status[b] = MP_EINVAL;
    }
}

// A warp reads one granule of one head back, keys and values.
template <typename T, int D>
__global__ void __launch_bounds__(kReadThreads)
    k_kv_read(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status, int per_seq) {
    const int lane = threadIdx.x % 32;
    const int64_t units = (int64_t)bt.n_seqs * per_seq * c.n_heads;
    const int64_t warps = (int64_t)gridDim.x * (kReadThreads / 32);
    for (int64_t u = (int64_t)blockIdx.x * (kReadThreads / 32) + threadIdx.x / 32; u < units; u += warps) {
        const int head = (int)(u % c.n_heads), b = (int)(u / c.n_heads / per_seq), j = (int)(u / c.n_heads % per_seq);
        const SeqView s = load_seq(bt, b, true);
        const int start = s.len - s.n;
        if (head == 0 && j == 0) {  // one warp looks the sequence's table over
            bool ok = s.st == MP_OK;
            if (s.n > 0)
                for (int col = start / c.block_tokens + lane; col <= (s.len - 1) / c.block_tokens; col += 32) {
                    const int p = __ldg(bt.table + (int64_t)b * bt.max_blocks + col);
                    ok &= p >= 0 && p < c.n_blocks;
                }
            ok = __all_sync(~0u, ok);
            if (lane == 0) status[b] = ok ? MP_OK : MP_EINVAL;
        }
        const int g = start / kGranule + j, base = g * kGranule;
        if (s.n == 0 || base >= s.len) continue;
        const int page = __ldg(bt.table + (int64_t)b * bt.max_blocks + base / c.block_tokens);
        if (page < 0 || page >= c.n_blocks) continue;
        const int from = max(start, base), past = min(s.len, base + kGranule);  // positions
        const int64_t at = block_byte(c, page, head) + (int64_t)(base % c.block_tokens) * D;
        const int64_t sc = (int64_t)page * c.n_heads + head;
        const float ks = __ldg(c.k_scale + sc), vs = __ldg(c.v_scale + sc);
        {
            T* out = static_cast<T*>(k.data) + (s.lo + base - start) * k.token_stride + head * k.head_stride;
#pragma unroll 4
            for (int i = lane; i < kGranule * (D / 16); i += 32) {
                const int t = i / (D / 16), d = i % (D / 16) * 16;
                if (base + t < from || base + t >= past) continue;
                const uint4 w = __ldg(reinterpret_cast<const uint4*>(c.k + at + key_byte<D>(t, d)));
                float x[16];
                e4m3_to_f32(w.x, x), e4m3_to_f32(w.y, x + 4), e4m3_to_f32(w.z, x + 8), e4m3_to_f32(w.w, x + 12);
#pragma unroll
                for (int q = 0; q < 16; ++q) x[q] *= ks;
                store_values<T, 16>(out + t * k.token_stride + d, wide, x);
            }
        }
        {
            // 16 tokens of 4 neighbouring values a thread
            T* out = static_cast<T*>(v.data) + (s.lo + base - start) * v.token_stride + head * v.head_stride;
            for (int i = lane; i < 2 * (D / 4); i += 32) {
                const int t0 = i / (D / 4) * 16, d = i % (D / 4) * 4;
                if (base + t0 + 16 <= from || base + t0 >= past) continue;
                uint4 w[4];
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    w[r] = __ldg(reinterpret_cast<const uint4*>(c.v + at + value_byte<D>(t0, d + r)));
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float x[4][4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) e4m3_to_f32(q == 0 ? w[r].x : q == 1 ? w[r].y : q == 2 ? w[r].z : w[r].w, x[r]);
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const int t = t0 + 4 * q + m;
                        if (base + t < from || base + t >= past) continue;
                        const float y[4] = {x[0][m] * vs, x[1][m] * vs, x[2][m] * vs, x[3][m] * vs};
                        store_values<T, 4>(out + t * v.token_stride + d, wide, y);
                    }
                }
            }
        }
    }
}

template <typename T, int D>
cudaError_t write_as(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                     int32_t* status, cudaStream_t stream) {
    const bool wide = rows_aligned(k) && rows_aligned(v);
    if (bt.max_tokens <= kWriteFewTokens) {
        k_kv_write_few<T, D><<<(unsigned)std::min(bt.n_seqs, 1 << 20), kWriteWarps * 32, 0, stream>>>(c, bt, k, v, wide, status);
        return cudaGetLastError();
    }
    cudaError_t e = cudaMemsetAsync(status, 0, sizeof(int32_t) * (size_t)bt.n_seqs, stream);
    if (e != cudaSuccess) return e;
    const int per_seq = (int)(((int64_t)bt.max_tokens + 2 * c.block_tokens - 2) / c.block_tokens);
    // as many heads a CTA as leave CTAs enough to fill the GPU several times over
    int heads = c.n_heads;
    const int64_t blocks = bt.n_tokens / c.block_tokens + bt.n_seqs;  // about as many as there are
    while (heads > 1 && blocks * ((c.n_heads + heads - 1) / heads) < kWriteCtas) heads = (heads + 1) / 2;
    const int64_t work = (int64_t)bt.n_seqs * per_seq * ((c.n_heads + heads - 1) / heads);
    const size_t smem = (size_t)c.block_tokens * D * sizeof(T);
    e = set_smem_limit((const void*)k_kv_write_many<T, D>, smem);
    if (e != cudaSuccess) return e;
    k_kv_write_many<T, D><<<(unsigned)std::min<int64_t>(work, 1 << 20), kWriteThreads, smem, stream>>>(c, bt, k, v, wide, status,
                                                                                                    per_seq, heads);
    return cudaGetLastError();
}

template <typename T, int D>
cudaError_t read_as(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                    int32_t* status, cudaStream_t stream) {
    const bool wide = rows_aligned(k) && rows_aligned(v);
    const int per_seq = (int)(((int64_t)bt.max_tokens + 2 * kGranule - 2) / kGranule);
    const int64_t units = (int64_t)bt.n_seqs * std::max(per_seq, 1) * c.n_heads;
    const int64_t ctas = (units + kReadThreads / 32 - 1) / (kReadThreads / 32);
    k_kv_read<T, D><<<(unsigned)std::min<int64_t>(ctas, 1 << 20), kReadThreads, 0, stream>>>(c, bt, k, v, wide, status,
                                                                                          std::max(per_seq, 1));
    return cudaGetLastError();
}

template <template <typename, int> class F, typename... A>
cudaError_t by_type(int32_t dtype, int32_t dim, A&... a) {
    if (dim == 64) {
        if (dtype == MP_F16) return F<__half, 64>::call(a...);
        if (dtype == MP_BF16) return F<__nv_bfloat16, 64>::call(a...);
        return F<float, 64>::call(a...);
    }
    if (dtype == MP_F16) return F<__half, 128>::call(a...);
    if (dtype == MP_BF16) return F<__nv_bfloat16, 128>::call(a...);
    return F<float, 128>::call(a...);
}
template <typename T, int D>
struct Write {
    template <typename... A>
    static cudaError_t call(A&... a) {
        return write_as<T, D>(a...);
    }
};
template <typename T, int D>
struct Read {
    template <typename... A>
    static cudaError_t call(A&... a) {
        return read_as<T, D>(a...);
    }
};

}  // namespace

cudaError_t launch_kv_write(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                            int32_t* status, cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    return by_type<Write>(k.dtype, c.head_dim, c, bt, k, v, status, stream);
}

cudaError_t launch_kv_read(const mp_kv_cache& c, const mp_kv_batch& bt, const mp_tokens& k, const mp_tokens& v,
                           int32_t* status, cudaStream_t stream) {
    if (bt.n_seqs == 0) return cudaSuccess;
    return by_type<Read>(k.dtype, c.head_dim, c, bt, k, v, status, stream);
}

}  // namespace mp
