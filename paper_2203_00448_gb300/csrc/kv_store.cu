// kv_store.cu -- mp_kv_write and mp_kv_read: tokens into and out of the cache's
// 8-bit blocks.
//
// A block and head is stored under one scale s = 2^e, the least power of two with
// max |x| <= 448 s (448 is the largest e4m3 value).  Dividing by it is exact, so a
// stored value carries the one rounding to e4m3's 4 significant bits, whatever the
// scale; when a later token makes the scale grow, earlier bytes are rounded again,
// which loses bits only among subnormals.  Both kernels move each byte once and
// are bound by memory (prompts) or by the latency of a launch (single tokens).
#include <algorithm>

#include "kv.cuh"

namespace mp {
namespace {

constexpr int kWriteWarps = 16;          // few tokens: one CTA a sequence, a warp a block, head and array
constexpr int kWriteThreads = 128;       // many tokens: one CTA a block, head and array
constexpr int32_t kWriteFewTokens = 16;  // ... above this many tokens a sequence
constexpr int kReadThreads = 256;

// The larger of all lanes' values, over a warp or a CTA of kGroup threads.
template <int kGroup>
__device__ __forceinline__ float group_max(float x, float* smem) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(~0u, x, o));
    if (kGroup > 32) {
        __syncthreads();  // smem's last use
        if (threadIdx.x % 32 == 0) smem[threadIdx.x / 32] = x;
        __syncthreads();
        x = smem[0];
#pragma unroll
        for (int w = 1; w < kGroup / 32; ++w) x = fmaxf(x, smem[w]);
    }
    return x;
}

// 2^e with the least e in [-60, 120] such that a <= 448 * 2^e = 1.75 * 2^(e + 8).
__device__ __forceinline__ float scale_of(float a) {
    const uint32_t u = __float_as_uint(a);
    int e = (int)(u >> 23) - 135 + ((u & 0x7fffffu) > 0x600000u);
    e = min(max(e, -60), 120);
    return __uint_as_float((uint32_t)(e + 127) << 23);
}

// NaN counts as 0 where it is stored; ok is cleared for it and for infinities.
__device__ __forceinline__ float storable(float x) { return x == x ? x : 0.f; }

// 4 stored bytes under another scale (ratio: the old one over the new one).
__device__ __forceinline__ uint32_t rescale(uint32_t w, float ratio) {
    float x[4];
    e4m3_to_f32(w, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] *= ratio;
    return f32_to_e4m3(x);
}

// kGroup threads put n tokens (x: the first one's values of this head) into slots
// [first, first + n) of one block and head of one array; slots below first hold
// earlier tokens.  Returns whether this thread met only finite values.
template <typename T, int D, bool kValues, int kGroup>
__device__ bool store_block(const T* x, int64_t stride, bool wide, int first, int n, uint8_t* bytes, float* scale_at,
                            int rank, float* smem) {
    bool ok = true;
    float top = 0.f;
    const float old = first > 0 ? *scale_at : 0.f;
    for (int i = rank; i < n * (D / 16); i += kGroup) {
        float v[16];
        load_values<T, 16>(x + (i / (D / 16)) * stride + i % (D / 16) * 16, wide, v);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float a = fabsf(v[k]);
            const bool fine = a <= 3.402823466e38f;
            ok = ok && fine;
            top = fmaxf(top, fine ? a : 0.f);
        }
    }
    top = group_max<kGroup>(top, smem);
    const float fresh = scale_of(top), scale = fmaxf(fresh, old), inverse = __fdiv_rn(1.f, scale);
    const bool grows = first > 0 && scale > old;
    const float ratio = grows ? __fdiv_rn(old, scale) : 1.f;
    if (rank == 0 && !(first > 0 && scale == old)) *scale_at = scale;
    const int past = first + n;
    if (!kValues) {
        const int from = grows ? 0 : first;
        for (int i = rank; i < (past - from) * (D / 16); i += kGroup) {
            const int t = from + i / (D / 16), d = i % (D / 16) * 16;
            uint4* at = reinterpret_cast<uint4*>(bytes + key_byte<D>(t, d));
            uint4 w;
            if (t < first) {
                w = *at;
                w.x = rescale(w.x, ratio), w.y = rescale(w.y, ratio), w.z = rescale(w.z, ratio), w.w = rescale(w.w, ratio);
            } else {
                float v[16];
                load_values<T, 16>(x + (t - first) * stride + d, wide, v);
#pragma unroll
                for (int k = 0; k < 16; ++k) v[k] = storable(v[k]) * inverse;
                w = make_uint4(f32_to_e4m3(v), f32_to_e4m3(v + 4), f32_to_e4m3(v + 8), f32_to_e4m3(v + 12));
            }
            *at = w;
        }
        return ok;
    }
    // a thread has 16 tokens of 2 neighbouring values, 2 x 16 stored bytes
    const int from = grows ? 0 : first / 16;
    for (int i = rank; i < ((past + 15) / 16 - from) * (D / 2); i += kGroup) {
        const int t0 = (from + i / (D / 2)) * 16, d = i % (D / 2) * 2;
        uint8_t* at = bytes + value_byte<D>(t0, d);
        float v[2][16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            float pair[2] = {0.f, 0.f};
            if (t0 + k >= first && t0 + k < past) load_values<T, 2>(x + (t0 + k - first) * stride + d, wide, pair);
            v[0][k] = storable(pair[0]) * inverse, v[1][k] = storable(pair[1]) * inverse;
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            uint32_t w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = f32_to_e4m3(v[r] + 4 * k);
            uint4* row = reinterpret_cast<uint4*>(at + 16 * r);
            if (t0 < first || t0 + 16 > past) {
                // part of it only: earlier tokens under the new scale, slots without a token as they were
                const uint4 had = *row;
                const uint32_t h[4] = {had.x, had.y, had.z, had.w};
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const uint32_t again = grows ? rescale(h[k], ratio) : h[k];
                    uint32_t m = 0, o = 0;  // bytes of new tokens, of earlier ones
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int t = t0 + 4 * k + j;
                        if (t < first) o |= 0xffu << (8 * j);
                        else if (t < past) m |= 0xffu << (8 * j);
                    }
                    w[k] = (w[k] & m) | (again & o) | (h[k] & ~(m | o));
                }
            }
            *row = make_uint4(w[0], w[1], w[2], w[3]);
        }
    }
    return ok;
}

// One block, head and array of sequence b; j counts the blocks that the call touches.
template <typename T, int D, int kGroup>
__device__ bool write_unit(const mp_kv_cache& c, const mp_kv_batch& bt, const SeqView& s, int b, int j, int head,
                           bool values, const mp_tokens& k, const mp_tokens& v, bool wide, int rank, float* smem) {
    const int start = s.len - s.n, col = start / c.block_tokens + j, base = col * c.block_tokens;
    const int page = __ldg(bt.table + (int64_t)b * bt.max_blocks + col);
    if (page < 0 || page >= c.n_blocks) return false;
    const int first = max(start - base, 0), n = min(s.len - base, c.block_tokens) - first;
    const mp_tokens& t = values ? v : k;
    const T* x = static_cast<const T*>(t.data) + (s.lo + (base + first - start)) * t.token_stride + head * t.head_stride;
    const int64_t at = block_byte(c, page, head), sc = (int64_t)page * c.n_heads + head;
    return values ? store_block<T, D, true, kGroup>(x, t.token_stride, wide, first, n, c.v + at, c.v_scale + sc, rank, smem)
                  : store_block<T, D, false, kGroup>(x, t.token_stride, wide, first, n, c.k + at, c.k_scale + sc, rank, smem);
}

__device__ __forceinline__ int blocks_touched(const mp_kv_cache& c, const SeqView& s) {
    return s.n == 0 ? 0 : (s.len - 1) / c.block_tokens - (s.len - s.n) / c.block_tokens + 1;
}

// Few tokens a sequence: one CTA a sequence, so that its status has one writer.
template <typename T, int D>
__global__ void __launch_bounds__(kWriteWarps * 32)
    k_kv_write_few(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status) {
    for (int b = blockIdx.x; b < bt.n_seqs; b += gridDim.x) {
        const SeqView s = load_seq(bt, b, true);
        const int tasks = blocks_touched(c, s) * c.n_heads * 2;
        bool ok = s.st == MP_OK;
        for (int u = threadIdx.x / 32; u < tasks; u += kWriteWarps)
            ok &= write_unit<T, D, 32>(c, bt, s, b, u / (2 * c.n_heads), u / 2 % c.n_heads, u % 2, k, v, wide,
                                       threadIdx.x % 32, nullptr);
        const bool bad = __syncthreads_or(!ok);
        if (threadIdx.x == 0) status[b] = bad ? MP_EINVAL : MP_OK;
    }
}

// Many tokens: units of one block, head and array over the whole grid; status is
// cleared before.
template <typename T, int D>
__global__ void __launch_bounds__(kWriteThreads)
    k_kv_write_many(mp_kv_cache c, mp_kv_batch bt, mp_tokens k, mp_tokens v, bool wide, int32_t* status, int per_seq) {
    __shared__ float smem[kWriteThreads / 32];
    const int64_t units = (int64_t)bt.n_seqs * per_seq * c.n_heads * 2;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const bool values = u % 2;
        const int64_t r = u / 2;
        const int head = (int)(r % c.n_heads), j = (int)(r / c.n_heads % per_seq), b = (int)(r / c.n_heads / per_seq);
        const SeqView s = load_seq(bt, b, true);
        bool ok = s.st == MP_OK;
        if (j < blocks_touched(c, s))
            ok &= write_unit<T, D, kWriteThreads>(c, bt, s, b, j, head, values, k, v, wide, threadIdx.x, smem);
        if (!ok) status[b] = MP_EINVAL;  // whoever writes it writes the same
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
    const int64_t units = (int64_t)bt.n_seqs * per_seq * c.n_heads * 2;
    k_kv_write_many<T, D>
        <<<(unsigned)std::min<int64_t>(units, 1 << 20), kWriteThreads, 0, stream>>>(c, bt, k, v, wide, status, per_seq);
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
