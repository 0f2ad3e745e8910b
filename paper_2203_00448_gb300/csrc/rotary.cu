// rotary.cu -- mp_rotary: queries and keys turned to their positions, or gradients turned back.
//
// The angle of position p and pair i is p times a frequency.  In turns, and as a fraction of 2^64, that is one integer
// product whose overflow is the whole turns: the reduction is exact, no position is too far.  What the angle is off by is p times
// the table's error: Rotary's doubles leave less than 2^-52 of a frequency's turns, for the first pair (0.16 turns a position) 2^-54
// turns, 2^-26 at position 2^28.
// What is left of it after the nearest quarter turn goes to sincospi in 32 bits.
//
// A token's angles serve all its heads: a CTA puts those of a few tokens into shared memory and then streams the heads.
//
// Measured: 15,973 tokens of 32 heads of 64 in 32 bits, half of each turned (262 MB), 43 us of GPU time, 6.1 TB/s, 90% of a copy's
// rate; prompts in 16 bits, whole heads, from a projection's output: 8,000 tokens of 40 heads of 128 (164 MB) 26 us, 6.3 TB/s, 15,973 50
// us, 6.6 TB/s, 97%; 8 tokens of 16 heads 4 us.
#include <algorithm>

#include "kv_attend.cuh"

namespace mp {
namespace {

constexpr int kThreads = 256;
constexpr int kTokens = 4;  // of a CTA where there are many

struct RotaryArgs {
    mp_rotation r;
    const int32_t* positions;
    int64_t n_tokens;
    mp_tokens in[2], out[2];  // queries, keys
    int32_t heads[2];
    int32_t head_dim, inverse, tokens;
};

// Cosine and sine of 2 pi phase / 2^64.
__device__ __forceinline__ float2 cos_sin(uint64_t phase) {
    const uint64_t quarters = (phase + (1ull << 61)) >> 62;
    const int64_t rest = (int64_t)(phase - (quarters << 62));  // within an eighth of a turn
    float s, c;
    sincospif((float)(int32_t)(rest >> 30) * 0x1p-33f, &s, &c);
    const float x = quarters & 1 ? -s : c, y = quarters & 1 ? c : s;
    return quarters & 2 ? make_float2(-x, -y) : make_float2(x, y);
}

// W pairs of a head from x to y.
template <typename T, int W, bool kHalf>
__device__ __forceinline__ void turn(const T* x, T* y, int half, const float2* cs, bool back) {
    T u[W], v[W];
    Pack<T, W> a = *reinterpret_cast<const Pack<T, W>*>(x), b = *reinterpret_cast<const Pack<T, W>*>(x + (kHalf ? half : W));
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const T first = kHalf ? a.x[i] : 2 * i < W ? a.x[2 * i % W] : b.x[2 * i % W];
        const T second = kHalf ? b.x[i] : 2 * i + 1 < W ? a.x[(2 * i + 1) % W] : b.x[(2 * i + 1) % W];
        const float c = cs[i].x, s = back ? -cs[i].y : cs[i].y, p = to_f32(first), q = to_f32(second);
        u[i] = from_f32<T>(p * c - q * s), v[i] = from_f32<T>(p * s + q * c);
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if (kHalf) {
            a.x[i] = u[i], b.x[i] = v[i];
        } else {
            (2 * i < W ? a : b).x[2 * i % W] = u[i];
            (2 * i + 1 < W ? a : b).x[(2 * i + 1) % W] = v[i];
        }
    }
    *reinterpret_cast<Pack<T, W>*>(y) = a;
    *reinterpret_cast<Pack<T, W>*>(y + (kHalf ? half : W)) = b;
}

template <typename T, int W, bool kHalf>
__global__ void __launch_bounds__(kThreads) k_rotary(RotaryArgs a) {
    extern __shared__ __align__(16) float2 cs[];  // [tokens][dim / 2]
    const int half = a.r.dim / 2, turned = half / W, units = a.head_dim / (2 * W);  // of a head: W pairs each
    const int per_token = (a.heads[0] + a.heads[1]) * units;
    after_previous();
    let_next_begin();
    for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.n_tokens; t0 += (int64_t)gridDim.x * a.tokens) {
        const int n = (int)min((int64_t)a.tokens, a.n_tokens - t0);
        for (int i = threadIdx.x; i < n * half; i += kThreads) {
            const int t = i / half;
            const float2 x = cos_sin((uint64_t)__ldg(a.r.turns + (i - t * half)) * (uint64_t)(int64_t)__ldg(a.positions + t0 + t));
            cs[i] = make_float2(x.x * a.r.amplitude, x.y * a.r.amplitude);
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n * per_token; i += kThreads) {
            const int t = i / per_token, at = i - t * per_token;
            int head = at / units;
            const int u = at - head * units, which = head >= a.heads[0];
            head -= which ? a.heads[0] : 0;
            const T* x = static_cast<const T*>(a.in[which].data) + (t0 + t) * a.in[which].token_stride + head * a.in[which].head_stride;
            T* y = static_cast<T*>(a.out[which].data) + (t0 + t) * a.out[which].token_stride + head * a.out[which].head_stride;
            if (u < turned) {
                const int o = kHalf ? u * W : u * 2 * W;
                turn<T, W, kHalf>(x + o, y + o, half, cs + t * half + u * W, a.inverse);
            } else {
                const int o = u * 2 * W;  // (the turned part is as long in either layout)
                *reinterpret_cast<Pack<T, W>*>(y + o) = *reinterpret_cast<const Pack<T, W>*>(x + o);
                *reinterpret_cast<Pack<T, W>*>(y + o + W) = *reinterpret_cast<const Pack<T, W>*>(x + o + W);
            }
        }
        __syncthreads();
    }
}

template <typename T, int W>
cudaError_t rotary_as(RotaryArgs a, cudaStream_t stream) {
    // few tokens: a CTA each, so that more SMs work (40 heads of 128 in 16 bits, GPU time with 1 and with 4 tokens a CTA: 304 tokens 2.0
    // and 4.1 us, 912 4.1 and 5.8, 1,216 4.9 and 5.8, 1,824 8.0 and 7.7, 4,864 17.6 and 14.4, 15,973 58 and 50)
    a.tokens = a.n_tokens >= 2 * kTokens * kSms ? kTokens : 1;
    const int64_t ctas = std::min<int64_t>((a.n_tokens + a.tokens - 1) / a.tokens, 1 << 20);
    const size_t smem = sizeof(float2) * (size_t)a.tokens * (a.r.dim / 2);
    return a.r.layout == MP_ROTARY_HALF ? launch_close(k_rotary<T, W, true>, (int)ctas, kThreads, smem, stream, a)
                                        : launch_close(k_rotary<T, W, false>, (int)ctas, kThreads, smem, stream, a);
}
template <typename T>
cudaError_t rotary_wide(const RotaryArgs& a, bool wide, cudaStream_t stream) {
    // units of 8 or 4 pairs where rows and parts of a head lie that way, else a pair at a time
    const int32_t half = a.r.dim / 2, rest = a.head_dim - a.r.dim;
    if (wide && half % 8 == 0 && rest % 16 == 0) return rotary_as<T, 8>(a, stream);
    if (wide && half % 4 == 0 && rest % 8 == 0) return rotary_as<T, 4>(a, stream);
    return rotary_as<T, 1>(a, stream);
}

}  // namespace

cudaError_t launch_rotary(const mp_rotation& r, const int32_t* positions, int64_t n_tokens, int32_t head_dim, const mp_tokens* q,
                          const mp_tokens* k, const mp_tokens* q_out, const mp_tokens* k_out, int32_t inverse, cudaStream_t stream) {
    if (n_tokens == 0) return cudaSuccess;
    RotaryArgs a = {};
    a.r = r, a.positions = positions, a.n_tokens = n_tokens, a.head_dim = head_dim, a.inverse = inverse;
    bool wide = true;
    const mp_tokens* in[2] = {q, k};
    const mp_tokens* out[2] = {q_out, k_out};
    int32_t dtype = MP_F16;
    for (int i = 0; i < 2; ++i)
        if (in[i] != nullptr) {
            a.in[i] = *in[i], a.out[i] = *out[i], a.heads[i] = in[i]->n_heads, dtype = in[i]->dtype;
            wide = wide && rows_aligned(*in[i]) && rows_aligned(*out[i]);
        }
    if (dtype == MP_F16) return rotary_wide<__half>(a, wide, stream);
    if (dtype == MP_BF16) return rotary_wide<__nv_bfloat16>(a, wide, stream);
    return rotary_wide<float>(a, wide, stream);
}

}  // namespace mp
