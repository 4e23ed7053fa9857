// The target of a verification: softmax of the logits mixed with the neighbours' weights (ralm_knnlm_target).
//
// Two passes over a row: its largest logit and the sum of exponentials under a running maximum, then the probabilities; what bounds them is
// memory, the second pass finds the row in L2.  A token's neighbours are added up by one thread in their order, on the
// probability formed again in fp32, so that the result is rounded once and does not depend on which thread came first.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

constexpr int NT = 1024;

// 8 numbers from anywhere that their type may lie: rows of an odd number of entries are aligned to nothing else (the hardware takes such accesses whole)
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int DT>
__device__ __forceinline__ void load8(const void *p, int64_t at, float (&x)[8])
{
    if constexpr (DT == DT_F32) {
        const f32x4_any *s = reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + at);
        const f32x4_any a = s[0], b = s[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
    } else {
        const u32x4_any w = *reinterpret_cast<const u32x4_any *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (DT == DT_BF16) x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
            else x[2 * j] = f16_bits_to_f32(w[j] & 0xffffu), x[2 * j + 1] = f16_bits_to_f32(w[j] >> 16);
        }
    }
}
template <int DT>
__device__ __forceinline__ float load1(const void *p, int64_t at)
{
    if constexpr (DT == DT_F32) return static_cast<const float *>(p)[at];
    const uint32_t b = static_cast<const uint16_t *>(p)[at];
    return DT == DT_BF16 ? __uint_as_float(b << 16) : f16_bits_to_f32(b);
}
template <int DT>
__device__ __forceinline__ void store1(void *p, int64_t at, float x)
{
    if constexpr (DT == DT_F32) static_cast<float *>(p)[at] = x;
    else if constexpr (DT == DT_BF16) static_cast<__bf16 *>(p)[at] = (__bf16)x;
    else static_cast<_Float16 *>(p)[at] = (_Float16)x;
}
template <int DT>
__device__ __forceinline__ void store8(void *p, int64_t at, const float (&x)[8])
{
    if constexpr (DT == DT_F32) {
        f32x4_any *d = reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + at);
        const f32x4_any a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        d[0] = a;
        d[1] = b;
    } else {
        u32x4_any w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if constexpr (DT == DT_BF16)
                w[j] = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]) << 16;
            else
                w[j] = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]) << 16;
        }
        *reinterpret_cast<u32x4_any *>(static_cast<uint16_t *>(p) + at) = w;
    }
}

// largest logit and sum of exp((x - largest) / T) of what a thread has seen; nothing: -inf, 0
struct Seen {
    float top, sum;
    __device__ __forceinline__ void join(float t, float s, float inv)
    {
        const float m = fmaxf(top, t);   // (a NaN lies in s)
        const float a = top == m ? sum : sum * expf((top - m) * inv), b = t == m ? s : s * expf((t - m) * inv);
        // -inf on both sides: nothing, or what made the sum NaN
        sum = a + b;
        top = m;
    }
};

template <int DT, int DO>
__global__ __launch_bounds__(NT) void target_kernel(const TargetParams p)
{
    __shared__ float tops[NT / 64], sums[NT / 64];
    __shared__ int32_t near_token[RALM_MAX_K];
    __shared__ float near_weight[RALM_MAX_K];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t row = blockIdx.x;
    const float inv = p.inv_temperature;
    const void *x = DT == DT_F32 ? static_cast<const void *>(static_cast<const float *>(p.logits) + row * p.logits_stride)
                                 : static_cast<const void *>(static_cast<const uint16_t *>(p.logits) + row * p.logits_stride);
    void *out = DO == DT_F32 ? static_cast<void *>(static_cast<float *>(p.out) + row * p.out_stride)
                             : static_cast<void *>(static_cast<uint16_t *>(p.out) + row * p.out_stride);
    const int V = p.V, V8 = V & ~7;
    Seen seen = {-__builtin_inff(), 0.f};
    auto take = [&](const float *y, int n) {
        float m = y[0];
        for (int j = 1; j < n; ++j) m = fmaxf(m, y[j]);
        float s = 0.f;
        for (int j = 0; j < n; ++j) s += y[j] == -__builtin_inff() ? 0.f : expf((y[j] - m) * inv);
        seen.join(m, s, inv);
    };
    for (int v = tid * 8; v < V8; v += NT * 8) {
        float y[8];
        load8<DT>(x, v, y);
        take(y, 8);
    }
    if (tid < V - V8) {
        const float y = load1<DT>(x, V8 + tid);
        take(&y, 1);
    }
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const float t = __shfl_xor(seen.top, s, 64), u = __shfl_xor(seen.sum, s, 64);
        seen.join(t, u, inv);
    }
    if (lane == 0) tops[wave] = seen.top, sums[wave] = seen.sum;
    for (int j = tid; j < p.k; j += NT) near_token[j] = p.tokens[row * p.k + j], near_weight[j] = p.weights[row * p.k + j];
    __syncthreads();
    seen = {-__builtin_inff(), 0.f};
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) seen.join(tops[w], sums[w], inv);
    const float share = p.share ? p.share[row] : p.share_all;
    const float top = seen.top, per = top == -__builtin_inff() && seen.sum == 0.f ? 0.f : (1.f - share) / seen.sum;
    auto prob = [&](float y) { return (y == -__builtin_inff() ? 0.f : expf((y - top) * inv)) * per; };   // per is NaN where the row is
    // a token's weights, by the thread of the first neighbour that has it; its logit is read before the row may be written over
    float mine = 0.f;
    int32_t token = -1;
    if (tid < p.k) {
        token = near_token[tid];
        if (token < 0 || token >= V) token = -1;
        for (int j = 0; token >= 0 && j < p.k; ++j) {
            if (near_token[j] != token) continue;
            if (j < tid) token = -1;
            else mine += near_weight[j];
        }
        if (token >= 0) mine = prob(load1<DT>(x, token)) + share * mine;
    }
    __syncthreads();
    for (int v = tid * 8; v < V8; v += NT * 8) {
        float y[8];
        load8<DT>(x, v, y);
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = prob(y[j]);
        store8<DO>(out, v, y);
    }
    if (tid < V - V8) store1<DO>(out, V8 + tid, prob(load1<DT>(x, V8 + tid)));
    __syncthreads();
    if (token >= 0) store1<DO>(out, token, mine);
}

template <int DT>
hipError_t launch(const TargetParams &p, hipStream_t stream)
{
    const dim3 grid((unsigned)p.Q);
    if (p.out_dtype == DT_F32) target_kernel<DT, DT_F32><<<grid, NT, 0, stream>>>(p);
    else if (p.out_dtype == DT_BF16) target_kernel<DT, DT_BF16><<<grid, NT, 0, stream>>>(p);
    else target_kernel<DT, DT_F16><<<grid, NT, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_knnlm_target(const TargetParams &p, hipStream_t stream)
{
    return p.dtype == DT_F32 ? launch<DT_F32>(p, stream) : p.dtype == DT_BF16 ? launch<DT_BF16>(p, stream) : launch<DT_F16>(p, stream);
}

}  // namespace ralm
