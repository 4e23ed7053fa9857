// A block's output into the residual stream and the stream's norm (ralm_residual_norm).
//
//   y = x or norm(x) post_weight + post_bias;  s = residual + scale gate y;  out = norm(s) weight + bias
//
// A row is read once and stays in registers as fp32 through all of it, statistics included: what bounds the kernel is memory.  The
// variance of a layer norm is the mean of squared differences from the mean, a second sum over the registers, and not the
// difference of two large sums.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

__device__ __forceinline__ float load1(const void *p, int dt, int64_t at)
{
    if (dt == DT_F32) return static_cast<const float *>(p)[at];
    const uint32_t b = static_cast<const uint16_t *>(p)[at];
    return dt == DT_BF16 ? __uint_as_float(b << 16) : f16_bits_to_f32(b);
}
__device__ __forceinline__ void store1(void *p, int dt, int64_t at, float x)
{
    if (dt == DT_F32) static_cast<float *>(p)[at] = x;
    else if (dt == DT_BF16) static_cast<__bf16 *>(p)[at] = (__bf16)x;
    else static_cast<_Float16 *>(p)[at] = (_Float16)x;
}
__device__ __forceinline__ void load8(const void *p, int dt, int64_t at, float (&x)[8])
{
    if (dt == DT_F32) {   // uniform
        const f32x4 *s = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + at);
        const f32x4 a = s[0], b = s[1];
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = a[j], x[4 + j] = b[j];
    } else {
        const uint4 v = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
        if (dt == DT_BF16) {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[2 * j] = __uint_as_float(w[j] << 16), x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[2 * j] = f16_bits_to_f32(w[j] & 0xffffu), x[2 * j + 1] = f16_bits_to_f32(w[j] >> 16);
        }
    }
}
__device__ __forceinline__ void store8(void *p, int dt, int64_t at, const float (&x)[8])
{
    if (dt == DT_F32) {
        f32x4 *d = reinterpret_cast<f32x4 *>(static_cast<float *>(p) + at);
        const f32x4 a = {x[0], x[1], x[2], x[3]}, b = {x[4], x[5], x[6], x[7]};
        d[0] = a;
        d[1] = b;
    } else {
        uint32_t w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (dt == DT_BF16)
                w[j] = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]) << 16;
            else
                w[j] = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]) << 16;
        }
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

template <int C>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), C, 0xf, 0xf, false));
}
// sum over the TPR threads of a row; `part` holds a word per wave and is used by two sums in turn (`which`), so one barrier a sum is enough
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float *part, int which)
{
    v = dpp_add<0xB1>(v);
    v = dpp_add<0x4E>(v);
    v = dpp_add<0x141>(v);
    v = dpp_add<0x140>(v);
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 4; ++r) s += __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), r * 16));
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        part += (which & 1) * W;
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
        __syncthreads();
        s = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) s += part[w];
    }
    return s;
}

// TPR threads a row, NV pieces of 8 numbers a thread.  VEC: pieces are loaded whole (D and all strides multiples of 8, bases of 16 bytes); otherwise
// number by number, neighbouring threads neighbouring numbers
template <int TPR, int NV, bool VEC>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(const ralm_norm_t p)
{
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1;   // rows of a workgroup
    __shared__ float part[TPR > 64 ? 2 * (TPR / 64) : 1];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (row >= p.T) return;   // whole waves, and no barrier where a workgroup has several rows
    const int D = p.D;
    const float mean_of = 1.f / (float)D;
    auto at = [&](int v, int j) { return VEC ? (v * TPR + t) * 8 + j : (v * 8 + j) * TPR + t; };
    auto load = [&](const void *s, int dt, int64_t base, int v, float (&x)[8], float other) {
        if constexpr (VEC) {
            if (at(v, 0) < D) {
                load8(s, dt, base + at(v, 0), x);
                return;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = other;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = at(v, j) < D ? load1(s, dt, base + at(v, j)) : other;
        }
    };
    auto store = [&](void *d, int dt, int64_t base, int v, const float (&x)[8]) {
        if constexpr (VEC) {
            if (at(v, 0) < D) store8(d, dt, base + at(v, 0), x);
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at(v, j) < D) store1(d, dt, base + at(v, j), x[j]);
        }
    };
    int sums = 0;
    float s[NV][8];
    // the norm of the row in s, times w plus b; numbers behind D are 0 before and count for nothing
    auto normed = [&](const void *w, const void *b) {
        float mean = 0.f;
        if (p.kind == RALM_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += s[v][j];
            mean = row_sum<TPR>(sum, part, sums++) * mean_of;
        }
        float sq = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = at(v, j) < D ? s[v][j] - mean : 0.f;
                sq += d * d;
            }
        const float r = 1.f / sqrtf(row_sum<TPR>(sq, part, sums++) * mean_of + p.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float g[8], o[8];
            if (w) load(w, p.param_dtype, 0, v, g, 0.f);
            if (b) load(b, p.param_dtype, 0, v, o, 0.f);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float y = (s[v][j] - mean) * r;
                if (w) y *= g[j];
                if (b) y += o[j];
                s[v][j] = at(v, j) < D ? y : 0.f;
            }
        }
    };
#pragma unroll
    for (int v = 0; v < NV; ++v) load(p.x, p.x_dtype, row * p.x_stride, v, s[v], 0.f);
    if (p.post) normed(p.post_weight, p.post_bias);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float g[8], r[8];
        if (p.gate) load(p.gate, p.x_dtype, p.gate_rows ? row * p.gate_stride : 0, v, g, 0.f);
        if (p.residual) load(p.residual, p.sum_dtype, row * p.residual_stride, v, r, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float y = s[v][j] * p.scale;
            if (p.gate) y *= g[j];
            if (p.residual) y += r[j];
            s[v][j] = at(v, j) < D ? y : 0.f;
        }
        if (p.sum) store(p.sum, p.sum_dtype, row * p.sum_stride, v, s[v]);
    }
    if (!p.out) return;
    normed(p.weight, p.bias);
#pragma unroll
    for (int v = 0; v < NV; ++v) store(p.out, p.out_dtype, row * p.out_stride, v, s[v]);
}

template <int TPR, int NV>
hipError_t launch(const ralm_norm_t &p, bool vec, hipStream_t stream)
{
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1, NT = TPR < 256 ? 256 : TPR;
    const dim3 grid((unsigned)((p.T + RPW - 1) / RPW));
    if (vec) norm_kernel<TPR, NV, true><<<grid, NT, 0, stream>>>(p);
    else norm_kernel<TPR, NV, false><<<grid, NT, 0, stream>>>(p);
    return hipGetLastError();
}

// Whether pieces of 8 numbers can be loaded whole: strides of rows, and bases
bool whole_pieces(const ralm_norm_t &p)
{
    auto fine = [](const void *a, int64_t stride) { return (reinterpret_cast<uintptr_t>(a) & 15) == 0 && stride % 8 == 0; };
    return p.D % 8 == 0 && fine(p.x, p.x_stride) && fine(p.residual, p.residual ? p.residual_stride : 0) && fine(p.sum, p.sum ? p.sum_stride : 0) &&
           fine(p.out, p.out ? p.out_stride : 0) && fine(p.gate, p.gate && p.gate_rows ? p.gate_stride : 0) && fine(p.weight, 0) && fine(p.bias, 0) &&
           fine(p.post_weight, 0) && fine(p.post_bias, 0);
}

}  // namespace

hipError_t launch_residual_norm(const ralm_norm_t &p, hipStream_t stream)
{
    const bool vec = whole_pieces(p);
    if (p.D <= 512) return launch<64, 1>(p, vec, stream);
    if (p.D <= 2048) return launch<256, 1>(p, vec, stream);
    if (p.D <= 4096) return launch<256, 2>(p, vec, stream);
    if (p.D <= 8192) return launch<256, 4>(p, vec, stream);
    if (p.D <= 16384) return launch<1024, 2>(p, vec, stream);
    return launch<1024, 4>(p, vec, stream);
}

}  // namespace ralm
