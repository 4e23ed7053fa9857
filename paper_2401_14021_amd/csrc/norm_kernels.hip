// A block's output into the residual stream and the stream's norm (ralm_residual_norm).
//
//   y = x or norm(x) post_weight + post_bias;  s = residual + scale gate y;  out = norm(s) weight + bias
//
// A row is read once and stays in registers as fp32 through all of it, statistics included: what bounds the kernel is memory (8192 rows of 4096, bf16, norms on both sides
// and a gate: 46 us, 5.8 TB/s, above a large copy's rate: part of the rows come from the last-level cache).  Not so beyond 16384 numbers a row: 1024 threads have 128
// registers each, and in all forms but those of bf16 or fp16 alone the compiler spills 8 to 120 of them, in the one for any types and lengths 231 (1000 rows of 32768, norms on both sides, us, at 5.1
// TB/s in brackets: bf16 56 (51), bf16 with an fp32 stream 95 (77), fp32 181 (103); 32767, bf16 with an fp32 stream 384 (77)).  The
// variance of a layer norm is the mean of squared differences from the mean, a second sum over the registers, and not the
// difference of two large sums.
#include <type_traits>

#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

__device__ __forceinline__ void store1(void *p, int dt, int64_t at, float x)
{
    if (dt == DT_F32) static_cast<float *>(p)[at] = x;
    else if (dt == DT_BF16) static_cast<__bf16 *>(p)[at] = (__bf16)x;
    else static_cast<_Float16 *>(p)[at] = (_Float16)x;
}
// 8 numbers from anywhere that their type may lie (the hardware takes such accesses whole): rows of an odd length need no form of their own
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

// 8 numbers as they lie in memory: a load that does not wait, whatever the type; they are widened where they are used.  (Widened at once behind a branch on the
// type, every load was waited for by itself: rows of 4096 as two pieces a thread took 78 us, as one piece 56.)
struct Raw {
    uint32_t w[8];
    __device__ __forceinline__ void load(const void *p, bool f32, int64_t at, int n)   // the first n of them, zeros behind
    {
        if (n >= 8) {
            const u32x4_any a = *reinterpret_cast<const u32x4_any *>(static_cast<const char *>(p) + at * (f32 ? 4 : 2));
            u32x4_any b = {0, 0, 0, 0};
            if (f32) b = *reinterpret_cast<const u32x4_any *>(static_cast<const char *>(p) + at * 4 + 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = a[j], w[4 + j] = b[j];
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n) break;
                if (f32) w[j] = static_cast<const uint32_t *>(p)[at + j];
                else w[j / 2] |= (uint32_t) static_cast<const uint16_t *>(p)[at + j] << (j & 1 ? 16 : 0);
            }
        }
    }
    __device__ __forceinline__ void load_whole(const void *p, bool f32, int64_t at)
    {
        const u32x4_any a = *reinterpret_cast<const u32x4_any *>(static_cast<const char *>(p) + at * (f32 ? 4 : 2));
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = a[j];
        if (!f32) return;
        const u32x4_any b = *reinterpret_cast<const u32x4_any *>(static_cast<const char *>(p) + at * 4 + 16);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[4 + j] = b[j];
    }
    __device__ __forceinline__ float at(int j, int dt) const
    {
        if (dt == DT_F32) return __uint_as_float(w[j]);
        const uint32_t b = j & 1 ? w[j / 2] >> 16 : w[j / 2] & 0xffffu;
        return dt == DT_BF16 ? __uint_as_float(b << 16) : f16_bits_to_f32(b);
    }
};
__device__ __forceinline__ void store8(void *p, int dt, int64_t at, const float (&x)[8])
{
    u32x4_any w;
    if (dt == DT_F32) {
        u32x4_any *d = reinterpret_cast<u32x4_any *>(static_cast<float *>(p) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[j]);
        d[0] = w;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = __float_as_uint(x[4 + j]);
        d[1] = w;
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if (dt == DT_BF16)
            w[j] = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]) << 16;
        else
            w[j] = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]) << 16;
    }
    *reinterpret_cast<u32x4_any *>(static_cast<uint16_t *>(p) + at) = w;
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

// TPR threads a row, NV pieces of 8 numbers a thread.  X, S, P: types of x and the result, of the stream and of the parameters, and rows of whole pieces; ANY: whatever the
// call says, number by number where a row ends inside a piece.  (With types and ends looked at in one kernel for all, two thirds of its instructions were moves between
// the branches: 8192 rows of 4096 took 69 us, now 46.)
constexpr int ANY = -1;
template <int TPR, int NV, int X, int S, int P>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_kernel(const ralm_norm_t p)
{
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1;   // rows of a workgroup
    constexpr bool WHOLE = X != ANY;
    static_assert(TPR == 64 || TPR >= 256, "a row is a wave's or a workgroup's");
    __shared__ float part[TPR > 64 ? 2 * (TPR / 64) : 1];
    const int t = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPW + threadIdx.x / TPR;
    if (row >= p.T) return;   // whole waves, and no barrier where a workgroup has several rows
    const int D = p.D;
    const int x_dt = WHOLE ? X : p.x_dtype, s_dt = WHOLE ? S : p.sum_dtype, p_dt = WHOLE ? P : p.param_dtype, o_dt = WHOLE ? X : p.out_dtype;
    const float mean_of = 1.f / (float)D;
    auto at = [&](int v) { return (v * TPR + t) * 8; };
    auto in = [&](int v, int j) { return WHOLE ? at(v) < D : at(v) + j < D; };
    auto load = [&](Raw(&raw)[NV], const void *from, int dt, int64_t base) __attribute__((always_inline)) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if constexpr (WHOLE) raw[v].load_whole(from, dt == DT_F32, base + (at(v) < D ? at(v) : 0));   // (pieces behind the row: its first one again)
            else raw[v].load(from, dt == DT_F32, base + at(v), D - at(v));
        }
    };
    auto store = [&](void *d, int dt, int64_t base, int v, const float (&x)[8]) __attribute__((always_inline)) {
        if (WHOLE ? at(v) < D : at(v) + 8 <= D) {
            store8(d, dt, base + at(v), x);
        } else if constexpr (!WHOLE) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (in(v, j)) store1(d, dt, base + at(v) + j, x[j]);
        }
    };
    int sums = 0;
    float s[NV][8];
    // the norm of the row in s, times w plus b
    auto normed = [&](const void *w, const void *b) __attribute__((always_inline)) {
        Raw g[NV], o[NV];
        if (w) load(g, w, p_dt, 0);
        if (b) load(o, b, p_dt, 0);
        if (p.kind == RALM_NORM_LAYER) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum += in(v, j) ? s[v][j] : 0.f;
            const float mean = row_sum<TPR>(sum, part, sums++) * mean_of;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[v][j] -= mean;
        }
        float sq = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float q = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) q += WHOLE || in(v, j) ? s[v][j] * s[v][j] : 0.f;
            sq += in(v, 0) ? q : 0.f;
        }
        const float r = 1.f / sqrtf(row_sum<TPR>(sq, part, sums++) * mean_of + p.eps);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[v][j] *= r;
        if (w) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[v][j] *= g[v].at(j, p_dt);
        }
        if (b) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < 8; ++j) s[v][j] += o[v].at(j, p_dt);
        }
    };
    // what is added and what it is multiplied with are under way while the first norm waits for its sums
    Raw x[NV], r[NV], g[NV];
    load(x, p.x, x_dt, row * p.x_stride);
    if (p.residual) load(r, p.residual, s_dt, row * p.residual_stride);
    if (p.gate) load(g, p.gate, x_dt, p.gate_rows ? row * p.gate_stride : 0);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[v][j] = x[v].at(j, x_dt);
    if (p.post) normed(p.post_weight, p.post_bias);
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 8; ++j) s[v][j] *= p.scale;
    if (p.gate) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[v][j] *= g[v].at(j, x_dt);
    }
    if (p.residual) {
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < 8; ++j) s[v][j] += r[v].at(j, s_dt);
    }
    if (p.sum) {
#pragma unroll
        for (int v = 0; v < NV; ++v) store(p.sum, s_dt, row * p.sum_stride, v, s[v]);
    }
    if (!p.out) return;
    normed(p.weight, p.bias);
#pragma unroll
    for (int v = 0; v < NV; ++v) store(p.out, o_dt, row * p.out_stride, v, s[v]);
}

template <int TPR, int NV>
hipError_t launch(const ralm_norm_t &p, hipStream_t stream)
{
    constexpr int RPW = TPR < 256 ? 256 / TPR : 1, NT = TPR < 256 ? 256 : TPR;
    const dim3 grid((unsigned)((p.T + RPW - 1) / RPW));
    const bool params = p.weight || p.bias || (p.post && (p.post_weight || p.post_bias));
    const int x = p.x_dtype, s = p.sum_dtype, w = params ? p.param_dtype : x;
    const bool plain = p.D % 8 == 0 && (!p.out || p.out_dtype == x) && (s == x || s == DT_F32) && (w == x || w == DT_F32);
    auto of = [&](auto x_tag) {
        constexpr int X = decltype(x_tag)::value;
        if (s == X && w == X) norm_kernel<TPR, NV, X, X, X><<<grid, NT, 0, stream>>>(p);
        else if (w == X) norm_kernel<TPR, NV, X, DT_F32, X><<<grid, NT, 0, stream>>>(p);
        else if (s == X) norm_kernel<TPR, NV, X, X, DT_F32><<<grid, NT, 0, stream>>>(p);
        else norm_kernel<TPR, NV, X, DT_F32, DT_F32><<<grid, NT, 0, stream>>>(p);
    };
    if (!plain) norm_kernel<TPR, NV, ANY, ANY, ANY><<<grid, NT, 0, stream>>>(p);
    else if (x == DT_BF16) of(std::integral_constant<int, DT_BF16>{});
    else if (x == DT_F16) of(std::integral_constant<int, DT_F16>{});
    else norm_kernel<TPR, NV, DT_F32, DT_F32, DT_F32><<<grid, NT, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_residual_norm(const ralm_norm_t &p, hipStream_t stream)
{
    // us, 30 million numbers, bf16, norms on both sides: D 1024 a wave 40, 256 threads 53; D 2048 a wave 41, 256 threads 41, 512 threads 52; D 4096 256 threads 42, 512
    // threads 42, 1024 threads 58; D 16384 512 threads 46, 1024 threads 57.  Four rows: 3.1 to 5.5, fewer pieces a thread first
    if (p.D <= 512) return launch<64, 1>(p, stream);
    if (p.D <= 1024) return launch<64, 2>(p, stream);
    if (p.D <= 2048) return launch<256, 1>(p, stream);
    if (p.D <= 4096) return launch<512, 1>(p, stream);
    if (p.D <= 8192) return launch<512, 2>(p, stream);
    if (p.D <= 16384) return launch<512, 4>(p, stream);
    return launch<1024, 4>(p, stream);
}

}  // namespace ralm
