// Rows times weights with bias, activation, gate and residual (ralm_linear).
//
// Weights are the A operand of the matrix instruction and the rows of x the B operand, so that a lane's results are four
// neighbouring outputs of one row: bias, activation, gate and residual are applied where the sums lie, and leave as one store.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

template <bool F16>
__device__ __forceinline__ f32x16 mfma32(const uint4 &a, const uint4 &b, const f32x16 &c)
{
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// ---- epilogue ----------------------------------------------------------------------------------

__device__ __forceinline__ float activated(float y, int act)
{
    switch (act) {   // uniform
    case RALM_ACT_RELU: return y < 0.f ? 0.f : y;   // NaN stays
    case RALM_ACT_GELU: return 0.5f * y * erfcf(-0.70710678f * y);
    case RALM_ACT_GELU_TANH:   // 0.5 y (1 + tanh u) = y / (1 + exp(-2 u))
        return y / (1.f + expf(-1.5957691216f * (y + 0.044715f * y * y * y)));
    case RALM_ACT_SILU: return y / (1.f + expf(-y));
    default: return y;
    }
}

template <bool F16>
__device__ __forceinline__ float widened(uint32_t b) { return F16 ? f16_bits_to_f32(b & 0xffffu) : __uint_as_float(b << 16); }

// Four neighbouring outputs n .. n + 3 of row t from their sums; `vec`: base and stride of out and residual are aligned to four elements
template <bool F16, bool GATED, bool OUT32>
__device__ __forceinline__ void finish4(const LinearParams &p, int64_t t, int n, float (&y)[4], const float (&up)[4], bool vec)
{
    if (t >= p.T || n >= p.N) return;
    const uint16_t *bias = static_cast<const uint16_t *>(p.bias);
    const int m = p.N - n < 4 ? p.N - n : 4;
    float r[4] = {0.f, 0.f, 0.f, 0.f};
    const bool whole = vec && m == 4;
    if (p.residual) {
        const int64_t at = t * p.residual_stride + n;
        if constexpr (OUT32) {
            const float *s = static_cast<const float *>(p.residual) + at;
            if (whole) {
                const f32x4 v = *reinterpret_cast<const f32x4 *>(s);
                r[0] = v[0], r[1] = v[1], r[2] = v[2], r[3] = v[3];
            } else {
                for (int j = 0; j < m; ++j) r[j] = s[j];
            }
        } else {
            const uint16_t *s = static_cast<const uint16_t *>(p.residual) + at;
            if (whole) {
                const uint2 v = *reinterpret_cast<const uint2 *>(s);
                r[0] = widened<F16>(v.x & 0xffffu), r[1] = widened<F16>(v.x >> 16), r[2] = widened<F16>(v.y & 0xffffu), r[3] = widened<F16>(v.y >> 16);
            } else {
                for (int j = 0; j < m; ++j) r[j] = widened<F16>(s[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v = y[j], u = GATED ? up[j] : 0.f;
        if (bias && j < m) {
            v += widened<F16>(bias[n + j]);
            if constexpr (GATED) u += widened<F16>(bias[p.N + n + j]);
        }
        v = activated(v, p.act);
        if constexpr (GATED) v *= u;
        y[j] = r[j] + v;
    }
    const int64_t at = t * p.out_stride + n;
    if constexpr (OUT32) {
        float *d = static_cast<float *>(p.out) + at;
        if (whole) {
            const f32x4 v = {y[0], y[1], y[2], y[3]};
            *reinterpret_cast<f32x4 *>(d) = v;
        } else {
            for (int j = 0; j < m; ++j) d[j] = y[j];
        }
    } else {
        uint16_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = F16 ? __builtin_bit_cast(uint16_t, (_Float16)y[j]) : __builtin_bit_cast(uint16_t, (__bf16)y[j]);
        uint16_t *d = static_cast<uint16_t *>(p.out) + at;
        if (whole) {
            const uint2 v = {b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16};
            *reinterpret_cast<uint2 *>(d) = v;
        } else {
            for (int j = 0; j < m; ++j) d[j] = b[j];
        }
    }
}
template <bool OUT32>
__device__ __forceinline__ bool quads_aligned(const LinearParams &p)
{
    constexpr uint64_t B = OUT32 ? 15 : 7;
    return ((reinterpret_cast<uint64_t>(p.out) | reinterpret_cast<uint64_t>(p.residual)) & B) == 0 && ((p.out_stride | p.residual_stride) & 3) == 0;
}

// ---- first form: tiles of 128 weights x 64 rows through registers into LDS -----------------------

// 16 bytes of a row, zeros outside the matrix
__device__ __forceinline__ uint4 piece(const uint16_t *base, int64_t stride, int64_t row, int64_t rows, int k, int K)
{
    if (row >= rows || k >= K) return make_uint4(0, 0, 0, 0);
    return *reinterpret_cast<const uint4 *>(base + row * stride + k);
}

template <bool F16, bool GATED, bool OUT32>
__global__ __launch_bounds__(256) void linear_kernel(const LinearParams p)
{
    constexpr int BM = 128, BN = 64, PITCH = 72;   // elements: 64 and 8 of padding
    __shared__ __align__(16) uint16_t a[BM * PITCH], b[BN * PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // gated: the tile's lower 64 rows are gates, the upper 64 what they are multiplied with
    constexpr int COLS = GATED ? BM / 2 : BM;
    const int n_tiles = (p.N + COLS - 1) / COLS;
    const int n0 = (int)(blockIdx.x % n_tiles) * COLS;
    const int64_t t0 = (int64_t)(blockIdx.x / n_tiles) * BN;
    const uint16_t *x = static_cast<const uint16_t *>(p.x), *w = static_cast<const uint16_t *>(p.w);
    const bool vec = quads_aligned<OUT32>(p);
    f32x16 acc[2][2];   // [gate, up or the upper 32 weights][32 rows]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    // wave (wn, wt): weights 32 wn' .., two blocks of them; rows 0 .. 63
    const int wn = wave;
    for (int k0 = 0; k0 < p.K; k0 += 64) {
        __syncthreads();
        for (int c = tid; c < BM * 8; c += 256) {
            const int row = c >> 3, k = (c & 7) * 8;
            uint4 v;
            if constexpr (GATED) {
                const int col = n0 + (row & 63);
                v = col < p.N ? piece(w, p.w_stride, (int64_t)(row >> 6) * p.N + col, 2 * (int64_t)p.N, k0 + k, p.K) : make_uint4(0, 0, 0, 0);
            } else {
                v = piece(w, p.w_stride, n0 + row, p.N, k0 + k, p.K);
            }
            *reinterpret_cast<uint4 *>(a + row * PITCH + k) = v;
        }
        for (int c = tid; c < BN * 8; c += 256) {
            const int row = c >> 3, k = (c & 7) * 8;
            *reinterpret_cast<uint4 *>(b + row * PITCH + k) = piece(x, p.x_stride, t0 + row, p.T, k0 + k, p.K);
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const int at = kk * 16 + (lane >> 5) * 8;
            if constexpr (GATED) {
                // waves 0, 1: rows 0 .. 31 of x, waves 2, 3: 32 .. 63
                const uint4 g = *reinterpret_cast<const uint4 *>(a + ((wn & 1) * 32 + (lane & 31)) * PITCH + at);
                const uint4 u = *reinterpret_cast<const uint4 *>(a + (64 + (wn & 1) * 32 + (lane & 31)) * PITCH + at);
                const uint4 r = *reinterpret_cast<const uint4 *>(b + ((wn >> 1) * 32 + (lane & 31)) * PITCH + at);
                acc[0][0] = mfma32<F16>(g, r, acc[0][0]);
                acc[1][0] = mfma32<F16>(u, r, acc[1][0]);
            } else {
                const uint4 g = *reinterpret_cast<const uint4 *>(a + (wn * 32 + (lane & 31)) * PITCH + at);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint4 r = *reinterpret_cast<const uint4 *>(b + (j * 32 + (lane & 31)) * PITCH + at);
                    acc[0][j] = mfma32<F16>(g, r, acc[0][j]);
                }
            }
        }
    }
#pragma unroll
    for (int j = 0; j < (GATED ? 1 : 2); ++j) {
        const int64_t t = t0 + (GATED ? wn >> 1 : j) * 32 + (lane & 31);
        const int n = n0 + (GATED ? wn & 1 : wn) * 32 + (lane >> 5) * 4;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            float y[4], up[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) y[v] = acc[0][j][c * 4 + v], up[v] = acc[1][j][c * 4 + v];
            finish4<F16, GATED, OUT32>(p, t, n + c * 8, y, up, vec);
        }
    }
}

template <bool F16, bool GATED, bool OUT32>
hipError_t launch(const LinearParams &p, hipStream_t stream)
{
    const int64_t n_tiles = (p.N + (GATED ? 63 : 127)) / (GATED ? 64 : 128), t_tiles = (p.T + 63) / 64;
    linear_kernel<F16, GATED, OUT32><<<dim3((unsigned)(n_tiles * t_tiles)), 256, 0, stream>>>(p);
    return hipGetLastError();
}
template <bool F16>
hipError_t launch_of(const LinearParams &p, hipStream_t stream)
{
    const bool o32 = p.out_dtype == DT_F32;
    if (p.gated) return o32 ? launch<F16, true, true>(p, stream) : launch<F16, true, false>(p, stream);
    return o32 ? launch<F16, false, true>(p, stream) : launch<F16, false, false>(p, stream);
}

}  // namespace

hipError_t launch_linear(const LinearParams &p, hipStream_t stream)
{
    return p.dtype == DT_F16 ? launch_of<true>(p, stream) : launch_of<false>(p, stream);
}

}  // namespace ralm
