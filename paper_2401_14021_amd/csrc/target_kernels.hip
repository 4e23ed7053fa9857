// The target of a verification: softmax of the logits mixed with the neighbours' weights (ralm_knnlm_target).
//
// target_row_kernel   a workgroup holds a row in registers: it is read once; what bounds it is memory
// target_stat_kernel, target_mix_kernel   few rows, or rows of more than 65536 entries: workgroups of 4096 entries leave their largest logit and sum of exponentials,
//                     then read their entries again, from L2 or the last-level cache, and write
//
// Exponentials are 2^((x - top) c), c = log2 e / T: the difference first, so that logits of any size are safe; results below 2^-126 are 0.  The largest logit counts as at
// least the lowest finite number, so that entries of -inf are 0 without being looked at, and a row of nothing else sums to 0.  A token's neighbours are added up by one thread in
// their order, on the probability formed again in fp32: the result is rounded once and does not depend on which thread came first.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

// 4 numbers from anywhere that their type may lie: rows of an odd number of entries are aligned to nothing else (the hardware takes such accesses whole).  Neighbouring lanes'
// fours lie side by side in every type
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

template <int DT>
__device__ __forceinline__ void load4(const void *p, int64_t at, float (&x)[4])
{
    if constexpr (DT == DT_F32) {
        const f32x4_any a = *reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = a[j];
    } else {
        const u32x2_any w = *reinterpret_cast<const u32x2_any *>(static_cast<const uint16_t *>(p) + at);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
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
__device__ __forceinline__ void store4(void *p, int64_t at, const float (&x)[4])
{
    if constexpr (DT == DT_F32) {
        const f32x4_any a = {x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + at) = a;
    } else {
        u32x2_any w;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            if constexpr (DT == DT_BF16)
                w[j] = __builtin_bit_cast(uint16_t, (__bf16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)x[2 * j + 1]) << 16;
            else
                w[j] = __builtin_bit_cast(uint16_t, (_Float16)x[2 * j]) | (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x[2 * j + 1]) << 16;
        }
        *reinterpret_cast<u32x2_any *>(static_cast<uint16_t *>(p) + at) = w;
    }
}

constexpr float LOWEST = -3.402823466e38f;

__device__ __forceinline__ float exp_of(float y, float top, float c) { return __builtin_amdgcn_exp2f((y - top) * c); }

template <int C>
__device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), C, 0xf, 0xf, false));
}
// over the lanes of a wave, without LDS: 16 lanes by exchanges, then the four sixteens
template <bool MAX>
__device__ __forceinline__ float wave_all(float v)
{
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    v = op(v, dpp<0xB1>(v));
    v = op(v, dpp<0x4E>(v));
    v = op(v, dpp<0x141>(v));
    v = op(v, dpp<0x140>(v));
    auto at = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
    return op(op(at(0), at(16)), op(at(32), at(48)));
}
// over a workgroup of NT threads; words: NT / 64 floats of LDS.  All threads
template <int NT, bool MAX>
__device__ __forceinline__ float group_all(float v, float *words)
{
    v = wave_all<MAX>(v);
    if ((threadIdx.x & 63) == 0) words[threadIdx.x >> 6] = v;
    __syncthreads();
    v = words[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v = MAX ? fmaxf(v, words[w]) : v + words[w];
    return v;
}

// The entries v0 .. v1 - 1 of a row, 4 NV a thread; what lies behind is -inf
template <int DT, int NT, int NV>
__device__ __forceinline__ void load_entries(const void *x, int v0, int v1, float (&y)[NV][4])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int at = v0 + (i * NT + (int)threadIdx.x) * 4;
        if (at + 4 <= v1) {
            load4<DT>(x, at, y[i]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) y[i][j] = at + j < v1 ? load1<DT>(x, at + j) : -__builtin_inff();
        }
    }
}
// 16-bit entries as they lie in memory, in half the registers; their exponentials are formed twice
template <int DT, int NT, int NV>
struct Packed {
    u32x2_any w[NV];
    __device__ __forceinline__ void load(const void *x, int n)
    {
        const uint16_t *from = static_cast<const uint16_t *>(x);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = (i * NT + (int)threadIdx.x) * 4;
            if (at + 4 <= n) {
                w[i] = *reinterpret_cast<const u32x2_any *>(from + at);
            } else {
                constexpr uint32_t NONE = DT == DT_BF16 ? 0xff80u : 0xfc00u;   // -inf
                uint32_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) b[j] = at + j < n ? from[at + j] : NONE;
                w[i][0] = b[0] | b[1] << 16;
                w[i][1] = b[2] | b[3] << 16;
            }
        }
    }
    // between two uses: the compiler would keep what it formed for the first one
    __device__ __forceinline__ void anew()
    {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            uint32_t a = w[i][0], b = w[i][1];
            asm("" : "+v"(a), "+v"(b));
            w[i][0] = a;
            w[i][1] = b;
        }
    }
    __device__ __forceinline__ float at(int i, int j) const
    {
        const uint32_t v = w[i][j / 2];
        if constexpr (DT == DT_BF16) return __uint_as_float(j & 1 ? v & 0xffff0000u : v << 16);
        else return f16_bits_to_f32(j & 1 ? v >> 16 : v & 0xffffu);
    }
};
template <int DT>
__device__ __forceinline__ void store_four(void *x, int at, int end, const float (&y)[4])
{
    if (at + 4 <= end) {
        store4<DT>(x, at, y);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (at + j < end) store1<DT>(x, at + j, y[j]);
    }
}
template <int DT, int NT, int NV>
__device__ __forceinline__ void store_entries(void *x, int v0, int v1, const float (&y)[NV][4])
{
#pragma unroll
    for (int i = 0; i < NV; ++i) store_four<DT>(x, v0 + (i * NT + (int)threadIdx.x) * 4, v1, y[i]);
}
template <int NV>
__device__ __forceinline__ float max_of(const float (&y)[NV][4])
{
    float m = LOWEST;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = fmaxf(m, y[i][j]);   // (a NaN shows in the sum)
    return m;
}
// y becomes its exponential
template <int NV>
__device__ __forceinline__ float exps_of(float (&y)[NV][4], float top, float c)
{
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float t = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y[i][j] = exp_of(y[i][j], top, c);
            t += y[i][j];
        }
        s += t;
    }
    return s;
}

// The tokens in [v0, v1) that a row's neighbours have, each with the sum of its weights in their order: a thread gets up to M of them, tokens of -1 are none.  Up to DIRECT
// neighbours each looks for its token in front of it; more are sorted by token and place first (40 rows of 50257, us: no
// neighbours 8.4, 64 10.7, 256 9.9 (18.6 unsorted), 1024 11.6).
constexpr int DIRECT = 64;
struct Near {
    alignas(16) int32_t token[DIRECT];
    alignas(16) float weight[RALM_MAX_K];
    u64 keys[RALM_MAX_K];
    int count;
};
template <int NT, int M>
__device__ __forceinline__ void gather_near(Near &near, const TargetParams &p, int64_t row, int v0, int v1, int32_t (&token)[M], float (&sum)[M])
{
    static_assert(NT >= DIRECT && NT * M >= RALM_MAX_K, "a place for every neighbour");
    const int tid = threadIdx.x, k = p.k;
    const int32_t *tokens = p.tokens + row * k;
    const float *weights = p.weights + row * k;
#pragma unroll
    for (int i = 0; i < M; ++i) token[i] = -1, sum[i] = 0.f;
    if (k <= DIRECT) {
        const int k4 = (k + 3) & ~3;
        if (tid < k4) {
            const int32_t t = tid < k ? tokens[tid] : -1;
            token[0] = t >= v0 && t < v1 ? t : -1;
            near.token[tid] = token[0];
            near.weight[tid] = tid < k ? weights[tid] : 0.f;
        }
        __syncthreads();
        if (tid < k4) {   // (by whole fours and without branches: one at a time, 64 neighbours took 3 us)
            const int32_t own = token[0];
            bool later = false;
#pragma unroll 4
            for (int j = 0; j < k4; j += 4) {
                const int4 t = *reinterpret_cast<const int4 *>(near.token + j);
                const float4 w = *reinterpret_cast<const float4 *>(near.weight + j);
                sum[0] += t.x == own ? w.x : 0.f;
                sum[0] += t.y == own ? w.y : 0.f;
                sum[0] += t.z == own ? w.z : 0.f;
                sum[0] += t.w == own ? w.w : 0.f;
                later |= (t.x == own && j < tid) || (t.y == own && j + 1 < tid) || (t.z == own && j + 2 < tid) || (t.w == own && j + 3 < tid);
            }
            if (later) token[0] = -1;   // the first one's thread has them all
        }
        return;
    }
    if (tid == 0) near.count = 0;
    __syncthreads();
    for (int j = tid; j < k; j += NT) {
        const int32_t t = tokens[j];
        near.weight[j] = weights[j];
        if (t >= v0 && t < v1) near.keys[atomicAdd(&near.count, 1)] = (u64)(uint32_t)t << 32 | (uint32_t)j;
    }
    __syncthreads();
    const int n = near.count;
    int size = 2;
    while (size < n) size <<= 1;   // at most RALM_MAX_K, a power of two
    for (int j = n + tid; j < size; j += NT) near.keys[j] = ~0ull;
    __syncthreads();
    sort_keys<NT, false>(near.keys, size);
#pragma unroll
    for (int i = 0; i < M; ++i) {
        const int j = tid + i * NT;
        if (j >= n) continue;
        const uint32_t t = (uint32_t)(near.keys[j] >> 32);
        if (j > 0 && (uint32_t)(near.keys[j - 1] >> 32) == t) continue;
        token[i] = (int32_t)t;
        for (int e = j; e < n && (uint32_t)(near.keys[e] >> 32) == t; ++e) sum[i] += near.weight[(uint32_t)near.keys[e]];
    }
}

template <int DT>
__device__ __forceinline__ const void *row_of(const void *p, int64_t at)
{
    return DT == DT_F32 ? static_cast<const void *>(static_cast<const float *>(p) + at) : static_cast<const void *>(static_cast<const uint16_t *>(p) + at);
}

// The model's share of a row over its sum of exponentials: NaN where the row is, 0 where there is nothing
__device__ __forceinline__ float share_of_model(float share, float sum) { return sum == 0.f ? 0.f : (1.f - share) / sum; }

// Workgroups of 512 threads share a CU, so that a row's phases have others beside them: two of up to 128 registers, three where 16-bit entries are kept as they lie
// (kernels alone, 1300 rows of 32000, bf16 to fp32: a workgroup of 1024 threads, alone, 74, two 63, three 54 us, 4.6 TB/s; bf16 to bf16 55, 47.  A stream of
// calls, bf16 to fp32, takes 58 each.  Four spill: 68.  Shorter rows gain
// nothing by it, and longer ones need 1024 threads' registers: 600 rows of 50257 52 us, packed 55.)
template <int DT, int DO, int NT, int NV>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(NT == 512 && (NV == 8 || (NV == 16 && DT != DT_F32)) ? 6 : 4))) void target_row_kernel(const TargetParams p)
{
    constexpr int M = (RALM_MAX_K + NT - 1) / NT;
    __shared__ Near near;
    __shared__ float words[2][NT / 64];
    const int64_t row = blockIdx.x;
    const void *x = row_of<DT>(p.logits, row * p.logits_stride);
    void *out = const_cast<void *>(row_of<DO>(p.out, row * p.out_stride));
    constexpr bool PACKED = DT != DT_F32 && NT == 512 && NV == 16;
    float y[PACKED ? 1 : NV][4];
    Packed<DT, NT, PACKED ? NV : 1> packed;
    if constexpr (PACKED) packed.load(x, p.V);
    else load_entries<DT, NT, NV>(x, 0, p.V, y);
    int32_t token[M];
    float sum[M], logit[M];
    gather_near<NT, M>(near, p, row, 0, p.V, token, sum);
#pragma unroll
    for (int i = 0; i < M; ++i) logit[i] = token[i] >= 0 ? load1<DT>(x, token[i]) : 0.f;   // before the row may be written over
    const float share = p.share ? p.share[row] : p.share_all;
    float top, all, per;
    if constexpr (PACKED) {
        top = LOWEST;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) top = fmaxf(top, packed.at(i, j));   // (a NaN shows in the sum)
        top = group_all<NT, true>(top, words[0]);
        packed.anew();
        all = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float t = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) t += exp_of(packed.at(i, j), top, p.scale);
            all += t;
        }
        all = group_all<NT, false>(all, words[1]);
        packed.anew();
        per = share_of_model(share, all);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) e[j] = exp_of(packed.at(i, j), top, p.scale) * per;
            store_four<DO>(out, (i * NT + (int)threadIdx.x) * 4, p.V, e);
        }
    } else {
        top = group_all<NT, true>(max_of<NV>(y), words[0]);
        all = group_all<NT, false>(exps_of<NV>(y, top, p.scale), words[1]);
        per = share_of_model(share, all);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < 4; ++j) y[i][j] *= per;
        }
        store_entries<DO, NT, NV>(out, 0, p.V, y);
    }
    __syncthreads();   // the entries of tokens are written again, by others
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (token[i] >= 0) store1<DO>(out, token[i], exp_of(logit[i], top, p.scale) * per + share * sum[i]);
}

constexpr int PART_NT = 256, PART_NV = TARGET_PART / (PART_NT * 4);

template <int DT>
__global__ __launch_bounds__(PART_NT) void target_stat_kernel(const TargetParams p)
{
    __shared__ float words[2][PART_NT / 64];
    const int64_t row = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - row * p.parts), v0 = part * TARGET_PART, v1 = p.V - v0 < TARGET_PART ? p.V : v0 + TARGET_PART;
    float y[PART_NV][4];
    load_entries<DT, PART_NT, PART_NV>(row_of<DT>(p.logits, row * p.logits_stride), v0, v1, y);
    const float top = group_all<PART_NT, true>(max_of<PART_NV>(y), words[0]);
    const float sum = group_all<PART_NT, false>(exps_of<PART_NV>(y, top, p.scale), words[1]);
    if (threadIdx.x == 0) p.stats[row * p.parts + part] = make_float2(top, sum);
}

template <int DT, int DO>
__global__ __launch_bounds__(PART_NT) void target_mix_kernel(const TargetParams p)
{
    constexpr int M = (RALM_MAX_K + PART_NT - 1) / PART_NT;
    __shared__ Near near;
    __shared__ float words[2][PART_NT / 64];
    const int64_t row = blockIdx.x / p.parts;
    const int part = (int)(blockIdx.x - row * p.parts), v0 = part * TARGET_PART, v1 = p.V - v0 < TARGET_PART ? p.V : v0 + TARGET_PART;
    const void *x = row_of<DT>(p.logits, row * p.logits_stride);
    void *out = const_cast<void *>(row_of<DO>(p.out, row * p.out_stride));
    float y[PART_NV][4];
    load_entries<DT, PART_NT, PART_NV>(x, v0, v1, y);
    int32_t token[M];
    float sum[M], logit[M];
    gather_near<PART_NT, M>(near, p, row, v0, v1, token, sum);
#pragma unroll
    for (int i = 0; i < M; ++i) logit[i] = token[i] >= 0 ? load1<DT>(x, token[i]) : 0.f;
    // a thread for every part: at most RALM_MAX_VOCABULARY / TARGET_PART
    static_assert(RALM_MAX_VOCABULARY <= PART_NT * TARGET_PART, "parts of a row");
    const float2 stat = (int)threadIdx.x < p.parts ? p.stats[row * p.parts + threadIdx.x] : make_float2(LOWEST, 0.f);
    const float share = p.share ? p.share[row] : p.share_all;
    const float top = group_all<PART_NT, true>(stat.x, words[0]);
    const float all = group_all<PART_NT, false>(stat.y == 0.f ? 0.f : stat.y * exp_of(stat.x, top, p.scale), words[1]);
    const float per = share_of_model(share, all);
#pragma unroll
    for (int i = 0; i < PART_NV; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) y[i][j] = exp_of(y[i][j], top, p.scale) * per;
    store_entries<DO, PART_NT, PART_NV>(out, v0, v1, y);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i)
        if (token[i] >= 0) store1<DO>(out, token[i], exp_of(logit[i], top, p.scale) * per + share * sum[i]);
}

template <int DT, int DO>
hipError_t launch(const TargetParams &p, hipStream_t stream)
{
    if (p.parts > 0) {
        const dim3 grid((unsigned)(p.Q * p.parts));
        target_stat_kernel<DT><<<grid, PART_NT, 0, stream>>>(p);
        target_mix_kernel<DT, DO><<<grid, PART_NT, 0, stream>>>(p);
    } else {
        const dim3 grid((unsigned)p.Q);
        if (p.V <= 1024) target_row_kernel<DT, DO, 256, 1><<<grid, 256, 0, stream>>>(p);
        else if (p.V <= 4096) target_row_kernel<DT, DO, 256, 4><<<grid, 256, 0, stream>>>(p);
        else if (p.V <= 8192) target_row_kernel<DT, DO, 512, 4><<<grid, 512, 0, stream>>>(p);
        else if (p.V <= 16384) target_row_kernel<DT, DO, 512, 8><<<grid, 512, 0, stream>>>(p);
        else if (p.V <= 32768) target_row_kernel<DT, DO, 512, 16><<<grid, 512, 0, stream>>>(p);
        else target_row_kernel<DT, DO, 1024, 16><<<grid, 1024, 0, stream>>>(p);
    }
    return hipGetLastError();
}
template <int DT>
hipError_t launch_of(const TargetParams &p, hipStream_t stream)
{
    return p.out_dtype == DT_F32 ? launch<DT, DT_F32>(p, stream) : p.out_dtype == DT_BF16 ? launch<DT, DT_BF16>(p, stream) : launch<DT, DT_F16>(p, stream);
}

}  // namespace

// Workgroups of a row, 0: a row is one workgroup's.  us, a row's workgroup and shared rows (16 neighbours, fp32): V 8000, 1 row 5.2, 7.1; V 32000, 8 rows 8.2, 7.6, 64
// rows 10.1, 10.2, 256 rows 17, 22; V 50257, 8 rows 11.5, 8.0, 128 rows 17.8, 17.8, 600 rows 63, 70
int target_parts(int64_t Q, int32_t V)
{
    if (V <= 65536 && (Q >= TARGET_FEW || V <= 8192)) return 0;
    return (V + TARGET_PART - 1) / TARGET_PART;
}

hipError_t launch_knnlm_target(const TargetParams &p, hipStream_t stream)
{
    return p.dtype == DT_F32 ? launch_of<DT_F32>(p, stream) : p.dtype == DT_BF16 ? launch_of<DT_BF16>(p, stream) : launch_of<DT_F16>(p, stream);
}

}  // namespace ralm
