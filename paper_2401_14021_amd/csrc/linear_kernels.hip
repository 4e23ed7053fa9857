// Rows times weights with bias, activation, gate and residual (ralm_linear).
//
// Weights are the A operand of the matrix instruction and the rows of x the B operand, so that a lane's results are four neighbouring outputs of one row:
// bias, activation, gate and residual are applied to fours.  Three kernels, one rule between them (linear_plan):
//
//  linear_few_kernel   few rows, small weights: what bounds it is the latency of a launch and of one trip to memory
//  linear_tile_kernel  tiles through LDS; few rows: bound by the weights' way from memory, the depth split over workgroups; many rows: by the matrix cores
//  linear_join_kernel  sums of a split depth, and the epilogue
#include <math.h>

#include <type_traits>

#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

// ---- epilogue ----------------------------------------------------------------------------------

// Phi(-a), a >= 0, as exp(-a^2 / 2) t P(t) with t = 1 / (1 + p a): t P(t) is what an exponential leaves of the normal distribution's tail, which varies slowly; P is a polynomial fitted
// over 0 <= a <= 14.5 for the least relative error.  (The library's erfc took 37 us of the 240 of 1387 rows x 16384 outputs, which no multiply hides.)
//
// EXACT, for fp32 outputs: 10 coefficients (3.5e-9 of the value), the square with its rounding error: 16 2^-24 of the value.  Otherwise 7 (9.6e-7) and the square as it
// is, 2^-17 of the value, 1/64 of a rounding to bf16, 1/16 of one to fp16; both down to 2^-118.
// (1387 rows, K 4096, N 16384: 7 coefficients 195 us, 10 and the corrections 198.)
template <bool EXACT>
__device__ __forceinline__ float normal_tail(float a)
{
    constexpr double C = -0.72134752044448170;   // -log2 e / 2
    constexpr float C_HIGH = (float)C, C_LOW = (float)(C - (double)C_HIGH);
    if constexpr (EXACT) {
        a = fminf(a, 16.f);   // infinities would be NaN in the corrections
        const float d = fmaf(0.3f, a, 1.f), t0 = __builtin_amdgcn_rcpf(d), t = fmaf(fmaf(-d, t0, 1.f), t0, t0);
        float s = -2.062346414e-02f;
        s = fmaf(s, t, 1.124355868e-01f);
        s = fmaf(s, t, -2.282135338e-01f);
        s = fmaf(s, t, 1.917844415e-01f);
        s = fmaf(s, t, -7.942341268e-02f);
        s = fmaf(s, t, 9.615679085e-02f);
        s = fmaf(s, t, 7.838965952e-02f);
        s = fmaf(s, t, 1.102354228e-01f);
        s = fmaf(s, t, 1.195718125e-01f);
        s = fmaf(s, t, 1.196866930e-01f) * t;
        const float q = a * a, q_low = fmaf(a, a, -q), h = q * C_HIGH;
        const float low = fmaf(q_low, C_HIGH, fmaf(q, C_LOW, fmaf(q, C_HIGH, -h)));   // what the exponent h lacks
        const float e = __builtin_amdgcn_exp2f(h);
        return s * fmaf(e, low * 0.69314718f, e);
    } else {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.36f, a, 1.f));
        float s = 4.678247124e-02f;
        s = fmaf(s, t, -1.788265556e-01f);
        s = fmaf(s, t, 1.796776205e-01f);
        s = fmaf(s, t, 2.742663398e-02f);
        s = fmaf(s, t, 1.394000649e-01f);
        s = fmaf(s, t, 1.418303847e-01f);
        s = fmaf(s, t, 1.437089741e-01f) * t;
        return s * __builtin_amdgcn_exp2f(a * a * C_HIGH);
    }
}

template <bool EXACT>
__device__ __forceinline__ float activated(float y, int act)
{
    switch (act) {   // uniform
    case RALM_ACT_RELU: return y < 0.f ? 0.f : y;   // NaN stays
    case RALM_ACT_GELU: {
        const float low = normal_tail<EXACT>(fabsf(y));
        return y * (y > 0.f ? 1.f - low : low);   // (y - y low would be NaN at infinity)
    }
    case RALM_ACT_GELU_TANH:   // 0.5 y (1 + tanh u) = y / (1 + exp(-2 u))
        return y * __builtin_amdgcn_rcpf(1.f + __expf(-1.5957691216f * (y + 0.044715f * y * y * y)));
    case RALM_ACT_SILU: return y * __builtin_amdgcn_rcpf(1.f + __expf(-y));
    default: return y;
    }
}

template <bool F16>
__device__ __forceinline__ float widened(uint32_t b) { return F16 ? f16_bits_to_f32(b & 0xffffu) : __uint_as_float(b << 16); }

// the bias of four neighbouring outputs and, behind it, of what they multiply
template <bool F16, bool GATED>
struct Bias4 {
    float y[4], up[4];
    __device__ __forceinline__ Bias4(const LinearParams &p, int n)
    {
        const uint16_t *bias = static_cast<const uint16_t *>(p.bias);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = bias && n + j < p.N;
            y[j] = in ? widened<F16>(bias[n + j]) : 0.f;
            up[j] = GATED && in ? widened<F16>(bias[p.N + n + j]) : 0.f;
        }
    }
};

// Quads of outputs from anywhere that their type may lie: rows of an odd number are aligned to nothing else (the hardware takes such accesses whole)
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// Four neighbouring outputs n .. n + 3 of row t from their sums
template <bool F16, bool GATED, bool OUT32>
__device__ __forceinline__ void finish4(const LinearParams &p, int64_t t, int n, const f32x4 &sum, const f32x4 &up, const Bias4<F16, GATED> &bias)
{
    if (t >= p.T || n >= p.N) return;
    const int m = p.N - n < 4 ? p.N - n : 4;
    float y[4], r[4] = {0.f, 0.f, 0.f, 0.f};
    if (p.residual) {
        const int64_t at = t * p.residual_stride + n;
        if constexpr (OUT32) {
            const float *s = static_cast<const float *>(p.residual) + at;
            if (m == 4) {
                const f32x4_any v = *reinterpret_cast<const f32x4_any *>(s);
                r[0] = v[0], r[1] = v[1], r[2] = v[2], r[3] = v[3];
            } else {
                for (int j = 0; j < m; ++j) r[j] = s[j];
            }
        } else {
            const uint16_t *s = static_cast<const uint16_t *>(p.residual) + at;
            if (m == 4) {
                const u32x2_any v = *reinterpret_cast<const u32x2_any *>(s);
                r[0] = widened<F16>(v[0] & 0xffffu), r[1] = widened<F16>(v[0] >> 16), r[2] = widened<F16>(v[1] & 0xffffu), r[3] = widened<F16>(v[1] >> 16);
            } else {
                for (int j = 0; j < m; ++j) r[j] = widened<F16>(s[j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float v = activated<OUT32>(sum[j] + bias.y[j], p.act);
        if constexpr (GATED) v *= up[j] + bias.up[j];
        y[j] = r[j] + v;
    }
    const int64_t at = t * p.out_stride + n;
    if constexpr (OUT32) {
        float *d = static_cast<float *>(p.out) + at;
        if (m == 4) {
            const f32x4_any v = {y[0], y[1], y[2], y[3]};
            *reinterpret_cast<f32x4_any *>(d) = v;
        } else {
            for (int j = 0; j < m; ++j) d[j] = y[j];
        }
    } else {
        uint16_t b[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) b[j] = F16 ? __builtin_bit_cast(uint16_t, (_Float16)y[j]) : __builtin_bit_cast(uint16_t, (__bf16)y[j]);
        uint16_t *d = static_cast<uint16_t *>(p.out) + at;
        if (m == 4) {
            const u32x2_any v = {b[0] | (uint32_t)b[1] << 16, b[2] | (uint32_t)b[3] << 16};
            *reinterpret_cast<u32x2_any *>(d) = v;
        } else {
            for (int j = 0; j < m; ++j) d[j] = b[j];
        }
    }
}

// ---- few rows: weights straight from memory to the matrix cores ----------------------------------
//
// A workgroup owns 16 RT weights (gated: RT / 2 blocks of gates and as many of what they multiply) and 16 TT rows of x; its W waves share the depth out in
// strips of 64 and meet once, at the end.  Every weight is used by one wave, so it goes from memory into the registers that the multiply reads, without LDS
// and without a barrier; so do the rows of x, which come from L2.  A lane's 16 bytes of two loads are half of its row's 128-byte line each.  D strips a wave
// are under way.  1 row: K = N = 1024 4.3 us, a launch and two trips to memory; K 4096, N 6144 12.6 us, 4.0 TB/s of weights.
template <bool F16>
__device__ __forceinline__ f32x4 mfma16(const uint4 &a, const uint4 &b, const f32x4 &c)
{
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

template <bool F16, bool GATED, bool OUT32, int RT, int TT, int W, int D>
__global__ __launch_bounds__(W * 64) void linear_few_kernel(const LinearParams p, const int n_tiles, const int t_tiles)
{
    constexpr int CB = GATED ? RT / 2 : RT;   // blocks of 16 outputs
    extern __shared__ __align__(16) unsigned char smem[];
    f32x4 *part = reinterpret_cast<f32x4 *>(smem);   // [W][RT][TT][64]
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    // the row tiles that share weights run on one XCD, one after the other
    const int j = (int)(blockIdx.x >> 3);
    const int n_tile = j / t_tiles * 8 + (int)(blockIdx.x & 7);
    if (n_tile >= n_tiles) return;
    const int n0 = n_tile * CB * 16;
    const int t0 = j % t_tiles * TT * 16;
    const int r = lane & 15, c = lane >> 4;
    const uint16_t *wp[RT], *xp[TT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        int n = n0 + (i % CB) * 16 + r;
        n = n < p.N ? n : p.N - 1;   // rows behind the last one are read again and not stored
        wp[i] = static_cast<const uint16_t *>(p.w) + (int64_t)(i < CB ? n : p.N + n) * p.w_stride + c * 8;
    }
#pragma unroll
    for (int i = 0; i < TT; ++i) {
        int t = t0 + i * 16 + r;
        t = t < (int)p.T ? t : (int)p.T - 1;
        xp[i] = static_cast<const uint16_t *>(p.x) + (int64_t)t * p.x_stride + c * 8;
    }
    const int strips = (p.K + 63) / 64;
    const int n_mine = wave < strips ? (strips - wave + W - 1) / W : 0;
    uint4 a[D][RT][2], b[D][TT][2];
    auto load = [&](int i, int d) __attribute__((always_inline)) {
        const int k0 = (wave + i * W) * 64;
        if (k0 + 64 <= p.K) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int q = 0; q < RT; ++q) a[d][q][h] = *reinterpret_cast<const uint4 *>(wp[q] + k0 + 32 * h);
#pragma unroll
                for (int q = 0; q < TT; ++q) b[d][q][h] = *reinterpret_cast<const uint4 *>(xp[q] + k0 + 32 * h);
            }
        } else {
            // the depth ends inside the strip: zeros on both sides, so that nothing that lies behind counts
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const bool in = k0 + 32 * h + c * 8 < p.K;
#pragma unroll
                for (int q = 0; q < RT; ++q) a[d][q][h] = in ? *reinterpret_cast<const uint4 *>(wp[q] + k0 + 32 * h) : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int q = 0; q < TT; ++q) b[d][q][h] = in ? *reinterpret_cast<const uint4 *>(xp[q] + k0 + 32 * h) : make_uint4(0, 0, 0, 0);
            }
        }
    };
    f32x4 acc[RT][TT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int q = 0; q < TT; ++q) acc[i][q] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](int d) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < RT; ++i)
#pragma unroll
                for (int q = 0; q < TT; ++q) acc[i][q] = mfma16<F16>(a[d][i][h], b[d][q][h], acc[i][q]);
    };
    // whole groups of D strips, then the rest; what is loaded depends on no condition but at the end
    const int groups = n_mine / D, rest = n_mine - groups * D;
    int i = 0;
    if (groups > 0) {
#pragma unroll
        for (int d = 0; d < D; ++d) load(d, d);
        for (int g = 1; g < groups; ++g) {
#pragma unroll
            for (int d = 0; d < D; ++d) {
                multiply(d);
                load(i + D + d, d);
            }
            i += D;
        }
#pragma unroll
        for (int d = 0; d < D; ++d) {
            multiply(d);
            if (d < rest) load(i + D + d, d);
        }
        i += D;
    } else {
#pragma unroll
        for (int d = 0; d < D; ++d)
            if (d < rest) load(d, d);
    }
#pragma unroll
    for (int d = 0; d < D; ++d)
        if (d < rest) multiply(d);
#pragma unroll
    for (int i2 = 0; i2 < RT; ++i2)
#pragma unroll
        for (int q = 0; q < TT; ++q) part[((wave * RT + i2) * TT + q) * 64 + lane] = acc[i2][q];
    __syncthreads();
    for (int e = tid; e < CB * TT * 64; e += W * 64) {
        f32x4 y = part[e], up = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (GATED) up = part[CB * TT * 64 + e];
        // in the order of the waves
        for (int w = 1; w < W; ++w) {
            y += part[w * RT * TT * 64 + e];
            if constexpr (GATED) up += part[w * RT * TT * 64 + CB * TT * 64 + e];
        }
        const int l = e & 63, q = (e >> 6) % TT, blk = (e >> 6) / TT;
        const int n = n0 + blk * 16 + (l >> 4) * 4;
        finish4<F16, GATED, OUT32>(p, t0 + q * 16 + (l & 15), n, y, up, Bias4<F16, GATED>(p, n));
    }
}

// ---- many rows: tiles through LDS ------------------------------------------------------------------
//
// A workgroup owns BM weights x BN rows of x and walks the depth in strips of 64 elements, which go from memory straight into LDS: a ring of S strips, 2 where LDS holds no more
// and 3 for narrow tiles, which wait for memory (T 64, K 4096, N 6144, 128 x 64: 2 strips 20.3 us, 3 18.3, 4 18.1, 6 18.3).  The loads that refill a strip's slot are
// issued once every wave has read its last operands from it.  Operand reads of a k-step travel under the multiplies of the one
// before; the 16-byte chunks of a row are swizzled so that 16 rows' reads of a chunk are free of bank conflicts.
//
// Multiplies of 16 x 16 x 32: half the accumulator traffic of 32 x 32 x 16, 3 to 7 % faster in every tile (8192^3, 256 x 256: 804, 778 us at the time).  8 waves of 128 x 64
// each are faster than 4 of 128 x 128, whose SIMDs have nothing else to do at a rendezvous (778, 828).  Of 778 us the loads take 92 (timed with the strips left
// where they are: 686), the operand reads some 45 more.
#define RALM_LDS __attribute__((address_space(3)))
#define RALM_SCHED_FENCE() __builtin_amdgcn_sched_barrier(0)

// slot of a row's chunk c: c ^ swizzle(row).  (Free of conflicts for 16 rows x 4 chunks a read; with bit 3 of the row folded in, as 32 rows x 2 chunks
// like it, the LDS worked twice as long: 8192^3 784 us, now 766.)
__device__ __forceinline__ int swizzle(int row) { return row & 7; }

// what a load of a chunk behind the end of a row reads
__device__ const uint4 zero_chunk = {0u, 0u, 0u, 0u};

// 64 lanes x 16 bytes to 1 KB of LDS; not tracked by the compiler, waited for by count.  From a base and the lanes' 32-bit offsets, or from the lanes' own addresses.
__device__ __forceinline__ void dma(const unsigned char *base, uint32_t voff, uint32_t lds_base)
{
    asm volatile(RALM_M0_THEN "global_load_lds_dwordx4 %1, %2" ::"s"(lds_base), "v"(voff), "s"(base) : "memory");
}
__device__ __forceinline__ void dma_at(const unsigned char *at, uint32_t lds_base)
{
    asm volatile(RALM_M0_THEN "global_load_lds_dwordx4 %1, off" ::"s"(lds_base), "v"(at) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_vmcnt()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

template <bool F16, bool GATED, bool OUT32, int WM, int WN, int TM, int TN, int S>
__global__ __launch_bounds__(WM *WN * 64) void linear_tile_kernel(const LinearParams p, const LinearPlan plan, const int n_tiles, const int t_tiles)
{
    constexpr int BM = WM * TM * 16, BN = WN * TN * 16, NW = WM * WN;
    constexpr int NA = BM / 8 / NW, NB = BN / 8 / NW, LPS = NA + NB;   // loads of a wave per strip, 8 rows each
    constexpr int A_BYTES = BM * 128, STAGE = (BM + BN) * 128;
    constexpr int COLS = GATED ? BM / 2 : BM, HALF = TM * 8;
    constexpr bool TOUCH = NW == 8;
    constexpr int NM = TM * TN, NR = TM + TN;
    constexpr int RV = NR + 6 < NM ? NR + 6 : NM - 1;   // the rendezvous follows this multiply of a strip's first k-step
    constexpr int PLACES = NM - 1 - RV + NM - NR;   // multiplies that loads are issued behind: those of the first k-step after the rendezvous, those of the second after its reads
    static_assert(NR <= NM - 1, "a k-step's reads are issued behind its multiplies");
    static_assert(!GATED || TM % 2 == 0, "gates and what they multiply lie in one wave");
    extern __shared__ __align__(16) unsigned char smem[];
    const uint32_t lds0 = (uint32_t)(size_t)(RALM_LDS unsigned char *)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroup b runs on XCD b % 8: an XCD gets consecutive tiles, in patches 4 row tiles high, whose weights and rows its L2 holds together
    const int tiles = n_tiles * t_tiles, total = tiles * plan.parts, per = (total + 7) / 8;
    int id = (int)(blockIdx.x & 7) * per + (int)(blockIdx.x >> 3);
    if (id >= total || (int)(blockIdx.x >> 3) >= per) return;
    const int part = id / tiles;
    id -= part * tiles;
    const int rise = t_tiles <= 8 ? t_tiles : 4;
    const int patch = id / (rise * n_tiles), high = t_tiles - patch * rise < rise ? t_tiles - patch * rise : rise, in = id - patch * rise * n_tiles;
    const int64_t t0 = (int64_t)(patch * rise + in % high) * BN;
    const int n0 = in / high * COLS;

    const unsigned char *wb = static_cast<const unsigned char *>(p.w), *xb = static_cast<const unsigned char *>(p.x);
    const uint32_t ws = (uint32_t)p.w_stride * 2, xs = (uint32_t)p.x_stride * 2;   // at most 2^23 bytes: 256 rows fit 32 bits
    // gated: a wave's rows are its outputs' gates, then what they multiply, N rows on: two bases
    const unsigned char *wbase = wb + (int64_t)n0 * ws, *ubase = GATED ? wbase + (int64_t)p.N * ws : wbase, *xbase = xb + t0 * xs;
    const int lr = lane >> 3, lc = lane & 7;
    uint32_t a_voff[NA], b_voff[NB];
    bool a_up[NA];
#pragma unroll
    for (int j = 0; j < NA; ++j) {
        const int row = (wave * NA + j) * 8 + lr;
        int col = row;
        a_up[j] = false;
        if constexpr (GATED) {
            const int q = row % (2 * HALF);   // a load's 8 rows are of one kind
            col = row / (2 * HALF) * HALF + q % HALF;
            a_up[j] = ((wave * NA + j) * 8) % (2 * HALF) >= HALF;
        }
        col = n0 + col < p.N ? col : p.N - 1 - n0;
        a_voff[j] = (uint32_t)col * ws + (uint32_t)((lc ^ swizzle(row)) << 4);
    }
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        const int row = (wave * NB + j) * 8 + lr;
        const int t = t0 + row < p.T ? row : (int)(p.T - 1 - t0);
        b_voff[j] = (uint32_t)t * xs + (uint32_t)((lc ^ swizzle(row)) << 4);
    }
    const int strips = (p.K + 63) / 64, first = part * plan.part_strips;
    const int KT = strips - first < plan.part_strips ? strips - first : plan.part_strips;   // at least one
    const int tail = first + KT == strips ? p.K & 63 : 0;                                     // elements of the last strip, 0: all
    // Few rows, whose x an XCD's L2 holds: neighbouring tiles begin at other strips of their part and go round, or rows that lie a power of two apart would keep a few
    // channels of the memory busy at a time (weights from HBM, us: T 16, K 16384, N 4096 in 8 parts 42, 30; T 45, K 4096, 22528 gated rows 48.6, 43.7).  A part of 13 strips begins at the same one in
    // every tile, one of 26 at two, and the part that holds a broken strip at its first
    const int begin = !TOUCH && p.T * p.K <= 1 << 20 && !tail ? in / high * 13 % KT : 0;
    int until = KT - begin;
    wbase += (int64_t)(first + begin) * 128;
    xbase += (int64_t)(first + begin) * 128;
    ubase += (int64_t)(first + begin) * 128;
    // TAIL: the strip may end behind the rows
    auto issue = [&](int idx, int slot, auto tail_tag) __attribute__((always_inline)) {
        const bool is_a = idx < NA;
        const int j = is_a ? idx : idx - NA;
        const uint32_t to = lds0 + slot * STAGE + (is_a ? 0 : A_BYTES) + (wave * (is_a ? NA : NB) + j) * 1024;
        const unsigned char *base = is_a ? (GATED && a_up[j] ? ubase : wbase) : xbase;
        const uint32_t voff = is_a ? a_voff[is_a ? j : 0] : b_voff[is_a ? 0 : j];
        if constexpr (decltype(tail_tag)::value) {
            // chunk of the row that this lane fetches: behind the end it is zeros
            const int row = (wave * (is_a ? NA : NB) + j) * 8 + lr;
            const int chunk = lc ^ swizzle(row);
            dma_at(chunk * 8 < tail ? base + voff : reinterpret_cast<const unsigned char *>(&zero_chunk), to);
        } else {
            dma(base, voff, to);
        }
    };
    // The loads of a strip are under way for the time of one, which a line from HBM may exceed.  So workgroups of 8 waves, alone on their CUs, touch a strip's lines AHEAD
    // strips before its loads, to have them in this XCD's L2: one dword a line, into a corner of LDS that nobody reads; a quarter of the weights' rows by each of four
    // neighbours that share them, and of the rows of x likewise.  Weights from HBM, us: 1387 rows, K 4096, N 16384 186, 183 (256 x 256: 213, 200); 4096 rows 455, 428;
    // 8192 rows, K 16384, N 4096 835, 797.  Tiles of 128 x 128, which share CUs, lost 4 % by it.
    constexpr int AHEAD = 2, ROWS_A = BM / 4 / (NW / 2), ROWS_B = BN / 4 / (NW / 2);   // rows that a wave touches
    const unsigned char *touch_base = xbase;
    uint32_t touch_voff = 0;
    if constexpr (TOUCH) {
        if (wave < NW / 2) {
            const int share = in % 4, row = share * (BM / 4) + wave * ROWS_A + lane * ROWS_A / 64, col = GATED ? row % COLS : row;
            touch_base = GATED && share >= 2 ? ubase : wbase;
            touch_voff = (uint32_t)(n0 + col < p.N ? col : p.N - 1 - n0) * ws;
        } else {
            const int row = in / high % 4 * (BN / 4) + (wave - NW / 2) * ROWS_B + lane * ROWS_B / 64;
            touch_voff = (uint32_t)(t0 + row < p.T ? row : (int)(p.T - 1 - t0)) * xs;
        }
    }
    auto touch = [&](int strip) __attribute__((always_inline)) {
        const unsigned char *at = touch_base + (int64_t)(strip < KT ? strip : KT - 1) * 128;   // every strip begins inside the rows
        asm volatile(RALM_M0_THEN "global_load_lds_dword %1, %2" ::"s"(lds0 + S * STAGE + wave * 256), "v"(touch_voff), "s"(at) : "memory");
    };
    auto next = [&]() __attribute__((always_inline)) {
        const int64_t step = !TOUCH && --until == 0 ? 128 - KT * 128 : 128;
        wbase += step;
        xbase += step;
        if constexpr (GATED) ubase += step;
    };
#pragma unroll
    for (int s = 0; s < S; ++s) {
        if (s < KT) {
            if (s == KT - 1 && tail) {
#pragma unroll
                for (int idx = 0; idx < LPS; ++idx) issue(idx, s, std::true_type{});
            } else {
#pragma unroll
                for (int idx = 0; idx < LPS; ++idx) issue(idx, s, std::false_type{});
            }
            next();
        }
    }

    const int fr = lane & 15, hi = lane >> 4;
    const int sw = swizzle(fr);
    const int a_off = (wm * TM * 16 + fr) * 128 + ((hi ^ sw) << 4);
    const int b_off = A_BYTES + (wn * TN * 16 + fr) * 128 + ((hi ^ sw) << 4);
    uint4 fa[2][TM], fb[2][TN];
    auto read = [&](int set, int slot, int kk, int idx) __attribute__((always_inline)) {
        const unsigned char *at = smem + slot * STAGE;
        // in the order in which the multiplies need them: A0, all of B, then A1 ..
        if (idx == 0 || idx > TN) {
            const int i = idx == 0 ? 0 : idx - TN;
            fa[set][i] = *reinterpret_cast<const uint4 *>(at + (a_off ^ (kk << 6)) + i * 16 * 128);
        } else {
            fb[set][idx - 1] = *reinterpret_cast<const uint4 *>(at + (b_off ^ (kk << 6)) + (idx - 1) * 16 * 128);
        }
    };
    f32x4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // behind the loads of every strip there is one touch (of the first strips: one in all)
    if constexpr (TOUCH) touch(2);
    // waits until but `strips` strips' loads are complete, as far as that many are under way
    auto wait_but = [&](int strips) __attribute__((always_inline)) {
        if (strips >= S - 1) wait_vmcnt<(S - 1) * LPS + TOUCH>();
        else if (S > 2 && strips == S - 2) wait_vmcnt<(S > 2 ? S - 2 : 0) * LPS + TOUCH>();
        else if (S > 3 && strips == S - 3) wait_vmcnt<(S > 3 ? S - 3 : 0) * LPS + TOUCH>();
        else if (S > 4 && strips == S - 4) wait_vmcnt<(S > 4 ? S - 4 : 0) * LPS + TOUCH>();
        else if (S > 5 && strips == S - 5) wait_vmcnt<(S > 5 ? S - 5 : 0) * LPS + TOUCH>();
        else wait_vmcnt<TOUCH>();
    };
    static_assert(S >= 2 && S <= 6 && (S - 1) * LPS + TOUCH < 64 && (S == 2 || !TOUCH), "loads under way");
    wait_but(KT - 1 < S - 1 ? KT - 1 : S - 1);
    __syncthreads();
#pragma unroll
    for (int idx = 0; idx < NR; ++idx) read(0, 0, 0, idx);

    int kt = 0;
    // One strip.  LOADS: the strip behind the next one is loaded; TAIL: it may end behind the rows; LAST: there is no next one
    int slot = 0;
    auto stage = [&](auto loads_tag, auto tail_tag, auto last_tag) __attribute__((always_inline)) {
        constexpr bool LOADS = decltype(loads_tag)::value, LAST = decltype(last_tag)::value;
        const int after = slot + 1 == S ? 0 : slot + 1;
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            if constexpr (NW == 8) {
                // two waves share a SIMD: the one further along its strip goes first, so that they take turns
                if (kk == 0) __builtin_amdgcn_s_setprio(0);
                else __builtin_amdgcn_s_setprio(1);
            }
            const int cur = kk;
            RALM_SCHED_FENCE();
#pragma unroll
            for (int m = 0; m < NM; ++m) {
                acc[m / TN][m % TN] = mfma16<F16>(fa[cur][m / TN], fb[cur][m % TN], acc[m / TN][m % TN]);
                if (m < NR && !(LAST && kk == 1)) read(cur ^ 1, kk == 1 ? after : slot, kk ^ 1, m);
                if (kk == 0 && m == RV && !LAST) {
                    // the next strip is complete (what is under way are the strips behind it, and a touch), and every wave has read this one
                    if constexpr (LOADS) wait_vmcnt<(S - 2) * LPS + TOUCH>();
                    else wait_but(KT - 2 - kt);
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
                if (LOADS && (kk == 0 ? m > RV : m >= NR)) {
                    const int at = kk == 0 ? m - RV - 1 : NM - 1 - RV + m - NR;
#pragma unroll
                    for (int l = 0; l < LPS; ++l)
                        if (l * PLACES / LPS == at) issue(l < NB ? NA + l : l - NB, slot, tail_tag);
                }
                RALM_SCHED_FENCE();
            }
        }
        if constexpr (LOADS) {
            if constexpr (TOUCH) touch(kt + 2 + AHEAD);
            next();
        }
        slot = after;
    };
    for (; kt < KT - S - (tail ? 1 : 0); ++kt) stage(std::true_type{}, std::false_type{}, std::false_type{});
    if (kt < KT - S) {
        stage(std::true_type{}, std::true_type{}, std::false_type{});
        ++kt;
    }
    for (; kt < KT - 1; ++kt) stage(std::false_type{}, std::false_type{}, std::false_type{});
    stage(std::false_type{}, std::false_type{}, std::true_type{});
    wait_vmcnt<0>();   // touches: before LDS is anybody else's
    __syncthreads();   // other waves read operands where the sums go
    // The sums by way of LDS, 32 rows of x at a time, so that a row's outputs leave side by side, and in a loop: written out for every register, the code below would be
    // fetched from memory for every tile.  A wave's place is its own.
    constexpr int WIDTH = TM * 16, PITCH = WIDTH + 4, OUTS = GATED ? WIDTH / 2 : WIDTH, LANES = OUTS / 4, ROWS = 64 / LANES;
    static_assert(NW * 32 * PITCH * 4 <= 160 * 1024, "LDS of the epilogue");
    float *own = reinterpret_cast<float *>(smem) + wave * 32 * PITCH;
    const int n_lane = (lane % LANES) * 4, n = n0 + wm * OUTS + n_lane;
    const Bias4<F16, GATED> bias(p, n);
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                *reinterpret_cast<f32x4 *>(own + (c * 16 + fr) * PITCH + i * 16 + hi * 4) = acc[i][j + c];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 4
        for (int r = lane / LANES; r < 32; r += ROWS) {
            const f32x4 y = *reinterpret_cast<const f32x4 *>(own + r * PITCH + n_lane);
            f32x4 up = y;
            if constexpr (GATED) up = *reinterpret_cast<const f32x4 *>(own + r * PITCH + OUTS + n_lane);
            const int64_t t = t0 + (wn * TN + j) * 16 + r;
            if (plan.parts == 1) {
                finish4<F16, GATED, OUT32>(p, t, n, y, up, bias);
            } else if (t < p.T && n < p.N) {
                float *to = plan.sums + ((int64_t)part * p.T + t) * plan.pitch + n;   // places behind N are the pitch's
                *reinterpret_cast<f32x4 *>(to) = y;
                if constexpr (GATED) *reinterpret_cast<f32x4 *>(to + plan.pitch / 2) = up;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

// Sums of the parts of a depth, in their order, and what follows: 3 to 4 us for 64 rows of 6144 in 4 parts, a launch and one trip to L2
template <bool F16, bool GATED, bool OUT32>
__global__ __launch_bounds__(256) void linear_join_kernel(const LinearParams p, const LinearPlan plan)
{
    const int quads = (p.N + 3) / 4;
    const uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const int64_t t = i / (uint32_t)quads;
    if (t >= p.T) return;
    const int n = (int)(i - (uint32_t)t * quads) * 4;
    const float *from = plan.sums + t * plan.pitch + n;
    const int64_t part = p.T * plan.pitch;
    f32x4 y = f32x4{0.f, 0.f, 0.f, 0.f}, up = y;
#pragma unroll 4
    for (int k = 0; k < plan.parts; ++k) {
        y += *reinterpret_cast<const f32x4 *>(from + k * part);
        if constexpr (GATED) up += *reinterpret_cast<const f32x4 *>(from + k * part + plan.pitch / 2);
    }
    finish4<F16, GATED, OUT32>(p, t, n, y, up, Bias4<F16, GATED>(p, n));
}

// ---- launches ----------------------------------------------------------------------------------------

template <bool F16, bool GATED, bool OUT32, int RT, int TT, int W, int D>
hipError_t launch_few(const LinearParams &p, hipStream_t stream)
{
    constexpr int CB = GATED ? RT / 2 : RT;
    const int n_tiles = (p.N + CB * 16 - 1) / (CB * 16), t_tiles = (int)((p.T + TT * 16 - 1) / (TT * 16));
    const size_t lds = (size_t)W * RT * TT * 64 * 16;
    auto kernel = linear_few_kernel<F16, GATED, OUT32, RT, TT, W, D>;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (once != hipSuccess) return once;
    kernel<<<dim3((unsigned)((n_tiles + 7) / 8 * 8 * t_tiles)), W * 64, lds, stream>>>(p, n_tiles, t_tiles);
    return hipGetLastError();
}
template <bool F16, bool GATED, bool OUT32, int WM, int WN, int TM, int TN, int S = 2>
hipError_t launch_tile(const LinearParams &p, const LinearPlan &plan, hipStream_t stream)
{
    constexpr int BM = WM * TM * 16, BN = WN * TN * 16, COLS = GATED ? BM / 2 : BM;
    const int64_t n_tiles = (p.N + COLS - 1) / COLS, t_tiles = (p.T + BN - 1) / BN;
    const size_t ring = S * (size_t)(BM + BN) * 128 + (WM * WN == 8 ? 8 * 256 : 0), sums = (size_t)WM * WN * 32 * (TM * 16 + 4) * 4, lds = ring > sums ? ring : sums;
    auto kernel = linear_tile_kernel<F16, GATED, OUT32, WM, WN, TM, TN, S>;
    static const hipError_t once = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (once != hipSuccess) return once;
    kernel<<<dim3((unsigned)((n_tiles * t_tiles * plan.parts + 7) / 8 * 8)), WM * WN * 64, lds, stream>>>(p, plan, (int)n_tiles, (int)t_tiles);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || plan.parts == 1) return e;
    const int64_t quads = (int64_t)p.T * ((p.N + 3) / 4);
    linear_join_kernel<F16, GATED, OUT32><<<dim3((unsigned)((quads + 255) / 256)), 256, 0, stream>>>(p, plan);
    return hipGetLastError();
}

template <bool F16, bool GATED, bool OUT32>
hipError_t launch(const LinearParams &p, const LinearPlan &plan, hipStream_t stream)
{
    switch (plan.form) {
    case LINEAR_FEW_16: return launch_few<F16, GATED, OUT32, GATED ? 2 : 1, 1, 8, 4>(p, stream);   // (gated: 16 gates and 16 that they multiply)
    case LINEAR_FEW_32: return launch_few<F16, GATED, OUT32, GATED ? 4 : 2, 1, 8, GATED ? 2 : 4>(p, stream);
    case LINEAR_64x64: return launch_tile<F16, GATED, OUT32, 1, 2, 4, 2, 3>(p, plan, stream);
    case LINEAR_128x64: return launch_tile<F16, GATED, OUT32, 2, 2, 4, 2, 3>(p, plan, stream);
    case LINEAR_128x128: return launch_tile<F16, GATED, OUT32, 2, 2, 4, 4>(p, plan, stream);
    case LINEAR_256x192: return launch_tile<F16, GATED, OUT32, 4, 2, 4, 6>(p, plan, stream);
    default: return launch_tile<F16, GATED, OUT32, 2, 4, 8, 4>(p, plan, stream);
    }
}
template <bool F16>
hipError_t launch_of(const LinearParams &p, const LinearPlan &plan, hipStream_t stream)
{
    const bool o32 = p.out_dtype == DT_F32;
    if (p.gated) return o32 ? launch<F16, true, true>(p, plan, stream) : launch<F16, true, false>(p, plan, stream);
    return o32 ? launch<F16, false, true>(p, plan, stream) : launch<F16, false, false>(p, plan, stream);
}

}  // namespace

// Which form, and over how many workgroups the depth is split: the one that a simple model of the time (us) says is fastest.
//
//   few   a start, a wave's share of the strips times what shares a CU, and what goes through the L1 caches (up to 16 rows of x for every 16 to 64 weights)
//   tiles a start; for every round of workgroups its strips, each as long as the multiplies of the workgroups that share a CU, as a latency, or as the weights' way from
//         memory, whichever is longest, and an epilogue; for parts a second launch and the way of their sums to memory and back
//
// The constants are a fit to 9000 measured calls (K 256 to 16384, N 500 to 50257, T 1 to 4096, gated and not, 1 to 16 parts; weights from HBM where they are more than a
// few MB).  Over these sizes the form that is taken is 1.2 % slower than the fastest one in the mean and 24 % at most (T 16, K 6144, N 2048: 14.6, 11.8 us).  What it
// decides between, us: T 1, K = N = 1024: few 4.7, tiles 7.5; T 64, K 4096, N 6144: few 25, tiles of 128 x 64 in 4 parts 16.7; T 1387, K 4096, N 6144: tiles of
// 128 x 128 100, of 256 x 192 74, of 256 x 256 85.
//
// consider(form, parts, us) for everything that may be taken
template <class F>
static void linear_candidates(int64_t T, int32_t N, int32_t K, int32_t gated, F consider)
{
    struct Tile {
        int32_t form, bm, bn, per_cu;
        float latency, multiply, epilogue;
    };
    static const Tile tiles[] = {{LINEAR_64x64, 64, 64, 3, 0.35f, 0.364f, 1.48f},
                                 {LINEAR_128x64, 128, 64, 2, 0.01f, 0.421f, 3.22f},
                                 {LINEAR_128x128, 128, 128, 2, 0.95f, 0.53f, 3.02f},
                                 {LINEAR_256x192, 256, 192, 1, 0.6f, 1.17f, 6.3f},
                                 {LINEAR_256x256, 256, 256, 1, 0.35f, 1.34f, 8.8f}};
    static const int32_t parts_of[] = {1, 2, 3, 4, 6, 8, 12, 16};
    constexpr int CUS = 256;
    const int64_t rows = (int64_t)N << gated;
    const int32_t strips = (K + 63) / 64;
    auto ceil_div = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    if (T <= 256) {
        static const float strip[] = {0.249f, 0.593f, 2.256f};   // of 16, 32, 64 weights
        for (int f = 0; f < 2; ++f) {
            const int kind = f + gated, bm = 16 << kind;
            const float wgs = (float)(ceil_div(rows, bm) * ceil_div(T, 16)), load = wgs / 210.f;
            consider(f ? LINEAR_FEW_32 : LINEAR_FEW_16, 1,
                     0.84f + (float)ceil_div(strips, 8) * strip[kind] * (load > 1.f ? load : 1.f) + wgs * (float)(bm + (T < 16 ? T : 16)) * (float)K * (2.f / 11.9e6f));
        }
    }
    for (const Tile &tile : tiles) {
        const int64_t t_tiles = ceil_div(T, tile.bn), all = ceil_div(rows, tile.bm) * t_tiles;
        const int64_t slots = CUS * tile.per_cu;
        auto strip = [&](int64_t wgs, int per_cu) {
            const float m = per_cu * tile.multiply, bytes = (float)wgs / (float)t_tiles * tile.bm * 128.f;
            const float w = fmaxf(tile.latency + bytes / 53.5e6f, bytes / 8.7e6f);
            return m > w ? m : w;
        };
        for (int32_t parts : parts_of) {
            // at least two strips a part; sums of less than 2^31 numbers
            if (parts > 1 && (strips / parts < 2 || T * rows > LINEAR_MAX_SUMS / parts)) break;
            const int64_t wgs = all * parts, full = wgs / slots, rest = wgs - full * slots;
            const float n = (float)ceil_div(strips, parts);
            float t = 0.62f + (float)full * (n * strip(slots, tile.per_cu) + tile.epilogue);
            if (rest) t += n * strip(rest, (int)ceil_div(rest, CUS)) + tile.epilogue;
            if (parts > 1) t += 2.92f + (float)parts * (float)(T * rows) * (8.f / 4.7e6f);
            consider(tile.form, parts, t);
        }
    }
}

LinearPlan linear_plan(int64_t T, int32_t N, int32_t K, int32_t gated)
{
    LinearPlan plan;
    float best = 0.f;
    plan.form = -1;
    plan.parts = 1;
    linear_candidates(T, N, K, gated, [&](int32_t form, int32_t parts, float t) {
        if (plan.form < 0 || t < best) plan.form = form, plan.parts = parts, best = t;
    });
    const int32_t strips = (K + 63) / 64;
    plan.part_strips = (strips + plan.parts - 1) / plan.parts;
    plan.parts = (strips + plan.part_strips - 1) / plan.part_strips;   // none without a strip
    plan.pitch = (int64_t)((N + 3) / 4 * 4) << gated;
    plan.sums = nullptr;
    return plan;
}

// The most parts x rows that any call of up to T rows has.  From 257 rows on, 64 at a time: among them every form has the same tiles, and its time is a constant
// plus parts x rows x another one for all forms.  So what is fastest for more of the rows has no more parts than what is for the first one, except that roundings of
// fp32 may show where two are as fast; forms within 1e-5 of the fastest count as well.
int64_t linear_most_sums(int64_t T, int32_t N, int32_t K, int32_t gated)
{
    int64_t most = 0;
    for (int64_t t = 1; t <= T && t <= 256; ++t) {
        const int32_t parts = linear_plan(t, N, K, gated).parts;
        if (parts > 1 && parts * t > most) most = parts * t;
    }
    const int64_t rows = (int64_t)N << gated;
    const int32_t strips = (K + 63) / 64;
    for (int64_t t = 257; t <= T && t * rows <= LINEAR_MAX_SUMS / 2; t += 64) {
        const int64_t last = T - t < 64 ? T : t + 63;
        float best = 3.4e38f;
        linear_candidates(t, N, K, gated, [&](int32_t, int32_t, float us) { best = fminf(best, us); });
        int32_t parts = 1;
        linear_candidates(t, N, K, gated, [&](int32_t, int32_t p, float us) {
            if (us <= best * (1.f + 1e-5f) && p > parts) parts = p;
        });
        const int32_t each = (strips + parts - 1) / parts;
        parts = (strips + each - 1) / each;
        if (parts > 1 && parts * last > most) most = parts * last;
    }
    return most;
}

hipError_t launch_linear(const LinearParams &p, const LinearPlan &plan, hipStream_t stream)
{
    return p.dtype == DT_F16 ? launch_of<true>(p, plan, stream) : launch_of<false>(p, plan, stream);
}

}  // namespace ralm
