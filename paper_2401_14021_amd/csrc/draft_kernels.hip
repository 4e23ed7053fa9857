// Verification of drafted tokens against the target's probabilities, from given random numbers.
//
// Draft i, token x, is accepted with probability min(1, p_i(x) / q_i(x)): iff u_i q_i(x) < p_i(x).  At the first one that is not, the
// request's next token is drawn from max(p - q, 0), divided by its sum; behind drafts that were all accepted, from the target's next row.  The tokens are
// then distributed as the target's own.
//
// Everything is done in whole numbers: a probability is P = floor(p 2^36), a random number m = floor(u 2^24).  The multiplication by 2^36 and
// the floor are exact in fp32, differences and sums in 64 bits, so no order of summation can show and a token is the same however a row is
// split: the smallest one whose running sum exceeds floor(m S / 2^24), S the sum of all.
//
//  draft_sums_kernel   a wave per 1024 entries of a request's row, or some of them where there are many: accepts (again in every wave: 3
//                      loads in a row, no launch of their own) and the sums of the entries
//  draft_pick_kernel   a workgroup per request: the 1024 entries in which the running sum passes the line, and the entry
// Rows are read once, but for the 1024 entries that hold the token.  What bounds a small call is the chain offsets -> drafts ->
// probabilities -> row, a large one the conversion of the entries (two to doubles, a difference, a maximum and a sum of doubles each).
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "kv_kernels.h"

namespace ralm {

namespace {

constexpr float FIX = 68719476736.0f;   // 2^36

template <int DT>
__device__ __forceinline__ float entry(const void *p, int64_t i)
{
    if constexpr (DT == DT_F32) return static_cast<const float *>(p)[i];
    const uint16_t h = static_cast<const uint16_t *>(p)[i];
    return DT == DT_F16 ? f16_bits_to_f32(h) : __uint_as_float((uint32_t)h << 16);
}
// floor(p 2^36) of a probability as a whole number in fp32; NaN counts as 0
__device__ __forceinline__ float fixed(float p) { return floorf(fminf(fmaxf(p, 0.0f), 1.0f) * FIX); }
__device__ __forceinline__ u64 random24(float u) { return (u64)(fminf(fmaxf(u, 0.0f), 0.99999994f) * 16777216.0f); }

// N entries of a row from i on, which is aligned to its type alone: one load of up to 16 bytes; zeros behind V
template <int DT, int N>
__device__ __forceinline__ void entries(const void *row, int64_t i, int V, float (&x)[N])
{
    if (i + N <= V) {
        if constexpr (DT == DT_F32) {
            __builtin_memcpy(x, static_cast<const float *>(row) + i, 4 * N);
        } else {
            uint16_t h[N];
            __builtin_memcpy(h, static_cast<const uint16_t *>(row) + i, 2 * N);
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = DT == DT_F16 ? f16_bits_to_f32(h[j]) : __uint_as_float((uint32_t)h[j] << 16);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = i + j < V ? entry<DT>(row, i + j) : 0.0f;
    }
}

// one request's drafts [first, first + count); count of accepted ones, by all lanes of a wave
template <int DT>
__device__ __forceinline__ int accepted_of(const DraftParams &p, int64_t r, int64_t first, int count)
{
    for (int at = 0; at < count; at += 64) {
        const int i = at + (threadIdx.x & 63);
        bool good = true;
        if (i < count) {
            const int64_t d = first + i;
            const int32_t x = p.draft_ids[d];
            good = false;
            if (x >= 0 && x < p.V) {
                const u64 P = (u64)fixed(entry<DT>(p.target_probs, (d + r) * p.target_stride + x));
                const u64 Q = p.draft_probs ? (u64)fixed(entry<DT>(p.draft_probs, d * p.draft_stride + x)) : (u64)FIX;
                good = random24(p.u[d]) * Q < P << 24;
            }
        }
        const uint64_t bad = __ballot(!good);
        if (bad) return at + __builtin_ctzll(bad);
    }
    return count;
}

// the rows that the next token is drawn from: q NULL where none is taken off; hot: the entry that a draft without probabilities takes off, or -1
struct Rows {
    const char *p, *q;
    int hot;
};
template <int DT>
__device__ __forceinline__ Rows rows_of(const DraftParams &p, int64_t r, int64_t first, int count, int n)
{
    constexpr int es = DT == DT_F32 ? 4 : 2;
    Rows w;
    w.p = static_cast<const char *>(p.target_probs) + (first + r + n) * p.target_stride * es;
    w.q = n < count && p.draft_probs ? static_cast<const char *>(p.draft_probs) + (first + n) * p.draft_stride * es : nullptr;
    w.hot = n < count && !p.draft_probs ? p.draft_ids[first + n] : -1;
    return w;
}
// N entries' weights (whole numbers)
template <int DT, int N>
__device__ __forceinline__ void weights(const Rows &w, int64_t i, int V, double (&x)[N])
{
    float p[N], q[N] = {};
    entries<DT, N>(w.p, i, V, p);
    if (w.q) entries<DT, N>(w.q, i, V, q);
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = i + j == w.hot ? 0.0 : fmax((double)fixed(p[j]) - (double)fixed(q[j]), 0.0);
}
// the sum of chunk c's weights, by all lanes of a wave; 1024 entries of at most 2^36 are exact in a double
template <int DT>
__device__ __forceinline__ u64 chunk_sum(const Rows &w, int64_t c, int V)
{
    constexpr int N = DT == DT_F32 ? 4 : 8;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < DRAFT_CHUNK / (64 * N); ++i) {
        double x[N];
        weights<DT, N>(w, c * DRAFT_CHUNK + i * (64 * N) + (threadIdx.x & 63) * N, V, x);
#pragma unroll
        for (int j = 0; j < N; j += 4) sum += (x[j] + x[j + 1]) + (x[j + 2] + x[j + 3]);
    }
    return (u64)wave64_sum(sum);
}
__device__ __forceinline__ int64_t clamp_row(int64_t o, int64_t n) { return o < 0 ? 0 : o > n ? n : o; }

// per: chunks of a wave
template <int DT>
__global__ __launch_bounds__(256) void draft_sums_kernel(DraftParams p, int per)
{
    const int lane = threadIdx.x & 63;
    const int64_t waves = (p.chunks + per - 1) / per;   // of a request
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (unit >= p.R * waves) return;
    const int64_t r = unit / waves, c0 = unit % waves * per, c1 = c0 + per < p.chunks ? c0 + per : p.chunks;
    const int64_t first = clamp_row(p.offsets[r], p.Qt), end = clamp_row(p.offsets[r + 1], p.Qt);
    const int count = end > first ? (int)(end - first) : 0;
    const int n = accepted_of<DT>(p, r, first, count);
    if (c0 == 0 && lane == 0) p.accepted[r] = n;
    const Rows w = rows_of<DT>(p, r, first, count, n);
    for (int64_t c = c0; c < c1; ++c) {
        const u64 sum = chunk_sum<DT>(w, c, p.V);
        if (lane == 0) p.sums[r * p.chunks + c] = sum;
    }
}

__device__ __forceinline__ u64 shfl_up_u64(u64 v, int s)
{
    return (u64)(uint32_t)__shfl_up((int)(uint32_t)(v >> 32), s, 64) << 32 | (uint32_t)__shfl_up((int)(uint32_t)v, s, 64);
}
// the sum of v over the threads in front of this one, and over all 256
__device__ __forceinline__ u64 sum_before(u64 v, u64 *red, u64 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 incl = v;
    for (int s = 1; s < 64; s <<= 1) {
        const u64 up = shfl_up_u64(incl, s);
        if (lane >= s) incl += up;
    }
    __syncthreads();
    if (lane == 63) red[wave] = incl;
    __syncthreads();
    u64 before = 0;
    total = 0;
    for (int w = 0; w < 4; ++w) {
        before += w < wave ? red[w] : 0;
        total += red[w];
    }
    return before + incl - v;
}

template <int DT>
__global__ __launch_bounds__(256) void draft_pick_kernel(DraftParams p)
{
    __shared__ u64 red[4];
    __shared__ int64_t s_chunk;
    __shared__ u64 s_before;
    const int64_t r = blockIdx.x;
    const int tid = threadIdx.x;
    const int64_t first = clamp_row(p.offsets[r], p.Qt), end = clamp_row(p.offsets[r + 1], p.Qt);
    const int count = end > first ? (int)(end - first) : 0;
    u64 *sums = p.sums + r * p.chunks;
    const u64 m = random24(p.u_next[r]);
    Rows w = rows_of<DT>(p, r, first, count, p.accepted[r]);
    // neighbouring chunks per thread
    const int64_t per = (p.chunks + 255) / 256, c0 = tid * per, c1 = c0 + per < p.chunks ? c0 + per : p.chunks;
    u64 mine, before, S;
    for (int again = 0;; ++again) {
        mine = 0;
        for (int64_t c = c0; c < c1; ++c) mine += sums[c];
        before = sum_before(mine, red, S);
        if (S != 0 || again || (!w.q && w.hot < 0)) break;
        // nothing is left beside the draft: the target alone
        w.q = nullptr;
        w.hot = -1;
        for (int64_t c = tid >> 6; c < p.chunks; c += 4) {
            const u64 sum = chunk_sum<DT>(w, c, p.V);
            if ((tid & 63) == 0) sums[c] = sum;
        }
        __threadfence_block();
        __syncthreads();
    }
    if (S == 0) {
        if (tid == 0) p.next[r] = -1;
        return;
    }
    const u64 t = __umul64hi(m, S) << 40 | (m * S) >> 24;   // < S
    u64 run = before;
    if (t >= run && t - run < mine) {   // one thread alone
        for (int64_t c = c0; c < c1; ++c) {
            const u64 x = sums[c];
            if (t - run < x) {
                s_chunk = c;
                s_before = run;
                break;
            }
            run += x;
        }
    }
    __syncthreads();
    const int64_t i = s_chunk * DRAFT_CHUNK + tid * 4;
    double y[4];
    weights<DT, 4>(w, i, p.V, y);
    u64 x[4], sum = 0, whole;
#pragma unroll
    for (int j = 0; j < 4; ++j) sum += x[j] = (u64)y[j];
    run = s_before + sum_before(sum, red, whole);
    if (t >= run && t - run < sum) {
        int j = 0;
        while (j < 3 && t - run >= x[j]) run += x[j++];
        p.next[r] = (int32_t)(i + j);
    }
}

template <int DT>
hipError_t verify_draft(const DraftParams &p, hipStream_t stream)
{
    // a wave of its own per chunk while all waves are on the chip at once (256 CUs, 16 waves each)
    const int per = (int)((p.R * p.chunks + 4095) / 4096), waves = (int)((p.chunks + per - 1) / per);
    draft_sums_kernel<DT><<<(unsigned)((p.R * waves + 3) / 4), 256, 0, stream>>>(p, per);
    draft_pick_kernel<DT><<<(unsigned)p.R, 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_verify_draft(const DraftParams &p, hipStream_t stream)
{
    return p.dtype == DT_F32 ? verify_draft<DT_F32>(p, stream) : p.dtype == DT_BF16 ? verify_draft<DT_BF16>(p, stream) : verify_draft<DT_F16>(p, stream);
}

}  // namespace ralm
