// C ABI of the operators around the generator's attention: argument checks (on the host, before any launch) and launches.  See include/ralm.h.
#include <hip/hip_runtime.h>
#include <math.h>

#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

using namespace ralm;

namespace {

constexpr int64_t MAX_ROWS = 1 << 22;       // keeps every launch below 2^32 work-items
constexpr int64_t MAX_STRIDE = 1 << 22;     // of x and w: 32-bit offsets inside a tile
constexpr int32_t MAX_K_LINEAR = 1 << 17;

ralm_status launched(hipError_t e)
{
    return e == hipSuccess ? RALM_OK : set_error(RALM_ERR_DEVICE, "launch failed: %s", hipGetErrorString(e));
}
bool aligned(const void *p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool known(int32_t dt) { return dt == RALM_F32 || dt == RALM_BF16 || dt == RALM_F16; }
size_t bytes_of(int32_t dt) { return dt == RALM_F32 ? 4 : 2; }

ralm_status check_linear(int64_t T, int32_t N, int32_t K, int32_t gated)
{
    if (gated != 0 && gated != 1) return set_error(RALM_ERR_RANGE, "gated must be 0 or 1");
    if (T < 0 || T > MAX_ROWS) return set_error(RALM_ERR_SHAPE, "T=%lld out of [0, 2^22]", (long long)T);
    if (N < 1 || N > (1 << 20) >> gated) return set_error(RALM_ERR_SHAPE, "N=%d out of [1, 2^20] (2^19 gated)", N);
    if (K < 8 || K > MAX_K_LINEAR || K % 8) return set_error(RALM_ERR_SHAPE, "K=%d must be a multiple of 8 in [8, 2^17]", K);
    if (T * N > 1LL << (36 - gated)) return set_error(RALM_ERR_SHAPE, "T x N beyond 2^36 (2^35 gated); split the rows");
    return RALM_OK;
}
size_t sums_bytes(const LinearPlan &plan, int64_t T) { return plan.parts > 1 ? (size_t)plan.parts * T * plan.pitch * 4 : 0; }

}  // namespace

extern "C" {

size_t ralm_linear_workspace_bytes(int64_t T, int32_t N, int32_t K, int32_t gated)
{
    if (check_linear(T, N, K, gated) != RALM_OK || T == 0) return 0;
    return (size_t)linear_most_sums(T, N, K, gated) * linear_plan(T, N, K, gated).pitch * 4;
}
size_t ralm_linear_workspace_bytes_exact(int64_t T, int32_t N, int32_t K, int32_t gated)
{
    if (check_linear(T, N, K, gated) != RALM_OK || T == 0) return 0;
    return sums_bytes(linear_plan(T, N, K, gated), T);
}

ralm_status ralm_linear(const void *x, int64_t x_stride, int64_t T, const void *w, int64_t w_stride, int32_t N, int32_t K, int32_t dtype,
                        const void *bias, int32_t act, int32_t gated, const void *residual, int64_t residual_stride, void *out, int64_t out_stride,
                        int32_t out_dtype, void *workspace, size_t workspace_bytes, void *stream)
{
    const ralm_status st = check_linear(T, N, K, gated);
    if (st != RALM_OK) return st;
    if (dtype != RALM_BF16 && dtype != RALM_F16) return set_error(RALM_ERR_DTYPE, "dtype must be RALM_BF16 or RALM_F16");
    if (out_dtype != dtype && out_dtype != RALM_F32) return set_error(RALM_ERR_DTYPE, "out_dtype must be dtype or RALM_F32");
    if (act < RALM_ACT_NONE || act > RALM_ACT_SILU) return set_error(RALM_ERR_RANGE, "act=%d unknown", act);
    if (T == 0) return RALM_OK;
    if (!x || !w || !out) return set_error(RALM_ERR_NULL, "x/w/out is NULL");
    if (x_stride == 0) x_stride = K;
    if (w_stride == 0) w_stride = K;
    if (out_stride == 0) out_stride = N;
    if (residual_stride == 0) residual_stride = N;
    if (x_stride < K || w_stride < K || out_stride < N || (residual && residual_stride < N))
        return set_error(RALM_ERR_SHAPE, "a stride is shorter than its row");
    if (x_stride > MAX_STRIDE || w_stride > MAX_STRIDE) return set_error(RALM_ERR_SHAPE, "strides of x and w beyond 2^22 elements");
    if (x_stride % 8 || w_stride % 8 || !aligned(x, 16) || !aligned(w, 16))
        return set_error(RALM_ERR_ALIGN, "x and w must be 16-byte aligned, their strides multiples of 8 elements");
    if (!aligned(out, bytes_of(out_dtype)) || !aligned(residual, bytes_of(out_dtype)) || !aligned(bias, 2))
        return set_error(RALM_ERR_ALIGN, "out, residual and bias must be aligned to their type");
    if (out == x || out == w || out == bias) return set_error(RALM_ERR_SHAPE, "out is x, w or bias");
    if (residual == out && residual_stride != out_stride) return set_error(RALM_ERR_SHAPE, "residual is out with another stride");
    LinearPlan plan = linear_plan(T, N, K, gated);
    if (plan.parts > 1) {
        if (!workspace || !aligned(workspace, 16)) return set_error(RALM_ERR_WORKSPACE, "workspace is NULL or not 16-byte aligned");
        if (workspace_bytes < sums_bytes(plan, T)) return set_error(RALM_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, sums_bytes(plan, T));
        plan.sums = static_cast<float *>(workspace);
    }
    LinearParams p;
    p.x = x, p.w = w;
    p.x_stride = x_stride, p.w_stride = w_stride;
    p.T = T;
    p.N = N, p.K = K, p.dtype = dtype;
    p.bias = bias;
    p.act = act, p.gated = gated;
    p.residual = residual;
    p.residual_stride = residual ? residual_stride : 0;
    p.out = out;
    p.out_stride = out_stride;
    p.out_dtype = out_dtype;
    return launched(launch_linear(p, plan, static_cast<hipStream_t>(stream)));
}

ralm_status ralm_residual_norm(const ralm_norm_t *norm, void *stream)
{
    if (!norm) return set_error(RALM_ERR_NULL, "norm is NULL");
    ralm_norm_t p = *norm;
    if (p.T < 0 || p.T > MAX_ROWS || p.D < 1 || p.D > RALM_MAX_NORM)
        return set_error(RALM_ERR_SHAPE, "T=%lld out of [0, 2^22] or D=%d out of [1, %d]", (long long)p.T, p.D, RALM_MAX_NORM);
    if (p.T * p.D > 1LL << 36) return set_error(RALM_ERR_SHAPE, "T x D beyond 2^36; split the rows");
    if (p.kind != RALM_NORM_RMS && p.kind != RALM_NORM_LAYER) return set_error(RALM_ERR_RANGE, "kind=%d unknown", p.kind);
    if ((p.post != 0 && p.post != 1) || (p.gate && p.gate_rows != 0 && p.gate_rows != 1)) return set_error(RALM_ERR_RANGE, "post and gate_rows must be 0 or 1");
    if (!(p.eps >= 0.f) || !isfinite(p.eps) || !isfinite(p.scale)) return set_error(RALM_ERR_RANGE, "eps must not be negative, eps and scale finite");
    if (!known(p.x_dtype) || !known(p.param_dtype) || !known(p.sum_dtype) || !known(p.out_dtype)) return set_error(RALM_ERR_DTYPE, "dtype unknown");
    if (p.T == 0) return RALM_OK;
    if (!p.x || (!p.sum && !p.out)) return set_error(RALM_ERR_NULL, "x is NULL, or both sum and out");
    int64_t *strides[] = {&p.x_stride, &p.gate_stride, &p.residual_stride, &p.sum_stride, &p.out_stride};
    for (int64_t *s : strides) {
        if (*s == 0) *s = p.D;
    }
    if (p.x_stride < p.D || (p.gate && p.gate_rows && p.gate_stride < p.D) || (p.residual && p.residual_stride < p.D) || (p.sum && p.sum_stride < p.D) ||
        (p.out && p.out_stride < p.D))
        return set_error(RALM_ERR_SHAPE, "a stride is shorter than its row");
    const size_t xb = bytes_of(p.x_dtype), wb = bytes_of(p.param_dtype), sb = bytes_of(p.sum_dtype);
    if (!aligned(p.x, xb) || !aligned(p.gate, xb) || !aligned(p.residual, sb) || !aligned(p.sum, sb) || !aligned(p.out, bytes_of(p.out_dtype)) ||
        !aligned(p.weight, wb) || !aligned(p.bias, wb) || !aligned(p.post_weight, wb) || !aligned(p.post_bias, wb))
        return set_error(RALM_ERR_ALIGN, "pointers must be aligned to their type");
    if ((p.sum && p.sum == p.out) || (p.out && p.out == p.residual)) return set_error(RALM_ERR_SHAPE, "out is sum or residual");
    if ((p.sum && p.sum == p.residual && p.sum_stride != p.residual_stride) ||
        (p.sum && p.sum == p.x && (p.sum_stride != p.x_stride || p.sum_dtype != p.x_dtype)) ||
        (p.out && p.out == p.x && (p.out_stride != p.x_stride || p.out_dtype != p.x_dtype)))
        return set_error(RALM_ERR_SHAPE, "an output is an input of another type or stride");
    for (const void *in : {p.gate, p.weight, p.bias, p.post_weight, p.post_bias}) {
        if (in && (in == p.sum || in == p.out)) return set_error(RALM_ERR_SHAPE, "an output is the gate or a parameter");
    }
    return launched(launch_residual_norm(p, static_cast<hipStream_t>(stream)));
}

size_t ralm_knnlm_target_workspace_bytes(int64_t Q, int32_t V)
{
    if (Q < 1 || Q > (1 << 20) || V < 1 || V > RALM_MAX_VOCABULARY) return 0;
    // of up to Q rows: fewer of them may be split where many are not
    size_t most = (size_t)Q * target_parts(Q, V);
    const int64_t few = Q < TARGET_FEW ? Q : TARGET_FEW - 1;
    if (few * target_parts(few, V) > (int64_t)most) most = (size_t)few * target_parts(few, V);
    return most * sizeof(float2);
}

ralm_status ralm_knnlm_target(const void *logits, int64_t logits_stride, int64_t Q, int32_t V, int32_t dtype, float temperature, const int32_t *tokens,
                              const float *weights, int32_t k, const float *share, float share_all, void *out, int64_t out_stride, int32_t out_dtype,
                              void *workspace, size_t workspace_bytes, void *stream)
{
    if (Q < 0 || Q > (1 << 20)) return set_error(RALM_ERR_SHAPE, "Q=%lld out of [0, 2^20]", (long long)Q);
    if (V < 1 || V > RALM_MAX_VOCABULARY) return set_error(RALM_ERR_SHAPE, "V=%d out of [1, %d]", V, RALM_MAX_VOCABULARY);
    if (k < 0 || k > RALM_MAX_K) return set_error(RALM_ERR_K, "k=%d out of [0, %d]", k, RALM_MAX_K);
    if (!known(dtype) || !known(out_dtype)) return set_error(RALM_ERR_DTYPE, "dtype unknown");
    if (!(temperature > 0.f) || !isfinite(temperature) || !isfinite((float)(1.4426950408889634 / (double)temperature))) return set_error(RALM_ERR_RANGE, "temperature must be positive and finite");
    if (!share && !(share_all >= 0.f && share_all <= 1.f)) return set_error(RALM_ERR_RANGE, "share_all must be in [0, 1]");
    if (Q == 0) return RALM_OK;
    if (!logits || !out || (k > 0 && (!tokens || !weights))) return set_error(RALM_ERR_NULL, "a pointer is NULL");
    if (logits_stride == 0) logits_stride = V;
    if (out_stride == 0) out_stride = V;
    if (logits_stride < V || out_stride < V) return set_error(RALM_ERR_SHAPE, "a stride is shorter than its row");
    if (!aligned(logits, bytes_of(dtype)) || !aligned(out, bytes_of(out_dtype)) || !aligned(tokens, 4) || !aligned(weights, 4) || !aligned(share, 4))
        return set_error(RALM_ERR_ALIGN, "pointers must be aligned to their type");
    if (logits == out && (dtype != out_dtype || logits_stride != out_stride)) return set_error(RALM_ERR_SHAPE, "out is logits of another type or stride");
    const int parts = target_parts(Q, V);
    if (Q * parts >= 1 << 24) return set_error(RALM_ERR_SHAPE, "Q x V beyond 2^36; split the batch");
    if (parts > 0) {
        const size_t need = (size_t)Q * parts * sizeof(float2);
        if (!workspace || !aligned(workspace, 16)) return set_error(RALM_ERR_WORKSPACE, "workspace is NULL or not 16-byte aligned");
        if (workspace_bytes < need) return set_error(RALM_ERR_WORKSPACE, "workspace too small: %zu < %zu bytes", workspace_bytes, need);
    }
    TargetParams p;
    p.logits = logits;
    p.logits_stride = logits_stride;
    p.Q = Q;
    p.V = V, p.dtype = dtype;
    p.scale = (float)(1.4426950408889634 / (double)temperature);
    p.parts = parts;
    p.stats = static_cast<float2 *>(workspace);
    p.tokens = tokens;
    p.weights = weights;
    p.k = k;
    p.share = share;
    p.share_all = share_all;
    p.out = out;
    p.out_stride = out_stride;
    p.out_dtype = out_dtype;
    return launched(launch_knnlm_target(p, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
