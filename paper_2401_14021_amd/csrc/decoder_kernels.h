// Launchers of the operators around the generator's attention (internal to libralm.so): products with epilogues, norms of the
// residual stream, rotary positions into the 4-bit cache, the target of a verification.  Every launcher only enqueues work on
// `stream`; argument validation happens in decoder_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kv_kernels.h"

namespace ralm {

struct LinearParams {
    const void *x, *w;
    int64_t x_stride, w_stride;   // elements
    int64_t T;
    int32_t N, K, dtype;
    const void *bias;
    int32_t act, gated;
    const void *residual;
    int64_t residual_stride;
    void *out;
    int64_t out_stride;
    int32_t out_dtype;
};
// weights x rows of a workgroup
enum { LINEAR_FEW_16, LINEAR_FEW_32, LINEAR_64x64, LINEAR_128x64, LINEAR_128x128, LINEAR_256x192, LINEAR_256x256 };
struct LinearPlan {
    int32_t form;
    int32_t parts, part_strips;   // of the depth: workgroups that share it, strips of 64 each
    int64_t pitch;                // of the parts' sums, [parts][T][pitch]
    float *sums;
};
constexpr int64_t LINEAR_MAX_SUMS = 1LL << 31;   // numbers that a split depth leaves
LinearPlan linear_plan(int64_t T, int32_t N, int32_t K, int32_t gated);
int64_t linear_most_sums(int64_t T, int32_t N, int32_t K, int32_t gated);   // parts x rows, of any number of rows up to T; 0: nothing is split
hipError_t launch_linear(const LinearParams &p, const LinearPlan &plan, hipStream_t stream);

hipError_t launch_residual_norm(const ralm_norm_t &p, hipStream_t stream);

struct KvRotary {
    const void *q;
    void *q_out;
    int64_t q_token, q_head, o_token, o_head;   // strides in elements
    int32_t n_q_heads;
    const double *freqs;
    int32_t half;          // pairs of a head that turn
    int32_t interleaved;
    double amplitude;
    const int32_t *shift;  // [R] or NULL
};
hipError_t launch_kv_append_rotary(const KvView &kv, const KvRows &rows, const KvRotary &turn, hipStream_t stream);

struct TargetParams {
    const void *logits;
    int64_t logits_stride;
    int64_t Q;
    int32_t V, dtype;
    float scale;           // log2 e / temperature
    const int32_t *tokens;
    const float *weights;
    int32_t k;
    const float *share;
    float share_all;
    void *out;
    int64_t out_stride;
    int32_t out_dtype;
    int32_t parts;         // workgroups of a row, from target_parts
    float2 *stats;         // [Q][parts]: largest logit and sum of exponentials
};
constexpr int TARGET_PART = 4096;   // entries of a workgroup that shares a row
constexpr int TARGET_FEW = 128;   // rows from which a workgroup takes one whole
int target_parts(int64_t Q, int32_t V);
hipError_t launch_knnlm_target(const TargetParams &p, hipStream_t stream);

}  // namespace ralm
