// Launchers of the generator's operators (internal to libralm.so): the 4-bit paged cache, attention over it, its pages, and the
// verification of drafted tokens.  Every launcher only enqueues work on `stream`; argument validation happens in kv_api.hip.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/ralm.h"

namespace ralm {

// the calling thread's error text (ralm_last_error); returns st
ralm_status set_error(ralm_status st, const char *fmt, ...);

// Layout of the cache.  A page holds page_tokens tokens of every layer and head, [layer][head][tile][17 d] bytes; a tile is 16 tokens of
// one head:
//   8 d   keys    [16 tokens][d / 2]                  two codes a byte, the lower one first
//   8 d   values  [4 quads][16][4 tokens][d / 32]     the n-th sixteenth of the head, of four neighbouring tokens beside each other
//   d / 2 powers of the keys    [16 tokens][d / 32]
//   d / 2 powers of the values  [4 quads][d / 32][4 tokens]
// That is how the matrix instructions of the attention consume them: a lane reads a quarter of a key and its power, and a sixteenth of four
// values and theirs, as one piece each, and the 64 lanes' pieces of a tile lie one behind the other.
constexpr int KV_TILE = 16, KV_BLOCK = 32;
__host__ __device__ inline int kv_tile_bytes(int d) { return 17 * d; }

struct KvView {
    uint8_t *pages;
    int64_t page_bytes;    // of all layers and heads
    int64_t layer_bytes;   // from the page's begin to the layer's
    int64_t head_bytes;
    int32_t n_pages, n_heads, d;
    int32_t tile_shift;    // tiles of a page: 1 << tile_shift
    const int32_t *table;  // [R, max_pages]
    const int32_t *lens;   // [R]
    int32_t R, max_pages;
};

// One call's new tokens: request r's are those in front of its length.
struct KvRows {
    void *k, *v;           // read (append) or written (read)
    int32_t dtype;
    int64_t k_token, k_head, v_token, v_head;   // strides in elements
    const int64_t *offsets;
    int64_t n;
    const int32_t *start;  // place of a request's first token; NULL: its length minus its number of tokens
};
hipError_t launch_kv_append(const KvView &kv, const KvRows &rows, hipStream_t stream);
hipError_t launch_kv_read(const KvView &kv, const KvRows &rows, hipStream_t stream);

struct KvAttention {
    const void *q;
    int32_t dtype;
    int64_t q_token, q_head;
    void *out;
    int64_t out_token, out_head;
    float *lse;            // [Qt, heads] or NULL
    const int64_t *offsets;
    int64_t Qt;
    int32_t group;         // query heads per key/value head
    float scale;           // of the scores, times log2 e
    int32_t window, sinks;
    // the launch, from kv_attention_plan
    int32_t row_tiles, parts, part_tiles;
    int32_t max_rows;      // queries x group, as far as the host knows
    int32_t by_length;     // 1: workgroups are handed out by the requests' lengths
    float *part_out;       // [parts][Qt * heads][d], sums that are not divided yet
    float *part_stat;      // [parts][Qt * heads][2], largest score and sum
};
struct KvAttentionPlan {
    int32_t rows;          // query rows of a workgroup
    int32_t waves;         // of a workgroup
    int32_t by_length;
    int32_t max_rows;      // of a request and key/value head, as far as the host knows
    int32_t row_tiles;     // workgroups that share the row tiles of a request and key/value head and part
    int32_t parts, part_tiles;
};
constexpr int64_t KV_MAX_GROUPS = 1 << 23;                // workgroups of a launch: below 2^32 work-items
constexpr int64_t KV_MAX_PAIRS = KV_MAX_GROUPS - 8;       // of request and key/value head, whose places are made up to eights
// max_q: most queries of a request, 0 where that is not known
KvAttentionPlan kv_attention_plan(int64_t R, int32_t n_heads, int32_t group, int32_t d, int64_t Qt, int64_t max_q, int64_t max_len,
                                  int32_t window, int32_t sinks);
hipError_t launch_kv_attention(const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream);

struct KvPages {
    uint8_t *pages;
    int64_t page_bytes;
    int32_t n_pages, page_tokens, max_pages, R;
    int32_t *table, *lens, *refs;
};
constexpr int KV_COUNT_PAGES = 4096, KV_COUNT_REQUESTS = 256;   // of a workgroup that counts
size_t kv_pages_scratch_words(int64_t n_pages, int64_t R);
hipError_t launch_kv_reserve(const KvPages &kv, const int32_t *grow, int32_t *granted, int32_t *scratch, hipStream_t stream);
hipError_t launch_kv_fork(const KvPages &kv, const int32_t *src, const int32_t *dst, const int32_t *keep, int64_t n, hipStream_t stream);
hipError_t launch_kv_truncate(const KvPages &kv, const int32_t *new_lens, hipStream_t stream);
hipError_t launch_kv_copy_pages(const KvPages &kv, const int32_t *src, const int32_t *dst, int64_t n, hipStream_t stream);
hipError_t launch_kv_compact(const KvPages &kv, int32_t *table_out, int32_t *refs_out, int32_t *used, int32_t *scratch, hipStream_t stream);

struct DraftParams {
    const int32_t *draft_ids;
    const void *draft_probs, *target_probs;
    int64_t draft_stride, target_stride;   // elements from row to row
    int32_t dtype, V;
    const float *u, *u_next;
    const int64_t *offsets;
    int64_t Qt, R;
    int32_t *accepted, *next;
    unsigned long long *sums;   // [R][chunks]
    int64_t chunks;
};
constexpr int DRAFT_CHUNK = 1024;   // entries of a row that a wave sums up
__host__ __device__ inline int64_t draft_chunks(int32_t V) { return ((int64_t)V + DRAFT_CHUNK - 1) / DRAFT_CHUNK; }
hipError_t launch_verify_draft(const DraftParams &p, hipStream_t stream);

// the request that owns row t of `offsets` (non-decreasing, [R + 1]), asked by all lanes of a wave for the same t: -1 if there is none.
// 64 places are looked at at a time, so that 4096 requests are two trips to memory.
__device__ __forceinline__ int owner_of(const int64_t *offsets, int R, int64_t t)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = R + 1;   // the last place in [lo, lo + n) whose offset is <= t
    while (n > 0) {
        const int step = (n + 63) / 64;
        const int at = lo + lane * step;
        const bool below = lane * step < n && offsets[at] <= t;
        const uint64_t b = __ballot(below);
        const int c = __builtin_amdgcn_readfirstlane(b == 0 ? 0 : 64 - __builtin_clzll(b));
        if (c == 0) return -1;
        const int last = (c - 1) * step;
        if (step == 1) {
            lo += last;
            break;
        }
        n = n - last < step ? n - last : step;
        lo += last;
    }
    return lo < R ? lo : -1;
}

}  // namespace ralm
