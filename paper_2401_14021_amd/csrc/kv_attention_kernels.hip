// Attention over the 4-bit paged cache.
//
//   out[i, h] = sum_j softmax_j(scale q[i, h] . K[j, h / G]) V[j, h / G]     over the tokens j that query i sees
//
// A request's queries are its last tokens; a row is one query of one head, and the rows of a key/value head (queries x G) are taken
// together.  One pass over the tokens with a running maximum m and sum l per row: p = 2^(s - m), out = sum p V / l.
//
// What the layout of the cache is for: with S^T = K Q^T (16 tokens x 16 rows per v_mfma_f32_16x16x32_bf16) lane (g, n) = (lane / 16, lane % 16) feeds the
// g-th quarter of token n's key - one piece of memory, one or two powers - and gets the scores of row n for tokens 4 g .. 4 g + 3.  Two such
// tiles are the eight tokens of that lane in O^T = V^T P^T, where it feeds the n-th sixteenth of the head for the same eight tokens: two more
// pieces of memory.  So neither scores nor operands pass through LDS or from lane to lane; only the maximum is joined across the four
// lanes of a row, and only when it grows by more than 2^8 (p then stays below 2^8).
//
// 4-bit codes become bf16 in one instruction for two (v_cvt_scalef32_pk_bf16_fp4, which applies the power); bf16 holds them exactly and has
// fp32's range.  p is rounded to bf16 for its product with V (at most 2^-8 of it, as the rounding of a bf16 output); fp16
// queries, and p for them, are split into two bf16 numbers whose products are added: nothing of the query is lost and p keeps 16 bits.
// Scores, m, l and out are fp32.
//
// Masks: a step of 32 tokens that every row sees takes no test at all.  In the others a token that a row does not see gets the
// score -inf; its value counts with p = 0, so powers behind the last token (pages that were never written) and of tokens that hold NaN are
// set aside first (guard_values), as 0 * NaN would reach rows that do not see the token.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "kv_kernels.h"

namespace ralm {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr float MINUS_INF = -__builtin_inff();

__device__ __forceinline__ f32x4 mfma(const uint4 &a, const uint4 &b, const f32x4 &c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}
// codes 2 B, 2 B + 1 of a word as two bf16 numbers
template <int B>
__device__ __forceinline__ uint32_t two(uint32_t codes, float power)
{
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, power, B));
}
__device__ __forceinline__ uint32_t two_at(uint32_t codes, float power, int b)   // b: a constant behind unrolling
{
    return b == 0 ? two<0>(codes, power) : b == 1 ? two<1>(codes, power) : b == 2 ? two<2>(codes, power) : two<3>(codes, power);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)   // one instruction on gfx950
{
    bf16x2 v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ float low(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float high(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// what a lane holds of one tile
template <int D>
struct Piece {
    uint32_t k[D / 32], v[D / 32];
    uint32_t k_power, v_power;   // one or two bytes; a byte per token
};
template <int W>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[W])
{
    if constexpr (W == 2) {
        const uint2 x = *reinterpret_cast<const uint2 *>(p);
        w[0] = x.x, w[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < W / 4; ++i) {
            const uint4 x = *reinterpret_cast<const uint4 *>(p + 16 * i);
            w[4 * i] = x.x, w[4 * i + 1] = x.y, w[4 * i + 2] = x.z, w[4 * i + 3] = x.w;
        }
    }
}
template <int D>
__device__ __forceinline__ void load_piece(const uint8_t *tile, int g, int n, Piece<D> &x)
{
    load_words<D / 32>(tile + n * (D / 2) + g * (D / 8), x.k);
    load_words<D / 32>(tile + 8 * D + g * (2 * D) + n * (D / 8), x.v);
    const uint8_t *kp = tile + 16 * D + n * (D / 32);
    x.k_power = D == 64 ? kp[g >> 1] : D == 128 ? kp[g] : *reinterpret_cast<const uint16_t *>(kp + 2 * g);
    x.v_power = *reinterpret_cast<const uint32_t *>(tile + 16 * D + D / 2 + g * (D / 8) + n * D / 512 * 4);
}

// Which tiles the rows [row0, row1) of a request's key/value head see, as a list: the first `sinks` tiles, then those from `lo` on
struct Span {
    int sinks, lo, n;       // n: tiles of the list
    int part, parts;        // tiles of a part, number of parts
};
__device__ __forceinline__ int tiles_up_to(int last) { return last < 0 ? 0 : (last >> 4) + 1; }
__device__ __forceinline__ Span span_of(const KvAttention &a, int p_first, int p_last)
{
    Span s;
    const int from = a.window > 0 && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
    s.lo = from >> 4;
    const int first_tiles = tiles_up_to(a.sinks - 1);
    s.sinks = a.window > 0 ? (first_tiles < s.lo ? first_tiles : s.lo) : 0;
    const int n = s.sinks + tiles_up_to(p_last) - s.lo;
    s.n = n < 0 || p_last < 0 ? 0 : n;
    const int per = (s.n + a.parts - 1) / a.parts;
    s.part = a.part_tiles > per ? a.part_tiles : (per + 1) / 2 * 2;
    s.parts = s.n == 0 ? 1 : (s.n + s.part - 1) / s.part;
    return s;
}

struct Request {
    int64_t first;    // row of q and out
    int count, len;   // queries, tokens
};
__device__ __forceinline__ Request request_of(const KvView &kv, const KvAttention &a, int r)
{
    Request x;
    int64_t o0 = a.offsets[r], o1 = a.offsets[r + 1];
    o0 = o0 < 0 ? 0 : o0 > a.Qt ? a.Qt : o0;
    o1 = o1 < o0 ? o0 : o1 > a.Qt ? a.Qt : o1;
    x.first = o0;
    x.count = (int)(o1 - o0);
    const int64_t most = ((int64_t)kv.max_pages << kv.tile_shift) * KV_TILE;
    const int64_t len = kv.lens[r];
    x.len = (int)(len < 0 ? 0 : len > most ? most : len);
    return x;
}

// A workgroup's place: the row tiles of a key/value head are neighbours on one XCD (workgroup b runs on XCD b % 8), whose L2 then holds what
// they all read
struct Place {
    int r, h, rt, part;
};
__device__ __forceinline__ Place place_of(const KvView &kv, const KvAttention &a, int parts)
{
    const uint32_t pairs = (uint32_t)kv.R * kv.n_heads, per = (uint32_t)a.row_tiles * parts;
    const uint32_t b = blockIdx.x, xcd = b & 7u, i = b >> 3;
    Place x;
    const uint32_t pair = i / per * 8 + xcd, rest = i % per;
    x.r = pair < pairs ? (int)(pair / kv.n_heads) : -1;
    x.h = (int)(pair % kv.n_heads);
    x.part = (int)(rest / a.row_tiles);
    x.rt = a.row_tiles - 1 - (int)(rest % a.row_tiles);   // the last rows see the most tokens: first
    return x;
}

template <int D>
constexpr int lds_bytes(int nq, bool rows) { return rows ? 16 : 4 * 16 * (D + 4) * 4 + 2 * 4 * 16 * nq * 4; }

// ROWS: each of the four waves has NQ * 16 rows of its own and goes over all tokens of the part (many rows); else all waves have the same
// NQ * 16 rows and share out the part's tokens, 32 at a time (few rows).
template <int D, int NQ, bool HALF, bool ROWS>
__global__ __launch_bounds__(256) void kv_attention_kernel(KvView kv, KvAttention a)
{
    constexpr int KI = D / 32, NI = D / 16;   // multiplies per tile: scores, outputs
    constexpr int RW = NQ * 16;               // rows of a wave
    constexpr int RG = ROWS ? 4 * RW : RW;    // of the workgroup
    constexpr int STRIDE = ROWS ? 1 : 4;      // steps of a wave: every STRIDE-th
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const Place at = place_of(kv, a, a.parts);
    if (at.r < 0) return;
    const Request rq = request_of(kv, a, at.r);
    const int rows = rq.count * a.group;
    const int tile_mask = (1 << kv.tile_shift) - 1;
    const uint8_t *pool = kv.pages + kv.layer_bytes + at.h * kv.head_bytes;
    const int32_t *table = kv.table + (int64_t)at.r * kv.max_pages;

    for (int rt = at.rt; rt * RG < rows; rt += a.row_tiles) {
        const int row_a = rt * RG, row_b = (rows < row_a + RG ? rows : row_a + RG) - 1;   // the workgroup's first and last row
        const int p0 = rq.len - rq.count;                                                // place of the first query
        const Span sp = span_of(a, p0 + row_a / a.group, p0 + row_b / a.group);
        if (at.part >= sp.parts) continue;

        // this wave's rows
        const int w_a = ROWS ? row_a + wave * RW : row_a;
        const int w_b = row_b < w_a + RW - 1 ? row_b : w_a + RW - 1;
        const bool any_rows = w_a <= row_b;
        int pos[NQ];                // place of the row's query; -1: no row
        int64_t q_row[NQ];
        int q_head[NQ];
        uint4 qf[NQ][KI], ql[HALF ? NQ : 1][HALF ? KI : 1];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const int row = w_a + t * 16 + n;
            const bool real = row <= row_b;
            const int i = real ? row / a.group : 0;
            q_head[t] = at.h * a.group + (real ? row - i * a.group : 0);
            q_row[t] = rq.first + i;
            pos[t] = real ? p0 + i : -1;
            const uint16_t *q = static_cast<const uint16_t *>(a.q) + q_row[t] * a.q_token + q_head[t] * a.q_head + g * (D / 4);
#pragma unroll
            for (int j = 0; j < KI; ++j) {
                uint4 x = make_uint4(0, 0, 0, 0);
                if (real) x = *reinterpret_cast<const uint4 *>(q + 8 * j);
                if constexpr (HALF) {
                    const uint32_t u[4] = {x.x, x.y, x.z, x.w};
                    uint32_t hi[4], lo[4];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const float f0 = f16_bits_to_f32(u[c] & 0xffffu), f1 = f16_bits_to_f32(u[c] >> 16);
                        hi[c] = pack_bf16(f0, f1);
                        lo[c] = pack_bf16(f0 - low(hi[c]), f1 - high(hi[c]));
                    }
                    qf[t][j] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    ql[t][j] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                } else {
                    qf[t][j] = x;
                }
            }
        }
        const int see_first = any_rows ? p0 + w_a / a.group : 0, see_last = any_rows ? p0 + w_b / a.group : -1;   // places of the wave's rows

        f32x4 o[NQ][NI];
        float m[NQ], l[NQ];
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            m[t] = MINUS_INF;
            l[t] = 0.0f;
#pragma unroll
            for (int i = 0; i < NI; ++i) o[t][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }

        // the wave's tiles: [v0, v1) of the span's list
        const int v0 = at.part * sp.part;
        int v1 = v0 + sp.part < sp.n ? v0 + sp.part : sp.n;
        const int own = sp.sinks + tiles_up_to(see_last) - sp.lo;   // tiles that the wave's last row sees
        v1 = own < v1 ? own : v1;
        const int steps = v1 > v0 ? ((v1 - v0 + 1) / 2 + STRIDE - 1 - (ROWS ? 0 : wave)) / STRIDE : 0;
        const int step0 = ROWS ? 0 : wave;

        // The wave's next 32 steps, two tiles each, a lane per tile: where the tile lies, whether it is there, and whether all of the wave's
        // rows see all of it.  One look at the table for 1024 tokens, and two instructions per tile to have its address.
        int64_t tile_at = 0;
        uint64_t there = 0, plain = 0;
        auto tile_of = [&](int k, int u) {
            const int v = v0 + 2 * (step0 + k * STRIDE) + u;
            return v < sp.sinks ? v : v - sp.sinks + sp.lo;
        };
        auto look_up = [&](int k) {
            const int v = v0 + 2 * (step0 + (k + (lane >> 1)) * STRIDE) + (lane & 1);
            const int tile = v < sp.sinks ? v : v - sp.sinks + sp.lo;
            const int slot = tile >> kv.tile_shift;
            const int id = v < v1 && slot < kv.max_pages ? table[slot] : -1;
            const bool ok = id >= 0 && id < kv.n_pages;
            tile_at = (ok ? id : 0) * kv.page_bytes + (tile & tile_mask) * kv_tile_bytes(D);
            there = __ballot(ok);
            plain = __ballot(ok && tile * 16 + 15 <= see_first && (a.window == 0 || tile * 16 > see_last - a.window || tile * 16 + 15 < a.sinks));
        };
        auto load_step = [&](int k, Piece<D> (&x)[2]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int l = 2 * (k & 31) + u;
                const uint32_t lo = __builtin_amdgcn_readlane((int)tile_at, l), hi = __builtin_amdgcn_readlane((int)(tile_at >> 32), l);
                load_piece<D>(pool + ((uint64_t)hi << 32 | lo), g, n, x[u]);
            }
        };
        // what the loads of a step need to be told of it: whether its tiles are there, and plain (two bits each)
        auto flags_of = [&](int k) { return (uint32_t)(there >> (2 * (k & 31)) & 3u) | (uint32_t)(plain >> (2 * (k & 31)) & 3u) << 2; };

        auto step = [&](Piece<D> (&x)[2], uint32_t flags, int k) {
            // scores, not scaled yet
            f32x4 s[NQ][2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint4 kf[KI];
#pragma unroll
                for (int j = 0; j < KI; ++j) {
                    const float power = __uint_as_float((D == 256 ? (j >= KI / 2 ? x[u].k_power >> 8 : x[u].k_power & 255u) : x[u].k_power) << 23);
                    kf[j] = make_uint4(two<0>(x[u].k[j], power), two<1>(x[u].k[j], power), two<2>(x[u].k[j], power), two<3>(x[u].k[j], power));
                }
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    f32x4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int j = 0; j < KI; ++j) {
                        c = mfma(kf[j], qf[t][j], c);
                        if constexpr (HALF) c = mfma(kf[j], ql[t][j], c);
                    }
                    s[t][u] = c;
                }
            }

            uint64_t odd[2] = {0, 0};   // lanes of values that hold a block without a finite power
            if (flags != 15u) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bool page = flags >> u & 1u;
                    const int j0 = tile_of(k, u) * 16 + 4 * g;
#pragma unroll
                    for (int t = 0; t < NQ; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int j = j0 + i;
                            const bool sees = page && j <= pos[t] && (a.window == 0 || j > pos[t] - a.window || j < a.sinks);
                            s[t][u][i] = sees ? s[t][u][i] : MINUS_INF;
                        }
                    // values: powers of tokens behind the last one, and of blocks that are NaN, count as the smallest
                    uint32_t keep = 0;
                    bool nan = false;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t b = (x[u].v_power >> (8 * i)) & 255u;
                        const bool in = page && j0 + i <= see_last;
                        keep |= in && b < 254u ? b << (8 * i) : 0u;
                        nan = nan || (in && b >= 254u);
                    }
                    odd[u] = __ballot(nan);
                    if (!nan) x[u].v_power = keep;
                }
            }

            // running maximum, p, sum
            uint4 pf[NQ], pl[HALF ? NQ : 1];
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                float top = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])),
                                  fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
                if (__any(top * a.scale > m[t] + 8.0f)) {
                    top = fmaxf(top, __shfl_xor(top, 16, 64));
                    top = fmaxf(top, __shfl_xor(top, 32, 64));
                    const float grown = fmaxf(m[t], top * a.scale);
                    const float shrink = m[t] == MINUS_INF ? 0.0f : __builtin_amdgcn_exp2f(m[t] - grown);
                    m[t] = grown;
                    l[t] *= shrink;
#pragma unroll
                    for (int i = 0; i < NI; ++i) o[t][i] *= shrink;
                }
                const float ref = m[t] == MINUS_INF ? 0.0f : m[t];
                float p[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][0][i], a.scale, -ref));
                    p[4 + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][1][i], a.scale, -ref));
                }
                l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
                uint32_t hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) hi[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
                pf[t] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                if constexpr (HALF) {
                    uint32_t lo[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) lo[i] = pack_bf16(p[2 * i] - low(hi[i]), p[2 * i + 1] - high(hi[i]));
                    pl[t] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
            }

            if (__builtin_expect((odd[0] | odd[1]) != 0, 0)) {
                // Blocks that are NaN in a step that not all rows see: they reach the rows that see them and no others.  A lane of O^T holds
                // the sixteenths 4 g .. 4 g + 3 of row n, the power of which lies with lane (quad, sixteenth)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
#pragma unroll 1
                    for (int quad = 0; quad < 4; ++quad)
#pragma unroll 1
                        for (int i = 0; i < 4; ++i) {
                            const int j = tile_of(k, u) * 16 + 4 * quad + i;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint32_t w = (uint32_t)__shfl((int)x[u].v_power, quad * 16 + 4 * g + e, 64);
                                const bool bad = (flags >> u & 1u) && j <= see_last && ((w >> (8 * i)) & 255u) >= 254u;
#pragma unroll
                                for (int t = 0; t < NQ; ++t) {
                                    const bool sees = bad && j <= pos[t] && (a.window == 0 || j > pos[t] - a.window || j < a.sinks);
#pragma unroll
                                    for (int c = 0; c < NI; ++c)
                                        if (sees) o[t][c][e] = __builtin_nanf("");
                                }
                            }
                        }
                    uint32_t keep = 0;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t b = (x[u].v_power >> (8 * i)) & 255u;
                        keep |= b < 254u ? b << (8 * i) : 0u;
                    }
                    x[u].v_power = keep;
                }
            }

            // outputs: token i of the lane's eight is token i % 4 of tile i / 4
            float power[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int sh = 8 * (i & 3);
                const uint32_t vp = x[i >> 2].v_power;
                power[i] = __uint_as_float(sh == 24 ? vp >> 1 & 0x7f800000u : vp << (23 - sh) & 0x7f800000u);
            }
#pragma unroll
            for (int c = 0; c < NI / 2; ++c) {   // codes 2 c, 2 c + 1 of the lane's sixteenth
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int byte = (i & 3) * (D / 32) + c;
                    w[i] = two_at(x[i >> 2].v[byte >> 2], power[i], byte & 3);
                }
                uint4 even, second;
                even = make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u),
                                  __builtin_amdgcn_perm(w[5], w[4], 0x05040100u), __builtin_amdgcn_perm(w[7], w[6], 0x05040100u));
                second = make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u),
                                    __builtin_amdgcn_perm(w[5], w[4], 0x07060302u), __builtin_amdgcn_perm(w[7], w[6], 0x07060302u));
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    o[t][2 * c] = mfma(even, pf[t], o[t][2 * c]);
                    o[t][2 * c + 1] = mfma(second, pf[t], o[t][2 * c + 1]);
                    if constexpr (HALF) {
                        o[t][2 * c] = mfma(even, pl[t], o[t][2 * c]);
                        o[t][2 * c + 1] = mfma(second, pl[t], o[t][2 * c + 1]);
                    }
                }
            }
        };

        // two steps a turn, the loads of the next one under way during each: no register is moved
        Piece<D> xa[2], xb[2];
        if (steps > 0) {
            look_up(0);
            load_step(0, xa);
        }
        for (int k = 0; k < steps; k += 2) {
            const uint32_t fa = flags_of(k), fb = flags_of(k + 1);
            if (k + 1 < steps) load_step(k + 1, xb);
            step(xa, fa, k);
            if (((k + 2) & 31) == 0 && k + 2 < steps) look_up(k + 2);
            if (k + 2 < steps) load_step(k + 2, xa);
            if (k + 1 < steps) step(xb, fb, k + 1);
        }

        // sums over the four lanes of a row
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            l[t] += __shfl_xor(l[t], 16, 64);
            l[t] += __shfl_xor(l[t], 32, 64);
        }

        const bool whole = sp.parts == 1;
        const int64_t all_rows = a.Qt * kv.n_heads * a.group;
        // numbers [at, at + 4) of a row of the output
        auto put4 = [&](int64_t row, int head, int d, const float (&y)[4]) {
            if (whole) {
                uint2 z;
                if constexpr (HALF) z = make_uint2(f32_to_f16_bits(y[0]) | f32_to_f16_bits(y[1]) << 16, f32_to_f16_bits(y[2]) | f32_to_f16_bits(y[3]) << 16);
                else z = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
                *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * a.out_token + head * a.out_head + d) = z;
            } else {
                float *dst = a.part_out + ((at.part * all_rows) + row * (kv.n_heads * a.group) + head) * D + d;
                *reinterpret_cast<float4 *>(dst) = make_float4(y[0], y[1], y[2], y[3]);
            }
        };
        auto put_stat = [&](int64_t row, int head, float mm, float ll) {
            const int64_t i = row * (kv.n_heads * a.group) + head;
            if (whole) {
                if (a.lse) a.lse[i] = ll == 0.0f ? MINUS_INF : (mm + __builtin_amdgcn_logf(ll)) * 0.69314718055994531f;
            } else {
                a.part_stat[(at.part * all_rows + i) * 2] = mm;
                a.part_stat[(at.part * all_rows + i) * 2 + 1] = ll;
            }
        };
        if constexpr (ROWS) {
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                if (w_a + t * 16 + n > row_b) continue;
                const float f = whole ? (l[t] == 0.0f ? 0.0f : 1.0f / l[t]) : 1.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < NI; c += 4) {
                        const float y[4] = {o[t][c][e] * f, o[t][c + 1][e] * f, o[t][c + 2][e] * f, o[t][c + 3][e] * f};
                        put4(q_row[t], q_head[t], (4 * g + e) * NI + c, y);
                    }
                if (g == 0) put_stat(q_row[t], q_head[t], m[t], l[t]);
            }
        } else {
            // the four waves' sums meet in LDS, one tile of 16 rows at a time
            constexpr int LD = D + 4;
            float *so = reinterpret_cast<float *>(smem);                       // [4][16][LD]
            float *sm = so + 4 * 16 * LD, *sl = sm + 4 * RW;                   // [4][RW]
            __syncthreads();
            if (g == 0) {
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    sm[wave * RW + t * 16 + n] = m[t];
                    sl[wave * RW + t * 16 + n] = l[t];
                }
            }
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                if (row_a + t * 16 > row_b) break;
                __syncthreads();
                float big = MINUS_INF;
                for (int w = 0; w < 4; ++w) big = fmaxf(big, sm[w * RW + t * 16 + n]);
                const float f = m[t] == MINUS_INF ? 0.0f : __builtin_amdgcn_exp2f(m[t] - big);
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < NI; c += 4)
                        *reinterpret_cast<float4 *>(so + (wave * 16 + n) * LD + (4 * g + e) * NI + c) =
                            make_float4(o[t][c][e] * f, o[t][c + 1][e] * f, o[t][c + 2][e] * f, o[t][c + 3][e] * f);
                __syncthreads();
                // 16 threads per row
                const int row = threadIdx.x >> 4, i16 = threadIdx.x & 15;
                const int at_row = row_a + t * 16 + row;
                if (at_row <= row_b) {
                    float mm = MINUS_INF, ll = 0.0f;
                    for (int w = 0; w < 4; ++w) mm = fmaxf(mm, sm[w * RW + t * 16 + row]);
                    for (int w = 0; w < 4; ++w) {
                        const float mw = sm[w * RW + t * 16 + row];
                        ll += mw == MINUS_INF ? 0.0f : sl[w * RW + t * 16 + row] * __builtin_amdgcn_exp2f(mw - mm);
                    }
                    const float fin = whole ? (ll == 0.0f ? 0.0f : 1.0f / ll) : 1.0f;
                    const int i = at_row / a.group, head = at.h * a.group + at_row - i * a.group;
#pragma unroll
                    for (int c = 0; c < D; c += 64) {
                        float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                        for (int w = 0; w < 4; ++w) {
                            const float4 v = *reinterpret_cast<const float4 *>(so + (w * 16 + row) * LD + c + i16 * 4);
                            y[0] += v.x, y[1] += v.y, y[2] += v.z, y[3] += v.w;
                        }
                        for (int e = 0; e < 4; ++e) y[e] *= fin;
                        put4(rq.first + i, head, c + i16 * 4, y);
                    }
                    if (i16 == 0) put_stat(rq.first + i, head, mm, ll);
                }
            }
            __syncthreads();
        }
    }
}

// Joins the parts of rows that were split, a wave per row: lane p has part p's maximum and factor, and the sums are read D / 64 numbers a lane, eight
// parts under way at once.  Bound by those trips to memory: few rows have many parts.
constexpr int MAX_PARTS = 64;
template <int D, bool HALF>
__global__ __launch_bounds__(256) void kv_join_kernel(KvView kv, KvAttention a, int group_rows, int slices)
{
    const int lane = threadIdx.x & 63;
    const int slice = blockIdx.x % slices;                         // of the row tile's rows
    const uint32_t unit = blockIdx.x / slices;
    const int rt0 = (int)(unit % a.row_tiles), pair = (int)(unit / a.row_tiles);
    const int r = pair / kv.n_heads, h = pair % kv.n_heads;
    const Request rq = request_of(kv, a, r);
    const int rows = rq.count * a.group, heads = kv.n_heads * a.group;
    const int64_t all_rows = a.Qt * heads;
    for (int rt = rt0; rt * group_rows < rows; rt += a.row_tiles) {
        const int row_a = rt * group_rows, row_b = (rows < row_a + group_rows ? rows : row_a + group_rows) - 1;
        const int q0 = rq.len - rq.count;
        const Span sp = span_of(a, q0 + row_a / a.group, q0 + row_b / a.group);
        if (sp.parts == 1) continue;
        for (int row = row_a + slice * 4 + (int)(threadIdx.x >> 6); row <= row_b; row += slices * 4) {
            const int i = row / a.group, head = h * a.group + row - i * a.group;
            const int64_t x = (rq.first + i) * heads + head;
            const float2 stat = lane < sp.parts ? *reinterpret_cast<const float2 *>(a.part_stat + (lane * all_rows + x) * 2) : make_float2(MINUS_INF, 0.0f);
            float m = stat.x;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) m = fmaxf(m, __shfl_xor(m, s, 64));
            const float f = stat.x == MINUS_INF ? 0.0f : __builtin_amdgcn_exp2f(stat.x - m);   // 0: a part of which the row sees nothing
            float l = f * stat.y;
#pragma unroll
            for (int s = 1; s < 64; s <<= 1) l += __shfl_xor(l, s, 64);
            float y[D / 64] = {};
            const float *src = a.part_out + x * D + lane * (D / 64);
            for (int p0 = 0; p0 < sp.parts; p0 += 8) {
                float v[8][D / 64];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int64_t p = p0 + e < sp.parts ? p0 + e : sp.parts - 1;
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) v[e][c] = src[p * all_rows * D + c];
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float fp = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), (p0 + e) & 63));   // 0 behind the last part
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) y[c] += fp == 0.0f || p0 + e >= sp.parts ? 0.0f : fp * v[e][c];   // what a part of factor 0 holds may be anything
                }
            }
            const float over = l == 0.0f ? 0.0f : 1.0f / l;
            uint16_t *dst = static_cast<uint16_t *>(a.out) + (rq.first + i) * a.out_token + head * a.out_head + lane * (D / 64);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) dst[c] = HALF ? f32_to_f16_bits(y[c] * over) : pack_bf16(y[c] * over, 0.0f);
            if (lane == 0 && a.lse) a.lse[x] = l == 0.0f ? MINUS_INF : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
        }
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <int D, int NQ, bool HALF, bool ROWS>
hipError_t run(const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream)
{
    const int64_t groups = ceil_div((int64_t)kv.R * kv.n_heads, 8) * 8 * plan.row_tiles;
    const int lds = lds_bytes<D>(NQ, ROWS);
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&kv_attention_kernel<D, NQ, HALF, ROWS>),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    kv_attention_kernel<D, NQ, HALF, ROWS><<<(unsigned)(groups * plan.parts), 256, lds, stream>>>(kv, a);
    if (plan.parts > 1) {
        // four rows of a row tile per workgroup, if there are that many
        const int most = (int)ceil_div(plan.rows < a.max_rows ? plan.rows : a.max_rows, 4);
        kv_join_kernel<D, HALF><<<(unsigned)((int64_t)kv.R * kv.n_heads * plan.row_tiles * most), 256, 0, stream>>>(kv, a, plan.rows, most);
    }
    return hipGetLastError();
}
template <int D, bool HALF>
hipError_t run_form(const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream)
{
    if (plan.form == KV_FORM_TOKENS16) return run<D, 1, HALF, false>(kv, a, plan, stream);
    if constexpr (D < 256)
        if (plan.form == KV_FORM_TOKENS32) return run<D, 2, HALF, false>(kv, a, plan, stream);
    return run<D, D == 256 ? 1 : 2, HALF, true>(kv, a, plan, stream);
}

}  // namespace

KvAttentionPlan kv_attention_plan(int64_t R, int32_t n_heads, int32_t group, int32_t d, int64_t max_q, int64_t max_len, int32_t window,
                                  int32_t sinks)
{
    KvAttentionPlan p;
    const int64_t rows = (max_q < 1 ? 1 : max_q) * group;
    p.form = rows <= 16 ? KV_FORM_TOKENS16 : rows <= 32 && d < 256 ? KV_FORM_TOKENS32 : KV_FORM_ROWS;   // 32 rows of 256 numbers do not fit the registers
    p.rows = p.form == KV_FORM_TOKENS16 ? 16 : p.form == KV_FORM_TOKENS32 ? 32 : d == 256 ? 64 : 128;
    p.row_tiles = (int32_t)ceil_div(rows, p.rows);
    p.max_rows = (int32_t)(rows < 0x7fffffff ? rows : 0x7fffffff);
    // tokens that a row tile may see
    int64_t seen = max_len < 1 ? 1 : max_len;
    if (window > 0) {
        const int64_t most = (int64_t)window + sinks + (p.rows + group - 1) / group + 32;
        seen = most < seen ? most : seen;
    }
    const int64_t tiles = ceil_div(seen, KV_TILE);
    const int64_t groups = R * n_heads * p.row_tiles;
    // three workgroups for each of the 256 CUs, which is what their registers allow, if the parts do not get shorter than two steps of each wave
    const int64_t least = p.form == KV_FORM_ROWS ? 8 : 16;
    int64_t parts = ceil_div(768, groups);
    if (parts > ceil_div(tiles, least)) parts = ceil_div(tiles, least);
    if (parts > MAX_PARTS) parts = MAX_PARTS;
    p.part_tiles = (int32_t)(ceil_div(ceil_div(tiles, parts), 8) * 8);
    p.parts = (int32_t)ceil_div(tiles, p.part_tiles);
    return p;
}

hipError_t launch_kv_attention(const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream)
{
    const bool half = a.dtype == DT_F16;
    if (kv.d == 64) return half ? run_form<64, true>(kv, a, plan, stream) : run_form<64, false>(kv, a, plan, stream);
    if (kv.d == 128) return half ? run_form<128, true>(kv, a, plan, stream) : run_form<128, false>(kv, a, plan, stream);
    return half ? run_form<256, true>(kv, a, plan, stream) : run_form<256, false>(kv, a, plan, stream);
}

}  // namespace ralm
