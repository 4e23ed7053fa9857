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
// fp32's range.  p is rounded to bf16 for its product with V (at most 2^-8 of it, as the rounding of a bf16 output: 0.0023 of the outputs' size from 64 bits
// where the output's rounding alone is 0.0017); with 16 bits of p chunks of prompts took 18 % more, windows 14 %, single tokens 2 to 5 %.  fp16
// queries, and p for them, are split into two bf16 numbers whose products are added: nothing of the query is lost and p keeps 16 bits.
// Scores, m, l and out are fp32.
//
// Masks: a step of 32 tokens that every row sees takes no test at all.  In the others a token that a row does not see gets the
// score -inf; its value counts with p = 0, so powers behind the last token (pages that were never written) and of tokens that hold NaN are
// set aside first (guard_values), as 0 * NaN would reach rows that do not see the token.
//
// What bounds it (counters): vector instructions and multiplies, which overlap only in part on a SIMD (a wave of each side by side takes 355 us where alone they take
// 248 and 245).  A step of 16 rows (bf16, 128 numbers) is 290 instructions: 200 vector ones, 96 of which make operands of codes and 16 are multiplies, 8 loads, the rest scalar.
// Six contexts of 115000 tokens, 8 x 4 heads of 128: 141 us, 5.5 TB/s of cache, vector instructions issue in 54 % of the cycles, the multiplies are busy in 16 %; a
// single token's other limit is the chain offsets -> pages -> codes -> sums (8 us for 640 tokens).  Prompt chunks: 395 us for 274 GFLOP, 690 TFLOP/s; 74 % and 31 %.
// Tried there and slower: operands converted once per workgroup and passed on through LDS (442 us: a fifth fewer instructions, but the waves wait for each other
// and for LDS), 48 or 64 rows a wave with the queries in LDS (476 to 490 us), one set of registers for a step's codes to have four waves a
// SIMD (156 instead of 141 us for the long contexts), loads two and three steps ahead (162 to 165).  fp4 codes as operands of the block-scaled multiply, with the
// query as two fp8 numbers, need no conversion of the keys, but its sums were found to be good to 1e-4 of the products' magnitude only.
#include <atomic>

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
__device__ __forceinline__ void load_keys(const uint8_t *tile, int g, int n, Piece<D> &x)
{
    load_words<D / 32>(tile + n * (D / 2) + g * (D / 8), x.k);
    const uint8_t *kp = tile + 16 * D + n * (D / 32);
    x.k_power = D == 64 ? kp[g >> 1] : D == 128 ? kp[g] : *reinterpret_cast<const uint16_t *>(kp + 2 * g);
}
template <int D>
__device__ __forceinline__ void load_values(const uint8_t *tile, int g, int n, Piece<D> &x)
{
    load_words<D / 32>(tile + 8 * D + g * (2 * D) + n * (D / 8), x.v);
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
    s.part = a.part_tiles > per ? a.part_tiles : (per + 3) / 4 * 4;
    s.parts = s.n == 0 ? 1 : (s.n + s.part - 1) / s.part;
    return s;
}

// the v-th tile of a span's list
__device__ __forceinline__ int listed_tile(const Span &s, int v) { return v < s.sinks ? v : v - s.sinks + s.lo; }

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

// The request that is the rank-th longest (equal ones in their order), R <= 64, by all lanes of every wave; lds: 64 words, in which the waves write the same,
// and each reads what its own lanes wrote: they are in step, and the fences keep the compiler from moving a read in front of the writes.
// 64 comparisons of what 16 reads bring: with a read of a lane's register per request this took 2.5 us of a call.
__device__ __forceinline__ int longest_request(const KvView &kv, int rank, uint32_t *lds)
{
    const uint32_t lane = threadIdx.x & 63;
    const int32_t len = (int)lane < kv.R ? kv.lens[lane] : 0;
    // no two alike; lanes without a request come last.  Beyond 2^25 tokens lengths count as equal
    const uint32_t key = (uint32_t)(len < 0 ? 0 : len > 1 << 25 ? 1 << 25 : len) * 64u + (63u - lane);
    lds[lane] = key;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    uint32_t before = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const uint4 k = reinterpret_cast<const uint4 *>(lds)[j];
        before += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
    }
    return __builtin_ctzll(__ballot(before == (uint32_t)rank));
}

// A workgroup's place: the row tiles of a key/value head are neighbours on one XCD (workgroup b runs on XCD b % 8), whose L2 then holds what
// they all read
struct Place {
    int r, h, rt, part;
};
__device__ __forceinline__ Place place_of(const KvView &kv, const KvAttention &a, int parts, uint32_t *lds)
{
    const uint32_t pairs = (uint32_t)kv.R * kv.n_heads, per = (uint32_t)a.row_tiles * parts;
    const uint32_t b = blockIdx.x, xcd = b & 7u, i = b >> 3;
    Place x;
    uint32_t pair = i / per * 8 + xcd;
    const uint32_t rest = i % per;
    x.part = (int)(rest / a.row_tiles);
    x.rt = a.row_tiles - 1 - (int)(rest % a.row_tiles);   // the last rows see the most tokens: first
    if (pair >= pairs) {
        x.r = -1;
        x.h = 0;
        return x;
    }
    if (a.by_length) {
        // A few workgroups per CU that start at once: 32 CUs of an XCD get the longest 32 in order, the next 32 in reverse, and so on, so that every CU
        // has about as many tokens
        const uint32_t n = (pairs - xcd + 7) / 8, round = i / 32 * 32, last = round + 32 < n ? round + 32 : n;
        if (a.by_length == 1 && (i & 32u)) pair = (last - 1 - (i - round)) * 8 + xcd;   // 2: many rounds of workgroups, the longest first
        x.r = longest_request(kv, (int)(pair / kv.n_heads), lds);
    } else {
        x.r = (int)(pair / kv.n_heads);
    }
    x.h = (int)(pair % kv.n_heads);
    return x;
}

// NQ * 16 rows of a key/value head that a wave works on
template <int D, int NQ, bool HALF>
struct Block {
    static constexpr int KI = D / 32, NI = D / 16;   // multiplies per tile: scores, outputs
    int pos[NQ];             // place of the row's query; -1: no row
    uint4 qf[NQ][KI], ql[HALF ? NQ : 1][HALF ? KI : 1];
    f32x4 o[NQ][NI];
    float m[NQ], l[NQ];
    int see_first, see_last;   // places of the first and last row's query; -1: no rows

    // rows row_a .. row_b (at most) of request rq
    __device__ __forceinline__ void begin(const KvAttention &a, const Request &rq, int h, int row_a, int row_b)
    {
        const int lane = threadIdx.x & 63, g = lane >> 4, n = lane & 15;
        const int p0 = rq.len - rq.count;
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            const int row = row_a + t * 16 + n;
            const bool real = row <= row_b;
            const int i = real ? row / a.group : 0, head = h * a.group + (real ? row - i * a.group : 0);
            pos[t] = real ? p0 + i : -1;
            const uint16_t *q = static_cast<const uint16_t *>(a.q) + (rq.first + i) * a.q_token + head * a.q_head + g * (D / 4);
#pragma unroll
            for (int j = 0; j < KI; ++j) {
                uint4 x = make_uint4(0, 0, 0, 0), y = x;
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
                    x = make_uint4(hi[0], hi[1], hi[2], hi[3]);
                    y = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                }
                qf[t][j] = x;
                if constexpr (HALF) ql[t][j] = y;
            }
            m[t] = MINUS_INF;
            l[t] = 0.0f;
#pragma unroll
            for (int i2 = 0; i2 < NI; ++i2) o[t][i2] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
        const int last = row_b < row_a + NQ * 16 - 1 ? row_b : row_a + NQ * 16 - 1;
        see_first = row_a <= row_b ? p0 + row_a / a.group : 0;
        see_last = row_a <= row_b ? p0 + last / a.group : -1;
    }
    __device__ __forceinline__ bool sees(const KvAttention &a, int t, int j) const
    {
        return j <= pos[t] && (a.window == 0 || j > pos[t] - a.window || j < a.sinks);
    }
    // whether all rows see all of a tile
    __device__ __forceinline__ bool all_see(const KvAttention &a, int tile) const
    {
        return tile * 16 + 15 <= see_first && (a.window == 0 || tile * 16 > see_last - a.window || tile * 16 + 15 < a.sinks);
    }
    __device__ __forceinline__ void mask(const KvAttention &a, f32x4 (&s)[2], int t, int u, bool page, int j0) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) s[u][i] = page && sees(a, t, j0 + i) ? s[u][i] : MINUS_INF;
    }
    // running maximum, p, sum: the weights of the lane's eight tokens for its row of block t
    __device__ __forceinline__ void weigh(const KvAttention &a, int t, const f32x4 (&s)[2], uint4 &pf, uint4 &pl)
    {
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
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
            p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[0][i], a.scale, -ref));
            p[4 + i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[1][i], a.scale, -ref));
        }
        l[t] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
        uint32_t hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) hi[i] = pack_bf16(p[2 * i], p[2 * i + 1]);
        pf = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if constexpr (HALF) {
            uint32_t lo[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) lo[i] = pack_bf16(p[2 * i] - low(hi[i]), p[2 * i + 1] - high(hi[i]));
            pl = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
    }
    // Values of a tile (first token j0, powers v_power by lane) whose power is not finite: NaN for the rows that see them and no others.  A lane of O^T
    // holds the sixteenths 4 g .. 4 g + 3 of row n, the power of which lies with lane (quad, sixteenth)
    __device__ __forceinline__ void spoil(const KvAttention &a, uint32_t v_power, bool page, int j0)
    {
        const int g = (threadIdx.x & 63) >> 4;
#pragma unroll 1
        for (int quad = 0; quad < 4; ++quad)
#pragma unroll 1
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t w = (uint32_t)__shfl((int)v_power, quad * 16 + 4 * g + e, 64);
                    const bool bad = page && ((w >> (8 * i)) & 255u) >= 254u;
#pragma unroll
                    for (int t = 0; t < NQ; ++t)
#pragma unroll
                        for (int c = 0; c < NI; ++c)
                            if (bad && sees(a, t, j0 + 4 * quad + i)) o[t][c][e] = __builtin_nanf("");
                }
    }
    // sums over the four lanes of a row
    __device__ __forceinline__ void end()
    {
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            l[t] += __shfl_xor(l[t], 16, 64);
            l[t] += __shfl_xor(l[t], 32, 64);
        }
    }
};

// what values' powers count as: those of tokens behind j_last, and those that are not finite, as the smallest.  bad: whether there were any of
// the latter
__device__ __forceinline__ uint32_t guard_values(uint32_t v_power, bool page, int j0, int j_last, bool &bad)
{
    uint32_t keep = 0;
    bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t b = (v_power >> (8 * i)) & 255u;
        const bool in = page && j0 + i <= j_last;
        keep |= in && b < 254u ? b << (8 * i) : 0u;
        bad = bad || (in && b >= 254u);
    }
    return keep;
}
// the four powers of a word as fp32
__device__ __forceinline__ void powers(uint32_t v_power, float *p)
{
    p[0] = __uint_as_float(v_power << 23);
    p[1] = __uint_as_float(v_power << 15 & 0x7f800000u);
    p[2] = __uint_as_float(v_power << 7 & 0x7f800000u);
    p[3] = __uint_as_float(v_power >> 1 & 0x7f800000u);
}
template <int D>
__device__ __forceinline__ float k_power_of(uint32_t k_power, int j)
{
    return __uint_as_float((D == 256 ? (j >= D / 64 ? k_power >> 8 : k_power & 255u) : k_power) << 23);
}
// operand of the j-th multiply of a tile's scores
__device__ __forceinline__ uint4 k_operand(uint32_t codes, float power) { return make_uint4(two<0>(codes, power), two<1>(codes, power), two<2>(codes, power), two<3>(codes, power)); }
// operands of the multiplies for codes 2 c and 2 c + 1 of the lane's sixteenth: token i of the lane's eight is token i % 4 of tile i / 4
template <int D>
__device__ __forceinline__ void v_operands(const uint32_t (&va)[D / 32], const uint32_t (&vb)[D / 32], const float (&power)[8], int c, uint4 &even, uint4 &odd)
{
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int byte = (i & 3) * (D / 32) + c;
        w[i] = two_at(i < 4 ? va[byte >> 2] : vb[byte >> 2], power[i], byte & 3);
    }
    even = make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x05040100u), __builtin_amdgcn_perm(w[3], w[2], 0x05040100u),
                      __builtin_amdgcn_perm(w[5], w[4], 0x05040100u), __builtin_amdgcn_perm(w[7], w[6], 0x05040100u));
    odd = make_uint4(__builtin_amdgcn_perm(w[1], w[0], 0x07060302u), __builtin_amdgcn_perm(w[3], w[2], 0x07060302u),
                     __builtin_amdgcn_perm(w[5], w[4], 0x07060302u), __builtin_amdgcn_perm(w[7], w[6], 0x07060302u));
}

// results of a row: to the output where nothing was split, else to the part's place
template <int D, bool HALF>
struct Sink {
    const KvAttention &a;
    int heads, part;
    bool whole;
    int64_t all_rows;
    __device__ __forceinline__ Sink(const KvView &kv, const KvAttention &a_, int part_, bool whole_)
        : a(a_), heads(kv.n_heads * a_.group), part(part_), whole(whole_), all_rows(a_.Qt * kv.n_heads * a_.group) {}
    // numbers d .. d + 3 of a row
    __device__ __forceinline__ void put4(int64_t row, int head, int d, float y0, float y1, float y2, float y3) const
    {
        if (whole) {
            uint2 z;
            if constexpr (HALF) z = make_uint2(f32_to_f16_bits(y0) | f32_to_f16_bits(y1) << 16, f32_to_f16_bits(y2) | f32_to_f16_bits(y3) << 16);
            else z = make_uint2(pack_bf16(y0, y1), pack_bf16(y2, y3));
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + row * a.out_token + head * a.out_head + d) = z;
        } else {
            *reinterpret_cast<float4 *>(a.part_out + (part * all_rows + row * heads + head) * D + d) = make_float4(y0, y1, y2, y3);
        }
    }
    __device__ __forceinline__ void put_stat(int64_t row, int head, float m, float l) const
    {
        const int64_t i = row * heads + head;
        if (whole) {
            if (a.lse) a.lse[i] = l == 0.0f ? MINUS_INF : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994531f;
        } else {
            *reinterpret_cast<float2 *>(a.part_stat + (part * all_rows + i) * 2) = make_float2(m, l);
        }
    }
};

// ROWS: each of a workgroup's waves has NQ * 16 rows of its own and goes over all tokens of the part (many rows; the waves never wait for each
// other).  Else all have the same NQ * 16 rows and share out the part's tokens, 32 at a time, and their sums meet in LDS (few rows).  Four waves, or eight
// where there is at most a workgroup for every CU.
template <int D, int NQ, bool ROWS, int WAVES>
constexpr int lds_bytes() { return ROWS ? 256 : WAVES * 16 * (D + 4) * 4 + 2 * WAVES * 16 * NQ * 4; }

template <int D, int NQ, bool HALF, bool ROWS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void kv_attention_kernel(KvView kv, KvAttention a)
{
    using B = Block<D, NQ, HALF>;
    constexpr int KI = B::KI, NI = B::NI, RW = NQ * 16, RG = ROWS ? WAVES * RW : RW;   // rows of a wave, of the workgroup
    constexpr int STRIDE = ROWS ? 1 : WAVES;                                              // a wave's steps are every STRIDE-th
    extern __shared__ __align__(16) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const Place at = place_of(kv, a, a.parts, reinterpret_cast<uint32_t *>(smem));
    if (at.r < 0) return;
    const Request rq = request_of(kv, a, at.r);
    const int rows = rq.count * a.group;
    const int tile_mask = (1 << kv.tile_shift) - 1;
    const uint8_t *pool = kv.pages + kv.layer_bytes + at.h * kv.head_bytes;
    const int32_t *table = kv.table + (int64_t)at.r * kv.max_pages;

    for (int rt = at.rt; rt * RG < rows; rt += a.row_tiles) {
        const int row_a = rt * RG, row_b = (rows < row_a + RG ? rows : row_a + RG) - 1;
        const int q0 = rq.len - rq.count;   // place of the first query
        const Span sp = span_of(a, q0 + row_a / a.group, q0 + row_b / a.group);
        if (at.part >= sp.parts) continue;
        B b;
        b.begin(a, rq, at.h, ROWS ? row_a + wave * RW : row_a, row_b);

        // this wave's tiles: of the part's, [v0, v1) of the span's list, those that its last row sees; its steps are pairs of them
        const int own = sp.sinks + tiles_up_to(b.see_last) - sp.lo;
        const int v0 = at.part * sp.part, end = v0 + sp.part < sp.n ? v0 + sp.part : sp.n, v1 = own < end ? own : end;
        const int step0 = ROWS ? 0 : wave;
        const int steps = v1 > v0 ? ((v1 - v0 + 1) / 2 + STRIDE - 1 - step0) / STRIDE : 0;

        // The wave's next 32 steps, two tiles each, a lane per tile: where the tile lies, whether it is there, and whether all rows see all of
        // it.  One look at the table for 1024 tokens, and two instructions per tile to have its address.
        int64_t tile_at = 0;
        uint64_t there = 0, plain = 0;
        auto tile_of = [&](int k, int u) { return listed_tile(sp, v0 + 2 * (step0 + k * STRIDE) + u); };
        auto look_up = [&](int k) {
            const int v = v0 + 2 * (step0 + (k + (lane >> 1)) * STRIDE) + (lane & 1);
            const int tile = listed_tile(sp, v);
            const int slot = tile >> kv.tile_shift;
            const int id = v < v1 && slot < kv.max_pages ? table[slot] : -1;
            const bool ok = id >= 0 && id < kv.n_pages;
            tile_at = (ok ? id : 0) * kv.page_bytes + (tile & tile_mask) * kv_tile_bytes(D);
            there = __ballot(ok);
            plain = __ballot(ok && b.all_see(a, tile));
        };
        auto tile_ptr = [&](int k, int u) {
            const int l = 2 * (k & 31) + u;
            const uint32_t lo = __builtin_amdgcn_readlane((int)tile_at, l), hi = __builtin_amdgcn_readlane((int)(tile_at >> 32), l);
            return pool + ((uint64_t)hi << 32 | lo);
        };
        auto load_step = [&](int k, Piece<D> (&x)[2]) {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint8_t *tile = tile_ptr(k, u);
                load_keys<D>(tile, g, n, x[u]);
                load_values<D>(tile, g, n, x[u]);
            }
        };
        // of a step: whether its tiles are there, and plain (two bits each)
        auto flags_of = [&](int k) { return (uint32_t)(there >> (2 * (k & 31)) & 3u) | (uint32_t)(plain >> (2 * (k & 31)) & 3u) << 2; };

        auto step = [&](Piece<D> (&x)[2], uint32_t flags, int k) {
            uint4 kf[2][KI];
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int j = 0; j < KI; ++j) kf[u][j] = k_operand(x[u].k[j], k_power_of<D>(x[u].k_power, j));
            uint4 pf[NQ], pl[HALF ? NQ : 1];
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                f32x4 s[2] = {f32x4{0.0f, 0.0f, 0.0f, 0.0f}, f32x4{0.0f, 0.0f, 0.0f, 0.0f}};   // scores, not scaled yet
#pragma unroll
                for (int j = 0; j < KI; ++j) {
                    s[0] = mfma(kf[0][j], b.qf[t][j], s[0]);
                    s[1] = mfma(kf[1][j], b.qf[t][j], s[1]);
                    if constexpr (HALF) {
                        s[0] = mfma(kf[0][j], b.ql[t][j], s[0]);
                        s[1] = mfma(kf[1][j], b.ql[t][j], s[1]);
                    }
                }
                if (flags != 15u) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) b.mask(a, s, t, u, flags >> u & 1u, tile_of(k, u) * 16 + 4 * g);
                }
                b.weigh(a, t, s, pf[t], pl[HALF ? t : 0]);
            }
            uint64_t bad[2] = {0, 0};   // lanes of values that hold a block without a finite power
            uint32_t raw[2] = {0, 0};
            if (flags != 15u) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    bool nan;
                    raw[u] = x[u].v_power;
                    x[u].v_power = guard_values(x[u].v_power, flags >> u & 1u, tile_of(k, u) * 16 + 4 * g, b.see_last, nan);
                    bad[u] = __ballot(nan);
                }
            }
            if (__builtin_expect((bad[0] | bad[1]) != 0, 0)) {
#pragma unroll
                for (int u = 0; u < 2; ++u) b.spoil(a, raw[u], flags >> u & 1u, tile_of(k, u) * 16);
            }
            float power[8];
            powers(x[0].v_power, power);
            powers(x[1].v_power, power + 4);
#pragma unroll
            for (int c = 0; c < NI / 2; ++c) {
                uint4 even, odd;
                v_operands<D>(x[0].v, x[1].v, power, c, even, odd);
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    b.o[t][2 * c] = mfma(even, pf[t], b.o[t][2 * c]);
                    b.o[t][2 * c + 1] = mfma(odd, pf[t], b.o[t][2 * c + 1]);
                    if constexpr (HALF) {
                        b.o[t][2 * c] = mfma(even, pl[t], b.o[t][2 * c]);
                        b.o[t][2 * c + 1] = mfma(odd, pl[t], b.o[t][2 * c + 1]);
                    }
                }
            }
        };

        // Two steps a turn with registers of their own, so that none is moved; the loads of the step behind a step are under way during it.  More of them
        // gain nothing: a wave that is alone on its SIMD takes 0.63 us a step, which are its 290 instructions in a row, about 5 cycles each.
        Piece<D> xa[2], xb[2];
        uint32_t fa = 0, fb = 0;
        auto request = [&](int k, Piece<D> (&to)[2], uint32_t &f) {
            if (k >= steps) return;
            if ((k & 31) == 0) look_up(k);
            f = flags_of(k);
            load_step(k, to);
        };
        request(0, xa, fa);
        for (int k = 0; k < steps; k += 2) {
            request(k + 1, xb, fb);
            step(xa, fa, k);
            request(k + 2, xa, fa);
            if (k + 1 < steps) step(xb, fb, k + 1);
        }
        b.end();

        const Sink<D, HALF> sink(kv, a, at.part, sp.parts == 1);
        if constexpr (ROWS) {
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                const int row = row_a + wave * RW + t * 16 + n;
                if (row > row_b) continue;
                const int i = row / a.group, head = at.h * a.group + row - i * a.group;
                const float f = sink.whole ? (b.l[t] == 0.0f ? 0.0f : 1.0f / b.l[t]) : 1.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int c = 0; c < NI; c += 4)
                        sink.put4(rq.first + i, head, (4 * g + e) * NI + c, b.o[t][c][e] * f, b.o[t][c + 1][e] * f, b.o[t][c + 2][e] * f, b.o[t][c + 3][e] * f);
                if (g == 0) sink.put_stat(rq.first + i, head, b.m[t], b.l[t]);
            }
            continue;
        }
        // the waves' sums meet in LDS, one tile of 16 rows at a time
        constexpr int LD = D + 4, TPR = WAVES * 4;                         // threads per row
        float *so = reinterpret_cast<float *>(smem);                       // [WAVES][16][LD]
        float *sm = so + WAVES * 16 * LD, *sl = sm + WAVES * RW;           // [WAVES][RW]
        __syncthreads();
        if (g == 0) {
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                sm[wave * RW + t * 16 + n] = b.m[t];
                sl[wave * RW + t * 16 + n] = b.l[t];
            }
        }
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            if (row_a + t * 16 > row_b) break;
            __syncthreads();
            float big = MINUS_INF;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) big = fmaxf(big, sm[w * RW + t * 16 + n]);
            const float f = b.m[t] == MINUS_INF ? 0.0f : __builtin_amdgcn_exp2f(b.m[t] - big);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int c = 0; c < NI; c += 4)
                    *reinterpret_cast<float4 *>(so + (wave * 16 + n) * LD + (4 * g + e) * NI + c) =
                        make_float4(b.o[t][c][e] * f, b.o[t][c + 1][e] * f, b.o[t][c + 2][e] * f, b.o[t][c + 3][e] * f);
            __syncthreads();
            const int row = threadIdx.x / TPR, i0 = threadIdx.x % TPR;
            const int at_row = row_a + t * 16 + row;
            if (at_row <= row_b) {
                float mm = MINUS_INF, ll = 0.0f;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) mm = fmaxf(mm, sm[w * RW + t * 16 + row]);
#pragma unroll
                for (int w = 0; w < WAVES; ++w) {
                    const float mw = sm[w * RW + t * 16 + row];
                    const float lw = sl[w * RW + t * 16 + row];
                    // a wave without a maximum saw nothing (its sum is 0) or keys that are all NaN (its sum is)
                    ll += mw == MINUS_INF ? lw : lw * __builtin_amdgcn_exp2f(mw - mm);
                }
                const float fin = sink.whole ? (ll == 0.0f ? 0.0f : 1.0f / ll) : 1.0f;
                const int i = at_row / a.group, head = at.h * a.group + at_row - i * a.group;
#pragma unroll
                for (int c0 = 0; c0 < D; c0 += 4 * TPR) {
                    const int c = c0 + i0 * 4;
                    if (4 * TPR > D && c >= D) continue;
                    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int w = 0; w < WAVES; ++w) {
                        const float4 v = *reinterpret_cast<const float4 *>(so + (w * 16 + row) * LD + c);
                        y[0] += v.x, y[1] += v.y, y[2] += v.z, y[3] += v.w;
                    }
                    sink.put4(rq.first + i, head, c, y[0] * fin, y[1] * fin, y[2] * fin, y[3] * fin);
                }
                if (i0 == 0) sink.put_stat(rq.first + i, head, mm, ll);
            }
        }
        __syncthreads();
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
            const float f = stat.x == MINUS_INF ? 0.0f : __builtin_amdgcn_exp2f(stat.x - m);
            float l = stat.x == MINUS_INF ? stat.y : f * stat.y;   // without a maximum: 0, or NaN
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
                    const float fp = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), (p0 + e) & 63));
                    // every part has written its sums, zeros for rows that see none of it: NaN values come through a factor of 0
#pragma unroll
                    for (int c = 0; c < D / 64; ++c) y[c] += p0 + e >= sp.parts ? 0.0f : fp * v[e][c];
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

template <auto KERNEL>
hipError_t run(int waves, int lds, const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream)
{
    const int64_t groups = ceil_div((int64_t)kv.R * kv.n_heads, 8) * 8 * plan.row_tiles * plan.parts;
    static std::atomic<bool> attr_done{false};   // per kernel; setting it twice is harmless
    if (lds > 65536 && !attr_done.load(std::memory_order_acquire)) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
        attr_done.store(true, std::memory_order_release);
    }
    KERNEL<<<(unsigned)groups, 64 * waves, lds, stream>>>(kv, a);
    return hipGetLastError();
}
template <int D, bool HALF>
hipError_t run_form(const KvView &kv, const KvAttention &a, const KvAttentionPlan &plan, hipStream_t stream)
{
    constexpr int N = D == 256 ? 1 : 2;   // 32 rows a wave: not with 256 numbers a head, whose operands and sums do not fit the registers
    auto finish = [&](hipError_t e) {
        if (e != hipSuccess || plan.parts == 1) return e;
        // four rows of a row tile per workgroup, if there are that many
        const int most = (int)ceil_div(plan.rows < a.max_rows ? plan.rows : a.max_rows, 4);
        kv_join_kernel<D, HALF><<<(unsigned)((int64_t)kv.R * kv.n_heads * plan.row_tiles * most), 256, 0, stream>>>(kv, a, plan.rows, most);
        return hipGetLastError();
    };
    constexpr bool EIGHT1 = D <= 128, EIGHT2 = D == 64 || (D == 128 && !HALF);   // eight waves: half the registers a wave
    if (plan.rows == 64 * N) return finish(run<kv_attention_kernel<D, N, HALF, true, 4>>(4, lds_bytes<D, N, true, 4>(), kv, a, plan, stream));
    if (plan.waves == 8) {
        if constexpr (EIGHT1)
            if (plan.rows == 16) return finish(run<kv_attention_kernel<D, 1, HALF, false, 8>>(8, lds_bytes<D, 1, false, 8>(), kv, a, plan, stream));
        if constexpr (EIGHT2)
            if (plan.rows == 32) return finish(run<kv_attention_kernel<D, 2, HALF, false, 8>>(8, lds_bytes<D, 2, false, 8>(), kv, a, plan, stream));
    }
    if (plan.rows == 16) return finish(run<kv_attention_kernel<D, 1, HALF, false, 4>>(4, lds_bytes<D, 1, false, 4>(), kv, a, plan, stream));
    return finish(run<kv_attention_kernel<D, N, HALF, false, 4>>(4, lds_bytes<D, N, false, 4>(), kv, a, plan, stream));
}

}  // namespace

KvAttentionPlan kv_attention_plan(int64_t R, int32_t n_heads, int32_t group, int32_t d, int64_t Qt, int64_t max_q, int64_t max_len,
                                  int32_t window, int32_t sinks)
{
    KvAttentionPlan p;
    // Where the most queries of a request are not known, the form is that for their mean: 64 single tokens over 200 to 4000 (8 x 4 heads x 128) take 44 us so,
    // 32 with the hint and 127 in the form for one request that has them all; one chunk of 512 among them 166, 295 and 221.
    const int64_t mean_q = max_q > 0 ? max_q : ceil_div(Qt, R);
    const int64_t rows = (mean_q < 1 ? 1 : mean_q) * group;
    // Waves with rows of their own where that gives two workgroups per CU whose waves have nearly all of their rows; else waves that share out the tokens of
    // 32 rows.  us in a graph, shared out and of their own: 8 chunks of 700 to 1500 tokens 492, 415; 32 requests, 8 x 8 heads x 128, 2000 tokens, 32 of
    // them new 111, 105; 24 new 91, 103; 16 new 66, 74; 8 x 8 x 4 heads, 3000 tokens, 256 new 148, 141; 128 new 80, 100; one of 512 new 29, 54.
    const int32_t wave_rows = rows <= 16 || d == 256 ? 16 : 32;
    const int64_t four = ceil_div(rows, 4 * wave_rows);
    const bool many = R * n_heads * four >= 512 && rows * 10 >= four * 4 * wave_rows * 9;
    p.rows = many ? 4 * wave_rows : wave_rows;
    const int64_t row_tiles = ceil_div(rows, p.rows), max_rows = max_q > 0 ? rows : (Qt < 1 ? 1 : Qt) * group;
    p.max_rows = (int32_t)(max_rows < 0x7fffffff ? max_rows : 0x7fffffff);
    // tokens that a row tile may see
    int64_t seen = max_len < 1 ? 1 : max_len;
    if (window > 0) {
        const int64_t most = (int64_t)window + sinks + (p.rows + group - 1) / group + 32;
        seen = most < seen ? most : seen;
    }
    const int64_t tiles = ceil_div(seen, KV_TILE);
    const int64_t groups = R * n_heads * row_tiles;
    // Waves and parts.  A wave takes 0.63 us for a step of 32 tokens however few waves there are, and a split costs 5 us: the join, and what every part does once.
    // So nothing is split that fills the chip's 256 CUs as it is or is short (80 tiles of 128 numbers).  Where there is at most a workgroup per CU
    // it has eight waves, and parts make up one per CU; three of four waves each where parts stay long.  One workgroup more than are resident would be a round of its own.
    // All of this is measured with, and true of, 16 rows of 128 bf16 numbers, whose 166 registers let three waves on a SIMD; the plan knows no other form.  Those of 64
    // numbers hold two to four waves (125 to 191 registers); of 128 numbers two with 32 rows of bf16 (231 to 253) or 16 rows of fp16 (186 to 194), one with 32 rows of
    // fp16 (265 to 268); of 256 numbers two in bf16 (243 to 253), one in fp16 (271 to 277): there three workgroups a CU are two or three rounds, and where the kernel has no
    // form of eight waves (256 numbers; 32 rows of 128 fp16 numbers) four do the work of the eight.
    // us in a graph, 4 waves unsplit, 8 waves unsplit, best split: 1 context, 32 heads x 640 tokens 7.9, 7.8, 9.0; x 1280 -, 10.4, 10.2; x 2048 15.0, 13.2,
    // 9.8; 8 x 4 heads x 32768 188, 135, 17.6; 32 requests, 8 x 8 heads, 4 drafts x 2000 26.4, 22.6, 30; 6 x 115000 756, -, 142 (16 parts of 4 waves; 8 of 8
    // waves 148); 64 requests, 8 x 4 heads x 2000 26.8, -, 33.
    p.waves = 4;
    int64_t parts = 1;
    if (groups <= 256) {
        const bool is_short = tiles * d <= 80 * 128;
        const int64_t one = 256 / groups, three = 768 / groups;
        if (three <= MAX_PARTS && tiles >= three * 128) {
            parts = three;
        } else {
            p.waves = 8;
            if (!is_short) parts = one;
        }
        if (parts > tiles / 16) parts = tiles / 16;   // two steps of each of four waves
        if (parts > MAX_PARTS) parts = MAX_PARTS;
        if (parts < 1) parts = 1;
    }
    p.part_tiles = (int32_t)(ceil_div(ceil_div(tiles, parts), 8) * 8);   // a step of every wave
    p.parts = (int32_t)ceil_div(tiles, p.part_tiles);
    // Row tiles: those of the request with the most rows.  Where only the mean is known, up to twice as many, or 32 workgroups per CU: one that finds no rows costs
    // 2.5 ns, one too few goes through several row tiles in turn.  An odd number, as those with rows would meet on a part of the CUs otherwise (2 and 4
    // row tiles of 64 single tokens: 60 and 70 us, 5: 45).  More than a launch has workgroups for are gone through in turn too.
    const int64_t pairs = ceil_div(R * n_heads, 8) * 8 * p.parts, room = KV_MAX_GROUPS / pairs;
    int64_t shared = row_tiles;
    if (max_q <= 0) {
        const int64_t all = ceil_div(max_rows, p.rows);
        shared = 2 * row_tiles - 1 > 8192 / pairs ? 2 * row_tiles - 1 : 8192 / pairs;
        if (shared > all) shared = all;
        shared -= shared % 2 == 0;
    }
    p.row_tiles = (int32_t)(shared < room ? shared : room);
    // 64 requests of 200 to 4000 tokens 38.6 -> 32.6 us, of 2000 each 26.6 -> 27.4; chunks of prompts 435 -> 421
    p.by_length = R > 1 && R <= 64 && groups > 256 ? (p.row_tiles == 1 && !many ? 1 : 2) : 0;
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
