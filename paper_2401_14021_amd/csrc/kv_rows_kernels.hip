// Keys and values into the 4-bit cache and back.
//
//  kv_append_kernel  blocks of 32 numbers x: 2^e with the smallest e for which max|x| <= 6 * 2^e, codes of x / 2^e on the grid
//                    +-{0, .5, 1, 1.5, 2, 3, 4, 6}, nearest, ties to the even code.  The division by a power of two is exact, so the
//                    only rounding is that of the code itself (one instruction for two numbers).  The exponent is chosen so that
//                    nothing saturates: the largest number of a block lands in (3, 6].
//  kv_read_kernel    the numbers that the codes stand for; exact in every type that holds the power.
//
// Both move bytes: what bounds them is memory for prompts (10400 tokens x 32 heads x 128, bf16: 42 to 51 us in, 4.4 to 5.3 TB/s; 34 us out, 42 when neighbouring
// tokens lay on different XCDs) and the chain offsets -> length -> page -> store for single tokens (3.7 us).  One wave per token and K or V: eight numbers a
// lane and step (16 bytes of a 16-bit type), four lanes per block, so that the block's maximum is two exchanges.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "decoder_kernels.h"

namespace ralm {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

// eight numbers of a row as they are: 16-bit types are looked through and converted two at a time, without being widened
template <int DT>
struct Eight {
    uint32_t w[DT == DT_F32 ? 8 : 4];
    __device__ __forceinline__ void load(const void *p, int64_t at)
    {
        if constexpr (DT == DT_F32) {
            const uint4 *s = reinterpret_cast<const uint4 *>(static_cast<const float *>(p) + at);
            const uint4 a = s[0], b = s[1];
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
        } else {
            const uint4 a = *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(p) + at);
            w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
        }
    }
    // the largest magnitude of the 32 numbers that four neighbouring lanes hold, as the bits of an fp32 number: magnitudes are in the order of
    // whole numbers, NaN beyond infinity
    __device__ __forceinline__ uint32_t top() const
    {
        if constexpr (DT == DT_F32) {
            uint32_t t = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) t = max(t, w[j] & 0x7fffffffu);
            t = max(t, lane_xor<1>(t));
            return max(t, lane_xor<2>(t));
        } else {
            auto larger = [](uint32_t x, uint32_t y) {
                return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, x), __builtin_bit_cast(u16x2, y)));
            };
            uint32_t t = larger(larger(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), larger(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
            t = larger(t, lane_xor<1>(t));
            t = larger(t, lane_xor<2>(t));
            t = max(t & 0xffffu, t >> 16);
            return DT == DT_BF16 ? t << 16 : __float_as_uint(f16_bits_to_f32(t));
        }
    }
    // their codes for the power `unit`
    __device__ __forceinline__ uint32_t codes(float unit) const
    {
        uint32_t c = 0;
        if constexpr (DT == DT_F32) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[0]), __uint_as_float(w[1]), unit, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[2]), __uint_as_float(w[3]), unit, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[4]), __uint_as_float(w[5]), unit, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, __uint_as_float(w[6]), __uint_as_float(w[7]), unit, 3);
        } else if constexpr (DT == DT_BF16) {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[0]), unit, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[1]), unit, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[2]), unit, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, w[3]), unit, 3);
        } else {
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[0]), unit, 0);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[1]), unit, 1);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[2]), unit, 2);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(c, __builtin_bit_cast(f16x2, w[3]), unit, 3);
        }
        return c;
    }
};

template <int DT>
__device__ __forceinline__ void store8(void *p, int64_t at, const float (&x)[8])
{
    const float4 a = make_float4(x[0], x[1], x[2], x[3]), b = make_float4(x[4], x[5], x[6], x[7]);
    if constexpr (DT == DT_F32) {
        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(p) + at);
        d[0] = a;
        d[1] = b;
    } else {
        // bf16: a block's numbers have two bits behind the leading one and the exponents of fp32; NaN keeps its high half
        uint4 r;
        if constexpr (DT == DT_F16) {
            r = pack8<DT_F16>(a, b);
        } else {
            r.x = __float_as_uint(x[0]) >> 16 | (__float_as_uint(x[1]) & 0xffff0000u);
            r.y = __float_as_uint(x[2]) >> 16 | (__float_as_uint(x[3]) & 0xffff0000u);
            r.z = __float_as_uint(x[4]) >> 16 | (__float_as_uint(x[5]) & 0xffff0000u);
            r.w = __float_as_uint(x[6]) >> 16 | (__float_as_uint(x[7]) & 0xffff0000u);
        }
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = r;
    }
}

// where a token lies: its tile of head 0 of the layer, and its row in the tile; NULL if it has no place.  owned: whether it is any request's
// r, at: its request and place
__device__ __forceinline__ uint8_t *place_of(const KvView &kv, const KvRows &rows, int64_t t, int &row, bool &owned, int &r, int64_t &at)
{
    owned = false;
    r = owner_of(rows.offsets, kv.R, t);
    if (r < 0) return nullptr;
    const int64_t o0 = rows.offsets[r], o1 = rows.offsets[r + 1];
    if (t < o0 || t >= o1) return nullptr;
    owned = true;
    at = rows.start ? (int64_t)rows.start[r] + (t - o0) : (int64_t)kv.lens[r] - (o1 - t);
    const int64_t slot = at >> (kv.tile_shift + 4);
    if (at < 0 || slot >= kv.max_pages) return nullptr;
    const int32_t page = kv.table[(int64_t)r * kv.max_pages + slot];
    if (page < 0 || page >= kv.n_pages) return nullptr;
    row = (int)(at & 15);
    const int tile = (int)(at >> 4) & ((1 << kv.tile_shift) - 1);
    return kv.pages + page * kv.page_bytes + kv.layer_bytes + (int64_t)tile * kv_tile_bytes(kv.d);
}
__device__ __forceinline__ uint8_t *place_of(const KvView &kv, const KvRows &rows, int64_t t, int &row, bool &owned)
{
    int r;
    int64_t at;
    return place_of(kv, rows, t, row, owned, r, at);
}

// byte of a tile where the codes of numbers 8 c .. 8 c + 7 of token `row` begin (D = 64: the second half lies D / 8 bytes on)
template <int D>
__device__ __forceinline__ int k_codes(int row, int c) { return row * (D / 2) + 4 * c; }
template <int D>
__device__ __forceinline__ int v_codes(int row, int c)
{
    constexpr int U = D / 16;   // codes of a sixteenth
    return 8 * D + ((row >> 2) * 16 + 8 * c / U) * (D / 8) + (row & 3) * (D / 32) + (8 * c % U) / 2;
}
template <int D>
__device__ __forceinline__ int k_power(int row, int b) { return 16 * D + row * (D / 32) + b; }
template <int D>
__device__ __forceinline__ int v_power(int row, int b) { return 16 * D + D / 2 + ((row >> 2) * (D / 32) + b) * 4 + (row & 3); }

// Workgroup b runs on XCD b % 8: an XCD gets neighbouring tokens, so that what they share of a line (values of four tokens lie beside each other)
// comes together in its L2
__device__ __forceinline__ int64_t unit_of_wave()
{
    const uint32_t per = (gridDim.x + 7) / 8, b = (blockIdx.x & 7u) * per + (blockIdx.x >> 3);
    return (int64_t)b * 4 + (threadIdx.x >> 6);
}

// a piece's codes and, by the first lane of the four that share it, their power
template <int D, int DT>
__device__ __forceinline__ void store_piece(uint8_t *tile, bool values, int row, int c, const Eight<DT> &x)
{
    const uint32_t top = x.top();
    int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u);
    e = e < 1 ? 1 : e > 252 ? 252 : e;   // 6 * 2^125 at most: 2^128 would be infinite in fp32 (the conversion saturates)
    const bool odd = top >= 0x7f800000u;
    uint32_t w = x.codes(__uint_as_float((uint32_t)e << 23));
    if (odd) {
        w = 0;
        e = 255;
    }
    if (!values) {
        *reinterpret_cast<uint32_t *>(tile + k_codes<D>(row, c)) = w;
    } else if constexpr (D == 64) {
        *reinterpret_cast<uint16_t *>(tile + v_codes<D>(row, c)) = (uint16_t)w;
        *reinterpret_cast<uint16_t *>(tile + v_codes<D>(row, c) + D / 8) = (uint16_t)(w >> 16);
    } else {
        *reinterpret_cast<uint32_t *>(tile + v_codes<D>(row, c)) = w;
    }
    if ((c & 3) == 0) tile[values ? v_power<D>(row, c >> 2) : k_power<D>(row, c >> 2)] = (uint8_t)e;
}

template <int D, int DT>
__global__ __launch_bounds__(256) void kv_append_kernel(KvView kv, KvRows rows)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = unit_of_wave();
    const int64_t t = unit >> 1;
    const bool values = unit & 1;
    if (t >= rows.n) return;
    const void *src = values ? rows.v : rows.k;
    const int64_t ts = values ? rows.v_token : rows.k_token, hs = values ? rows.v_head : rows.k_head;
    constexpr int C = D / 8;   // pieces of a head
    const int pieces = kv.n_heads * C;
    // Four steps' loads under way at once, the first of them while the token's place is looked up.  A multiple of four pieces: the lanes of a block come
    // together
    Eight<DT> x[4];
    auto load4 = [&](int i0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 64 * u;
            if (i < pieces) x[u].load(src, t * ts + i / C * hs + 8 * (i % C));
        }
    };
    load4(lane);
    int row = 0;
    bool owned;
    uint8_t *at = place_of(kv, rows, t, row, owned);
    if (!at) return;
    for (int i0 = lane; i0 < pieces; i0 += 256) {
        if (i0 != lane) load4(i0);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 64 * u, h = i / C, c = i % C;
            if (i >= pieces) break;
            store_piece<D>(at + h * kv.head_bytes, values, row, c, x[u]);
        }
    }
}

template <int D, int DT>
__global__ __launch_bounds__(256) void kv_read_kernel(KvView kv, KvRows rows)
{
    const int lane = threadIdx.x & 63;
    const int64_t unit = unit_of_wave();
    const int64_t t = unit >> 1;
    const bool values = unit & 1;
    if (t >= rows.n) return;
    void *dst = values ? rows.v : rows.k;
    const int64_t ts = values ? rows.v_token : rows.k_token, hs = values ? rows.v_head : rows.k_head;
    int row = 0;
    bool owned;
    const uint8_t *at = place_of(kv, rows, t, row, owned);
    if (!owned) return;   // the caller's row stays as it is
    constexpr int C = D / 8;
    const int pieces = kv.n_heads * C;
    for (int i = lane; i < pieces; i += 64) {
        const int h = i / C, c = i % C;
        uint32_t w = 0, e = 0;   // a token without a place reads as zeros
        if (at) {
            const uint8_t *tile = at + h * kv.head_bytes;
            if (!values) {
                w = *reinterpret_cast<const uint32_t *>(tile + k_codes<D>(row, c));
            } else if constexpr (D == 64) {
                w = *reinterpret_cast<const uint16_t *>(tile + v_codes<D>(row, c));
                w |= (uint32_t) * reinterpret_cast<const uint16_t *>(tile + v_codes<D>(row, c) + D / 8) << 16;
            } else {
                w = *reinterpret_cast<const uint32_t *>(tile + v_codes<D>(row, c));
            }
            e = tile[values ? v_power<D>(row, c >> 2) : k_power<D>(row, c >> 2)];
        }
        const float p = __uint_as_float(e << 23);
        float x[8];
        const auto a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 0);
        const auto b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 1);
        const auto f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 2);
        const auto g = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, p, 3);
        x[0] = a[0], x[1] = a[1], x[2] = b[0], x[3] = b[1], x[4] = f[0], x[5] = f[1], x[6] = g[0], x[7] = g[1];
        store8<DT>(dst, t * ts + h * hs + 8 * c, x);
    }
}

// ---- rotary positions on the way in ----------------------------------------------------------------

// Numbers as they are and back.  A turned number is a sum in 64 bits that becomes fp32 and then its type: two sides that form the
// angle alike agree to 2^-50, so that a key's codes do not depend on who formed them.
template <int DT>
__device__ __forceinline__ double number(const void *p, int64_t at)
{
    if constexpr (DT == DT_F32) return static_cast<const float *>(p)[at];
    const uint32_t b = static_cast<const uint16_t *>(p)[at];
    return DT == DT_BF16 ? __uint_as_float(b << 16) : f16_bits_to_f32(b);
}
template <int DT>
__device__ __forceinline__ uint32_t bits_of(double x)
{
    float f = (float)x;
    asm("" : "+v"(f));   // two roundings, as documented: the compiler would make one of them
    if constexpr (DT == DT_F32) return __float_as_uint(f);
    else if constexpr (DT == DT_BF16) return __builtin_bit_cast(uint16_t, (__bf16)f);
    else return __builtin_bit_cast(uint16_t, (_Float16)f);
}
template <int DT>
__device__ __forceinline__ double number_of(const Eight<DT> &x, int j)
{
    if constexpr (DT == DT_F32) return __uint_as_float(x.w[j]);
    const uint32_t b = j & 1 ? x.w[j / 2] >> 16 : x.w[j / 2] & 0xffffu;
    return DT == DT_BF16 ? __uint_as_float(b << 16) : f16_bits_to_f32(b);
}
template <int DT>
__device__ __forceinline__ void pack(Eight<DT> &x, const double (&y)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if constexpr (DT == DT_F32) x.w[j] = bits_of<DT>(y[j]);
        else if (j & 1) x.w[j / 2] |= bits_of<DT>(y[j]) << 16;
        else x.w[j / 2] = bits_of<DT>(y[j]);
    }
}
template <int DT>
__device__ __forceinline__ void store_eight(void *p, int64_t at, const Eight<DT> &x)
{
    if constexpr (DT == DT_F32) {
        uint4 *d = reinterpret_cast<uint4 *>(static_cast<float *>(p) + at);
        d[0] = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
        d[1] = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
    } else {
        *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p) + at) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
    }
}

// A workgroup takes a token: its place and the cosines and sines of its angles, once for all heads, while the first of its queries, keys and values are under way;
// then all of them.  12018 tokens of 32 + 8 heads of 128, bf16: 56 us, 4.6 TB/s (59 with loads behind the place and the angles); 64 tokens 5.0, the chain of
// offsets, length, page and angle.
// WHOLE: partners lie in pieces of 8 that are loaded whole (interleaved ones in the same piece, others where half is a multiple of 8); otherwise 256 pieces at a time, whole
// heads, meet in LDS, where a number finds its partner at any distance (half 50: 69 us, pair by pair from memory 136; 64 tokens 6.4, 9).
template <int D, int DT, bool WHOLE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void kv_append_rotary_kernel(KvView kv, KvRows rows, KvRotary p)
{
    constexpr int C = D / 8;   // pieces of a head
    __shared__ double2 turns[D / 2];
    __shared__ uint32_t met[WHOLE ? 1 : 256 * (DT == DT_F32 ? 8 : 4)];
    const int tid = threadIdx.x;
    // tokens beside each other on one XCD, as in the append
    const uint32_t per = (gridDim.x + 7) / 8, b = (blockIdx.x & 7u) * per + (blockIdx.x >> 3);
    const int64_t t = b;
    if (t >= rows.n) return;
    static_assert(WHOLE || !INTERLEAVED, "interleaved pairs lie in whole pieces");
    const int half = p.half;

    // Queries by units: a piece of the lower half with its partner in the upper one, then pieces that do not turn; interleaved, every piece by itself
    const int low = WHOLE && !INTERLEAVED ? half / 8 : 0, units = C - low, q_units = p.n_q_heads * units;
    auto load_q = [&](int i, Eight<DT> &x, Eight<DT> &z) __attribute__((always_inline)) {
        const int h = i / units, c = i - h * units;
        const int64_t in = t * p.q_token + h * p.q_head;
        x.load(p.q, in + 8 * (c < low ? c : c + low));
        if (c < low) z.load(p.q, in + 8 * c + half);
    };
    auto finish_q = [&](int i, Eight<DT> &x, Eight<DT> &z) __attribute__((always_inline)) {
        const int h = i / units, c = i - h * units;
        const int64_t to = t * p.o_token + h * p.o_head;
        if constexpr (INTERLEAVED) {
            if (8 * c < 2 * half) {
                double y[8];
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const bool turn = 4 * c + j / 2 < half;   // (a piece may hold the last pair and what does not turn)
                    const double2 cs = turns[turn ? 4 * c + j / 2 : 0];
                    const double u = number_of<DT>(x, j), v = number_of<DT>(x, j + 1);
                    y[j] = turn ? u * cs.x - v * cs.y : u;
                    y[j + 1] = turn ? v * cs.x + u * cs.y : v;
                }
                pack<DT>(x, y);
            }
        } else if (c < low) {
            double y[8], w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double2 cs = turns[8 * c + j];
                const double u = number_of<DT>(x, j), v = number_of<DT>(z, j);
                y[j] = u * cs.x - v * cs.y;
                w[j] = v * cs.x + u * cs.y;
            }
            pack<DT>(x, y);
            pack<DT>(z, w);
            store_eight<DT>(p.q_out, to + 8 * c + half, z);
        }
        store_eight<DT>(p.q_out, to + 8 * (c < low ? c : c + low), x);
    };
    // Keys, each piece by itself with the partners that it needs read too, then values as they are
    const int k_units = kv.n_heads * C;
    auto load_kv = [&](int i, Eight<DT> &x, Eight<DT> &z) __attribute__((always_inline)) {
        const bool values = i >= k_units;
        const int u = values ? i - k_units : i, h = u / C, c = u % C;
        const int64_t in = values ? t * rows.v_token + h * rows.v_head : t * rows.k_token + h * rows.k_head;
        x.load(values ? rows.v : rows.k, in + 8 * c);
        if (WHOLE && !INTERLEAVED && !values && 8 * c < 2 * half) z.load(rows.k, in + (8 * c < half ? 8 * c + half : 8 * c - half));
    };
    auto finish_kv = [&](int i, Eight<DT> &x, Eight<DT> &z, uint8_t *at, int row) __attribute__((always_inline)) {
        const bool values = i >= k_units;
        const int u = values ? i - k_units : i, h = u / C, c = u % C;
        if (WHOLE && !values && 8 * c < 2 * half) {
            double y[8];
            if constexpr (INTERLEAVED) {
#pragma unroll
                for (int j = 0; j < 8; j += 2) {
                    const bool turn = 4 * c + j / 2 < half;
                    const double2 cs = turns[turn ? 4 * c + j / 2 : 0];
                    const double e = number_of<DT>(x, j), f = number_of<DT>(x, j + 1);
                    y[j] = turn ? e * cs.x - f * cs.y : e;
                    y[j + 1] = turn ? f * cs.x + e * cs.y : f;
                }
            } else {
                const bool lower = 8 * c < half;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const double2 cs = turns[(lower ? 8 * c : 8 * c - half) + j];
                    const double e = number_of<DT>(x, j), f = number_of<DT>(z, j);
                    y[j] = lower ? e * cs.x - f * cs.y : e * cs.x + f * cs.y;
                }
            }
            pack<DT>(x, y);
        }
        store_piece<D>(at + h * kv.head_bytes, values, row, c, x);
    };

    Eight<DT> q0, q1, k0, k1;
    if (tid < q_units) load_q(tid, q0, q1);
    if (tid < 2 * k_units) load_kv(tid, k0, k1);
    int row = 0, r = 0;
    int64_t place = 0;
    bool owned = false;
    uint8_t *at = place_of(kv, rows, t, row, owned, r, place);   // every wave for itself
    if (!owned) return;
    if (p.shift) place += p.shift[r];
    for (int j = tid; j < half; j += 256) {
        double c, s;
        sincos((double)place * p.freqs[j], &s, &c);
        turns[j] = make_double2(c * p.amplitude, s * p.amplitude);
    }
    __syncthreads();
    if constexpr (WHOLE) {
        for (int i = tid; i < q_units; i += 256) {
            if (i != tid) load_q(i, q0, q1);
            finish_q(i, q0, q1);
        }
    } else {
        // x with its partners from the pieces of this pass, which begins with whole heads; all threads
        auto turn = [&](Eight<DT> &x, bool turned, int c) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (DT == DT_F32) met[8 * tid + j] = x.w[j];
                else if (j < 4) met[4 * tid + j] = x.w[j];
            }
            __syncthreads();
            if (turned && 8 * c < 2 * half) {
                const int head = 8 * (tid - c);
                double y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int e = 8 * c + j;
                    const bool lower = e < half, turns_too = e < 2 * half;
                    const double2 cs = turns[lower ? e : turns_too ? e - half : 0];
                    const double u = number_of<DT>(x, j), v = number<DT>(met, head + (lower ? e + half : turns_too ? e - half : e));
                    y[j] = !turns_too ? u : lower ? u * cs.x - v * cs.y : u * cs.x + v * cs.y;
                }
                pack<DT>(x, y);
            }
            __syncthreads();
        };
        for (int i0 = 0; i0 < q_units; i0 += 256) {
            const int i = i0 + tid, h = i / C, c = i % C;
            if (i0 > 0 && i < q_units) load_q(i, q0, q1);
            turn(q0, i < q_units, c);
            if (i < q_units) store_eight<DT>(p.q_out, t * p.o_token + h * p.o_head + 8 * c, q0);
        }
        for (int i0 = 0; i0 < k_units; i0 += 256) {
            const int i = i0 + tid;
            if (i0 > 0 && i < 2 * k_units) load_kv(i, k0, k1);
            turn(k0, i < k_units, i % C);
            if (at && i < 2 * k_units) finish_kv(i, k0, k1, at, row);
        }
        if (!at) return;
        for (int i = (k_units + 255) / 256 * 256 + tid; i < 2 * k_units; i += 256) {   // values alone
            load_kv(i, k0, k1);
            finish_kv(i, k0, k1, at, row);
        }
        return;
    }
    if (!at) return;
    for (int i = tid; i < 2 * k_units; i += 256) {
        if (i != tid) load_kv(i, k0, k1);
        finish_kv(i, k0, k1, at, row);
    }
}

template <int D, int DT>
hipError_t rotary_of(const KvView &kv, const KvRows &rows, const KvRotary &p, hipStream_t stream)
{
    const dim3 grid((unsigned)((rows.n + 7) / 8 * 8));
    if (p.interleaved) kv_append_rotary_kernel<D, DT, true, true><<<grid, 256, 0, stream>>>(kv, rows, p);
    else if (p.half % 8 == 0) kv_append_rotary_kernel<D, DT, true, false><<<grid, 256, 0, stream>>>(kv, rows, p);
    else kv_append_rotary_kernel<D, DT, false, false><<<grid, 256, 0, stream>>>(kv, rows, p);
    return hipGetLastError();
}
template <int D>
hipError_t rotary_any(const KvView &kv, const KvRows &rows, const KvRotary &p, hipStream_t stream)
{
    return rows.dtype == DT_F32    ? rotary_of<D, DT_F32>(kv, rows, p, stream)
           : rows.dtype == DT_BF16 ? rotary_of<D, DT_BF16>(kv, rows, p, stream)
                                   : rotary_of<D, DT_F16>(kv, rows, p, stream);
}

template <int D>
hipError_t rows_of(bool append, const KvView &kv, const KvRows &rows, hipStream_t stream)
{
    const dim3 grid((unsigned)((rows.n * 2 + 31) / 32 * 8));   // whole rounds of the 8 XCDs
    if (append) {
        if (rows.dtype == DT_F32) kv_append_kernel<D, DT_F32><<<grid, 256, 0, stream>>>(kv, rows);
        else if (rows.dtype == DT_BF16) kv_append_kernel<D, DT_BF16><<<grid, 256, 0, stream>>>(kv, rows);
        else kv_append_kernel<D, DT_F16><<<grid, 256, 0, stream>>>(kv, rows);
    } else {
        if (rows.dtype == DT_F32) kv_read_kernel<D, DT_F32><<<grid, 256, 0, stream>>>(kv, rows);
        else if (rows.dtype == DT_BF16) kv_read_kernel<D, DT_BF16><<<grid, 256, 0, stream>>>(kv, rows);
        else kv_read_kernel<D, DT_F16><<<grid, 256, 0, stream>>>(kv, rows);
    }
    return hipGetLastError();
}

hipError_t any_rows(bool append, const KvView &kv, const KvRows &rows, hipStream_t stream)
{
    return kv.d == 64 ? rows_of<64>(append, kv, rows, stream) : kv.d == 128 ? rows_of<128>(append, kv, rows, stream) : rows_of<256>(append, kv, rows, stream);
}

}  // namespace

hipError_t launch_kv_append(const KvView &kv, const KvRows &rows, hipStream_t stream) { return any_rows(true, kv, rows, stream); }
hipError_t launch_kv_read(const KvView &kv, const KvRows &rows, hipStream_t stream) { return any_rows(false, kv, rows, stream); }
hipError_t launch_kv_append_rotary(const KvView &kv, const KvRows &rows, const KvRotary &p, hipStream_t stream)
{
    return kv.d == 64 ? rotary_any<64>(kv, rows, p, stream) : kv.d == 128 ? rotary_any<128>(kv, rows, p, stream) : rotary_any<256>(kv, rows, p, stream);
}

}  // namespace ralm
