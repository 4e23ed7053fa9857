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
#include "kv_kernels.h"

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
__device__ __forceinline__ uint8_t *place_of(const KvView &kv, const KvRows &rows, int64_t t, int &row, bool &owned)
{
    owned = false;
    const int r = owner_of(rows.offsets, kv.R, t);
    if (r < 0) return nullptr;
    const int64_t o0 = rows.offsets[r], o1 = rows.offsets[r + 1];
    if (t < o0 || t >= o1) return nullptr;
    owned = true;
    const int64_t at = rows.start ? (int64_t)rows.start[r] + (t - o0) : (int64_t)kv.lens[r] - (o1 - t);
    const int64_t slot = at >> (kv.tile_shift + 4);
    if (at < 0 || slot >= kv.max_pages) return nullptr;
    const int32_t page = kv.table[(int64_t)r * kv.max_pages + slot];
    if (page < 0 || page >= kv.n_pages) return nullptr;
    row = (int)(at & 15);
    const int tile = (int)(at >> 4) & ((1 << kv.tile_shift) - 1);
    return kv.pages + page * kv.page_bytes + kv.layer_bytes + (int64_t)tile * kv_tile_bytes(kv.d);
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
            const uint32_t top = x[u].top();
            int e = (int)(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u);
            e = e < 1 ? 1 : e > 252 ? 252 : e;   // 6 * 2^125 at most: 2^128 would be infinite in fp32 (the conversion saturates)
            const bool odd = top >= 0x7f800000u;
            uint32_t w = x[u].codes(__uint_as_float((uint32_t)e << 23));
            if (odd) {
                w = 0;
                e = 255;
            }
            uint8_t *tile = at + h * kv.head_bytes;
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

}  // namespace ralm
