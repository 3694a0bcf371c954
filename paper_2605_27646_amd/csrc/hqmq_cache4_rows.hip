// Rows into the pages of a 4-bit cache and back (include/hqmq_cache4.h, hqmq_cache4_write and hqmq_cache4_read).
//
// A lane takes 8 channels (16 bytes of a row, one dword of codes) of one token.  Four consecutive positions, which are one block of
// the V layout, lie beside each other in a wave, so that the 64 dwords of a 128-channel head and four tokens are 256 bytes in a
// row of the cache; the four lanes of a group are 4 lanes apart and share their extrema by rotations inside 16 lanes.
#include "hqmq_cache4_device.h"

namespace hqmq {

namespace {

constexpr int kRowThreads = 256;
constexpr int kMostBlocks = 1 << 16;  // of a grid along the positions
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Extremum over lanes l, l + 4, l + 8, l + 12 of 16.
template <int kCtrl>
__device__ __forceinline__ float rotated(float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), kCtrl, 0xf, 0xf, false));
}
__device__ __forceinline__ float group_max(float x)
{
    x = fmaxf(x, rotated<0x124>(x));
    return fmaxf(x, rotated<0x128>(x));
}

template <bool kBf16>
__device__ __forceinline__ float widened(uint32_t bits)
{
    bits = (bits & 0x7fffu) > (kBf16 ? 0x7f80u : 0x7c00u) ? 0u : bits;  // a NaN counts as 0
    const float x = kBf16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    return __builtin_amdgcn_fmed3f(x, -49152.f, 49152.f);
}

// What a thread works on: 8 channels of kv head h, the same for every block of positions that it goes through.
struct Unit {
    int h, w, t;    // head, dword of the row, token of four
    bool there, is_v;
};
__device__ __forceinline__ Unit unit_of(const Cache4 &c)
{
    const int per_head = 16 * c.NG;  // 4 tokens of 4 NG dwords
    const int per_role = (c.H * per_head + kRowThreads - 1) / kRowThreads;
    Unit u;
    u.is_v = (int)blockIdx.y >= per_role;
    const int i = ((int)blockIdx.y - (u.is_v ? per_role : 0)) * kRowThreads + (int)threadIdx.x;
    u.t = i & 3;
    u.h = i / per_head;
    u.w = (i - u.h * per_head) >> 2;
    u.there = u.h < c.H;
    return u;
}

// The cache's page of a position, or -1.
__device__ __forceinline__ int page_of(const Cache4 &c, const Cache4Seqs &b, int seq, int pos)
{
    const int page = b.table[(int64_t)seq * b.pitch + (pos >> c.page_shift)];
    return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

}  // namespace

// Bound by memory for prompts, by launch and latency for a step's rows.
template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void k_cache4_write(Cache4 c, Cache4Seqs b, Cache4Rows k, Cache4Rows v)
{
    const int seq = blockIdx.z;
    const Cache4Seq s = cache4_seq(b, c.page_shift, seq);
    const Unit u = unit_of(c);
    const Cache4Rows &rows = u.is_v ? v : k;
    uint8_t *const codes = u.is_v ? c.v_codes : c.k_codes;
    uint8_t *const scales = u.is_v ? c.v_scales : c.k_scales;
    const int ch = 8 * u.w, row_bytes = 16 * c.NG;
    for (int block = (max(s.pos0, 0) >> 2) + (int)blockIdx.x; 4 * block < s.length && s.n > 0; block += (int)gridDim.x) {
        const int pos = 4 * block + u.t;
        const int page = u.there && pos >= s.pos0 && pos < s.length ? page_of(c, b, seq, pos) : -1;
        uint4v bits = uint4v{0u, 0u, 0u, 0u};
        if (page >= 0 && ch < c.D) {
            const uint16_t *src = rows.data + (int64_t)(s.first_row + (pos - s.pos0)) * rows.row + u.h * rows.head + ch;
            if (rows.wide) {
                bits = *reinterpret_cast<const uint4v *>(src);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (ch + e < c.D)
                        bits[e / 2] |= (uint32_t)src[e] << (16 * (e & 1));
            }
        }
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = widened<kBf16>((bits[e / 2] >> (16 * (e & 1))) & 0xffffu);
        uint32_t code = 0, scale;
        if (kFormat == HQMQ_CACHE4_FLOAT) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                top = fmaxf(top, fabsf(x[e]));
            top = group_max(top);
            // 7 / 4 has the fraction bits 0x600000: an exponent more for anything above
            const int exponent = min(max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 2, 127 - 23), 127 + 13);
            scale = (uint32_t)exponent;
            const float unit = e8m0(scale);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], unit, 0);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], unit, 1);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], unit, 2);
            code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], unit, 3);
        } else {
            const int n = min(max(c.D - ch, 0), 8);
            float high = -1.0e30f, low = 1.0e30f;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) {
                    high = fmaxf(high, x[e]);
                    low = fminf(low, x[e]);
                }
            high = group_max(high);
            low = -group_max(-low);
            if (low > high)  // channels past the head's only
                low = high = 0.f;
            float fifteenth = (high - low) * (1.f / 15.f);
            asm("" : "+v"(fifteenth));  // rounded to fp32 before fp16: v_fma_mixlo_f16 would round the product once
            const _Float16 s16 = (_Float16)fifteenth, m16 = (_Float16)low;
            scale = __builtin_bit_cast(uint32_t, cache4_h2{s16, m16});
            const float step = (float)s16, least = (float)m16, inverse = step > 0.f ? 1.f / step : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float q = (x[e] - least) * inverse;
                float r = rintf(q);
                // three roundings put q up to 16 * 3 * 2^-24 off: next to the middle of two codes the exact quotient decides
                if (fabsf(fabsf(q - r) - 0.5f) < 1.0e-5f)
                    r = (float)rint(((double)x[e] - (double)least) / (double)step);
                const uint32_t q4 = (uint32_t)__builtin_amdgcn_fmed3f(r, 0.f, 15.f);
                code |= (e < n ? q4 : 0u) << (4 * e);
            }
        }
        if (page < 0)
            continue;
        const int slot = pos & ((1 << c.page_shift) - 1);
        const int64_t row0 = ((int64_t)page * c.H + u.h) << c.page_shift;  // of the head's page
        int64_t scale_at = row0 * c.NG;
        if (!u.is_v) {
            *reinterpret_cast<uint32_t *>(codes + (row0 + slot) * row_bytes + 4 * u.w) = code;
            scale_at += slot * c.NG + (u.w >> 2);
        } else {
            const Cache4Place p = cache4_v_place(c.NG, u.w, u.t);
            uint8_t *at = codes + (row0 + (slot & ~3)) * row_bytes + p.at;
            if (p.bytes == 4) {
                *reinterpret_cast<uint32_t *>(at) = code;
            } else if (p.bytes == 2) {
                *reinterpret_cast<uint16_t *>(at) = (uint16_t)code;
                *reinterpret_cast<uint16_t *>(at + 8) = (uint16_t)(code >> 16);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    at[4 * r] = (uint8_t)(code >> (8 * r));
            }
            scale_at += (slot & ~3) * c.NG + (u.w >> 2) * 4 + u.t;
        }
        if ((u.w & 3) == 0) {
            if (kFormat == HQMQ_CACHE4_FLOAT)
                scales[scale_at] = (uint8_t)scale;
            else
                reinterpret_cast<uint32_t *>(scales)[scale_at] = scale;
        }
    }
}

template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void k_cache4_read(Cache4 c, Cache4Seqs b, Cache4Rows k, Cache4Rows v)
{
    const int seq = blockIdx.z;
    const Cache4Seq s = cache4_seq(b, c.page_shift, seq);
    const Unit u = unit_of(c);
    const Cache4Rows &rows = u.is_v ? v : k;
    const uint8_t *const codes = u.is_v ? c.v_codes : c.k_codes;
    const uint8_t *const scales = u.is_v ? c.v_scales : c.k_scales;
    const int ch = 8 * u.w, row_bytes = 16 * c.NG;
    if (!u.there || ch >= c.D)
        return;
    for (int block = (s.pos0 >> 2) + (int)blockIdx.x; 4 * block < s.length; block += (int)gridDim.x) {
        const int pos = 4 * block + u.t;
        if (pos < s.pos0 || pos >= s.length)
            continue;
        const int page = pos >= 0 ? page_of(c, b, seq, pos) : -1;
        uint4v bits = uint4v{0u, 0u, 0u, 0u};
        if (page >= 0) {
            const int slot = pos & ((1 << c.page_shift) - 1);
            const int64_t row0 = ((int64_t)page * c.H + u.h) << c.page_shift;
            int64_t scale_at = row0 * c.NG;
            uint32_t code;
            if (!u.is_v) {
                code = *reinterpret_cast<const uint32_t *>(codes + (row0 + slot) * row_bytes + 4 * u.w);
                scale_at += slot * c.NG + (u.w >> 2);
            } else {
                const Cache4Place p = cache4_v_place(c.NG, u.w, u.t);
                const uint8_t *at = codes + (row0 + (slot & ~3)) * row_bytes + p.at;
                if (p.bytes == 4)
                    code = *reinterpret_cast<const uint32_t *>(at);
                else if (p.bytes == 2)
                    code = *reinterpret_cast<const uint16_t *>(at) | (uint32_t) * reinterpret_cast<const uint16_t *>(at + 8) << 16;
                else
                    code = at[0] | (uint32_t)at[4] << 8 | (uint32_t)at[8] << 16 | (uint32_t)at[12] << 24;
                scale_at += (slot & ~3) * c.NG + (u.w >> 2) * 4 + u.t;
            }
            cache4_h2 y[4];
            if (kFormat == HQMQ_CACHE4_FLOAT) {
                const float unit = e8m0(scales[scale_at]);
                y[0] = e2m1_pair<0>(code, unit);
                y[1] = e2m1_pair<1>(code, unit);
                y[2] = e2m1_pair<2>(code, unit);
                y[3] = e2m1_pair<3>(code, unit);
            } else {
                const cache4_h2 sm = __builtin_bit_cast(cache4_h2, reinterpret_cast<const uint32_t *>(scales)[scale_at]);
                const cache4_h2 ss = {sm[0], sm[0]}, mm = {sm[1], sm[1]};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t two = code >> (8 * e);
                    y[e] = int4_pair((two & 0xfu) | (two & 0xf0u) << 12, ss, mm);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (kBf16) {
                    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                    bits[e] = __builtin_bit_cast(uint32_t, b2{(__bf16)(float)y[e][0], (__bf16)(float)y[e][1]});
                } else {
                    bits[e] = __builtin_bit_cast(uint32_t, y[e]);
                }
            }
        }
        uint16_t *dst = rows.data + (int64_t)(s.first_row + (pos - s.pos0)) * rows.row + u.h * rows.head + ch;
        if (rows.wide) {
            *reinterpret_cast<uint4v *>(dst) = bits;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (ch + e < c.D)
                    dst[e] = (uint16_t)(bits[e / 2] >> (16 * (e & 1)));
        }
    }
}

namespace {

dim3 rows_grid(const Cache4 &c, const Cache4Seqs &b, int max_rows)
{
    const int per_role = (c.H * 16 * c.NG + kRowThreads - 1) / kRowThreads;
    const int blocks = max_rows == 1 ? 1 : (max_rows - 1) / 4 + 2;  // wherever in a block of four the first position lies
    return dim3((unsigned)(blocks < kMostBlocks ? blocks : kMostBlocks), (unsigned)(2 * per_role), (unsigned)b.n_seqs);
}

}  // namespace

hipError_t launch_cache4_write(const Cache4 &c, const Cache4Seqs &b, int max_rows, bool bf16, const Cache4Rows &k, const Cache4Rows &v,
                               hipStream_t stream)
{
    const dim3 grid = rows_grid(c, b, max_rows);
    const auto kernel = c.format == HQMQ_CACHE4_FLOAT ? (bf16 ? k_cache4_write<HQMQ_CACHE4_FLOAT, true> : k_cache4_write<HQMQ_CACHE4_FLOAT, false>)
                                                      : (bf16 ? k_cache4_write<HQMQ_CACHE4_INT, true> : k_cache4_write<HQMQ_CACHE4_INT, false>);
    kernel<<<grid, kRowThreads, 0, stream>>>(c, b, k, v);
    return hipGetLastError();
}

hipError_t launch_cache4_read(const Cache4 &c, const Cache4Seqs &b, int max_rows, bool bf16, const Cache4Rows &k, const Cache4Rows &v,
                              hipStream_t stream)
{
    const dim3 grid = rows_grid(c, b, max_rows);
    const auto kernel = c.format == HQMQ_CACHE4_FLOAT ? (bf16 ? k_cache4_read<HQMQ_CACHE4_FLOAT, true> : k_cache4_read<HQMQ_CACHE4_FLOAT, false>)
                                                      : (bf16 ? k_cache4_read<HQMQ_CACHE4_INT, true> : k_cache4_read<HQMQ_CACHE4_INT, false>);
    kernel<<<grid, kRowThreads, 0, stream>>>(c, b, k, v);
    return hipGetLastError();
}

}  // namespace hqmq
