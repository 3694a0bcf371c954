// Rows into the pages of a 4-bit cache and back (include/hqmq_cache4.h, hqmq_cache4_write and hqmq_cache4_read).
//
// A lane takes 8 channels (16 bytes of a row, a dword of codes) of the four tokens of one block of the V layout: rows are moved
// 1 KB a wave and instruction, V's codes of the four tokens are 16 consecutive bytes, and the four lanes of a group lie beside each
// other.  One token a lane, the four of a block in lanes of their own, moved rows in pieces of 256 bytes: 2 x 32768 tokens of 8 heads
// x 96 read back in 100 us, this way 60 (255 MB, 4.3 TB/s); 7246 rows of 8 heads x 128 written 15 and 10.3 us.
//
// Bound by memory for prompts, by launch and latency for a step's rows (3 to 3.5 us), and between them by issue where integers are written:
// 1200 rows of 8 heads x 128 6.0 us, 5.2 were no tie to be decided, 4.1 in the float format.  A workgroup takes one block of positions, which
// leaves lanes without work where its heads are fewer than 256 lanes take: 65536 rows of 1 x 128 read in 14.7 us and written in 27.4,
// where 8192 rows of 8 x 128, as many bytes, take 8.7 each.
#include <type_traits>

#include "hqmq_cache4_device.h"

namespace hqmq {

namespace {

constexpr int kRowThreads = 256;
constexpr int64_t kMostGroups = 1 << 22;  // empty ones take some 0.3 ns each
constexpr int64_t kFewGroups = 1024;      // up to here empty workgroups cost less than the search for a place's sequence
constexpr int kPastAll = 1 << 28;  // blocks of four positions that a sequence has at most
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Maximum over the four lanes of a group.
__device__ __forceinline__ float group_max(float x)
{
    x = fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0xb1, 0xf, 0xf, false)));  // lanes 1 0 3 2
    return fmaxf(x, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x4e, 0xf, 0xf, false)));  // lanes 2 3 0 1
}

template <bool kBf16>
__device__ __forceinline__ float widened(uint32_t bits)
{
    return kBf16 ? __uint_as_float(bits << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
}

// The largest magnitude of 8 channels, as its bits.  NaN become 0 and what is larger than 49152 that, which is rare: found by integers, two
// channels an instruction.
template <bool kBf16>
__device__ __forceinline__ uint32_t cleaned(uint4v &bits)
{
    typedef unsigned short us2 __attribute__((ext_vector_type(2)));
    constexpr uint32_t kNan = kBf16 ? 0x7f80u : 0x7c00u, kMost = kBf16 ? 0x4740u : 0x7a00u;
    const auto top_of = [&] {
        us2 y = {0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y = __builtin_elementwise_max(y, __builtin_bit_cast(us2, bits[e] & 0x7fff7fffu));
        return max((uint32_t)y[0], (uint32_t)y[1]);
    };
    uint32_t top = top_of();
    if (__builtin_expect(top > kMost, 0)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const auto clean = [&](uint32_t y) { return (y & 0x7fffu) > kNan ? 0u : (y & 0x8000u) | min(y & 0x7fffu, kMost); };
            bits[e] = clean(bits[e] & 0xffffu) | clean(bits[e] >> 16) << 16;
        }
        top = top_of();
    }
    return top;
}

// What a thread works on: 8 channels of a kv head, the same for every block of positions that it goes through.
struct Unit {
    int h, w;  // head, dword of the row
    bool there, is_v;
};
__device__ __forceinline__ Unit unit_of(const Cache4 &c, Divisor by_row)
{
    const int words = 4 * c.NG, n = c.H * words;
    int i = (int)(blockIdx.y * kRowThreads + threadIdx.x);
    Unit u;
    u.is_v = i >= n;
    i -= u.is_v ? n : 0;
    u.h = divided(i, by_row);
    u.w = i - u.h * words;
    u.there = u.h < c.H;
    return u;
}

// The sequence of this workgroup and which of its blocks of four positions is the first to take.
__device__ __forceinline__ bool place_of(const Cache4Seqs &b, const Cache4Flat &flat, int &seq, int &turn)
{
    seq = blockIdx.z;
    turn = blockIdx.x;
    if (flat.on) {
        const int place = (int)(blockIdx.x + gridDim.x * blockIdx.z);
        seq = cache4_seq_at(b, flat, place);
        turn = seq < 0 ? -1 : place - cache4_first(b, flat, seq);
    }
    return turn >= 0;  // starts that do not ascend have no places
}

// The page of the block of four positions that begins at pos (0 or above), or -1: a page holds whole blocks.
__device__ __forceinline__ int page_of(const Cache4 &c, const Cache4Seqs &b, int seq, int pos)
{
    const int page = const_ints(b.table)[(int64_t)seq * b.pitch + (pos >> c.page_shift)];
    return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

// V's dwords of four tokens in the order of its layout, and back (the same exchange): whole, by halves or by bytes.
__device__ __forceinline__ uint4v interleaved(uint4v x, int bytes)
{
    const auto perm = [](uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); };
    if (bytes == 4)
        return x;
    if (bytes == 2)  // run r: halves r of the four
        return uint4v{perm(x[1], x[0], 0x05040100u), perm(x[3], x[2], 0x05040100u), perm(x[1], x[0], 0x07060302u), perm(x[3], x[2], 0x07060302u)};
    const uint32_t a = perm(x[1], x[0], 0x05010400u), b = perm(x[1], x[0], 0x07030602u);  // bytes 0 0 1 1, 2 2 3 3 of two
    const uint32_t d = perm(x[3], x[2], 0x05010400u), e = perm(x[3], x[2], 0x07030602u);
    return uint4v{perm(d, a, 0x05040100u), perm(d, a, 0x07060302u), perm(e, b, 0x05040100u), perm(e, b, 0x07060302u)};
}
__device__ __forceinline__ uint4v separated(uint4v y, int bytes)
{
    if (bytes != 2)
        return interleaved(y, bytes);  // a transposition of 4 x 4 bytes
    const auto perm = [](uint32_t hi, uint32_t lo, uint32_t sel) { return __builtin_amdgcn_perm(hi, lo, sel); };
    return uint4v{perm(y[2], y[0], 0x05040100u), perm(y[2], y[0], 0x07060302u), perm(y[3], y[1], 0x05040100u), perm(y[3], y[1], 0x07060302u)};
}

// 8 channels as a dword of codes and the group's scale (a byte, or step and minimum).
template <int kFormat, bool kBf16>
__device__ __forceinline__ uint2 quantised(uint4v bits, int n)  // n: how many of them there are, others are zeros
{
    const uint32_t top = cleaned<kBf16>(bits);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        x[e] = widened<kBf16>((bits[e / 2] >> (16 * (e & 1))) & 0xffffu);
    uint32_t code = 0;
    if (kFormat == HQMQ_CACHE4_FLOAT) {
        const float most = group_max(widened<kBf16>(top));
        // 7 / 4 has the fraction bits 0x600000: an exponent more for anything above
        const int exponent = min(max((int)((__float_as_uint(most) + 0x1fffffu) >> 23) - 2, 127 - 23), 127 + 13);
        const float unit = e8m0((uint32_t)exponent);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0], x[1], unit, 0);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2], x[3], unit, 1);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4], x[5], unit, 2);
        code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6], x[7], unit, 3);
        return make_uint2(code, (uint32_t)exponent);
    }
    float high = x[0], low = x[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
        high = fmaxf(high, x[e]);
        low = fminf(low, x[e]);
    }
    if (__builtin_expect(n < 8, 0)) {  // without the zeros past the head's last channel
        high = -1.0e30f, low = 1.0e30f;
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < n) {
                high = fmaxf(high, x[e]);
                low = fminf(low, x[e]);
            }
    }
    high = group_max(high);
    low = -group_max(-low);
    if (low > high)  // channels past the head's only
        low = high = 0.f;
    float fifteenth = (high - low) * (1.f / 15.f);
    asm("" : "+v"(fifteenth));  // rounded to fp32 before fp16: v_fma_mixlo_f16 would round the product once
    const _Float16 s16 = (_Float16)fifteenth, m16 = (_Float16)low;
    const float step = (float)s16, least = (float)m16, inverse = step > 0.f ? __builtin_amdgcn_rcpf(step) : 0.f;
    float r[8], far = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float q = __builtin_amdgcn_fmed3f((x[e] - least) * inverse, 0.f, 15.f);
        r[e] = rintf(q);
        far = fmaxf(far, fabsf(q - r[e]));
    }
    // Two roundings and a reciprocal that is good to one last place put q up to 16 * 4 * 2^-24 off.  Next to the middle of two codes the
    // exact difference d + rest from it decides: the middle has 5 bits and the step 11, and d is within a factor of two of their product.
    if (far > 0.5f - 1.0e-5f) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float d = x[e] - least, back = d - x[e], rest = (x[e] - (d - back)) - (least + back);
            const float lower = floorf(d * inverse), over = (d - (lower + 0.5f) * step) + rest;
            const bool up = over > 0.f || (over == 0.f && ((int)lower & 1));
            r[e] = step > 0.f ? __builtin_amdgcn_fmed3f(lower + (up ? 1.f : 0.f), 0.f, 15.f) : 0.f;
        }
    }
    // four codes as one number, which fp32 holds, and both of these as integers
    const float first = fmaf(4096.f, r[3], fmaf(256.f, r[2], fmaf(16.f, r[1], r[0])));
    const float second = fmaf(4096.f, r[7], fmaf(256.f, r[6], fmaf(16.f, r[5], r[4])));
    code = (uint32_t)second << 16 | (uint32_t)first;
    if (__builtin_expect(n < 8, 0))
        code &= (1u << (4 * max(n, 0))) - 1u;
    return make_uint2(code, __builtin_bit_cast(uint32_t, cache4_h2{s16, m16}));
}

// And back, in the rows' type.
template <int kFormat, bool kBf16>
__device__ __forceinline__ uint4v values(uint32_t code, uint32_t scale)
{
    cache4_h2 y[4];
    if (kFormat == HQMQ_CACHE4_FLOAT) {
        const float unit = e8m0(scale);
        y[0] = e2m1_pair<0>(code, unit);
        y[1] = e2m1_pair<1>(code, unit);
        y[2] = e2m1_pair<2>(code, unit);
        y[3] = e2m1_pair<3>(code, unit);
    } else {
        const cache4_h2 sm = __builtin_bit_cast(cache4_h2, scale), ss = {sm[0], sm[0]}, mm = {sm[1], sm[1]};
        const uint32_t even = code & 0x0f0f0f0fu, odd = code >> 4 & 0x0f0f0f0fu;
        const uint32_t lo = __builtin_amdgcn_perm(odd, even, 0x05010400u), hi = __builtin_amdgcn_perm(odd, even, 0x07030602u);  // a code a byte
        y[0] = int4_pair<false>(lo, ss, mm);
        y[1] = int4_pair<true>(lo, ss, mm);
        y[2] = int4_pair<false>(hi, ss, mm);
        y[3] = int4_pair<true>(hi, ss, mm);
    }
    uint4v bits;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (kBf16) {
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            bits[e] = __builtin_bit_cast(uint32_t, b2{(__bf16)(float)y[e][0], (__bf16)(float)y[e][1]});
        } else {
            bits[e] = __builtin_bit_cast(uint32_t, y[e]);
        }
    }
    return bits;
}

}  // namespace

template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void k_cache4_write(Cache4 c, Cache4Seqs b, Cache4Rows k, Cache4Rows v, Divisor by_row, Cache4Flat flat)
{
    typedef std::conditional_t<kFormat == HQMQ_CACHE4_FLOAT, uint8_t, uint32_t> Scale;
    int seq, turn;
    if (!place_of(b, flat, seq, turn))
        return;
    const Cache4Seq s = cache4_seq(b, c.page_shift, seq);
    const Unit u = unit_of(c, by_row);
    const Cache4Rows rows = u.is_v ? v : k;
    uint8_t *const codes = u.is_v ? c.v_codes : c.k_codes;
    Scale *const scales = reinterpret_cast<Scale *>(u.is_v ? c.v_scales : c.k_scales);
    const int ch = 8 * u.w, row_bytes = 16 * c.NG, n_ch = min(max(c.D - ch, 0), 8);
    const int tail = c.D & 7;
    const bool short_head = c.D < 8, last = n_ch > 0 && n_ch < 8;
    const uint16_t *const src = rows.data + u.h * rows.head + (last && !short_head ? c.D - 8 : ch);
    for (int block = (max(s.pos0, 0) >> 2) + turn; 4 * (int64_t)block < s.length && s.n > 0; block += flat.on ? kPastAll : (int)gridDim.x) {
        const int pos = 4 * block, first = max(s.pos0 - pos, 0), end = min(s.length - pos, 4);  // the block's tokens first .. end - 1
        const int page = page_of(c, b, seq, pos);
        if (page < 0)  // uniform
            continue;
        uint4v bits[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            bits[t] = uint4v{0u, 0u, 0u, 0u};
            if (t >= first && t < end && u.there && n_ch > 0 && !short_head) {
                const uint16_t *at = src + (int64_t)(s.first_row + (pos + t - s.pos0)) * rows.row;
                bits[t] = load8(at);
            }
        }
        if (tail) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (!short_head)
                    bits[t] = last ? last_of(bits[t], tail) : bits[t];
                else if (t >= first && t < end && u.there && n_ch > 0)
                    bits[t] = load_some(src + (int64_t)(s.first_row + (pos + t - s.pos0)) * rows.row, tail);
        }
        uint4v code, scale;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint2 y = quantised<kFormat, kBf16>(bits[t], n_ch);
            code[t] = y.x;
            scale[t] = y.y;
        }
        if (!u.there)
            continue;
        const int slot = pos & ((1 << c.page_shift) - 1);
        const int64_t row0 = (((int64_t)page * c.H + u.h) << c.page_shift) + slot;  // the block's first token
        const int group = u.w >> 2;
        const bool leads = (u.w & 3) == 0;  // of its group
        if (!u.is_v) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t >= first && t < end) {
                    *reinterpret_cast<uint32_t *>(codes + (row0 + t) * row_bytes + 4 * u.w) = code[t];
                    if (leads)
                        scales[(row0 + t) * c.NG + group] = (Scale)scale[t];
                }
            continue;
        }
        const Cache4Place p = cache4_v_place(c.NG, u.w, 0);
        uint8_t *const at = codes + row0 * row_bytes + p.at;
        Scale *const scale_at = scales + row0 * c.NG + 4 * group;
        if (end - first == 4) {
            *reinterpret_cast<uint4v *>(at) = interleaved(code, p.bytes);
            if (leads) {
                if (kFormat == HQMQ_CACHE4_FLOAT)
                    *reinterpret_cast<uint32_t *>(scale_at) = scale[0] | scale[1] << 8 | scale[2] << 16 | scale[3] << 24;
                else
                    *reinterpret_cast<uint4v *>(scale_at) = scale;
            }
            continue;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t < first || t >= end)
                continue;
            if (p.bytes == 4) {
                *reinterpret_cast<uint32_t *>(at + 4 * t) = code[t];
            } else if (p.bytes == 2) {
                *reinterpret_cast<uint16_t *>(at + 2 * t) = (uint16_t)code[t];
                *reinterpret_cast<uint16_t *>(at + 2 * t + 8) = (uint16_t)(code[t] >> 16);
            } else {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    at[t + 4 * r] = (uint8_t)(code[t] >> (8 * r));
            }
            if (leads)
                scale_at[t] = (Scale)scale[t];
        }
    }
}

template <int kFormat, bool kBf16>
__global__ __launch_bounds__(kRowThreads) void k_cache4_read(Cache4 c, Cache4Seqs b, Cache4Rows k, Cache4Rows v, Divisor by_row, Cache4Flat flat)
{
    typedef std::conditional_t<kFormat == HQMQ_CACHE4_FLOAT, uint8_t, uint32_t> Scale;
    int seq, turn;
    if (!place_of(b, flat, seq, turn))
        return;
    const Cache4Seq s = cache4_seq(b, c.page_shift, seq);
    const Unit u = unit_of(c, by_row);
    const Cache4Rows rows = u.is_v ? v : k;
    const uint8_t *const codes = u.is_v ? c.v_codes : c.k_codes;
    const Scale *const scales = reinterpret_cast<const Scale *>(u.is_v ? c.v_scales : c.k_scales);
    const int ch = 8 * u.w, row_bytes = 16 * c.NG;
    if (!u.there || ch >= c.D)
        return;
    uint16_t *const dst = rows.data + u.h * rows.head + ch;
    for (int block = (s.pos0 >> 2) + turn; 4 * (int64_t)block < s.length; block += flat.on ? kPastAll : (int)gridDim.x) {
        const int pos = 4 * block, first = max(s.pos0 - pos, 0), end = min(s.length - pos, 4);
        const int page = pos >= 0 ? page_of(c, b, seq, pos) : -1;
        uint4v code = uint4v{0u, 0u, 0u, 0u}, scale = code;
        if (page >= 0) {  // uniform; all of the block's four tokens lie in the cache
            const int slot = pos & ((1 << c.page_shift) - 1);
            const int64_t row0 = (((int64_t)page * c.H + u.h) << c.page_shift) + slot;
            if (!u.is_v) {
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    code[t] = *reinterpret_cast<const uint32_t *>(codes + (row0 + t) * row_bytes + 4 * u.w);
                    scale[t] = scales[(row0 + t) * c.NG + (u.w >> 2)];
                }
            } else {
                const Cache4Place p = cache4_v_place(c.NG, u.w, 0);
                code = separated(*reinterpret_cast<const uint4v *>(codes + row0 * row_bytes + p.at), p.bytes);
                const Scale *const scale_at = scales + row0 * c.NG + 4 * (u.w >> 2);
                if (kFormat == HQMQ_CACHE4_FLOAT) {
                    const uint32_t y = *reinterpret_cast<const uint32_t *>(scale_at);
                    scale = uint4v{y & 0xffu, y >> 8 & 0xffu, y >> 16 & 0xffu, y >> 24};
                } else {
                    scale = *reinterpret_cast<const uint4v *>(scale_at);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            if (t < first || t >= end)
                continue;
            uint4v bits = uint4v{0u, 0u, 0u, 0u};
            if (page >= 0)
                bits = values<kFormat, kBf16>(code[t], scale[t]);
            uint16_t *const at = dst + (int64_t)(s.first_row + (pos + t - s.pos0)) * rows.row;
            if (ch + 8 <= c.D)
                store8(at, bits);
            else
                store_some(at, bits, c.D & 7);
        }
    }
}

namespace {

// Blocks of four positions: as many as the largest sequence needs, wherever in one of them its first position lies; beyond
// kMostGroups workgroups in all they take turns.  Where that would leave most of many workgroups without rows, places along all rows
// (2048 rows among 63 single ones, 8 heads x 128: 12.9 us without, 5.4 with; among 255 41 and 6).
dim3 rows_grid(const Cache4 &c, const Cache4Seqs &b, int max_rows, Cache4Flat &flat)
{
    const int64_t per_block = ((int64_t)2 * c.H * 4 * c.NG + kRowThreads - 1) / kRowThreads;
    const int64_t blocks = max_rows == 1 ? 1 : (max_rows - 1) / 4 + 2, room = kMostGroups / (per_block * b.n_seqs);
    flat = Cache4Flat{0, 1, 2, 2};
    const int64_t places = cache4_places(flat, b.n_rows, b.n_seqs);
    if (b.starts && b.n_seqs > 1 && blocks * b.n_seqs > kFewGroups && 2 * blocks * b.n_seqs > 3 * places) {
        flat.on = 1;
        const int64_t z = (places + (1 << 22) - 1) >> 22;
        return dim3((unsigned)((places + z - 1) / z), (unsigned)per_block, (unsigned)z);
    }
    return dim3((unsigned)(blocks < room ? blocks : room < 1 ? 1 : room), (unsigned)per_block, (unsigned)b.n_seqs);
}

}  // namespace

template <int kFormat>
static const void *rows_kernel(bool write, bool bf16)
{
    if (write)
        return bf16 ? reinterpret_cast<const void *>(&k_cache4_write<kFormat, true>) : reinterpret_cast<const void *>(&k_cache4_write<kFormat, false>);
    return bf16 ? reinterpret_cast<const void *>(&k_cache4_read<kFormat, true>) : reinterpret_cast<const void *>(&k_cache4_read<kFormat, false>);
}

hipError_t launch_cache4_rows(bool write, const Cache4 &c, const Cache4Seqs &b, int max_rows, bool bf16, const Cache4Rows &k, const Cache4Rows &v,
                              hipStream_t stream)
{
    Cache4 cc = c;
    Cache4Seqs bc = b;
    Cache4Rows kc = k, vc = v;
    Divisor by_row = make_divisor((uint32_t)(4 * c.NG));
    Cache4Flat flat;
    const dim3 grid = rows_grid(c, b, max_rows, flat);
    void *args[] = {&cc, &bc, &kc, &vc, &by_row, &flat};
    const void *kernel = c.format == HQMQ_CACHE4_FLOAT ? rows_kernel<HQMQ_CACHE4_FLOAT>(write, bf16) : rows_kernel<HQMQ_CACHE4_INT>(write, bf16);
    return hipLaunchKernel(kernel, grid, dim3(kRowThreads), args, 0, stream);
}

}  // namespace hqmq
