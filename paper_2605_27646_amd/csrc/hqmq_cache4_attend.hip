// Causal attention over a paged cache held in 4 bits (include/hqmq_cache4.h, hqmq_cache4_attend).
//
// A workgroup takes 16, 32 or 64 query rows of a kv head (row r = j G + g is query head g of the sequence's row j) and a share of
// the tokens; its waves take steps of 32 tokens in turn and join their sums in LDS at the end.  The codes go from memory to
// the operands of v_mfma_f32_16x16x32_f16 without crossing lanes, by three choices of order:
//   S^T = K Q^T   lane (token l % 16, quarter l / 16) reads a quarter of a key's codes, a run of 8 NG channels, and the query operand
//                 has the same channels in the same places;
//   P^T           the scores come as lane (query l % 16, tokens 4 (l / 16) .. + 3) of each 16 tokens, which two of together are the
//                 eight tokens of that lane in the operand P^T as they stand;
//   O^T = V^T P^T lane (run l % 16, l / 16) reads the codes of those eight tokens for a run of 8 (4, 2) channels, two blocks of four
//                 tokens of the V layout, and product e takes channel e of every run.
// A query's maximum and sum belong to one column, so every factor is one per lane.
//
// Bound by memory for generation steps of many long sequences (64 of up to 8192 tokens, 8 heads x 128: 69 to 73 us, 301 MB at 4.2 to 4.4 TB/s,
// vector instructions issue for a third of the time), by a workgroup's start and the join for short ones (130 tokens 6 us, of which
// one step is 1), and by issue for prompts (1024 tokens of two sequences behind 15000, bf16: 437 us, 1.19 PFLOP/s, 425 to 455 over inputs
// and machines; of the kernel's 428 us in a trace vector instructions are 70 % and matrix instructions 48 %; of the former 37 % are exponentials,
// 33 % the reconstruction for 64 rows).  With fp16 rows the second product runs twice: 629 us.
//
// Registers: 64 rows of 128 channels and 32 of 256 need all 256, and 8 to 25 more that are kept in scratch (28 to 72 bytes a lane).  A step
// reads 2 to 9 words of them back and writes 2 at most, beside its 64 to 128 matrix instructions.
#include <algorithm>
#include <type_traits>

#include "hqmq_cache4_device.h"

namespace hqmq {

namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef cache4_h2 half2_t;
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

constexpr int kStep = 32;             // tokens that a wave takes at a time
constexpr int kMergeThreads = 256;
constexpr float kNothing = -3.0e38f;  // "no token seen yet": less than any exponent, finite, so that of two of them the difference is 0
constexpr float kTop4 = 7.f;          // weights are taken relative to 2^-kTop4 of the largest score,
constexpr float kRise4 = 15.f;        // and relative to a newer one once they would pass 2^kRise4 (fp16 ends at 2^16)
constexpr int kFarOnly = 0x7fffffff;
constexpr float kMost4 = 0x1p127f;    // exponents and factors end here
constexpr float kLog2e4 = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Waves of a workgroup.  For up to 16 rows eight, of which two workgroups fill a compute unit's registers.
constexpr int attend_waves(int blocks) { return blocks == 1 ? 8 : 4; }

// Blocks of rows whose sums are joined at a time: two workgroups fit a compute unit's LDS, heads of more than 128 channels one of eight waves.
constexpr int attend_pass(int NG, int blocks) { return blocks == 1 || NG > 4 ? 1 : 2; }
// A row's pitch there: 4 banks past a multiple of all, so that the 16 rows of a wave's store go to all banks once.
constexpr int attend_pitch(int NG) { return 32 * NG + 4 + 32 * (NG & 1); }

constexpr size_t attend_shared_bytes(int NG, int blocks)  // queries, then the waves' sums of the rows that are joined
{
    const size_t queries = (size_t)blocks * NG * 64 * 16;
    const size_t join = (size_t)attend_waves(blocks) * attend_pass(NG, blocks) * 16 * attend_pitch(NG) * 4;
    return queries > join ? queries : join;
}
constexpr size_t attend_lds_bytes(int NG, int blocks)
{
    return attend_shared_bytes(NG, blocks) + (size_t)blocks * 16 * (8 + 12 * attend_waves(blocks) + 8);
}

// Maximum or sum over the four lanes that hold a query's column.
__device__ __forceinline__ float column_max(float x)
{
    auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ uint32_t column_max(uint32_t x)
{
    auto y = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    x = max((uint32_t)y[0], (uint32_t)y[1]);
    y = __builtin_amdgcn_permlane32_swap(x, x, false, false);
    return max((uint32_t)y[0], (uint32_t)y[1]);
}
__device__ __forceinline__ float column_sum(float x)
{
    auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// n words from an address that is a multiple of 4 n bytes from one of 16.
#define HQMQ_GLOBAL __attribute__((address_space(1)))
typedef const HQMQ_GLOBAL uint8_t *Bytes;  // of the cache: an address that the compiler knows to be in memory, though it is made opaque
template <int n>
struct Words {
    uint32_t w[n];
};
template <int n>
__device__ __forceinline__ Words<n> load_words(Bytes p)
{
    typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
    Words<n> out;
    if constexpr (n % 4 == 0) {
#pragma unroll
        for (int i = 0; i < n / 4; ++i) {
            const uint4v y = reinterpret_cast<const HQMQ_GLOBAL uint4v *>(p)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                out.w[4 * i + e] = y[e];
        }
    } else if constexpr (n % 2 == 0) {
#pragma unroll
        for (int i = 0; i < n / 2; ++i) {
            const uint2v y = reinterpret_cast<const HQMQ_GLOBAL uint2v *>(p)[i];
            out.w[2 * i] = y[0];
            out.w[2 * i + 1] = y[1];
        }
    } else {
#pragma unroll
        for (int i = 0; i < n; ++i)
            out.w[i] = reinterpret_cast<const HQMQ_GLOBAL uint32_t *>(p)[i];
    }
    return out;
}

// The parts of the V layout for NG groups.
template <int NG>
struct Parts {
    static constexpr int whole = NG / 4, n = whole + (NG / 2 & 1) + (NG & 1);
    // of part p: groups, words of a lane's 4 tokens before it, channels of a lane before it
    static constexpr int groups(int p) { return p < whole ? 4 : p == whole && (NG & 2) ? 2 : 1; }
    static constexpr int before(int p) { return p <= whole ? 4 * p : 4 * whole + 2; }
};

// What a lane holds of 16 tokens, as loaded.
template <int kFormat, int NG>
struct KStage {
    static constexpr int kScales = NG == 1 || NG == 2 || NG == 4 ? 1 : 2;
    // a byte stays one until it is used: widening it where it is loaded would wait for it
    typedef std::conditional_t<kFormat == HQMQ_CACHE4_FLOAT, uint8_t, uint32_t> Scale;
    Words<NG> code;
    Scale scale[kScales];
};
template <int kFormat, int NG>
struct VStage {
    static constexpr int kWords = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    Words<NG> code;
    Words<kWords> scale[Parts<NG>::n];
};

// 16 tokens of a head in one page: where they begin in each of the cache's buffers, one address for the wave.
struct Tile {
    Bytes k_codes, k_scales, v_codes, v_scales;
};
// head: the first token of the head in page 0
template <int kFormat, int NG>
__device__ __forceinline__ Tile tile_at(const Tile &head, const Cache4 &c, int page, int slot)
{
    const uint64_t codes = ((uint64_t)(uint32_t)page * (uint32_t)(c.H * NG) << (c.page_shift + 4)) + (uint32_t)(16 * NG * slot);
    const uint64_t scales = codes >> (kFormat == HQMQ_CACHE4_FLOAT ? 4 : 2);
    Tile t = {head.k_codes + codes, head.k_scales + scales, head.v_codes + codes, head.v_scales + scales};
    asm("" : "+s"(t.k_codes), "+s"(t.k_scales), "+s"(t.v_codes), "+s"(t.v_scales));  // scalar bases: a lane's share is a 32-bit offset
    return t;
}

// A lane's places behind a tile's addresses.
template <int kFormat, int NG>
struct Places {
    static constexpr uint32_t kScale = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    using P = Parts<NG>;
    uint32_t k_code, k_scale[KStage<kFormat, NG>::kScales], v_code[P::n], v_scale[P::n];
    __device__ __forceinline__ explicit Places(uint32_t lane)
    {
        const uint32_t token = lane & 15, run = token, quarter = lane >> 4;
        k_code = token * (16 * NG) + 4 * NG * quarter;
        k_scale[0] = kScale * (token * NG + (quarter * NG >> 2));
        k_scale[KStage<kFormat, NG>::kScales - 1] = kScale * (token * NG + ((quarter * NG + (KStage<kFormat, NG>::kScales > 1 ? NG - 1 : 0)) >> 2));
#pragma unroll
        for (int p = 0; p < P::n; ++p) {
            v_code[p] = quarter * (64 * NG) + 4 * P::groups(p) * run + 64 * P::before(p);
            v_scale[p] = kScale * (4 * (quarter * NG + P::before(p) + (run * P::groups(p) >> 4)));
        }
    }
    // Widening an offset where it is used, in every step, makes it an offset to a scalar base; kept as 64 bits it would be added to each.
    __device__ __forceinline__ void keep_narrow_k()
    {
        asm volatile("" : "+v"(k_code));
#pragma unroll
        for (int i = 0; i < KStage<kFormat, NG>::kScales; ++i)
            asm volatile("" : "+v"(k_scale[i]));
    }
    __device__ __forceinline__ void keep_narrow_v()
    {
#pragma unroll
        for (int p = 0; p < P::n; ++p) {
            asm volatile("" : "+v"(v_code[p]));
            asm volatile("" : "+v"(v_scale[p]));
        }
    }
};

template <int kFormat, int NG>
__device__ __forceinline__ void load_k(KStage<kFormat, NG> &s, const Tile &tile, const Places<kFormat, NG> &at)
{
    typedef typename KStage<kFormat, NG>::Scale Scale;
    s.code = load_words<NG>(tile.k_codes + at.k_code);
#pragma unroll
    for (int i = 0; i < KStage<kFormat, NG>::kScales; ++i)
        s.scale[i] = *reinterpret_cast<const HQMQ_GLOBAL Scale *>(tile.k_scales + at.k_scale[i]);
}

template <int kFormat, int NG>
__device__ __forceinline__ void load_v(VStage<kFormat, NG> &s, const Tile &tile, const Places<kFormat, NG> &place)
{
    using P = Parts<NG>;
#pragma unroll
    for (int p = 0; p < P::n; ++p) {
        const Bytes at = tile.v_codes + place.v_code[p];
        if (P::groups(p) == 4) {
            const Words<4> w = load_words<4>(at);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s.code.w[(P::before(p) + i) % NG] = w.w[i];
        } else if (P::groups(p) == 2) {
            const Words<2> w = load_words<2>(at);
            s.code.w[P::before(p)] = w.w[0];
            s.code.w[(P::before(p) + 1) % NG] = w.w[1];
        } else {
            s.code.w[P::before(p)] = load_words<1>(at).w[0];
        }
        s.scale[p] = load_words<VStage<kFormat, NG>::kWords>(tile.v_scales + place.v_scale[p]);
    }
}

// Of the lane's four tokens those before `first` and from `end` on become zeros, whatever lies there.
template <int kFormat, int NG>
__device__ __forceinline__ void blank_v(VStage<kFormat, NG> &s, int first, int end)
{
    using P = Parts<NG>;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const bool gone = t < first || t >= end;
#pragma unroll
        for (int p = 0; p < P::n; ++p) {
            const int at = P::before(p);
            if (P::groups(p) == 4)
                s.code.w[(at + t) % NG] = gone ? 0u : s.code.w[(at + t) % NG];
            else if (P::groups(p) == 2)
                s.code.w[(at + t / 2) % NG] &= gone ? (t & 1 ? 0x0000ffffu : 0xffff0000u) : 0xffffffffu;
            else
                s.code.w[at] &= gone ? ~(0xffu << (8 * t)) : 0xffffffffu;
            if (kFormat == HQMQ_CACHE4_FLOAT)
                s.scale[p].w[0] = gone ? (s.scale[p].w[0] & ~(0xffu << (8 * t))) | 127u << (8 * t) : s.scale[p].w[0];
            else
                s.scale[p].w[t % VStage<kFormat, NG>::kWords] = gone ? 0u : s.scale[p].w[t % VStage<kFormat, NG>::kWords];
        }
    }
}

// The operand of channels 8 w .. 8 w + 7 of the lane's run, in their order (float) or as 0 2 4 6 1 3 5 7 (int).
template <int kFormat, int NG>
__device__ __forceinline__ half8_t k_operand(const KStage<kFormat, NG> &s, int w, int lane)
{
    const int quarter = lane >> 4;
    auto scale = s.scale[0];
    if (KStage<kFormat, NG>::kScales > 1)
        scale = (quarter * NG + w) >> 2 == quarter * NG >> 2 ? scale : s.scale[KStage<kFormat, NG>::kScales - 1];
    const uint32_t code = s.code.w[w];
    half2_t y[4];
    if (kFormat == HQMQ_CACHE4_FLOAT) {
        const float unit = e8m0(scale);
        y[0] = e2m1_pair<0>(code, unit);
        y[1] = e2m1_pair<1>(code, unit);
        y[2] = e2m1_pair<2>(code, unit);
        y[3] = e2m1_pair<3>(code, unit);
    } else {
        const half2_t sm = __builtin_bit_cast(half2_t, (uint32_t)scale), ss = {sm[0], sm[0]}, mm = {sm[1], sm[1]};
        const uint32_t even = code & 0x0f0f0f0fu, odd = code >> 4 & 0x0f0f0f0fu;
        y[0] = int4_pair<false>(even, ss, mm);
        y[1] = int4_pair<true>(even, ss, mm);
        y[2] = int4_pair<false>(odd, ss, mm);
        y[3] = int4_pair<true>(odd, ss, mm);
    }
    return __builtin_bit_cast(half8_t, uint4v{__builtin_bit_cast(uint32_t, y[0]), __builtin_bit_cast(uint32_t, y[1]),
                                              __builtin_bit_cast(uint32_t, y[2]), __builtin_bit_cast(uint32_t, y[3])});
}

// Channels 2 kByte and 2 kByte + 1 of the lane's run in part kPart, the eight tokens of two stages each.
template <int kFormat, int NG, int kPart, int kByte>
__device__ __forceinline__ void v_operands(const VStage<kFormat, NG> (&s)[2], half8_t &even, half8_t &odd)
{
    using P = Parts<NG>;
    constexpr int at = P::before(kPart), groups = P::groups(kPart);
    uint32_t e[4], o[4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const uint32_t *code = s[x].code.w + at;
        if (kFormat == HQMQ_CACHE4_FLOAT) {
            const uint32_t scales = s[x].scale[kPart].w[0];
            uint32_t y[4];
            const auto pair = [&](auto token) {
                constexpr int t = decltype(token)::value;
                constexpr int word = groups == 4 ? t : groups == 2 ? t / 2 : 0, byte = groups == 4 ? kByte : groups == 2 ? kByte + 2 * (t & 1) : t;
                y[t] = __builtin_bit_cast(uint32_t, e2m1_pair<byte>(code[word], e8m0((scales >> (8 * t)) & 0xffu)));
            };
            pair(std::integral_constant<int, 0>{});
            pair(std::integral_constant<int, 1>{});
            pair(std::integral_constant<int, 2>{});
            pair(std::integral_constant<int, 3>{});
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[2 * x + i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], 0x05040100u);
                o[2 * x + i] = __builtin_amdgcn_perm(y[2 * i + 1], y[2 * i], 0x07060302u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t a = s[x].scale[kPart].w[(2 * i) % VStage<kFormat, NG>::kWords], b = s[x].scale[kPart].w[(2 * i + 1) % VStage<kFormat, NG>::kWords];
                const half2_t step = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(b, a, 0x05040100u));
                const half2_t least = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(b, a, 0x07060302u));
                uint32_t both;  // bytes of the tokens 2 i and 2 i + 1 side by side
                if (groups == 4)  // of two pairs of channels, and this one's half
                    both = __builtin_amdgcn_perm(code[(2 * i + 1) % NG], code[(2 * i) % NG], kByte < 2 ? 0x05010400u : 0x07030602u);
                else if (groups == 2)
                    both = __builtin_amdgcn_perm(0u, code[i % NG], 0x03010200u);
                else  // of both pairs of tokens
                    both = code[0];
                const uint32_t low = both & 0x0f0f0f0fu, high = both >> 4 & 0x0f0f0f0fu;
                if (groups > 1 ? kByte & 1 : i) {
                    e[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair<true>(low, step, least));
                    o[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair<true>(high, step, least));
                } else {
                    e[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair<false>(low, step, least));
                    o[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair<false>(high, step, least));
                }
            }
        }
    }
    even = __builtin_bit_cast(half8_t, uint4v{e[0], e[1], e[2], e[3]});
    odd = __builtin_bit_cast(half8_t, uint4v{o[0], o[1], o[2], o[3]});
}

template <int i, int n, typename F>
__device__ __forceinline__ void unrolled(F &&f)
{
    if constexpr (i < n) {
        f(std::integral_constant<int, i>{});
        unrolled<i + 1, n>(f);
    }
}

// Waves of a SIMD that the registers are to leave room for.
constexpr int attend_occupancy(int NG, int blocks) { return blocks == 1 && NG <= 4 ? 4 : 2; }

}  // namespace

// Four channels of a result, or the n of them that there are (any number).
template <bool kBf16>
__device__ __forceinline__ void store_four(uint16_t *dst, f4 y, int n)
{
    uint32_t bits[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        if (kBf16) {
            typedef __bf16 b2 __attribute__((ext_vector_type(2)));
            bits[e] = __builtin_bit_cast(uint32_t, b2{(__bf16)y[2 * e], (__bf16)y[2 * e + 1]});
        } else {
            bits[e] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)y[2 * e], (_Float16)y[2 * e + 1]});
        }
    }
    if (n >= 4) {
        struct __attribute__((packed, aligned(2))) Four {
            uint64_t bits;
        };
        reinterpret_cast<Four *>(dst)->bits = (uint64_t)bits[1] << 32 | bits[0];
    } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < n)
                dst[e] = (uint16_t)(bits[e / 2] >> (16 * (e & 1)));
    }
}
// The logarithm of a sum of weights l relative to 2^m.
__device__ __forceinline__ float lse_of(float m, float l) { return l > 0.f ? kLn2 * (m + __builtin_amdgcn_logf(l)) : -__builtin_inff(); }

template <int kFormat, int NG, int kBlocks, bool kBf16>
__global__ __launch_bounds__(64 * attend_waves(kBlocks), attend_occupancy(NG, kBlocks)) void k_cache4_attend(Cache4Attend a)
{
    using P = Parts<NG>;
    constexpr int kRows = 16 * kBlocks, kChannels = 2 * NG;  // of a lane
    constexpr int kWaves = attend_waves(kBlocks), kPitch = attend_pitch(NG);
    static_assert(kBlocks <= kWaves, "a wave stages a block of queries");
    // fp16 rows take weights in two parts.  bf16 rows take the first alone, 11 bits for results of 8: it moves a tenth of the results to the
    // neighbouring bf16 number, the error against 64 bits is 0.5 to 0.7 % above that of rounding alone, and two parts take half as much matrix
    // work again (the chunk above: 629 us with fp16 rows).  The sum stays that of the fp32 weights, because lse has 24 bits.
    constexpr bool kFine = !kBf16;
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr size_t kShared = attend_shared_bytes(NG, kBlocks);
    half8_t *const queries = reinterpret_cast<half8_t *>(lds);           // [kBlocks][NG][lane]
    float *const join = reinterpret_cast<float *>(lds);                  // [kWaves][kPass][16][kPitch], when the queries are done with
    float *const factor = reinterpret_cast<float *>(lds + kShared);      // [kRows]: from products to exponents of 2
    int *const position = reinterpret_cast<int *>(factor + kRows);       // [kRows]: -1 - 2^30 and less: no row
    float *const stats = reinterpret_cast<float *>(position + kRows);    // [kWaves][kRows][2]
    float *const row_factors = stats + kWaves * kRows * 2;               // [kRows][kWaves]
    int64_t *const row_at_lds = reinterpret_cast<int64_t *>(row_factors + kWaves * kRows);  // [kRows]

    const int tid = threadIdx.x;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Cache4 &c = a.c;
    const int h = blockIdx.x, rest = divided((int)blockIdx.y, a.by_splits), split = (int)blockIdx.y - rest * a.n_splits;
    // the longest first: a causal prompt's last rows see the most
    int seq = blockIdx.z, first_tile = a.n_tiles - 1 - rest;
    if (a.flat.on) {
        const int place = a.n_tiles - 1 - (rest + (int)(blockIdx.z * gridDim.y));  // z: only where nothing is split
        seq = place < 0 ? -1 : cache4_seq_at(a.b, a.flat, place);
        first_tile = seq < 0 ? -1 : place - cache4_first(a.b, a.flat, seq);
        if (first_tile < 0)  // starts that do not ascend have no tiles
            return;
    }
    const int page_mask = (1 << c.page_shift) - 1;
    const uint64_t head_rows = (uint64_t)h << c.page_shift;
    constexpr int kScale = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    const Tile head = {(Bytes)c.k_codes + head_rows * (16 * NG), (Bytes)c.k_scales + head_rows * (kScale * NG),
                       (Bytes)c.v_codes + head_rows * (16 * NG), (Bytes)c.v_scales + head_rows * (kScale * NG)};
    const ConstInts table = const_ints(a.b.table + (int64_t)seq * a.b.pitch);
    const Cache4Seq s = cache4_seq(a.b, c.page_shift, seq);
    const int n_rows = s.n * a.G, n_heads = c.H * a.G;

    for (int tile = first_tile; (int64_t)tile * kRows < n_rows; tile += a.n_tiles) {  // a second one only with fewer places than tiles
        const int r0 = tile * kRows;
        int lane = tid & 63;
        asm volatile("" : "+v"(lane));  // what is made of it stays inside a tile's turn, of which there is one as a rule
        const int col = lane & 15, quarter = lane >> 4;
        // ---- what the rows see -----------------------------------------------------------------------------------------
        const int j_first = divided(r0, a.by_G), j_last = min(divided(r0 + kRows - 1, a.by_G), s.n - 1);
        const int end = s.pos0 + j_last + 1, all_end = s.pos0 + j_first + 1;  // all_end: every row sees what is before it,
        const int begin = a.window ? max(0, s.pos0 + j_first + 1 - a.window) & ~(kStep - 1) : 0;
        int all_begin = a.window ? s.pos0 + j_last + 1 - a.window : 0;  // and from here on
        // Without a window the first pages are looked up before the length is there: no length puts them past the table.
        const int64_t share = (int64_t)begin + (int64_t)split * a.split_tokens;
        const int from = (int)min(share, (int64_t)(a.b.pitch << c.page_shift));
        int page[2];
        const auto look_up = [&](int step, int last) {  // pages of a step's two halves; past the share's end: those of its last step
            const int token = min(from + kStep * step, last);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                page[x] = table[min((token + 16 * x) >> c.page_shift, a.b.pitch - 1)];
        };
        look_up(wave, 0x7fffffdf);
        const int to = split == a.n_splits - 1 ? end : (int)min(share + a.split_tokens, (int64_t)end);
        const int n_steps = to > from ? (to - from + kStep - 1) / kStep : 0;
        const int last = from + kStep * max(n_steps - 1, 0);
        KStage<kFormat, NG> ks[2] = {};
        VStage<kFormat, NG> vs[2] = {};
        Places<kFormat, NG> places(lane);
        Tile tiles[2];
        bool bad[2];
        const auto tiles_of = [&](int token) {  // of the pages that were looked up last
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                bad[x] = (uint32_t)page[x] >= (uint32_t)c.n_pages;
                tiles[x] = tile_at<kFormat, NG>(head, c, bad[x] ? 0 : page[x], (token + 16 * x) & page_mask);
            }
        };
        // ---- the wave's block of queries and its first step are on their way together --------------------------------------
        const int query = r0 + 16 * wave + col, query_j = divided(query, a.by_G), first_ch = 8 * NG * quarter;
        const bool there = wave < kBlocks && query < n_rows;
        uint4v bits[NG];
#pragma unroll
        for (int w = 0; w < NG; ++w)
            bits[w] = uint4v{0u, 0u, 0u, 0u};
        if (there) {
            const uint16_t *src = a.q.data + (int64_t)(s.first_row + query_j) * a.q.row + (int64_t)(h * a.G + (query - query_j * a.G)) * a.q.head;
            int D = c.D;
            asm volatile("" : "+s"(D));  // what is compared with it is not kept in registers from tile to tile
            if (__builtin_expect(D % 8 == 0, 1)) {
#pragma unroll
                for (int w = 0; w < NG; ++w)
                    if (first_ch + 8 * w < D)
                        bits[w] = load8(src + (first_ch + 8 * w));
            } else if (NG == 1 && D < 8) {
                if (first_ch == 0)
                    bits[0] = load_some(src, D);
            } else {
#pragma unroll
                for (int w = 0; w < NG; ++w)
                    if (first_ch + 8 * w < D)
                        bits[w] = load8(src + min(first_ch + 8 * w, D - 8));
#pragma unroll
                for (int w = 0; w < NG; ++w)
                    bits[w] = first_ch + 8 * w > D - 8 && first_ch + 8 * w < D ? last_of(bits[w], D & 7) : bits[w];
            }
        }
        if (wave < n_steps) {
            tiles_of(from + kStep * wave);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                load_k(ks[x], tiles[x], places);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                load_v(vs[x], tiles[x], places);
            look_up(wave + kWaves, last);
        }
        // ---- queries to LDS, as operands
        if (wave < kBlocks) {
            float f = fabsf(a.scale) * kLog2e4;
            uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;  // a negative scale goes into the queries' signs
            asm volatile("" : "+s"(flip));
            typedef unsigned short us2 __attribute__((ext_vector_type(2)));
            us2 tops = {0, 0};
#pragma unroll
            for (int w = 0; w < NG; ++w)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    tops = __builtin_elementwise_max(tops, __builtin_bit_cast(us2, bits[w][e] & 0x7fff7fffu));
            uint32_t top = max((uint32_t)tops[0], (uint32_t)tops[1]);
            top = column_max(top);
            // A query that holds an infinity or a NaN has no scores: its sums are formed of zeros, and what it gives is NaN.
            const bool lost = top >= (kBf16 ? 0x7f80u : 0x7c00u);
            if (__builtin_expect(lost, 0)) {
                top = 0;
#pragma unroll
                for (int w = 0; w < NG; ++w)
                    bits[w] = uint4v{0u, 0u, 0u, 0u};
            }
            if (kBf16) {
                // A power of two brings the row's largest magnitude to 2^14 .. 2^15, where fp16 has all its bits down to 2^-28 of it.
                const int up = 141 - (int)(top >> 7);
                f = ldexpf(f, -up);
                top = 0x7800u;  // as fp16 from here on
#pragma unroll
                for (int w = 0; w < NG; ++w)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        bits[w][e] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)ldexpf(__uint_as_float(bits[w][e] << 16), up),
                                                                          (_Float16)ldexpf(__uint_as_float(bits[w][e] & 0xffff0000u), up)});
            }
#pragma unroll
            for (int w = 0; w < NG; ++w) {
                uint4v x = bits[w] ^ uint4v{flip, flip, flip, flip};
                if (kFormat == HQMQ_CACHE4_INT)  // channels 0 2 4 6 1 3 5 7
                    x = uint4v{__builtin_amdgcn_perm(x[1], x[0], 0x05040100u), __builtin_amdgcn_perm(x[3], x[2], 0x05040100u),
                               __builtin_amdgcn_perm(x[1], x[0], 0x07060302u), __builtin_amdgcn_perm(x[3], x[2], 0x07060302u)};
                queries[(wave * NG + w) * 64 + lane] = __builtin_bit_cast(half8_t, x);
            }
            if (quarter == 0) {
                // Products stay below 2^40: with a factor as small as the first they all become 0, but minus infinity stays what it is.
                f = fminf(fmaxf(f, 0x1p-120f), kMost4);
                // A fused product differs from the rounded one in a reference by up to half a last place, and where exponents pass 2^27 weights
                // would pass 2^15.  A row that can come there, with keys below 2^16, has the same rounded product in both: its factor is marked.
                factor[16 * wave + col] = f * (float)__builtin_bit_cast(_Float16, (uint16_t)top) > 2048.f / (32 * NG) ? -f : f;
                row_at_lds[16 * wave + col] = lost;
                position[16 * wave + col] = there ? s.pos0 + query_j : -0x7fffffff;
            }
        }
        __syncthreads();
        float scale[kBlocks];
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb)
            scale[nb] = factor[16 * nb + col];
        bool far = false;
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb)
            far |= scale[nb] < 0.f;
        if (__builtin_expect(__any(far), 0)) {
            all_begin = kFarOnly;  // no step is without a look at its products
#pragma unroll
            for (int nb = 0; nb < kBlocks; ++nb)
                scale[nb] = 1.f;
        }

        f4 o[kChannels][kBlocks];
        float ref[kBlocks], sum[kBlocks];
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb) {
            ref[nb] = kNothing;
            sum[nb] = 0.f;
#pragma unroll
            for (int e = 0; e < kChannels; ++e)
                o[e][nb] = f4{0.f, 0.f, 0.f, 0.f};
        }

        for (int step = wave; step < n_steps; step += kWaves) {
            const int token = from + kStep * step;
            const bool bad_now[2] = {bad[0], bad[1]};
            // ---- scores
            int at = lane;
            if (kBlocks * NG > 8)
                asm volatile("" : "+v"(at));  // the operands of many queries are read again, not kept in registers
            // A wave that feeds the matrix cores goes first, so that another's exponentials and conversions fill the time between: 1024 tokens
            // of two prompts 454 us without, 449 in this product, 428 in both; with 32 rows and weights in two parts the second costs 2 %.
            f4 x[2][kBlocks];
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int nb = 0; nb < kBlocks; ++nb)
                    x[i][nb] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < NG; ++w) {
                    const half8_t key = k_operand(ks[i], w, lane);
#pragma unroll
                    for (int nb = 0; nb < kBlocks; ++nb)
                        x[i][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(key, queries[(nb * NG + w) * 64 + at], x[i][nb], 0, 0, 0);
                }
            }
            __builtin_amdgcn_s_setprio(0);
            tiles_of(min(token + kStep * kWaves, last));
            places.keep_narrow_k();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_k(ks[i], tiles[i], places);
            // ---- unseen tokens, and products that are rounded
            if (token + kStep > all_end || token < all_begin || bad_now[0] || bad_now[1]) {
                if (__builtin_expect(all_begin == kFarOnly, 0)) {
#pragma unroll
                    for (int nb = 0; nb < kBlocks; ++nb) {
                        const float f = fabsf(factor[16 * nb + col]);
#pragma unroll
                        for (int i = 0; i < 2; ++i)
#pragma unroll
                            for (int r = 0; r < 4; ++r)
                                x[i][nb][r] = fminf(x[i][nb][r] * f, kMost4);
                    }
                }
#pragma unroll
                for (int nb = 0; nb < kBlocks; ++nb) {
                    const int pos = position[16 * nb + col], low = a.window ? max(pos, -1) + 1 - a.window : 0;
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int r = 0; r < 4; ++r) {
                            const int t = token + 16 * i + 4 * quarter + r;
                            x[i][nb][r] = t <= pos && t >= low && !bad_now[i] ? x[i][nb][r] : -__builtin_inff();
                        }
                }
            }
            // ---- a newer reference for the weights: rare but for a wave's first step
            float top[kBlocks];
            bool rise = false;
#pragma unroll
            for (int nb = 0; nb < kBlocks; ++nb) {
                top[nb] = fmaxf(fmaxf(fmaxf(x[0][nb][0], x[0][nb][1]), fmaxf(x[0][nb][2], x[0][nb][3])),
                                fmaxf(fmaxf(x[1][nb][0], x[1][nb][1]), fmaxf(x[1][nb][2], x[1][nb][3])));
                rise |= fmaf(top[nb], scale[nb], -ref[nb]) > kRise4;
            }
            if (__any(rise)) {
#pragma unroll
                for (int nb = 0; nb < kBlocks; ++nb) {
                    const float newer = fmaxf(ref[nb], column_max(top[nb] * scale[nb]) - kTop4);
                    const float f = __builtin_amdgcn_exp2f(ref[nb] - newer);
                    ref[nb] = newer;
                    sum[nb] *= f;
#pragma unroll
                    for (int e = 0; e < kChannels; ++e)
                        o[e][nb] *= f4{f, f, f, f};
                }
            }
            // ---- weights
            float minus = -1.f;
            asm("" : "+s"(minus));  // a product that the compiler keeps: one instruction takes the fp16 factor as it is
            half8_t hi[kBlocks], lo[kBlocks];
#pragma unroll
            for (int nb = 0; nb < kBlocks; ++nb) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; r += 2) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(x[i][nb][r], scale[nb], -ref[nb]));
                        const float q = __builtin_amdgcn_exp2f(fmaf(x[i][nb][r + 1], scale[nb], -ref[nb]));
                        sum[nb] += p;
                        sum[nb] += q;
                        const half2_t rounded = {(_Float16)p, (_Float16)q};
                        hi[nb][4 * i + r] = rounded[0];
                        hi[nb][4 * i + r + 1] = rounded[1];
                        if (kFine) {
                            const half2_t rest = {(_Float16)fmaf((float)rounded[0], minus, p), (_Float16)fmaf((float)rounded[1], minus, q)};
                            lo[nb][4 * i + r] = rest[0];
                            lo[nb][4 * i + r + 1] = rest[1];
                        }
                    }
            }
            // ---- values: a token that none of the sequence's rows sees may hold anything
            const bool too_early = a.window && token < all_end - a.window;
            if (__builtin_expect(token + kStep > s.length || too_early || bad_now[0] || bad_now[1], 0)) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int base = token + 16 * i + 4 * quarter;
                    blank_v(vs[i], too_early ? all_end - a.window - base : 0, bad_now[i] ? 0 : s.length - base);
                }
            }
            if (kBlocks > 2)
                __builtin_amdgcn_s_setprio(1);
            unrolled<0, P::n>([&](auto part) {
                constexpr int p = decltype(part)::value;
                unrolled<0, P::groups(p)>([&](auto byte) {
                    constexpr int b = decltype(byte)::value;
                    half8_t even, odd;
                    v_operands<kFormat, NG, p, b>(vs, even, odd);
                    constexpr int e = 2 * P::before(p) + 2 * b;
#pragma unroll
                    for (int nb = 0; nb < kBlocks; ++nb) {
                        o[e][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, hi[nb], o[e][nb], 0, 0, 0);
                        o[e + 1][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, hi[nb], o[e + 1][nb], 0, 0, 0);
                    }
                    if (kFine) {
#pragma unroll
                        for (int nb = 0; nb < kBlocks; ++nb) {
                            o[e][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(even, lo[nb], o[e][nb], 0, 0, 0);
                            o[e + 1][nb] = __builtin_amdgcn_mfma_f32_16x16x32_f16(odd, lo[nb], o[e + 1][nb], 0, 0, 0);
                        }
                    }
                });
            });
            if (kBlocks > 2)
                __builtin_amdgcn_s_setprio(0);
            places.keep_narrow_v();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_v(vs[i], tiles[i], places);
            look_up(step + 2 * kWaves, last);
        }

        // ---- the waves' sums joined, kPass blocks of rows at a time -----------------------------------------------------------
        int thread = tid;
        asm volatile("" : "+v"(thread));  // addresses are formed here, not kept in registers through the steps
        const int col_now = thread & 15, quarter_now = (thread & 63) >> 4;
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb) {
            const float total = column_sum(sum[nb]);
            if (quarter_now == 0)
                *reinterpret_cast<float2 *>(stats + (wave * kRows + 16 * nb + col_now) * 2) = make_float2(ref[nb], total);
        }
        __syncthreads();  // the queries are done with
        if (thread < kRows) {  // what a row's channels have in common: the waves' factors, and where they go; -1: nowhere
            float2 part[kWaves];
            float m = kNothing, l = 0.f, f[kWaves];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                part[w] = *reinterpret_cast<const float2 *>(stats + (w * kRows + thread) * 2);
                m = fmaxf(m, part[w].x);
            }
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                f[w] = __builtin_amdgcn_exp2f(part[w].x - m);
                l = fmaf(part[w].y, f[w], l);
            }
            uint32_t nan = 0x7fc00000u;
            asm volatile("" : "+v"(nan));  // its bits: the compiler is told that no float is one
            const bool none = row_at_lds[thread] != 0 && l > 0.f;  // of a query without scores
            const int r = r0 + thread, j = divided(r, a.by_G), in_head = h * a.G + (r - j * a.G);
            const int64_t row_at = (int64_t)(s.first_row + j) * n_heads + in_head;
            int64_t at = -1;
            if (r < n_rows) {
                if (a.n_splits > 1) {
                    const int64_t part_at = row_at * a.n_splits + split;
                    *reinterpret_cast<float2 *>(a.part_ml + 2 * part_at) = make_float2(m, none ? -1.f : l);
                    at = l > 0.f ? part_at * (32 * NG) : -1;
                } else {
                    const float inverse = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w)
                        f[w] = __uint_as_float(none ? nan : __float_as_uint(f[w] * inverse));
                    at = (int64_t)(s.first_row + j) * a.out.row + (int64_t)in_head * a.out.head;
                    if (a.lse)
                        reinterpret_cast<uint32_t *>(a.lse)[row_at] = none ? nan : __float_as_uint(lse_of(m, l));
                }
            }
#pragma unroll
            for (int w = 0; w < kWaves; w += 4)
                *reinterpret_cast<f4 *>(row_factors + thread * kWaves + w) = f4{f[w], f[w + 1], f[w + 2], f[w + 3]};
            row_at_lds[thread] = at;
        }
        constexpr int kPass = attend_pass(NG, kBlocks), kUnits = 8 * NG;  // a thread takes 4 channels of a row
#pragma unroll 1
        for (int first = 0; first < kBlocks; first += kPass) {
            unrolled<0, kBlocks>([&](auto t) {
                constexpr int nb = decltype(t)::value;
                if (first == nb / kPass * kPass) {
                    float *const mine = join + ((wave * kPass + nb % kPass) * 16 + col_now) * kPitch;
                    unrolled<0, P::n>([&](auto part) {
                        constexpr int p = decltype(part)::value, kRun = 2 * P::groups(p), kWide = kRun < 4 ? 2 : 4;
                        typedef float wide __attribute__((ext_vector_type(kWide)));
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int e0 = 0; e0 < kRun; e0 += kWide) {
                                wide y;
#pragma unroll
                                for (int e = 0; e < kWide; ++e)
                                    y[e] = o[2 * P::before(p) + e0 + e][nb][r];
                                *reinterpret_cast<wide *>(mine + 32 * P::before(p) + kRun * (4 * quarter_now + r) + e0) = y;
                            }
                    });
                }
            });
            __syncthreads();
#pragma unroll 2
            for (int unit = thread; unit < kPass * 16 * kUnits; unit += 64 * kWaves) {
                const int row = (int)((uint32_t)unit / kUnits), ch = 4 * (unit - row * kUnits);
                const int64_t at = row_at_lds[16 * first + row];
                f4 total = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    const float f = row_factors[(16 * first + row) * kWaves + w];
                    const f4 y = *reinterpret_cast<const f4 *>(join + (w * kPass * 16 + row) * kPitch + ch);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        total[e] = fmaf(f, y[e], total[e]);
                }
                if (at < 0)
                    continue;
                if (a.n_splits > 1)
                    *reinterpret_cast<f4 *>(a.part_acc + at + ch) = total;
                else
                    store_four<kBf16>(a.out.data + at + ch, total, c.D - ch);
            }
            __syncthreads();
        }
    }
}

// Maximum, or sum, over a wave: inside rows of 16 lanes and then across them, without LDS.
template <int kCtrl, int kRows>
__device__ __forceinline__ float moved(float x, float otherwise)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(otherwise), __float_as_int(x), kCtrl, kRows, 0xf, false));
}
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, moved<0x111, 0xf>(x, kNothing));  // shifted right by 1, 2, 4, 8 lanes of a row
    x = fmaxf(x, moved<0x112, 0xf>(x, kNothing));
    x = fmaxf(x, moved<0x114, 0xf>(x, kNothing));
    x = fmaxf(x, moved<0x118, 0xf>(x, kNothing));
    x = fmaxf(x, moved<0x142, 0xa>(x, kNothing));  // lane 15 to the next row, lane 31 to the last two
    x = fmaxf(x, moved<0x143, 0xc>(x, kNothing));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ float wave_sum(float x)
{
    x += moved<0x111, 0xf>(x, 0.f);
    x += moved<0x112, 0xf>(x, 0.f);
    x += moved<0x114, 0xf>(x, 0.f);
    x += moved<0x118, 0xf>(x, 0.f);
    x += moved<0x142, 0xa>(x, 0.f);
    x += moved<0x143, 0xc>(x, 0.f);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

// The splits' sums of a row, relative to the largest reference.  A workgroup takes one row and head: its four waves take splits in
// turn, as many at a time as rows of 4-channel lanes fit a wave, and join their sums in LDS.  Every wave forms the factors by itself
// and asks for the sums before it has them.
constexpr int kMostSplits = 128;
template <int NG, bool kBf16>
__global__ __launch_bounds__(kMergeThreads) void k_cache4_merge(Cache4Attend a)
{
    constexpr int kLanes = 8 * NG, kInWave = 64 / kLanes, kAtOnce = kInWave * (kMergeThreads / 64);  // lanes of a split, splits at once
    constexpr int kAhead = NG <= 4 ? 8 : 4, kMls = kMostSplits / 64;
    __shared__ __align__(16) f4 partial[kAtOnce][kLanes];
    const int tid = threadIdx.x, lane = tid & 63, n_heads = a.c.H * a.G;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int in_wave = lane / kLanes, ch = 4 * (lane - in_wave * kLanes);
    const bool works = in_wave < kInWave;
    const int mine = kInWave * wave + in_wave;  // splits mine, mine + kAtOnce, ..
    const int64_t n = (int64_t)a.b.n_rows * n_heads;
    const int first_row = a.b.starts ? const_ints(a.b.starts)[0] : 0, end_row = a.b.starts ? const_ints(a.b.starts)[a.b.n_seqs] : a.b.n_rows;
    for (int64_t row_at = blockIdx.x; row_at < n; row_at += gridDim.x) {
        const int row = (int)((uint32_t)row_at / (uint32_t)n_heads), head = (int)row_at - row * n_heads;
        if (row < first_row || row >= end_row)
            continue;
        const float *acc = a.part_acc + row_at * a.n_splits * (32 * NG) + ch;
        const auto load = [&](int s) { return *reinterpret_cast<const f4 *>(acc + (int64_t)min(s, a.n_splits - 1) * (32 * NG)); };
        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + row_at * a.n_splits;
        float2 z[kMls];
#pragma unroll
        for (int i = 0; i < kMls; ++i)
            z[i] = ml[min(lane + 64 * i, a.n_splits - 1)];
        f4 y[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            y[i] = load(mine + i * kAtOnce);
        float m = kNothing, l = 0.f, f[kMls];
        bool none = false;
#pragma unroll
        for (int i = 0; i < kMls; ++i)
            none |= z[i].y < 0.f;  // a query without scores
        none = __any(none);
        uint32_t nan = 0x7fc00000u;
        asm volatile("" : "+v"(nan));
#pragma unroll
        for (int i = 0; i < kMls; ++i)
            m = fmaxf(m, lane + 64 * i < a.n_splits && z[i].y > 0.f ? z[i].x : kNothing);
        m = wave_max(m);
#pragma unroll
        for (int i = 0; i < kMls; ++i) {
            const bool there = lane + 64 * i < a.n_splits && z[i].y > 0.f;  // of a split that saw nothing there are no sums
            f[i] = there ? __builtin_amdgcn_exp2f(z[i].x - m) : 0.f;
            l = fmaf(there ? z[i].y : 0.f, f[i], l);
        }
        l = wave_sum(l);
        f4 total = f4{0.f, 0.f, 0.f, 0.f};
        const auto add = [&](int s, f4 x) {
            float w = __shfl(f[0], s & 63);
#pragma unroll
            for (int i = 1; i < kMls; ++i) {
                const float v = __shfl(f[i], s & 63);
                w = s >> 6 == i ? v : w;
            }
            w = works && s < a.n_splits ? w : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                total[e] = fmaf(w, w > 0.f ? x[e] : 0.f, total[e]);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            add(mine + i * kAtOnce, y[i]);
        for (int s = kAhead * kAtOnce; s < a.n_splits; s += kAtOnce)  // as often for every lane: they ask each other for factors
            add(s + mine, load(s + mine));
        if (works)
            partial[mine][ch / 4] = total;
        __syncthreads();
        if (tid < kLanes) {
            total = partial[0][tid];
#pragma unroll
            for (int i = 1; i < kAtOnce; ++i)
                total += partial[i][tid];
            const float inverse = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                total[e] = __uint_as_float(none ? nan : __float_as_uint(total[e] * inverse));
            store_four<kBf16>(a.out.data + (int64_t)row * a.out.row + (int64_t)head * a.out.head + 4 * tid, total, a.c.D - 4 * tid);
            if (a.lse && tid == 0)
                reinterpret_cast<uint32_t *>(a.lse)[row_at] = none ? nan : __float_as_uint(lse_of(m, l));
        }
        __syncthreads();
    }
}

// How a call is cut.  Times are of 8 kv heads x 128 channels in the float format, 4 query heads a kv head, unless said otherwise, and of
// calls whose max_length is the longest length.  Tokens are shared out by max_length, so that shorter sequences leave parts without
// tokens: with room for 131072, one step of one sequence of 8192 tokens 21 us for 10, of eight 55 for 19.
//   - Rows of a workgroup: 16 as long as that makes no more than a workgroup for each compute unit, 32 up to twice that many, then 64;
//     never so many that a smaller form would hold all rows of a sequence.  More rows share the reconstruction, fewer keep more units
//     at work.  16 / 32 / 64 rows: 20 new tokens behind 2000 12.7 / 14.3 / 17.7 us, 128 behind 8000 38 / 41 / 43, 512 behind 8000
//     112 / 88 / 87, 1024 of two sequences behind 15000 728 / 565 / 481.  Heads of more than 128 channels have no room for 64.
//   - Tokens are split only where there are fewer workgroups than compute units, which the second kernel costs 4 us and more for many
//     rows (32 sequences of 4000 tokens, 2 x 16 rows, 4 heads: 22 us as they are, 29 in two): into enough for two workgroups a unit
//     (6 sequences of up to 12345 tokens, 5 rows x 8 query heads, 4 heads x 96 integers: 28 us, with one a unit 31), but no more than
//     32 where that is enough for one (one sequence of 32768 tokens: 64 parts 16.0 us, 32 14.9), of two steps of each wave at least
//     (two sequences of 8000: 13.5 us, with one step 14.4, with four 14.9) or of one, if that makes 16 at most (one of 4000: 10.5 us,
//     with two steps 11.4).  Four steps are not split (8 sequences of up to 1500 tokens, 5 rows: 13.1 us, in two 14.9).
//   - Where a launch of the largest sequence's tiles for each would be mostly empty, places are dealt along all rows and a workgroup finds
//     its sequence (2048 rows among 63 single ones: 192 us without, 93 with; among 255 360 and 116; later steps brought these to 76 and 103).
constexpr int kUnits = 256;  // compute units
constexpr int kFewSplits = 32;
constexpr int kOneStepSplits = 16;
constexpr int kWholeRounds = 4;
constexpr int kFewPlaces = 1024;

Cache4Plan plan_cache4_attend(const Cache4 &c, const Cache4Seqs &b, int max_rows, int max_length, int G, int window)
{
    Cache4Plan p;
    const int64_t rows = (int64_t)max_rows * G, heads = (int64_t)c.H * b.n_seqs;
    const auto tiles_of = [&](int blocks) { return (rows + 16 * blocks - 1) / (16 * blocks); };
    const auto flat_of = [&](int blocks) { return Cache4Flat{1, G, blocks == 1 ? 4 : blocks == 2 ? 5 : 6, 1}; };
    const auto places_of = [&](int blocks) {  // of one head, as many as there can be work for
        return b.starts ? std::min(tiles_of(blocks) * b.n_seqs, cache4_places(flat_of(blocks), b.n_rows, b.n_seqs)) : tiles_of(blocks) * b.n_seqs;
    };
    p.blocks = 1;
    while (p.blocks < (c.NG > 4 ? 2 : 4) && tiles_of(p.blocks) > 1 && places_of(p.blocks) * c.H > kUnits * p.blocks)
        p.blocks *= 2;
    p.flat = flat_of(p.blocks);
    const int64_t places = places_of(p.blocks);
    p.flat.on = b.starts && b.n_seqs > 1 && tiles_of(p.blocks) * heads > kFewPlaces && 2 * tiles_of(p.blocks) * b.n_seqs > 3 * places;
    // More tiles than places take turns, so that what the host believes of the rows never makes more workgroups than work could fill.
    p.n_tiles = (int32_t)(p.flat.on ? places : std::min(tiles_of(p.blocks), std::max<int64_t>(std::min<int64_t>(512, ((int64_t)1 << 20) / heads), 1)));
    int64_t span = max_length;
    if (window)
        span = std::min(span, (int64_t)window + std::min<int64_t>(max_rows, 16 * p.blocks / G + 1));
    const int64_t groups = places * c.H, round = kStep * attend_waves(p.blocks);
    int64_t splits = 1;
    const int64_t rounds = (span + round - 1) / round;
    if (groups < kUnits && rounds > kWholeRounds) {
        splits = std::max<int64_t>(kUnits / groups, std::min<int64_t>(2 * kUnits / groups, kFewSplits));
        splits = std::min({splits, std::max<int64_t>((rounds + 1) / 2, std::min<int64_t>(rounds, kOneStepSplits)), (int64_t)kMostSplits});
    }
    p.split_tokens = (int32_t)((span + splits * round - 1) / (splits * round) * round);
    p.n_splits = (int32_t)((span + p.split_tokens - 1) / p.split_tokens);
    p.ml_bytes = p.acc_bytes = 0;
    if (p.n_splits > 1) {
        const uint64_t parts = (uint64_t)b.n_rows * c.H * G * p.n_splits;
        p.ml_bytes = (parts * 8 + 255) / 256 * 256;
        p.acc_bytes = parts * 32 * c.NG * 4;
    }
    return p;
}

namespace {

template <int kFormat, int NG, bool kBf16>
const void *attend_kernel(int blocks)
{
    if (blocks == 1)
        return reinterpret_cast<const void *>(&k_cache4_attend<kFormat, NG, 1, kBf16>);
    if constexpr (NG <= 4) {
        if (blocks == 4)
            return reinterpret_cast<const void *>(&k_cache4_attend<kFormat, NG, 4, kBf16>);
    }
    return reinterpret_cast<const void *>(&k_cache4_attend<kFormat, NG, 2, kBf16>);
}
template <int kFormat, bool kBf16>
const void *attend_kernel(int NG, int blocks)
{
    switch (NG) {
    case 1: return attend_kernel<kFormat, 1, kBf16>(blocks);
    case 2: return attend_kernel<kFormat, 2, kBf16>(blocks);
    case 3: return attend_kernel<kFormat, 3, kBf16>(blocks);
    case 4: return attend_kernel<kFormat, 4, kBf16>(blocks);
    case 6: return attend_kernel<kFormat, 6, kBf16>(blocks);
    default: return attend_kernel<kFormat, 8, kBf16>(blocks);
    }
}

}  // namespace

template <int NG>
static const void *merge_kernel(bool bf16)
{
    return bf16 ? reinterpret_cast<const void *>(&k_cache4_merge<NG, true>) : reinterpret_cast<const void *>(&k_cache4_merge<NG, false>);
}
static const void *merge_kernel(int NG, bool bf16)
{
    switch (NG) {
    case 1: return merge_kernel<1>(bf16);
    case 2: return merge_kernel<2>(bf16);
    case 3: return merge_kernel<3>(bf16);
    case 4: return merge_kernel<4>(bf16);
    case 6: return merge_kernel<6>(bf16);
    default: return merge_kernel<8>(bf16);
    }
}

static const void *attend_kernel(int format, bool bf16, int NG, int blocks)
{
    if (format == HQMQ_CACHE4_FLOAT)
        return bf16 ? attend_kernel<HQMQ_CACHE4_FLOAT, true>(NG, blocks) : attend_kernel<HQMQ_CACHE4_FLOAT, false>(NG, blocks);
    return bf16 ? attend_kernel<HQMQ_CACHE4_INT, true>(NG, blocks) : attend_kernel<HQMQ_CACHE4_INT, false>(NG, blocks);
}

hipError_t prepare_cache4_kernels()
{
    for (int format : {HQMQ_CACHE4_FLOAT, HQMQ_CACHE4_INT})
        for (int NG : {1, 2, 3, 4, 6, 8})
            for (int blocks : {1, 2, 4})
                for (int bf16 = 0; bf16 < 2; ++bf16) {
                    if (attend_lds_bytes(NG, blocks) <= 64 * 1024 || (NG > 4 && blocks > 2))
                        continue;
                    const hipError_t err = hipFuncSetAttribute(attend_kernel(format, bf16 != 0, NG, blocks), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                               (int)attend_lds_bytes(NG, blocks));
                    if (err != hipSuccess)
                        return err;
                }
    return hipSuccess;
}

hipError_t launch_cache4_attend(const Cache4Attend &a, const Cache4Plan &plan, bool bf16, hipStream_t stream)
{
    const void *kernel = attend_kernel(a.c.format, bf16, a.c.NG, plan.blocks);
    dim3 grid((unsigned)a.c.H, (unsigned)(plan.n_tiles * plan.n_splits), (unsigned)a.b.n_seqs);
    if (plan.flat.on) {
        grid.z = (grid.y + 32767) / 32768;
        grid.y = (grid.y + grid.z - 1) / grid.z;
    }
    Cache4Attend args = a;
    void *list[] = {&args};
    hipError_t err = hipLaunchKernel(kernel, grid, dim3(64 * attend_waves(plan.blocks)), list, attend_lds_bytes(a.c.NG, plan.blocks), stream);
    if (err != hipSuccess || plan.n_splits == 1)
        return err;
    const dim3 rows((unsigned)std::min<int64_t>((int64_t)a.b.n_rows * a.c.H * a.G, 1 << 20));
    return hipLaunchKernel(merge_kernel(a.c.NG, bf16), rows, dim3(kMergeThreads), list, 0, stream);
}

}  // namespace hqmq
