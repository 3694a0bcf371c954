// Causal attention over a paged cache held in 4 bits (include/hqmq_cache4.h, hqmq_cache4_attend).
//
// A workgroup takes 16, 32 or 64 query rows of a kv head (row r = j G + g is query head g of the sequence's row j) and a share of
// the tokens; its four waves take steps of 32 tokens in turn and join their sums in LDS at the end.  The codes go from memory to
// the operands of v_mfma_f32_16x16x32_f16 without crossing lanes, by three choices of order:
//   S^T = K Q^T   lane (token l % 16, quarter l / 16) reads a quarter of a key's codes, a run of 8 NG channels, and the query operand
//                 has the same channels in the same places;
//   P^T           the scores come as lane (query l % 16, tokens 4 (l / 16) .. + 3) of each 16 tokens, which two of together are the
//                 eight tokens of that lane in the operand P^T as they stand;
//   O^T = V^T P^T lane (run l % 16, l / 16) reads the codes of those eight tokens for a run of 8 (4, 2) channels, two blocks of four
//                 tokens of the V layout, and product e takes channel e of every run.
// A query's maximum and sum belong to one column, so every factor is one per lane.
#include <algorithm>

#include "hqmq_cache4_device.h"

namespace hqmq {

namespace {

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef cache4_h2 half2_t;
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4, kThreads4 = 64 * kWaves, kStep = 32;
constexpr float kNothing = -1.0e30f;  // "no token seen yet": finite, so that differences stay finite
constexpr float kTop4 = 7.f;          // weights are taken relative to 2^-kTop4 of the largest score,
constexpr float kRise4 = 15.f;        // and relative to a newer one once they would pass 2^kRise4 (fp16 ends at 2^16)
constexpr float kLog2e4 = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kPartChannels = 128;    // of V at most, as a part of its layout
constexpr int kJoinPitch = kPartChannels + 4;

constexpr size_t attend_lds_bytes(int NG, int blocks)
{
    const size_t queries = (size_t)blocks * NG * 64 * 16, join = (size_t)kWaves * 16 * kJoinPitch * 4;
    return (queries > join ? queries : join) + (size_t)blocks * 16 * 8 + (size_t)kWaves * blocks * 16 * 2 * 4;
}

// Maximum or sum over the four lanes that hold a query's column.
__device__ __forceinline__ float column_max(float x)
{
    auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
    y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
__device__ __forceinline__ float column_sum(float x)
{
    auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(y[0]) + __uint_as_float(y[1]);
}

// n words from an address that is a multiple of 4 n bytes from one of 16.
template <int n>
struct Words {
    uint32_t w[n];
};
template <int n>
__device__ __forceinline__ Words<n> load_words(const uint8_t *p)
{
    struct __attribute__((packed, aligned(n % 4 == 0 ? 16 : n % 2 == 0 ? 8 : 4))) Raw {
        uint32_t w[n];
    };
    const Raw r = *reinterpret_cast<const Raw *>(p);
    Words<n> out;
#pragma unroll
    for (int i = 0; i < n; ++i)
        out.w[i] = r.w[i];
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
    Words<NG> code;
    uint32_t scale[kScales];
};
template <int kFormat, int NG>
struct VStage {
    static constexpr int kWords = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    Words<NG> code;
    Words<kWords> scale[Parts<NG>::n];
};

// 16 tokens of a head in one page: where they begin in each of the cache's buffers (one address for the wave), and where the lane's
// share lies behind that (the same for all).
struct Tile {
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
};
template <int kFormat, int NG>
__device__ __forceinline__ Tile tile_at(const Cache4 &c, int page, int h, int slot)
{
    constexpr int kScale = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    const int64_t row = (((int64_t)page * c.H + h) << c.page_shift) + slot;
    return Tile{c.k_codes + row * (16 * NG), c.k_scales + row * (kScale * NG), c.v_codes + row * (16 * NG), c.v_scales + row * (kScale * NG)};
}

template <int kFormat, int NG>
__device__ __forceinline__ void load_k(KStage<kFormat, NG> &s, const Tile &tile, int lane)
{
    const uint32_t token = lane & 15, quarter = lane >> 4, first = quarter * NG >> 2, last = (quarter * NG + NG - 1) >> 2;
    s.code = load_words<NG>(tile.k_codes + (token * (16 * NG) + 4 * NG * quarter));
    const auto scale_of = [&](uint32_t g) -> uint32_t {
        return kFormat == HQMQ_CACHE4_FLOAT ? (uint32_t)tile.k_scales[token * NG + g] : load_words<1>(tile.k_scales + 4 * (token * NG + g)).w[0];
    };
    s.scale[0] = scale_of(first);
    if (KStage<kFormat, NG>::kScales > 1)
        s.scale[KStage<kFormat, NG>::kScales - 1] = scale_of(last);
}

template <int kFormat, int NG>
__device__ __forceinline__ void load_v(VStage<kFormat, NG> &s, const Tile &tile, int lane)
{
    constexpr uint32_t kScale = kFormat == HQMQ_CACHE4_FLOAT ? 1 : 4;
    const uint32_t quarter = lane >> 4, run = lane & 15;
    using P = Parts<NG>;
#pragma unroll
    for (int p = 0; p < P::n; ++p) {
        const uint8_t *at = tile.v_codes + (quarter * (64 * NG) + 4 * P::groups(p) * run + 64 * P::before(p));
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
        s.scale[p] = load_words<VStage<kFormat, NG>::kWords>(tile.v_scales + kScale * (4 * (quarter * NG + P::before(p) + (run * P::groups(p) >> 4))));
    }
}

// Tokens of the lane's four at or behind `end` (of these four) become zeros, whatever lies there.
template <int kFormat, int NG>
__device__ __forceinline__ void blank_v(VStage<kFormat, NG> &s, int end)
{
    using P = Parts<NG>;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const bool gone = t >= end;
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

// The operand of channels 8 w .. 8 w + 7 of the lane's run, in their order (float) or in that of kIntOrder (int).
template <int kFormat, int NG>
__device__ __forceinline__ half8_t k_operand(const KStage<kFormat, NG> &s, int w, int lane)
{
    const int quarter = lane >> 4;
    uint32_t scale = s.scale[0];
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
        const half2_t sm = __builtin_bit_cast(half2_t, scale), ss = {sm[0], sm[0]}, mm = {sm[1], sm[1]};
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = int4_pair(code >> (4 * e), ss, mm);
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
                uint32_t both;  // the byte of token 2 i at bits 0..7, that of token 2 i + 1 at 16..23
                if (groups == 4)
                    both = __builtin_amdgcn_perm(code[(2 * i + 1) % NG], code[(2 * i) % NG], 0x0c040c00u + 0x00010001u * kByte);
                else if (groups == 2)
                    both = code[i % NG] >> (8 * kByte);
                else
                    both = __builtin_amdgcn_perm(0u, code[0], 0x0c010c00u + 0x00020002u * i);
                e[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair(both, step, least));
                o[2 * x + i] = __builtin_bit_cast(uint32_t, int4_pair(both >> 4, step, least));
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

// Workgroups of a compute unit that the registers are to leave room for.
constexpr int attend_occupancy(int NG, int blocks) { return blocks == 1 ? (NG <= 4 ? 4 : 2) : 2; }

}  // namespace

template <int kFormat, int NG, int kBlocks, bool kBf16>
__global__ __launch_bounds__(kThreads4, attend_occupancy(NG, kBlocks)) void k_cache4_attend(Cache4Attend a)
{
    using P = Parts<NG>;
    constexpr int kRows = 16 * kBlocks, kChannels = 2 * NG;  // of a lane
    constexpr bool kFine = !kBf16;
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr size_t kShared = std::max((size_t)kBlocks * NG * 64 * 16, (size_t)kWaves * 16 * kJoinPitch * 4);
    half8_t *const queries = reinterpret_cast<half8_t *>(lds);           // [kBlocks][NG][lane]
    float *const join = reinterpret_cast<float *>(lds);                  // [kWaves][16][kJoinPitch], when the queries are done with
    float *const factor = reinterpret_cast<float *>(lds + kShared);      // [kRows]: from products to exponents of 2
    int *const position = reinterpret_cast<int *>(factor + kRows);       // [kRows]: -1 - 2^30 and less: no row
    float *const stats = reinterpret_cast<float *>(position + kRows);    // [kWaves][kRows][2]

    const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, quarter = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const Cache4 &c = a.c;
    const int h = (int)(blockIdx.x % (uint32_t)c.H), rest = (int)(blockIdx.x / (uint32_t)c.H);
    const int split = rest % a.n_splits, seq = blockIdx.y;
    const int page_mask = (1 << c.page_shift) - 1;
    const ConstInts table = const_ints(a.b.table + (int64_t)seq * a.b.pitch);
    const Cache4Seq s = cache4_seq(a.b, c.page_shift, seq);
    const int n_rows = s.n * a.G, n_heads = c.H * a.G;

    // the longest first: a causal prompt's last rows see the most
    for (int tile = a.n_tiles - 1 - rest / a.n_splits; tile * kRows < n_rows; tile += a.n_tiles) {
        const int r0 = tile * kRows;
        // ---- what the rows see -----------------------------------------------------------------------------------------
        const int j_first = r0 / a.G, j_last = min((r0 + kRows - 1) / a.G, s.n - 1);
        const int end = s.pos0 + j_last + 1, all_end = s.pos0 + j_first + 1;  // all_end: every row sees what is before it,
        const int begin = a.window ? max(0, s.pos0 + j_first + 1 - a.window) & ~(kStep - 1) : 0;
        const int all_begin = a.window ? s.pos0 + j_last + 1 - a.window : 0;  // and from here on
        const int64_t share = (int64_t)begin + (int64_t)split * a.split_tokens;
        const int from = (int)min(share, (int64_t)max(end, 0));
        const int to = split == a.n_splits - 1 ? end : (int)min(share + a.split_tokens, (int64_t)max(end, 0));
        const int n_steps = to > from ? (to - from + kStep - 1) / kStep : 0;

        // Pages of a step's two halves; -1 for none.  Past the share's end: those of its last step.
        const int last = from + kStep * max(n_steps - 1, 0);
        int page[2];
        const auto look_up = [&](int step) {
            const int token = min(from + kStep * step, last);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                page[x] = __builtin_amdgcn_readfirstlane(table[min((token + 16 * x) >> c.page_shift, a.b.pitch - 1)]);
        };
        KStage<kFormat, NG> ks[2];
        VStage<kFormat, NG> vs[2];
        Tile tiles[2];
        bool bad[2];
        const auto tiles_of = [&](int token) {  // of the pages that were looked up last
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                bad[x] = (uint32_t)page[x] >= (uint32_t)c.n_pages;
                tiles[x] = tile_at<kFormat, NG>(c, bad[x] ? 0 : page[x], h, (token + 16 * x) & page_mask);
            }
        };
        if (wave < n_steps) {
            look_up(wave);
            tiles_of(from + kStep * wave);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                load_k(ks[x], tiles[x], lane);
#pragma unroll
            for (int x = 0; x < 2; ++x)
                load_v(vs[x], tiles[x], lane);
            look_up(wave + kWaves);
        }

        // ---- queries to LDS, as operands -------------------------------------------------------------------------------
        for (int nb = wave; nb < kBlocks; nb += kWaves) {
            const int r = r0 + 16 * nb + col;
            const bool there = r < n_rows;
            const int j = r / a.G;
            const uint16_t *src = a.q.data + (int64_t)(s.first_row + j) * a.q.row + (int64_t)(h * a.G + (r - j * a.G)) * a.q.head;
            uint4v bits[NG];
#pragma unroll
            for (int w = 0; w < NG; ++w) {
                const int ch = 8 * (quarter * NG + w);
                bits[w] = uint4v{0u, 0u, 0u, 0u};
                if (there && ch < c.D) {
                    if (a.q.wide) {
                        bits[w] = *reinterpret_cast<const uint4v *>(src + ch);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (ch + e < c.D)
                                bits[w][e / 2] |= (uint32_t)src[ch + e] << (16 * (e & 1));
                    }
                }
            }
            float f = fabsf(a.scale) * kLog2e4;
            const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;  // a negative scale goes into the queries' signs
            if (kBf16) {
                // A power of two brings the row's largest magnitude to 2^14 .. 2^15, where fp16 has all its bits down to 2^-28 of it.
                uint32_t top = 0;
#pragma unroll
                for (int w = 0; w < NG; ++w)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        top = max(top, max(bits[w][e] & 0x7fffu, bits[w][e] >> 16 & 0x7fffu));
                top = max(top, (uint32_t)__shfl_xor((int)top, 16));
                top = max(top, (uint32_t)__shfl_xor((int)top, 32));
                const int up = 141 - (int)(top >> 7);
                f = ldexpf(f, -up);
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
                if (kFormat == HQMQ_CACHE4_INT)  // channels 0 4 1 5 2 6 3 7
                    x = uint4v{__builtin_amdgcn_perm(x[2], x[0], 0x05040100u), __builtin_amdgcn_perm(x[2], x[0], 0x07060302u),
                               __builtin_amdgcn_perm(x[3], x[1], 0x05040100u), __builtin_amdgcn_perm(x[3], x[1], 0x07060302u)};
                queries[(nb * NG + w) * 64 + lane] = __builtin_bit_cast(half8_t, x);
            }
            if (quarter == 0) {
                // Products stay below 2^40: with a factor this small they all become 0, but minus infinity stays what it is.
                factor[16 * nb + col] = fmaxf(f, 0x1p-120f);
                position[16 * nb + col] = there ? s.pos0 + j : -0x7fffffff;
            }
        }
        __syncthreads();
        float scale[kBlocks];
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb)
            scale[nb] = factor[16 * nb + col];

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
            f4 x[2][kBlocks];
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
            tiles_of(min(token + kStep * kWaves, last));
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_k(ks[i], tiles[i], lane);
            // ---- unseen tokens
            if (token + kStep > all_end || token < all_begin || bad_now[0] || bad_now[1]) {
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
            half8_t hi[kBlocks], lo[kBlocks];
#pragma unroll
            for (int nb = 0; nb < kBlocks; ++nb) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float p = __builtin_amdgcn_exp2f(fmaf(x[i][nb][r], scale[nb], -ref[nb]));
                        sum[nb] += p;
                        const _Float16 rounded = (_Float16)p;
                        hi[nb][4 * i + r] = rounded;
                        if (kFine)
                            lo[nb][4 * i + r] = (_Float16)(p - (float)rounded);
                    }
            }
            // ---- values: a token that is none of the sequence's may hold anything
            if (token + kStep > s.length || bad_now[0] || bad_now[1]) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    blank_v(vs[i], bad_now[i] ? 0 : s.length - (token + 16 * i + 4 * quarter));
            }
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
#pragma unroll
            for (int i = 0; i < 2; ++i)
                load_v(vs[i], tiles[i], lane);
            look_up(step + 2 * kWaves);
        }

        // ---- the four waves' sums joined -------------------------------------------------------------------------------
#pragma unroll
        for (int nb = 0; nb < kBlocks; ++nb) {
            const float total = column_sum(sum[nb]);
            if (quarter == 0) {
                stats[(wave * kRows + 16 * nb + col) * 2] = ref[nb];
                stats[(wave * kRows + 16 * nb + col) * 2 + 1] = total;
            }
        }
        __syncthreads();
        const bool whole_result = a.n_splits == 1;
        unrolled<0, kBlocks>([&](auto block) {
            constexpr int nb = decltype(block)::value;
            const auto joined = [&](int row, float &ref_all, float &sum_all) {
                ref_all = kNothing;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    ref_all = fmaxf(ref_all, stats[(w * kRows + row) * 2]);
                sum_all = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    sum_all += stats[(w * kRows + row) * 2 + 1] * __builtin_amdgcn_exp2f(stats[(w * kRows + row) * 2] - ref_all);
            };
            float ref_all, sum_all;
            joined(16 * nb + col, ref_all, sum_all);
            const float f = __builtin_amdgcn_exp2f(ref[nb] - ref_all);
            unrolled<0, P::n>([&](auto part) {
                constexpr int p = decltype(part)::value, kRun = 2 * P::groups(p), kUnits = 4 * P::groups(p);
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int e = 0; e < kRun; ++e)
                        join[(wave * 16 + col) * kJoinPitch + kRun * (4 * quarter + r) + e] = f * o[2 * P::before(p) + e][nb][r];
                __syncthreads();
                if (tid < 16 * kUnits) {
                    const int row = tid / kUnits, ch0 = 8 * (tid % kUnits), r = r0 + 16 * nb + row;
                    float m, l;
                    joined(16 * nb + row, m, l);
                    f4 total[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
                    for (int w = 0; w < kWaves; ++w)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            total[i] += *reinterpret_cast<const f4 *>(join + (w * 16 + row) * kJoinPitch + ch0 + 4 * i);
                    if (r < n_rows) {
                        const int j = r / a.G, head = h * a.G + (r - j * a.G), ch = 32 * P::before(p) + ch0;
                        const int64_t row_at = (int64_t)(s.first_row + j) * n_heads + head;
                        if (!whole_result) {
                            const int64_t at = row_at * a.n_splits + split;
                            if (l > 0.f) {
                                f4 *dst = reinterpret_cast<f4 *>(a.part_acc + at * (32 * NG) + ch);
                                dst[0] = total[0];
                                dst[1] = total[1];
                            }
                            if (ch == 0) {
                                a.part_ml[2 * at] = m;
                                a.part_ml[2 * at + 1] = l;
                            }
                        } else {
                            const float inverse = l > 0.f ? 1.f / l : 0.f;
                            uint4v bits;
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float u = total[e / 2][2 * (e & 1)] * inverse, v = total[e / 2][2 * (e & 1) + 1] * inverse;
                                if (kBf16) {
                                    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
                                    bits[e] = __builtin_bit_cast(uint32_t, b2{(__bf16)u, (__bf16)v});
                                } else {
                                    bits[e] = __builtin_bit_cast(uint32_t, half2_t{(_Float16)u, (_Float16)v});
                                }
                            }
                            uint16_t *dst = a.out.data + (int64_t)(s.first_row + j) * a.out.row + (int64_t)head * a.out.head + ch;
                            if (a.out.wide) {
                                if (ch < c.D)
                                    *reinterpret_cast<uint4v *>(dst) = bits;
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (ch + e < c.D)
                                        dst[e] = (uint16_t)(bits[e / 2] >> (16 * (e & 1)));
                            }
                            if (a.lse && ch == 0)
                                a.lse[row_at] = l > 0.f ? kLn2 * (m + __builtin_amdgcn_logf(l)) : -__builtin_inff();
                        }
                    }
                }
                __syncthreads();
            });
        });
    }
}

// The splits' sums of a row, relative to the largest reference.  A workgroup takes one row and head: its four waves take splits in
// turn, as many at a time as rows of 4-channel lanes fit a wave, and join their sums in LDS.
constexpr int kMostSplits = 128;
template <bool kBf16>
__global__ __launch_bounds__(kThreads4) void k_cache4_merge(Cache4Attend a)
{
    __shared__ __align__(16) float weight[kMostSplits];
    __shared__ __align__(16) f4 partial[kThreads4];
    __shared__ float whole[2];
    const int tid = threadIdx.x, n_heads = a.c.H * a.G, width = 32 * a.c.NG, lanes = width / 4, at_once = kThreads4 / lanes;
    const int mine = tid / lanes, ch = 4 * (tid - mine * lanes);
    const int64_t n = (int64_t)a.b.n_rows * n_heads;
    for (int64_t row_at = blockIdx.x; row_at < n; row_at += gridDim.x) {
        const int row = (int)(row_at / n_heads), head = (int)(row_at - (int64_t)row * n_heads);
        if (a.b.starts && (row < a.b.starts[0] || row >= a.b.starts[a.b.n_seqs]))
            continue;
        __syncthreads();
        if (tid < 64) {
            const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + row_at * a.n_splits;
            float2 y[kMostSplits / 64];
            float m = kNothing, l = 0.f;
#pragma unroll
            for (int i = 0; i < kMostSplits / 64; ++i) {
                y[i] = tid + 64 * i < a.n_splits ? ml[tid + 64 * i] : make_float2(kNothing, 0.f);
                m = fmaxf(m, y[i].y > 0.f ? y[i].x : kNothing);
            }
#pragma unroll
            for (int d = 32; d; d >>= 1)
                m = fmaxf(m, __shfl_xor(m, d));
#pragma unroll
            for (int i = 0; i < kMostSplits / 64; ++i) {
                const float f = y[i].y > 0.f ? __builtin_amdgcn_exp2f(y[i].x - m) : 0.f;
                weight[tid + 64 * i] = f;
                l = fmaf(y[i].y, f, l);
            }
#pragma unroll
            for (int d = 32; d; d >>= 1)
                l += __shfl_xor(l, d);
            if (tid == 0) {
                whole[0] = m;
                whole[1] = l;
            }
        }
        __syncthreads();
        f4 total = f4{0.f, 0.f, 0.f, 0.f};
        if (mine < at_once) {
            const float *acc = a.part_acc + row_at * a.n_splits * width + ch;
#pragma unroll 4
            for (int s = mine; s < a.n_splits; s += at_once) {
                const float f = weight[s];
                const f4 y = *reinterpret_cast<const f4 *>(acc + (int64_t)s * width);
                if (f > 0.f)  // of a split that saw nothing there are no sums
                    total += f4{f, f, f, f} * y;
            }
        }
        partial[tid] = total;
        __syncthreads();
        if (tid < lanes) {
            for (int i = 1; i < at_once; ++i)
                total += partial[tid + i * lanes];
            const float l = whole[1], inverse = l > 0.f ? 1.f / l : 0.f;
            uint16_t *dst = a.out.data + (int64_t)row * a.out.row + (int64_t)head * a.out.head + ch;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (ch + e < a.c.D) {
                    const float y = total[e] * inverse;
                    dst[e] = kBf16 ? __builtin_bit_cast(uint16_t, (__bf16)y) : __builtin_bit_cast(uint16_t, (_Float16)y);
                }
            if (a.lse && tid == 0)
                a.lse[row_at] = l > 0.f ? kLn2 * (whole[0] + __builtin_amdgcn_logf(l)) : -__builtin_inff();
        }
    }
}

Cache4Plan plan_cache4_attend(const Cache4 &c, const Cache4Seqs &b, int max_rows, int max_length, int G, int window)
{
    Cache4Plan p;
    const int64_t rows = (int64_t)max_rows * G;
    p.blocks = rows <= 16 ? 1 : rows <= 32 || c.NG > 4 ? 2 : 4;
    const int64_t heads = (int64_t)c.H * b.n_seqs;
    const int64_t most_tiles = ((int64_t)1 << 22) / c.H > 0 ? ((int64_t)1 << 22) / c.H : 1;
    p.n_tiles = (int32_t)std::min((rows + 16 * p.blocks - 1) / (16 * p.blocks), most_tiles);
    int64_t span = max_length;
    if (window)
        span = std::min(span, (int64_t)window + std::min<int64_t>(max_rows, 16 * p.blocks / G + 1));
    const int64_t round = kStep * kWaves, rr = getenv("HQ_R") ? atoi(getenv("HQ_R")) : 2, most = std::max<int64_t>((span + rr * round - 1) / (rr * round), 1);
    const int64_t wanted = (getenv("HQ_S") ? atoi(getenv("HQ_S")) : 512) / std::max<int64_t>(p.n_tiles * heads, 1);
    p.n_splits = (int32_t)std::max<int64_t>(std::min<int64_t>(std::min(wanted, most), kMostSplits), 1);
    p.split_tokens = (int32_t)((span + p.n_splits * round - 1) / (p.n_splits * round) * round);
    p.n_splits = (int32_t)std::max<int64_t>((span + p.split_tokens - 1) / p.split_tokens, 1);
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

hipError_t launch_cache4_attend(const Cache4Attend &a, const Cache4Plan &plan, bool bf16, hipStream_t stream)
{
    const bool f = a.c.format == HQMQ_CACHE4_FLOAT;
    const void *kernel = f ? (bf16 ? attend_kernel<HQMQ_CACHE4_FLOAT, true>(a.c.NG, plan.blocks) : attend_kernel<HQMQ_CACHE4_FLOAT, false>(a.c.NG, plan.blocks))
                           : (bf16 ? attend_kernel<HQMQ_CACHE4_INT, true>(a.c.NG, plan.blocks) : attend_kernel<HQMQ_CACHE4_INT, false>(a.c.NG, plan.blocks));
    const dim3 grid((unsigned)((int64_t)a.c.H * plan.n_tiles * plan.n_splits), (unsigned)a.b.n_seqs);
    Cache4Attend args = a;
    void *list[] = {&args};
    hipError_t err = hipLaunchKernel(kernel, grid, dim3(kThreads4), list, attend_lds_bytes(a.c.NG, plan.blocks), stream);
    if (err != hipSuccess || plan.n_splits == 1)
        return err;
    const dim3 rows((unsigned)std::min<int64_t>((int64_t)a.b.n_rows * a.c.H * a.G, 1 << 20));
    if (bf16)
        k_cache4_merge<true><<<rows, kThreads4, 0, stream>>>(args);
    else
        k_cache4_merge<false><<<rows, kThreads4, 0, stream>>>(args);
    return hipGetLastError();
}

}  // namespace hqmq
