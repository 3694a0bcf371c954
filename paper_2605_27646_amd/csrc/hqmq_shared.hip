// Attention of many sequences over one packed prefix (include/hqmq_serve.h, hqmq_attend_shared): O = softmax(Q K^T scale) V
// with the n_share * G query rows of a kv head against one reconstruction of its K and V.
#include <type_traits>

#include "hqmq_serve_device.h"

namespace hqmq {

namespace {

constexpr int kThreadsShared = 512;
constexpr int kGroupThreads = 256;  // a group of four waves works on tiles of its own
constexpr int kPay = 128;           // outlier payloads of a tile and side kept in LDS
constexpr float kNoToken = -1.0e30f;
constexpr float kTop = 10.f;        // weights are taken relative to 2^-kTop of the largest score,
constexpr float kRise = 15.f;       // and relative to a newer one once they would pass 2^kRise
constexpr uint32_t kBigScale = 0x77ffu;  // 32752 as fp16 bits: below it no product of a unit codeword leaves the fp16 range

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

// Tokens of a tile: 2048 chunks of K and V together, eight for each of a group's threads (24 chunks per row: 1536).
template <int kNc>
constexpr int tile_tokens() { return kNc == 16 ? 64 : 32; }
template <int kNc>
constexpr int key_pitch() { return 4 * kNc + 8; }  // halves; an odd number of 16-byte slots: rows fall on all banks
template <int kNc>
constexpr int value_pitch() { return tile_tokens<kNc>() + 8; }

// LDS of a group, in 32-bit words: keys [tokens][key_pitch] halves | values [D rows][value_pitch] halves | code words of K, of V |
// flags, scales, offsets of K, of V | payloads of K, of V
template <int kNc>
struct GroupLds {
    static constexpr int kTok = tile_tokens<kNc>();
    static constexpr int keys = kTok * key_pitch<kNc>() / 2;
    static constexpr int values = 4 * kNc * value_pitch<kNc>() / 2;
    static constexpr int rows = 3 * kTok;
    static constexpr int pay = 2 * kPay + 4;  // and a slot past the last that is read and not used
    __host__ __device__ static constexpr int words(int row_words) { return (kTok * row_words + 2 + 3) / 4 * 4; }  // + a word read past the last
    __host__ __device__ static constexpr int total(int row_words) { return keys + values + 2 * (words(row_words) + rows + pay); }
};
static_assert(GroupLds<32>::keys % 4 == 0 && GroupLds<24>::keys % 4 == 0 && GroupLds<16>::keys % 4 == 0, "16-byte reads of what follows");
static_assert(GroupLds<32>::values % 4 == 0 && GroupLds<24>::values % 4 == 0 && GroupLds<16>::values % 4 == 0, "16-byte reads of what follows");

// Codeword directions divided by the radius codes' range L, so that a chunk is (radius code * scale, exact in fp32) times an
// entry, rounded once.  kTable: per side 13 S entries (12 primaries with a positive first non-zero component, then zeros for
// primaries past the 24), else the S secondaries and the 24 primaries.
template <bool kTable>
__host__ __device__ constexpr size_t side_floats(int S) { return (size_t)(kTable ? 13 : 1) * S * 4; }

// Row of V^T in LDS for component e of chunk c: blocks of 32 rows are the operands of one product; in a product's result a lane
// then holds all four components of a chunk.
__device__ __forceinline__ int value_row(int c, int e) { return 32 * (c >> 3) + 8 * e + (c & 7); }

__device__ __forceinline__ float4_t product(const float P[4], float4_t q)
{
    float4_t d;
    d[0] = fmaf(-P[3], q[3], fmaf(-P[2], q[2], fmaf(-P[1], q[1], P[0] * q[0])));
    d[1] = fmaf(-P[3], q[2], fmaf(P[2], q[3], fmaf(P[1], q[0], P[0] * q[1])));
    d[2] = fmaf(P[3], q[1], fmaf(P[2], q[0], fmaf(-P[1], q[3], P[0] * q[2])));
    d[3] = fmaf(P[3], q[0], fmaf(-P[2], q[1], fmaf(P[1], q[2], P[0] * q[3])));
    return d;
}

}  // namespace

template <int kNc, bool kTable, bool kPow2, int kCols>
__global__ __launch_bounds__(kThreadsShared, 2) void k_shared(Geometry g, SharedArgs a)
{
    using L = GroupLds<kNc>;
    constexpr int kTok = L::kTok, kD = 4 * kNc;
    constexpr int kLoads = (kTok * (kNc * 24 / 32) + kGroupThreads - 1) / kGroupThreads;  // code words per thread and side, at the largest w
    constexpr bool kWide = kCols >= 32;           // 32x32x16 products, else 16x16x32
    constexpr int kCb = kWide ? kCols / 32 : 1;   // blocks of columns (query rows) of a wave
    constexpr int kSteps = kWide ? kD / 16 : kD / 32;
    constexpr int kBlocks = kWide ? kD / 32 : kD / 16;
    constexpr int kRegs = kWide ? 16 : 4;         // of a block's result
    using acc_t = std::conditional_t<kWide, float16_t, float4_t>;
    extern __shared__ __align__(16) float lds[];
    uint2 *lut = reinterpret_cast<uint2 *>(lds);  // [48] of a primary: byte offset of its rows in a table (number without one), sign bit
    float *prim = lds + 96;                       // [24][4], without tables
    float *dir_k = prim + (kTable ? 0 : 96);
    float *dir_v = dir_k + side_floats<kTable>(g.S);
    uint32_t *groups = reinterpret_cast<uint32_t *>(dir_v + side_floats<kTable>(g.S));

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int group = wave >> 2, gt = tid & (kGroupThreads - 1), gw = wave & 3;
    const int seg = blockIdx.y, b = seg / g.H, h = seg % g.H;
    const uint32_t row_words = kNc == 32 ? (uint32_t)g.w : (uint32_t)g.row_words;
    const uint32_t w = g.w, w_idx = g.w_idx;

    uint32_t *mine = groups + group * L::total((int)row_words);
    _Float16 *keys = reinterpret_cast<_Float16 *>(mine);
    _Float16 *values = reinterpret_cast<_Float16 *>(mine + L::keys);
    uint32_t *words[2], *row_part[2];
    uint2 *pays[2];
    {
        uint32_t *p = mine + L::keys + L::values;
        const int nw = L::words((int)row_words);
        words[0] = p;
        words[1] = p + nw;
        row_part[0] = p + 2 * nw;
        row_part[1] = row_part[0] + L::rows;
        pays[0] = reinterpret_cast<uint2 *>(row_part[1] + L::rows);
        pays[1] = pays[0] + L::pay / 2;
    }

    // ---- columns of this wave: query rows r of the kv head ---------------------------------------------------------
    const int n_rows = a.n_share * a.G;
    const int col0 = (int)blockIdx.z * 4 * kCols + gw * kCols;
    const int col = kWide ? (lane & 31) : (lane & 15);
    const int kgrp = kWide ? (lane >> 5) : (lane >> 4);  // which 8 of a product's terms the lane supplies, which rows of a result it holds
    const bool has_cols = col0 < n_rows;                 // uniform
    const uint32_t flip = a.qscale < 0.f ? 0x80008000u : 0u;
    const float qscale = fabsf(a.qscale);                // a negative scale goes into the queries' signs
    half8_t qf[kCb][kSteps];
    int vis[kCb];
    int least = g.T, most = 0;
#pragma unroll
    for (int cb = 0; cb < kCb; ++cb) {
        const int r = col0 + 32 * cb + col;
        const bool there = r < n_rows;
        const int rr = there ? r : 0, m = rr / a.G;
        const size_t head = ((size_t)(b * a.n_share + m) * g.H + h) * a.G + (rr - m * a.G);
        const _Float16 *q = a.q + head * kD + 8 * kgrp;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            uint4v v = *reinterpret_cast<const uint4v *>(q + (kWide ? 16 : 32) * s);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = there ? v[i] ^ flip : 0u;
            qf[cb][s] = __builtin_bit_cast(half8_t, v);
        }
        vis[cb] = g.T;
        if (a.visible) {
            if (there)
                vis[cb] = min(max(a.visible[head], 0), g.T);
            least = min(least, vis[cb]);
        }
        most = max(most, there ? vis[cb] : 0);
    }

    // ---- the tables --------------------------------------------------------------------------------------------------
    {
        const double over_L = 1.0 / (double)((1 << g.b_r) - 1);
        const float *sk = a.k.sec + (size_t)h * g.S * 4, *sv = a.v.sec + (size_t)h * g.S * 4;
        for (int i = tid; i < 2 * g.S; i += kThreadsShared) {
            const bool is_v = i >= g.S;
            const int s = is_v ? i - g.S : i;
            const float4_t q = *reinterpret_cast<const float4_t *>((is_v ? sv : sk) + 4 * s);
            float4_t *dst = reinterpret_cast<float4_t *>(is_v ? dir_v : dir_k) + s;
            double x[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                x[e] = (double)q[e] * over_L;
            if (!kTable) {
                *dst = float4_t{(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
            } else {
#pragma unroll
                for (int c = 0; c < 13; ++c) {
                    double P[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        P[e] = c < 4 ? (c == e ? 1.0 : 0.0) : (c == 12 ? 0.0 : (e == 0 ? 0.5 : ((((c - 4) >> (3 - e)) & 1) ? -0.5 : 0.5)));
                    float4_t d;
                    d[0] = (float)fma(-P[3], x[3], fma(-P[2], x[2], fma(-P[1], x[1], P[0] * x[0])));
                    d[1] = (float)fma(-P[3], x[2], fma(P[2], x[3], fma(P[1], x[0], P[0] * x[1])));
                    d[2] = (float)fma(P[3], x[1], fma(P[2], x[0], fma(-P[1], x[3], P[0] * x[2])));
                    d[3] = (float)fma(P[3], x[0], fma(-P[2], x[1], fma(P[1], x[2], P[0] * x[3])));
                    dst[(size_t)c * g.S] = d;
                }
            }
        }
        if (tid < 48) {
            const uint32_t p = tid;
            uint32_t c = 12u, neg = 0u;
            if (p < 8) {
                c = p >> 1;
                neg = p & 1u;
            } else if (p < 24) {
                const uint32_t bits = p - 8u;
                neg = bits >> 3;
                c = 4u + ((neg ? ~bits : bits) & 7u);
            }
            lut[p] = make_uint2(kTable ? c * (uint32_t)g.S * 16u : c * 16u, neg << 31);
        }
        if (!kTable && tid < 96) {
            const int c = tid >> 2, e = tid & 3;
            prim[tid] = c < 4 ? (c == e ? 1.f : 0.f) : (c >= 12 ? 0.f : (e == 0 ? 0.5f : ((((c - 4) >> (3 - e)) & 1) ? -0.5f : 0.5f)));
        }
    }

    // ---- the tiles of this workgroup -----------------------------------------------------------------------------------
    const int begin = (int)blockIdx.x * a.rows_per_split;
    int end = min(g.T, begin + a.rows_per_split);
    if (a.visible) {  // nothing that no row of the workgroup sees is read; every wave needs the same end
        int *both = reinterpret_cast<int *>(mine);
        for (int d = 32; d > 0; d /= 2)
            most = max(most, __shfl_xor(most, d));
        for (int d = 32; d > 0; d /= 2)
            least = min(least, __shfl_xor(least, d));
        if (lane == 0)
            both[gw] = most;
        __syncthreads();
        end = min(end, max(max(both[0], both[1]), max(both[2], both[3])));
        least = __builtin_amdgcn_readfirstlane(least);
        end = __builtin_amdgcn_readfirstlane(end);
        __syncthreads();
    }
    const int n_tiles = end > begin ? (end - begin + kTok - 1) / kTok : 0;
    const int n_mine = (n_tiles + 1 - group) >> 1;  // tiles group, group + 2, ...

    float m_ref[kCb], l_run[kCb];
    acc_t acc[kCb][kBlocks];
#pragma unroll
    for (int cb = 0; cb < kCb; ++cb) {
        m_ref[cb] = kNoToken;
        l_run[cb] = 0.f;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
            for (int i = 0; i < kRegs; ++i)
                acc[cb][k][i] = 0.f;
    }

    // ---- a tile's packed rows on their way to LDS ------------------------------------------------------------------------
    uint32_t cw[2][kLoads], fw = 0u, sg = 0u, ro = 0u;
    uint32_t list0[2], listn[2];  // window of the outlier list: first entry and length
    uint2 pay = make_uint2(0u, 0u);
    uint32_t pay_base[2] = {0u, 0u}, pay_n[2] = {0u, 0u};  // of the tile in LDS
    const AttendSide *const sides[2] = {&a.k, &a.v};
    auto tile_start = [&](int j) { return begin + (2 * j + group) * kTok; };
    auto request = [&](int j) {
        const int t0 = tile_start(j);
        const int nr = min(kTok, end - t0);
        const int64_t R0 = (int64_t)seg * g.T + t0;
        const uint32_t last = (uint32_t)nr * row_words - 1u;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const uint32_t *src = sides[s]->codes + R0 * row_words;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                cw[s][i] = src[min((uint32_t)gt + kGroupThreads * i, last)];
            list0[s] = sides[s]->row_off[R0];
            listn[s] = sides[s]->row_off[R0 + nr];
        }
        if (gt < 2 * kTok) {
            const int s = gt / kTok, row = gt % kTok, r = min(row, nr - 1);
            const bool there = row < nr;
            fw = (s ? a.v.flags : a.k.flags)[R0 + r];
            sg = (s ? a.v.sigma : a.k.sigma)[R0 + r];
            ro = (s ? a.v.row_off : a.k.row_off)[R0 + r];
            fw = there ? fw : 0u;
            sg = there ? sg : 0u;
        }
    };
    auto request_payloads = [&]() {
        const int s = gt >> 7;  // uniform
        const AttendSide &sd = s ? a.v : a.k;
        const uint32_t base = s ? list0[1] : list0[0], n = (s ? listn[1] : listn[0]) - base;
        const uint32_t in_list = (uint64_t)base < sd.outlier_capacity ? (uint32_t)min((uint64_t)n, sd.outlier_capacity - base) : 0u;
        const uint32_t slot = (uint32_t)gt & (kPay - 1);
        pay = make_uint2(0u, 0u);
        if (slot < in_list)
            pay = reinterpret_cast<const uint2 *>(sd.outliers)[base + (uint64_t)slot];
    };
    auto stage = [&]() {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int nw = L::words((int)row_words);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (gt + kGroupThreads * i < nw)
                    words[s][gt + kGroupThreads * i] = cw[s][i];
            pay_base[s] = list0[s];
            pay_n[s] = listn[s] - list0[s];
        }
        if (gt < 2 * kTok) {
            uint32_t *dst = row_part[gt / kTok] + gt % kTok;
            dst[0] = fw;
            dst[kTok] = sg;
            dst[2 * kTok] = ro;
        }
        pays[gt >> 7][gt & (kPay - 1)] = pay;
    };

    // ---- reconstruction ----------------------------------------------------------------------------------------------------
    const uint32_t idx_mask = (1u << w_idx) - 1u;
    const uint32_t div_shift = 32u - (uint32_t)__clz((int)(48u * (uint32_t)g.S * (uint32_t)g.S));
    const uint32_t div_mul = ((1u << div_shift) + (uint32_t)g.S - 1u) / (uint32_t)g.S;  // k / S = k * div_mul >> div_shift for k < 48 S, in 32 bits while
                                                                                                   // the tables fit (S < 300)
    auto read_code = [&](int s, int row, uint32_t c) {
        const uint32_t bit = c * w;
        const uint32_t *rw = words[s] + row * row_words + (bit >> 5);
        return __builtin_amdgcn_alignbit(rw[1], rw[0], bit & 31u);
    };
    auto chunk = [&](auto fast_tag, int s, uint32_t code, float scale, uint32_t slot, bool flagged) {
        constexpr bool kFast = decltype(fast_tag)::value;
        uint32_t p, s_idx;
        if (kPow2) {
            p = (code >> g.log2_S) & 31u;
            s_idx = code & ((uint32_t)g.S - 1u);
        } else {
            const uint32_t kk = code & idx_mask;
            p = kTable ? __umul24(kk, div_mul) >> div_shift : (uint32_t)((float)kk * g.inv_S);
            s_idx = kk - __umul24(p, (uint32_t)g.S);
        }
        const uint2 l = lut[p];
        const char *dir = reinterpret_cast<const char *>(s ? dir_v : dir_k) + (s_idx << 4);
        float4_t d;
        if (kTable) {
            d = *reinterpret_cast<const float4_t *>(dir + l.x);
        } else {
            const float4_t P = *reinterpret_cast<const float4_t *>(reinterpret_cast<const char *>(prim) + l.x);
            const float Pa[4] = {P[0], P[1], P[2], P[3]};
            d = product(Pa, *reinterpret_cast<const float4_t *>(dir));
        }
        const float r = __uint_as_float(__float_as_uint((float)__builtin_amdgcn_ubfe(code, w_idx, w - w_idx) * scale) | l.y);
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            y[e] = r * d[e];
            if (!kFast)
                y[e] = __builtin_amdgcn_fmed3f(y[e], -65504.f, 65504.f);  // the decode saturates
        }
        half4_t out;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            out[e] = (_Float16)y[e];
        uint2 o = __builtin_bit_cast(uint2, out);
        uint2 v = pays[s][min(slot, (uint32_t)kPay)];
        if (!kFast && slot >= (uint32_t)kPay && flagged) {  // past the staged ones: straight from the list
            const AttendSide &sd = s ? a.v : a.k;
            const uint64_t at = (uint64_t)pay_base[s] + slot;
            v = at < sd.outlier_capacity ? reinterpret_cast<const uint2 *>(sd.outliers)[at] : make_uint2(0u, 0u);
        }
        o.x = flagged ? v.x : o.x;
        o.y = flagged ? v.y : o.y;
        return o;
    };
    auto scale_of = [&](int s, int row) { return (float)__builtin_bit_cast(_Float16, (uint16_t)row_part[s][kTok + row]); };
    auto decode_keys = [&](auto fast_tag) {
#pragma unroll
        for (int u0 = 0; u0 < kTok * kNc / 2; u0 += kGroupThreads) {
            const int u = u0 + gt;
            if (kTok * kNc / 2 % kGroupThreads != 0 && u >= kTok * kNc / 2)
                break;
            const int row = u / (kNc / 2), c = 2 * (u % (kNc / 2));
            const uint32_t word = row_part[0][row];
            const uint32_t slot = row_part[0][2 * kTok + row] - pay_base[0] + __popc(word & ((1u << c) - 1u));
            const float scale = scale_of(0, row);
            const bool f0 = (word >> c) & 1u, f1 = (word >> c) & 2u;
            const uint2 x = chunk(fast_tag, 0, read_code(0, row, c), scale, slot, f0);
            const uint2 y = chunk(fast_tag, 0, read_code(0, row, c + 1), scale, slot + (f0 ? 1u : 0u), f1);
            *reinterpret_cast<uint4v *>(keys + row * key_pitch<kNc>() + 4 * c) = uint4v{x.x, x.y, y.x, y.y};
        }
    };
    auto decode_values = [&](auto fast_tag) {
        const int u = gt;
        if (kNc * kTok / 4 < kGroupThreads && u >= kNc * kTok / 4)
            return;
        static_assert(kNc * kTok / 4 <= kGroupThreads, "one chunk of four tokens per thread");
        const int c = u % kNc, quad = u / kNc;
        const uint4v word = *reinterpret_cast<const uint4v *>(row_part[1] + 4 * quad);
        const uint4v off = *reinterpret_cast<const uint4v *>(row_part[1] + 2 * kTok + 4 * quad);
        uint2 v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t slot = off[i] - pay_base[1] + __popc(word[i] & ((1u << c) - 1u));
            v[i] = chunk(fast_tag, 1, read_code(1, 4 * quad + i, c), scale_of(1, 4 * quad + i), slot, (word[i] >> c) & 1u);
        }
        // where the four tokens stand in the order in which a product takes a block of scores as its operand
        const int at = kWide ? 4 * ((quad & ~3) | ((quad & 1) << 1) | ((quad >> 1) & 1)) : 4 * ((quad & ~7) | ((quad & 3) << 1) | ((quad >> 2) & 1));
        const uint32_t lo = 0x05040100u, hi = 0x07060302u;
        _Float16 *dst = values + value_row(c, 0) * value_pitch<kNc>() + at;
        const auto put = [&](int e, uint32_t x, uint32_t y) {
            *reinterpret_cast<uint2 *>(dst + 8 * e * value_pitch<kNc>()) = make_uint2(x, y);
        };
        put(0, __builtin_amdgcn_perm(v[1].x, v[0].x, lo), __builtin_amdgcn_perm(v[3].x, v[2].x, lo));
        put(1, __builtin_amdgcn_perm(v[1].x, v[0].x, hi), __builtin_amdgcn_perm(v[3].x, v[2].x, hi));
        put(2, __builtin_amdgcn_perm(v[1].y, v[0].y, lo), __builtin_amdgcn_perm(v[3].y, v[2].y, lo));
        put(3, __builtin_amdgcn_perm(v[1].y, v[0].y, hi), __builtin_amdgcn_perm(v[3].y, v[2].y, hi));
    };
    auto decode = [&]() {
        // uniform per wave: what can leave the fp16 range or lies past the staged payloads is taken with care
        bool big = false;
        for (int row = lane; row < kTok; row += 64)
            big |= row_part[0][kTok + row] >= kBigScale || row_part[1][kTok + row] >= kBigScale;
        const bool care = __any(big);
        if (!care && pay_n[0] <= (uint32_t)kPay)
            decode_keys(std::true_type{});
        else
            decode_keys(std::false_type{});
        if (!care && pay_n[1] <= (uint32_t)kPay)
            decode_values(std::true_type{});
        else
            decode_values(std::false_type{});
    };

    // ---- the two products of a tile and the softmax between them --------------------------------------------------------------
    const auto over_lanes = [&](float v, auto f) {  // over the lanes that hold other rows of the same column
        if (!kWide) {
            const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
            v = f(__uint_as_float(x[0]), __uint_as_float(x[1]));
        }
        const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
    };
    auto attend = [&](int j, auto between) {
#pragma unroll
        for (int sub = 0; sub < kTok; sub += 32) {
            const int t0 = tile_start(j) + sub;
            float s[kCb][16];  // wide: token 8 (i / 4) + 4 kgrp + i % 4; else (8 of them) 16 (i / 4) + 4 kgrp + i % 4
            constexpr int kS = kWide ? 16 : 8;
            if constexpr (kWide) {
                float16_t sc[kCb];
#pragma unroll
                for (int cb = 0; cb < kCb; ++cb)
                    sc[cb] = float16_t{0.f};
                const _Float16 *kp = keys + (sub + (lane & 31)) * key_pitch<kNc>() + 8 * kgrp;
#pragma unroll
                for (int st = 0; st < kSteps; ++st) {
                    const half8_t kf = *reinterpret_cast<const half8_t *>(kp + 16 * st);
#pragma unroll
                    for (int cb = 0; cb < kCb; ++cb)
                        sc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf, qf[cb][st], sc[cb], 0, 0, 0);
                }
#pragma unroll
                for (int cb = 0; cb < kCb; ++cb)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        s[cb][i] = sc[cb][i];
            } else {
                float4_t sc[2] = {float4_t{0.f, 0.f, 0.f, 0.f}, float4_t{0.f, 0.f, 0.f, 0.f}};
                const _Float16 *kp = keys + (sub + (lane & 15)) * key_pitch<kNc>() + 8 * kgrp;
#pragma unroll
                for (int st = 0; st < kSteps; ++st)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const half8_t *>(kp + 16 * u * key_pitch<kNc>() + 32 * st),
                                                                       qf[0][st], sc[u], 0, 0, 0);
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    s[0][i] = sc[i >> 2][i & 3];
            }
            const bool whole = t0 + 32 <= end && t0 + 32 <= least;  // uniform: every row sees every token
            half8_t ph[kCb][2], pl[kCb][2];
#pragma unroll
            for (int cb = 0; cb < kCb; ++cb) {
                float mul = qscale;
                if (!whole) {
                    const int seen = min(end, vis[cb]) - t0 - 4 * kgrp;
#pragma unroll
                    for (int i = 0; i < kS; ++i)
                        s[cb][i] = (kWide ? 8 : 16) * (i >> 2) + (i & 3) < seen ? s[cb][i] * qscale : 3.f * kNoToken;
                    mul = 1.f;
                }
                float top = s[cb][0];
#pragma unroll
                for (int i = 1; i < kS; ++i)
                    top = fmaxf(top, s[cb][i]);
                top = over_lanes(top * mul, [](float x, float y) { return fmaxf(x, y); });
                // Weights are 2^(s - m_ref): with m_ref 10 below the largest score seen they reach 2^10, their fp16 parts hold weights
                // down to 2^-24 of the largest as normal numbers, and m_ref is raised (and what was summed scaled) only when a score
                // would pass 2^15, so hardly ever after the first tiles.
                const bool raise = top - m_ref[cb] > kRise;
                if (__any(raise)) {
                    const float m_new = raise ? top - kTop : m_ref[cb];
                    const float corr = __builtin_amdgcn_exp2f(m_ref[cb] - m_new);
                    m_ref[cb] = m_new;
                    l_run[cb] *= corr;
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                        for (int i = 0; i < kRegs; ++i)
                            acc[cb][k][i] *= corr;
                }
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < kS; ++i) {
                    const float p = __builtin_amdgcn_exp2f(fmaf(s[cb][i], mul, -m_ref[cb]));
                    sum += p;
                    const _Float16 hi = (_Float16)p;
                    ph[cb][i >> 3][i & 7] = hi;
                    pl[cb][i >> 3][i & 7] = (_Float16)(p - (float)hi);  // the weight in 22 bits
                }
                l_run[cb] += sum;
            }
            if (sub == 0)
                between();
            const _Float16 *vp = values + (kWide ? (lane & 31) : (lane & 15)) * value_pitch<kNc>() + sub + 8 * kgrp;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) {
                if constexpr (kWide) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const half8_t vf = *reinterpret_cast<const half8_t *>(vp + 32 * k * value_pitch<kNc>() + 16 * u);
#pragma unroll
                        for (int cb = 0; cb < kCb; ++cb) {
                            acc[cb][k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, ph[cb][u], acc[cb][k], 0, 0, 0);
                            acc[cb][k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf, pl[cb][u], acc[cb][k], 0, 0, 0);
                        }
                    }
                } else {
                    const half8_t vf = *reinterpret_cast<const half8_t *>(vp + 16 * k * value_pitch<kNc>());
                    acc[0][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, ph[0][0], acc[0][k], 0, 0, 0);
                    acc[0][k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, pl[0][0], acc[0][k], 0, 0, 0);
                }
            }
        }
    };

    // ---- phases: while one group multiplies a tile, the other reconstructs its next -----------------------------------------------
    if (group == 0 && n_mine > 0) {
        request(0);
        request_payloads();
        stage();
    }
    __syncthreads();
    const int n0 = (n_tiles + 1) >> 1, n1 = n_tiles >> 1;
    const int last = max(2 * n0, n1 > 0 ? 2 * n1 + 1 : 0);
    for (int ph = 1; ph <= last; ++ph) {
        if ((ph + group) & 1) {
            if ((ph - 1 - group) / 2 < n_mine)
                decode();
        } else {
            const int j = (ph - 2 - group) / 2;  // -1 in the second group's first phase
            const bool more = j + 1 < n_mine;
            if (more)
                request(j + 1);
            const auto payloads = [&]() {
                if (more)
                    request_payloads();
            };
            if (has_cols && j >= 0 && j < n_mine)
                attend(j, payloads);
            else
                payloads();
            if (more)
                stage();
        }
        __syncthreads();
    }

    // ---- the second group's state joins the first's, which writes the workgroup's ------------------------------------------------
    float *xch = lds + (size_t)gw * 64 * (kCb * (kBlocks * kRegs + 2)) + lane;  // over everything: no wave reads tiles or tables any more
#pragma unroll
    for (int cb = 0; cb < kCb; ++cb)
        l_run[cb] = over_lanes(l_run[cb], [](float x, float y) { return x + y; });
    if (group == 1 && has_cols) {
        int at = 0;
#pragma unroll
        for (int cb = 0; cb < kCb; ++cb) {
            xch[64 * at++] = m_ref[cb];
            xch[64 * at++] = l_run[cb];
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                for (int i = 0; i < kRegs; ++i)
                    xch[64 * at++] = acc[cb][k][i];
        }
    }
    __syncthreads();
    if (group == 1 || !has_cols)
        return;
    int at = 0;
#pragma unroll
    for (int cb = 0; cb < kCb; ++cb) {
        const float m2 = xch[64 * at++], l2 = xch[64 * at++];
        const float m = fmaxf(m_ref[cb], m2);
        const float c1 = __builtin_amdgcn_exp2f(m_ref[cb] - m), c2 = __builtin_amdgcn_exp2f(m2 - m);
        const int r = col0 + 32 * cb + col;
        const bool there = r < n_rows;
        const int rr = there ? r : 0, q = rr / a.G;
        const size_t head = ((size_t)(b * a.n_share + q) * g.H + h) * a.G + (rr - q * a.G);
        const size_t part = head * a.part_pitch + blockIdx.x;
        if (there && kgrp == 0) {
            a.part_ml[2 * part] = m;
            a.part_ml[2 * part + 1] = fmaf(l_run[cb], c1, l2 * c2);
        }
        float *dst = a.part_acc + part * 128;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
            float o[kRegs];
#pragma unroll
            for (int i = 0; i < kRegs; ++i)
                o[i] = fmaf(acc[cb][k][i], c1, xch[64 * at++] * c2);
            if (!there)
                continue;
            if constexpr (kWide) {  // row 8 e + c % 8 of block c / 8: the lane has chunks 8 k + 4 kgrp + 0 .. 3
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<float4_t *>(dst + 4 * (8 * k + 4 * kgrp + i)) = float4_t{o[i], o[4 + i], o[8 + i], o[12 + i]};
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * k + 4 * kgrp + i;
                    dst[4 * (8 * (row >> 5) + (row & 7)) + ((row >> 3) & 3)] = o[i];
                }
            }
        }
    }
}

// Columns of a wave: 16, 32 or 64, the fewest with which four waves hold all query rows of a kv head.
static int shared_cols(const Geometry &g, int n_rows)
{
    return n_rows <= 64 ? 16 : n_rows <= 128 ? 32 : 64;
}

static size_t shared_lds_bytes(const Geometry &g, int cols, bool table)
{
    const int group = g.n_c == 32 ? GroupLds<32>::total(g.row_words) : g.n_c == 24 ? GroupLds<24>::total(g.row_words) : GroupLds<16>::total(g.row_words);
    const size_t loop = 96 + (table ? 2 * side_floats<true>(g.S) : 96 + 2 * side_floats<false>(g.S)) + 2 * (size_t)group;
    const size_t merge = (size_t)4 * (cols * g.D + 2 * 64 * (cols > 32 ? 2 : 1));
    return (loop > merge ? loop : merge) * sizeof(float);
}

SharedPlan plan_shared(const Geometry &g, int G, int n_share)
{
    const int tok = g.n_c == 16 ? 64 : 32;
    const int n_rows = G * n_share, per_wg = 4 * shared_cols(g, n_rows);
    const int64_t per = (int64_t)g.B * g.H * ((n_rows + per_wg - 1) / per_wg), pairs = (g.T + 2 * tok - 1) / (2 * tok);
    int64_t want = 256 / per;  // one workgroup per compute unit
    want = want < 1 ? 1 : want < pairs ? want : pairs;
    const int64_t pairs_per = (pairs + want - 1) / want;
    return {(int32_t)((pairs + pairs_per - 1) / pairs_per), (int32_t)(pairs_per * 2 * tok)};
}

namespace {
template <int kNc, bool kTable, bool kPow2>
const void *shared_kernel(int cols)
{
    return cols == 16 ? reinterpret_cast<const void *>(&k_shared<kNc, kTable, kPow2, 16>)
         : cols == 32 ? reinterpret_cast<const void *>(&k_shared<kNc, kTable, kPow2, 32>)
                      : reinterpret_cast<const void *>(&k_shared<kNc, kTable, kPow2, 64>);
}
template <int kNc>
const void *shared_kernel(bool table, bool pow2, int cols)
{
    if (!table)
        return shared_kernel<kNc, false, false>(cols);
    return pow2 ? shared_kernel<kNc, true, true>(cols) : shared_kernel<kNc, true, false>(cols);
}
const void *shared_kernel(int n_c, bool table, bool pow2, int cols)
{
    return n_c == 32 ? shared_kernel<32>(table, pow2, cols) : n_c == 24 ? shared_kernel<24>(table, pow2, cols) : shared_kernel<16>(table, pow2, cols);
}
}  // namespace

hipError_t prepare_shared_kernels()
{
    for (int n_c : {32, 24, 16})
        for (int cols : {16, 32, 64})
            for (int form = 0; form < 3; ++form) {
                const hipError_t err = hipFuncSetAttribute(shared_kernel(n_c, form > 0, form > 1, cols), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsPerCu);
                if (err != hipSuccess)
                    return err;
            }
    return hipSuccess;
}

hipError_t launch_shared(const Geometry &g, const SharedArgs &a, hipStream_t stream)
{
    if (g.D != 128 && g.D != 96 && g.D != 64)
        return hipErrorInvalidValue;
    const int n_rows = a.G * a.n_share, cols = shared_cols(g, n_rows);
    const bool table = shared_lds_bytes(g, cols, true) <= kLdsPerCu, pow2 = (g.S & (g.S - 1)) == 0;
    const dim3 grid((unsigned)a.n_splits, (unsigned)(g.B * g.H), (unsigned)((n_rows + 4 * cols - 1) / (4 * cols)));
    Geometry gc = g;
    SharedArgs ac = a;
    void *args[] = {&gc, &ac};
    return hipLaunchKernel(shared_kernel(g.n_c, table, pow2, cols), grid, dim3(kThreadsShared), args, shared_lds_bytes(g, cols, table), stream);
}

}  // namespace hqmq
