// Attention of many sequences over one packed prefix (include/hqmq_serve.h, hqmq_attend_shared): O = softmax(Q K^T scale) V
// with the n_share * G query rows of a kv head against one reconstruction of its K and V.
//
// Both products are formed with the tokens as rows, S^T = K Q^T and O^T = V^T P^T: a lane then has scores of one query row, so that the
// softmax's maximum and sum are the lane's own up to two swaps, and a block of weights, rounded, is the second product's operand as it
// stands.  Reconstructed keys and values (transposed) go through LDS, where the waves of a workgroup share them.  Workgroups split the
// prefix; sums and maxima of the splits, in fp32, are joined by the merge of hqmq_attend where there is more than one.
//
// What bounds it depends on the rows.  Up to 64 of them the reconstruction, 40 vector instructions and some 60 cycles of LDS per 64 chunks,
// but neither unit by itself: 8 heads x 32771 tokens x 64, 24 rows a head, 27 us, of which vector instructions issue for 48 % and the LDS
// works for 43 %, while waves wait for 48 % of their cycles (reconstruct, barrier, multiply, barrier; 64 heads x 2049 x 96, 12 rows and
// their own tokens: 31 us, 50, 37 and 49 %).  256 rows, 8 heads x 32768 x 128: 74 us for encoded normal values, 82 for channels of different
// gain and uniformly drawn codewords, 420 to 460 TFLOP/s, where a large product of two matrices would take 30.  Of the 82 vector instructions
// have 47 %, the matrix cores 25, the LDS 31, and waves wait for 44 % of their cycles: a barrier for every 32 tokens between those that
// reconstruct and those that multiply.  Measured at 256 rows, with one fp16 number per weight: two groups of four waves that reconstruct and
// multiply in turn 124 us, eight alike 104, four that reconstruct for eight 86, and with a tile's weights computed between the last one's
// products and rows written in whole lines 64.  64 columns per wave spill (247 us).
//
// The weights enter the second product as fp16 pairs, 22 bits, whatever the number of rows.  One fp16 number each, 11 bits, would take
// 63 us instead of 74 at 256 rows x 128, 42 instead of 47 x 64, 51 instead of 54 at 96 rows x 128, and a row in which one token has nearly all
// of the weight would be off by up to 2^-11 of it besides the result's own rounding.
#include "hqmq_limits.h"
#include "hqmq_packed.h"

namespace hqmq {

namespace {

constexpr int kMakers = 256;        // threads that fetch and reconstruct tiles: four waves
constexpr int kLoads = 3;           // code words of a tile and side per thread
constexpr int kPay = 128;           // outlier payloads of a tile and side kept in LDS

// Tokens of a tile: 1024 chunks of K and of V (24 chunks per row: 768), four for each of a side's threads.
template <int kNc>
constexpr int tile_tokens() { return kNc == 16 ? 64 : 32; }
template <int kNc>
constexpr int key_pitch() { return 4 * kNc + 8; }  // halves; an odd number of 16-byte slots: rows fall on all banks
template <int kNc>
constexpr int value_pitch() { return tile_tokens<kNc>() + 8; }

// A tile in LDS, in 32-bit words: keys [tokens][key_pitch] halves; values [D rows][value_pitch] halves
template <int kNc>
struct TileLds {
    static constexpr int keys = tile_tokens<kNc>() * key_pitch<kNc>() / 2;
    static constexpr int values = 4 * kNc * value_pitch<kNc>() / 2;
    static_assert(keys % 4 == 0 && values % 4 == 0, "16-byte accesses");
    // of a form with so many tiles in flight: of two, the values one longer
    __host__ __device__ static constexpr int value_bufs(int bufs) { return bufs == 2 ? 3 : 1; }
    __host__ __device__ static constexpr int total(int bufs) { return bufs * keys + value_bufs(bufs) * values; }
};
// A tile's packed rows of one side: code words (room for the largest w) | flags, scales, places in the outlier list's window | payloads,
// with a slot past the last that is read and not used | whether the tile wants care, the window's first entry
template <int kNc>
struct StageLds {
    static constexpr int kTok = tile_tokens<kNc>();
    static constexpr int words = kLoads * kMakers;
    static_assert(kTok * (kNc * 24 / 32) <= words, "w <= 24");
    static constexpr int pays = words + 3 * kTok;
    static constexpr int about = pays + 2 * kPay + 2;
    static constexpr int total = about + 2;
    static_assert(words % 4 == 0 && kTok % 4 == 0 && total % 4 == 0, "16-byte reads");
};

// Row of V^T in LDS for component e of chunk c: blocks of 32 rows are the operands of one product; in a product's result a lane
// then holds all four components of a chunk.
__device__ __forceinline__ int value_row(int c, int e) { return 32 * (c >> 3) + 8 * e + (c & 7); }

// How a workgroup works: waves that multiply, query rows (columns) of each, tiles in LDS, waves per SIMD.  With one tile in LDS four
// waves reconstruct a tile and then multiply it, and the workgroups that share a compute unit fill each other's waits; with two, four
// waves more reconstruct the next tile while these multiply.
// By rows of a kv head: 16 columns per wave and three workgroups per compute unit up to 64 (two per compute unit, which spills nothing:
// 24 rows x 64 27.5 -> 30 us, 12 x 96 25.2 -> 26.6, 130 tokens 6.8 -> 6.2), 32 columns up to 128, two tiles and eight waves of them above;
// more than 256 rows are blocks of 256, each with a reconstruction of its own.
// Both sides, 8 heads x 32768 x 128 in us: 48 rows small 49.3, middle 51.8; 64 rows 51.5, 51.9 (x 64: 33.1, 34.1); 65 rows 77.3, 52.3.
// Middle / large: 65 rows 52.4 / 51.7, 128 rows 57.4 / 55.2 and, 128 rows, 8 x 2000 x 128 27.2 / 22.8, but 320 heads of 500 tokens 48.7 / 56.5, of 80
// rows 46.6 / 54.9, 512 heads of 300 x 64 20.9 / 27.0, 8 of 500 13.2 / 14.5: two workgroups per compute unit take many heads and few tiles better.
// 129 rows 86.7 / 62.0, 256 94.3 / 73.0.  Blocks of 256: 257 rows 110, 384 115, 512 127, 1024 240.
template <int kTakers_, int kCols_, int kBufs_, int kPerSimd_>
struct Form {
    static constexpr int kTakers = kTakers_, kCols = kCols_, kBufs = kBufs_, kPerSimd = kPerSimd_;
    static constexpr int kThreads = 64 * kTakers + (kBufs == 2 ? kMakers : 0);
    static constexpr bool kTogether = kBufs == 1 && kCols == 16;  // a launch may hold prefixes and own tokens
};
using FormSmall = Form<4, 16, 1, 3>;
using FormMiddle = Form<4, 32, 1, 2>;
using FormLarge = Form<8, 32, 2, 3>;

}  // namespace

template <int kNc, bool kTable, bool kPow2, typename F>
__global__ __launch_bounds__(F::kThreads, F::kPerSimd) void k_shared(Geometry g, SharedArgs a, SharedArgs own, int n_first)
{
    int block = (int)blockIdx.x;
    if (F::kTogether && block >= n_first) {  // uniform
        block -= n_first;
        a = own;
    }
    const int split = block % a.n_splits, seg = block / a.n_splits;
    using Tile = TileLds<kNc>;
    using Stage = StageLds<kNc>;
    constexpr int kTok = tile_tokens<kNc>(), kD = 4 * kNc;
    constexpr int kCols = F::kCols, kBufs = F::kBufs, kThreads = F::kThreads, kWaves = kThreads / 64;
    constexpr bool kWide = kCols == 32;           // 32x32x16 products, else 16x16x32
    constexpr int kSteps = kWide ? kD / 16 : kD / 32;
    constexpr int kBlocks = kWide ? kD / 32 : kD / 16;
    constexpr int kRegs = kWide ? 16 : 4;         // of a block's result
    using acc_t = std::conditional_t<kWide, float16_t, float4_t>;
    extern __shared__ __align__(16) float lds[];
    uint32_t *key_tiles = reinterpret_cast<uint32_t *>(lds + kLutFloats + 2 * direction_floats<kTable>(g.S));
    uint32_t *value_tiles = key_tiles + kBufs * Tile::keys;
    uint32_t *stages = key_tiles + Tile::total(kBufs);  // [kBufs][K, V]

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool maker = kBufs == 1 || wave < 4, taker = kBufs == 1 || wave >= 4;  // uniform
    const int st = tid & (kMakers - 1);
    const int b = seg / g.H, h = seg % g.H;
    const uint32_t row_words = kNc == 32 ? (uint32_t)g.w : (uint32_t)g.row_words;
    const uint32_t w = g.w;

    // ---- columns of this wave: query rows r of the kv head ---------------------------------------------------------
    const int n_rows = a.n_share * a.G;
    const int col0 = ((int)blockIdx.z * F::kTakers + (kBufs == 1 ? wave : wave - 4)) * kCols;
    const int col = lane & (kCols - 1);
    const int kgrp = lane / kCols;         // which 8 of a product's terms the lane supplies, which rows of a result it holds
    const bool has_cols = taker && col0 < n_rows;  // uniform
    const uint32_t flip = a.qscale < 0.f ? 0x80008000u : 0u;
    const float qscale = fabsf(a.qscale);  // a negative scale goes into the queries' signs
    const int r = col0 + col;
    const bool there = taker && r < n_rows;
    size_t head;
    {
        const int rr = there ? r : 0, m = rr / a.G;
        head = ((size_t)(b * a.n_share + m) * g.H + h) * a.G + (rr - m * a.G);
    }
    half8_t qf[kSteps];
    {
        const _Float16 *q = a.q + head * kD + 8 * kgrp;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            uint4v v = *reinterpret_cast<const uint4v *>(q + (kWide ? 16 : 32) * s);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = there ? v[i] ^ flip : 0u;
            qf[s] = __builtin_bit_cast(half8_t, v);
        }
    }
    int vis = a.T;
    if (a.visible && there)
        vis = min(seen_tokens(a.visible[head]), a.T);

    build_tables<kTable>(lds, g, a.k.sec + (size_t)h * g.S * 4, a.v.sec + (size_t)h * g.S * 4, 2, tid, kThreads);
    const Decoder<kTable, kPow2> decoder(lds, g);

    // ---- the tiles of this workgroup -----------------------------------------------------------------------------------
    const int begin = split * a.rows_per_split;
    int end = min(a.T, begin + a.rows_per_split);
    int least = a.T;      // every query row of the wave sees the tokens below
    if (a.visible) {      // what no row of the workgroup sees is not read
        int *most_of = reinterpret_cast<int *>(key_tiles);
        int most = there ? vis : 0;
        least = vis;
        for (int d = 32; d > 0; d /= 2) {
            most = max(most, __shfl_xor(most, d));
            least = min(least, __shfl_xor(least, d));
        }
        if (lane == 0)
            most_of[wave] = most;
        __syncthreads();
        most = 0;
        for (int i = 0; i < kWaves; ++i)
            most = max(most, most_of[i]);
        end = __builtin_amdgcn_readfirstlane(min(end, most));
        least = __builtin_amdgcn_readfirstlane(least);
        __syncthreads();
    }
    const int n_tiles = end > begin ? (end - begin + kTok - 1) / kTok : 0;

    float m_ref = kNoToken, l_run = 0.f;
    acc_t acc[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k)
#pragma unroll
        for (int i = 0; i < kRegs; ++i)
            acc[k][i] = 0.f;

    // ---- a tile's packed rows on their way to LDS ------------------------------------------------------------------------
    // Every load is issued a tile's time or more before its value is needed, and without a condition: tokens past the last read as
    // zeros (no flags, a scale of zero) behind the last payload.  The outlier list's bounds come a tile before rows and payloads.
    // Waves 0 and 1 look after K's rows and payloads, 2 and 3 after V's; all of them fetch code words of both.
    const bool of_v = (wave & 2) != 0, row_wave = (wave & 1) == 0;
    const uint32_t n_tok = (uint32_t)max(end - begin, 0);
    const int64_t first_row = (int64_t)seg * a.T + begin;
    const rsrc_t code_k = buffer_of(a.k.codes + first_row * row_words, n_tok * row_words);
    const rsrc_t code_v = buffer_of(a.v.codes + first_row * row_words, n_tok * row_words);
    const rsrc_t flag_b = buffer_of((of_v ? a.v.flags : a.k.flags) + first_row, n_tok);
    const rsrc_t scale_b = buffer_of((of_v ? a.v.sigma : a.k.sigma) + first_row, n_tok);
    const rsrc_t place_b = buffer_of((of_v ? a.v.row_off : a.k.row_off) + first_row, n_tok + 1u);
    const uint2 *const list = reinterpret_cast<const uint2 *>(of_v ? a.v.outliers : a.k.outliers);
    const uint2 *const no_list = reinterpret_cast<const uint2 *>(of_v ? a.v.codes : a.k.codes);  // any two words: a row has three or more
    const uint32_t capacity = (uint32_t)min(of_v ? a.v.outlier_capacity : a.k.outlier_capacity, (uint64_t)0xffffffffu);
    uint32_t code_at = 4u * st, row_at = 4u * (lane & (kTok - 1)), bound_at = (lane & 1) * kTok;
    uint32_t cw[2][kLoads], fw = 0u, ro = 0u, bounds = 0u;
    uint16_t sg = 0u;  // as loaded: widening it before it is staged would wait for it
    uint2 pay = make_uint2(0u, 0u);
    uint32_t next_base = 0u, next_n = 0u, next_in_list = 0u;  // window of the outlier list, of the tile on its way
    auto request_bounds = [&]() {  // even lanes: first entry of the next tile's window, odd ones: the entry behind it
        bounds = __builtin_amdgcn_raw_buffer_load_b32(place_b, 4u * min(bound_at, n_tok), 0, 0);
        bound_at += kTok;
    };
    auto request = [&]() {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            cw[0][i] = __builtin_amdgcn_raw_buffer_load_b32(code_k, code_at + 4u * kMakers * i, 0, 0);
            cw[1][i] = __builtin_amdgcn_raw_buffer_load_b32(code_v, code_at + 4u * kMakers * i, 0, 0);
        }
        fw = __builtin_amdgcn_raw_buffer_load_b32(flag_b, row_at, 0, 0);
        sg = __builtin_amdgcn_raw_buffer_load_b16(scale_b, row_at >> 1, 0, 0);
        ro = __builtin_amdgcn_raw_buffer_load_b32(place_b, min(row_at, 4u * n_tok), 0, 0);
        code_at += 4u * kTok * row_words;
        row_at += 4u * kTok;
        next_base = (uint32_t)__builtin_amdgcn_readlane((int)bounds, 0);
        next_n = (uint32_t)__builtin_amdgcn_readlane((int)bounds, 1) - next_base;
        next_in_list = min(next_n, capacity - min(next_base, capacity));
        const uint2 *src = next_in_list ? list + next_base : no_list;
        pay = src[min((uint32_t)st & (kPay - 1), max(next_in_list, 1u) - 1u)];
    };
    auto stage = [&](int buf) {
        uint32_t *dst = stages + 2 * buf * Stage::total;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            dst[st + kMakers * i] = cw[0][i];
            dst[Stage::total + st + kMakers * i] = cw[1][i];
        }
        uint32_t *mine = dst + (of_v ? Stage::total : 0);
        if (row_wave) {
            uint32_t *rp = mine + Stage::words + (lane & (kTok - 1));
            rp[0] = fw;
            rp[kTok] = (uint32_t)sg;
            rp[2 * kTok] = ro - next_base;
            // what can leave the fp16 range, or payloads past the staged ones, send the tile down a careful form
            const bool care = __any((uint32_t)sg >= kBigScale) || next_n > (uint32_t)kPay;
            *reinterpret_cast<uint2 *>(mine + Stage::about) = make_uint2(care ? 1u : 0u, next_base);
        }
        const uint32_t slot = (uint32_t)st & (kPay - 1);
        reinterpret_cast<uint2 *>(mine + Stage::pays)[slot] = slot < next_in_list ? pay : make_uint2(0u, 0u);
    };

    // ---- reconstruction ----------------------------------------------------------------------------------------------------
    auto read_code = [&](const uint32_t *sp, int row, uint32_t c) {
        const uint32_t bit = c * w;
        const uint32_t *rw = sp + row * row_words + (bit >> 5);
        return __builtin_amdgcn_alignbit(rw[1], rw[0], bit & 31u);
    };
    auto pre = [&](auto fast_tag, const uint32_t *sp, uint32_t code, uint32_t slot) {
        return decoder.template pre<decltype(fast_tag)::value, kPay>(reinterpret_cast<const uint2 *>(sp + Stage::pays), code, slot);
    };
    auto direction = [&](int s, const Chunk &f) { return decoder.direction(s, f); };
    auto finish = [&](auto fast_tag, int s, uint32_t base, const Chunk &f, float4_t d, uint32_t scale, bool flagged) {
        return decoder.template finish<decltype(fast_tag)::value, kPay>(s ? a.v : a.k, base, f, d, scale_value(scale), flagged);
    };
    // A thread's part of a tile: two pairs of neighbouring chunks of K, one chunk of V in four neighbouring tokens.  Threads beyond a
    // tile's last unit (24 chunks per row) do that one again.
    constexpr int kKeyUnits = kTok * kNc / 2, kValueUnits = kTok * kNc / 4;
    static_assert(kKeyUnits <= 2 * kMakers && kValueUnits <= kMakers, "a thread's four chunks of a side");
    // side: 0 keys, 1 values, 2 both at once, for which only waves that do not multiply have the registers
    auto decode = [&](auto side_tag, int buf, int value_buf) {
        constexpr bool kKeys = decltype(side_tag)::value != 1, kValues = decltype(side_tag)::value != 0;
        const uint32_t *sk = stages + 2 * buf * Stage::total, *sv = sk + Stage::total;
        const uint2 about_k = *reinterpret_cast<const uint2 *>(sk + Stage::about), about_v = *reinterpret_cast<const uint2 *>(sv + Stage::about);
        int row[2], c[2];
        uint32_t code[8], word[2], scale[2], off[2];
#pragma unroll
        for (int i = 0; kKeys && i < 2; ++i) {
            const int u = min(st + kMakers * i, kKeyUnits - 1);
            row[i] = u / (kNc / 2);
            c[i] = 2 * (u % (kNc / 2));
            code[2 * i] = read_code(sk, row[i], c[i]);
            code[2 * i + 1] = read_code(sk, row[i], c[i] + 1);
            const uint32_t *rp = sk + Stage::words + row[i];
            word[i] = rp[0];
            scale[i] = rp[kTok];
            off[i] = rp[2 * kTok];
        }
        const int vu = min(st, kValueUnits - 1), vc = vu % kNc, quad = vu / kNc;
        uint4v vword = {}, vscale = {}, voff = {};
        if (kValues) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                code[4 + i] = read_code(sv, 4 * quad + i, vc);
            const uint32_t *vp = sv + Stage::words + 4 * quad;
            vword = *reinterpret_cast<const uint4v *>(vp);
            vscale = *reinterpret_cast<const uint4v *>(vp + kTok);
            voff = *reinterpret_cast<const uint4v *>(vp + 2 * kTok);
        }
        // where the four tokens stand in the order in which a product takes a block of scores as its operand
        const int at = 4 * (kWide ? (quad & ~3) | ((quad & 1) << 1) | ((quad >> 1) & 1) : (quad & ~7) | ((quad & 3) << 1) | ((quad >> 2) & 1));
        _Float16 *keys = reinterpret_cast<_Float16 *>(key_tiles + buf * Tile::keys);
        _Float16 *values = reinterpret_cast<_Float16 *>(value_tiles + value_buf * Tile::values) + value_row(vc, 0) * value_pitch<kNc>() + at;
        const auto form = [&](auto fast_tag) {
            bool flag[4];
            Chunk f[8];
            float4_t d[8];
#pragma unroll
            for (int i = 0; kKeys && i < 2; ++i) {
                flag[2 * i] = (word[i] >> c[i]) & 1u;
                flag[2 * i + 1] = (word[i] >> c[i]) & 2u;
                const uint32_t slot = off[i] + __popc(word[i] & ((1u << c[i]) - 1u));
                f[2 * i] = pre(fast_tag, sk, code[2 * i], slot);
                f[2 * i + 1] = pre(fast_tag, sk, code[2 * i + 1], slot + (flag[2 * i] ? 1u : 0u));
            }
            if (kKeys && kValues)
                __builtin_amdgcn_sched_barrier(0);  // the order of the steps: it is what overlaps their LDS round trips
#pragma unroll
            for (int i = 0; kKeys && i < 4; ++i)
                d[i] = direction(0, f[i]);
#pragma unroll
            for (int i = 0; kValues && i < 4; ++i)
                f[4 + i] = pre(fast_tag, sv, code[4 + i], voff[i] + __popc(vword[i] & ((1u << vc) - 1u)));
            if (kKeys && kValues)
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                if (kKeys) {
                    const uint2 x = finish(fast_tag, 0, about_k.y, f[2 * i], d[2 * i], scale[i], flag[2 * i]);
                    const uint2 y = finish(fast_tag, 0, about_k.y, f[2 * i + 1], d[2 * i + 1], scale[i], flag[2 * i + 1]);
                    *reinterpret_cast<uint4v *>(keys + row[i] * key_pitch<kNc>() + 4 * c[i]) = uint4v{x.x, x.y, y.x, y.y};
                }
                if (kValues) {
                    d[4 + 2 * i] = direction(1, f[4 + 2 * i]);
                    d[5 + 2 * i] = direction(1, f[5 + 2 * i]);
                }
                if (kKeys && kValues)
                    __builtin_amdgcn_sched_barrier(0);
            }
            if (!kValues)
                return;
            uint2 v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] = finish(fast_tag, 1, about_v.y, f[4 + i], d[4 + i], vscale[i], (vword[i] >> vc) & 1u);
            const uint32_t lo = 0x05040100u, hi = 0x07060302u;
            const auto put = [&](int e, uint32_t x, uint32_t y) {
                *reinterpret_cast<uint2 *>(values + 8 * e * value_pitch<kNc>()) = make_uint2(x, y);
            };
            put(0, __builtin_amdgcn_perm(v[1].x, v[0].x, lo), __builtin_amdgcn_perm(v[3].x, v[2].x, lo));
            put(1, __builtin_amdgcn_perm(v[1].x, v[0].x, hi), __builtin_amdgcn_perm(v[3].x, v[2].x, hi));
            put(2, __builtin_amdgcn_perm(v[1].y, v[0].y, lo), __builtin_amdgcn_perm(v[3].y, v[2].y, lo));
            put(3, __builtin_amdgcn_perm(v[1].y, v[0].y, hi), __builtin_amdgcn_perm(v[3].y, v[2].y, hi));
        };
        if (__builtin_amdgcn_readfirstlane((int)((kKeys ? about_k.x : 0u) | (kValues ? about_v.x : 0u))) == 0)
            form(std::true_type{});
        else
            form(std::false_type{});
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
    constexpr int kS = kWide ? 16 : 8;  // scores of a lane and 32 tokens; wide: token 8 (i / 4) + 4 kgrp + i % 4; else 16 (i / 4) + 4 kgrp + i % 4
    constexpr int kU = kWide ? 2 : 1;   // products of 32 tokens' values per block
    half8_t held[2][kU] = {};           // two tiles in LDS: the last tile's weights, whose values are still to come
    // Weights enter the products as pairs of fp16 values: 22 bits.
    const auto set_pairs = [](half8_t (*to)[kU], int i, float p0, float p1) {  // of weights i and i + 1
        typedef float float2_t __attribute__((ext_vector_type(2)));
        typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
        const half2_t hi = __builtin_convertvector(float2_t{p0, p1}, half2_t);
        const uint32_t both = __builtin_bit_cast(uint32_t, hi);
        float r0, r1;  // p - hi in one instruction each; the compiler converts first
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r0) : "v"(both), "v"(p0));
        asm("v_fma_mix_f32 %0, %1, -1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r1) : "v"(both), "v"(p1));
        const half2_t lo = __builtin_convertvector(float2_t{r0, r1}, half2_t);
        to[0][i >> 3][i & 7] = hi[0];
        to[0][i >> 3][(i & 7) + 1] = hi[1];
        to[1][i >> 3][i & 7] = lo[0];
        to[1][i >> 3][(i & 7) + 1] = lo[1];
    };
    // Scores of 32 tokens from t0 on, the factor that is still missing from them, and m_ref raised if need be.
    // Weights are 2^(s - m_ref): with m_ref some 10 below the largest score seen they reach 2^10, their fp16 values are normal numbers
    // down to 2^-24 of the largest, and m_ref is raised (and what was summed scaled) only when a score would pass 2^15, so hardly
    // ever after the first tiles.  It is a whole number: scaling by a power of two rounds nothing, but for held weights that become
    // subnormal fp16 numbers: these are off by 2^-25 at most, 2^-34 of the largest weight.
    auto scores = [&](const _Float16 *keys, int t0, float *s) {
        if constexpr (kWide) {
            float16_t sc = float16_t{0.f};
            const _Float16 *kp = keys + (lane & 31) * key_pitch<kNc>() + 8 * kgrp;
#pragma unroll
            for (int x = 0; x < kSteps; ++x)
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8_t *>(kp + 16 * x), qf[x], sc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                s[i] = sc[i];
        } else {
            float4_t sc[2] = {float4_t{0.f, 0.f, 0.f, 0.f}, float4_t{0.f, 0.f, 0.f, 0.f}};
            const _Float16 *kp = keys + (lane & 15) * key_pitch<kNc>() + 8 * kgrp;
#pragma unroll
            for (int x = 0; x < kSteps; ++x)
#pragma unroll
                for (int u = 0; u < 2; ++u)
                    sc[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(*reinterpret_cast<const half8_t *>(kp + 16 * u * key_pitch<kNc>() + 32 * x),
                                                                   qf[x], sc[u], 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                s[i] = sc[i >> 2][i & 3];
        }
        float mul = qscale;
        if (t0 + 32 > end || t0 + 32 > least) {  // uniform: some query row does not see every token
            const int seen = min(end, vis) - t0 - 4 * kgrp;
#pragma unroll
            for (int i = 0; i < kS; ++i)
                s[i] = (kWide ? 8 : 16) * (i >> 2) + (i & 3) < seen ? s[i] * qscale : 3.f * kNoToken;
            mul = 1.f;
        }
        float top = s[0];
#pragma unroll
        for (int i = 1; i < kS; ++i)
            top = fmaxf(top, s[i]);
        top = over_lanes(top * mul, [](float x, float y) { return fmaxf(x, y); });
        const bool raise = top - m_ref > kRise;
        if (__any(raise)) {
            const float m_new = raise ? ceilf(top) - kTop : m_ref;
            const float corr = __builtin_amdgcn_exp2f(m_ref - m_new);
            m_ref = m_new;
            l_run *= corr;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                for (int i = 0; i < kRegs; ++i)
                    acc[k][i] *= corr;
            if constexpr (kBufs == 2)  // in fp32: the factor alone may be less than any fp16 number, or a coarse one
#pragma unroll
                for (int i = 0; i < kS; i += 2) {
                    const half8_t hi = held[0][i >> 3], lo = held[1][i >> 3];
                    set_pairs(held, i, ((float)hi[i & 7] + (float)lo[i & 7]) * corr, ((float)hi[(i & 7) + 1] + (float)lo[(i & 7) + 1]) * corr);
                }
        }
        return mul;
    };
    auto value_operand = [&](const _Float16 *values, int k, int u) {
        return *reinterpret_cast<const half8_t *>(values + ((kWide ? 32 : 16) * k + (lane & (kWide ? 31 : 15))) * value_pitch<kNc>() + 8 * kgrp + 16 * u);
    };
    auto multiply = [&](half8_t v, half8_t p, int k) {
        if constexpr (kWide)
            acc[k] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v, p, acc[k], 0, 0, 0);
        else
            acc[k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p, acc[k], 0, 0, 0);
    };
    auto weights = [&](const float *s, float mul, int i, half8_t (*to)[kU]) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(s[i], mul, -m_ref)), p1 = __builtin_amdgcn_exp2f(fmaf(s[i + 1], mul, -m_ref));
        l_run += p0;
        l_run += p1;
        set_pairs(to, i, p0, p1);
    };
    // One tile in LDS: scores, weights, products with the values.
    auto attend = [&](int j) {
#pragma unroll
        for (int sub = 0; sub < kTok; sub += 32) {
            float s[kS];
            const float mul = scores(reinterpret_cast<const _Float16 *>(key_tiles) + sub * key_pitch<kNc>(), begin + j * kTok + sub, s);
            half8_t p[2][kU];
#pragma unroll
            for (int i = 0; i < kS; i += 2)
                weights(s, mul, i, p);
            const _Float16 *values = reinterpret_cast<const _Float16 *>(value_tiles) + sub;
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                half8_t v[kBlocks];
#pragma unroll
                for (int k = 0; k < kBlocks; ++k)
                    v[k] = value_operand(values, k, u);
#pragma unroll
                for (int half = 0; half < 2; ++half)
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k)
                        multiply(v[k], p[half][u], k);
            }
        }
    };
    // Two tiles: the weights of these 32 tokens between the products of the last ones' with their values, so that vector and matrix
    // instructions issue side by side.
    auto attend_held = [&](const _Float16 *keys, const _Float16 *last_values, int t0, bool first) {
        float s[kS];
        const float mul = scores(keys, t0, s);
        half8_t next[2][kU];
        if (first) {
#pragma unroll
            for (int i = 0; i < kS; i += 2)
                weights(s, mul, i, next);
        } else {
#pragma unroll
            for (int n = 0; n < kU * kBlocks; ++n) {
                const int u = n / kBlocks, k = n % kBlocks;
                const half8_t v = value_operand(last_values, k, u);
                multiply(v, held[0][u], k);
                const int i0 = 2 * (n * kS / 2 / (kU * kBlocks)), i1 = 2 * ((n + 1) * kS / 2 / (kU * kBlocks));
#pragma unroll
                for (int i = i0; i < i1; i += 2)
                    weights(s, mul, i, next);
                multiply(v, held[1][u], k);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int u = 0; u < kU; ++u)
                held[half][u] = next[half][u];
    };

    // ---- the loop -------------------------------------------------------------------------------------------------------------
    if (maker && n_tiles > 0) {
        request_bounds();
        request();
        request_bounds();
        stage(0);
        request();
        request_bounds();
    }
    lds_barrier();
    if constexpr (kBufs == 1) {
        for (int j = 0; j < n_tiles; ++j) {
            decode(std::integral_constant<int, 0>{}, 0, 0);
            decode(std::integral_constant<int, 1>{}, 0, 0);
            lds_barrier();
            if (has_cols)
                attend(j);
            stage(0);
            request();
            request_bounds();
            lds_barrier();
        }
    } else if (maker) {
        if (n_tiles > 0) {
            decode(std::integral_constant<int, 2>{}, 0, 0);
            stage(1);
            request();
            request_bounds();
        }
        lds_barrier();
        int v = 0;
        for (int j = 1; j <= n_tiles; ++j) {  // past the last tile: zeros, which nothing reads
            v = v == 2 ? 0 : v + 1;
            decode(std::integral_constant<int, 2>{}, j & 1, v);
            stage((j + 1) & 1);
            request();
            request_bounds();
            lds_barrier();
        }
    } else {
        const _Float16 *keys = reinterpret_cast<const _Float16 *>(key_tiles), *values = reinterpret_cast<const _Float16 *>(value_tiles);
        const _Float16 *last = values;
        lds_barrier();
        int v = 0;
        for (int j = 0; j < n_tiles; ++j) {
            const _Float16 *kt = keys + 2 * (j & 1) * Tile::keys, *vt = values + 2 * v * Tile::values;
            if (has_cols) {
#pragma unroll
                for (int sub = 0; sub < kTok; sub += 32)
                    attend_held(kt + sub * key_pitch<kNc>(), sub ? vt + sub - 32 : last, begin + j * kTok + sub, j == 0 && sub == 0);
            }
            last = vt + kTok - 32;
            v = v == 2 ? 0 : v + 1;
            lds_barrier();
        }
        if (has_cols && n_tiles > 0)
#pragma unroll
            for (int n = 0; n < kU * kBlocks; ++n)
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    multiply(value_operand(last, n % kBlocks, n / kBlocks), held[half][n / kBlocks], n % kBlocks);
    }
    if constexpr (kBufs == 2)
        lds_barrier();  // what follows is written over the last values, which slower waves may still read

    // ---- the wave's columns of this share: through LDS, so that a row's sums leave in whole lines -------------------------------------
    l_run = over_lanes(l_run, [](float x, float y) { return x + y; });
    if (!has_cols)
        return;
    // The only share writes the result itself: 256 x 8 heads of 64 tokens x 64, 64 rows, 25 us instead of 101 with partial sums and the merge.
    const float factor = !a.out ? 1.f : l_run > 0.f ? 1.f / l_run : 0.f;  // a row that saw no token: zeros
    if (a.out) {
        if (there && kgrp == 0 && a.lse)
            a.lse[head] = l_run > 0.f ? (m_ref + __builtin_amdgcn_logf(l_run)) * 0.693147180559945309417f : -__builtin_inff();
    } else if (there && kgrp == 0) {
        float *ml = a.part_ml + 2 * (head * a.part_pitch + a.split0 + split);
        ml[0] = m_ref;
        ml[1] = l_run;
    }
    constexpr int kPitch = 32 + 4;  // 32 dimensions, a line of 128 bytes, at a time
    float *out = reinterpret_cast<float *>(key_tiles) + (kBufs == 1 ? wave : wave - 4) * kCols * kPitch;  // tiles and packed rows are done with
#pragma unroll
    for (int part = 0; part < kD / 32; ++part) {
        constexpr int kOf = kWide ? 1 : 2;  // blocks of a part
#pragma unroll
        for (int k = 0; k < kOf; ++k)
#pragma unroll
            for (int i = 0; i < kRegs; ++i) {
                const int row = kWide ? 8 * (i >> 2) + 4 * kgrp + (i & 3) : 16 * k + 4 * kgrp + i;  // 8 e + c % 8
                out[col * kPitch + 4 * (row & 7) + (row >> 3)] = acc[kOf * part + k][i] * factor;
            }
        wave_lds_sync();
#pragma unroll
        for (int i = lane; i < kCols * 8; i += 64) {
            const int c = i >> 3, d = 4 * (i & 7), rr = col0 + c;
            if (rr < n_rows) {
                const int m = rr / a.G;
                const size_t hd = ((size_t)(b * a.n_share + m) * g.H + h) * a.G + (rr - m * a.G);
                if (a.out) {
                    const float4_t x = *reinterpret_cast<const float4_t *>(out + c * kPitch + d);
                    half4_t y;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        y[e] = (_Float16)x[e];
                    *reinterpret_cast<half4_t *>(a.out + hd * kD + 32 * part + d) = y;
                    continue;
                }
                *reinterpret_cast<float4_t *>(a.part_acc + (hd * a.part_pitch + a.split0 + split) * 128 + 32 * part + d) =
                    *reinterpret_cast<const float4_t *>(out + c * kPitch + d);
            }
        }
        wave_lds_sync();
    }
}

bool shared_is_small(int n_rows) { return n_rows <= 64; }

namespace {

enum SharedForm { kSmall, kMiddle, kLarge };  // up to 64, 128 and 256 query rows per workgroup
struct SharedChoice {
    SharedForm form;
    bool table;
    int rows, threads, resident;  // query rows and threads of a workgroup, workgroups of a compute unit
    size_t lds;
};
SharedChoice choose_shared(const Geometry &g, int n_rows)
{
    SharedChoice c;
    c.form = shared_is_small(n_rows) ? kSmall : n_rows <= 128 ? kMiddle : kLarge;
    int most = 0;
    const auto fit = [&](auto lds, size_t table_room) {
        c.table = lds(true) <= table_room;
        c.lds = lds(c.table);
        c.resident = (int)(kLdsPerCu / c.lds);
        c.resident = c.resident < most ? c.resident : most;
    };
    c.rows = c.form == kSmall ? 64 : c.form == kMiddle ? 128 : 256;
    c.threads = c.form == kLarge ? FormLarge::kThreads : c.form == kMiddle ? FormMiddle::kThreads : FormSmall::kThreads;
    most = c.form == kSmall ? FormSmall::kPerSimd : c.form == kMiddle ? FormMiddle::kPerSimd : 1;
    const int bufs = c.form == kLarge ? FormLarge::kBufs : 1;
    const int tile = g.n_c == 32 ? TileLds<32>::total(bufs) : g.n_c == 24 ? TileLds<24>::total(bufs) : TileLds<16>::total(bufs);
    const int stage = g.n_c == 32 ? StageLds<32>::total : g.n_c == 24 ? StageLds<24>::total : StageLds<16>::total;
    fit([&](bool table) {
        return (kLutFloats + 2 * (table ? direction_floats<true>(g.S) : direction_floats<false>(g.S)) + tile + (size_t)bufs * 2 * stage) * sizeof(float);
    }, c.form == kLarge ? kLdsPerCu : kLdsPerCu / 2);
    return c;
}

template <int kNc, typename F>
const void *shared_kernel(bool table, bool pow2)
{
    if (!table)
        return reinterpret_cast<const void *>(&k_shared<kNc, false, false, F>);
    return pow2 ? reinterpret_cast<const void *>(&k_shared<kNc, true, true, F>) : reinterpret_cast<const void *>(&k_shared<kNc, true, false, F>);
}
template <int kNc>
const void *shared_kernel(SharedForm form, bool table, bool pow2)
{
    return form == kSmall ? shared_kernel<kNc, FormSmall>(table, pow2) : form == kMiddle ? shared_kernel<kNc, FormMiddle>(table, pow2)
                                                                                          : shared_kernel<kNc, FormLarge>(table, pow2);
}
const void *shared_kernel(int n_c, SharedForm form, bool table, bool pow2)
{
    return n_c == 32 ? shared_kernel<32>(form, table, pow2) : n_c == 24 ? shared_kernel<24>(form, table, pow2) : shared_kernel<16>(form, table, pow2);
}

}  // namespace

SharedPlan plan_shared(const Geometry &g, int G, int n_share, bool alone)
{
    const SharedChoice c = choose_shared(g, G * n_share);
    const int tok = g.n_c == 16 ? tile_tokens<16>() : tile_tokens<32>();
    const int64_t per = (int64_t)g.B * g.H * ((G * n_share + c.rows - 1) / c.rows), tiles = (g.T + tok - 1) / tok;
    int64_t want = (int64_t)256 * c.resident / per;  // what the chip holds at once
    want = want > kMostSharedSplits ? kMostSharedSplits : want;
    if (alone && tiles <= kTilesAlone)
        want = 1;
    want = want < 1 ? 1 : want < tiles ? want : tiles;
    const int64_t tiles_per = (tiles + want - 1) / want;
    return {(int32_t)((tiles + tiles_per - 1) / tiles_per), (int32_t)(tiles_per * tok)};
}

hipError_t prepare_shared_kernels()
{
    for (int n_c : {32, 24, 16})
        for (SharedForm form : {kSmall, kMiddle, kLarge})
            for (int t = 0; t < 3; ++t) {
                const hipError_t err = hipFuncSetAttribute(shared_kernel(n_c, form, t > 0, t > 1), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsPerCu);
                if (err != hipSuccess)
                    return err;
            }
    return hipSuccess;
}

hipError_t launch_shared(const Geometry &g, const SharedArgs &a, const SharedArgs *own, hipStream_t stream)
{
    if (g.D != 128 && g.D != 96 && g.D != 64)
        return hipErrorInvalidValue;
    const int n_rows = a.G * a.n_share;
    const SharedChoice c = choose_shared(g, n_rows);
    if (own && c.form != kSmall)
        return hipErrorInvalidValue;
    int n_first = a.n_splits * g.B * g.H;
    const int n_own = own ? own->n_splits * g.B * a.n_share * g.H : 0;
    const dim3 grid((unsigned)(n_first + n_own), 1, (unsigned)((n_rows + c.rows - 1) / c.rows));
    Geometry gc = g;
    SharedArgs ac = a, oc = own ? *own : a;
    void *args[] = {&gc, &ac, &oc, &n_first};
    return hipLaunchKernel(shared_kernel(g.n_c, c.form, c.table, (g.S & (g.S - 1)) == 0), grid, dim3(c.threads), args, c.lds, stream);
}

}  // namespace hqmq
