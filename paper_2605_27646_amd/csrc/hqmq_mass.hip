// The attention weight that cached tokens accumulate (include/hqmq_serve.h, hqmq_attend_mass): a token's weights
// e^{scale <q, K_hat_t> - lse} summed over the query rows of its kv head.
//
// A wave takes 32 tokens of its own: every lane reconstructs half a key (lane (token l % 32, half l / 32) the chunks kM half ..
// kM half + kM - 1), which is the operand of v_mfma_f32_32x32x16_f16 as it stands and stays in registers while the query rows go past
// in blocks of 32 from LDS.  With the rows as the other operand a lane receives the scores of one token, so that their weights are
// summed in it, in one fixed order.
//
// One pass over the keys; no wave waits for another but for the tables and the query rows.  Bound by latency for short caches (8 heads of
// 777 tokens 6 us: launch, tables, one tile), by vector instructions for few rows (8 heads x 32768 x 128, 4 rows a head: 15.5 us, 25.6 MB at
// 1.65 TB/s; most of them reconstruct) and by the exponentials for many (16 heads of 8001 tokens x 64, 128 rows: 11.5 us).
//
// The exponent is fma(score, scale, -lse), small wherever the weight is not, and only then taken to base 2: with log2 e inside the scale
// and inside lse, each rounded once, the weights of a row whose scores are near 50 were off by 1e-6, the same way in all of them.
#include "hqmq_packed.h"

namespace hqmq {

namespace {

constexpr int kMassWaves = 16, kMassThreads = 64 * kMassWaves;
constexpr int kMassRows = 128;   // query rows in LDS at a time
constexpr int kMassPay = 64;     // outlier payloads of a wave's 32 tokens kept in LDS
constexpr float kLog2e = 1.44269504088896340736f;

// A wave's packed rows in LDS, in words: code words (room for the largest w) | flags, scales, places in the outlier list's window |
// payloads, with a slot past the last that is read and not used
template <int kNc>
struct MassStage {
    static constexpr int kLoads = (24 * kNc + 63) / 64;
    static constexpr int rows = 64 * kLoads + 4, pays = rows + 96, total = pays + 2 * kMassPay + 4;
};

}  // namespace

template <int kNc, bool kTable, bool kPow2>
__global__ __launch_bounds__(kMassThreads, 4) void k_mass(Geometry g, MassArgs a, int tiles_per_split)
{
    using Stage = MassStage<kNc>;
    constexpr int kD = 4 * kNc, kM = kNc / 2, kQPitch = kD + 8;
    extern __shared__ __align__(16) float lds[];
    _Float16 *queries = reinterpret_cast<_Float16 *>(lds + kLutFloats + direction_floats<kTable>(g.S));  // [kMassRows][kQPitch]
    float *row_lse = reinterpret_cast<float *>(queries + kMassRows * kQPitch);                           // [kMassRows]
    int *row_vis = reinterpret_cast<int *>(row_lse + kMassRows);                                         // [kMassRows]
    int *row_limits = row_vis + kMassRows;  // [kMassRows / 64]: whether row_vis counts for any of these rows
    uint32_t *stages = reinterpret_cast<uint32_t *>(row_limits + kMassRows / 64 + 2);  // aligned to 16 bytes

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int seg = blockIdx.y, b = seg / g.H, h = seg % g.H;
    const uint32_t row_words = kNc == 32 ? (uint32_t)g.w : (uint32_t)g.row_words, w = g.w;
    uint32_t *mine = stages + wave * Stage::total;
    const uint2 *pays = reinterpret_cast<const uint2 *>(mine + Stage::pays);
    const int n_rows = a.n_share * a.G, n_groups = (n_rows + kMassRows - 1) / kMassRows;
    const float scale = fabsf(a.scale);  // a negative scale goes into the queries' signs

    const auto load_rows = [&](int group) {
        const uint32_t flip = a.scale < 0.f ? 0x80008000u : 0u;
        const int first = group * kMassRows, n = min(n_rows - first, kMassRows);
        const auto head_of = [&](int r) {
            const int m = (first + r) / a.G;
            return ((size_t)(b * a.n_share + m) * g.H + h) * a.G + (first + r - m * a.G);
        };
        const int padded = (n + 31) / 32 * 32;
        for (int i = tid; i < padded * (kD / 8); i += kMassThreads) {
            const int r = i / (kD / 8), d = 8 * (i % (kD / 8));
            uint4v q = uint4v{0u, 0u, 0u, 0u};
            if (r < n)
                q = *reinterpret_cast<const uint4v *>(a.q + head_of(r) * kD + d);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                q[e] ^= flip;
            *reinterpret_cast<uint4v *>(queries + r * kQPitch + d) = q;
        }
        if (tid < kMassRows) {  // whole waves
            // Rows that are not there, and those that saw nothing (an lse of minus infinity), see no token: a weight of zero would
            // not do, as their score is not a number where the key is not finite.
            float lse = 0.f;
            int vis = 0;
            if (tid < n) {
                lse = a.lse[head_of(tid)];
                vis = a.visible ? a.visible[head_of(tid)] : g.T;
                if (lse == -__builtin_inff()) {
                    lse = 0.f;
                    vis = 0;
                }
            }
            row_lse[tid] = lse;
            row_vis[tid] = vis;
            const bool some = ballot(vis < g.T) != 0ull;
            if (lane == 0)
                row_limits[wave] = some;
        }
    };

    // ---- this wave's tiles ------------------------------------------------------------------------------------------------
    const int first_tile = (int)blockIdx.x * tiles_per_split;
    const int n_tiles = min((g.T + 31) / 32 - first_tile, tiles_per_split);
    const int64_t first_row = (int64_t)seg * g.T + 32 * (int64_t)first_tile;
    const uint32_t n_tok = (uint32_t)min(g.T - 32 * first_tile, 32 * tiles_per_split);
    // Tokens past the last read as zeros (no flags, a scale of zero) behind the last payload; every load is issued a tile's time before its value is needed.
    const rsrc_t codes = buffer_of(a.k.codes + first_row * row_words, n_tok * row_words);
    const rsrc_t flags_b = buffer_of(a.k.flags + first_row, n_tok);
    const rsrc_t scales = buffer_of(a.k.sigma + first_row, n_tok);
    const rsrc_t places = buffer_of(a.k.row_off + first_row, n_tok + 1u);
    const uint2 *const list = reinterpret_cast<const uint2 *>(a.k.outliers);
    const uint2 *const no_list = reinterpret_cast<const uint2 *>(a.k.codes);  // any two words: a row has three or more
    const uint32_t capacity = (uint32_t)min(a.k.outlier_capacity, (uint64_t)0xffffffffu);
    uint32_t code_at = 4u * (32u * row_words * wave + lane), row_at = 4u * (32u * wave + (lane & 31)), bound_at = 32u * (wave + (lane & 1));
    uint32_t cw[Stage::kLoads], fw, ro, bounds, next_base, next_n, next_in_list;
    uint16_t sg;  // as loaded: widening it before it is staged would wait for it
    uint2 pay;
    const auto request_bounds = [&]() {  // even lanes: first entry of the next tile's window, odd ones: the entry behind it
        bounds = __builtin_amdgcn_raw_buffer_load_b32(places, 4u * min(bound_at, n_tok), 0, 0);
        bound_at += 32u * kMassWaves;
    };
    const auto request = [&]() {
#pragma unroll
        for (int i = 0; i < Stage::kLoads; ++i)
            cw[i] = __builtin_amdgcn_raw_buffer_load_b32(codes, code_at + 256u * i, 0, 0);
        fw = __builtin_amdgcn_raw_buffer_load_b32(flags_b, row_at, 0, 0);
        sg = __builtin_amdgcn_raw_buffer_load_b16(scales, row_at >> 1, 0, 0);
        ro = __builtin_amdgcn_raw_buffer_load_b32(places, min(row_at, 4u * n_tok), 0, 0);
        code_at += 4u * 32u * kMassWaves * row_words;
        row_at += 4u * 32u * kMassWaves;
        next_base = (uint32_t)__builtin_amdgcn_readlane((int)bounds, 0);
        next_n = (uint32_t)__builtin_amdgcn_readlane((int)bounds, 1) - next_base;
        next_in_list = min(next_n, capacity - min(next_base, capacity));
        const uint2 *src = next_in_list ? list + next_base : no_list;
        pay = src[min((uint32_t)lane, max(next_in_list, 1u) - 1u)];
    };
    request_bounds();
    request();
    request_bounds();
    build_tables<kTable>(lds, g, a.k.sec + (size_t)h * g.S * 4, nullptr, 1, tid, kMassThreads);
    load_rows(0);
    const Decoder<kTable, kPow2> decoder(lds, g);
    lds_barrier();
    if (n_groups == 1 && wave >= n_tiles)
        return;  // no tile, and no more barriers

    half8_t key[kM / 2];
    const auto reconstruct = [&]() {
#pragma unroll
        for (int i = 0; i < Stage::kLoads; ++i)
            mine[lane + 64 * i] = cw[i];
        if (lane < 32) {
            uint32_t *rp = mine + Stage::rows + lane;
            rp[0] = fw;
            rp[32] = (uint32_t)sg;
            rp[64] = ro - next_base;
        }
        reinterpret_cast<uint2 *>(mine + Stage::pays)[lane] = (uint32_t)lane < next_in_list ? pay : make_uint2(0u, 0u);
        // what can leave the fp16 range, or payloads past the staged ones, send the tile down a careful form
        const bool care = __any((uint32_t)sg >= kBigScale) || next_n > (uint32_t)kMassPay;
        const uint32_t base = next_base;
        request();
        request_bounds();
        wave_lds_sync();
        int row = lane & 31, half = lane >> 5;
        asm volatile("" : "+v"(row), "+v"(half));  // the addresses of the chunks are not kept through the loop
        const uint32_t c0 = (uint32_t)(kM * half), word = mine[Stage::rows + row], flags = word >> c0;
        const float sigma = scale_value(mine[Stage::rows + 32 + row]);
        uint32_t slot = mine[Stage::rows + 64 + row] + __popc(word & ((1u << c0) - 1u));
        const uint32_t *rw = mine + row * row_words;
        const uint32_t bit0 = c0 * w;
        constexpr int kBatch = 4;
#pragma unroll
        for (int m0 = 0; m0 < kM; m0 += kBatch) {
            Chunk f[kBatch];
            float4_t y[kBatch];
#pragma unroll
            for (int m = 0; m < kBatch; ++m) {
                const uint32_t bit = bit0 + (uint32_t)(m0 + m) * w;
                const uint32_t *at = rw + (bit >> 5);
                f[m] = decoder.template pre<false, kMassPay>(pays, __builtin_amdgcn_alignbit(at[1], at[0], bit), slot);
                slot += (flags >> (m0 + m)) & 1u;
            }
#pragma unroll
            for (int m = 0; m < kBatch; ++m)
                y[m] = decoder.scaled(f[m], decoder.direction(0, f[m]), sigma);
            if (care) {  // uniform and rare
#pragma unroll
                for (int m = 0; m < kBatch; ++m) {
                    y[m] = decoder.saturated(y[m]);
                    if (f[m].slot >= (uint32_t)kMassPay && ((flags >> (m0 + m)) & 1u))
                        f[m].pay = decoder.far_payload(a.k, base, f[m]);
                }
            }
#pragma unroll
            for (int m = 0; m < kBatch; m += 2) {
                const uint2 x = decoder.packed(f[m], y[m], (flags >> (m0 + m)) & 1u), z = decoder.packed(f[m + 1], y[m + 1], (flags >> (m0 + m + 1)) & 1u);
                uint4v both = uint4v{x.x, x.y, z.x, z.y};
                asm volatile("" : "+v"(both));  // here, not where it is used: one batch's registers at a time
                key[(m0 + m) / 2] = __builtin_bit_cast(half8_t, both);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The weights of the rows in LDS, summed over those that this lane has (8 (i / 4) + 4 (lane / 32) + i % 4 of each block).
    const auto weigh = [&](int n, int t) {
        const int half = lane >> 5;
        float sum = 0.f;
        for (int r0 = 0; r0 < n; r0 += 32) {
            const bool limits = __builtin_amdgcn_readfirstlane(row_limits[r0 / 64]) != 0;
            float16_t sc = float16_t{0.f};
            const _Float16 *q = queries + (r0 + (lane & 31)) * kQPitch + 4 * kM * half;
#pragma unroll
            for (int s = 0; s < kM / 2; ++s)
                sc = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const half8_t *>(q + 8 * s), key[s], sc, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r0 + 8 * i >= n)  // uniform
                    break;
                const float4_t lse = *reinterpret_cast<const float4_t *>(row_lse + r0 + 8 * i + 4 * half);
                if (!limits) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        sum += __builtin_amdgcn_exp2f(kLog2e * fmaf(sc[4 * i + e], scale, -lse[e]));
                } else {
                    const int4 vis = *reinterpret_cast<const int4 *>(row_vis + r0 + 8 * i + 4 * half);
                    const int v[4] = {vis.x, vis.y, vis.z, vis.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = __builtin_amdgcn_exp2f(kLog2e * fmaf(sc[4 * i + e], scale, -lse[e]));
                        sum += t < v[e] ? p : 0.f;
                    }
                }
            }
        }
        return sum;
    };
    const auto store = [&](int tile, float sum) {
        const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(y[0]) + __uint_as_float(y[1]);
        const int t = 32 * (first_tile + tile) + (lane & 31);
        if (lane < 32 && t < g.T) {
            const int64_t at = (int64_t)seg * g.T + t;
            a.mass_out[at] = a.mass_in ? fmaf(a.decay, a.mass_in[at], sum) : sum;
        }
    };
    for (int tile0 = 0; tile0 < n_tiles; tile0 += kMassWaves) {  // as often for every wave: with many rows they change hands
        const int tile = tile0 + wave;
        float sum = 0.f;
        reconstruct();  // past the last tile: zeros
        for (int group = 0; group < n_groups; ++group) {
            if (n_groups > 1) {
                lds_barrier();
                load_rows(group);
                lds_barrier();
            }
            sum += weigh(min(n_rows - group * kMassRows, kMassRows), 32 * (first_tile + tile) + (lane & 31));
        }
        if (tile < n_tiles)
            store(tile, sum);
    }
}

namespace {
size_t mass_lds_bytes(const Geometry &g, bool table)
{
    const int stage = g.n_c == 32 ? MassStage<32>::total : g.n_c == 24 ? MassStage<24>::total : MassStage<16>::total;
    return (kLutFloats + (table ? direction_floats<true>(g.S) : direction_floats<false>(g.S)) + (size_t)kMassRows * (g.D + 8) / 2 + 2 * kMassRows + kMassRows / 64 + 2 +
            (size_t)kMassWaves * stage) * sizeof(float);
}
template <int kNc>
const void *mass_kernel(bool table, bool pow2)
{
    if (!table)
        return reinterpret_cast<const void *>(&k_mass<kNc, false, false>);
    return pow2 ? reinterpret_cast<const void *>(&k_mass<kNc, true, true>) : reinterpret_cast<const void *>(&k_mass<kNc, true, false>);
}
const void *mass_kernel(int n_c, bool table, bool pow2)
{
    return n_c == 32 ? mass_kernel<32>(table, pow2) : n_c == 24 ? mass_kernel<24>(table, pow2) : mass_kernel<16>(table, pow2);
}
}  // namespace

hipError_t prepare_mass_kernels()
{
    for (int n_c : {32, 24, 16})
        for (int t = 0; t < 3; ++t) {
            const hipError_t err = hipFuncSetAttribute(mass_kernel(n_c, t > 0, t > 1), hipFuncAttributeMaxDynamicSharedMemorySize, (int)kLdsPerCu);
            if (err != hipSuccess)
                return err;
        }
    return hipSuccess;
}

hipError_t launch_mass(const Geometry &g, const MassArgs &a, hipStream_t stream)
{
    if (g.D != 128 && g.D != 96 && g.D != 64)
        return hipErrorInvalidValue;
    const bool table = mass_lds_bytes(g, true) <= kLdsPerCu, pow2 = (g.S & (g.S - 1)) == 0;
    const int segs = g.B * g.H, tiles = (g.T + 31) / 32;
    int splits = segs < 256 ? 256 / segs : 1;  // one workgroup per compute unit
    splits = splits < tiles ? splits : tiles;
    int per = (tiles + splits - 1) / splits;
    const dim3 grid((unsigned)((tiles + per - 1) / per), (unsigned)segs);
    Geometry gc = g;
    MassArgs ac = a;
    void *args[] = {&gc, &ac, &per};
    return hipLaunchKernel(mass_kernel(g.n_c, table, pow2), grid, dim3(kMassThreads), args, mass_lds_bytes(g, table), stream);
}

}  // namespace hqmq
