// Reconstruction of packed chunks from per-head tables of codeword directions in LDS, for the kernels that serve a batch from
// packed caches.
#pragma once

#include <type_traits>

#include "hqmq_serve_device.h"

namespace hqmq {
namespace {

constexpr float kNoToken = -1.0e30f;     // "no token seen yet": finite, so that differences stay finite
constexpr float kTop = 10.f;             // softmax weights are taken relative to 2^-kTop of the largest score,
constexpr float kRise = 15.f;            // and relative to a newer one once they would pass 2^kRise
constexpr uint32_t kBigScale = 0x77ffu;  // 32752 as fp16 bits: below it no product of a unit codeword leaves the fp16 range

typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));

typedef __amdgpu_buffer_rsrc_t rsrc_t;
// n elements from p on, as a buffer: what lies past them reads as zero
template <typename T>
__device__ __forceinline__ rsrc_t buffer_of(const T *p, uint32_t n) { return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(n * (uint32_t)sizeof(T)), 0x00020000); }

// A barrier for what goes through LDS: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The 24 primaries are +-u w^m with u one of 1, i, j, k, w = (1 + i + j + k) / 2 and m = 0, 1, 2.  A product with u reorders the
// components (e takes that of e ^ u) and flips signs, which costs nothing on the packed fp16 result, rounding being symmetric: two
// byte permutes and two exclusive ors.  So a table of three entries per secondary, w^m (x) q_s, serves all 24.
struct Primary {
    uint32_t m, select, flip_lo, flip_hi;  // select: of the result's first dword; the second's is select ^ 0x04040404
};
struct Primaries {
    Primary p[32];
};
constexpr Primaries make_primaries()
{
    Primaries out{};
    const int w[3][4] = {{2, 0, 0, 0}, {1, 1, 1, 1}, {-1, 1, 1, 1}};                               // twice w^m
    const int sign[4][4] = {{1, 1, 1, 1}, {-1, 1, -1, 1}, {-1, 1, 1, -1}, {-1, -1, 1, 1}};  // of component e ^ u in u (x) x
    for (int p = 0; p < 32; ++p) {
        int P[4] = {0, 0, 0, 0};  // twice the primary
        if (p < 8)
            P[p >> 1] = (p & 1) ? -2 : 2;
        else if (p < 24)
            for (int e = 0; e < 4; ++e)
                P[e] = ((p - 8) >> (3 - e)) & 1 ? -1 : 1;
        out.p[p] = Primary{0u, 0x03020100u, 0u, 0u};  // past the 24: any that stays in the table
        for (int u = 0; p < 24 && u < 4; ++u)
            for (int m = 0; m < 3; ++m)
                for (int s = -1; s < 2; s += 2) {
                    bool same = true;
                    for (int e = 0; e < 4; ++e)
                        same = same && P[e] == s * sign[u][e] * w[m][e ^ u];
                    if (!same)
                        continue;
                    const uint32_t lo = 2u * (0u ^ u), hi = 2u * (1u ^ u);
                    uint32_t flip[2] = {0u, 0u};
                    for (int e = 0; e < 4; ++e)
                        if (s * sign[u][e] < 0)
                            flip[e >> 1] |= 0x8000u << (16 * (e & 1));
                    out.p[p] = Primary{(uint32_t)m, lo | (lo + 1u) << 8 | hi << 16 | (hi + 1u) << 24, flip[0], flip[1]};
                }
    }
    return out;
}
__constant__ const Primaries kPrimaries = make_primaries();

// The tables of a workgroup in LDS: [48] a Primary, with the byte offset of its entries | directions [sides][3 or 1][S][4].  A direction
// is divided by the radius codes' range L, so that a chunk is (radius code * scale, exact in fp32) times it, rounded once; it is taken
// in fp64 and rounded once too.  kTable: three entries per secondary, else the secondaries alone, for codebooks whose table does not fit.
constexpr int kLutFloats = 4 * 48;
template <bool kTable>
__host__ __device__ constexpr size_t direction_floats(int S) { return (size_t)(kTable ? 3 : 1) * S * 4; }

template <bool kTable>
__device__ __forceinline__ void build_tables(float *lds, const Geometry &g, const float *sec_k, const float *sec_v, int sides, int tid, int threads)
{
    const double over_L = 1.0 / (double)((1 << g.b_r) - 1);
    for (int i = tid; i < sides * g.S; i += threads) {
        const bool is_v = i >= g.S;
        const int s = is_v ? i - g.S : i;
        const float4_t q = *reinterpret_cast<const float4_t *>((is_v ? sec_v : sec_k) + 4 * s);
        float4_t *dst = reinterpret_cast<float4_t *>(lds + kLutFloats + (is_v ? direction_floats<kTable>(g.S) : 0)) + s;
        const double x0 = q[0] * over_L, x1 = q[1] * over_L, x2 = q[2] * over_L, x3 = q[3] * over_L;
        dst[0] = float4_t{(float)x0, (float)x1, (float)x2, (float)x3};
        if (kTable) {  // w (x) x = ((1, 1, 1, 1) (x) x) / 2, and w^2 = w - 1
            const double y0 = 0.5 * (x0 - x1 - x2 - x3), y1 = 0.5 * (x0 + x1 - x2 + x3);
            const double y2 = 0.5 * (x0 + x1 + x2 - x3), y3 = 0.5 * (x0 - x1 + x2 + x3);
            dst[g.S] = float4_t{(float)y0, (float)y1, (float)y2, (float)y3};
            dst[2 * g.S] = float4_t{(float)(y0 - x0), (float)(y1 - x1), (float)(y2 - x2), (float)(y3 - x3)};
        }
    }
    if (tid < 48) {
        const Primary p = kPrimaries.p[min(tid, 31)];
        reinterpret_cast<uint4v *>(lds)[tid] = uint4v{kTable ? p.m * (uint32_t)g.S * 16u : p.m, p.select, p.flip_lo, p.flip_hi};
    }
}

// One chunk in three steps, so that the LDS round trips of neighbouring chunks overlap: its primary and payload (pre), the codeword's
// direction (direction), the arithmetic (finish).  code: the chunk's w bits, with others above them.  slot: place in the staged
// window of payloads (kSlots of them and one more that may be read) that the chunk takes if it is flagged.  kFast: nothing can leave the
// fp16 range and the whole window is staged.
struct Chunk {
    uint32_t code, s_idx, slot;
    uint4v l;
    uint2 pay;
};
template <bool kTable, bool kPow2>
struct Decoder {
    const float *lds;
    uint32_t S, w_idx, r_bits, idx_mask, log2_S;
    float inv_S;
    __device__ Decoder(const float *tables, const Geometry &g)
        : lds(tables), S((uint32_t)g.S), w_idx((uint32_t)g.w_idx), r_bits((uint32_t)(g.w - g.w_idx)), idx_mask((1u << g.w_idx) - 1u),
          log2_S((uint32_t)g.log2_S), inv_S(g.inv_S)
    {
    }
    template <bool kFast, int kSlots>
    __device__ __forceinline__ Chunk pre(const uint2 *pays, uint32_t code, uint32_t slot) const
    {
        Chunk f;
        uint32_t p;
        if (kPow2) {
            p = (code >> log2_S) & 31u;
            f.s_idx = code & (S - 1u);
        } else {
            const uint32_t kk = code & idx_mask;
            p = (uint32_t)((float)kk * inv_S);
            f.s_idx = kk - __umul24(p, S);
        }
        f.code = code;
        f.slot = slot;
        f.l = reinterpret_cast<const uint4v *>(lds)[p];
        f.pay = pays[kFast ? slot : min(slot, (uint32_t)kSlots)];
        return f;
    }
    __device__ __forceinline__ float4_t direction(int side, const Chunk &f) const
    {
        const char *at = reinterpret_cast<const char *>(lds + kLutFloats + (side ? direction_floats<kTable>((int)S) : 0)) + (f.s_idx << 4);
        if (kTable)
            return *reinterpret_cast<const float4_t *>(at + f.l[0]);
        const float4_t x = *reinterpret_cast<const float4_t *>(at);
        const float4_t y = {0.5f * (x[0] - x[1] - x[2] - x[3]), 0.5f * (x[0] + x[1] - x[2] + x[3]), 0.5f * (x[0] + x[1] + x[2] - x[3]),
                            0.5f * (x[0] - x[1] + x[2] + x[3])};
        return f.l[0] == 0u ? x : f.l[0] == 1u ? y : y - x;
    }
    // The four values in fp32, of a row with this scale.
    __device__ __forceinline__ float4_t scaled(const Chunk &f, float4_t d, float sigma) const
    {
        const float r = (float)__builtin_amdgcn_ubfe(f.code, w_idx, r_bits) * sigma;
        return float4_t{r * d[0], r * d[1], r * d[2], r * d[3]};
    }
    static __device__ __forceinline__ float4_t saturated(float4_t y)  // as the decode does
    {
        return float4_t{__builtin_amdgcn_fmed3f(y[0], -65504.f, 65504.f), __builtin_amdgcn_fmed3f(y[1], -65504.f, 65504.f),
                        __builtin_amdgcn_fmed3f(y[2], -65504.f, 65504.f), __builtin_amdgcn_fmed3f(y[3], -65504.f, 65504.f)};
    }
    // The payload of a flagged chunk past the staged ones: straight from the list.  base: the window's first entry.
    static __device__ __forceinline__ uint2 far_payload(const AttendSide &sd, uint32_t base, const Chunk &f)
    {
        const uint64_t at = (uint64_t)base + f.slot;
        return at < sd.outlier_capacity ? reinterpret_cast<const uint2 *>(sd.outliers)[at] : make_uint2(0u, 0u);
    }
    // The chunk: its values rounded to fp16, in their places and with their signs, or its payload.
    static __device__ __forceinline__ uint2 packed(const Chunk &f, float4_t y, bool flagged)
    {
        half4_t out;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            out[e] = (_Float16)y[e];
        const uint2 o = __builtin_bit_cast(uint2, out);
        const uint32_t lo = __builtin_amdgcn_perm(o.y, o.x, f.l[1]) ^ f.l[2], hi = __builtin_amdgcn_perm(o.y, o.x, f.l[1] ^ 0x04040404u) ^ f.l[3];
        return make_uint2(flagged ? f.pay.x : lo, flagged ? f.pay.y : hi);
    }
    template <bool kFast, int kSlots>
    __device__ __forceinline__ uint2 finish(const AttendSide &sd, uint32_t base, Chunk f, float4_t d, float sigma, bool flagged) const
    {
        float4_t y = scaled(f, d, sigma);
        if (!kFast) {
            y = saturated(y);
            if (f.slot >= (uint32_t)kSlots && flagged)
                f.pay = far_payload(sd, base, f);
        }
        return packed(f, y, flagged);
    }
};

__device__ __forceinline__ float scale_value(uint32_t half_bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)half_bits); }

}  // namespace
}  // namespace hqmq
