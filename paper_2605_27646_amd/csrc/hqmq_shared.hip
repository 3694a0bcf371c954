// Attention of many sequences over one packed prefix (include/hqmq_serve.h, hqmq_attend_shared).  A workgroup takes 16
// query rows of a kv head over a share of the prefix, tiles of 32 tokens reconstructed into LDS; its partial state is
// merged with those of the other shares, and of the sequences' own tokens, by the merge of the single-query attention.
#include "hqmq_serve_device.h"

namespace hqmq {

namespace {
constexpr int kRows = 16, kTile = 32;
constexpr float kNone = -1.0e30f;  // "no token seen yet": finite, so that differences stay finite
}

template <int kNc>
__global__ __launch_bounds__(256) void k_shared_rows(Geometry g, SharedArgs a)
{
    constexpr int kD = 4 * kNc, kPer = kD / 16;
    __shared__ float qs[kRows][kD + 1];
    __shared__ __align__(16) _Float16 ks[kTile][kD + 8], vs[kTile][kD + 8];
    __shared__ float ps[kRows][kTile + 1];
    const int tid = threadIdx.x, r = tid >> 4, j = tid & 15;
    const int seg = blockIdx.y, b = seg / g.H, h = seg % g.H;
    const int row = blockIdx.z * kRows + r, n_rows = a.n_share * a.G;
    const bool there = row < n_rows;
    const int m = there ? row / a.G : 0, gq = there ? row % a.G : 0;
    const size_t head = ((size_t)(b * a.n_share + m) * g.H + h) * a.G + gq;
    int vis = there ? g.T : 0;
    if (there && a.visible)
        vis = min(vis, a.visible[head]);
    for (int d = j; d < kD; d += 16)
        qs[r][d] = (float)a.q[head * kD + d];
    float mx = kNone, sum = 0.f, acc[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        acc[i] = 0.f;
    const int begin = blockIdx.x * a.rows_per_split, end = min(g.T, begin + a.rows_per_split);
    const float *sk = a.k.sec + (size_t)h * g.S * 4, *sv = a.v.sec + (size_t)h * g.S * 4;
    for (int t0 = begin; t0 < end; t0 += kTile) {
        __syncthreads();
        for (int i = tid; i < kTile * kNc; i += 256) {
            const int t = i / kNc, c = i % kNc;
            uint2 kc = make_uint2(0u, 0u), vc = kc;
            if (t0 + t < end) {
                const int64_t at = (int64_t)seg * g.T + t0 + t;
                kc = chunk_from_memory(g, a.k, sk, at, c);
                vc = chunk_from_memory(g, a.v, sv, at, c);
            }
            *reinterpret_cast<uint2 *>(&ks[t][4 * c]) = kc;
            *reinterpret_cast<uint2 *>(&vs[t][4 * c]) = vc;
        }
        __syncthreads();
        float s[2] = {0.f, 0.f};
        for (int d = 0; d < kD; ++d) {
            s[0] = fmaf(qs[r][d], (float)ks[j][d], s[0]);
            s[1] = fmaf(qs[r][d], (float)ks[j + 16][d], s[1]);
        }
        float top = mx;
        const int seen = min(end, vis) - t0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s[i] = j + 16 * i < seen ? s[i] * a.qscale : 3.f * kNone;
            top = fmaxf(top, s[i]);
        }
        for (int d = 1; d < 16; d *= 2)
            top = fmaxf(top, __shfl_xor(top, d));
        const float corr = __builtin_amdgcn_exp2f(mx - top);
        mx = top;
        sum *= corr;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float p = __builtin_amdgcn_exp2f(s[i] - mx);
            sum += p;
            ps[r][j + 16 * i] = p;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            float o = acc[i] * corr;
            for (int t = 0; t < kTile; ++t)
                o = fmaf(ps[r][t], (float)vs[t][j * kPer + i], o);
            acc[i] = o;
        }
    }
    for (int d = 1; d < 16; d *= 2)
        sum += __shfl_xor(sum, d);
    if (!there)
        return;
    const size_t at = head * a.part_pitch + blockIdx.x;
    if (j == 0) {
        a.part_ml[2 * at] = mx;
        a.part_ml[2 * at + 1] = sum;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i)
        a.part_acc[at * 128 + j * kPer + i] = acc[i];
}

SharedPlan plan_shared(const Geometry &g, int G, int n_share)
{
    const int64_t per = (int64_t)g.B * g.H * ((G * n_share + kRows - 1) / kRows), tiles = (g.T + kTile - 1) / kTile;
    int64_t want = (512 + per - 1) / per;
    want = want < tiles ? want : tiles;
    const int64_t tiles_per = (tiles + want - 1) / want;
    return {(int32_t)((tiles + tiles_per - 1) / tiles_per), (int32_t)(tiles_per * kTile)};
}

hipError_t launch_shared(const Geometry &g, const SharedArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)a.n_splits, (unsigned)(g.B * g.H), (unsigned)((a.G * a.n_share + kRows - 1) / kRows));
    if (g.D == 128)
        hipLaunchKernelGGL(k_shared_rows<32>, grid, dim3(256), 0, stream, g, a);
    else if (g.D == 96)
        hipLaunchKernelGGL(k_shared_rows<24>, grid, dim3(256), 0, stream, g, a);
    else if (g.D == 64)
        hipLaunchKernelGGL(k_shared_rows<16>, grid, dim3(256), 0, stream, g, a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace hqmq
