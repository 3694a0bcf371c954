// The attention weight that cached tokens accumulate (include/hqmq_serve.h, hqmq_attend_mass).  A thread per token: its
// reconstructed key stays in registers while all query rows of the kv head go past.
#include "hqmq_serve_device.h"

namespace hqmq {

template <int kNc>
__global__ __launch_bounds__(256) void k_mass_tokens(Geometry g, MassArgs a)
{
    constexpr int kD = 4 * kNc;
    const int seg = blockIdx.y, b = seg / g.H, h = seg % g.H;
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= g.T)
        return;
    const int64_t row = (int64_t)seg * g.T + t;
    uint2 key[kNc];
#pragma unroll
    for (int c = 0; c < kNc; ++c)
        key[c] = chunk_from_memory(g, a.k, a.k.sec + (size_t)h * g.S * 4, row, c);
    float sum = 0.f;
    for (int r = 0; r < a.n_share * a.G; ++r) {
        const size_t head = ((size_t)(b * a.n_share + r / a.G) * g.H + h) * a.G + r % a.G;
        const float lse = a.lse[head];
        if (lse < -1.0e30f || (a.visible && t >= a.visible[head]))
            continue;
        const half4_t *q = reinterpret_cast<const half4_t *>(a.q + head * kD);
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < kNc; ++c) {
            const half4_t kc = __builtin_bit_cast(half4_t, key[c]), qc = q[c];
#pragma unroll
            for (int i = 0; i < 4; ++i)
                s = fmaf((float)qc[i], (float)kc[i], s);
        }
        sum += __builtin_amdgcn_exp2f(fmaf(s, a.qscale, -lse * 1.44269504088896340736f));
    }
    a.mass_out[row] = a.mass_in ? fmaf(a.decay, a.mass_in[row], sum) : sum;
}

hipError_t launch_mass(const Geometry &g, const MassArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)((g.T + 255) / 256), (unsigned)(g.B * g.H));
    if (g.D == 128)
        hipLaunchKernelGGL(k_mass_tokens<32>, grid, dim3(256), 0, stream, g, a);
    else if (g.D == 96)
        hipLaunchKernelGGL(k_mass_tokens<24>, grid, dim3(256), 0, stream, g, a);
    else if (g.D == 64)
        hipLaunchKernelGGL(k_mass_tokens<16>, grid, dim3(256), 0, stream, g, a);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace hqmq
