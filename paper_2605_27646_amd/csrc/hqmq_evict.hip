// The tokens that a cache keeps, and their packed rows moved into a cache of their own (include/hqmq_serve.h,
// hqmq_evict_select and hqmq_evict_compact).
#include "hqmq_serve_device.h"

namespace hqmq {

namespace {

// The rank order of masses as unsigned numbers: larger mass, larger key; -0 and +0 equal; every NaN below -infinity.
// On the bit patterns: the build tells the compiler that no arithmetic sees a NaN.
__device__ __forceinline__ uint32_t mass_key(uint32_t bits)
{
    const uint32_t magnitude = bits & 0x7fffffffu;
    if (magnitude > 0x7f800000u)
        return 0u;
    return magnitude == 0u ? 0x80000000u : (bits >> 31 ? ~bits : bits | 0x80000000u);
}

constexpr int kSelThreads = 1024;

__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t *red)
{
    for (int d = 32; d > 0; d /= 2)
        v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t s = 0;
    for (int i = 0; i < kSelThreads / 64; ++i)
        s += red[i];
    return s;
}

}  // namespace

// A workgroup per (b, h).  The key of the last token kept is found bit by bit from the top (a count of the keys at or
// above a candidate decides a bit); then the tokens in order: all above it, and of those that equal it the first ones.
__global__ __launch_bounds__(kSelThreads) void k_evict_select(SelectArgs a)
{
    __shared__ uint32_t red[kSelThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t seg = blockIdx.x;
    const int b = (int)(seg / a.H);
    const int len = a.length ? min(max(a.length[b], 0), a.T) : a.T;
    const uint32_t *mass = reinterpret_cast<const uint32_t *>(a.mass) + seg * a.T;
    int32_t *keep = a.keep + seg * a.n_keep;
    uint32_t *kept = reinterpret_cast<uint32_t *>(a.kept_mass) + seg * a.n_keep;
    const int n = min(len, a.n_keep);
    if (tid == 0)
        a.n_kept[seg] = n;
    for (int j = n + tid; j < a.n_keep; j += kSelThreads) {
        keep[j] = -1;
        if (a.kept_mass)
            kept[j] = 0u;
    }
    const bool all = len <= a.n_keep;
    const int lo = all ? len : a.n_sink, hi = all ? len : len - a.n_recent;
    const uint32_t want = all ? 0u : (uint32_t)(a.n_keep - a.n_sink - a.n_recent);  // of the tokens lo .. hi - 1, which are more
    uint32_t last = 0u;
    for (int bit = 31; bit >= 0 && want > 0; --bit) {
        const uint32_t candidate = last | (1u << bit);
        uint32_t c = 0;
        for (int t = lo + tid; t < hi; t += kSelThreads)
            c += mass_key(mass[t]) >= candidate;
        if (block_sum(c, red) >= want)
            last = candidate;
    }
    uint32_t above = 0;
    for (int t = lo + tid; t < hi; t += kSelThreads)
        above += mass_key(mass[t]) > last;
    const uint32_t equal_wanted = want - (want > 0 ? block_sum(above, red) : 0u);
    uint32_t done = 0, equal_done = 0;
    for (int t0 = 0; t0 < len; t0 += kSelThreads) {
        const int t = t0 + tid;
        uint32_t key = 0;
        bool mid = t >= lo && t < hi, eq = false, in = t < len && !mid;
        if (mid && want > 0) {
            key = mass_key(mass[t]);
            in = key > last;
            eq = key == last;
        }
        const unsigned long long me = ballot(eq);
        __syncthreads();
        if (lane == 0)
            red[wave] = (uint32_t)__popcll(me);
        __syncthreads();
        uint32_t before = equal_done, total = 0;
        for (int i = 0; i < kSelThreads / 64; ++i) {
            before += i < wave ? red[i] : 0u;
            total += red[i];
        }
        equal_done += total;
        in |= eq && before + (uint32_t)__popcll(me & ((1ull << lane) - 1ull)) < equal_wanted;
        const unsigned long long mi = ballot(in);
        __syncthreads();
        if (lane == 0)
            red[wave] = (uint32_t)__popcll(mi);
        __syncthreads();
        before = done;
        total = 0;
        for (int i = 0; i < kSelThreads / 64; ++i) {
            before += i < wave ? red[i] : 0u;
            total += red[i];
        }
        done += total;
        if (in) {
            const uint32_t at = before + (uint32_t)__popcll(mi & ((1ull << lane) - 1ull));
            keep[at] = t;
            if (a.kept_mass)
                kept[at] = mass[t];
        }
    }
}

hipError_t launch_evict_select(const SelectArgs &a, hipStream_t stream)
{
    hipLaunchKernelGGL(k_evict_select, dim3((unsigned)(a.B * a.H)), dim3(kSelThreads), 0, stream, a);
    return hipGetLastError();
}

// ---- compaction: outliers per workgroup of 256 rows, then every workgroup finds its place and moves its rows ----------

__device__ __forceinline__ int64_t source_row(const CompactShape &s, const CompactTensor &t, int seg, int j)
{
    const int k = t.keep[(int64_t)seg * s.n_keep + j];
    return k >= 0 && k < s.T ? (int64_t)seg * s.T + k : -1;
}

__global__ __launch_bounds__(kCompactRows) void k_compact_count(CompactShape s, CompactBatch batch)
{
    __shared__ uint32_t red[kCompactRows / 64];
    const CompactTensor &t = batch.t[blockIdx.z];
    const int seg = blockIdx.y, j = blockIdx.x * kCompactRows + threadIdx.x;
    uint32_t c = 0;
    if (j < s.n_keep) {
        const int64_t from = source_row(s, t, seg, j);
        c = from >= 0 ? __popc(t.in.flags[from]) : 0;
    }
    for (int d = 32; d > 0; d /= 2)
        c += __shfl_xor(c, d);
    if ((threadIdx.x & 63) == 0)
        red[threadIdx.x >> 6] = c;
    __syncthreads();
    if (threadIdx.x == 0)
        s.totals[blockIdx.z * s.totals_stride + (uint64_t)seg * s.blocks_per_seg + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(kCompactRows) void k_compact_move(CompactShape s, CompactBatch batch)
{
    __shared__ uint32_t red[2][kCompactRows / 64], base_s;
    const CompactTensor &t = batch.t[blockIdx.z];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int seg = blockIdx.y, j = blockIdx.x * kCompactRows + tid, segs = s.B * s.H;
    const uint32_t *totals = s.totals + blockIdx.z * s.totals_stride;
    const int64_t me = (int64_t)seg * s.blocks_per_seg + blockIdx.x;
    uint32_t before = 0;
    for (int64_t i = tid; i < me; i += kCompactRows)
        before += totals[i];
    for (int d = 32; d > 0; d /= 2)
        before += __shfl_xor(before, d);
    const int64_t from = j < s.n_keep ? source_row(s, t, seg, j) : -1;
    const uint32_t word = from >= 0 ? t.in.flags[from] : 0u;
    uint32_t scan = __popc(word);
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(scan, d);
        scan += lane >= d ? o : 0u;
    }
    if (lane == 63)
        red[1][wave] = scan;
    if (lane == 0)
        red[0][wave] = before;
    __syncthreads();
    uint32_t at = scan - __popc(word);
    for (int i = 0; i < kCompactRows / 64; ++i)
        at += red[0][i] + (i < wave ? red[1][i] : 0u);
    const int64_t to = (int64_t)seg * s.n_keep + j;
    if (j < s.n_keep) {
        t.out.flags[to] = word;
        t.out.sigma[to] = from >= 0 ? t.in.sigma[from] : (uint16_t)0;
        t.out.row_off[to] = at;
        for (int i = 0; i < s.row_words; ++i)
            t.out.codes[to * s.row_words + i] = from >= 0 ? t.in.codes[from * s.row_words + i] : 0u;
        const uint32_t src = from >= 0 ? t.in.row_off[from] : 0u;
        for (int i = 0; i < __popc(word); ++i) {
            const uint64_t f = (uint64_t)src + i, o = (uint64_t)at + i;
            if (o < t.out_capacity)
                reinterpret_cast<uint2 *>(t.out.outliers)[o] =
                    f < t.in_capacity ? reinterpret_cast<const uint2 *>(t.in.outliers)[f] : make_uint2(0u, 0u);
        }
        if (to == (int64_t)segs * s.n_keep - 1) {
            const uint32_t total = at + __popc(word);
            t.out.row_off[to + 1] = total;
            t.out.n_outliers[s.H] = total;
            *t.out.status = *t.in.status | (total > t.out_capacity ? HQMQ_STATUS_OUTLIER_OVERFLOW : 0u);
        }
    }
    if (blockIdx.x == 0 && seg < s.H) {  // the head's count: its batch entries' workgroups
        uint32_t c = 0;
        for (int b = 0; b < s.B; ++b)
            for (int i = tid; i < s.blocks_per_seg; i += kCompactRows)
                c += totals[((int64_t)b * s.H + seg) * s.blocks_per_seg + i];
        for (int d = 32; d > 0; d /= 2)
            c += __shfl_xor(c, d);
        if (tid == 0)
            base_s = 0;
        __syncthreads();
        if (lane == 0)
            atomicAdd(&base_s, c);
        __syncthreads();
        if (tid == 0)
            t.out.n_outliers[seg] = base_s;
    }
}

hipError_t launch_evict_compact(const CompactShape &s, const CompactBatch &batch, int n_tensors, hipStream_t stream)
{
    const dim3 grid((unsigned)s.blocks_per_seg, (unsigned)(s.B * s.H), (unsigned)n_tensors);
    hipLaunchKernelGGL(k_compact_count, grid, dim3(kCompactRows), 0, stream, s, batch);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    hipLaunchKernelGGL(k_compact_move, grid, dim3(kCompactRows), 0, stream, s, batch);
    return hipGetLastError();
}

}  // namespace hqmq
