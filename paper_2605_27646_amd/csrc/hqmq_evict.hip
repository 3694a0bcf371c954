// The tokens that a cache keeps, and their packed rows moved into a cache of their own (include/hqmq_serve.h,
// hqmq_evict_select and hqmq_evict_compact).
#include <type_traits>

#include "hqmq_serve_device.h"

namespace hqmq {

namespace {

// The rank order of masses as unsigned numbers: larger mass, larger key; -0 and +0 equal; every NaN (1) below -infinity.  0 is left
// for what is not there, the largest number for tokens that are kept anyway.
// On the bit patterns: the build tells the compiler that no arithmetic sees a NaN.
__device__ __forceinline__ uint32_t mass_key(uint32_t bits)
{
    const uint32_t magnitude = bits & 0x7fffffffu;
    if (magnitude > 0x7f800000u)
        return 1u;
    return (magnitude == 0u ? 0x80000000u : (bits >> 31 ? ~bits : bits | 0x80000000u)) + 1u;
}
constexpr uint32_t kKeptKey = 0xffffffffu;

constexpr int kDigit0 = 12, kDigit1 = 10, kDigit2 = 10;  // of a key, from the top
static_assert(kDigit0 + kDigit1 + kDigit2 == 32, "a key");

__device__ __forceinline__ uint32_t wave_scan(uint32_t v, int lane)  // inclusive
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(v, d);
        v += lane >= d ? o : 0u;
    }
    return v;
}

}  // namespace

// A workgroup per (b, h); a wave has kPer * 64 tokens in a row (of every kThreads * kPer), lane by lane, so that it reads whole lines and
// finds the places of what it keeps with ballots.  The key of the last token kept is found digit by digit from the top: a histogram in LDS of
// the keys that share the digits found so far, and a scan of it.  Keys stay in registers; cache lines beyond kThreads * kPer tokens
// (kLoop) are read again for each digit, from the L2.
// Bound by latency: one workgroup's loads, three histograms and scans, and the ballots.
template <int kThreads, int kPer, bool kLoop>
__global__ __launch_bounds__(kThreads) void k_evict_select(SelectArgs a)
{
    constexpr int kWaves = kThreads / 64, kSpan = kThreads * kPer;
    __shared__ uint32_t hist[1 << kDigit0];
    __shared__ uint32_t wave_sum[2][kWaves], found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t seg = blockIdx.x;
    const int b = (int)(seg / a.H);
    const int len = a.length ? min(max(a.length[b], 0), a.T) : a.T;
    const uint32_t *mass = reinterpret_cast<const uint32_t *>(a.mass) + seg * a.T;
    int32_t *keep = a.keep + seg * a.n_keep;
    uint32_t *kept = reinterpret_cast<uint32_t *>(a.kept_mass) + seg * a.n_keep;
    const int n = min(len, a.n_keep);
    const int lo = a.n_sink, hi = len - a.n_recent;
    const int mine = wave * kPer * 64 + lane;

    uint32_t key[kPer], raw[kPer];
    const auto load = [&](int span) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int t = span + mine + 64 * j;
            raw[j] = mass[min(t, a.T - 1)];
        }
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const int t = span + mine + 64 * j;
            const uint32_t k = t < lo || t >= hi ? kKeptKey : mass_key(raw[j]);
            key[j] = t < len ? k : 0u;
        }
    };
    load(0);
    if (tid == 0)
        a.n_kept[seg] = n;
    for (int j = n + tid; j < a.n_keep; j += kThreads) {
        keep[j] = -1;
        if (a.kept_mass)
            kept[j] = 0u;
    }

    // ---- keys above `last` are kept, and of those equal to it the first `ties` -------------------------------------------------
    uint32_t last = 0u, ties = 0u;
    if (len > a.n_keep) {
        uint32_t rank = (uint32_t)n, prefix = 0u;
        const auto digit = [&](auto shift_tag, auto bits_tag) {
            constexpr int kShift = decltype(shift_tag)::value, kBits = decltype(bits_tag)::value, kBins = 1 << kBits;
            constexpr int kEach = kBins / kThreads > 0 ? kBins / kThreads : 1;  // bins of a thread, the highest of them with the first
            for (int i = tid; i < kBins; i += kThreads)
                hist[i] = 0u;
            __syncthreads();
            for (int span = 0; span < a.T; span += kSpan) {
                if (kLoop)
                    load(span);
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    const bool in = kShift + kBits == 32 ? key[j] != 0u : (kShift + kBits < 32 && key[j] >> ((kShift + kBits) & 31) == prefix && key[j] != 0u);
                    if (in)
                        atomicAdd(&hist[(key[j] >> kShift) & (kBins - 1)], 1u);
                }
                if (!kLoop)
                    break;
            }
            __syncthreads();
            uint32_t c[kEach], sum = 0u;
            const int top = kBins - 1 - tid * kEach;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                c[i] = top - i >= 0 ? hist[top - i] : 0u;
                sum += c[i];
            }
            const uint32_t scan = wave_scan(sum, lane);
            if (lane == 63)
                wave_sum[0][wave] = scan;
            __syncthreads();
            uint32_t above = scan - sum;
            for (int i = 0; i < wave; ++i)
                above += wave_sum[0][i];
            if (above < rank && rank <= above + sum) {  // one thread
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    if (above < rank && rank <= above + c[i]) {
                        found[0] = (uint32_t)(top - i);
                        found[1] = rank - above;
                        found[2] = c[i];
                    }
                    above += c[i];
                }
            }
            __syncthreads();
            prefix = prefix << kBits | found[0];
            rank = found[1];
            return found[2] == rank;  // every key with these digits is kept
        };
        bool whole = digit(std::integral_constant<int, 32 - kDigit0>{}, std::integral_constant<int, kDigit0>{});
        int shift = 32 - kDigit0;
        if (!whole) {
            whole = digit(std::integral_constant<int, kDigit2>{}, std::integral_constant<int, kDigit1>{});
            shift = kDigit2;
        }
        if (!whole) {
            whole = digit(std::integral_constant<int, 0>{}, std::integral_constant<int, kDigit2>{});
            shift = 0;
        }
        last = prefix << shift;
        if (whole)
            last = max(last, 1u) - 1u;
        else
            ties = rank;
    }

    // ---- places, in token order --------------------------------------------------------------------------------------------------
    uint32_t kept_before = 0u, ties_before = 0u;
    for (int span = 0; span < a.T; span += kSpan) {
        if (kLoop)
            load(span);
        uint32_t n_above = 0u, n_equal = 0u;  // of the wave
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            n_above += (uint32_t)__popcll(ballot(key[j] > last));
            if (ties != 0u)
                n_equal += (uint32_t)__popcll(ballot(key[j] == last));
        }
        __syncthreads();  // the last reads of these words
        if (lane == 0) {
            wave_sum[0][wave] = n_above;
            wave_sum[1][wave] = n_equal;
        }
        __syncthreads();
        uint32_t at = kept_before, equal = ties_before;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) {
            const uint32_t e = wave_sum[1][i], k = wave_sum[0][i] + (min(ties_before + e, ties) - min(ties_before, ties));
            if (i < wave) {
                at += k;
                equal += e;
            }
            kept_before += k;
            ties_before += e;
        }
        const auto place = [&](bool with_ties) {
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                const unsigned long long below = (1ull << lane) - 1ull;
                bool in = key[j] > last;
                if (with_ties) {
                    const unsigned long long same = ballot(key[j] == last);
                    in = in || (of_mask(same) && equal + (uint32_t)__popcll(same & below) < ties);
                    equal += (uint32_t)__popcll(same);
                }
                const unsigned long long kept_mask = ballot(in);
                if (in) {
                    const uint32_t to = at + (uint32_t)__popcll(kept_mask & below);
                    keep[to] = span + mine + 64 * j;
                    if (a.kept_mass)
                        kept[to] = raw[j];
                }
                at += (uint32_t)__popcll(kept_mask);
            }
        };
        if (ties == 0u)
            place(false);
        else
            place(true);
        if (!kLoop)
            break;
    }
}

// Threads and tokens of a thread by the tokens of a head: as many waves as can share them, up to 16, and the keys in registers up to
// 32768 tokens.
hipError_t launch_evict_select(const SelectArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.B * a.H));
    if (a.T <= 256 * 4)
        hipLaunchKernelGGL((k_evict_select<256, 4, false>), grid, dim3(256), 0, stream, a);
    else if (a.T <= 1024 * 4)
        hipLaunchKernelGGL((k_evict_select<1024, 4, false>), grid, dim3(1024), 0, stream, a);
    else if (a.T <= 1024 * 8)
        hipLaunchKernelGGL((k_evict_select<1024, 8, false>), grid, dim3(1024), 0, stream, a);
    else if (a.T <= 1024 * 16)
        hipLaunchKernelGGL((k_evict_select<1024, 16, false>), grid, dim3(1024), 0, stream, a);
    else if (a.T <= 1024 * 32)
        hipLaunchKernelGGL((k_evict_select<1024, 32, false>), grid, dim3(1024), 0, stream, a);
    else
        hipLaunchKernelGGL((k_evict_select<1024, 32, true>), grid, dim3(1024), 0, stream, a);
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
