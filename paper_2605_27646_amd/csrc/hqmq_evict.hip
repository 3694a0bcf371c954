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
constexpr uint32_t kKeptKey = 0xffffffffu, kZeroKey = 0x80000001u;

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

__device__ __forceinline__ uint32_t wave_total(uint32_t v)
{
#pragma unroll
    for (int d = 32; d > 0; d /= 2)
        v += __shfl_xor(v, d);
    return v;
}

// The tokens of a head, and the keys of kThreads * kPer of them from `first` on: a wave has kPer * 64 in a row, lane by lane, so that it
// reads whole lines and finds the places of what it keeps with ballots.
struct Head {
    const uint32_t *mass;
    int T, len, lo, hi, n_keep;  // lo .. hi - 1: the tokens that are not kept anyway
    __device__ __forceinline__ Head(const SelectArgs &a, int64_t seg)
    {
        T = a.T;
        len = a.length ? min(max(a.length[seg / a.H], 0), a.T) : a.T;
        mass = reinterpret_cast<const uint32_t *>(a.mass) + seg * a.T;
        lo = a.n_sink;
        hi = len - a.n_recent;
        n_keep = a.n_keep;
    }
    __device__ __forceinline__ uint32_t key(int t, uint32_t raw) const
    {
        const uint32_t k = t < lo || t >= hi ? kKeptKey : mass_key(raw);
        return t < len ? k : 0u;
    }
};
template <int kPer>
struct Keys {
    uint32_t key[kPer];
    int mine;  // the token of key[0]; key[j]'s is 64 j further
    __device__ __forceinline__ bool any(const Head &h) const { return __builtin_amdgcn_readfirstlane(mine) < h.len; }  // in the wave
    __device__ __forceinline__ void load(const Head &h, int first, int wave, int lane)
    {
        mine = first + wave * kPer * 64 + lane;
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            key[j] = h.mass[min(mine + 64 * j, h.T - 1)];
        // most waves: weights' sums, which are not negative, of tokens that are neither kept anyway nor missing
        uint32_t most = key[0];
#pragma unroll
        for (int j = 1; j < kPer; ++j)
            most = max(most, key[j]);
        const int from = first + wave * kPer * 64;
        if (from >= h.lo && from + 64 * kPer <= h.hi && ballot(most > 0x7f800000u) == 0ull) {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                key[j] += kZeroKey;
        } else {
#pragma unroll
            for (int j = 0; j < kPer; ++j)
                key[j] = h.key(mine + 64 * j, key[j]);
        }
    }
};

// The keys' digit of kBits bits above kShift, of those that share the digits above it with prefix, added to hist in LDS.  (Keys of 0 too:
// they are below every key that a rank can ask for.)  Where a quarter of
// a wave's first keys have one digit (a value that many tokens have would be added one by one: 32768 equal masses 100 us instead of 34), a
// wave adds the keys that have its first lane's digit at once.
template <int kShift, int kBits, int kPer>
__device__ __forceinline__ void count_digit(const Keys<kPer> &k, uint32_t prefix, uint32_t *hist, int lane)
{
    const auto bin_of = [&](uint32_t x) { return (x >> kShift) & ((1u << kBits) - 1u); };
    const auto counts = [&](uint32_t x) { return kShift + kBits >= 32 || x >> ((kShift + kBits) & 31) == prefix; };
    const auto common = [&](int l) {
        const uint32_t its = (uint32_t)__builtin_amdgcn_readlane((int)bin_of(k.key[0]), l);
        return __popcll(ballot(counts(k.key[0]) && bin_of(k.key[0]) == its)) >= 16;
    };
    if (common(0) || common(21) || common(42)) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            const uint32_t bin = bin_of(k.key[j]);
            const bool in = counts(k.key[j]);
            const unsigned long long all = ballot(in);
            if (all == 0ull)
                continue;
            const int first = (int)__ffsll((unsigned long long)all) - 1;
            const uint32_t its = (uint32_t)__builtin_amdgcn_readlane((int)bin, first);
            const unsigned long long same = ballot(in && bin == its);
            if (lane == first)
                atomicAdd(&hist[its], (uint32_t)__popcll(same));
            else if (in && bin != its)
                atomicAdd(&hist[bin], 1u);
        }
    } else {
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (counts(k.key[j]))
                atomicAdd(&hist[bin_of(k.key[j])], 1u);
    }
}

// From a histogram, kEach bins of it in this thread (bin kBins - 1 - kEach * tid - i in c[i]), the bin that holds the key of the given rank
// from the top: found[0], found[1] its rank there, found[2] the bin's keys.
template <int kThreads, int kEach>
__device__ __forceinline__ void find_bin(const uint32_t *c, int top, uint32_t rank, uint32_t *wave_sum, uint32_t *found, int wave, int lane)
{
    uint32_t sum = 0u;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        sum += c[i];
    const uint32_t scan = wave_scan(sum, lane);
    if (lane == 63)
        wave_sum[wave] = scan;
    __syncthreads();
    uint32_t above = scan - sum;
    for (int i = 0; i < wave; ++i)
        above += wave_sum[i];
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
}

// The tokens above `last`, and the first `ties` of those equal to it, to their places.  at, equal: how many of either this wave's tokens
// come behind.
template <int kPer>
__device__ __forceinline__ void place_keys(const Keys<kPer> &k, uint32_t last, uint32_t ties, uint32_t at, uint32_t equal, const Head &head, int32_t *keep, uint32_t *kept, int lane)
{
    const unsigned long long below = (1ull << lane) - 1ull;
    const uint32_t *mass = head.mass;
    const int lo = head.lo, hi = head.hi;
    const auto place = [&](auto plain_tag) {
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            bool in = k.key[j] > last;
            if (!decltype(plain_tag)::value && ties != 0u) {
                const unsigned long long same = ballot(k.key[j] == last);
                in = in || (of_mask(same) && equal + (uint32_t)__popcll(same & below) < ties);
                equal += (uint32_t)__popcll(same);
            }
            const unsigned long long kept_mask = ballot(in);
            if (in) {
                const uint32_t to = at + (uint32_t)__popcll(kept_mask & below);
                keep[to] = k.mine + 64 * j;
                if (kept)
                    kept[to] = decltype(plain_tag)::value ? k.key[j] - kZeroKey : mass[k.mine + 64 * j];
            }
            at += (uint32_t)__popcll(kept_mask);
        }
    };
    // most waves: no ties, and of the keys only those of positive masses, which tell the masses
    const int first = k.mine - lane;
    if (ties == 0u && last >= kZeroKey && first >= lo && first + 64 * kPer <= hi)
        place(std::true_type{});
    else
        place(std::false_type{});
}
template <int kPer>
__device__ __forceinline__ void count_kept(const Keys<kPer> &k, uint32_t last, uint32_t ties, uint32_t &above, uint32_t &equal)
{
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        above += (uint32_t)__popcll(ballot(k.key[j] > last));
        if (ties != 0u)
            equal += (uint32_t)__popcll(ballot(k.key[j] == last));
    }
}

// Counts, and -1 and zeros behind the kept tokens of a head that has fewer than n_keep.
__device__ __forceinline__ void fill_rest(const SelectArgs &a, int64_t seg, int n, int tid, int threads)
{
    if (tid == 0)
        a.n_kept[seg] = n;
    for (int j = n + tid; j < a.n_keep; j += threads) {
        a.keep[seg * a.n_keep + j] = -1;
        if (a.kept_mass)
            a.kept_mass[seg * a.n_keep + j] = 0.f;
    }
}

}  // namespace

// A workgroup per (b, h), its keys in registers.  The key of the last token kept is found digit by digit from the top: a histogram in LDS of
// the keys that share the digits found so far, and a scan of it.
// Bound by latency and by what one compute unit loads and issues: 8 heads of 600 tokens 6.4 us, of 8192 10, of 32768 22 (0.5 us for every
// 1024 tokens).
template <int kThreads, int kPer>
__global__ __launch_bounds__(kThreads) void k_evict_select(SelectArgs a)
{
    constexpr int kWaves = kThreads / 64;
    __shared__ uint32_t hist[1 << kDigit0];
    __shared__ uint32_t wave_sum[2][kWaves], found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t seg = blockIdx.x;
    const Head head(a, seg);
    const int n = min(head.len, a.n_keep);
    Keys<kPer> k;
    k.load(head, 0, wave, lane);
    fill_rest(a, seg, n, tid, kThreads);

    // ---- keys above `last` are kept, and of those equal to it the first `ties` -------------------------------------------------
    uint32_t last = 0u, ties = 0u;
    if (head.len > a.n_keep) {
        uint32_t rank = (uint32_t)n, prefix = 0u;
        const auto digit = [&](auto shift_tag, auto bits_tag) {
            constexpr int kShift = decltype(shift_tag)::value, kBits = decltype(bits_tag)::value, kBins = 1 << kBits;
            constexpr int kEach = kBins / kThreads;
            for (int i = tid; i < kBins; i += kThreads)
                hist[i] = 0u;
            __syncthreads();
            if (k.any(head))
                count_digit<kShift, kBits>(k, prefix, hist, lane);
            __syncthreads();
            uint32_t c[kEach];
            const int top = kBins - 1 - tid * kEach;
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                c[i] = hist[top - i];
            find_bin<kThreads, kEach>(c, top, rank, wave_sum[0], found, wave, lane);
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
    uint32_t above = 0u, equal = 0u;  // of the wave
    count_kept(k, last, ties, above, equal);
    __syncthreads();
    if (lane == 0) {
        wave_sum[0][wave] = above;
        wave_sum[1][wave] = equal;
    }
    __syncthreads();
    above = equal = 0u;  // of the waves before it
    for (int i = 0; i < wave; ++i) {
        above += wave_sum[0][i];
        equal += wave_sum[1][i];
    }
    place_keys(k, last, ties, above + min(equal, ties), equal, head, a.keep + seg * a.n_keep,
               a.kept_mass ? reinterpret_cast<uint32_t *>(a.kept_mass) + seg * a.n_keep : nullptr, lane);
}

// Longer heads are shared by workgroups in four launches: the histogram of each digit, left in the workspace for the next launch to sum,
// and the places.  Every workgroup finds the last digit for itself, and, from the same counts, how many tokens the workgroups before it
// keep: no launch of its own for either.  A workgroup takes 8192 tokens, or several times as many where more than kMostSelectParts would
// share a head: each reads the histograms of all of them.
// Bound by latency: four launches with a chain of loads each, of keys and of counts that another XCD wrote.  8 heads of 40000 tokens
// 23.6 us, of 131072 28.5; 32 of 131072 45.7.
constexpr int kPartThreads = 1024, kPartPer = 8, kPart = kPartThreads * kPartPer, kMostSelectParts = 64;
constexpr int kDigitBits[3] = {kDigit0, kDigit1, kDigit2}, kDigitShift[3] = {32 - kDigit0, kDigit2, 0};
// What the digits so far say.
struct PartState {
    uint32_t prefix, rank;   // the digits of the last key kept, its rank among the keys that have them
    uint32_t digits, whole;  // how many; whether all keys with them are kept: no further digit then
    uint32_t above;          // tokens with larger keys (whole: or these digits) in the workgroups before this one
};
// A workspace, in 32-bit words: histograms of the three digits [segs][parts][bins], and the PartState after the first two
// [2][segs][parts][8].
struct PartLayout {
    uint64_t hist[3], state[2], total;
    int parts, loads;  // workgroups of a head, kPart tokens that each takes in turn
    __host__ __device__ PartLayout(int64_t segs, int T)
    {
        const int all = (T + kPart - 1) / kPart;
        loads = (all + kMostSelectParts - 1) / kMostSelectParts;
        parts = (all + loads - 1) / loads;
        uint64_t at = 0;
        const int bits[3] = {kDigit0, kDigit1, kDigit2};
        for (int d = 0; d < 3; ++d) {
            hist[d] = at;
            at += (uint64_t)segs * parts << bits[d];
        }
        for (int d = 0; d < 2; ++d) {
            state[d] = at;
            at += (uint64_t)segs * parts * 8;
        }
        total = at;
    }
};

template <int kStep>  // 0, 1, 2: that digit's histogram; 3: the places
__global__ __launch_bounds__(kPartThreads) void k_evict_select_part(SelectArgs a, uint32_t *ws)
{
    constexpr int kWaves = kPartThreads / 64;
    __shared__ uint32_t hist[1 << kDigit0];
    __shared__ uint32_t wave_sum[2][kWaves], found[3];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t seg = blockIdx.y;
    const int part = blockIdx.x;
    const Head head(a, seg);
    const PartLayout l((int64_t)a.B * a.H, a.T);
    const int n = min(head.len, a.n_keep);
    const bool all = head.len <= a.n_keep;  // kept whole: nothing to find
    if (kStep < 3 && all)
        return;
    const int first = part * l.loads * kPart;
    Keys<kPartPer> k;
    k.load(head, first, wave, lane);

    PartState st{0u, (uint32_t)n, 0u, 0u, 0u};
    uint32_t equal_before = 0u;  // tokens with the last key itself in the workgroups before this one
    if constexpr (kStep > 0) {
        constexpr int kD = kStep - 1, kBins = 1 << kDigitBits[kD], kEach = kBins / kPartThreads;
        typedef uint32_t bins_t __attribute__((ext_vector_type(kEach)));
        if (kD > 0 && !all)
            st = *reinterpret_cast<const PartState *>(ws + l.state[kD > 0 ? kD - 1 : 0] + (seg * l.parts + part) * 8);
        if (!all && st.whole == 0u) {
            const int low = kBins - kEach * (tid + 1);  // this thread's bins, the lowest of them
            const uint32_t *h = ws + l.hist[kD] + seg * l.parts * kBins + low;
            uint32_t c[kEach] = {}, before[kEach] = {};  // from the highest bin down: of all parts, of those before this one
            for (int p = 0; p < l.parts; p += 8) {       // eight loads on their way at a time
                bins_t x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u)
                    x[u] = *reinterpret_cast<const bins_t *>(h + (int64_t)min(p + u, l.parts - 1) * kBins);
#pragma unroll
                for (int u = 0; u < 8; ++u)
#pragma unroll
                    for (int i = 0; i < kEach; ++i) {
                        c[i] += p + u < l.parts ? x[u][kEach - 1 - i] : 0u;
                        before[i] += p + u < part ? x[u][kEach - 1 - i] : 0u;
                    }
            }
            find_bin<kPartThreads, kEach>(c, low + kEach - 1, st.rank, wave_sum[0], found, wave, lane);
            st.prefix = st.prefix << kDigitBits[kD] | found[0];
            st.rank = found[1];
            st.digits = kD + 1;
            st.whole = found[2] == found[1] ? 1u : 0u;
            uint32_t above = 0u, same = 0u;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const uint32_t bin = (uint32_t)(low + kEach - 1 - i);
                above += bin > found[0] || (bin == found[0] && st.whole != 0u) ? before[i] : 0u;
                same += bin == found[0] && st.whole == 0u ? before[i] : 0u;
            }
            above = wave_total(above);
            same = wave_total(same);
            if (lane == 0) {
                wave_sum[0][wave] = above;
                wave_sum[1][wave] = same;
            }
            __syncthreads();
            for (int i = 0; i < kWaves; ++i) {
                st.above += wave_sum[0][i];
                equal_before += wave_sum[1][i];
            }
        }
        if (kStep < 3 && tid == 0)
            *reinterpret_cast<PartState *>(ws + l.state[kD < 2 ? kD : 0] + (seg * l.parts + part) * 8) = st;
    }
    if constexpr (kStep < 3) {
        if (st.whole != 0u)
            return;
        constexpr int kBins = 1 << kDigitBits[kStep];
        for (int i = tid; i < kBins; i += kPartThreads)
            hist[i] = 0u;
        __syncthreads();
        for (int x = 0; x < l.loads; ++x) {
            if (x > 0)
                k.load(head, first + x * kPart, wave, lane);
            if (k.any(head))
                count_digit<kDigitShift[kStep], kDigitBits[kStep]>(k, st.prefix, hist, lane);
        }
        __syncthreads();
        uint32_t *h = ws + l.hist[kStep] + (seg * l.parts + part) * kBins;
        for (int i = tid; i < kBins; i += kPartThreads)
            h[i] = hist[i];
    } else {
        if (part == 0)
            fill_rest(a, seg, n, tid, kPartThreads);
        // keys above `last` are kept, and of those equal to it the first `ties`
        uint32_t last = 0u, ties = 0u;
        if (all) {
            st.above = (uint32_t)min(first, head.len);
        } else {
            last = st.prefix << (st.digits == 1u ? kDigitShift[0] : st.digits == 2u ? kDigitShift[1] : kDigitShift[2]);
            if (st.whole != 0u)
                last = max(last, 1u) - 1u;
            else
                ties = st.rank;
        }
        uint32_t above_before = st.above;
        for (int x = 0; x < l.loads; ++x) {
            if (x > 0)
                k.load(head, first + x * kPart, wave, lane);
            uint32_t above = 0u, equal = 0u;  // of the wave
            count_kept(k, last, ties, above, equal);
            __syncthreads();
            if (lane == 0) {
                wave_sum[0][wave] = above;
                wave_sum[1][wave] = equal;
            }
            __syncthreads();
            uint32_t above_here = above_before, equal_here = equal_before;  // of what comes before the wave's tokens
            for (int i = 0; i < kWaves; ++i) {
                const uint32_t more = wave_sum[0][i], same = wave_sum[1][i];
                above_here += i < wave ? more : 0u;
                equal_here += i < wave ? same : 0u;
                above_before += more;
                equal_before += same;
            }
            place_keys(k, last, ties, above_here + min(equal_here, ties), equal_here, head, a.keep + seg * a.n_keep,
                       a.kept_mass ? reinterpret_cast<uint32_t *>(a.kept_mass) + seg * a.n_keep : nullptr, lane);
        }
    }
}

// One workgroup takes a head of up to 32768 tokens, with as many waves as can share them, up to 16: there the two ways take the same time.
static bool select_in_parts(int T) { return T > 1024 * 32; }

uint64_t evict_select_workspace_bytes(int B, int H, int T)
{
    return select_in_parts(T) ? PartLayout((int64_t)B * H, T).total * sizeof(uint32_t) : 0;
}

hipError_t launch_evict_select(const SelectArgs &a, uint32_t *workspace, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.B * a.H));
    if (select_in_parts(a.T)) {
        const dim3 parts((unsigned)PartLayout((int64_t)a.B * a.H, a.T).parts, (unsigned)(a.B * a.H));
        hipLaunchKernelGGL(k_evict_select_part<0>, parts, dim3(kPartThreads), 0, stream, a, workspace);
        hipLaunchKernelGGL(k_evict_select_part<1>, parts, dim3(kPartThreads), 0, stream, a, workspace);
        hipLaunchKernelGGL(k_evict_select_part<2>, parts, dim3(kPartThreads), 0, stream, a, workspace);
        hipLaunchKernelGGL(k_evict_select_part<3>, parts, dim3(kPartThreads), 0, stream, a, workspace);
    } else if (a.T <= 256 * 4)
        hipLaunchKernelGGL((k_evict_select<256, 4>), grid, dim3(256), 0, stream, a);
    else if (a.T <= 1024 * 4)
        hipLaunchKernelGGL((k_evict_select<1024, 4>), grid, dim3(1024), 0, stream, a);
    else if (a.T <= 1024 * 8)
        hipLaunchKernelGGL((k_evict_select<1024, 8>), grid, dim3(1024), 0, stream, a);
    else if (a.T <= 1024 * 16)
        hipLaunchKernelGGL((k_evict_select<1024, 16>), grid, dim3(1024), 0, stream, a);
    else
        hipLaunchKernelGGL((k_evict_select<1024, 32>), grid, dim3(1024), 0, stream, a);
    return hipGetLastError();
}

// ---- compaction ------------------------------------------------------------------------------------------------------------------
// A launch counts the outliers of every 64 and every 256 kept rows; in the last a workgroup takes 64 rows, sums what comes before them
// (where there are more than kCompactDirect counts, from a third launch's sums of kCompactGroup of them each), and moves code words and
// payloads lane by lane along the new tensor, so that they are written in whole lines.
// Bound by latency: the chain of loads from a kept index over its flags to its payloads, in each of the two launches.

namespace {
constexpr int kMoveThreads = 256, kMoveRows = 64;
constexpr int kMoveList = 512;  // payloads of 64 rows that are moved line by line; more than a quarter of the chunks: row by row
static_assert(kCompactRows == 4 * kMoveRows, "a count for every wave");

__device__ __forceinline__ int64_t source_row(const CompactShape &s, const CompactTensor &t, int seg, int j)
{
    if (j >= s.n_keep)
        return -1;
    const int k = t.keep[(int64_t)seg * s.n_keep + j];
    return k >= 0 && k < s.T ? (int64_t)seg * s.T + k : -1;
}
}  // namespace

__global__ __launch_bounds__(kCompactRows) void k_compact_count(CompactShape s, CompactBatch batch)
{
    __shared__ uint32_t sub[4];
    const CompactTensor &t = batch.t[blockIdx.z];
    const int seg = blockIdx.y;
    const int64_t from = source_row(s, t, seg, blockIdx.x * kCompactRows + threadIdx.x);
    const uint32_t c = wave_total(from >= 0 ? __popc(t.in.flags[from]) : 0u);
    if ((threadIdx.x & 63) == 0)
        sub[threadIdx.x >> 6] = c;
    __syncthreads();
    uint32_t *totals = s.totals + blockIdx.z * s.totals_stride;
    const int64_t block = (int64_t)seg * s.blocks_per_seg + blockIdx.x, blocks = (int64_t)s.B * s.H * s.blocks_per_seg;
    if (threadIdx.x == 0)
        totals[block] = sub[0] + sub[1] + sub[2] + sub[3];
    if (threadIdx.x < 4)
        totals[blocks + 4 * block + threadIdx.x] = sub[threadIdx.x];
}

// groups[i]: the outliers of kCompactGroup blocks.
__global__ __launch_bounds__(kMoveThreads) void k_compact_groups(CompactShape s)
{
    __shared__ uint32_t red[kMoveThreads / 64];
    const int tid = threadIdx.x;
    const int64_t blocks = (int64_t)s.B * s.H * s.blocks_per_seg, first = (int64_t)blockIdx.x * kCompactGroup;
    uint32_t *totals = s.totals + blockIdx.y * s.totals_stride;
    uint32_t c = 0u;
    for (int64_t i = first + tid; i < min(first + kCompactGroup, blocks); i += kMoveThreads)
        c += totals[i];
    c = wave_total(c);
    if ((tid & 63) == 0)
        red[tid >> 6] = c;
    __syncthreads();
    if (tid == 0)
        totals[5 * blocks + blockIdx.x] = red[0] + red[1] + red[2] + red[3];
}

__global__ __launch_bounds__(kMoveThreads) void k_compact_move(CompactShape s, CompactBatch batch)
{
    __shared__ int64_t row_of[kMoveRows];
    __shared__ uint32_t red[2][kMoveThreads / 64], list[kMoveList];
    const CompactTensor &t = batch.t[blockIdx.z];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int seg = blockIdx.y, j0 = blockIdx.x * kMoveRows, n = min(s.n_keep - j0, kMoveRows);
    const uint32_t *totals = s.totals + blockIdx.z * s.totals_stride;
    const int64_t blocks = (int64_t)s.B * s.H * s.blocks_per_seg;
    const int64_t block = (int64_t)seg * s.blocks_per_seg + blockIdx.x / 4;
    const int64_t to0 = (int64_t)seg * s.n_keep + j0;

    // every wave looks at the rows, so that none waits for another's loads; the code words are on their way before flags and counts are
    // looked at
    const int64_t from = source_row(s, t, seg, j0 + lane);
    if (wave == 0)
        row_of[lane] = from;
    const uint32_t word = from >= 0 ? t.in.flags[from] : 0u;
    const uint32_t src = from >= 0 ? t.in.row_off[from] : 0u;
    const uint16_t sigma = from >= 0 ? t.in.sigma[from] : (uint16_t)0;
    uint32_t before = tid < (int)(blockIdx.x & 3) ? totals[blocks + 4 * block + tid] : 0u;
    const int64_t n_groups = blocks > kCompactDirect ? block / kCompactGroup : 0;
    for (int64_t i = tid; i < n_groups; i += kMoveThreads)
        before += totals[5 * blocks + i];
    for (int64_t i = n_groups * kCompactGroup + tid; i < block; i += kMoveThreads)
        before += totals[i];
    __syncthreads();
    constexpr int kWords = (kMoveRows * 24 + kMoveThreads - 1) / kMoveThreads;  // of a thread: a row has 24 at most
    const int n_words = n * s.row_words;
    uint32_t code[kWords];
#pragma unroll
    for (int u = 0; u < kWords; ++u) {
        const int i = min(tid + kMoveThreads * u, n_words - 1), r = i / s.row_words;
        const int64_t row = row_of[r];
        code[u] = t.in.codes[max(row, (int64_t)0) * s.row_words + (i - r * s.row_words)];
        code[u] = row >= 0 ? code[u] : 0u;
    }
    before = wave_total(before);
    if (lane == 0)
        red[0][wave] = before;
    if (blockIdx.x == 0 && seg < s.H) {  // the head's count: its batch entries' rows
        uint32_t c = 0;
        for (int64_t i = tid; i < (int64_t)s.B * s.blocks_per_seg; i += kMoveThreads)
            c += totals[(i / s.blocks_per_seg * s.H + seg) * s.blocks_per_seg + i % s.blocks_per_seg];
        c = wave_total(c);
        if (lane == 0)
            red[1][wave] = c;
    }
    const uint32_t mine = __popc(word), scan = wave_scan(mine, lane), sum = (uint32_t)__builtin_amdgcn_readlane((int)scan, 63);
    const bool listed = sum <= (uint32_t)kMoveList;
    if (wave == 0 && listed)
        for (uint32_t i = 0; i < mine; ++i)
            list[scan - mine + i] = src + i;
    __syncthreads();
    const uint32_t base = red[0][0] + red[0][1] + red[0][2] + red[0][3], at = base + scan - mine;
    if (tid == 0 && blockIdx.x == 0 && seg < s.H)
        t.out.n_outliers[seg] = red[1][0] + red[1][1] + red[1][2] + red[1][3];

#pragma unroll
    for (int u = 0; u < kWords; ++u)
        if (tid + kMoveThreads * u < n_words)
            t.out.codes[to0 * s.row_words + tid + kMoveThreads * u] = code[u];
    const uint2 *pay = reinterpret_cast<const uint2 *>(t.in.outliers);
    uint2 *out = reinterpret_cast<uint2 *>(t.out.outliers);
    if (listed) {
        for (uint32_t i = tid; i < sum; i += kMoveThreads) {
            const uint64_t f = list[i], o = (uint64_t)base + i;
            if (o < t.out_capacity)
                out[o] = f < t.in_capacity ? pay[f] : make_uint2(0u, 0u);
        }
    } else {
        for (uint32_t i = wave; i < mine; i += kMoveThreads / 64) {
            const uint64_t f = (uint64_t)src + i, o = (uint64_t)at + i;
            if (o < t.out_capacity)
                out[o] = f < t.in_capacity ? pay[f] : make_uint2(0u, 0u);
        }
    }
    if (wave == 1 && lane < n) {
        const int64_t to = to0 + lane;
        t.out.flags[to] = word;
        t.out.row_off[to] = at;
        t.out.sigma[to] = sigma;
        if (to == (int64_t)s.B * s.H * s.n_keep - 1) {
            const uint32_t total = at + mine;
            t.out.row_off[to + 1] = total;
            t.out.n_outliers[s.H] = total;
            *t.out.status = *t.in.status | (total > t.out_capacity ? HQMQ_STATUS_OUTLIER_OVERFLOW : 0u);
        }
    }
}

hipError_t launch_evict_compact(const CompactShape &s, const CompactBatch &batch, int n_tensors, hipStream_t stream)
{
    hipLaunchKernelGGL(k_compact_count, dim3((unsigned)s.blocks_per_seg, (unsigned)(s.B * s.H), (unsigned)n_tensors), dim3(kCompactRows), 0, stream, s, batch);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess)
        return err;
    const int64_t blocks = (int64_t)s.B * s.H * s.blocks_per_seg;
    if (blocks > kCompactDirect) {
        hipLaunchKernelGGL(k_compact_groups, dim3((unsigned)((blocks + kCompactGroup - 1) / kCompactGroup), (unsigned)n_tensors), dim3(kMoveThreads), 0, stream, s);
        err = hipGetLastError();
        if (err != hipSuccess)
            return err;
    }
    const dim3 grid((unsigned)((s.n_keep + kMoveRows - 1) / kMoveRows), (unsigned)(s.B * s.H), (unsigned)n_tensors);
    hipLaunchKernelGGL(k_compact_move, grid, dim3(kMoveThreads), 0, stream, s, batch);
    return hipGetLastError();
}

}  // namespace hqmq
