// Declarations shared by the kernels of the paged 4-bit cache (hqmq_cache4_rows.hip, hqmq_cache4_attend.hip) and the C ABI
// (hqmq_api.hip).  Not part of the public ABI (include/hqmq_cache4.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "hqmq_cache4.h"

namespace hqmq {

// Groups of 32 channels that a row of D channels takes: a part of the V layout is 4, 2 or 1 of them.
constexpr int cache4_groups(int D) { return D <= 128 ? (D + 31) / 32 : (D + 63) / 64 * 2; }

struct Cache4 {
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int32_t n_pages, page_shift, H, D;
    int32_t NG;      // groups of a row
    int32_t format;
};

struct Cache4Seqs {
    const int32_t *table, *lengths, *starts;  // starts: null for n_rows / n_seqs rows each
    int32_t n_seqs, n_rows, pitch;
    int32_t rows_each;                        // where starts is null
};

struct Cache4Rows {
    uint16_t *data;
    int64_t row, head;  // element strides
};

// 8 channels of a row, at any address that is a multiple of 2 (memory takes vector accesses of any alignment here).
typedef uint32_t cache4_u4 __attribute__((ext_vector_type(4)));
struct __attribute__((packed, aligned(2))) Cache4Eight {
    cache4_u4 bits;
};
__device__ __forceinline__ cache4_u4 load8(const uint16_t *p) { return reinterpret_cast<const Cache4Eight *>(p)->bits; }
__device__ __forceinline__ void store8(uint16_t *p, cache4_u4 bits) { reinterpret_cast<Cache4Eight *>(p)->bits = bits; }

// The last n of a head's channels, 1 .. 7 and the same for all lanes: in pieces of 4, 2 and 1, or, where 8 precede the head's end, these
// without the first 8 - n of them (no lane waits for what another branch has loaded).
struct __attribute__((packed, aligned(2))) Cache4Four {
    uint64_t bits;
};
struct __attribute__((packed, aligned(2))) Cache4Two {
    uint32_t bits;
};
__device__ __forceinline__ cache4_u4 load_some(const uint16_t *p, int n)
{
    uint64_t four = 0, rest = 0;
    if (n & 4)
        four = reinterpret_cast<const Cache4Four *>(p)->bits;
    if (n & 1)
        rest = (uint64_t)p[n - 1] << (16 * (n & 2));
    if (n & 2)
        rest |= reinterpret_cast<const Cache4Two *>(p + (n & 4))->bits;
    const uint64_t low = n & 4 ? four : rest, high = n & 4 ? rest : 0;
    return cache4_u4{(uint32_t)low, (uint32_t)(low >> 32), (uint32_t)high, (uint32_t)(high >> 32)};
}
__device__ __forceinline__ void store_some(uint16_t *p, cache4_u4 bits, int n)
{
    const uint64_t low = (uint64_t)bits[1] << 32 | bits[0];
    uint64_t rest = low;
    if (n & 4) {
        reinterpret_cast<Cache4Four *>(p)->bits = low;
        rest = (uint64_t)bits[3] << 32 | bits[2];
    }
    if (n & 2)
        reinterpret_cast<Cache4Two *>(p + (n & 4))->bits = (uint32_t)rest;
    if (n & 1)
        p[n - 1] = (uint16_t)(rest >> (16 * (n & 2)));
}
__device__ __forceinline__ cache4_u4 last_of(cache4_u4 x, int n)
{
    const int back = 8 - n;
    if (back & 4)
        x = cache4_u4{x[2], x[3], 0u, 0u};
    if (back & 2)
        x = cache4_u4{x[1], x[2], x[3], 0u};
    if (back & 1)
        x = cache4_u4{__builtin_amdgcn_alignbit(x[1], x[0], 16), __builtin_amdgcn_alignbit(x[2], x[1], 16), __builtin_amdgcn_alignbit(x[3], x[2], 16),
                      x[3] >> 16};
    return x;
}

// Division of numbers below 2^30 by one that the host knows: with l = ceil(log2 d) and m = ceil(2^(30 + l) / d), which is at most 2^31
// (2^l < 2 d) and makes products below 2^61, m is less than 1 above 2^(30 + l) / d.  So n m / 2^(30 + l) exceeds n / d by less than
// n / 2^(30 + l) <= n / (2^30 d) < 1 / d, and has the same whole part: the next one is 1 / d away at least.
struct Divisor {
    uint32_t mul, shift;
};
inline Divisor make_divisor(uint32_t d)
{
    uint32_t l = 0;
    while ((1u << l) < d)
        ++l;
    return Divisor{(uint32_t)(((1ull << (30 + l)) + d - 1) / d), 30 + l};
}
__host__ __device__ __forceinline__ int divided(int n, Divisor d) { return (int)((uint64_t)(uint32_t)n * d.mul >> d.shift); }

// What no kernel writes while it runs, so that uniform loads of it are scalar ones (which do not wait for the vector loads before them).
typedef const __attribute__((address_space(4))) int32_t *ConstInts;
__device__ __forceinline__ ConstInts const_ints(const int32_t *p) { return (ConstInts)p; }

// Sequence i of a batch: its tokens, its rows and the position of the first of them (negative: more rows than tokens).
struct Cache4Seq {
    int32_t length, first_row, n, pos0;
};
__device__ __forceinline__ Cache4Seq cache4_seq(const Cache4Seqs &b, int page_shift, int i)
{
    Cache4Seq s;
    const int most = b.pitch << page_shift;
    s.length = min(max(const_ints(b.lengths)[i], 0), most);
    if (b.starts) {  // inside the tensors, whatever they hold
        s.first_row = min(max(const_ints(b.starts)[i], 0), b.n_rows);
        s.n = min(max(const_ints(b.starts)[i + 1], s.first_row), b.n_rows) - s.first_row;
    } else {
        s.first_row = i * b.rows_each;
        s.n = b.rows_each;
    }
    s.pos0 = s.length - s.n;
    return s;
}

// Places of a launch along the rows of all sequences, where a place for each of the largest sequence's tiles would leave most of them
// empty: sequence i has those from first(i) = (starts[i] mul >> shift) + extra i on, at least mul n_i / 2^shift + extra of them.
struct Cache4Flat {
    int32_t on, mul, shift, extra;
};
__device__ __forceinline__ int cache4_first(const Cache4Seqs &b, const Cache4Flat &f, int i)
{
    return (int)((int64_t)min(max(const_ints(b.starts)[i], 0), b.n_rows) * f.mul >> f.shift) + f.extra * i;
}
// The sequence of a place, the last whose first place is not behind it, or -1: every lane of the wave asks for one of 64 in each round.
__device__ __forceinline__ int cache4_seq_at(const Cache4Seqs &b, const Cache4Flat &f, int place)
{
    int from = 0, n = b.n_seqs;
    const int lane = threadIdx.x & 63;
    do {
        const int step = (n + 63) / 64, i = lane * step;
        const bool before = i < n && cache4_first(b, f, from + i) <= place;
        const int count = __popcll(__builtin_amdgcn_ballot_w64(before));
        if (count == 0)  // in the first round only
            return -1;
        from += (count - 1) * step;
        n = min(step, n - (count - 1) * step);
    } while (n > 1);
    return __builtin_amdgcn_readfirstlane(from);
}
inline int64_t cache4_places(const Cache4Flat &f, int64_t n_rows, int64_t n_seqs) { return (n_rows * f.mul >> f.shift) + f.extra * n_seqs; }

// ---- codes ------------------------------------------------------------------------------------------------------------

typedef _Float16 cache4_h2 __attribute__((ext_vector_type(2)));

// Two values of a byte of e2m1 codes times a power of two (exact in fp16), byte kByte of the word.
template <int kByte>
__device__ __forceinline__ cache4_h2 e2m1_pair(uint32_t word, float scale)
{
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, kByte);
}

// Integer codes c in the two low (kHigh: high) bytes of a word times s plus m, rounded once.  A byte 0 .. 15 read as an fp8 number
// (4 bits of exponent, 3 of mantissa, the smallest ones denormal) is c 2^-9 for each of them, so one conversion with a scale of
// 2^9 gives both codes as fp16 numbers.
template <bool kHigh>
__device__ __forceinline__ cache4_h2 int4_pair(uint32_t bytes, cache4_h2 s, cache4_h2 m)
{
    return __builtin_elementwise_fma(__builtin_bit_cast(cache4_h2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(bytes, 512.f, kHigh)), s, m);
}

__device__ __forceinline__ float e8m0(uint32_t byte) { return __uint_as_float(byte << 23); }

// Where dword w (channels 8 w .. 8 w + 7) of token t of a block of four lies in the block of V codes: first byte, and how many runs
// of how many bytes it is split into, kStep(t) apart.
struct Cache4Place {
    int32_t at, runs, bytes;  // run r at `at` + r * 4 * bytes
};
__device__ __forceinline__ Cache4Place cache4_v_place(int NG, int w, int t)
{
    const int whole = NG & ~3;  // groups in parts of 128 channels
    const int w64 = 4 * whole, w32 = 4 * (NG & ~1);
    if (w < w64)
        return {16 * w + 4 * t, 1, 4};
    if (w < w32)
        return {16 * w64 + 16 * (w - w64) + 2 * t, 2, 2};
    return {16 * w32 + 16 * (w - w32) + t, 4, 1};
}

// ---- launches ---------------------------------------------------------------------------------------------------------

hipError_t launch_cache4_rows(bool write, const Cache4 &c, const Cache4Seqs &b, int max_rows, bool bf16, const Cache4Rows &k, const Cache4Rows &v,
                              hipStream_t stream);

struct Cache4Attend {
    Cache4 c;
    Cache4Seqs b;
    Cache4Rows q, out;
    float *lse;                // [n_rows][H * G] or null
    float *part_acc;           // [n_rows * H * G][n_splits][32 NG]: weighted sums of a split, relative to 2^part_ml[0]
    float *part_ml;            // [n_rows * H * G][n_splits][2]: reference (log2 domain) and sum of the weights, 0: nothing seen
    float scale;
    int32_t G, window;
    Divisor by_G, by_splits;
    Cache4Flat flat;
    int32_t n_tiles, n_splits; // workgroups along the rows (of a sequence, or of all where flat.on) and along the tokens
    int32_t split_tokens;      // of each split but the last, which goes to the end
};
struct Cache4Plan {
    int32_t blocks;            // of 16 query rows that a workgroup takes at a time: 1, 2 or 4
    int32_t n_tiles, n_splits, split_tokens;
    Cache4Flat flat;
    uint64_t ml_bytes, acc_bytes;
};
Cache4Plan plan_cache4_attend(const Cache4 &c, const Cache4Seqs &b, int max_rows, int max_length, int G, int window);
hipError_t prepare_cache4_kernels();  // once per device, before the first launch_cache4_attend on it
hipError_t launch_cache4_attend(const Cache4Attend &a, const Cache4Plan &plan, bool bf16, hipStream_t stream);

}  // namespace hqmq
