// Declarations shared by the kernels that serve a batch from packed caches (hqmq_shared.hip, hqmq_mass.hip,
// hqmq_evict.hip) and the C ABI (hqmq_api.hip).  Not part of the public ABI (include/hqmq_serve.h).
#pragma once

#include "hqmq_device.h"
#include "hqmq_serve.h"

namespace hqmq {

// Query rows of a kv head: row r = m * G + g is query head h * G + g of sequence b * n_share + m.
struct SharedArgs {
    AttendSide k, v;
    const _Float16 *q;       // [B * n_share][H * G][D]
    const int32_t *visible;  // [B * n_share][H * G] or null
    float *part_ml;          // [B * n_share * H * G][part_pitch][2]: maximum (log2 domain) and weight sum of a split
    float *part_acc;         // [..][part_pitch][128]: weighted value sums
    _Float16 *out;           // [B * n_share][H * G][D], and lse [B * n_share][H * G] or null: one share only, no partial sums; else null
    float *lse;
    float qscale;            // softmax scale * log2(e)
    int32_t T, G, n_share;
    int32_t n_splits, rows_per_split;  // workgroups along the prefix and its tokens per workgroup
    int32_t split0, part_pitch;        // the first one's place in the partial arrays, and how many places there are, the own tokens' included
};
constexpr int kMostSharedSplits = 512;  // and as many of the own tokens: kMostParts in all
struct SharedPlan {
    int32_t n_splits, rows_per_split;
};
// alone: without own tokens, so that a prefix of kTilesAlone tiles is one share and needs no merge.  One share / one per tile and the merge,
// 2 sequences, 8 heads x 128: one tile 6.0 / 8.3 us, two 7.6 / 8.3, three 8.5 / 8.3, five 12.5 / 9.8.
constexpr int kTilesAlone = 2;
SharedPlan plan_shared(const Geometry &g, int G, int n_share, bool alone);
hipError_t prepare_shared_kernels();  // once per device, before the first launch_shared on it
bool shared_is_small(int n_rows);     // of a kv head: a launch of prefixes can take the sequences' own tokens with it
// own: of the sequences' own tokens (B * n_share batch entries), or null
hipError_t launch_shared(const Geometry &g, const SharedArgs &a, const SharedArgs *own, hipStream_t stream);

struct MassArgs {
    AttendSide k;
    const _Float16 *q;
    const float *lse;        // [B * n_share][H * G], natural logarithm
    const int32_t *visible;
    const float *mass_in;    // null: decay is 0
    float *mass_out;
    float scale, decay;
    int32_t G, n_share;
};
hipError_t prepare_mass_kernels();  // once per device, before the first launch_mass on it
hipError_t launch_mass(const Geometry &g, const MassArgs &a, hipStream_t stream);

struct SelectArgs {
    const float *mass;
    const int32_t *length;
    int32_t *keep, *n_kept;
    float *kept_mass;
    int32_t B, H, T, n_sink, n_recent, n_keep;
};
uint64_t evict_select_workspace_bytes(int B, int H, int T);
hipError_t launch_evict_select(const SelectArgs &a, uint32_t *workspace, hipStream_t stream);

struct CompactTensor {
    EncodedPtrs in, out;
    const int32_t *keep;
    uint64_t in_capacity, out_capacity;
};
constexpr int kMaxCompactBatch = 24;  // 24 * 136 B of descriptors stay inside the 4 KiB of kernel arguments
struct CompactBatch {
    CompactTensor t[kMaxCompactBatch];
};
struct CompactShape {
    int32_t B, H, T, n_keep, row_words;
    int32_t blocks_per_seg;  // per (b, h), of kCompactRows rows each
    uint32_t *totals;        // [tensor]: outliers of each block [B * H * blocks_per_seg], of each quarter of one [4 * B * H * blocks_per_seg],
                             // and of kCompactGroup blocks each, if there are more than kCompactDirect
    uint64_t totals_stride;  // of a tensor, in entries
};
constexpr int kCompactRows = 256;
// Summing the blocks before it costs a workgroup 1.7 us per 1000 of them, the launch that makes the groups 4.6 us (4096 blocks 56.9 us
// without, 4104 with it 52.3).
constexpr int kCompactGroup = 1024, kCompactDirect = 2560;
hipError_t launch_evict_compact(const CompactShape &s, const CompactBatch &batch, int n_tensors, hipStream_t stream);

}  // namespace hqmq
