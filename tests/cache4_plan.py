"""How hqmq_cache4_attend cuts a call, asked of the library's own functions compiled for the host."""
from __future__ import annotations

import ctypes as C
import functools
import tempfile
from typing import NamedTuple

import cache4_cpp
from cache4_cpp import between

ASK = """
extern "C" void plan(int H, int D, int page_size, int n_seqs, int pages_per_seq, int has_starts, int max_rows, int max_length, int n_rows, int n_q_heads,
                     int window, int *out)
{
    static const int32_t some[1] = {};
    const hqmq_cache4_params p = {1, page_size, H, D, HQMQ_CACHE4_FLOAT};
    const hqmq_cache4_batch b = {n_seqs, pages_per_seq, max_rows, max_length, some, some, has_starts ? some : nullptr};
    const Cache4Plan plan = cache4_plan(&p, &b, n_rows, n_q_heads, window);
    const int all[5] = {plan.blocks, plan.n_tiles, plan.n_splits, plan.split_tokens, plan.flat.on};
    std::copy(all, all + 5, out);
}
"""


class Plan(NamedTuple):
    blocks: int        # of 16 query rows of a workgroup
    n_tiles: int
    n_splits: int
    split_tokens: int
    flat: bool


@functools.lru_cache(maxsize=None)
def _host() -> C.CDLL:
    device, kernels, api = "hqmq_cache4_device.h", "hqmq_cache4_attend.hip", "hqmq_api.hip"
    code = (between(device, "constexpr int cache4_groups", "// 8 channels of a row") + between(device, "struct Cache4Flat {", "__device__ __forceinline__ int cache4_first")
            + between(device, "inline int64_t cache4_places", "// ---- codes") + between(device, "struct Cache4Plan {", "Cache4Plan plan_cache4_attend")
            + between(kernels, "constexpr int kStep", "constexpr int kMergeThreads") + between(kernels, "constexpr int attend_waves", "// Blocks of rows whose sums")
            + between(kernels, "constexpr int kMostSplits", "template") + between(kernels, "constexpr int kUnits = 256", "namespace {\n\ntemplate")
            + between(api, "static Cache4 make_cache4(", 'extern "C" int32_t hqmq_cache4_sizes') + between(api, "static Cache4Seqs make_cache4_seqs", "static Cache4Rows make")
            + between(api, "static Cache4Plan cache4_plan", 'extern "C" uint64_t hqmq_cache4_attend_workspace_bytes') + ASK)
    with tempfile.TemporaryDirectory() as folder:
        host = cache4_cpp.compiled(folder, code)
    host.plan.restype, host.plan.argtypes = None, [C.c_int] * 11 + [C.POINTER(C.c_int)]
    return host


def plan(H, D, page_size, n_seqs, pages_per_seq, n_rows, n_q_heads, starts=True, max_rows=2 ** 30, max_length=2 ** 30, window=0) -> Plan:
    out = (C.c_int * 5)()
    _host().plan(H, D, page_size, n_seqs, pages_per_seq, starts, max_rows, max_length, n_rows, n_q_heads, window, out)
    return Plan(*out[:4], bool(out[4]))
