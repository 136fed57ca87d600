// What the kernels of prompt attention and of the paged cache share: their arguments, vector types
// and the places of sequences and pages.
#pragma once

#include <hip/hip_runtime.h>

#include "ds_internal.h"

namespace ds {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- prompt attention
constexpr int kPromptRows = 128;   // rows (token * G + head of the group) of a workgroup

struct PromptArgs {
    const void *q, *K, *V;
    void *out;
    const int32_t *q_start, *kv_start, *kv_len;   // (paged: kv_len by table row)
    const int32_t *rows, *table;                  // paged only
    int64_t q_stride, out_stride, kv_stride, kv_head_stride, kv_elems;
    int n_seqs, Hkv, G, total_q, n_tiles;
    int n_pages, page_log2, max_pages, n_table;   // paged only
};
struct PromptPlan {
    int G, n_tiles;
    size_t total;
};
bool make_prompt_plan(const ds_prompt_t &m, PromptPlan *p);
hipError_t launch_prompt(PromptArgs a, bool paged, int dtype, hipStream_t st);

// Row tiles of packed sequences, numbered without a prefix sum: sequence s has its tiles from number
// floor(q_start[s] G / 128) + s on, which leaves room for the part tile that each one may end in.
__device__ __forceinline__ int tile_base(int q_start, int G, int s) { return (int)((int64_t)q_start * G / kPromptRows) + s; }

// The sequence whose tiles a number falls among, the last one that starts at or before it: 64 starts looked at at
// a time, by every wavefront for itself.  (Starts that do not ascend give some sequence.)
__device__ __forceinline__ int find_sequence(const int32_t *q_start, int n, int G, int slot)
{
    const int lane = threadIdx.x & 63;
    int first = 0, end = n;
    while (end - first > 1) {
        const int step = (end - first + 63) / 64, i = first + lane * step;
        const bool before = i < end && tile_base(q_start[min(i, n - 1)], G, i) <= slot;
        const int k = __builtin_popcountll(__ballot(before));
        first += max(k - 1, 0) * step;
        end = min(end, first + step);
    }
    return first;
}

}  // namespace ds
