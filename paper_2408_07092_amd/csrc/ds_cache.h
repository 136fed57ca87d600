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
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int kMostTokens = 1 << 30;  // of a sequence: what the kernels step past its end stays within 32 bits

// A running maximum before any score, and where every score is -infinity: what is folded in later takes its weight
// away (2^(kLeast - m) = 0), and the weights of scores of -infinity are 0, not 2^(-inf + inf).
constexpr float kLeast = -3e38f;

// n / d of 0 <= n < 2^31 by a product: with 2^(l-1) < d <= 2^l and m = floor(2^(31+l) / d) + 1, m d lies between 2^(31+l) and
// 2^(31+l) + 2^l, so n m / 2^(31+l) exceeds n / d by less than 1 / d.  (A division of the compiler's is a chain of some 25
// instructions, and a workgroup's beginning had ten of them.)
struct Quotient {
    uint32_t m;
    int shift;
    void set(uint32_t d)
    {
        int l = 0;
        while ((1ull << l) < d) ++l;
        m = (uint32_t)((1ull << (31 + l)) / d + 1);
        shift = 31 + l;
    }
    __device__ __forceinline__ int of(int n) const { return (int)((uint64_t)(uint32_t)n * m >> shift); }
};

// ---------------------------------------------------------------- prompt attention
constexpr int kPromptRows = 128;   // rows (token * G + head of the group) of a workgroup
constexpr int kPromptParts = 64;   // parts that keys are split into at most: a lane of the join for each

struct PromptArgs {
    const void *q, *K, *V;
    void *out;
    const int32_t *q_start, *kv_start, *kv_len;   // (paged: kv_len by table row)
    const int32_t *rows, *table;                  // paged only
    int64_t q_stride, out_stride, kv_stride, kv_head_stride, kv_elems;
    float2 *part_ml;                              // [n_split][total_q][Hq]: maximum and sum of a row over a part of the keys
    float *part_acc;                              // [n_split][total_q][Hq][d]: its numerator
    Quotient by_G, by_Hkv, by_Hq;
    int n_seqs, Hq, Hkv, G, total_q, n_tiles, n_split, cus;
    int n_pages, page_log2, max_pages, n_table;   // paged only
};
struct PromptPlan {
    int G, n_tiles, n_split;
    size_t off_acc, total;
};
void make_prompt_plan(const ds_prompt_t &m, PromptPlan *p, size_t workspace_bytes = SIZE_MAX);   // total: 256 at least
hipError_t launch_prompt(PromptArgs a, bool paged, int dtype, hipStream_t st);

// Row tiles of packed sequences, numbered without a prefix sum: sequence s has its tiles from number
// floor(q_start[s] G / 128) + s on, which leaves room for the part tile that each one may end in.
__device__ __forceinline__ int tile_base(int q_start, int G, int s) { return (int)((int64_t)q_start * G / kPromptRows) + s; }

// The last i of [0, n) whose key is at or before x, keys ascending: 64 of them looked at at a time, by every
// wavefront for itself (x the same in all lanes).  Keys that do not ascend give some i.
template <class Key>
__device__ __forceinline__ int last_at_or_before(int n, int x, Key key)
{
    const int lane = threadIdx.x & 63;
    int first = 0, end = n;
    while (end - first > 1) {
        const int step = (end - first + 63) / 64, i = first + lane * step;
        const bool before = i < end && key(min(i, n - 1)) <= x;
        const int k = __builtin_popcountll(__ballot(before));
        first += max(k - 1, 0) * step;
        end = min(end, first + step);
    }
    return first;
}

// ---------------------------------------------------------------- paged decode
constexpr int kPiece = 64;         // tokens that a share is counted in: 16 for each wavefront of a workgroup
constexpr int kLead = 3;           // pieces that a unit counts for besides its own
constexpr int kWhole = 4;          // a unit of up to so many pieces is not cut
constexpr int kShareAtLeast = 2;   // pieces

struct PagedArgs {
    const void *q, *K, *V;
    float *out, *part;
    uint32_t *arrived;             // per sequence and unit, zero between calls
    const int32_t *rows, *lens, *table;
    Quotient by_units, by_passes;
    int n, Hkv, G, passes;         // passes of 16 heads over a KV head's rows
    bool join_here;                // parts are joined by the workgroup that is last, not by a launch after this one
    int n_pages, page_log2, max_pages, n_table;
};
struct PagedPlan {
    int G, passes, GH, wgs;
    bool join_here;
    size_t off_arrived, total;
};
void make_paged_plan(const ds_pages_t &g, int n, int Hq, int max_len, PagedPlan *p);
hipError_t launch_paged(PagedArgs a, const PagedPlan &p, int dtype, hipStream_t st);

struct AppendPagedArgs {
    const u32x4 *k_new, *v_new;
    u32x4 *K, *V;
    const int32_t *new_start, *rows, *start, *table;
    int64_t new_stride;            // 16-byte pieces from token to token
    int n, total_new, Hkv;
    int n_pages, page_log2, max_pages, n_table;
};
hipError_t launch_append_paged(const AppendPagedArgs &a, hipStream_t st);

// ---------------------------------------------------------------- the books of a paged cache
constexpr int kPagesListed = 2048; // rows that a call may list

struct PagesArgs {
    int32_t *refs, *table, *lens;
    const int32_t *rows;               // fork: the sources
    const int32_t *n_new, *dst;        // extend; fork
    int32_t *start;                    // extend
    int4 *copies;                      // fork and compact: {from, to, tokens, 0}
    int32_t *n_copies, *status;
    int n, n_pages, page_log2, max_pages, n_rows;
};
struct CopyPagesArgs {
    u32x4 *K, *V;
    const int4 *copies;
    const int32_t *n_copies;
    int max_copies, Hkv, n_pages, page_log2;
};
hipError_t launch_pages_extend(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_fork(const PagesArgs &a, hipStream_t st);
hipError_t launch_pages_free(const PagesArgs &a, hipStream_t st);
size_t pages_workspace(int n_pages);
hipError_t launch_pages_compact(const PagesArgs &a, void *ws, hipStream_t st);
hipError_t launch_pages_copy(const CopyPagesArgs &a, hipStream_t st);

}  // namespace ds
