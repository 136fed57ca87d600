// The books of a paged cache, kept on the device so that a serving step that takes and gives back pages
// can be captured: who holds which page (table, lens), and how often a page is held (refs, 0 = free).
//
// What is given out is always the lowest free pages, ascending, in the order of the call's list, so the
// books follow from the calls alone and not from how they ran.  The counts themselves are the free list:
// one workgroup looks through them, 16 K pages a round, until it has enough.  Its time is latency (a
// round of loads, a scan over the workgroup, a few barriers); the copies of pages are what moves data.
#include <algorithm>

#include "ds_device.h"
#include "ds_cache.h"

namespace ds {

constexpr int kBooks = 1024, kBookWaves = kBooks / 64;  // threads of the workgroup that keeps the books
constexpr int kListed = kPagesListed / kBooks;          // list entries of a thread
constexpr int kFound = 4096;                            // free pages that are remembered in LDS

__device__ __forceinline__ int pages_in(const PagesArgs &a, int tokens) { return tokens > 0 ? ((tokens - 1) >> a.page_log2) + 1 : 0; }
__device__ __forceinline__ bool length_ok(const PagesArgs &a, int64_t tokens) { return tokens >= 0 && tokens <= (int64_t)a.max_pages << a.page_log2; }

struct BooksLds {
    uint32_t seen[65536 / 32];        // a bit for every row
    uint32_t w[kBookWaves];
    uint32_t bad;
};

// Marks row r; whether it was marked already or is none.
__device__ __forceinline__ bool mark(const PagesArgs &a, uint32_t *seen, int r)
{
    if (r < 0 || r >= a.n_rows) return true;
    const uint32_t bit = 1u << (r & 31);
    return (atomicOr(&seen[r >> 5], bit) & bit) != 0u;
}

// The counts of 16 pages (pages that are none count as held), and which of them are free (bit i: the i-th).
struct Counts {
    typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
    i32x4 v[4];
    __device__ __forceinline__ Counts(const int32_t *refs, int n_pages, int mine)
    {
        if (mine + 16 <= n_pages) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<const i32x4 *>(refs + mine + 4 * i);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i / 4][i % 4] = mine + i < n_pages ? refs[mine + i] : 1;
        }
    }
    __device__ __forceinline__ uint32_t free() const
    {
        uint32_t f = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) f |= v[i / 4][i % 4] <= 0 ? 1u << i : 0u;
        return f;
    }
};

// Goes through the free pages in ascending order, take(rank, page) for each, until `want` have been seen; how many
// there are, or want if there are as many.  All threads of the workgroup call it.  first: the counts of the thread's
// pages of the first round, which a caller can have asked for before.  take may write the count of the page that it is given (in
// the first round it is read no more, in the others a thread has read its 16 before).
template <class Take>
__device__ __forceinline__ uint32_t each_free(const int32_t *refs, int n_pages, uint32_t want, uint32_t *s_w, const Counts &first, Take take)
{
    uint32_t have = 0;
    for (int p0 = 0; p0 < n_pages && have < want; p0 += kBooks * 16) {
        const int mine = p0 + (int)threadIdx.x * 16;
        uint32_t free = p0 == 0 ? first.free() : Counts(refs, n_pages, mine).free(), total;
        uint32_t rank = have + block_exclusive_scan<kBookWaves>((uint32_t)__builtin_popcount(free), s_w, &total);
        for (; free && rank < want; free &= free - 1u, ++rank) take(rank, mine + __builtin_ctz(free));
        have += total;
    }
    return min(have, want);
}

// Rows grow: see ds_pages_extend.
__global__ __launch_bounds__(kBooks) void k_pages_extend(PagesArgs a)
{
    __shared__ BooksLds s;
    __shared__ uint32_t first[kPagesListed];   // pages that the list's entries before this one need
    __shared__ int32_t found[kFound];
    const int tid = threadIdx.x;
    const Counts counts0(a.refs, a.n_pages, tid * 16);   // (asked for first: what they wait for is not needed before)
    for (int i = tid; i < 65536 / 32; i += kBooks) s.seen[i] = 0u;
    if (tid == 0) s.bad = 0u;
    __syncthreads();
    int row[kListed], len[kListed], more[kListed];
    uint32_t need[kListed], sum = 0;
#pragma unroll
    for (int k = 0; k < kListed; ++k) {
        const int i = tid * kListed + k;
        row[k] = len[k] = more[k] = 0;
        need[k] = 0u;
        if (i < a.n) {
            row[k] = a.rows[i];
            more[k] = a.n_new[i];
            uint32_t code = mark(a, s.seen, row[k]) ? DS_PAGES_ROWS : 0;
            if (code == 0) {
                len[k] = a.lens[row[k]];
                if (more[k] < 0 || !length_ok(a, len[k]) || !length_ok(a, (int64_t)len[k] + more[k])) code = DS_PAGES_LENGTH;
            }
            if (code) atomicMax(&s.bad, code);
            else need[k] = min((uint32_t)(pages_in(a, len[k] + more[k]) - pages_in(a, len[k])), (uint32_t)a.n_pages + 1u);
        }
        sum += need[k];
    }
    uint32_t total;
    uint32_t before = block_exclusive_scan<kBookWaves>(sum, s.w, &total);  // (2048 entries of 2^20 + 1 pages at most: no overflow)
#pragma unroll
    for (int k = 0; k < kListed; ++k) {
        if (tid * kListed + k < a.n) first[tid * kListed + k] = before;
        before += need[k];
    }
    __syncthreads();
    uint32_t code = s.bad;
    auto give = [&](uint32_t rank, int page) {
        int lo = 0, hi = a.n;               // the last entry that starts at or before the rank: the one it belongs to
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first[mid] <= rank) lo = mid;
            else hi = mid;
        }
        const int r = a.rows[lo];
        a.table[(size_t)r * a.max_pages + pages_in(a, a.lens[r]) + (rank - first[lo])] = page;
        a.refs[page] = 1;
    };
    if (code == 0 && total > 0) {
        if (total > (uint32_t)a.n_pages) {
            code = DS_PAGES_NO_ROOM;
        } else {
            const uint32_t got = each_free(a.refs, a.n_pages, total, s.w, counts0, [&](uint32_t rank, int page) {
                if (rank < kFound) found[rank] = page;
            });
            __syncthreads();
            if (got < total) {
                code = DS_PAGES_NO_ROOM;
            } else if (total <= kFound) {
                for (uint32_t rank = tid; rank < total; rank += kBooks) give(rank, found[rank]);
            } else {
                each_free(a.refs, a.n_pages, total, s.w, counts0, give);
            }
        }
    }
    __syncthreads();   // (give reads the lengths)
#pragma unroll
    for (int k = 0; k < kListed; ++k) {
        const int i = tid * kListed + k;
        if (i < a.n) {
            a.start[i] = code ? -1 : len[k];
            if (!code) a.lens[row[k]] = len[k] + more[k];
        }
    }
    if (tid == 0) *a.status = (int32_t)code;
}

// dst shares src's full pages: wavefront (w, y) of n_waves by n_y takes every n_waves-th entry of the list, and every
// n_y-th 256 pages of it.
constexpr int kShared = 256;
__device__ __forceinline__ void share_pages(const PagesArgs &a, int w, int n_waves, int y, int n_y)
{
    constexpr int kFlight = kShared / 64;
    const int lane = threadIdx.x & 63;
    for (int i = w; i < a.n; i += n_waves) {
        const int32_t *from = a.table + (size_t)a.rows[i] * a.max_pages;
        int32_t *to = a.table + (size_t)a.dst[i] * a.max_pages;
        const int full = a.lens[a.rows[i]] >> a.page_log2;
        for (int j0 = y * kShared + lane; j0 < full; j0 += n_y * kShared) {
            int p[kFlight];
#pragma unroll
            for (int k = 0; k < kFlight; ++k) p[k] = from[min(j0 + 64 * k, full - 1)];
#pragma unroll
            for (int k = 0; k < kFlight; ++k)
                if (j0 + 64 * k < full) {
                    to[j0 + 64 * k] = p[k];
                    if ((uint32_t)p[k] < (uint32_t)a.n_pages) atomicAdd(&a.refs[p[k]], 1);
                }
        }
    }
}

// Sequences branch: see ds_pages_fork.  rows: the sources.  share: the full pages too (else a launch of its own does them).
__global__ __launch_bounds__(kBooks) void k_pages_fork(PagesArgs a, int share)
{
    __shared__ BooksLds s;
    __shared__ int32_t found[kPagesListed];
    const int tid = threadIdx.x;
    const Counts counts0(a.refs, a.n_pages, tid * 16);
    for (int i = tid; i < 65536 / 32; i += kBooks) s.seen[i] = 0u;
    if (tid == 0) s.bad = 0u;
    __syncthreads();
    int src[kListed], dst[kListed], len[kListed];
    uint32_t half = 0;   // bit k: entry k's last page is partly filled
#pragma unroll
    for (int k = 0; k < kListed; ++k) {
        const int i = tid * kListed + k;
        src[k] = dst[k] = len[k] = 0;
        if (i < a.n) {
            src[k] = a.rows[i];
            dst[k] = a.dst[i];
            uint32_t code = src[k] < 0 || src[k] >= a.n_rows || mark(a, s.seen, dst[k]) ? DS_PAGES_ROWS : 0;
            if (code == 0) {
                len[k] = a.lens[src[k]];
                if (a.lens[dst[k]] != 0) code = DS_PAGES_ROWS;
                else if (!length_ok(a, len[k])) code = DS_PAGES_LENGTH;
            }
            if (code) atomicMax(&s.bad, code);
            else if (len[k] & ((1 << a.page_log2) - 1)) half |= 1u << k;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kListed; ++k)   // a row that is branched is none that a branch goes to
        if (tid * kListed + k < a.n && src[k] >= 0 && src[k] < a.n_rows && (s.seen[src[k] >> 5] >> (src[k] & 31) & 1u))
            atomicMax(&s.bad, (uint32_t)DS_PAGES_ROWS);
    uint32_t total;
    uint32_t rank = block_exclusive_scan<kBookWaves>((uint32_t)__builtin_popcount(half), s.w, &total);
    uint32_t code = s.bad;
    if (code == 0 && total > 0) {
        const uint32_t got = each_free(a.refs, a.n_pages, total, s.w, counts0, [&](uint32_t r, int page) { found[r] = page; });
        if (got < total) code = DS_PAGES_NO_ROOM;
    }
    __syncthreads();
    if (!code) {
        // (lens of the branches come last: share_pages reads those of the sources, which are other rows)
        const int wave = tid >> 6, n_y = max(1, kBookWaves / a.n);
        if (share) share_pages(a, wave / n_y, kBookWaves / n_y, wave % n_y, n_y);
#pragma unroll
        for (int k = 0; k < kListed; ++k)
            if (tid * kListed + k < a.n) {
                if (half >> k & 1u) {
                    const int full = len[k] >> a.page_log2, page = found[rank];
                    a.table[(size_t)dst[k] * a.max_pages + full] = page;
                    a.refs[page] = 1;
                    a.copies[rank] = make_int4(a.table[(size_t)src[k] * a.max_pages + full], page, len[k] & ((1 << a.page_log2) - 1), 0);
                    ++rank;
                }
                a.lens[dst[k]] = len[k];
            }
    }
    if (tid == 0) {
        *a.n_copies = code ? 0 : (int32_t)total;
        *a.status = (int32_t)code;
    }
}
__global__ __launch_bounds__(kWG) void k_pages_share(PagesArgs a)
{
    if (*a.status == 0) share_pages(a, (int)blockIdx.x, (int)gridDim.x, (int)(blockIdx.y * (kWG / 64) + (threadIdx.x >> 6)), (int)(gridDim.y * (kWG / 64)));
}

// Rows end: see ds_pages_free.  A workgroup for each row; each looks at the whole list, so that all agree on it.
__global__ __launch_bounds__(kWG) void k_pages_free(PagesArgs a)
{
    __shared__ uint32_t seen[65536 / 32], s_bad;
    const int tid = threadIdx.x;
    for (int i = tid; i < (a.n_rows + 31) / 32; i += kWG) seen[i] = 0u;
    if (tid == 0) s_bad = 0u;
    __syncthreads();
    for (int i = tid; i < a.n; i += kWG) {   // (a length that another workgroup has set to 0 by now was right before)
        const int r = a.rows[i];
        const uint32_t code = mark(a, seen, r) ? DS_PAGES_ROWS : length_ok(a, a.lens[r]) ? DS_PAGES_DONE : DS_PAGES_LENGTH;
        if (code) atomicMax(&s_bad, code);
    }
    __syncthreads();
    const uint32_t bad = s_bad;
    if (blockIdx.x == 0 && tid == 0) *a.status = (int32_t)bad;
    if (bad) return;
    const int row = a.rows[blockIdx.x];
    const int held = pages_in(a, a.lens[row]);
    int32_t *entry = a.table + (size_t)row * a.max_pages;
    constexpr int kFlight = 8;
    for (int j0 = tid; j0 < held; j0 += kWG * kFlight) {
        int p[kFlight];
#pragma unroll
        for (int k = 0; k < kFlight; ++k) p[k] = entry[min(j0 + kWG * k, held - 1)];
#pragma unroll
        for (int k = 0; k < kFlight; ++k)
            if (j0 + kWG * k < held) {
                if ((uint32_t)p[k] < (uint32_t)a.n_pages) atomicSub(&a.refs[p[k]], 1);
                entry[j0 + kWG * k] = -1;
            }
    }
    __syncthreads();
    if (tid == 0) a.lens[row] = 0;
}

// The live pages behind the first n_live go to the free ones among them: see ds_pages_compact.  Leaves n_live and where
// those pages went in the workspace: ws[0], and ws[4 + page], where a page behind the front that nobody holds stays (an entry of the
// table may name one if the books were not in order); ws[4 + n_pages ..] lists the free ones.
__global__ __launch_bounds__(kBooks) void k_pages_compact(PagesArgs a, int32_t *ws)
{
    __shared__ uint32_t s_w[kBookWaves], s_bad;
    const int tid = threadIdx.x;
    int32_t *map = ws + 4, *holes = map + a.n_pages;
    const Counts counts0(a.refs, a.n_pages, tid * 16);
    bool bad = !length_ok(a, a.lens[min(tid, a.n_rows - 1)]);
    if (tid == 0) s_bad = 0u;
    __syncthreads();
    for (int r = tid + kBooks; r < a.n_rows; r += kBooks) bad |= !length_ok(a, a.lens[r]);
    if (bad) s_bad = 1u;   // (seen by all behind the barriers of each_free)
    const int n_live = a.n_pages - (int)each_free(a.refs, a.n_pages, (uint32_t)a.n_pages, s_w, counts0, [](uint32_t, int) {});
    if (s_bad) {
        if (tid == 0) {
            ws[0] = a.n_pages;   // (k_pages_remap finds nothing to do)
            *a.n_copies = 0;
            *a.status = DS_PAGES_LENGTH;
        }
        return;
    }
    // holes (free, before n_live) and movers (held, from n_live on), ascending: as many of one as of the other
    uint32_t n_holes = 0, n_movers = 0;
    for (int p0 = 0; p0 < a.n_pages; p0 += kBooks * 16) {
        const int mine = p0 + tid * 16;
        const uint32_t there = mine + 16 <= a.n_pages ? 0xffffu : mine < a.n_pages ? (1u << (a.n_pages - mine)) - 1u : 0u;
        const uint32_t front = mine + 16 <= n_live ? 0xffffu : mine < n_live ? (1u << (n_live - mine)) - 1u : 0u;
        const uint32_t free = p0 == 0 ? counts0.free() : Counts(a.refs, a.n_pages, mine).free();
        uint32_t hole = free & front, mover = ~free & there & ~front, total;
        const uint32_t rank = block_exclusive_scan<kBookWaves>((uint32_t)__builtin_popcount(hole) | (uint32_t)__builtin_popcount(mover) << 16, s_w, &total);
        uint32_t h = n_holes + (rank & 0xffffu), m = n_movers + (rank >> 16);   // (16384 of each in a round at most)
        for (; hole; hole &= hole - 1u) holes[h++] = mine + __builtin_ctz(hole);
        for (; mover; mover &= mover - 1u) a.copies[m++].x = mine + __builtin_ctz(mover);
        // (all of them for now: the movers' entries are written below)
        if (mine >= n_live && mine + 16 <= a.n_pages) {
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<int4 *>(map + mine + i) = make_int4(mine + i, mine + i + 1, mine + i + 2, mine + i + 3);
        } else {
            for (int i = max(mine, n_live); i < min(mine + 16, a.n_pages); ++i) map[i] = i;
        }
        n_holes += total & 0xffffu;
        n_movers += total >> 16;
    }
    __syncthreads();
    for (uint32_t i = tid; i < n_holes; i += kBooks) {
        const int from = a.copies[i].x, to = holes[i];
        a.copies[i] = make_int4(from, to, 1 << a.page_log2, 0);
        map[from] = to;
        a.refs[to] = a.refs[from];
        a.refs[from] = 0;
    }
    if (tid == 0) {
        ws[0] = n_live;
        *a.n_copies = (int32_t)n_holes;
        *a.status = DS_PAGES_DONE;
    }
}
__global__ __launch_bounds__(kWG) void k_pages_remap(PagesArgs a, const int32_t *ws)
{
    const int row = blockIdx.x, held = min(pages_in(a, a.lens[row]), a.max_pages), n_live = ws[0];
    int32_t *entry = a.table + (size_t)row * a.max_pages;
    for (int j = blockIdx.y * kWG + threadIdx.x; j < held; j += gridDim.y * kWG) {
        const int p = entry[j];
        if (p >= n_live && p < a.n_pages) entry[j] = ws[4 + p];
    }
}

// Copies the listed pages' rows, K's and V's: 16 lanes to a row of 256 bytes, a workgroup 64 rows of an entry at a
// time.  Bound by memory, a read and a write of every row.
__global__ __launch_bounds__(kWG) void k_pages_copy(CopyPagesArgs a)
{
    const int n = min(max(*a.n_copies, 0), a.max_copies), P = 1 << a.page_log2;
    const int groups = (2 * a.Hkv * P) / 64;      // of 64 rows, in an entry (P is 16 or more and there are two pools ..
    const int rest = (2 * a.Hkv * P) % 64;        // .. so what is left is 32 rows, or none)
    const int per = groups + (rest ? 1 : 0);
    const uint32_t all = (uint32_t)n * (uint32_t)per;   // (2^28 at most)
    for (uint32_t w = blockIdx.x; w < all; w += gridDim.x) {
        const int4 e = a.copies[w / (uint32_t)per];
        if ((uint32_t)e.x >= (uint32_t)a.n_pages || (uint32_t)e.y >= (uint32_t)a.n_pages) continue;
        const int r0 = (int)(w % (uint32_t)per) * 64 + (threadIdx.x >> 4);
        u32x4 v[4];
        size_t to[4];
        bool on[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int r = r0 + 16 * k, x = r >> a.page_log2, t = r & (P - 1);   // x: head of K, then head of V
            on[k] = x < 2 * a.Hkv && t < e.z;
            const int h = x < a.Hkv ? x : x - a.Hkv;
            const size_t in_page = (size_t)(h * P + t) * 16 + (threadIdx.x & 15), page = (size_t)a.Hkv * P * 16;
            to[k] = e.y * page + in_page;
            v[k] = (u32x4)(0u);
            if (on[k]) v[k] = (x < a.Hkv ? a.K : a.V)[e.x * page + in_page];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (on[k]) ((r0 + 16 * k) >> a.page_log2 < a.Hkv ? a.K : a.V)[to[k]] = v[k];
    }
}

// ---------------------------------------------------------------- launchers
hipError_t launch_pages_extend(const PagesArgs &a, hipStream_t st)
{
    DS_LAUNCH(KID_PAGES_EXTEND, k_pages_extend, dim3(1), dim3(kBooks), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_pages_fork(const PagesArgs &a, hipStream_t st)
{
    // The workgroup that keeps the books shares the full pages too if each of its wavefronts has 256 of them at most; more are
    // worth a launch.  (us of a fork and the freeing of its branches, one launch and two: one row of 256 pages 6.6 and 7.7,
    // 16 of 256 9.0 and 10.0, 4 of 512 8.7 and 9.4; on the other side 32 of 64 9.3 and 9.0, 16 of 1024 13.9 and 10.8,
    // 256 of 64 25 and 9.5.)
    const int n_y = std::max(1, kBookWaves / a.n), per = (a.max_pages + kShared - 1) / kShared;
    const bool alone = a.n <= kBookWaves && per <= n_y;
    DS_LAUNCH(KID_PAGES_FORK, k_pages_fork, dim3(1), dim3(kBooks), 0, st, a, alone ? 1 : 0);
    if (!alone) DS_LAUNCH(KID_PAGES_FORK, k_pages_share, dim3(a.n, std::min((per + kWG / 64 - 1) / (kWG / 64), 64)), dim3(kWG), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_pages_free(const PagesArgs &a, hipStream_t st)
{
    DS_LAUNCH(KID_PAGES_FREE, k_pages_free, dim3(a.n), dim3(kWG), 0, st, a);
    return hipGetLastError();
}

size_t pages_workspace(int n_pages) { return ((size_t)n_pages * 2 * 4 + 16 + 255) / 256 * 256; }

hipError_t launch_pages_compact(const PagesArgs &a, void *ws, hipStream_t st)
{
    DS_LAUNCH(KID_PAGES_COMPACT, k_pages_compact, dim3(1), dim3(kBooks), 0, st, a, static_cast<int32_t *>(ws));
    DS_LAUNCH(KID_PAGES_COMPACT, k_pages_remap, dim3(a.n_rows, std::min((a.max_pages + kWG - 1) / kWG, 64)), dim3(kWG), 0, st, a, static_cast<const int32_t *>(ws));
    return hipGetLastError();
}

hipError_t launch_pages_copy(const CopyPagesArgs &a, hipStream_t st)
{
    const int64_t work = (int64_t)a.max_copies * (((2 * a.Hkv << a.page_log2) + 63) / 64);
    DS_LAUNCH(KID_PAGES_COPY, k_pages_copy, dim3((unsigned)std::min<int64_t>(work, device_caps().cus * 8)), dim3(kWG), 0, st, a);
    return hipGetLastError();
}

}  // namespace ds
