// Attention over whole prompts: causal, grouped heads, packed sequences of unlike lengths, with the
// keys in rows of any stride (packed, or the contiguous caches) or in pages.
//
//   O[i] = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(s_ij - m_i),   s_ij = log2(e)/sqrt(d) q_i . k_j
//
// over the keys j <= i + nk - nq, in one pass over the keys with a running maximum m and a
// running sum.  Bound by the matrix units: 4 d flops a pair against a few bytes for each row.  8K tokens of 32 heads take
// 528 us (1.04 PFLOP/s), two of 8K in groups of 4 982 us; a library product of 16384 x 16384 x 16384 reaches 1.3 to 1.37.  What
// holds it there is power: the same launch on zeros takes 365 us, and on random data the clock is at 1.6 to 1.7 GHz, with
// the matrix units busy in 60 % of the cycles.  Short prompts are bound by a workgroup's steps one after the other, 1.2 us each
// with the compute unit to itself (97 tokens 6.6 us, 500 in groups of 4 14.8, 1500 of 32 heads 39).
//
// The G query heads of a KV head are rows of one matrix: row token * G + g.  A workgroup takes 128 of
// these rows, a wavefront 32, and walks the keys in tiles of 64 that all of its wavefronts share from LDS.  Two
// workgroups share a compute unit, 64 KiB and 240 registers a lane each.  (Two of 8K tokens in groups of 4, before the
// loads went between the products: 1081 us; with eight wavefronts to a workgroup and three tiles on their way 1102; with 64 rows to a wavefront, which
// halves the reads of LDS but leaves one wavefront to a SIMD, 1394, and at best, long after, 1096 beside 1031.  Eight wavefronts of which four take each half of the keys: 1500
// tokens 42 -> 37, but packed prompts 63 -> 76 and 8K tokens 527 -> 560.)
// Everything is computed transposed, so that a query row is a column and lives in one lane (and the
// lane 32 away, which has the other half of the keys): its maximum, sum and rescaling are
// scalars of the lane, and the weights come out of the first product in the layout that the
// second one reads, with no exchange between lanes.
//   S^T[key][row]  = K[key][:] . Q[row][:]          32x32x16, K from LDS, Q in registers
//   O^T[ch][row]  += V^T[ch][key] . P^T[key][row]   32x32x16, V^T by transposing LDS reads
// Lane roles (lo = lane % 32, hi = lane / 32): of S^T and O^T a lane holds column lo, and of each 32 rows
// 8 (i / 4) + 4 hi + i % 4, i = 0..15.  As the second operand of P.V, eight keys of a lane are
// 16 c + 4 hi + {0..3} and 16 c + 8 + 4 hi + {0..3}: the V^T operand is read in the same order.
#include <algorithm>
#include <type_traits>

#include "ds_device.h"
#include "ds_cache.h"

namespace ds {

constexpr float kPromptScale = 1.4426950408889634f * 0.08838834764831845f;  // log2(e) / sqrt(128)
constexpr int kKeys = 64;                                  // keys of a tile
constexpr int kTileBytes = kKeys * kD * 2;
constexpr int kAheadK = 2, kAheadV = 4;                    // LDS is read so many pairs of products, or products, ahead of them
// The running maximum is raised only when a row's exceeds it by more than this (in the log2 domain), so
// that most tiles rescale nothing; weights carry the factor 2^kRoom besides, which cancels in the quotient.  They
// are at most 2^(7 + 8), within fp16, and normal fp16 numbers down to 2^-21 of the row's largest.
constexpr float kSlack = 8.0f, kRoom = 7.0f;

template <class T>
struct Mma;
template <>
struct Mma<_Float16> {
    typedef half8 vec8;
    typedef _Float16 vec2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x16 dot(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float add2(vec2 p, float l) { return __builtin_amdgcn_fdot2(p, (vec2)(_Float16)1.0f, l, false); }
};
template <>
struct Mma<__bf16> {
    typedef bf16x8 vec8;
    typedef __bf16 vec2 __attribute__((ext_vector_type(2)));
    static __device__ __forceinline__ f32x16 dot(vec8 a, vec8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ float add2(vec2 p, float l) { return __builtin_amdgcn_fdot2_f32_bf16(p, (vec2)(__bf16)1.0f, l, false); }
};

// Where the 16-byte piece c of a tile's row r lies in LDS: rows of 256 bytes would put a column of
// pieces on the same four banks.  Of V, which the transposing read takes two pieces of each of four rows at a time from, at
// v_piece(r, c); of K, read a piece of each of 32 rows at a time, at r * 16 + (c ^ (r & 15)).
__device__ __forceinline__ int v_piece(int r, int c) { return r * 16 + (c ^ ((r & 3) << 2)); }

__device__ __forceinline__ float halves_max(float v)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r.x), __uint_as_float(r.y));
}
__device__ __forceinline__ float halves_sum(float v)
{
    const u32x2 r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r.x) + __uint_as_float(r.y);
}

// Sixteen bytes of every lane, at base + off bytes, from memory into LDS past the registers: to `at` (bytes, the wavefront's)
// + 16 lane.  Written out because the compiler, not knowing which buffer a transposing read reads, would wait for every
// load in flight ahead of each of them; the loads are waited for by wait_tiles.  (m0, the place in LDS, is used for
// nothing else in this kernel.)
__device__ __forceinline__ void load_to_lds(const void *base, uint32_t off, uint32_t at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(at), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void wait_tiles()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// The V operand of a product: keys 16 c .., channels 32 d .. of rows that lie from vb on.  (The steps of k_prompt have it written out: called from
// there, the compiler moves the reads from their places among the products, 500 tokens in groups of 4 14.5 -> 15.0 us.)
template <class T>
__device__ __forceinline__ typename Mma<T>::vec8 v_operand(const u32x4 *vb, int c, int d)
{
    const int lane = threadIdx.x & 63;
    const int r = 16 * c + (lane >> 5) * 4 + (lane & 15) / 4, piece = d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2;
    const char *v0 = reinterpret_cast<const char *>(vb + v_piece(r, piece)) + (lane & 1) * 8;
    const char *v1 = reinterpret_cast<const char *>(vb + v_piece(r + 8, piece)) + (lane & 1) * 8;
    const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v0);
    const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v1);
    const s16x8 v = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
    return __builtin_bit_cast(typename Mma<T>::vec8, v);
}

// A wavefront's 32 rows once more, by itself and 32 keys at a time, for those whose numerator is not finite: a value that is
// not finite comes into rows of the same tile that do not see its key as well, 0 times it being NaN, and sums of
// large bf16 values overflow.  last: the last key that some row sees; my_last: that the lane's row sees; all rows see the keys before
// `clear`.  In tiles that hold others, values that are not finite are taken out of the products and added to the rows that
// see them.  Weights are 2^(s - m + *room), in bf16 such that they add up to 1 at most: no numerator exceeds the largest
// value.  lds: 8 KiB of the wavefront's own.
// Nothing is on its way while it computes: where all rows come here a call takes five times as long (4096 tokens, 16 / 8 heads, a NaN in the
// first value 90 -> 447 us, in all of them 495; the same in pages of 64 105 -> 484 and 534).
template <class T, class At>
__device__ __forceinline__ void rows_again(const T *q, const T *K, const T *V, int last, int my_last, int clear, At at, u32x4 *lds, float *room, float *m, float *l, f32x16 (&O)[4])
{
    typedef typename Mma<T>::vec8 vec8;
    typedef T vec4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63, lo = lane & 31, hi = lane >> 5;
    *room = std::is_same_v<T, __bf16> ? -(float)(last > 0 ? 32 - __builtin_clz(last) : 0) : kRoom;
    *m = kLeast;
    *l = 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = (f32x16)(0.0f);
    vec8 qx[8];
#pragma unroll
    for (int x = 0; x < 8; ++x) qx[x] = *reinterpret_cast<const vec8 *>(q + x * 16 + hi * 8);
#pragma unroll 1
    for (int t0 = 0; t0 <= last; t0 += 32) {
        const T *k = K + at(min(t0 + lo, last)) + hi * 8;
        f32x16 S = (f32x16)(0.0f);
        vec8 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const vec8 *>(V + at(min(t0 + 4 * i + (lane >> 4), last)) + (lane & 15) * 8);
#pragma unroll
        for (int x = 0; x < 8; ++x) S = Mma<T>::dot(*reinterpret_cast<const vec8 *>(k + x * 16), qx[x], S);
        uint32_t beyond = 0u;   // bit i: v[i] was not finite somewhere
        if (t0 + 32 > clear) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (!(fabsf((float)v[i][j]) < __builtin_inff())) {
                        v[i][j] = (T)0.0f;
                        beyond |= 1u << i;
                    }
        }
        __builtin_amdgcn_wave_barrier();   // (the reads of the tile before come first)
#pragma unroll
        for (int i = 0; i < 8; ++i) lds[v_piece(4 * i + (lane >> 4), lane & 15)] = __builtin_bit_cast(u32x4, v[i]);
        __builtin_amdgcn_wave_barrier();
        float top = kNegInf;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (t0 + 8 * (i / 4) + 4 * hi + i % 4 > my_last) S[i] = kNegInf;
            top = fmaxf(top, S[i]);
        }
        const float mn = fmaxf(*m, halves_max(top) * kPromptScale), f = __builtin_amdgcn_exp2f(*m - mn), shift = *room - mn;
        *m = mn;
        *l *= f;
#pragma unroll
        for (int d = 0; d < 4; ++d) O[d] *= f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            vec8 P;
#pragma unroll
            for (int j = 0; j < 8; ++j) P[j] = (T)__builtin_amdgcn_exp2f(__builtin_fmaf(S[8 * c + j], kPromptScale, shift));   // (rounded as in the tiles' steps)
#pragma unroll
            for (int j = 0; j < 8; j += 2) *l = Mma<T>::add2((typename Mma<T>::vec2){P[j], P[j + 1]}, *l);
#pragma unroll
            for (int d = 0; d < 4; ++d) O[d] = Mma<T>::dot(v_operand<T>(lds, c, d), P, O[d]);
        }
#pragma unroll 1
        for (int i = 0; i < 8; ++i) {
            const uint64_t found = __ballot(beyond >> i & 1u);
#pragma unroll 1
            for (int r = 0; r < 4; ++r) {
                if ((found >> (16 * r) & 0xffffu) == 0u) continue;
                const int j = t0 + 4 * i + r;
                const T *row = V + at(min(j, last)) + 4 * hi;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const vec4 x = *reinterpret_cast<const vec4 *>(row + d * 32 + e * 8);
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            if (j <= my_last && !(fabsf((float)x[y]) < __builtin_inff())) O[d][4 * e + y] += (float)x[y];
                    }
            }
        }
    }
}

template <class T, bool PAGED>
__global__ __launch_bounds__(kWG, 2) void k_prompt(PromptArgs a)
{
    typedef typename Mma<T>::vec8 vec8;
    extern __shared__ __attribute__((aligned(16))) u32x4 tiles[];  // K, K, V, V: 16-byte pieces
    constexpr int kPieces = kTileBytes / 16;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 31, hi = lane >> 5;
    // Work is handed out from the last row tiles, which see most, to the first.  Where all of it is on the device at once, one
    // workgroup to some compute units and two to the others (workgroups i and cus + i, as they are dealt out), the
    // heaviest are to have theirs alone, and of the others the heaviest the lightest beside them.  (us, in order and so: one
    // prompt of 1500 tokens, 32 heads 41.4 and 39.1, of 1900 47.3 and 43.5, of 1500 in groups of 4 35.9 and 32.7.)
    int rank = blockIdx.x;
    const int W = gridDim.x, twice = W - a.cus;
    if (twice > 0 && twice <= a.cus) rank = rank < twice ? a.cus - twice + rank : rank < a.cus ? rank - twice : W - 1 - (rank - a.cus);
    const int kvh = rank - a.by_Hkv.of(rank) * a.Hkv;
    const int slot = a.n_tiles - 1 - a.by_Hkv.of(rank);
    // ---- the sequence and its rows
    const int s = last_at_or_before(a.n_seqs, slot, [&](int i) { return tile_base(a.q_start[i], a.G, i); });
    const int qs = a.q_start[s], qe = a.q_start[s + 1];
    const int word0 = PAGED ? (a.rows ? a.rows[s] : s) : a.kv_start[s], word1 = PAGED ? 0 : a.kv_len[s];   // (with these, not after them)
    if (qs < 0 || qe < qs || qe > a.total_q) return;
    const int n_rows = (qe - qs) * a.G;
    const int r0 = (slot - tile_base(qs, a.G, s)) * kPromptRows;
    if (r0 < 0 || r0 >= n_rows) return;
    bool bad = false;
    int nk;
    int64_t kv0 = 0;
    const int32_t *pages = nullptr;
    if constexpr (PAGED) {
        const int row = word0;
        bad = row < 0 || row >= a.n_table;
        nk = bad ? 0 : a.kv_len[row];
        pages = a.table + (size_t)(bad ? 0 : row) * a.max_pages;
        bad |= nk < 0 || (int64_t)nk > (int64_t)a.max_pages << a.page_log2;
    } else {
        nk = word1;
        kv0 = word0;
        bad = nk < 0 || nk > kMostTokens || kv0 < 0 || (nk > 0 && (kv0 + nk - 1) * a.kv_stride + (int64_t)(a.Hkv - 1) * a.kv_head_stride + kD > a.kv_elems);
        kv0 = kv0 * a.kv_stride + (int64_t)kvh * a.kv_head_stride;
    }
    if (bad) nk = 0;
    const int last_row = min(n_rows, r0 + kPromptRows) - 1;
    const int seen = max(0, min(nk, a.by_G.of(last_row) + nk - (qe - qs) + 1));    // keys that some row of the workgroup sees
    // ---- its part of them, where the keys are split; from here on keys count from its first
    const int all_kt = (seen + kKeys - 1) / kKeys, part_kt = a.n_split == 1 ? all_kt : (all_kt + a.n_split - 1) / a.n_split;
    const int kt0 = min((int)blockIdx.y * part_kt, all_kt), n_kt = min(part_kt, all_kt - kt0);
    const int first_key = kt0 * kKeys;
    const int before = nk - (qe - qs) - first_key;   // keys ahead of the sequence's first row's own
    nk = min(nk - first_key, n_kt * kKeys);
    if constexpr (!PAGED) kv0 += first_key * a.kv_stride;
    const int my_row = r0 + wave * 32 + lo;
    const bool on = my_row < n_rows;
    const int my_last = on ? min(a.by_G.of(my_row) + before, nk - 1) : -1; // last key that the lane's row sees
    // tiles that some row of the wavefront sees, and those that all of its rows see whole
    const int n_mine = min(n_kt, max(0, a.by_G.of(min(r0 + wave * 32 + 31, n_rows - 1)) + before + kKeys) / kKeys);
    const int n_clear = r0 + wave * 32 >= n_rows ? 0 : max(0, min(a.by_G.of(r0 + wave * 32) + before + 1, nk)) / kKeys;

    vec8 q[8];
    {
        const int row = min(my_row, n_rows - 1), own = a.by_G.of(row);
        const T *src = static_cast<const T *>(a.q) + (size_t)(qs + own) * a.q_stride + (size_t)(kvh * a.G + row - own * a.G) * kD + hi * 8;
#pragma unroll
        for (int x = 0; x < 8; ++x) q[x] = *reinterpret_cast<const vec8 *>(src + x * 16);
    }
    f32x16 O[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = (f32x16)(0.0f);
    float m = kLeast, l = 0.0f;

    // ---- tiles: of each 16 rows a wavefront brings four, a lane one piece.  The pieces of a row change places on the
    // way (see v_piece), by the lane's place in memory, since in LDS a load's lanes lie side by side.
    // Rows past the last key re-read it (their weight is 0, and 0 times whatever lies behind it need not be).
    const int lane_row = 4 * wave + (lane >> 4);
    const uint32_t row_bytes = PAGED ? kD * 2 : (uint32_t)a.kv_stride * 2;   // (64 rows are within 2^31 bytes)
    const uint32_t k_off = ((lane & 15) ^ lane_row) * 16, v_off = ((lane & 15) ^ ((lane >> 4) << 2)) * 16, row_off = lane_row * row_bytes;
    const T *Kp = static_cast<const T *>(a.K) + kv0, *Vp = static_cast<const T *>(a.V) + kv0;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)tiles + wave * 1024;
    // Paged: lane i % 4 of `of` holds the page of a tile's rows 16 i .. (16 rows that start at a multiple of 16 are in one page)
    auto page_ids = [&](int kt) {
        int p = 0;
        if constexpr (PAGED) {
            if (nk > 0) p = pages[(first_key + min(kt * kKeys + (lane & 3) * 16, nk - 1)) >> a.page_log2];
            if ((uint32_t)p >= (uint32_t)a.n_pages) {
                if (kt < n_kt) bad = true;
                p = 0;
            }
        }
        return p;
    };
    // rows 16 i .. of tile kt: the wavefront's four of them
    auto load_rows = [&](const T *base, uint32_t off, int kt, int i, int buffer, int of, auto whole) {
        const int t0 = kt * kKeys + i * 16;
        const uint32_t at = lds0 + buffer * kTileBytes + i * 4096;
        if constexpr (PAGED) {
            const int64_t p = __builtin_amdgcn_readlane(of, i);
            const int g0 = whole ? t0 : min(t0, nk - 1) & ~15;
            const T *src = base + (((p * a.Hkv + kvh) << a.page_log2) + ((first_key + g0) & ((1 << a.page_log2) - 1))) * kD;
            load_to_lds(src, off + (whole ? row_off : (uint32_t)(min(t0 + lane_row, nk - 1) - g0) * row_bytes), at);
        } else if constexpr (whole) {
            load_to_lds(base + t0 * a.kv_stride, off + row_off, at);
        } else {
            load_to_lds(base + kt * kKeys * a.kv_stride, off + (uint32_t)(min(t0 + lane_row, nk - 1) - kt * kKeys) * row_bytes, at);
        }
    };
    auto load_tile = [&](const T *base, uint32_t off, int kt, int buffer, int of) {
        if ((kt + 1) * kKeys <= nk) {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_rows(base, off, kt, i, buffer, of, std::true_type{});
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) load_rows(base, off, kt, i, buffer, of, std::false_type{});
        }
    };

    // Products and LDS reads keep the places that they have here; what the vector units do may move between them.  (Left
    // to itself the compiler reads right before it multiplies.  1500 tokens of 32 heads 44.0 -> 41.5 us, 500 in groups
    // of 4 16.4 -> 15.3.)
    auto pin = []() { __builtin_amdgcn_sched_barrier(0x2 | 0x4 | 0x400); };
    // S = K Q of a tile; between(x) is done ahead of the x-th pieces' products
    auto scores = [&](int buffer, f32x16 (&S)[2], auto between) {
        // (the places of pieces 2 x + hi of row lo are formed anew in every step: eight registers that the loop cannot spare)
        int at = (lo * 16 + (hi ^ (lo & 15))) * 16;
        asm volatile("" : "+v"(at));
        const char *kb = reinterpret_cast<const char *>(tiles + buffer * kPieces);
        vec8 k[8][2];
        auto read = [&](int x) {
#pragma unroll
            for (int b = 0; b < 2; ++b) k[x][b] = *reinterpret_cast<const vec8 *>(kb + b * 8192 + (at ^ x * 32));
        };
#pragma unroll
        for (int b = 0; b < 2; ++b) S[b] = (f32x16)(0.0f);
#pragma unroll
        for (int x = 0; x < kAheadK; ++x) read(x);
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            if (x + kAheadK < 8) read(x + kAheadK);
            between(x);
            pin();
#pragma unroll
            for (int b = 0; b < 2; ++b) S[b] = Mma<T>::dot(k[x][b], q[x], S[b]);
            pin();
        }
    };
    auto hide = [&](int kt, f32x16 (&S)[2]) {
        const int left = my_last - kt * kKeys - 4 * hi;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (b * 32 + 8 * (i / 4) + i % 4 > left) S[b][i] = kNegInf;
    };
    auto weights = [&](const f32x16 (&S)[2], vec8 (&P)[4], int c0 = 0, int c1 = 4) {
        const float shift = kRoom - m;
#pragma unroll
        for (int c = c0; c < c1; ++c)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                P[c][j] = (T)__builtin_amdgcn_exp2f(__builtin_fmaf(S[c / 2][8 * (c & 1) + j], kPromptScale, shift));  // (rounded once, to the type of V)
    };
    auto add_up = [&](const vec8 (&P)[4]) {   // (the rounded weights)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int j = 0; j < 8; j += 2) l = Mma<T>::add2((typename Mma<T>::vec2){P[c][j], P[c][j + 1]}, l);
    };
    // the V operand of products i = 4 c + d: keys 16 c .., channels 32 d ..
    auto read_v = [&](int buffer, int i) {
        const u32x4 *vb = tiles + (2 + buffer) * kPieces;
        const int c = i / 4, d = i % 4;
        // four keys by sixteen channels for each 16 lanes: lane 4 j + x brings row j, channels 4 x ..
        const int r = 16 * c + 4 * hi + (lane & 15) / 4, piece = d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2;
        const char *v0 = reinterpret_cast<const char *>(vb + v_piece(r, piece)) + (lane & 1) * 8;
        const char *v1 = reinterpret_cast<const char *>(vb + v_piece(r + 8, piece)) + (lane & 1) * 8;
        const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v0);
        const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v1);
        const s16x8 v = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
        return __builtin_bit_cast(vec8, v);
    };
    auto values = [&](int buffer, vec8 (&v)[kAheadV], const vec8 (&P)[4], int i0, int i1) {
#pragma unroll
        for (int i = i0; i < i1; ++i) {
            const vec8 now = v[i % kAheadV];
            if (i + kAheadV < 16) v[i % kAheadV] = read_v(buffer, i + kAheadV);
            pin();
            O[i % 4] = Mma<T>::dot(now, P[i / 4], O[i % 4]);
            pin();
        }
    };
    auto raise = [&](const f32x16 (&S)[2]) {
        float top = kNegInf;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, S[b][i]);
        top = halves_max(top) * kPromptScale;
        if (__any(top > m + kSlack)) {
            const float mn = fmaxf(m, top);
            const float f = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= f;
#pragma unroll
            for (int d = 0; d < 4; ++d) O[d] *= f;
        }
    };
    // (the loads of q are waited for here: inside the loop the wait would take in the next tile's loads as well)
#pragma unroll
    for (int x = 0; x < 8; ++x) asm volatile("" : "+v"(q[x]));

    int ids0 = page_ids(0), ids1 = page_ids(1);
    if (n_kt > 0) {
        load_tile(Kp, k_off, 0, 0, ids0);
        load_tile(Vp, v_off, 0, 2, ids0);
        if (n_kt > 1) load_tile(Kp, k_off, 1, 1, ids1);
    }
    ids0 = page_ids(2);
    wait_tiles();
    f32x16 S0[2], S1[2];
    if (n_mine > 0) scores(0, S0, [](int) {});
    // (Every wavefront reads the first K tile here, and what comes next brings another to its place: in the loop the barrier
    //  at the end of a step lies between the two.  Without further tiles nothing is brought.)
    if (n_kt > 1) __syncthreads();
    if (n_mine > 0) {
        if (n_clear < 1) hide(0, S0);
        raise(S0);
    }
    // A step: most of tile kt's weights while the matrix units form the scores of the next, the rest while they form its
    // values, with the sum of the weights and the next one's maximum (so that both halves have vector work, and registers do); the K tile after the next and the next V tile are on their way meanwhile, to
    // places whose tiles were done with before the last barrier.  odd: kt % 2
    auto bring = [&](int kt, int odd) {
        if (kt + 1 < n_kt) load_tile(Vp, v_off, kt + 1, 3 - odd, ids1);
        if (kt + 2 < n_kt) load_tile(Kp, k_off, kt + 2, odd, ids0);
        ids1 = ids0;
        ids0 = page_ids(kt + 3);
    };
    auto step = [&](int kt, int odd, f32x16 (&S)[2], f32x16 (&N)[2], auto hidden) {
        vec8 P[4], v[kAheadV];
        // (One load at a time between the products.  The eight of them in a row ahead of the step kept the wavefront from
        //  its products for as long as they take to be accepted: 8K tokens of 32 heads 581 -> 531 us, two of 8K in groups
        //  of 4 1073 -> 977, 512 on 20K in groups of 8 697 -> 638.  Behind the last K tile it comes again, to a place
        //  that nobody reads.)
        scores(1 - odd, N, [&](int x) {
            constexpr std::bool_constant<!hidden> whole{};
            if (x < 4) load_rows(Vp, v_off, kt + 1, x, 3 - odd, ids1, whole);
            else load_rows(Kp, k_off, hidden ? min(kt + 2, n_kt - 1) : kt + 2, x - 4, odd, ids0, whole);
            if (x == 7)
#pragma unroll
                for (int i = 0; i < kAheadV; ++i) v[i] = read_v(odd, i);
        });
        ids1 = ids0;
        ids0 = page_ids(kt + 3);
        weights(S, P, 0, 3);
        if constexpr (hidden) hide(kt + 1, N);
        values(odd, v, P, 0, 12);
        weights(S, P, 3, 4);
        values(odd, v, P, 12, 16);
        add_up(P);
        raise(N);
        wait_tiles();
    };
    int kt = 0;
    for (const int n_whole = nk / kKeys; kt + 2 < n_clear && kt + 3 < n_whole; kt += 2) {
        step(kt, 0, S0, S1, std::false_type{});
        step(kt + 1, 1, S1, S0, std::false_type{});
    }
    for (; kt + 1 < n_mine; ++kt) {
        step(kt, kt & 1, S0, S1, std::true_type{});
        S0[0] = S1[0];
        S0[1] = S1[1];
    }
    for (; kt < n_kt; ++kt) {   // (the wavefront's last tile, and those that only others see)
        bring(kt, kt & 1);
        if (kt < n_mine) {
            vec8 P[4], v[kAheadV];
#pragma unroll
            for (int i = 0; i < kAheadV; ++i) v[i] = read_v(kt & 1, i);
            weights(S0, P);
            values(kt & 1, v, P, 0, 16);
            add_up(P);
        }
        wait_tiles();
    }
    if constexpr (PAGED) {  // (a page that is not there: seen by the threads that would have read it)
        uint32_t *flag = reinterpret_cast<uint32_t *>(tiles);
        if (tid == 0) *flag = 0u;
        __syncthreads();
        if (bad) *flag = 1u;
        __syncthreads();
        bad = *flag != 0u;
    }
    // The lane's half of its row, from weights that carry 2^room: the result, or a part of it.
    auto write = [&](const auto &g, const Quotient &by_G, float room) {
        l = halves_sum(l);
        const int own = by_G.of(my_row), head = kvh * g.G + my_row - own * g.G;
        const int64_t token = qs + own;
        if (g.n_split > 1) {
            const int64_t row = ((int64_t)blockIdx.y * g.total_q + token) * g.Hq + head;
            if (my_last < 0) m = kNegInf;                // (a part without a key that the row sees)
            // (2^(s - m + room) is 2^(s - (m + kRoom - room) + kRoom))
            if (hi == 0) g.part_ml[row] = bad ? make_float2(0.0f, __builtin_nanf("")) : make_float2(m + (kRoom - room), l);
            if (l != 0.0f) {
                float *acc = g.part_acc + row * kD + 4 * hi;
#pragma unroll
                for (int d = 0; d < 4; ++d)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4 *>(acc + d * 32 + i * 8) = (f32x4){O[d][4 * i], O[d][4 * i + 1], O[d][4 * i + 2], O[d][4 * i + 3]};
            }
        } else {
            // (a row whose pages or places are not there is NaN, one that sees no key is zero)
            const float inv = bad ? __builtin_nanf("") : my_last < 0 ? 0.0f : 1.0f / l;
            T *dst = static_cast<T *>(g.out) + token * g.out_stride + (int64_t)head * kD + 8 * hi;
            // (four channels of a lane and the next four of the lane 32 away, exchanged for whole pieces of 16 bytes: 97 tokens of 32
            // heads 8.0 -> 7.4 us, 12 of 300 in groups of 4 32.4 -> 28.4, 8 of 2407 in pairs 443 -> 431.  Whole rows by way of LDS: no better.)
            typedef T vec4 __attribute__((ext_vector_type(4)));
            auto four = [&](int d, int i) {
                vec4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = (T)(O[d][4 * i + j] * inv);
                return __builtin_bit_cast(u32x2, x);
            };
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int i = 0; i < 4; i += 2) {
                    const u32x2 x = four(d, i), y = four(d, i + 1);
                    const u32x2 u = __builtin_amdgcn_permlane32_swap(x.x, y.x, false, false), v = __builtin_amdgcn_permlane32_swap(x.y, y.y, false, false);
                    *reinterpret_cast<u32x4 *>(dst + d * 32 + i * 8) = (u32x4){u.x, v.x, u.y, v.y};
                }
        }
    };
    if (on) write(a, a.by_G, kRoom);
    // Rows whose numerator is not finite are formed once more (looked for while they are being written).
    f32x16 all = (O[0] + O[1]) + (O[2] + O[3]);
#pragma unroll
    for (int n = 8; n > 0; n /= 2)
#pragma unroll
        for (int i = 0; i < n; ++i) all[i] += all[i + n];
    const uint64_t beyond = __ballot(on && !bad && !(fabsf(all[0]) < __builtin_inff()));
    if (const uint32_t anew = (uint32_t)beyond | (uint32_t)(beyond >> 32)) {
        // (The arguments are read again: those that only this part needs would be kept over the loop, which has no scalar registers
        //  left for them.)
        auto *end = (const __attribute__((address_space(4))) PromptArgs *)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(end));
        const Quotient by_G = {end->by_G.m, end->by_G.shift};
        const int own = by_G.of(min(my_row, n_rows - 1)), head = kvh * end->G + min(my_row, n_rows - 1) - own * end->G;
        const int last = min(by_G.of(min(r0 + wave * 32 + 31, n_rows - 1)) + before, nk - 1);   // (the rows' last keys ascend)
        auto at = [&](int j) -> int64_t {
            if constexpr (PAGED) {
                const int t = first_key + j;
                return ((((int64_t)pages[t >> end->page_log2] * end->Hkv + kvh) << end->page_log2) + (t & ((1 << end->page_log2) - 1))) * kD;
            } else {
                return kv0 + j * end->kv_stride;
            }
        };
        float room;
        // (the tiles are done with; the upper half of a wavefront's quarter of them does not hold the flag above)
        rows_again<T>(static_cast<const T *>(end->q) + (int64_t)(qs + own) * end->q_stride + (int64_t)head * kD, static_cast<const T *>(end->K),
                      static_cast<const T *>(end->V), last, my_last, n_clear * kKeys, at, tiles + wave * kPieces + kPieces / 2, &room, &m, &l, O);
        if (anew >> lo & 1u) write(*end, by_G, room);
    }
}

// Joins the parts of split keys, a wavefront for a row of a head:
//   y = sum_z acc_z 2^(m_z - M) / sum_z l_z 2^(m_z - M),  M = max_z m_z + 6,  z ascending
// (parts of large bf16 values add up to more than binary32 holds: 64 of them at most, each with a weight of 1/64 at most, do not).
template <class T>
__global__ __launch_bounds__(kWG) void k_prompt_join(PromptArgs a)
{
    typedef T vec2 __attribute__((ext_vector_type(2)));
    const int lane = threadIdx.x & 63;
    const int64_t rows = (int64_t)a.total_q * a.Hq;
    const int64_t row = (int64_t)blockIdx.x * (kWG / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= rows) return;
    const int token = a.by_Hq.of((int)row), head = (int)row - token * a.Hq;
    const int s = last_at_or_before(a.n_seqs, token, [&](int i) { return a.q_start[i]; });
    const int qs = a.q_start[s], qe = a.q_start[s + 1];
    if (qs < 0 || qe < qs || qe > a.total_q || token < qs || token >= qe) return;   // (no row of a sequence: left as it is)
    const float2 ml = lane < a.n_split ? a.part_ml[lane * rows + row] : make_float2(kNegInf, 0.0f);
    float M = ml.x;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor(M, o));
    static_assert(kPromptParts == 1 << 6);
    const float f = ml.x == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(ml.x - M - 6.0f);
    float L = f * ml.y;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) L += __shfl_xor(L, o);
    const uint64_t there = __ballot(ml.y != 0.0f);   // parts that have written a numerator
    float2 A = make_float2(0.0f, 0.0f);
    constexpr int kFlight = 8;
    for (int z0 = 0; z0 < a.n_split; z0 += kFlight) {
        float2 v[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const bool on = z0 + i < a.n_split && (there >> (z0 + i) & 1u);
            v[i] = on ? *reinterpret_cast<const float2 *>(a.part_acc + ((z0 + i) * rows + row) * kD + 2 * lane) : make_float2(0.0f, 0.0f);
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const float w = __shfl(f, (z0 + i) & 63);
            A.x += w * v[i].x;
            A.y += w * v[i].y;
        }
    }
    const float inv = M == kNegInf ? 0.0f : 1.0f / L;   // (no part with a key that the row sees: zero)
    *reinterpret_cast<vec2 *>(static_cast<T *>(a.out) + token * a.out_stride + (int64_t)head * kD + 2 * lane) = (vec2){(T)(A.x * inv), (T)(A.y * inv)};
}

// ---------------------------------------------------------------- launcher
void make_prompt_plan(const ds_prompt_t &m, PromptPlan *p, size_t workspace_bytes)
{
    p->G = m.Hq / m.Hkv;
    p->n_tiles = (int)((int64_t)m.total_q * p->G / kPromptRows) + m.n_seqs;
    p->n_split = 1;
    // Few rows over many keys: the keys are split, until two workgroups to a compute unit have work at most.  A part
    // saves its share of the steps, 1.2 us each (one workgroup's step is latency), and costs a numerator of every row,
    // written and read, and the join about 4 us.  (us, not split and split: 16 tokens on 30000, groups of 4, 818 -> 39; eight of
    // 16 on 2000 63 -> 31; two of 60 on 10000, single heads 237 -> 80; on the other side of the line 500 tokens 18 -> 24 in two
    // parts, 1000 in groups of 7 30 -> 42.)
    const int64_t wgs = (int64_t)p->n_tiles * m.Hkv, most = std::min<int64_t>(2 * device_caps().cus / wgs, kPromptParts);
    const double steps = 1.2 * m.max_kv / kKeys, row_part = (double)m.total_q * m.Hq * (2 * kD * 4) / 3e6;
    double best = steps;
    p->off_acc = 0;
    p->total = 256;
    for (int n = 2; n <= most; ++n) {
        const double us = steps / n + 4.0 + n * row_part;
        const size_t rows = (size_t)m.total_q * m.Hq * n, off_acc = (rows * 8 + 255) / 256 * 256, total = off_acc + rows * kD * 4;
        if (us < best && total <= workspace_bytes) {    // (what the parts do not fit in, fewer do, and none always)
            best = us;
            p->n_split = n;
            p->off_acc = off_acc;
            p->total = total;
        }
    }
}

typedef void (*PromptFn)(PromptArgs);
static PromptFn prompt_fn(bool paged, int dtype)
{
    if (dtype == DS_BF16) return paged ? k_prompt<__bf16, true> : k_prompt<__bf16, false>;
    return paged ? k_prompt<_Float16, true> : k_prompt<_Float16, false>;
}

hipError_t launch_prompt(PromptArgs a, bool paged, int dtype, hipStream_t st)
{
    a.cus = device_caps().cus;
    a.by_G.set(a.G);
    a.by_Hkv.set(a.Hkv);
    a.by_Hq.set(a.Hq);
    const PromptFn fn = prompt_fn(paged, dtype);
    DS_LAUNCH(KID_PROMPT, fn, dim3((unsigned)(a.n_tiles * a.Hkv), a.n_split), dim3(kWG), 4 * kTileBytes, st, a);
    if (a.n_split > 1) {
        const unsigned wgs = (unsigned)(((int64_t)a.total_q * a.Hq + kWG / 64 - 1) / (kWG / 64));
        const PromptFn join = dtype == DS_BF16 ? k_prompt_join<__bf16> : k_prompt_join<_Float16>;
        DS_LAUNCH(KID_PROMPT, join, dim3(wgs), dim3(kWG), 0, st, a);
    }
    return hipGetLastError();
}

}  // namespace ds
