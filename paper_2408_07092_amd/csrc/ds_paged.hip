// Dense decode attention of one new token of every sequence over a paged cache, and the writing of
// new tokens' rows into its pages.
//
// The attention reads every K and V row once and computes next to nothing on it: memory bound.  Lengths are
// known on the device only and may differ as they like, so the work is cut there: all the
// sequences' tokens, a KV head after the other, are one line of pieces of 64 tokens, of which every workgroup
// takes an equal, contiguous share, but for units of up to kWhole pieces, which are not cut (an end that falls into one
// moves to its nearer end: 101 sequences of up to 89 tokens, 2 groups of 16 13.8 -> 7.0 us).  A share covers the end of one unit (sequence and KV head), whole units, and
// the beginning of another, or a part of a single one; a unit's parts meet in the workspace, where
// the last workgroup to arrive joins them in their order along the cache.  Which part holds
// which tokens follows from the lengths and the launch alone, so results do not depend on who is last.
//
// One workgroup to a compute unit, each wavefront with two tiles of 16 tokens on their way (64 KiB a compute unit), streams best: 16
// sequences of 32K tokens (2.1 GB) take 319 us, 6.7 TB/s, one of 250K (512 MB) 86.  (As first measured: 322, and with one tile on
// its way and one, two or four workgroups 405, 318 and 347, with two tiles and two workgroups 332; 89, and 118 to 182 with one
// tile and two to four workgroups, whose parts cost more to join.  Three and four tiles: no difference.)  A unit's beginning and end (its query, the
// wavefronts' states, the part) cost a workgroup about what three pieces do, and count as kLead pieces: 48 sequences of 3 to 20000
// tokens 157 us without, 109, 102 and 100 with one, two and three (since then, with a head's states combined by a
// wavefront, 91 and the writing of the new rows 5).
//
// A wavefront takes 16 tokens at a time (within one page, as pages hold 16 or more), for up to 16 heads
// of the group at once:
//   S[token][head] = K[token][:] . q[head][:]       16x16x32, K and q from memory
//   O[head][ch]   += P[token][head] V[token][ch]    16x16x16, the weight as the sum of two numbers of V's type
// Lane roles (lo = lane % 16, hi = lane / 16): K token lo, 16-byte pieces at channels 8 (4 x + hi); q head lo, the
// same; S head lo, tokens 4 hi + r; V token 4 hi + r, channels 8 lo ..; O[e]: heads 4 hi + rr, channel 8 lo + e.
// One head alone leaves 15 of 16 columns of the matrix units idle, which costs nothing here: 16 tokens take
// about 500 clocks of one SIMD, and their 8 KiB about 700 of the compute unit's share of memory.
#include <algorithm>
#include <type_traits>

#include "ds_device.h"
#include "ds_cache.h"
#include "ds_attend_core.h"

namespace ds {

template <class T>
struct Mma16;
template <>
struct Mma16<_Float16> {
    typedef half8 vec8;
    typedef half4v vec4;
    static __device__ __forceinline__ f32x4 dot32(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 dot16(vec4 a, vec4 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x16f16(a, b, c, 0, 0, 0); }
};
template <>
struct Mma16<__bf16> {
    typedef bf16x8 vec8;
    typedef __bf16 vec4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x4 dot32(vec8 a, vec8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x4 dot16(vec4 a, vec4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
    }
};

// Tokens of table row `row`, or -1 if the row or its length cannot be.
__device__ __forceinline__ int row_tokens(const PagedArgs &a, int b, int *row)
{
    *row = a.rows ? a.rows[b] : b;
    if (*row < 0 || *row >= a.n_table) return -1;
    const int n = a.lens[*row];
    return n < 0 || (int64_t)n > (int64_t)a.max_pages << a.page_log2 ? -1 : n;
}
// ... and what they count for: the pieces, and kLead more for a unit's beginning and end.
__device__ __forceinline__ int pieces_of(int tokens) { return tokens > 0 ? (tokens - 1) / kPiece + 1 + kLead : 0; }

// The share of workgroup w of W: T / W pieces, the first T % W of them one more.
struct Shares {
    uint32_t each, more;
    __device__ __forceinline__ Shares(uint32_t T, uint32_t W) : each(T / W), more(T % W) {}
    __device__ __forceinline__ uint32_t start(uint32_t w) const { return w * each + min(w, more); }
    __device__ __forceinline__ uint32_t of(uint32_t x) const   // the workgroup that has piece x
    {
        return x < more * (each + 1) ? x / (each + 1) : (x - more) / each;
    }
};

// Joins the parts of a unit, which lie with workgroups w0 .. w1: for every head
//   y = sum_p acc_p 2^(m_p - M) / sum_p l_p 2^(m_p - M),  M = max_p m_p,
// a wavefront for a head, or two or four of them where there are fewer heads, 16 parts in flight, folded in
// an order that depends on the launch alone.  All threads call it.
template <int GH>
__device__ __forceinline__ void join_parts(const PagedArgs &a, int w0, int w1, int first_head, int n_heads, float *out, float (*red)[kD + 4])
{
    constexpr int kBatch = 16;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int share = n_heads >= 4 ? 1 : n_heads >= 2 ? 2 : 4, at_once = 4 / share;
    const int n = w1 - w0 + 1, sub = wave % share;
    for (int g0 = 0; g0 < n_heads; g0 += at_once) {
        const int g = g0 + wave / share;
        float M = kNegInf, L = 0.0f;
        float2 A = make_float2(0.0f, 0.0f);
        if (g < n_heads) {
            for (int i0 = sub; i0 < n; i0 += share * kBatch) {
                float2 ml[kBatch], v[kBatch];
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    const int w = w0 + min(i0 + i * share, n - 1);
                    const float *pc = a.part + (((size_t)w * 2 + (w == w0 ? 1 : 0)) * GH + first_head + g) * kPartStride;
                    ml[i] = ld_dev(reinterpret_cast<const float2 *>(pc));
                    v[i] = ld_dev(reinterpret_cast<const float2 *>(pc + 4 + 2 * lane));
                }
                float top = M;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    if (i0 + i * share >= n) ml[i].x = kNegInf;
                    top = fmaxf(top, ml[i].x);
                }
                const float f0 = M == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(M - top);
                M = top;
                L *= f0;
                A.x *= f0;
                A.y *= f0;
#pragma unroll
                for (int i = 0; i < kBatch; ++i)
                    if (ml[i].x != kNegInf) {
                        const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
                        L += f * ml[i].y;
                        A.x += f * v[i].x;
                        A.y += f * v[i].y;
                    }
            }
        }
        if (share > 1) {
            red[wave][2 * lane] = A.x;
            red[wave][2 * lane + 1] = A.y;
            if (lane == 0) {
                red[wave][kD] = M;
                red[wave][kD + 1] = L;
            }
            __syncthreads();
            if (sub == 0 && g < n_heads) {
                float top = kNegInf;
                for (int s = 0; s < share; ++s) top = fmaxf(top, red[wave + s][kD]);
                L = 0.0f;
                A = make_float2(0.0f, 0.0f);
                for (int s = 0; s < share; ++s) {
                    const float f = red[wave + s][kD] == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(red[wave + s][kD] - top);
                    L += f * red[wave + s][kD + 1];
                    A.x += f * red[wave + s][2 * lane];
                    A.y += f * red[wave + s][2 * lane + 1];
                }
            }
            __syncthreads();
        }
        if (sub == 0 && g < n_heads) *reinterpret_cast<float2 *>(out + (size_t)g * kD + 2 * lane) = make_float2(A.x / L, A.y / L);
    }
}

// Combines the wavefronts' states (maximum, sum, two of padding, numerator) to a unit's part, or to its rows of the
// output: a wavefront for a head, two channels a lane.  All threads call it.
template <int GH>
__device__ __forceinline__ void combine_states(const float (*wpart)[GH][kPartStride], int n_heads, float *part, float *out)
{
    const int lane = threadIdx.x & 63;
    __syncthreads();
#pragma unroll
    for (int g0 = 0; g0 < GH; g0 += 4) {
        const int g = g0 + (int)(threadIdx.x >> 6);
        if (g >= n_heads) break;
        float2 ml[4], v[4];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            ml[w] = *reinterpret_cast<const float2 *>(&wpart[w][g][0]);
            v[w] = *reinterpret_cast<const float2 *>(&wpart[w][g][4 + 2 * lane]);
        }
        const float M = fmaxf(fmaxf(ml[0].x, ml[1].x), fmaxf(ml[2].x, ml[3].x));
        float L = 0.0f;
        float2 A = make_float2(0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[w].x - M);
            L += f * ml[w].y;
            A.x += f * v[w].x;
            A.y += f * v[w].y;
        }
        if (out) {
            *reinterpret_cast<float2 *>(out + (size_t)g * kD + 2 * lane) = make_float2(A.x / L, A.y / L);
        } else {
            uint2 *pg = reinterpret_cast<uint2 *>(part + (size_t)g * kPartStride);
            st_dev(pg + 2 + lane, make_uint2(__float_as_uint(A.x), __float_as_uint(A.y)));
            if (lane == 0) st_dev(pg, make_uint2(__float_as_uint(M), __float_as_uint(L)));
        }
    }
}

// All pieces of the call's sequences, and those ahead of sequence `upto` (threads of a workgroup each take some).
__device__ __forceinline__ void count_pieces(const PagedArgs &a, int upto, uint32_t *s_w, uint32_t *total, uint32_t *before)
{
    uint32_t all = 0, ahead = 0;
    for (int b = threadIdx.x; b < a.n; b += kWG) {
        int row;
        const uint32_t k = (uint32_t)pieces_of(row_tokens(a, b, &row));
        all += k;
        if (b < upto) ahead += k;
    }
    block_exclusive_scan(all, s_w, total);
    block_exclusive_scan(ahead, s_w, before);
}
// (one sequence of 900 tokens, 32 heads, in shares of no less than two pieces 10.8 us, of four 11.7, of eight 14.0)
__device__ __forceinline__ uint32_t shares_of(uint32_t T_all, uint32_t wgs) { return max(1u, min(wgs, T_all / kShareAtLeast)); }

template <class T, int GH>
__global__ __launch_bounds__(kWG, 2) void k_paged(PagedArgs a)
{
    constexpr int kDepth = 2;   // tiles of a wavefront on their way
    typedef typename Mma16<T>::vec8 vec8;
    typedef typename Mma16<T>::vec4 vec4;
    __shared__ __attribute__((aligned(16))) float wpart[4][GH][kPartStride];
    __shared__ __attribute__((aligned(16))) float sc_sh[4][16];
    __shared__ uint32_t s_w[4], s_flag, s_at[2][4];
    float (*red)[kD + 4] = reinterpret_cast<float (*)[kD + 4]>(&wpart[0][0][0]);   // (4 of them; used after wpart)

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 15, hi = lane >> 4;
    const int units = a.Hkv * a.passes;   // of a sequence
    // ---- all pieces
    const int per = (a.n + kWG - 1) / kWG;
    uint32_t mine = 0;
    int n = 1, row = 0;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        n = 1;
        if (b < a.n) {
            n = row_tokens(a, b, &row);
            mine += (uint32_t)pieces_of(n);
        }
        // sequences without a token, or without a place: zero, or NaN
        for (uint64_t left = __ballot(n <= 0 && b % (int)gridDim.x == (int)blockIdx.x); left; left &= left - 1) {
            const int from = __builtin_ctzll(left), at = __shfl(b, from);
            const float x = __shfl(n, from) < 0 ? __builtin_nanf("") : 0.0f;
            const int row_out = a.Hkv * a.G * kD;
            for (int j = lane; j < row_out; j += 64) a.out[(size_t)at * row_out + j] = x;
        }
    }
    uint32_t total;
    uint32_t ahead = block_exclusive_scan(mine, s_w, &total);
    const uint32_t T_all = total * (uint32_t)units;
    const uint32_t W = shares_of(T_all, gridDim.x);
    if (blockIdx.x >= W || T_all == 0) return;
    const Shares shares(T_all, W);
    // ---- the sequences that the share's ends lie in
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t want = (uint32_t)a.by_units.of((int)shares.start(blockIdx.x + e));   // the piece of a sequence, counted over sequences
        if (ahead <= want && want < ahead + mine) {
            int b = tid * per;
            uint32_t at = ahead;
            if (per > 1)
                for (uint32_t k; (k = (uint32_t)pieces_of(n = row_tokens(a, b, &row))) <= want - at; ++b) at += k;
            s_at[e][0] = (uint32_t)b;
            s_at[e][1] = at;
            s_at[e][2] = (uint32_t)n;
            s_at[e][3] = (uint32_t)row;
        }
    }
    __syncthreads();
    // (an end within a short unit moves to the nearer end of it)
    auto end_of = [&](int e) {
        const uint32_t x = shares.start(blockIdx.x + e);
        if (x >= T_all) return T_all;
        const uint32_t first = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_at[e][1]) * (uint32_t)units;
        const uint32_t np = (uint32_t)pieces_of(__builtin_amdgcn_readfirstlane((int)s_at[e][2])), r = (x - first) % np;
        return np > kWhole + kLead ? x : 2 * r < np ? x - r : x - r + np;
    };
    uint32_t x = end_of(0);
    const uint32_t x_end = end_of(1);
    int b = __builtin_amdgcn_readfirstlane((int)s_at[0][0]);
    uint32_t seq0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_at[0][1]) * (uint32_t)units;       // first piece of sequence b
    n = __builtin_amdgcn_readfirstlane((int)s_at[0][2]);
    row = __builtin_amdgcn_readfirstlane((int)s_at[0][3]);

    while (x < x_end) {
        const uint32_t np = (uint32_t)pieces_of(n);
        if (x >= seq0 + np * (uint32_t)units) {    // on to the next sequence (also over those without a piece)
            seq0 += np * (uint32_t)units;
            n = row_tokens(a, ++b, &row);
            continue;
        }
        const int u = (int)((x - seq0) / np), h = a.by_passes.of(u), g0 = (u - h * a.passes) * 16;
        const uint32_t unit0 = seq0 + (uint32_t)u * np;
        // (a share that ends within a unit's lead leaves it to the next)
        const int p0 = max((int)(x - unit0) - kLead, 0), p1 = (int)min(np, x_end - unit0) - kLead;
        const int n_heads = min(16, a.G - g0);
        const size_t head0 = (size_t)b * a.Hkv * a.G + (size_t)h * a.G + g0;
        x = unit0 + kLead + p1;
        if (p1 <= 0) break;

        // ---- the wavefront's tiles: tokens 64 p + 16 wave ..
        vec8 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[i] = (vec8)(T)0;
            if (lo < n_heads) q[i] = *reinterpret_cast<const vec8 *>(static_cast<const T *>(a.q) + (head0 + lo) * kD + 8 * (4 * i + hi));
        }
        // Weights are 2^(s - m + lead), which cancels in the quotient: in fp16 so that their low parts are normal numbers, in bf16, whose
        // values reach as far as binary32's, so that the weights of all n tokens add up to 1 at most and no numerator, of a
        // wavefront, a part or the whole, exceeds the largest value.
        const float lead = std::is_same_v<T, __bf16> ? -(float)(n > 1 ? 32 - __builtin_clz(n - 1) : 0) : kPScaleLog2;
        float m = kLeast, l = 0.0f;
        f32x4 O[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) O[e] = (f32x4)(0.0f);
        bool bad = false;
        // (read as constants: by scalar loads, which do not queue behind the rows)
        const auto *pages = (const __attribute__((address_space(4))) int32_t *)(a.table + (size_t)row * a.max_pages);
        int t = p0 * kPiece + wave * 16;
        const int t_end = min(n, p1 * kPiece);
        const int t_last = t + (t_end - 1 - t) / kPiece * kPiece;   // the wavefront's last tile, if it has one
        auto place = [&](int p, int t) {   // element of the pools where the tile that starts with token t starts, in page p
            if ((uint32_t)p >= (uint32_t)a.n_pages) {
                bad = true;
                p = 0;
            }
            return ((((int64_t)p * a.Hkv + h) << a.page_log2) + (t & ((1 << a.page_log2) - 1))) * kD;
        };
        auto page_of = [&](int t) { return pages[min(t, t_last) >> a.page_log2]; };
        struct Rows {
            vec8 k[4], v[4];
        };
        auto issue_k = [&](Rows &rows, int64_t at) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                rows.k[i] = __builtin_nontemporal_load(reinterpret_cast<const vec8 *>(static_cast<const T *>(a.K) + at + lo * kD + 8 * (4 * i + hi)));
        };
        auto issue_v = [&](Rows &rows, int64_t at) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                rows.v[r] = __builtin_nontemporal_load(reinterpret_cast<const vec8 *>(static_cast<const T *>(a.V) + at + (4 * hi + r) * kD + 8 * lo));
        };
        // Folds the tile that starts with token t into the state; its rows' registers are loaded again, for the tile
        // kDepth ahead, as soon as they are used up: a wavefront has 16 KiB on their way.
        auto fold = [&](Rows &rows, int t, auto more, int64_t at) {
            __builtin_amdgcn_sched_barrier(0);
            f32x4 S = (f32x4)(0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) S = Mma16<T>::dot32(rows.k[i], q[i], S);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more()) issue_k(rows, at);
            __builtin_amdgcn_sched_barrier(0);
            float s[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] = t + 4 * hi + r < n ? S[r] * kScaleLog2 : kNegInf;
            if (t + 16 > n) {   // (rows of the page behind the last token: weight 0 times whatever is there must be 0)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (t + 4 * hi + r >= n) rows.v[r] = (vec8)(T)0;
            }
            const float mn = fmaxf(m, rows_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));  // (token t is there)
            const float sc = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            float p[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - mn + lead);
            l = l * sc + ((p[0] + p[1]) + (p[2] + p[3]));
            if (__any(sc != 1.0f)) {
                if (hi == 0) sc_sh[wave][lo] = sc;
                const f32x4 f = *reinterpret_cast<const f32x4 *>(&sc_sh[wave][4 * hi]);
#pragma unroll
                for (int e = 0; e < 8; ++e) O[e] *= f;
            }
            // a weight as the sum of two numbers of V's type: 22 bits in fp16, 16 in bf16
            vec4 p_hi, p_lo;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                p_hi[r] = (T)p[r];
                p_lo[r] = (T)(p[r] - (float)p_hi[r]);
            }
            // (four high parts, then the four low parts: two issues in a row into one accumulator would wait for each other)
#pragma unroll
            for (int e0 = 0; e0 < 8; e0 += 4) {
                vec4 v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (vec4){rows.v[0][e0 + e], rows.v[1][e0 + e], rows.v[2][e0 + e], rows.v[3][e0 + e]};
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e0 + e] = Mma16<T>::dot16(p_hi, v[e], O[e0 + e]);
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e0 + e] = Mma16<T>::dot16(p_lo, v[e], O[e0 + e]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (more()) issue_v(rows, at);
        };
        if (t < t_end) {
            Rows rows[kDepth];
            int page[kDepth];
#pragma unroll
            for (int d = 0; d < kDepth; ++d) page[d] = page_of(t + d * kPiece);
#pragma unroll
            for (int d = 0; d < kDepth; ++d) {
                const int64_t at = place(page[d], min(t + d * kPiece, t_last));
                issue_k(rows[d], at);
                issue_v(rows[d], at);
            }
            // (pages are looked up while the tiles before are computed; past its last tile a wavefront reads that
            //  one again, in the caches, so that no load is a choice and every wait is for the loads that it needs)
#pragma unroll
            for (int d = 0; d < kDepth; ++d) page[d] = page_of(t + (kDepth + d) * kPiece);
            for (; t + (kDepth - 1) * kPiece < t_end; t += kDepth * kPiece) {
#pragma unroll
                for (int d = 0; d < kDepth; ++d) {
                    const int64_t at = place(page[d], min(t + (kDepth + d) * kPiece, t_last));
                    page[d] = page_of(t + (2 * kDepth + d) * kPiece);
                    fold(rows[d], t + d * kPiece, std::true_type{}, at);
                }
            }
#pragma unroll
            for (int d = 0; d < kDepth - 1; ++d)
                if (t + d * kPiece < t_end) fold(rows[d], t + d * kPiece, std::false_type{}, 0);
        }
        // ---- the wavefronts' states as one part, or the result
        l = rows_sum(l);
        if (bad) {                                 // (a page that is not there: the unit comes out as NaN)
            m = 0.0f;
            l = __builtin_nanf("");
        }
        if (hi == 0 && lo < n_heads) *reinterpret_cast<float2 *>(&wpart[wave][lo][0]) = make_float2(m, l);
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
            if (4 * hi + rr < n_heads) {
#pragma unroll
                for (int e = 0; e < 8; e += 4)
                    *reinterpret_cast<f32x4 *>(&wpart[wave][4 * hi + rr][4 + 8 * lo + e]) = (f32x4){O[e][rr], O[e + 1][rr], O[e + 2][rr], O[e + 3][rr]};
            }
        const bool whole = p0 == 0 && p1 == (int)np - kLead;
        // (a share has at most one part of a unit that an earlier share began, and one of a unit that goes on)
        float *po = a.part + ((size_t)blockIdx.x * 2 + (p0 == 0 ? 1 : 0)) * GH * kPartStride;
        combine_states<GH>(wpart, n_heads, po, whole ? a.out + head0 * kD : nullptr);
        if (!whole && a.join_here) {
            const int w0 = (int)shares.of(unit0 + kLead), w1 = (int)shares.of(unit0 + np - 1);
            uint32_t *arrived = a.arrived + (size_t)b * units + u;
            if (last_arrival(arrived, (uint32_t)(w1 - w0 + 1), &s_flag)) {
                if (tid == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                join_parts<GH>(a, w0, w1, 0, n_heads, a.out + head0 * kD, red);
            }
        }
        __syncthreads();   // (wpart is written again)
    }
}

// The join as a launch of its own, a workgroup for every query head: where few units are cut into many parts, one
// workgroup at the end of the launch above would read a unit's parts for all of its heads.
template <int GH>
__global__ __launch_bounds__(kWG) void k_paged_join(PagedArgs a, uint32_t wgs)
{
    __shared__ __attribute__((aligned(16))) float red[4][kD + 4];
    __shared__ uint32_t s_w[4];
    const int Hq = a.Hkv * a.G, b = blockIdx.x / Hq, hq = blockIdx.x % Hq, units = a.Hkv * a.passes;
    uint32_t total, ahead;
    count_pieces(a, b, s_w, &total, &ahead);
    int row;
    const uint32_t np = (uint32_t)pieces_of(row_tokens(a, b, &row)), T_all = total * (uint32_t)units;
    if (np <= kWhole + kLead) return;
    const Shares shares(T_all, shares_of(T_all, wgs));
    const int h = hq / a.G, g = hq % a.G;
    const uint32_t unit0 = ahead * (uint32_t)units + (uint32_t)(h * a.passes + g / 16) * np;
    const int w0 = (int)shares.of(unit0 + kLead), w1 = (int)shares.of(unit0 + np - 1);
    if (w0 != w1) join_parts<GH>(a, w0, w1, g % 16, 1, a.out + (size_t)blockIdx.x * kD, red);
}

// Writes new tokens' rows into their pages: a wavefront takes a token and 16 of its 2 Hkv rows, four
// rows to an instruction, 16 lanes each.  Bound by memory: every row read once, written once.
__global__ __launch_bounds__(kWG) void k_append_paged(AppendPagedArgs a)
{
    const int wave = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * (kWG / 64) + (threadIdx.x >> 6))), lane = threadIdx.x & 63;
    const int parts = (2 * a.Hkv + 15) / 16;
    const int i = wave / parts, x0 = (wave % parts) * 16;
    if (i >= a.total_new) return;
    u32x4 v[4];   // (on their way while their place is looked up)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int x = x0 + 4 * e + (lane >> 4), h = x >> 1;
        if (h < a.Hkv) v[e] = (x & 1 ? a.v_new : a.k_new)[(size_t)i * a.new_stride + (size_t)h * 16 + (lane & 15)];
    }
    const int s = last_at_or_before(a.n, i, [&](int j) { return a.new_start[j]; });
    if (i < a.new_start[s] || i >= a.new_start[s + 1]) return;   // a row of no sequence
    const int row = a.rows ? a.rows[s] : s;
    const int start = a.start[s];
    if (row < 0 || row >= a.n_table || start < 0) return;
    const int64_t t = (int64_t)start + (i - a.new_start[s]);
    if (t >= (int64_t)a.max_pages << a.page_log2) return;
    const int p = a.table[(size_t)row * a.max_pages + (t >> a.page_log2)];
    if ((uint32_t)p >= (uint32_t)a.n_pages) return;
    const int in_page = (int)(t & ((1 << a.page_log2) - 1));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int x = x0 + 4 * e + (lane >> 4), h = x >> 1;
        if (h < a.Hkv) (x & 1 ? a.V : a.K)[((((size_t)p * a.Hkv + h) << a.page_log2) + in_page) * 16 + (lane & 15)] = v[e];
    }
}

// ---------------------------------------------------------------- launchers
void make_paged_plan(const ds_pages_t &g, int n, int Hq, int max_len, PagedPlan *p)
{
    p->G = Hq / g.Hkv;
    p->passes = (p->G + 15) / 16;
    p->GH = p->G <= 4 ? 4 : p->G <= 8 ? 8 : 16;
    const int64_t units = (int64_t)n * g.Hkv * p->passes, pieces = units * std::max<int64_t>(1, ((int64_t)max_len + kPiece - 1) / kPiece);
    // One workgroup to a compute unit reads fastest.  Where units are many and short it waits for one's lengths, page and rows after
    // the other's, and a second one is worth its bandwidth: 65 sequences of up to 24 tokens, 40 heads 25.5 us with one and 15.9 with two,
    // 32 of up to 200, 32 heads 26.8 and 25.1; on the other side 128 of up to 500, 8 groups of 8 50.2 and 52.5, one of 900, 32
    // heads 11.1 and 14.3.
    const int cus = device_caps().cus, at_once = pieces <= kWhole * units && units >= 4 * cus ? 2 : 1;
    p->wgs = (int)std::min<int64_t>(pieces, at_once * cus);
    // Up to eight parts a unit the last workgroup joins for all heads (32 units of 900 tokens 10.8 us, with a launch of its own
    // for the join 11.9); more are joined by a workgroup for each head (4 units of 250K tokens, 64 parts: 119 -> 110).
    p->join_here = p->wgs <= 8 * units;
    // Parts first, room for as many as there can be: the counters, which are zero between calls, are then never where calls
    // of other sequences have parts, and one workspace serves all of them.
    p->off_arrived = (size_t)2 * cus * 2 * p->GH * kPartStride * 4;
    p->total = (p->off_arrived + (size_t)units * 4 + 255) / 256 * 256;
}

hipError_t launch_paged(PagedArgs a, const PagedPlan &p, int dtype, hipStream_t st)
{
    a.by_units.set((uint32_t)(a.Hkv * a.passes));
    a.by_passes.set((uint32_t)a.passes);
    const bool bf = dtype == DS_BF16;
    void (*fn)(PagedArgs) = p.GH == 4   ? (bf ? k_paged<__bf16, 4> : k_paged<_Float16, 4>)
                            : p.GH == 8 ? (bf ? k_paged<__bf16, 8> : k_paged<_Float16, 8>)
                                        : (bf ? k_paged<__bf16, 16> : k_paged<_Float16, 16>);
    DS_LAUNCH(KID_PAGED, fn, dim3((unsigned)p.wgs), dim3(kWG), 0, st, a);
    if (!p.join_here) {
        void (*join)(PagedArgs, uint32_t) = p.GH == 4 ? k_paged_join<4> : p.GH == 8 ? k_paged_join<8> : k_paged_join<16>;
        DS_LAUNCH(KID_PAGED, join, dim3((unsigned)(a.n * a.Hkv * a.G)), dim3(kWG), 0, st, a, (uint32_t)p.wgs);
    }
    return hipGetLastError();
}

hipError_t launch_append_paged(const AppendPagedArgs &a, hipStream_t st)
{
    const int64_t waves = (int64_t)a.total_new * ((2 * a.Hkv + 15) / 16);
    DS_LAUNCH(KID_APPEND_PAGED, k_append_paged, dim3((unsigned)((waves + kWG / 64 - 1) / (kWG / 64))), dim3(kWG), 0, st, a);
    return hipGetLastError();
}

}  // namespace ds
