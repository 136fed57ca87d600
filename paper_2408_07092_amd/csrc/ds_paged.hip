// Dense decode attention of one new token of every sequence over a paged cache, and the writing of
// new tokens' rows into its pages.
//
// The attention reads every K and V row once and computes next to nothing on it: memory bound.  Lengths are
// known on the device only and may differ as they like, so the work is cut there: all the
// sequences' tokens, a KV head after the other, are one line of pieces of 64 tokens, of which every workgroup
// takes an equal, contiguous share.  A share covers the end of one unit (sequence and KV head), whole units, and
// the beginning of another, or a part of a single one; a unit's parts meet in the workspace, where
// the last workgroup to arrive joins them in their order along the cache.  Which part holds
// which tokens follows from the lengths and the launch alone, so results do not depend on who is last.
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
__device__ __forceinline__ int pieces_of(int tokens) { return tokens > 0 ? (tokens - 1) / kPiece + 1 : 0; }

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
// a wavefront for a head, or two or four of them where there are fewer heads, 12 or 16 parts in flight (as registers allow), folded in
// an order that depends on the launch alone.  All threads call it.
template <int GH>
__device__ __forceinline__ void join_parts(const PagedArgs &a, int w0, int w1, int n_heads, float *out, float (*red)[kD + 4])
{
    constexpr int kBatch = 12;
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
                    const float *pc = a.part + (((size_t)w * 2 + (w == w0 ? 1 : 0)) * GH + g) * kPartStride;
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

template <class T, int GH>
__global__ __launch_bounds__(kWG, GH > 8 ? 3 : 4) void k_paged(PagedArgs a)
{
    typedef typename Mma16<T>::vec8 vec8;
    typedef typename Mma16<T>::vec4 vec4;
    __shared__ __attribute__((aligned(16))) float wpart[4][GH][kPartStride];
    __shared__ __attribute__((aligned(16))) float sc_sh[4][16];
    __shared__ uint32_t s_w[4], s_flag, s_at[2];
    float (*red)[kD + 4] = reinterpret_cast<float (*)[kD + 4]>(&wpart[0][0][0]);   // (4 of them; used after wpart)

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 15, hi = lane >> 4;
    const int units = a.Hkv * a.passes;   // of a sequence
    // ---- all pieces, and where this workgroup's share starts
    const int per = (a.n + kWG - 1) / kWG;
    uint32_t mine = 0;
    for (int i = 0; i < per; ++i) {
        const int b = tid * per + i;
        int row, n = 1;
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
    const uint32_t W = max(1u, min(gridDim.x, T_all / (uint32_t)a.least));
    if (blockIdx.x >= W || T_all == 0) return;
    const Shares shares(T_all, W);
    uint32_t x = shares.start(blockIdx.x);
    const uint32_t x_end = shares.start(blockIdx.x + 1);
    const uint32_t want = x / (uint32_t)units;     // the piece of a sequence that the share starts in, counted over sequences
    if (ahead <= want && want < ahead + mine) {
        int b = tid * per, row;
        for (uint32_t k; (k = (uint32_t)pieces_of(row_tokens(a, b, &row))) <= want - ahead; ++b) ahead += k;
        s_at[0] = (uint32_t)b;
        s_at[1] = ahead;
    }
    __syncthreads();
    int b = __builtin_amdgcn_readfirstlane((int)s_at[0]);
    uint32_t seq0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)s_at[1]) * (uint32_t)units;       // first piece of sequence b

    while (x < x_end) {
        int row;
        const int n = row_tokens(a, b, &row);
        const uint32_t np = (uint32_t)pieces_of(n);
        if (x >= seq0 + np * (uint32_t)units) {    // (also over sequences without a piece)
            seq0 += np * (uint32_t)units;
            ++b;
            continue;
        }
        const int u = (int)((x - seq0) / np), h = u / a.passes, g0 = (u % a.passes) * 16;
        const uint32_t unit0 = seq0 + (uint32_t)u * np;
        const int p0 = (int)(x - unit0), p1 = (int)min(np, x_end - unit0);
        const int n_heads = min(16, a.G - g0);
        const size_t head0 = (size_t)b * a.Hkv * a.G + (size_t)h * a.G + g0;
        x = unit0 + p1;

        // ---- the wavefront's tiles: tokens 64 p + 16 wave ..
        vec8 q[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            q[i] = (vec8)(T)0;
            if (lo < n_heads) q[i] = *reinterpret_cast<const vec8 *>(static_cast<const T *>(a.q) + (head0 + lo) * kD + 8 * (4 * i + hi));
        }
        float m = kNegInf, l = 0.0f;
        f32x4 O[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) O[e] = (f32x4)(0.0f);
        bool bad = false;
        const int32_t *pages = a.table + (size_t)row * a.max_pages;
        vec8 kr[4], vr[4];
        auto place = [&](int p, int t) {   // element of the pools where the tile that starts with token t starts, in page p
            if ((uint32_t)p >= (uint32_t)a.n_pages) {
                bad = true;
                p = 0;
            }
            return ((((int64_t)p * a.Hkv + h) << a.page_log2) + (t & ((1 << a.page_log2) - 1))) * kD;
        };
        auto issue_k = [&](int64_t at) {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                kr[i] = __builtin_nontemporal_load(reinterpret_cast<const vec8 *>(static_cast<const T *>(a.K) + at + lo * kD + 8 * (4 * i + hi)));
        };
        auto issue_v = [&](int64_t at) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                vr[r] = __builtin_nontemporal_load(reinterpret_cast<const vec8 *>(static_cast<const T *>(a.V) + at + (4 * hi + r) * kD + 8 * lo));
        };
        int t = p0 * kPiece + wave * 16;
        const int t_end = min(n, p1 * kPiece);
        if (t < t_end) {
            // (a tile's page is looked up while the tile before the one before it is computed)
            const int last_entry = (n - 1) >> a.page_log2;
            int64_t at = place(pages[t >> a.page_log2], t);
            int page = pages[min((t + kPiece) >> a.page_log2, last_entry)];
            issue_k(at);
            issue_v(at);
            for (; t < t_end; t += kPiece) {
                const bool more = t + kPiece < t_end;
                if (more) at = place(page, t + kPiece);
                page = pages[min((t + 2 * kPiece) >> a.page_log2, last_entry)];
                __builtin_amdgcn_sched_barrier(0);
                f32x4 S = (f32x4)(0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) S = Mma16<T>::dot32(kr[i], q[i], S);
                __builtin_amdgcn_sched_barrier(0);
                if (more) issue_k(at);
                __builtin_amdgcn_sched_barrier(0);
                float s[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) s[r] = t + 4 * hi + r < n ? S[r] * kScaleLog2 : kNegInf;
                if (t + 16 > n) {   // (rows of the page behind the last token: weight 0 times whatever is there must be 0)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (t + 4 * hi + r >= n) vr[r] = (vec8)(T)0;
                }
                const float mn = fmaxf(m, rows_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]))));  // (token t is there)
                const float sc = m == kNegInf ? 0.0f : __builtin_amdgcn_exp2f(m - mn);
                m = mn;
                float p[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) p[r] = __builtin_amdgcn_exp2f(s[r] - mn + kPScaleLog2);
                l = l * sc + ((p[0] + p[1]) + (p[2] + p[3]));
                if (__any(sc != 1.0f)) {
                    if (hi == 0) sc_sh[wave][lo] = sc;
                    const f32x4 f = *reinterpret_cast<const f32x4 *>(&sc_sh[wave][4 * hi]);
#pragma unroll
                    for (int e = 0; e < 8; ++e) O[e] *= f;
                }
                // a weight as the sum of two numbers of V's type: 22 bits in fp16 (the scale keeps the low part normal), 16 in bf16
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
                    for (int e = 0; e < 4; ++e) v[e] = (vec4){vr[0][e0 + e], vr[1][e0 + e], vr[2][e0 + e], vr[3][e0 + e]};
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[e0 + e] = Mma16<T>::dot16(p_hi, v[e], O[e0 + e]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) O[e0 + e] = Mma16<T>::dot16(p_lo, v[e], O[e0 + e]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                __builtin_amdgcn_sched_barrier(0);
                if (more) issue_v(at);
            }
        }
        // ---- the wavefronts' states as one part, or the result
        l = rows_sum(l);
        if (bad) {                                 // (a page that is not there: the unit comes out as NaN)
            m = 0.0f;
            l = __builtin_nanf("");
        }
        if (hi == 0 && lo < n_heads) {
            wpart[wave][lo][0] = m;
            wpart[wave][lo][1] = l;
        }
#pragma unroll
        for (int rr = 0; rr < 4; ++rr)
            if (4 * hi + rr < n_heads) {
#pragma unroll
                for (int e = 0; e < 8; ++e) wpart[wave][4 * hi + rr][4 + 8 * lo + e] = O[e][rr];
            }
        const bool whole = p0 == 0 && p1 == (int)np;
        // (a share has at most one part of a unit that an earlier share began, and one of a unit that goes on)
        float *po = a.part + ((size_t)blockIdx.x * 2 + (p0 == 0 ? 1 : 0)) * GH * kPartStride;
        wg_combine_store<GH>(wpart, n_heads, po, kPartStride, whole ? a.out + head0 * kD : nullptr);
        if (!whole) {
            const int w0 = (int)shares.of(unit0), w1 = (int)shares.of(unit0 + np - 1);
            uint32_t *arrived = a.arrived + (size_t)b * units + u;
            if (last_arrival(arrived, (uint32_t)(w1 - w0 + 1), &s_flag)) {
                if (tid == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                join_parts<GH>(a, w0, w1, n_heads, a.out + head0 * kD, red);
            }
        }
        __syncthreads();   // (wpart is written again)
    }
}

// Writes new tokens' rows into their pages: a wavefront takes a token and 16 of its 2 Hkv rows, four
// rows to an instruction, 16 lanes each.  Bound by memory: every row read once, written once.
__global__ __launch_bounds__(kWG) void k_append_paged(AppendPagedArgs a)
{
    const int wave = (int)(blockIdx.x * (kWG / 64) + (threadIdx.x >> 6)), lane = threadIdx.x & 63;
    const int parts = (2 * a.Hkv + 15) / 16;
    const int i = wave / parts, x0 = (wave % parts) * 16;
    if (i >= a.total_new) return;
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
    u32x4 v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int x = x0 + 4 * e + (lane >> 4), h = x >> 1;
        if (h < a.Hkv) v[e] = (x & 1 ? a.v_new : a.k_new)[(size_t)i * a.new_stride + (size_t)h * 16 + (lane & 15)];
    }
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
    p->least = 2;
    const int64_t pieces = (int64_t)n * g.Hkv * p->passes * std::max(1, (max_len + kPiece - 1) / kPiece);
    p->wgs = (int)std::min<int64_t>(pieces, device_caps().cus * (p->GH > 8 ? 3 : 4));
    p->off_part = ((size_t)n * g.Hkv * p->passes * 4 + 255) / 256 * 256;
    p->total = (p->off_part + (size_t)p->wgs * 2 * p->GH * kPartStride * 4 + 255) / 256 * 256;
}

hipError_t launch_paged(PagedArgs a, const PagedPlan &p, int dtype, hipStream_t st)
{
    const dim3 grid((unsigned)p.wgs);
    const bool bf = dtype == DS_BF16;
    void (*fn)(PagedArgs) = p.GH == 4   ? (bf ? k_paged<__bf16, 4> : k_paged<_Float16, 4>)
                            : p.GH == 8 ? (bf ? k_paged<__bf16, 8> : k_paged<_Float16, 8>)
                                        : (bf ? k_paged<__bf16, 16> : k_paged<_Float16, 16>);
    DS_LAUNCH(KID_PAGED, fn, grid, dim3(kWG), 0, st, a);
    return hipGetLastError();
}

hipError_t launch_append_paged(const AppendPagedArgs &a, hipStream_t st)
{
    const int64_t waves = (int64_t)a.total_new * ((2 * a.Hkv + 15) / 16);
    DS_LAUNCH(KID_APPEND_PAGED, k_append_paged, dim3((unsigned)((waves + kWG / 64 - 1) / (kWG / 64))), dim3(kWG), 0, st, a);
    return hipGetLastError();
}

}  // namespace ds
