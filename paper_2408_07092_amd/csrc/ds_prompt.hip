// Attention over whole prompts: causal, grouped heads, packed sequences of unlike lengths, with the
// keys in rows of any stride (packed, or the contiguous caches) or in pages.
//
//   O[i] = sum_j p_ij v_j / sum_j p_ij,   p_ij = 2^(s_ij - m_i),   s_ij = log2(e)/sqrt(d) q_i . k_j
//
// over the keys j <= i + nk - nq, in one pass over the keys with a running maximum m and a
// running sum.  Bound by the matrix units: 4 d flops a pair against a few bytes for each row.
//
// The G query heads of a KV head are rows of one matrix: row token * G + g.  A workgroup takes 128 of
// these rows, a wavefront 32, and walks the keys in tiles of 64 that all of its wavefronts share from LDS.
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
// The running maximum is raised only when a row's exceeds it by more than this (in the log2 domain), so
// that most tiles rescale nothing; weights carry the factor 2^kRoom besides, which cancels in the quotient.  They
// are at most 2^(7 + 8), within fp16, and normal fp16 numbers down to 2^-21 of the row's largest.
constexpr float kSlack = 8.0f, kRoom = 7.0f;
constexpr float kLeast = -1e30f;                           // stands for "no key yet": 2^(s - kLeast) is never formed

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
// pieces on the same four banks.  K is read a piece of each of 32 rows at a time, V by the
// transposing read two pieces of each of four rows.
__device__ __forceinline__ int k_piece(int r, int c) { return r * 16 + (c ^ (r & 15)); }
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

// Sixteen bytes of every lane from memory into LDS, to `at` (bytes, the wavefront's) + 16 lane, past the registers.
// Written out because the compiler, not knowing which buffer a transposing read reads, would wait for every load
// in flight ahead of each of them; the loads are waited for by wait_tiles.  (m0, the place in LDS, is used for nothing
// else in this kernel.)
__device__ __forceinline__ void load_to_lds(const void *src, uint32_t at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(at), "v"(src) : "memory");
}
__device__ __forceinline__ void wait_tiles()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

template <class T, bool PAGED>
__global__ __launch_bounds__(kWG, 2) void k_prompt(PromptArgs a)
{
    typedef typename Mma<T>::vec8 vec8;
    extern __shared__ __attribute__((aligned(16))) u32x4 tiles[];  // K, K, V, V: 16-byte pieces
    constexpr int kPieces = kTileBytes / 16;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lo = lane & 31, hi = lane >> 5;
    const int kvh = blockIdx.x % a.Hkv;
    const int slot = a.n_tiles - 1 - (int)(blockIdx.x / a.Hkv);
    // ---- the sequence and its rows
    const int s = last_at_or_before(a.n_seqs, slot, [&](int i) { return tile_base(a.q_start[i], a.G, i); });
    const int qs = a.q_start[s], qe = a.q_start[s + 1];
    if (qs < 0 || qe < qs || qe > a.total_q) return;
    const int n_rows = (qe - qs) * a.G;
    const int r0 = (slot - tile_base(qs, a.G, s)) * kPromptRows;
    if (r0 < 0 || r0 >= n_rows) return;
    bool bad = false;
    int nk;
    int64_t kv0 = 0;
    const int32_t *pages = nullptr;
    if constexpr (PAGED) {
        const int row = a.rows ? a.rows[s] : s;
        bad = row < 0 || row >= a.n_table;
        nk = bad ? 0 : a.kv_len[row];
        pages = a.table + (size_t)(bad ? 0 : row) * a.max_pages;
        bad |= nk < 0 || (int64_t)nk > (int64_t)a.max_pages << a.page_log2;
    } else {
        nk = a.kv_len[s];
        kv0 = a.kv_start[s];
        bad = nk < 0 || nk > kMostTokens || kv0 < 0 || (nk > 0 && (kv0 + nk - 1) * a.kv_stride + (int64_t)(a.Hkv - 1) * a.kv_head_stride + kD > a.kv_elems);
        kv0 = kv0 * a.kv_stride + (int64_t)kvh * a.kv_head_stride;
    }
    if (bad) nk = 0;
    const int before = nk - (qe - qs);               // keys ahead of the sequence's first row's own
    const int last_row = min(n_rows, r0 + kPromptRows) - 1;
    const int seen = max(0, min(nk, last_row / a.G + before + 1));    // keys that some row of the workgroup sees
    const int n_kt = (seen + kKeys - 1) / kKeys;
    const int my_row = r0 + wave * 32 + lo;
    const bool on = my_row < n_rows;
    const int my_last = on ? min(my_row / a.G + before, nk - 1) : -1; // last key that the lane's row sees
    // tiles that some row of the wavefront sees, and those that all of its rows see whole
    const int n_mine = min(n_kt, max(0, (min(r0 + wave * 32 + 31, n_rows - 1)) / a.G + before + kKeys) / kKeys);
    const int n_clear = r0 + wave * 32 >= n_rows ? 0 : max(0, min((r0 + wave * 32) / a.G + before + 1, nk)) / kKeys;

    vec8 q[8];
    {
        const int row = min(my_row, n_rows - 1);
        const T *src = static_cast<const T *>(a.q) + (size_t)(qs + row / a.G) * a.q_stride + (size_t)(kvh * a.G + row % a.G) * kD + hi * 8;
#pragma unroll
        for (int x = 0; x < 8; ++x) q[x] = *reinterpret_cast<const vec8 *>(src + x * 16);
    }
    f32x16 O[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) O[d] = (f32x16)(0.0f);
    float m = kLeast, l = 0.0f;

    // ---- tiles: of each 16 rows a wavefront brings four, a lane one piece.  The pieces of a row change places on the
    // way (see k_piece), by the lane's place in memory, since in LDS a load's lanes lie side by side.
    // Rows past the last key re-read it (their weight is 0, and 0 times whatever lies behind it need not be).
    const int lane_row = 4 * wave + (lane >> 4);
    const int64_t step_row = PAGED ? kD : a.kv_stride;
    const T *Kp = static_cast<const T *>(a.K) + kv0 + lane_row * step_row + ((lane & 15) ^ lane_row) * 8;
    const T *Vp = static_cast<const T *>(a.V) + kv0 + lane_row * step_row + ((lane & 15) ^ ((lane >> 4) << 2)) * 8;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void *)tiles + wave * 1024;
    // Paged: lane i % 4 of `of` holds the page of a tile's rows 16 i .. (16 rows that start at a multiple of 16 are in one page)
    auto page_ids = [&](int kt) {
        int p = 0;
        if constexpr (PAGED) {
            if (nk > 0) p = pages[min(kt * kKeys + (lane & 3) * 16, nk - 1) >> a.page_log2];
            if ((uint32_t)p >= (uint32_t)a.n_pages) {
                if (kt < n_kt) bad = true;
                p = 0;
            }
        }
        return p;
    };
    auto load_tile = [&](const T *base, int kt, int buffer, int of) {
        const bool full = (kt + 1) * kKeys <= nk;
        const uint32_t at = lds0 + buffer * kTileBytes;
#pragma unroll
        for (int i = 0; i < kKeys / 16; ++i) {
            const int t0 = kt * kKeys + i * 16;
            const T *src = base;
            if constexpr (PAGED) {
                const int64_t p = __builtin_amdgcn_readlane(of, i);
                src += (((p * a.Hkv + kvh) << a.page_log2) + (min(t0, nk - 1) & ((1 << a.page_log2) - 1) & ~15)) * kD;
                if (full) load_to_lds(src, at + i * 4096);
                else load_to_lds(src + (min(t0 + lane_row, nk - 1) - (min(t0, nk - 1) & ~15) - lane_row) * kD, at + i * 4096);
            } else {
                src += t0 * a.kv_stride;
                if (full) load_to_lds(src, at + i * 4096);
                else load_to_lds(src + (int64_t)min(0, nk - 1 - t0 - lane_row) * a.kv_stride, at + i * 4096);
            }
        }
    };

    auto scores = [&](int buffer, f32x16 (&S)[2]) {
        const u32x4 *kb = tiles + buffer * kPieces;
#pragma unroll
        for (int b = 0; b < 2; ++b) S[b] = (f32x16)(0.0f);
#pragma unroll
        for (int x = 0; x < 8; ++x)
#pragma unroll
            for (int b = 0; b < 2; ++b)
                S[b] = Mma<T>::dot(__builtin_bit_cast(vec8, kb[k_piece(b * 32 + lo, 2 * x + hi)]), q[x], S[b]);
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
    auto values = [&](int buffer, const vec8 (&P)[4], int c0 = 0, int c1 = 4) {
        const u32x4 *vb = tiles + (2 + buffer) * kPieces;
#pragma unroll
        for (int c = c0; c < c1; ++c)
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                // four keys by sixteen channels for each 16 lanes: lane 4 j + x brings row j, channels 4 x ..
                const int r = 16 * c + 4 * hi + (lane & 15) / 4, piece = d * 4 + ((lane >> 4) & 1) * 2 + (lane & 3) / 2;
                const char *v0 = reinterpret_cast<const char *>(vb + v_piece(r, piece)) + (lane & 1) * 8;
                const char *v1 = reinterpret_cast<const char *>(vb + v_piece(r + 8, piece)) + (lane & 1) * 8;
                const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v0);
                const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)v1);
                const s16x8 v = {x0[0], x0[1], x0[2], x0[3], x1[0], x1[1], x1[2], x1[3]};
                O[d] = Mma<T>::dot(__builtin_bit_cast(vec8, v), P[c], O[d]);
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
        load_tile(Kp, 0, 0, ids0);
        load_tile(Vp, 0, 2, ids0);
        if (n_kt > 1) load_tile(Kp, 1, 1, ids1);
    }
    ids0 = page_ids(2);
    wait_tiles();
    f32x16 S0[2], S1[2];
    if (n_mine > 0) {
        scores(0, S0);
        if (n_clear < 1) hide(0, S0);
        raise(S0);
    }
    // A step: most of tile kt's weights while the matrix units form the scores of the next, the rest while they form its
    // values, with the sum of the weights and the next one's maximum (so that both halves have vector work, and registers do); the K tile after the next and the next V tile are on their way meanwhile, to
    // places whose tiles were done with before the last barrier.  odd: kt % 2
    auto bring = [&](int kt, int odd) {
        if (kt + 1 < n_kt) load_tile(Vp, kt + 1, 3 - odd, ids1);
        if (kt + 2 < n_kt) load_tile(Kp, kt + 2, odd, ids0);
        ids1 = ids0;
        ids0 = page_ids(kt + 3);
    };
    auto step = [&](int kt, int odd, f32x16 (&S)[2], f32x16 (&N)[2], auto hidden) {
        bring(kt, odd);
        vec8 P[4];
        scores(1 - odd, N);
        weights(S, P, 0, 3);
        if (hidden) hide(kt + 1, N);
        values(odd, P, 0, 3);
        weights(S, P, 3, 4);
        values(odd, P, 3, 4);
        add_up(P);
        raise(N);
        wait_tiles();
    };
    int kt = 0;
    for (; kt + 2 < n_clear; kt += 2) {
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
            vec8 P[4];
            weights(S0, P);
            values(kt & 1, P);
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
    if (!on) return;
    l = halves_sum(l);
    // (a row that sees no key is zero; one whose pages or places are not there is NaN)
    const float inv = bad ? __builtin_nanf("") : l > 0.0f ? 1.0f / l : 0.0f;
    T *dst = static_cast<T *>(a.out) + (size_t)(qs + my_row / a.G) * a.out_stride + (size_t)(kvh * a.G + my_row % a.G) * kD + 4 * hi;
    typedef T vec4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = (T)(O[d][4 * i + j] * inv);
            *reinterpret_cast<vec4 *>(dst + d * 32 + i * 8) = x;
        }
}

// ---------------------------------------------------------------- launcher
bool make_prompt_plan(const ds_prompt_t &m, PromptPlan *p)
{
    p->G = m.Hq / m.Hkv;
    p->n_tiles = (int)((int64_t)m.total_q * p->G / kPromptRows) + m.n_seqs;
    p->total = 256;
    return true;
}

typedef void (*PromptFn)(PromptArgs);
static PromptFn prompt_fn(bool paged, int dtype)
{
    if (dtype == DS_BF16) return paged ? k_prompt<__bf16, true> : k_prompt<__bf16, false>;
    return paged ? k_prompt<_Float16, true> : k_prompt<_Float16, false>;
}

hipError_t launch_prompt(PromptArgs a, bool paged, int dtype, hipStream_t st)
{
    const PromptFn fn = prompt_fn(paged, dtype);
    DS_LAUNCH(KID_PROMPT, fn, dim3((unsigned)(a.n_tiles * a.Hkv)), dim3(kWG), 4 * kTileBytes, st, a);
    return hipGetLastError();
}

}  // namespace ds
