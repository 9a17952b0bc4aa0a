// moa_prompt32.cuh -- the attention of moa_prompt.cuh in fp32.
//
// A CTA takes 64 query rows (the g heads of consecutive tokens) against the rows of one K/V head, 32 keys at a time, a
// warp 16 rows, on the warp-level TF32 MMA.  Every operand is split in two terms in registers, x = hi + lo with 11 bits
// each, and hi hi + hi lo + lo hi leaves 2^-22 of a product out.  The MMA cuts its sums off instead of rounding
// them (about 2^-23 per step), so a chain is 32 features of a score or 32 keys of a weighted sum long; chains are
// added in fp32.  The weights of a tile stay in registers: with keys 2t and 2t + 1 as columns t and t + 4 of the second
// product, the layout that the scores come in is the one that it takes.
//
// What bounds it is the issue of the splits (K and V of a tile are split by every warp) and the MMA.  Where there are few units the
// keys are cut into pieces, joined in order by the CTA that delivers the last one.
#pragma once

#include "moa_prompt.cuh"

namespace moa {

template <int D_, bool PAGED_>
struct Prompt32Cfg {
    static constexpr int D = D_, THREADS = 128, ROWS = 64, KEYS = 32;
    static constexpr bool PAGED = PAGED_;
    static constexpr int LD = D + 4;                       // floats of a row in shared memory: no two of a fragment's lanes share a bank
    static constexpr int OFF_K = ROWS * LD, OFF_V = OFF_K + 2 * KEYS * LD, OFF_NF = OFF_V + 2 * KEYS * LD;
    static constexpr size_t SMEM = sizeof(float) * (size_t)(OFF_NF + D);
};

// A number in two terms of 11 bits.
struct Two { uint32_t hi, lo; };
__device__ __forceinline__ Two in_two(float x)
{
    const float hi = tf32_rn(x);
    return {__float_as_uint(hi), __float_as_uint(x - hi)};
}

// Unit: sequence b's tiles of 64 rows have the numbers from start_b * g / 64 + b on, which no two sequences share.  The last
// numbers, whose rows see most keys, come first.
template <class C>
__device__ __forceinline__ long long prompt32_first(const PromptArgs &a, int b)
{
    return (long long)(a.token_start != nullptr ? a.token_start[b] : C::PAGED ? b : 0) * a.g / C::ROWS + b;
}

constexpr int kPrompt32Few = 512;       // sequences up to which a CTA has one unit

// Where the sequences are not all in order: the one that unit x is of, -1: none, looked for by the whole block.
struct Prompt32Find { PromptSeq s; int b; };
template <class C>
__device__ __noinline__ Prompt32Find prompt32_find(const PromptArgs &a, long long x)
{
    __shared__ Prompt32Find s_found;
    __shared__ int s_floor[C::THREADS / 32];
    const int tid = threadIdx.x, gs = (a.batch + C::THREADS - 1) / C::THREADS, b0 = min(tid * gs, a.batch), b1 = min(b0 + gs, a.batch);
    int floor = prompt_floor(a, b0, b1, s_floor), bad;
    __syncthreads();                                       // (the unit before has read its own)
    if (tid == 0) s_found.b = -1;
    __syncthreads();
    for (int b = b0; b < b1; ++b) {
        const PromptSeq s = prompt_seq<C::PAGED>(a, b, floor, bad);
        if (bad != 0 && blockIdx.x == 0) raise_status(bad);
        const long long tile = x - prompt32_first<C>(a, b);
        if (tile >= 0 && tile * C::ROWS < (long long)s.n * a.g) { s_found.s = s; s_found.b = b; }      // (one thread's, as no two share a token)
    }
    __syncthreads();
    return s_found;
}

// Piece `piece` of unit `u`; the whole block.  down(): whether this thread has seen an entry of token_start below the one before it.
template <class C, class Down>
__device__ __forceinline__ void prompt32_unit(const PromptArgs &a, int splits, int units, int piece, int u, const Down &down)
{
    constexpr int D = C::D, LD = C::LD, KEYS = C::KEYS, NT = D / 8;
    constexpr bool PAGED = C::PAGED;
    extern __shared__ __align__(16) float smem32[];
    __shared__ int s_flag[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int head = u % a.h_kv;
    const long long x = units / a.h_kv - 1 - u / a.h_kv;
    // The last sequence whose first number is at most x, by steps of 128 entries at a time.
    int b = 0, end = a.batch, floor = 0, bad;
    while (end - b > 1) {
        const int step = (end - b + C::THREADS - 1) / C::THREADS, at = b + tid * step;
        const int n = __syncthreads_count(at < end && prompt32_first<C>(a, at) <= x);
        b += max(n - 1, 0) * step;
        end = min(b + step, end);
    }
    PromptSeq s = prompt_seq<PAGED>(a, b, floor, bad);
    float *const sQ = smem32, *const sK = smem32 + C::OFF_K, *const sV = smem32 + C::OFF_V;
    int *const nf = reinterpret_cast<int *>(smem32 + C::OFF_NF);
    for (int f = tid; f < D; f += C::THREADS) nf[f] = 0x7fffffff;
    if (tid < 2) s_flag[tid] = 0;
    if (__syncthreads_or(down())) {                        // the entries do not ascend: the search has found anything
        const Prompt32Find found = prompt32_find<C>(a, x);
        if (found.b < 0) return;
        b = found.b; s = found.s;
    }
    const long long tile = x - prompt32_first<C>(a, b), all = (long long)s.n * a.g;
    if (tile < 0 || tile * C::ROWS >= all) return;
    const int row0 = (int)tile * C::ROWS, rows = (int)min((long long)C::ROWS, all - row0);
    const int least = prompt_sees(a, s, row0), sees = prompt_sees(a, s, row0 + rows - 1);
    // Pieces of this unit: 8 tiles each at the least, of those that were launched.
    const int tiles = (sees + KEYS - 1) / KEYS, pieces = max(1, min(splits, (tiles + 7) / 8));
    if (piece >= pieces) return;
    const int t0 = (int)((long long)tiles * piece / pieces), t1 = (int)((long long)tiles * (piece + 1) / pieces);

    // ---- copies
    constexpr int CPR = D / 4, RPI = C::THREADS / CPR;     // 16-byte chunks of a row, rows per pass of the block
    const int chunk = tid % CPR, rsub = tid / CPR;
    for (int r = rsub; r < C::ROWS; r += RPI) {
        const bool in = r < rows;
        const int row = row0 + (in ? r : 0), tok = div_g(a, row);
        const unsigned char *p = a.q + (long long)(s.first + tok) * a.q_st + ((long long)head * a.g + (row - tok * a.g)) * (D * 4) + 16 * chunk;
        cp16(smem_u32(sQ + r * LD + 4 * chunk), p, in);
    }
    auto copy = [&](int tl, int st) {
#pragma unroll
        for (int i = 0; i < KEYS / RPI; ++i) {
            const int r = RPI * i + rsub, row = tl * KEYS + r;
            const uint32_t kd = smem_u32(sK + (st * KEYS + r) * LD + 4 * chunk), vd = smem_u32(sV + (st * KEYS + r) * LD + 4 * chunk);
            bool in = row < sees;
            const unsigned char *kp = a.k, *vp = a.v;
            if (in) {
                if (PAGED) {
                    const int pi = (int)(((unsigned long long)(uint32_t)row * a.page_mul) >> a.page_sh), off = row - pi * a.page_size;
                    const int page = a.table[(long long)b * a.max_pages + pi];
                    if (page < 0 || page >= a.num_pages) {     // no such page: its scores are NaN
                        if (chunk == 0) raise_status(MOA_STATUS_PAGE_RANGE);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(kd), "r"(0x7fffffffu) : "memory");
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vd), "r"(0u) : "memory");
                        continue;
                    }
                    kp += page * a.k_sp + head * a.k_sh + off * a.k_sr;
                    vp += page * a.v_sp + head * a.v_sh + off * a.v_sr;
                } else {
                    kp += head * a.k_sh + (long long)(s.first + row) * a.k_sr;
                    vp += head * a.v_sh + (long long)(s.first + row) * a.v_sr;
                }
                kp += 16 * chunk; vp += 16 * chunk;
            }
            cp16(kd, kp, in);
            cp16(vd, vp, in);
        }
    };
    if (t0 < t1) copy(t0, 0);
    cp_commit();

    // this lane's rows of the unit: ra, ra + 8
    const int ra = 16 * warp + g;
    int lim[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) lim[e] = ra + 8 * e < rows ? prompt_sees(a, s, row0 + ra + 8 * e) : 0;
    const float scale = a.negate ? -a.qscale : a.qscale;
    float o[NT][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < NT; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;

    for (int tl = t0; tl < t1; ++tl) {
        const int st = (tl - t0) & 1;
        if (tl + 1 < t1) copy(tl + 1, st ^ 1);
        cp_commit();
        cp_wait<1>();
        __syncthreads();
        const float *const k = sK + st * KEYS * LD, *const v = sV + st * KEYS * LD;
        if (a.causal && (tl + 1) * KEYS > least) {         // rows that not every query sees: their V as 0 where it is not finite, and noted
            for (int i = tid; i < KEYS * D; i += C::THREADS) {
                const int r = i / D, f = i % D;
                float *const p = sV + (st * KEYS + r) * LD + f;
                if (!isfinite(*p)) { *p = 0.f; atomicMin(&nf[f], tl * KEYS + r); s_flag[0] = 1; }
            }
            __syncthreads();
        }
        // ---- scores
        float c[4][4];
#pragma unroll
        for (int n = 0; n < 4; ++n) c[n][0] = c[n][1] = c[n][2] = c[n][3] = 0.f;
#pragma unroll 1
        for (int d0 = 0; d0 < D; d0 += 32) {
            float z[4][4];
#pragma unroll
            for (int n = 0; n < 4; ++n) z[n][0] = z[n][1] = z[n][2] = z[n][3] = 0.f;
#pragma unroll
            for (int d = d0; d < d0 + 32; d += 8) {
                const float *const q = sQ + ra * LD + d + t;
                const Two a0 = in_two(q[0]), a1 = in_two(q[8 * LD]), a2 = in_two(q[4]), a3 = in_two(q[8 * LD + 4]);
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const float *const kk = k + (8 * n + g) * LD + d + t;
                    const Two b0 = in_two(kk[0]), b1 = in_two(kk[4]);
                    mma_tf32_16x8x8(z[n], a0.lo, a1.lo, a2.lo, a3.lo, b0.hi, b1.hi);
                    mma_tf32_16x8x8(z[n], a0.hi, a1.hi, a2.hi, a3.hi, b0.lo, b1.lo);
                    mma_tf32_16x8x8(z[n], a0.hi, a1.hi, a2.hi, a3.hi, b0.hi, b1.hi);
                }
            }
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) c[n][e] += z[n][e];
        }
        // ---- weights
        float f[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float top = -INFINITY;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float &y = c[n][2 * r + e];
                    y = tl * KEYS + 8 * n + 2 * t + e < lim[r] ? y * scale : -INFINITY;
                    top = max_nan(top, y);
                }
            top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
            float mn = max_nan(m[r], top);
            if (mn == INFINITY) mn = __uint_as_float(0x7fffffffu);             // (infinity less itself: the row is NaN)
            f[r] = mn == m[r] ? 1.f : m[r] == -INFINITY && mn == mn ? 0.f : fast_exp2(m[r] - mn);
            m[r] = mn;
            const float ref = mn == -INFINITY ? 0.f : mn;
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    c[n][2 * r + e] = fast_exp2(c[n][2 * r + e] - ref);
                    sum += c[n][2 * r + e];
                }
            l[r] = fmaf(l[r], f[r], sum);
        }
        // ---- weighted sum
        Two p[4][4];
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            p[n][0] = in_two(c[n][0]); p[n][1] = in_two(c[n][2]); p[n][2] = in_two(c[n][1]); p[n][3] = in_two(c[n][3]);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *const vv = v + (8 * i + 2 * t) * LD + 8 * n + g;
                const Two b0 = in_two(vv[0]), b1 = in_two(vv[LD]);
                mma_tf32_16x8x8(z, p[i][0].lo, p[i][1].lo, p[i][2].lo, p[i][3].lo, b0.hi, b1.hi);
                mma_tf32_16x8x8(z, p[i][0].hi, p[i][1].hi, p[i][2].hi, p[i][3].hi, b0.lo, b1.lo);
                mma_tf32_16x8x8(z, p[i][0].hi, p[i][1].hi, p[i][2].hi, p[i][3].hi, b0.hi, b1.hi);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = fmaf(o[n][e], f[e >> 1], z[e]);
        }
        __syncthreads();                                   // the tile is rewritten by the copies after the next
    }
    cp_wait<0>();
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
        l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
    }
    if (s_flag[0]) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (nf[8 * n + 2 * t + (e & 1)] < lim[e >> 1]) o[n][e] = __uint_as_float(0x7fffffffu);
    }
    auto out_row = [&](int r) {                            // r: of the unit
        const int row = row0 + r, tok = div_g(a, row);
        return reinterpret_cast<float *>(a.out + (long long)(s.first + tok) * a.o_st + ((long long)head * a.g + (row - tok * a.g)) * (D * 4));
    };
    if (pieces == 1) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            if (ra + 8 * r >= rows) continue;
            float *const to = out_row(ra + 8 * r);
            const float inv = lim[r] <= 0 ? 0.f : 1.f / l[r];
#pragma unroll
            for (int n = 0; n < NT; ++n)
                *reinterpret_cast<float2 *>(to + 8 * n + 2 * t) = make_float2(o[n][2 * r] * inv, o[n][2 * r + 1] * inv);
        }
        return;
    }
    // ---- a piece: (o, m, l) of every row into its slot; the last one joins them
    const long long slot = (long long)a.slot_rows * (D + 2);
    float *const part = a.slots + ((long long)u * splits + piece) * slot;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        if (ra + 8 * r >= rows) continue;
        float *const to = part + (ra + 8 * r) * (D + 2);
#pragma unroll
        for (int n = 0; n < NT; ++n)
            *reinterpret_cast<float2 *>(to + 8 * n + 2 * t) = make_float2(o[n][2 * r], o[n][2 * r + 1]);
        if (t == 0) *reinterpret_cast<float2 *>(to + D) = make_float2(m[r], l[r]);
    }
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        unsigned long long *word = a.tickets + u;
        const bool last = ticket_arrive(word, a.ticket_tag) + 1 == (unsigned)pieces;
        if (last) *word = 0;
        __threadfence();
        s_flag[1] = last;
    }
    __syncthreads();
    if (!s_flag[1]) return;
    const float *const p0 = a.slots + (long long)u * splits * slot;
    for (int i = tid; i < rows * (D / 2); i += C::THREADS) {
        const int r = i / (D / 2), col = i % (D / 2) * 2;
        float top = -INFINITY, total = 0.f, y0 = 0.f, y1 = 0.f;
        // (eight pieces' loads under way at once: left to the compiler, 148 pieces took 240 us in one build and 325 in another)
        constexpr int AT_ONCE = 8;
        const float *const mine = p0 + r * (D + 2);
        for (int p = 0; p < pieces; p += AT_ONCE) {
            float m8[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) m8[k] = p + k < pieces ? __ldcg(reinterpret_cast<const float2 *>(mine + (p + k) * slot + D)).x : -INFINITY;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) top = max_nan(top, m8[k]);
        }
        for (int p = 0; p < pieces; p += AT_ONCE) {
            float2 e[AT_ONCE], y[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const bool in = p + k < pieces;
                e[k] = in ? __ldcg(reinterpret_cast<const float2 *>(mine + (p + k) * slot + D)) : make_float2(-INFINITY, 0.f);
                y[k] = in ? __ldcg(reinterpret_cast<const float2 *>(mine + (p + k) * slot + col)) : make_float2(0.f, 0.f);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const float w = exp2_diff(e[k].x, top);
                total = fmaf(e[k].y, w, total);
                y0 = fmaf(y[k].x, w, y0); y1 = fmaf(y[k].y, w, y1);
            }
        }
        const float inv = prompt_sees(a, s, row0 + r) <= 0 ? 0.f : 1.f / total;
        *reinterpret_cast<float2 *>(out_row(r) + col) = make_float2(y0 * inv, y1 * inv);
    }
}

// MANY: more than kPrompt32Few sequences, and a CTA takes several units.
template <class C, bool MANY>
__global__ void __launch_bounds__(C::THREADS, 2) prompt32_kernel(const __grid_constant__ PromptArgs a, int splits, int units)
{
    launch_dependents();
    grid_dependency_wait();
    if (blockIdx.x == 0)
        for (int b = threadIdx.x; b < a.batch; b += C::THREADS) {
            int floor = 0, bad;
            prompt_seq<C::PAGED>(a, b, floor, bad);
            if (bad != 0) raise_status(bad);
        }
    // Every CTA looks whether the entries of token_start ascend: only then does a search find a unit's sequence.
    if constexpr (MANY) {
        int down = 0;
        if (a.token_start != nullptr)
            for (int b = threadIdx.x; b < a.batch; b += C::THREADS) down |= a.token_start[b + 1] < a.token_start[b];
        for (int i = blockIdx.x; i < units; i += gridDim.x) {          // (with so many units none is cut)
            if (i != blockIdx.x) __syncthreads();          // (the unit before has read what it keeps in shared memory)
            prompt32_unit<C>(a, 1, units, 0, i, [&] { return down; });
        }
    } else {
        constexpr int N = kPrompt32Few / C::THREADS;       // (they are on their way while the unit is looked for)
        int x[N] = {}, y[N] = {};
        if (a.token_start != nullptr)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int b = threadIdx.x + i * C::THREADS;
                if (b < a.batch) { x[i] = a.token_start[b]; y[i] = a.token_start[b + 1]; }
            }
        prompt32_unit<C>(a, splits, units, blockIdx.x % splits, blockIdx.x / splits, [&] {
            int down = 0;
#pragma unroll
            for (int i = 0; i < N; ++i) down |= y[i] < x[i];
            return down;
        });
    }
}

}  // namespace moa
