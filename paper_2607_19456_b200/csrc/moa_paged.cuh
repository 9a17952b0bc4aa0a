// moa_paged.cuh -- single-query attention over a paged cache held in fp32, bf16, fp16 or 4 bits.
//
// Steps I-III of Algorithm 1 in online-softmax form, as in the streaming kernels, on a cache whose
// rows are found through a page table.  What is different here:
//
//  - Work is dealt to WARPS.  The cached rows of every (sequence, kv head) unit are cut into tiles
//    of 16 rows; all tiles form one flat list, cut into equal contiguous ranges first for the CTAs,
//    then for the warps of a CTA.  A unit that lies inside one warp's range never leaves the warp;
//    only the (at most two) units that a range cuts go through shared memory, once, at the end of
//    the CTA.  Small caches (16 and 4 bits) have units that take a CTA a microsecond or two; a block
//    barrier for every unit, as the fp32 streaming kernels have, would cost as much again.
//  - Tiles come through per-lane 16-byte asynchronous copies into a ring of the warp's own: a page may
//    end inside a tile, and a bulk copy per tile and operand (an SM retires one per 70 cycles) would bring
//    4 bits no more than 15 bytes a cycle of the 24 that HBM has.  16 and 32 bits would have enough of them (58
//    and 117 at rows of 128); there the copies below reach the copy rate too (bf16, 4 x 131072 rows: 286 us
//    of 287).  The page numbers of a tile are read while the tile before it is issued.
//  - Both products run on the warp-level MMA with the cached operand as A (16 rows or 16 features),
//    heads as the 8 columns: S[16 rows x 8 heads] = K Q^T, O^T[16 features x 8 heads] += V^T P^T.
//    A query group of one head to eight costs the same.  What bounds the kernel is the copy in 16 and 32 bits,
//    instruction issue and the ALU in 4 (52 % and 45 % on 64 x 1024..8192 rows).
//
// Number formats of the products:
//  - bf16, fp16: the stored values are the A operand; q is the B operand as it is (the scale is
//    applied to the fp32 score).  The probabilities are split into two 16-bit terms, p = hi + lo,
//    so that their rounding (2^-9 for bf16) does not add to the one rounding of the output.  fp16 ends at
//    2^-24, so there p is taken 2^11 times as large (2^15 at most): what many light rows lose beside a heavy one
//    is 2^-36 of the heavy one's weight each (2^-25 with p as it is: 4096 rows 17 nats lower were lost whole).
//  - fp32: both operands split into two tf32 terms, three products (hi*hi, hi*lo, lo*hi), short chains.
//  - 4 bits: a code c in 0..15 is used as the fp16 bit pattern c, the subnormal c * 2^-24: unpacking
//    is one AND for two codes (another for the codes four bits up, which come out 16 times as large);
//    V's bytes are used whole, c0 + 16 c1, beside c0 alone: four instructions for eight codes.
//    The score of a row is scale * (s * <q, c> + m * sum(q)) with the row's (s, m); in the weighted
//    sum the weight of a row is p * s, and sum(p * (m + 8 s)) is kept beside it.  q is brought to fp16 by a
//    power of two per head that puts its largest value at 2^13, whatever bf16 value that is (what is rounded off is 2^-38
//    of the largest value, 2^-34 in the features of the high codes, which take q / 16); the weights are brought into
//    fp16's range by a power of two that follows the largest s seen.  For fp16 outputs they are split into two terms, as
//    above (one rounding of 2^-12 each made the outputs 1.45 times as far off as their own rounding does); for bf16
//    outputs one term is an eighth of the output's rounding and does not show (1.67e-3 against 1.66e-3 in the 2-norm).
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "moa_device.cuh"
#include "moa_mma.cuh"

namespace moa {

struct PagedArgs {
    const unsigned char *k, *v;      // pools
    const uint32_t *kp, *vp;         // 4-bit rows: (scale, least) pairs, [num_pages][h_stored][page_size]
    long long k_sp, k_sh, k_sr;      // byte strides: page, kv head, row
    long long v_sp, v_sh, v_sr;
    int num_pages, page_size;
    uint32_t page_mul;               // row / page_size = row * page_mul >> page_sh, for rows below 2^31
    int page_sh;
    // A tile of 16 rows lies in one page (page_size a power of two, 16 at least), and these byte strides
    // (page and row; pairs of a page) fit 32 bits: the copies' addresses are two multiply-adds each.
    int one_page;
    uint32_t k_sp32, k_sr32, v_sp32, v_sr32, p_sp32;
    const int32_t *table;            // [batch, max_pages]
    int max_pages;
    const int32_t *seq_lens;         // [batch]
    int len_max;                     // min(max_pages * page_size, INT_MAX - 64)
    const void *q;
    void *out;
    long long q_sb;                  // elements between the queries of consecutive sequences
    int dtype;                       // of q and out (MOA_F32, MOA_BF16, MOA_F16)
    int batch, h_q, h_stored;
    int share;                       // virtual kv heads per stored one
    int g_s;                         // query heads per virtual kv head
    int g_total;                     // query heads per stored kv head
    float qscale;                    // scale * log2(e)
    float *ws;                       // two partial slots per CTA
    unsigned long long *tickets;     // for every CTA: counter of the pieces of the unit that is cut at its end
    unsigned long long ticket_tag;
};

// W warps, S ring stages of TT tiles of 16 rows (K and V) each.  The ring and the slots of the first cut unit
// share the 227 KB of an SM; the slot of the last cut unit is the ring itself, empty by then.
// TERMS: fp16 terms that a weight of a 4-bit row is held in: two for fp16 outputs, one for bf16.
template <int FMT_, int D_, int NT_, int W_, int S_, int TT_, int TERMS_ = 1>
struct PagedCfg {
    static constexpr int FMT = FMT_, D = D_, NT = NT_, W = W_, S = S_, TT = TT_, TERMS = TERMS_;
    static constexpr int THREADS = W * 32, R = 16 * TT;    // rows of a stage
    static constexpr int ROWB = FMT == MOA_KV_F32 ? 4 * D : FMT == MOA_KV_INT4 ? D / 2 : 2 * D;   // bytes of a row
    static constexpr int CPR = ROWB / 16;                  // 16-byte chunks of a row
    static constexpr int NCH = 16 * CPR / 32;              // chunks a lane copies per tile and operand
    static constexpr int KB = 16 * ROWB;                   // bytes of one operand's tile
    static constexpr int PB = FMT == MOA_KV_INT4 ? 128 : 0;    // bytes of a tile's (scale, least) pairs: 16 of K, 16 of V
    static constexpr int TILE = 2 * KB + PB;
    static constexpr int STAGE = TT * TILE;
    static constexpr int WHOLE = 4 * W;                    // stages of a unit that is not cut when there are few units
    static constexpr int MT = D / 16;                      // 16-feature output tiles
    static constexpr int G = 8 * NT;                       // heads of a unit
    static constexpr int PS = D + 4;                       // floats of a partial: o[D], m, l, 2 pad
    static constexpr int SLOT = G * PS;                    // floats of a unit's partial
    static constexpr int KSTEPS = FMT == MOA_KV_F32 ? D / 8 : D / 16;
    static constexpr int QREGS = FMT == MOA_KV_F32 ? 4 : 2;    // B registers per k-step (fp32: two terms)
    // How far (log2) a score may pass the reference maximum before that moves, and what the probabilities are taken
    // larger by: weights held in fp16 reach 2^15.  (4 bits have the factor in PagedState::inv.)
    static constexpr float AHEAD = FMT == MOA_KV_F16 || FMT == MOA_KV_INT4 ? 4.0f : 8.0f;
    static constexpr float SHIFT = FMT == MOA_KV_F16 ? 11.0f : 0.0f;
    static constexpr size_t OFF_FIRST = (size_t)W * S * STAGE;
    static constexpr size_t OFF_PREF = OFF_FIRST + sizeof(float) * (size_t)W * SLOT;
    static constexpr size_t SMEM_BYTES = OFF_PREF + sizeof(long long) * THREADS;
    static_assert(W <= 16, "two segments per warp have to fit a warp's lanes");
    static_assert((size_t)S * STAGE >= sizeof(float) * SLOT, "the ring holds the last partial");
    static_assert(OFF_FIRST % 16 == 0 && OFF_PREF % 16 == 0, "alignment of the regions");
    static_assert(SMEM_BYTES <= 227 * 1024 - 1280, "shared memory of an SM, less the static part");
};

__device__ __forceinline__ void cp16(uint32_t dst, const void *src, bool full)
{
    const int n = full ? 16 : 0;                           // 0: the 16 bytes are zero-filled, src is not read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void *src, bool full)
{
    const int n = full ? 4 : 0;
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
template <bool BF16>
__device__ __forceinline__ void mma_16x8x16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                            uint32_t b0, uint32_t b1)
{
    if (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Two floats as one register of 16-bit values (lo in the low half), and the values they were rounded to.
template <bool BF16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi)
{
    uint32_t r;
    if (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool BF16>
__device__ __forceinline__ float2 unpack16(uint32_t r)
{
    if (BF16) return make_float2(__uint_as_float(r << 16), __uint_as_float(r & 0xffff0000u));
    return __half22float2(*reinterpret_cast<const __half2 *>(&r));
}
__device__ __forceinline__ float4 lds4(uint32_t addr)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
// One element of a tensor of `dtype` as a float, and four floats into one.
__device__ __forceinline__ float load_as_float(const void *p, long long i, int dtype)
{
    if (dtype == MOA_F32) return static_cast<const float *>(p)[i];
    if (dtype == MOA_BF16) return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return __half2float(static_cast<const __half *>(p)[i]);
}
__device__ __forceinline__ void store4(void *p, long long i, const float4 &v, int dtype)
{
    if (dtype == MOA_F32) *reinterpret_cast<float4 *>(static_cast<float *>(p) + i) = v;
    else {
        const uint2 r = dtype == MOA_BF16 ? make_uint2(pack16<true>(v.x, v.y), pack16<true>(v.z, v.w))
                                          : make_uint2(pack16<false>(v.x, v.y), pack16<false>(v.z, v.w));
        *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + i) = r;
    }
}
__device__ __forceinline__ void store1(void *p, long long i, float v, int dtype)
{
    if (dtype == MOA_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == MOA_BF16) static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
    else static_cast<__half *>(p)[i] = __float2half_rn(v);
}

__device__ __forceinline__ int page_index(const PagedArgs &a, int row)
{
    return (int)(((unsigned long long)(unsigned)row * a.page_mul) >> a.page_sh);
}

__device__ __forceinline__ int paged_len(const PagedArgs &a, int b)       // 0: nothing to attend to
{
    const int len = a.seq_lens[b];
    return (len >= 1 && len <= a.len_max) ? len : 0;
}

// Query head that is head g of virtual kv head vh of sequence b; -1: padding (or no such sequence).
__device__ __forceinline__ int paged_query_head(const PagedArgs &a, int b, int vh, int g)
{
    const int in_stored = (vh % a.share) * a.g_s + g;
    return (g < a.g_s && in_stored < a.g_total && b < a.batch) ? (vh / a.share) * a.g_total + in_stored : -1;
}

// A place in the flat list: stage i of the ub stages (of R rows) of unit (b, h).
struct TileCursor {
    int b, h, i, ub, len;
};
template <int R>
__device__ __forceinline__ void next_unit(const PagedArgs &a, int hv, TileCursor &c)
{
    c.i = 0;
    if (++c.h < hv) return;
    c.h = 0;
    do {
        if (++c.b >= a.batch) { c.b = a.batch; c.len = 0; c.ub = 1; return; }
        c.len = paged_len(a, c.b);
    } while (c.len == 0);
    c.ub = (c.len + R - 1) / R;
}

// Place of a 16-byte chunk c of row r in the shared tile of K and of V: what keeps the reads free of
// bank conflicts.
template <class C>
__device__ __forceinline__ void chunk_place(int r, int c, uint32_t &kd, uint32_t &vd)
{
    if constexpr (C::FMT == MOA_KV_INT4) {
        kd = r * C::ROWB + c * 16;
        vd = r * C::ROWB + ((c ^ (C::D == 128 ? (r >> 1) & 3 : (r >> 2) & 1)) << 4);
    } else if constexpr (C::FMT == MOA_KV_F32) {
        kd = r * C::ROWB + ((c ^ ((r & 1) << 2)) << 4);
        vd = r * C::ROWB + ((c ^ ((r & 3) << 1)) << 4);
    } else {
        kd = vd = r * C::ROWB + ((c ^ (r & 7)) << 4);
    }
}

// Copies of one tile whose rows may lie in several pages, end behind the sequence (zero-filled), or
// have pages that do not exist (zero-filled, reported).  A row per lane (lanes 16..31 repeat): `page` is
// that of row row0 + lane % 16.  True: a page does not exist.
template <class C>
__device__ __forceinline__ bool copy_ragged_tile(const PagedArgs &a, uint32_t dst, int page, int hs, int row0, int len)
{
    const int lane = threadIdx.x & 31, row = row0 + (lane & 15);
    long long ko = -1, vo = 0, po = 0;
    bool bad = false;
    if (row < len) {
        const int off = row - page_index(a, row) * a.page_size;
        bad = page < 0 || page >= a.num_pages;
        if (!bad) {
            ko = page * a.k_sp + hs * a.k_sh + off * a.k_sr;
            vo = page * a.v_sp + hs * a.v_sh + off * a.v_sr;
            po = ((long long)page * a.h_stored + hs) * a.page_size + off;
        }
    }
    const int c = lane % C::CPR;
#pragma unroll
    for (int i = 0; i < C::NCH; ++i) {
        const int r = lane / C::CPR + i * (32 / C::CPR);
        const long long k1 = __shfl_sync(0xffffffffu, ko, r), v1 = __shfl_sync(0xffffffffu, vo, r);
        uint32_t kd, vd;
        chunk_place<C>(r, c, kd, vd);
        cp16(dst + kd, k1 >= 0 ? a.k + k1 + c * 16 : a.k, k1 >= 0);
        cp16(dst + C::KB + vd, k1 >= 0 ? a.v + v1 + c * 16 : a.v, k1 >= 0);
    }
    if constexpr (C::PB != 0) cp4(dst + 2 * C::KB + lane * 4, (lane < 16 ? a.kp : a.vp) + po, ko >= 0);
    const bool any = __any_sync(0xffffffffu, bad);
    if (any && lane == 0) raise_status(MOA_STATUS_PAGE_RANGE);
    return any;
}

// Registers of one warp's unit: accumulators of O^T, reference maxima, sums.
template <class C>
struct PagedState {
    float acc[C::NT][C::MT][4];
    // Heads 8n + 2t and 8n + 2t + 1.  msub: m - SHIFT, what probabilities and sums are relative to, or 0 while m is -inf
    float m[C::NT][2], msub[C::NT][2], l[C::NT][2];
    float om[C::NT][2];                                    // 4 bits: sum of p * (least + 8 scale)
    float ref, inv;                                        // 4 bits: power of two, at least every row's scale so far; 2048 / ref
};

// n * i / of, in 32 bits where that suffices.
__device__ __forceinline__ long long split_at(long long n, int i, int of)
{
    return n <= 0x003fffff ? (long long)((unsigned)n * (unsigned)i / (unsigned)of) : n * i / of;      // (i <= of <= 1024)
}
// The part that stage j lies in, of `of` parts of n stages.
__device__ __forceinline__ int part_of(long long n, long long j, int of)
{
    return n <= 0x003fffff ? (int)(((unsigned)(j + 1) * (unsigned)of - 1u) / (unsigned)n) : (int)(((j + 1) * of - 1) / n);
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) paged_decode_kernel(const __grid_constant__ PagedArgs a)
{
    constexpr int FMT = C::FMT, D = C::D, NT = C::NT, W = C::W, S = C::S, MT = C::MT, PS = C::PS, G = C::G, TT = C::TT, R = C::R;
    constexpr bool BF = FMT == MOA_KV_BF16, Q4 = FMT == MOA_KV_INT4, F32 = FMT == MOA_KV_F32;
    extern __shared__ __align__(128) unsigned char smem[];
    float *first_slots = reinterpret_cast<float *>(smem + C::OFF_FIRST);
    long long *s_pref = reinterpret_cast<long long *>(smem + C::OFF_PREF);
    __shared__ long long s_warp[16];
    __shared__ bool s_large[16];
    __shared__ long long s_seg[32];                        // unit of segment 2 * warp + (0: first, 1: last), or -1
    __shared__ long long s_seg_lo[32];                     // flat index of that unit's first stage
    __shared__ int s_seg_ub[32], s_seg_vh[32], s_seg_b[32];    // its stages, virtual kv head, sequence
    __shared__ int s_done[2];

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const int hv = a.h_stored * a.share;
    const int dtype = F32 ? MOA_F32 : FMT == MOA_KV_BF16 ? MOA_BF16 : FMT == MOA_KV_F16 ? MOA_F16 : a.dtype;

    launch_dependents();
    if (lane < 2) s_seg[2 * warp + lane] = -1;             // (read behind the barrier at the end)
    if (warp == 0 && lane >= 2 * W) s_seg[lane] = -1;
    // Into L2 while the kernel before this one ends: what the first copies depend on (lengths, page table,
    // queries).  A hint, no access: what that kernel still writes is read from L2 as it stands then.
    {
        const long long id = (long long)blockIdx.x * C::THREADS + tid, lens_n = (a.batch + 31) / 32,
                        table_n = ((long long)a.batch * a.max_pages + 31) / 32,
                        q_n = ((long long)(a.batch - 1) * a.q_sb + a.h_q * D) * (dtype == MOA_F32 ? 4 : 2) / 128;
        const unsigned char *p = nullptr;
        if (id < lens_n) p = reinterpret_cast<const unsigned char *>(a.seq_lens) + id * 128;
        else if (id < lens_n + q_n) p = static_cast<const unsigned char *>(a.q) + (id - lens_n) * 128;
        else if (id < lens_n + q_n + table_n) p = reinterpret_cast<const unsigned char *>(a.table) + (id - lens_n - q_n) * 128;
        if (p != nullptr) asm volatile("prefetch.global.L2 [%0];" ::"l"(p));
    }
    grid_dependency_wait();

    // ---- lengths: stages per sequence and their prefix ---------------------------------------
    // Up to 128 sequences every warp does this for itself, four to a lane; more go through shared
    // memory, a run of sequences to a thread.
    const bool few = a.batch <= 128;
    const int per_thread = few ? 4 : (a.batch + C::THREADS - 1) / C::THREADS;
    int ln[4];                                             // few: lengths of sequences 4 * lane..., 0 where out of range
    long long mine = 0;
    bool large = false;
    auto zero_out = [&](int b) {                           // a sequence without rows
        const long long row_bytes = (long long)a.h_q * D * (dtype == MOA_F32 ? 4 : 2);
        for (long long i = tid; i < row_bytes / 16; i += C::THREADS)
            reinterpret_cast<uint4 *>(static_cast<unsigned char *>(a.out) + (long long)b * row_bytes)[i] = make_uint4(0u, 0u, 0u, 0u);
    };
    if (few) {
        unsigned zero = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) ln[i] = 4 * lane + i < a.batch ? a.seq_lens[4 * lane + i] : -1;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = 4 * lane + i;
            const bool here = b < a.batch && (unsigned)b % gridDim.x == blockIdx.x;
            if (here && ln[i] == 0) zero |= 1u << i;
            if (ln[i] < 0 || ln[i] > a.len_max) {
                if (here && warp == 0) raise_status(MOA_STATUS_SEQLEN_RANGE);
                ln[i] = 0;
            }
            mine += (ln[i] + R - 1) / R;
            large |= ln[i] > C::WHOLE * R;
        }
        if (__any_sync(0xffffffffu, zero != 0)) {
#pragma unroll 1
            for (int b = 0; b < a.batch; ++b)
                if (__shfl_sync(0xffffffffu, zero, b >> 2) >> (b & 3) & 1u) zero_out(b);
        }
    } else {
        bool empty = false;
#pragma unroll 1
        for (int i = 0; i < per_thread; ++i) {
            const int b = tid * per_thread + i;
            if (b >= a.batch) break;
            const int len = a.seq_lens[b];
            const bool here = (unsigned)b % gridDim.x == blockIdx.x;
            if (len < 0 || len > a.len_max) { if (here) raise_status(MOA_STATUS_SEQLEN_RANGE); }
            else { mine += (len + R - 1) / R; empty |= len == 0 && here; large |= len > C::WHOLE * R; }
        }
        if (__syncthreads_or(empty)) {
            for (int b = blockIdx.x; b < a.batch; b += gridDim.x)
                if (a.seq_lens[b] == 0) zero_out(b);
        }
    }
    large = __any_sync(0xffffffffu, large);
    long long pre = mine;                                  // stages per head of the sequences before this lane's (this thread's)
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const long long x = __shfl_up_sync(0xffffffffu, pre, off);
        if (lane >= off) pre += x;
    }
    long long total = __shfl_sync(0xffffffffu, pre, 31);
    pre -= mine;
    if (!few) {
        if (lane == 0) { s_warp[warp] = total; s_large[warp] = large; }
        __syncthreads();
        total = 0;
#pragma unroll 1
        for (int w = 0; w < W; ++w) {
            if (w < warp) pre += s_warp[w];
            total += s_warp[w];
            large |= s_large[w];
        }
        s_pref[tid] = pre;
        __syncthreads();
    }
    total *= hv;

    // ---- this CTA's range [c0, c1) of the flat list, this warp's [j0, j1), and the unit it begins in --
    // Few and small units: one for each CTA, none is cut, the list is the unit's own.  Else a CTA takes at
    // least W stages: a cut costs a partial, a counter round trip and a merge, about 3 us.
    const bool whole = few && !large && (long long)a.batch * hv <= gridDim.x;
    const int active = total < (long long)W * gridDim.x ? (int)((unsigned)(total + W - 1) / W) : (int)gridDim.x;
    TileCursor cc;
    cc.b = cc.h = cc.i = cc.len = 0;
    cc.ub = 1;
    long long c0, c1, j0, j1, unit_lo = 0;                 // unit_lo: flat index of the current unit's first stage
    if (whole) {
        cc.b = blockIdx.x / hv; cc.h = blockIdx.x % hv;
        if (cc.b >= a.batch) return;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int x = __shfl_sync(0xffffffffu, ln[i], cc.b >> 2);
            if ((cc.b & 3) == i) cc.len = x;
        }
        if (cc.len == 0) return;
        cc.ub = (cc.len + R - 1) / R;
        c0 = 0; c1 = cc.ub;
        j0 = split_at(c1, warp, W); j1 = split_at(c1, warp + 1, W);
        cc.i = (int)j0;
    } else {
        if (blockIdx.x >= active) return;                  // (also when there is nothing to do)
        c0 = split_at(total, blockIdx.x, active); c1 = split_at(total, blockIdx.x + 1, active);
        j0 = c0 + split_at(c1 - c0, warp, W); j1 = c0 + split_at(c1 - c0, warp + 1, W);
        if (j0 < j1) {
            long long at;
            int b, len = 0, ub = 0;
            if (few) {
                const int from = 31 - __clz(__ballot_sync(0xffffffffu, mine > 0 && pre * hv <= j0));
                at = __shfl_sync(0xffffffffu, pre, from) * hv;
                b = 4 * from - 1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int x = __shfl_sync(0xffffffffu, ln[i], from);
                    if (j0 < at + (long long)ub * hv) continue;        // found
                    at += (long long)ub * hv;
                    ++b; len = x; ub = (x + R - 1) / R;
                }
            } else {
                int lo = 0, hi = C::THREADS;
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (s_pref[mid] * hv <= j0) lo = mid; else hi = mid;
                }
                at = s_pref[lo] * hv;
#pragma unroll 1
                for (b = lo * per_thread; b < a.batch; ++b) {          // ends before: j0 < total
                    len = paged_len(a, b);
                    ub = (len + R - 1) / R;
                    if (j0 < at + (long long)ub * hv) break;
                    at += (long long)ub * hv;
                }
            }
            if (b < a.batch && ub > 0) {                   // (else the lengths have changed meanwhile: no rows, no output)
                const long long in = j0 - at;
                cc.b = b; cc.len = len; cc.ub = ub;
                cc.h = in <= 0x7fffffff ? (int)((unsigned)in / (unsigned)ub) : (int)(in / ub);
                cc.i = (int)(in - (long long)cc.h * ub);
            } else cc.b = a.batch;
            unit_lo = j0 - cc.i;
        }
    }

    unsigned char *ring = smem + (size_t)warp * S * C::STAGE;
    const uint32_t smem_u = smem_u32(smem), ring_u = smem_u + warp * S * C::STAGE;

    if (j0 < j1) {
        TileCursor lc = cc;
        const int n = (int)(j1 - j0);                      // (2^31 stages of one warp would be 8e13 rows)
        int to_load = n, unit_left;                        // stages not issued yet, in all and of the unit under `lc`
        uint32_t load_at = ring_u;
        unsigned bad_stages = 0, load_bit = 1;
        // Of the unit under `lc`: its K/V head's part of the pools, its row of the table, and up to where
        // its rows go whole stages of whole pages at a time.
        const unsigned char *kh, *vh;
        const uint32_t *ph;                                // this lane's operand of the pairs
        const int32_t *trow;
        int hs, row0, fast_end, page[TT];
        auto load_unit = [&]() {
            hs = a.share == 1 ? lc.h : lc.h / a.share;
            kh = a.k + hs * a.k_sh + (lane / C::CPR) * a.k_sr + (lane % C::CPR) * 16;
            vh = a.v + hs * a.v_sh + (lane / C::CPR) * a.v_sr + (lane % C::CPR) * 16;
            if (Q4) ph = (lane < 16 ? a.kp : a.vp) + (long long)hs * a.page_size + (lane & 15);
            trow = a.table + (long long)lc.b * a.max_pages;
            row0 = lc.i * R;
            unit_left = lc.ub - lc.i;
            fast_end = a.one_page ? lc.len - (R - 1) : 0;
        };
        // Page numbers of the stage's tiles, one stage ahead of their copies: of the tile, or of the lane's row
        // where tiles go by row.
        auto fetch_pages = [&]() {
            if (row0 < fast_end) {
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) page[tt] = trow[page_index(a, row0 + 16 * tt)];
            } else {
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    const int row = row0 + 16 * tt + (lane & 15);
                    page[tt] = row < lc.len ? trow[page_index(a, row)] : -1;
                }
            }
        };
        load_unit();
        fetch_pages();
        uint32_t kd0, vd0;
        chunk_place<C>(lane / C::CPR, lane % C::CPR, kd0, vd0);

        auto issue = [&]() {                               // copies of the stage under `lc`, then on to the next
            bool fast = row0 < fast_end;
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) fast = fast && (unsigned)page[tt] < (unsigned)a.num_pages;
            bad_stages &= ~load_bit;
            if (fast) {
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) {
                    const uint32_t dst = load_at + tt * C::TILE, pg = page[tt], off = (row0 + 16 * tt) & (a.page_size - 1);
                    const unsigned char *kr = kh + (unsigned long long)pg * a.k_sp32 + (unsigned long long)off * a.k_sr32;
                    const unsigned char *vr = vh + (unsigned long long)pg * a.v_sp32 + (unsigned long long)off * a.v_sr32;
#pragma unroll
                    for (int i = 0; i < C::NCH; ++i) {
                        // the place of row r + i * (32 / CPR), from the place of row r: the swizzle's bits and the row's are apart
                        constexpr int RS = 32 / C::CPR;
                        const uint32_t kx = Q4 ? 0 : F32 ? ((i * RS) & 1) << 6 : ((i * RS) & 7) << 4;
                        const uint32_t vx = Q4 ? 0 : F32 ? ((i * RS) & 3) << 5 : ((i * RS) & 7) << 4;
                        cp16(dst + (kd0 ^ kx) + i * RS * C::ROWB, kr + (unsigned long long)(i * RS) * a.k_sr32);
                        cp16(dst + C::KB + (vd0 ^ vx) + i * RS * C::ROWB, vr + (unsigned long long)(i * RS) * a.v_sr32);
                    }
                    if (Q4) cp4(dst + 2 * C::KB + lane * 4, ph + ((unsigned long long)pg * a.p_sp32 + off));
                }
            } else {
                bool bad = false;
#pragma unroll 1
                for (int tt = 0; tt < TT; ++tt) {
                    int pg = page[0];                      // (of the lane's row: a stage with a missing page has its tiles' numbers, which serve)
#pragma unroll
                    for (int k = 1; k < TT; ++k) pg = tt == k ? page[k] : pg;
                    bad |= copy_ragged_tile<C>(a, load_at + tt * C::TILE, pg, hs, row0 + 16 * tt, lc.len);
                }
                if (bad) bad_stages |= load_bit;
            }
            load_at += C::STAGE; load_bit <<= 1;
            if (load_bit == 1u << S) { load_at = ring_u; load_bit = 1; }
            if (--to_load > 0) {
                row0 += R;
                if (--unit_left == 0) {
                    next_unit<R>(a, hv, lc);
                    load_unit();
                }
                fetch_pages();
            }
        };
#pragma unroll 1
        for (int i = 0; i < S; ++i) {
            if (to_load > 0) issue();
            cp_commit();
        }

        // ---- the unit's query and state ----------------------------------------------------
        uint32_t qf[NT][C::KSTEPS][C::QREGS];
        float fa[NT][2], fm[NT][2];                        // 4 bits: factors of <q, c> and of the least value
        PagedState<C> s;
        auto begin_unit = [&]() {
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int qh = paged_query_head(a, cc.b, cc.h, 8 * n + g);
                const long long base = (long long)cc.b * a.q_sb + (long long)qh * D;
                if constexpr (F32) {
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (qh >= 0) x = *reinterpret_cast<const float4 *>(static_cast<const float *>(a.q) + base + 4 * (t + 4 * i));
                        const Split4 sp = split4(x);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            qf[n][2 * i + e][0] = sp.h[2 * e]; qf[n][2 * i + e][1] = sp.h[2 * e + 1];
                            qf[n][2 * i + e][C::QREGS - 2] = sp.l[2 * e]; qf[n][2 * i + e][C::QREGS - 1] = sp.l[2 * e + 1];
                        }
                    }
                } else if constexpr (!Q4) {
                    const uint16_t *q = static_cast<const uint16_t *>(a.q) + base;
#pragma unroll
                    for (int i = 0; i < C::KSTEPS; ++i) {
                        qf[n][i][0] = qh >= 0 ? *reinterpret_cast<const uint32_t *>(q + 16 * i + 2 * t) : 0u;
                        qf[n][i][1] = qh >= 0 ? *reinterpret_cast<const uint32_t *>(q + 16 * i + 2 * t + 8) : 0u;
                    }
                } else {
                    // Lane t holds features [t * D/4, (t+1) * D/4) of head g, in the order of the codes' words.
                    uint4 raw[D / 32];
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
                        raw[i] = qh >= 0 ? *reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(a.q) + base + t * (D / 4) + 8 * i)
                                         : make_uint4(0u, 0u, 0u, 0u);
                    float most = 0.f;
                    auto pair = [&](uint32_t r) { return dtype == MOA_BF16 ? unpack16<true>(r) : unpack16<false>(r); };
#pragma unroll
                    for (int i = 0; i < D / 32; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 f = pair(reinterpret_cast<const uint32_t *>(&raw[i])[e]);
                            most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
                        }
#pragma unroll
                    for (int off = 1; off < 4; off <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
                    // largest magnitude into [2^13, 2^14), from 2^127 down to 2^-113; below, times 2^126
                    int e = 13 - ((int)((__float_as_uint(most) >> 23) & 255u) - 127);
                    e = e > 126 ? 126 : e < -114 ? -114 : e;
                    const float up = __uint_as_float((uint32_t)(127 + e) << 23), up16 = up * 0.0625f;
                    float sum = 0.f;                       // of q times that power, which overflows where the score does, not before
#pragma unroll
                    for (int i = 0; i < D / 32; ++i) {     // word i: features 8i.. of the lane's; pairs (0,4) (1,5), then (2,6) (3,7)
                        const float2 f01 = pair(raw[i].x), f23 = pair(raw[i].y), f45 = pair(raw[i].z), f67 = pair(raw[i].w);
                        qf[n][2 * i][0] = pack16<false>(f01.x * up, f45.x * up);
                        qf[n][2 * i][1] = pack16<false>(f01.y * up16, f45.y * up16);
                        qf[n][2 * i + 1][0] = pack16<false>(f23.x * up, f67.x * up);
                        qf[n][2 * i + 1][1] = pack16<false>(f23.y * up16, f67.y * up16);
                        sum += fmaf(f01.x, up, f01.y * up) + fmaf(f23.x, up, f23.y * up) + (fmaf(f45.x, up, f45.y * up) + fmaf(f67.x, up, f67.y * up));
                    }
#pragma unroll
                    for (int off = 1; off < 4; off <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                    const float down = __uint_as_float((uint32_t)(127 - e) << 23) * a.qscale;
                    sum *= down;
#pragma unroll
                    for (int e2 = 0; e2 < 2; ++e2) {       // of heads 8n + 2t + e2: held by lanes with g = 2t + e2
                        fa[n][e2] = __shfl_sync(0xffffffffu, down, (2 * t + e2) * 4);
                        fm[n][e2] = __shfl_sync(0xffffffffu, sum, (2 * t + e2) * 4);
                    }
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s.acc[n][i][e] = 0.f;
#pragma unroll
                for (int e = 0; e < 2; ++e) { s.m[n][e] = -INFINITY; s.msub[n][e] = 0.f; s.l[n][e] = 0.f; s.om[n][e] = 0.f; }
            }
            s.ref = 5.9604644775390625e-8f;                // 2^-24, fp16's least positive value
            s.inv = 34359738368.0f;
        };

        // ---- one tile: scores, probabilities, weighted sum ----------------------------------
        auto process = [&](uint32_t st, int nr, bool bad) {
            float x[TT][NT][4];
            float2 vpar[TT][2];                            // 4 bits: V's (scale, least) of this lane's two rows
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                const uint32_t sk = st + tt * C::TILE;
                const unsigned char *skp = smem + (sk - smem_u);
                if constexpr (F32) {
                    float lh[NT][4] = {}, hl[NT][4] = {};
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[tt][n][e] = 0.f;
#pragma unroll
                    for (int i4 = 0; i4 < D / 16; i4 += 2) {   // chains of four large products, added in fp32
                        float hh[NT][4] = {};
#pragma unroll
                        for (int i = i4; i < i4 + 2; ++i) {
                            const unsigned char *p = skp + g * C::ROWB + (((t + 4 * i) ^ ((g & 1) << 2)) << 4);
                            const Split4 s0 = split4(*reinterpret_cast<const float4 *>(p));
                            const Split4 s1 = split4(*reinterpret_cast<const float4 *>(p + 8 * C::ROWB));
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint32_t ah[4] = {s0.h[2 * e], s1.h[2 * e], s0.h[2 * e + 1], s1.h[2 * e + 1]};
                                const uint32_t al[4] = {s0.l[2 * e], s1.l[2 * e], s0.l[2 * e + 1], s1.l[2 * e + 1]};
#pragma unroll
                                for (int n = 0; n < NT; ++n)
                                    mma3(hh[n], lh[n], hl[n], ah, al, qf[n][2 * i + e][0], qf[n][2 * i + e][1],
                                         qf[n][2 * i + e][C::QREGS - 2], qf[n][2 * i + e][C::QREGS - 1]);
                            }
                        }
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int e = 0; e < 4; ++e) x[tt][n][e] += hh[n][e];
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[tt][n][e] = (x[tt][n][e] + (lh[n][e] + hl[n][e])) * a.qscale;
                } else if constexpr (!Q4) {
                    float c[2][NT][4] = {};                // two chains: half the products wait for one another
#pragma unroll
                    for (int i = 0; i < C::KSTEPS; ++i) {
                        uint32_t r[4];
                        ldsm4(r, sk + (lane & 15) * C::ROWB + (((2 * i + (lane >> 4)) ^ (lane & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NT; ++n) mma_16x8x16<BF>(c[i & 1][n], r[0], r[1], r[2], r[3], qf[n][i][0], qf[n][i][1]);
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[tt][n][e] = (c[0][n][e] + c[1][n][e]) * a.qscale;
                } else {
                    constexpr int NW = D / 32;
                    uint32_t w0[NW], w1[NW];
                    const unsigned char *p = skp + g * C::ROWB + t * (D / 8);
                    if constexpr (NW == 4) {
                        *reinterpret_cast<uint4 *>(w0) = *reinterpret_cast<const uint4 *>(p);
                        *reinterpret_cast<uint4 *>(w1) = *reinterpret_cast<const uint4 *>(p + 8 * C::ROWB);
                    } else {
                        *reinterpret_cast<uint2 *>(w0) = *reinterpret_cast<const uint2 *>(p);
                        *reinterpret_cast<uint2 *>(w1) = *reinterpret_cast<const uint2 *>(p + 8 * C::ROWB);
                    }
                    const __half2 *par = reinterpret_cast<const __half2 *>(skp + 2 * C::KB);
                    const float2 k0 = __half22float2(par[g]), k1 = __half22float2(par[g + 8]);
                    const float ks0 = k0.x * 16777216.0f, ks1 = k1.x * 16777216.0f;        // codes are c * 2^-24
                    vpar[tt][0] = __half22float2(par[16 + g]);
                    vpar[tt][1] = __half22float2(par[24 + g]);
                    float c[NT][4] = {};
#pragma unroll
                    for (int w = 0; w < NW; ++w)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint32_t u0 = e ? w0[w] >> 8 : w0[w], u1 = e ? w1[w] >> 8 : w1[w];
                            const uint32_t a0 = u0 & 0x000f000fu, a2 = u0 & 0x00f000f0u, a1 = u1 & 0x000f000fu, a3 = u1 & 0x00f000f0u;
#pragma unroll
                            for (int n = 0; n < NT; ++n) mma_16x8x16<false>(c[n], a0, a1, a2, a3, qf[n][2 * w + e][0], qf[n][2 * w + e][1]);
                        }
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            x[tt][n][e] = fmaf(ks0, c[n][e] * fa[n][e], k0.y * fm[n][e]);
                            x[tt][n][2 + e] = fmaf(ks1, c[n][2 + e] * fa[n][e], k1.y * fm[n][e]);
                        }
                }
            }
            if (nr < R) {                                  // rows behind the last one
#pragma unroll
                for (int tt = 0; tt < TT; ++tt)
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            if (16 * tt + g >= nr) x[tt][n][e] = -INFINITY;
                            if (16 * tt + g + 8 >= nr) x[tt][n][2 + e] = -INFINITY;
                        }
            }
            // The reference maximum moves only when a score exceeds it by more than 8 (a factor of 256; 4, a factor
            // of 16, where weights are fp16): rarely after the first tiles.
            float top[NT][2], vtop = 0.f;
            bool up = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    top[n][e] = fmaxf(x[0][n][e], x[0][n][2 + e]);
#pragma unroll
                    for (int tt = 1; tt < TT; ++tt) top[n][e] = fmaxf(top[n][e], fmaxf(x[tt][n][e], x[tt][n][2 + e]));
                    up |= top[n][e] > s.m[n][e] + C::AHEAD;
                }
            if constexpr (Q4) {
#pragma unroll
                for (int tt = 0; tt < TT; ++tt) vtop = fmaxf(vtop, fmaxf(vpar[tt][0].x, vpar[tt][1].x));
                up |= vtop > s.ref;
            }
            if (__any_sync(0xffffffffu, up)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float most = top[n][e];
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
                        const float m_new = fmaxf(s.m[n][e], most);
                        const float sub_new = m_new == -INFINITY ? 0.f : m_new - C::SHIFT;
                        const float alpha = s.m[n][e] == -INFINITY ? 0.f : fast_exp2(s.msub[n][e] - sub_new);
                        s.m[n][e] = m_new;
                        s.msub[n][e] = sub_new;
                        s.l[n][e] *= alpha;
                        if (Q4) s.om[n][e] *= alpha;
#pragma unroll
                        for (int i = 0; i < MT; ++i) { s.acc[n][i][e] *= alpha; s.acc[n][i][2 + e] *= alpha; }
                    }
                if constexpr (Q4) {
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) vtop = fmaxf(vtop, __shfl_xor_sync(0xffffffffu, vtop, off));
                    if (vtop > s.ref) {                    // next power of two (2^16 at most: scales are fp16)
                        const float r = __uint_as_float((__float_as_uint(vtop) + 0x7fffffu) & 0x7f800000u);
                        const float f = s.ref / r;
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int i = 0; i < MT; ++i)
#pragma unroll
                                for (int e = 0; e < 4; ++e) s.acc[n][i][e] *= f;
                        s.ref = r;
                        s.inv = 2048.0f / r;               // exact: weights reach 2^15 at most
                    }
                }
            }
            if (bad) {                                     // a row whose page does not exist: the unit's result is NaN
#pragma unroll
                for (int n = 0; n < NT; ++n) s.l[n][0] = s.l[n][1] = __int_as_float(0x7fffffff);
            }
            uint32_t wt[TT][NT][2], wl[TT][NT][2];         // 4 bits: weights p * s as B operand, and their second terms
            uint32_t hi[TT][NT][2], lo[TT][NT][2];         // 16 bits: weights p in two terms as B operand
            float ls[NT][2];                               // 16 and 32 bits: the lane's probabilities of the stage, added up before they join
                                                           // the unit's (4 bits: one by one, 78 us instead of 79 on 64 x 1024..8192 rows)
#pragma unroll
            for (int tt = 0; tt < TT; ++tt) {
                const uint32_t sv = st + tt * C::TILE + C::KB;
                const unsigned char *svp = smem + (sv - smem_u);
                float p[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) p[n][e] = fast_exp2(x[tt][n][e] - s.msub[n][e & 1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (Q4) s.l[n][e] = (s.l[n][e] + p[n][e]) + p[n][2 + e];
                        else ls[n][e] = tt == 0 ? p[n][e] + p[n][2 + e] : ls[n][e] + (p[n][e] + p[n][2 + e]);
                    }
                }
                if constexpr (F32) {
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        // P^T as B operand: row t (+4) of each 8-row half, head g
                        uint32_t bh[4], bl[4];             // rows t, t+4, 8+t, 12+t
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            const int src = (t + (h & 1) * 4) * 4 + (g >> 1);
                            const float y0 = __shfl_sync(0xffffffffu, p[n][(h >> 1) * 2], src);
                            const float y1 = __shfl_sync(0xffffffffu, p[n][(h >> 1) * 2 + 1], src);
                            const float y = (g & 1) ? y1 : y0;
                            bh[h] = (__float_as_uint(y) + 0x1000u) & 0xFFFFE000u;
                            bl[h] = (__float_as_uint(y - __uint_as_float(bh[h])) + 0x1000u) & 0xFFFFE000u;
                        }
#pragma unroll
                        for (int i = 0; i < D / 32; ++i) {
                            Split4 v[2][2];
#pragma unroll
                            for (int h = 0; h < 4; ++h) {
                                const int r = t + (h & 1) * 4 + (h >> 1) * 8;
                                v[h >> 1][h & 1] = split4(*reinterpret_cast<const float4 *>(svp + r * C::ROWB + (((g + 8 * i) ^ ((r & 3) << 1)) << 4)));
                            }
#pragma unroll
                            for (int e = 0; e < 2; ++e) {  // output tile 2i + e: features 4(g + 8i) + 2e, + 1
                                float hh[4] = {}, lh[4] = {}, hl[4] = {};
#pragma unroll
                                for (int k = 0; k < 2; ++k) {
                                    const uint32_t ah[4] = {v[k][0].h[2 * e], v[k][0].h[2 * e + 1], v[k][1].h[2 * e], v[k][1].h[2 * e + 1]};
                                    const uint32_t al[4] = {v[k][0].l[2 * e], v[k][0].l[2 * e + 1], v[k][1].l[2 * e], v[k][1].l[2 * e + 1]};
                                    mma3(hh, lh, hl, ah, al, bh[2 * k], bh[2 * k + 1], bl[2 * k], bl[2 * k + 1]);
                                }
#pragma unroll
                                for (int z = 0; z < 4; ++z) s.acc[n][2 * i + e][z] += hh[z] + (lh[z] + hl[z]);
                            }
                        }
                    }
                } else if constexpr (!Q4) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t r = pack16<BF>(p[n][2 * h], p[n][2 * h + 1]);
                            const float2 f = unpack16<BF>(r);
                            hi[tt][n][h] = movmatrix_trans(r);
                            lo[tt][n][h] = movmatrix_trans(pack16<BF>(p[n][2 * h] - f.x, p[n][2 * h + 1] - f.y));
                        }
                } else {
                    const float s0 = vpar[tt][0].x * s.inv, s1 = vpar[tt][1].x * s.inv;
                    const float mid0 = fmaf(8.f, vpar[tt][0].x, vpar[tt][0].y), mid1 = fmaf(8.f, vpar[tt][1].x, vpar[tt][1].y);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float w0 = p[n][2 * h] * (h ? s1 : s0), w1 = p[n][2 * h + 1] * (h ? s1 : s0);
                            const uint32_t r = pack16<false>(w0, w1);
                            wt[tt][n][h] = movmatrix_trans(r);
                            if constexpr (C::TERMS == 2) {
                                const float2 f = unpack16<false>(r);
                                wl[tt][n][h] = movmatrix_trans(pack16<false>(w0 - f.x, w1 - f.y));
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 2; ++e) s.om[n][e] = fmaf(p[n][e], mid0, fmaf(p[n][2 + e], mid1, s.om[n][e]));
                    }
                }
            }
            if constexpr (!Q4) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) s.l[n][e] += ls[n][e];
            }
            // A stage's sum joins the unit's, in fp32.
            auto add_sum = [&](float (&to)[4], const float (&sum)[4]) {
#pragma unroll
                for (int z = 0; z < 4; z += 2) {
                    const uint64_t y = add2(pack2(__float_as_uint(to[z]), __float_as_uint(to[z + 1])),
                                            pack2(__float_as_uint(sum[z]), __float_as_uint(sum[z + 1])));
                    uint32_t y0, y1;
                    unpack2(y, y0, y1);
                    to[z] = __uint_as_float(y0);
                    to[z + 1] = __uint_as_float(y1);
                }
            };
            if constexpr (!F32 && !Q4) {
                // Weighted sum of the stage's rows, from zero, then added to the unit's in fp32: the MMA's accumulation
                // cuts off instead of rounding, and in one chain over 131072 rows of one sign that took 7e-4 off the sum.
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    float sum[NT][4] = {};
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) {
                        uint32_t r[4];
                        const int row = (lane & 7) + ((lane >> 4) << 3);
                        ldsm4t(r, st + tt * C::TILE + C::KB + row * C::ROWB + (((2 * i + ((lane >> 3) & 1)) ^ (row & 7)) << 4));
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            mma_16x8x16<BF>(sum[n], r[0], r[1], r[2], r[3], lo[tt][n][0], lo[tt][n][1]);
                            mma_16x8x16<BF>(sum[n], r[0], r[1], r[2], r[3], hi[tt][n][0], hi[tt][n][1]);
                        }
                    }
#pragma unroll
                    for (int n = 0; n < NT; ++n) add_sum(s.acc[n][i], sum[n]);
                }
            }
            if constexpr (Q4) {
                // Weighted sum of the stage's codes, from zero, then added to the unit's in fp32.  The sums are of c - 8:
                // with codes from 0 they would carry 7.5 steps of every row, which over 1e5 rows are 500 times
                // the result, and the rounding of the accumulation and of the weights would act on them (fp16 outputs at
                // 131072 rows, whose own rounding is 2.1e-4, are 2.4e-4 off the definition; with weights of one term 3.0e-4,
                // and with codes from 0 as well 7.4e-4).
                // What is to be taken off, 8 * sum of the rounded weights, comes as a product of its own with a
                // constant operand, which the sums start from.  Low features of a byte: its low code; the rows of
                // the high ones hold c0 + 16 c1 (so 136 comes off), taken apart at the end of the unit.
                float off[NT][4];
#pragma unroll
                for (int n = 0; n < NT; ++n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) off[n][e] = 0.f;
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt) {
                        if (C::TERMS == 2) mma_16x8x16<false>(off[n], 0x80088008u, 0x80888088u, 0x80088008u, 0x80888088u, wl[tt][n][0], wl[tt][n][1]);
                        mma_16x8x16<false>(off[n], 0x80088008u, 0x80888088u, 0x80088008u, 0x80888088u, wt[tt][n][0], wt[tt][n][1]);
                    }
                }
#pragma unroll
                for (int j = 0; j < D / 64; ++j) {
                    // A transposed load hands a lane the 16-bit units (four codes) of two neighbouring rows in one
                    // register: columns 16j.. of units, rows 0-7, 8-15; columns 16j + 8..: the same.
                    uint32_t r[TT][4];
                    const int row = (lane & 7) + (((lane >> 3) & 1) << 3), ch = 2 * j + (lane >> 4);
#pragma unroll
                    for (int tt = 0; tt < TT; ++tt)
                        ldsm4t(r[tt], st + tt * C::TILE + C::KB + row * C::ROWB + ((ch ^ (D == 128 ? (row >> 1) & 3 : (row >> 2) & 1)) << 4));
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {      // output tile 4j + 2i + e: features 4(8(2j + i) + g) + 2e, + 1
                            float sum[NT][4];
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int z = 0; z < 4; ++z) sum[n][z] = off[n][z];
#pragma unroll
                            for (int tt = 0; tt < TT; ++tt) {
                                const uint32_t a1 = e ? __byte_perm(r[tt][2 * i], 0u, 0x4341) : r[tt][2 * i] & 0x00ff00ffu;
                                const uint32_t a3 = e ? __byte_perm(r[tt][2 * i + 1], 0u, 0x4341) : r[tt][2 * i + 1] & 0x00ff00ffu;
#pragma unroll
                                for (int n = 0; n < NT; ++n) {
                                    if (C::TERMS == 2) mma_16x8x16<false>(sum[n], a1 & 0x000f000fu, a1, a3 & 0x000f000fu, a3, wl[tt][n][0], wl[tt][n][1]);
                                    mma_16x8x16<false>(sum[n], a1 & 0x000f000fu, a1, a3 & 0x000f000fu, a3, wt[tt][n][0], wt[tt][n][1]);
                                }
                            }
                            const int to = 4 * j + 2 * i + e;
#pragma unroll
                            for (int n = 0; n < NT; ++n) add_sum(s.acc[n][to], sum[n]);
                        }
                }
            }
        };

        // ---- end of a unit, or of this warp's part of it ------------------------------------
        // Feature of accumulator (i, half h): 16-bit: 16i + 8h + g; fp32 and 4 bits: 4(g + 8(i/2)) + 2(i%2) + h.  dst: a partial slot, or null for the output row.
        auto close = [&](float *dst) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float l = s.l[n][e], om = s.om[n][e];
#pragma unroll
                    for (int off = 4; off < 32; off <<= 1) {
                        l += __shfl_xor_sync(0xffffffffu, l, off);
                        if (Q4) om += __shfl_xor_sync(0xffffffffu, om, off);
                    }
                    const int head = 8 * n + 2 * t + e;
                    float f0 = 1.f, f1 = 1.f, add = 0.f;   // of even and of odd features
                    if (Q4) { f0 = s.ref * 8192.0f; f1 = s.ref * 512.0f; add = om; }         // 2^24 / 2048, and a 16th
                    long long at = -1;
                    if (dst != nullptr) {
                        if (g == 0) { dst[head * PS + D] = s.m[n][e] == -INFINITY ? -INFINITY : s.msub[n][e]; dst[head * PS + D + 1] = l; }
                    } else {
                        const int qh = paged_query_head(a, cc.b, cc.h, head);
                        if (qh >= 0) at = ((long long)cc.b * a.h_q + qh) * D;
                        const float inv = 1.0f / l;
                        f0 *= inv; f1 *= inv; add *= inv;
                    }
                    auto val = [&](int i, int h) {
                        return fmaf(Q4 && h ? s.acc[n][i][2 + e] - s.acc[n][i][e] : s.acc[n][i][2 * h + e], h ? f1 : f0, add);
                    };
                    if (Q4 || F32) {
#pragma unroll
                        for (int i = 0; i < MT; i += 2) {
                            const float4 v4 = make_float4(val(i, 0), val(i, 1), val(i + 1, 0), val(i + 1, 1));
                            const int d = 4 * (g + 4 * i);
                            if (dst != nullptr) *reinterpret_cast<float4 *>(dst + head * PS + d) = v4;
                            else if (at >= 0) store4(a.out, at + d, v4, dtype);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < MT; ++i)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const int d = 16 * i + 8 * h + g;
                                if (dst != nullptr) dst[head * PS + d] = val(i, h);
                                else if (at >= 0) store1(a.out, at + d, val(i, h), dtype);
                            }
                    }
                }
        };

        uint32_t stage_at = ring_u;
        unsigned stage_bit = 1;
#pragma unroll 1
        for (int left = n;;) {                             // unit by unit
            begin_unit();
            const int here = min(cc.ub - cc.i, left);
            int nr = cc.len - cc.i * R;                    // rows from this stage on
#pragma unroll 1
            for (int k = 0; k < here; ++k, nr -= R) {
                cp_wait<S - 1>();
                __syncwarp();
                process(stage_at, nr, (bad_stages & stage_bit) != 0);
                __syncwarp();                              // every lane is done with the stage
                stage_at += C::STAGE; stage_bit <<= 1;
                if (stage_bit == 1u << S) { stage_at = ring_u; stage_bit = 1; }
                if (to_load > 0) issue();
                cp_commit();
            }
            left -= here;
            const bool unit_ends = cc.i + here == cc.ub;
            float *dst = nullptr;                          // the whole unit: the output; else a partial
            if (!unit_ends || unit_lo < j0) {
                const int which = left == 0 ? 1 : 0;       // a cut unit that ends before the range does is its first
                if (which) { cp_wait<0>(); __syncwarp(); }
                dst = which ? reinterpret_cast<float *>(ring) : first_slots + (size_t)warp * C::SLOT;
                if (lane == 0) {
                    const int sg = 2 * warp + which;
                    s_seg[sg] = (long long)cc.b * hv + cc.h;
                    s_seg_lo[sg] = unit_lo; s_seg_ub[sg] = cc.ub; s_seg_vh[sg] = cc.h; s_seg_b[sg] = cc.b;
                }
            }
            close(dst);
            if (left == 0) break;
            unit_lo += cc.ub;
            next_unit<R>(a, hv, cc);
        }
    }
    __syncthreads();

    // ---- join the pieces of units that this CTA's warps share -------------------------------
    // Every warp works out the groups of segments for itself, a segment to a lane: one leads a group
    // when the valid segment before it belongs to another unit.  Then a warp takes a head (or two): the
    // segments' factors by shuffles, the features by its lanes.
    const long long u = s_seg[lane];
    const unsigned valid = __ballot_sync(0xffffffffu, u >= 0);
    if (valid == 0) return;                                // uniform for the CTA: nothing was cut
    const unsigned below = valid & ((1u << lane) - 1u);
    const long long pu = __shfl_sync(0xffffffffu, u, below ? 31 - __clz(below) : lane);
    const unsigned leaders = __ballot_sync(0xffffffffu, u >= 0 && (below == 0 || pu != u));
    const unsigned upto = leaders & (0xffffffffu >> (31 - lane)), after = lane < 31 ? leaders >> (lane + 1) : 0u;
    const int my_lead = upto ? 31 - __clz(upto) : 0, my_end = after ? lane + __ffs(after) - 1 : 31;
    auto members = [&](int lead) -> unsigned {             // segments of the group that segment `lead` leads
        const unsigned next = lead < 31 ? leaders >> (lead + 1) : 0u;
        return valid & (next ? (1u << (lead + __ffs(next))) - (1u << lead) : 0u - (1u << lead));
    };
    auto seg_slot = [&](int sg) -> uint32_t {              // shared address of its partial
        return smem_u + ((sg & 1) ? (sg >> 1) * (S * C::STAGE) : (int)C::OFF_FIRST + (sg >> 1) * (C::SLOT * 4));
    };
    constexpr int LPR = D / 4, HPW = (G + W - 1) / W;
    const int d = (lane % LPR) * 4;
    float f[HPW], M[HPW], L[HPW];                          // of this lane's segment; M and L of its group
#pragma unroll
    for (int k = 0; k < HPW; ++k) {
        const int head = warp + k * W;
        float m = -INFINITY, l = 0.f;
        if ((valid >> lane & 1u) && head < G) {
            const float4 ml = lds4(seg_slot(lane) + (head * PS + D) * 4);
            m = ml.x; l = ml.y;
        }
        M[k] = m;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const float x = __shfl_up_sync(0xffffffffu, M[k], off);
            if (lane - off >= my_lead) M[k] = fmaxf(M[k], x);
        }
        M[k] = __shfl_sync(0xffffffffu, M[k], my_end);
        f[k] = exp2_diff(m, M[k]);
        L[k] = f[k] * l;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const float x = __shfl_up_sync(0xffffffffu, L[k], off);
            if (lane - off >= my_lead) L[k] += x;
        }
        L[k] = __shfl_sync(0xffffffffu, L[k], my_end);
    }
    auto join = [&](int lead, int head, float fk) {        // this lane's four features of a group's sum
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (unsigned r = members(lead); r != 0;) {        // four under way at once (the last one again, unused, where there are fewer)
            float4 y[4];
            float x[4];
            int sg = 0;
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                const bool on = r != 0;
                sg = on ? __ffs(r) - 1 : sg;
                x[z] = __shfl_sync(0xffffffffu, fk, sg);
                if (!on) x[z] = 0.f;
                y[z] = lds4(seg_slot(sg) + (head * PS + d) * 4);
                if (!on) y[z] = make_float4(0.f, 0.f, 0.f, 0.f);
                r &= r - 1;
            }
#pragma unroll
            for (int z = 0; z < 4; ++z) {
                o.x = fmaf(x[z], y[z].x, o.x); o.y = fmaf(x[z], y[z].y, o.y); o.z = fmaf(x[z], y[z].z, o.z); o.w = fmaf(x[z], y[z].w, o.w);
            }
        }
        return o;
    };
    auto emit = [&](int b, int vh, int head, const float4 &o, float sum) {
        const int qh = paged_query_head(a, b, vh, head);
        const float inv = 1.0f / sum;
        if (qh >= 0 && lane < LPR)
            store4(a.out, ((long long)b * a.h_q + qh) * D + d, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv), dtype);
    };
    // Units cut between CTAs first (the first group, the last, or both): their partials leave and are
    // counted while the whole units are joined.  One release and one count per CTA and cut unit: fences of
    // several warps of an SM wait for one another.
    int lead_of[2] = {__ffs(leaders) - 1, 31 - __clz(leaders)}, first[2], last[2];
    bool cut[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int lead = lead_of[i];
        const long long lo = s_seg_lo[lead], hi = lo + s_seg_ub[lead];
        cut[i] = !whole && (lo < c0 || hi > c1) && (i == 0 || lead != lead_of[0]);
        first[i] = last[i] = 0;
        if (cut[i]) { first[i] = part_of(total, lo, active); last[i] = part_of(total, hi - 1, active); }
    }
    const bool any_cut = cut[0] || cut[1];
    if (any_cut) {
#pragma unroll
        for (int k = 0; k < HPW; ++k) {
            const int head = warp + k * W;
            if (head >= G) break;
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
                if (!(i ? cut[1] : cut[0])) continue;
                const int lead = i ? lead_of[1] : lead_of[0];
                float *p = a.ws + ((size_t)blockIdx.x * 2 + (s_seg_lo[lead] <= c0 ? 0 : 1)) * C::SLOT + head * PS;
                const float4 o = join(lead, head, f[k]);
                const float m = __shfl_sync(0xffffffffu, M[k], lead), l = __shfl_sync(0xffffffffu, L[k], lead);
                if (lane < LPR) *reinterpret_cast<float4 *>(p + d) = o;
                if (lane == 0) *reinterpret_cast<float2 *>(p + D) = make_float2(m, l);
            }
        }
        __syncthreads();
        if (tid < 2) {
            int done = 0;
            if (tid ? cut[1] : cut[0]) {
                unsigned long long *word = a.tickets + (tid ? first[1] : first[0]);
                asm volatile("fence.acq_rel.gpu;" ::: "memory");
                done = ticket_arrive(word, a.ticket_tag) == (unsigned)(tid ? last[1] - first[1] : last[0] - first[0]);
                if (done) {
                    *word = 0ull;
                    asm volatile("fence.acq_rel.gpu;" ::: "memory");
                }
            }
            s_done[tid] = done;
        }
    }
#pragma unroll 1
    for (unsigned r = leaders; r != 0; r &= r - 1) {
        const int lead = __ffs(r) - 1;
        if ((cut[0] && lead == lead_of[0]) || (cut[1] && lead == lead_of[1])) continue;
#pragma unroll
        for (int k = 0; k < HPW; ++k) {
            const int head = warp + k * W;
            if (head < G) emit(s_seg_b[lead], s_seg_vh[lead], head, join(lead, head, f[k]), __shfl_sync(0xffffffffu, L[k], lead));
        }
    }
    if (!any_cut) return;

    // ---- units cut between CTAs: the CTA that delivers the last piece joins them, in CTA order --------
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < 2; ++i) {
        if (!s_done[i]) continue;
        const int lead = i ? lead_of[1] : lead_of[0], c_first = i ? first[1] : first[0], c_last = i ? last[1] : last[0];
        const int slot0 = s_seg_lo[lead] == split_at(total, c_first, active) ? 0 : 1;      // a CTA's slot 0: the unit that its range begins in
        float top[HPW], sum[HPW], x[HPW];
        float4 o[HPW], oc[HPW];
#pragma unroll
        for (int k = 0; k < HPW; ++k) { top[k] = -INFINITY; sum[k] = 0.f; o[k] = oc[k] = make_float4(0.f, 0.f, 0.f, 0.f); }
#pragma unroll 1
        for (int c = c_first; c <= c_last; c += 32) {      // 32 partials' factors at once, one to a lane
            const int n = min(32, c_last - c + 1);
            auto part = [&](int z, int k) {                // partial of CTA c + z for this warp's head k
                return a.ws + ((size_t)(c + z) * 2 + (c + z > c_first ? 0 : slot0)) * C::SLOT + min(warp + k * W, G - 1) * PS;
            };
            constexpr int B = 8;                           // rows of a head under way at once, the first beside the factors
            float4 y[HPW][B];
            float2 ml[HPW];
            auto fetch = [&](int z0) {
#pragma unroll
                for (int k = 0; k < HPW; ++k)
#pragma unroll
                    for (int z = 0; z < B; ++z)
                        if (z0 + z < n) y[k][z] = __ldcg(reinterpret_cast<const float4 *>(part(z0 + z, k) + d));
            };
#pragma unroll
            for (int k = 0; k < HPW; ++k) ml[k] = __ldcg(reinterpret_cast<const float2 *>(part(min(lane, n - 1), k) + D));
            fetch(0);
#pragma unroll
            for (int k = 0; k < HPW; ++k) {
                if (lane >= n) ml[k] = make_float2(-INFINITY, 0.f);
                float top_new = fmaxf(top[k], ml[k].x);
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) top_new = fmaxf(top_new, __shfl_xor_sync(0xffffffffu, top_new, off));
                const float keep = exp2_diff(top[k], top_new);
                x[k] = exp2_diff(ml[k].x, top_new);
                float add = x[k] * ml[k].y;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) add += __shfl_xor_sync(0xffffffffu, add, off);
                sum[k] = fmaf(sum[k], keep, add);
                o[k].x *= keep; o[k].y *= keep; o[k].z *= keep; o[k].w *= keep;
                oc[k].x *= keep; oc[k].y *= keep; oc[k].z *= keep; oc[k].w *= keep;
                top[k] = top_new;
            }
#pragma unroll 1
            for (int z0 = 0; z0 < n; z0 += B) {
                if (z0 > 0) fetch(z0);
#pragma unroll
                for (int k = 0; k < HPW; ++k)
#pragma unroll
                    for (int z = 0; z < B; ++z)
                        if (z0 + z < n) comp_fma4(o[k], oc[k], y[k][z], __shfl_sync(0xffffffffu, x[k], z0 + z));
            }
        }
#pragma unroll
        for (int k = 0; k < HPW; ++k)
            if (warp + k * W < G) emit(s_seg_b[lead], s_seg_vh[lead], warp + k * W, o[k], sum[k]);
    }
}

}  // namespace moa
