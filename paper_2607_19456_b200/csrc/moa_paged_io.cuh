// moa_paged_io.cuh -- writing and reading the rows of a paged cache: the append, with the position
// rotation of queries and keys on the way, and the read-back into dense rows.
//
// Both are bound by memory.  A row (one head of one token) belongs to D/16 neighbouring threads of a
// warp, 16 features each, as two chunks of 8 (16 bytes in 16-bit types): under the rotation of
// halves the two chunks are each other's partners, so no value crosses threads.  A thread takes
// several heads of its token, all of q, all of k or all of v, in turn: the token's sequence, page,
// cosines and sines are found once, and the next row is under way while one is turned.
//
// Every product, sum and quotient below is rounded on its own (no contraction into fused
// multiply-adds): what a row holds is then defined by the formulas alone, and equals what any
// other IEEE evaluation of them gives, which matters where a value lies next to a border between
// two 4-bit codes.
#pragma once

#include "moa_paged.cuh"

namespace moa {

struct PagedIoArgs {
    unsigned char *k_pool, *v_pool;
    uint32_t *kp, *vp;
    long long k_sp, k_sh, k_sr;      // byte strides of the pools: page, kv head, row
    long long v_sp, v_sh, v_sr;
    int num_pages, page_size, page_shift, h_kv;
    const int32_t *table;
    int max_pages, batch;
    const int32_t *seq_lens;
    // append
    const void *q, *k, *v;
    void *q_out;
    long long q_st, k_st, v_st, o_st;    // elements between consecutive tokens
    int tokens, h_q;
    int run, q_runs, kv_runs;        // heads that a thread takes; runs of them in q, and in k (as many in v)
    const int32_t *token_start;      // [batch + 1], or null: token t belongs to sequence t
    const float *cos_sin;            // [rope_rows, rot]: rot/2 cosines, rot/2 sines
    int rope_rows, rot;
    int pairs;                       // features (2i, 2i+1) turn together; else (i, rot/2 + i)
    // read-back
    void *k_out, *v_out;
    const int32_t *row_start;
    int n_out;
};

// Eight consecutive elements of a row as floats, and back.
template <int DT>
__device__ __forceinline__ void load8(float (&x)[8], const void *p)
{
    if constexpr (DT == MOA_F32) {
        const float4 u = static_cast<const float4 *>(p)[0], w = static_cast<const float4 *>(p)[1];
        x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = w.x; x[5] = w.y; x[6] = w.z; x[7] = w.w;
    } else {
        const uint4 u = *static_cast<const uint4 *>(p);
        const uint32_t r[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack16<DT == MOA_BF16>(r[i]);
            x[2 * i] = f.x; x[2 * i + 1] = f.y;
        }
    }
}
template <int DT>
__device__ __forceinline__ void store8(void *p, const float (&x)[8])
{
    if constexpr (DT == MOA_F32) {
        static_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
        static_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        constexpr bool BF = DT == MOA_BF16;
        *static_cast<uint4 *>(p) = make_uint4(pack16<BF>(x[0], x[1]), pack16<BF>(x[2], x[3]), pack16<BF>(x[4], x[5]),
                                              pack16<BF>(x[6], x[7]));
    }
}

// (x, y) turned by the angle whose cosine and sine are c and s.
__device__ __forceinline__ void turn(float &x, float &y, float c, float s)
{
    const float u = __fsub_rn(__fmul_rn(x, c), __fmul_rn(y, s));
    y = __fadd_rn(__fmul_rn(y, c), __fmul_rn(x, s));
    x = u;
}

// A row in 4 bits: s = fp16((max - min) / 15), m = fp16(min), code = round((x - m) / s) in 0..15.
// The quotient by 15 is a product with fp32's nearest to 1/15.  Rows beyond fp16's range are held
// as if cut off there; a row with a value that is no number or infinite reads back as NaN.
// lo, hi: this thread's two chunks; the D/16 threads of a row are neighbours, `mask` their lanes.
template <int D>
__device__ __forceinline__ void pack_row(const float (&lo)[8], const float (&hi)[8], uint32_t &c_lo, uint32_t &c_hi,
                                         uint32_t &params, unsigned mask)
{
    float mn = lo[0], mx = lo[0];
    bool odd = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        mn = fminf(mn, fminf(lo[i], hi[i]));
        mx = fmaxf(mx, fmaxf(lo[i], hi[i]));
        odd |= !isfinite(lo[i]) || !isfinite(hi[i]);
    }
    int bad = odd;
#pragma unroll
    for (int off = 1; off < D / 16; off <<= 1) {
        mn = fminf(mn, __shfl_xor_sync(mask, mn, off));
        mx = fmaxf(mx, __shfl_xor_sync(mask, mx, off));
        bad |= __shfl_xor_sync(mask, bad, off);
    }
    const float top = 65504.0f;
    const __half s16 = __float2half_rn(fminf(__fmul_rn(__fsub_rn(mx, mn), 1.0f / 15.0f), top));
    const __half m16 = __float2half_rn(fminf(fmaxf(mn, -top), top));
    const float s = __half2float(s16), m = __half2float(m16);
    c_lo = c_hi = 0u;
    if (bad) { params = 0x7fff7fffu; return; }
    if (s > 0.f) {
        // round((x - m) / s): with the reciprocal, which is within 2^-22 of the quotient's 15 at most; a thread
        // that comes nearer than 2^-16 to a border between two codes divides.
        const float r = __frcp_rn(s);
        float c[16];
        bool near = false;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = i < 8 ? lo[i] : hi[i - 8];
            const float q = fminf(fmaxf(__fmul_rn(__fsub_rn(x, m), r), 0.f), 15.f);
            c[i] = rintf(q);
            near |= fabsf(q - c[i]) > 0.5f - 1.0f / 65536.0f;
        }
        if (near) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x = i < 8 ? lo[i] : hi[i - 8];
                c[i] = fminf(fmaxf(rintf(__fdiv_rn(__fsub_rn(x, m), s)), 0.f), 15.f);
            }
        }
        // Four codes make an exact number below 2^16, whose bits a float of 2^23 more shows.
        uint32_t h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            h[i] = __float_as_uint(fmaf(4096.f, c[4 * i + 3], fmaf(256.f, c[4 * i + 2], fmaf(16.f, c[4 * i + 1], c[4 * i]))) + 8388608.0f) & 0xffffu;
        c_lo = h[0] | h[1] << 16;
        c_hi = h[2] | h[3] << 16;
    }
    params = (uint32_t)__half_as_ushort(s16) | ((uint32_t)__half_as_ushort(m16) << 16);
}

// How the pairs that turn together lie: none, in a thread's two chunks (halves, rot a multiple of 16),
// next to each other, or anywhere (halves of another size: partners are fetched one by one).
enum PagedTurn { kTurnNone, kTurnChunks, kTurnPairs, kTurnAny };

// Two chunks of a row as they are loaded.
template <int DT> struct RowPart { uint4 u[DT == MOA_F32 ? 4 : 2]; };
template <int DT>
__device__ __forceinline__ void fetch(RowPart<DT> &r, const unsigned char *row, int d_lo, int d_hi)
{
    constexpr int ES = DT == MOA_F32 ? 4 : 2, N = DT == MOA_F32 ? 2 : 1;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        r.u[i] = *reinterpret_cast<const uint4 *>(row + d_lo * ES + 16 * i);
        r.u[N + i] = *reinterpret_cast<const uint4 *>(row + d_hi * ES + 16 * i);
    }
}

// FMT: of the pools; DT: of q, k, v.  The same for 16 and 32 bits.
template <int FMT, int DT, int D, int TURN>
__global__ void __launch_bounds__(256, TURN == kTurnAny ? 2 : DT == MOA_F32 || FMT == MOA_KV_INT4 ? 3 : 4) paged_append_kernel(const __grid_constant__ PagedIoArgs a)
{
    constexpr int TPR = D / 16, SLOTS = 256 / TPR, ES = DT == MOA_F32 ? 4 : 2, N = DT == MOA_F32 ? 2 : 1;
    launch_dependents();
    grid_dependency_wait();
    const int part = threadIdx.x % TPR;
    const unsigned mask = ((1u << TPR) - 1u) << (threadIdx.x & 31 & ~(TPR - 1));
    const long long item = (long long)blockIdx.x * SLOTS + threadIdx.x / TPR;     // run by run, the tokens of a run in order
    const int run = item <= 0xffffffffll ? (int)((unsigned)item / (unsigned)a.tokens) : (int)(item / a.tokens);
    const int tok = (int)(item - (long long)run * a.tokens);
    if (run >= a.q_runs + 2 * a.kv_runs) return;           // (the threads of a row leave together)
    const int kind = run < a.q_runs ? 0 : run < a.q_runs + a.kv_runs ? 1 : 2;      // q, k, v
    const int h0 = (run - (kind == 0 ? 0 : kind == 1 ? a.q_runs : a.q_runs + a.kv_runs)) * a.run;
    const int h1 = min(h0 + a.run, kind == 0 ? a.h_q : a.h_kv);

    // The first row is under way while its place is found.
    int d_lo = 16 * part, d_hi = 16 * part + 8;
    const bool turns = TURN != kTurnNone && kind != 2 && 16 * part < a.rot;
    if (TURN == kTurnChunks && turns) { d_lo = 8 * part; d_hi = a.rot / 2 + 8 * part; }
    const unsigned char *src = kind == 0 ? static_cast<const unsigned char *>(a.q) + tok * a.q_st * ES
                             : kind == 1 ? static_cast<const unsigned char *>(a.k) + tok * a.k_st * ES
                                         : static_cast<const unsigned char *>(a.v) + tok * a.v_st * ES;
    src += (long long)h0 * D * ES;
    RowPart<DT> next;
    fetch<DT>(next, src, d_lo, d_hi);

    // The token's sequence, position and row.
    int b = tok;
    long long pos;
    if (a.token_start != nullptr) {
        int lo = 0, hi = a.batch;                          // last b with token_start[b] <= tok
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.token_start[mid] <= tok) lo = mid; else hi = mid;
        }
        b = lo;
        const int first = a.token_start[b], next = a.token_start[b + 1];
        if (first > tok || tok >= next) return;            // behind the last sequence: left as it is
        pos = (long long)a.seq_lens[b] - ((long long)next - tok);
    } else {
        pos = (long long)a.seq_lens[b] - 1;
        if (pos == -1) return;                             // a padded batch: no token
    }
    const int pi = pos < 0 ? 0 : a.page_shift >= 0 ? (int)pos >> a.page_shift : (int)pos / a.page_size;
    int status = 0, off = 0;
    long long page = 0;
    if (pos < 0 || pi >= a.max_pages || (TURN != kTurnNone && pos >= a.rope_rows)) status = MOA_STATUS_APPEND_RANGE;
    else {
        page = a.table[(long long)b * a.max_pages + pi];
        off = (int)pos - pi * a.page_size;
        if (page < 0 || page >= a.num_pages) status = MOA_STATUS_PAGE_RANGE;
    }
    if (status != 0) {
        if (part == 0 && run == 0) raise_status(status);
        return;
    }

    // This thread's share of the token's cosines and sines.
    const int rot = a.rot, half = rot / 2;
    float cs[8], sn[8];
    const float *row = a.cos_sin + pos * rot;
    if constexpr (TURN == kTurnChunks || TURN == kTurnPairs) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool in = turns && (TURN == kTurnChunks || 8 * part + i < half);
            cs[i] = in ? row[8 * part + i] : 1.f;
            sn[i] = in ? row[half + 8 * part + i] : 0.f;
        }
    }
    unsigned char *dst = kind == 0 ? static_cast<unsigned char *>(a.q_out) + tok * a.o_st * ES
                       : kind == 1 ? a.k_pool + page * a.k_sp + off * a.k_sr : a.v_pool + page * a.v_sp + off * a.v_sr;
    const long long dst_step = kind == 0 ? D * ES : kind == 1 ? a.k_sh : a.v_sh;
    dst += h0 * dst_step;
    uint32_t *par = FMT == MOA_KV_INT4 && kind != 0 ? (kind == 1 ? a.kp : a.vp) + (page * a.h_kv + h0) * a.page_size + off : nullptr;

#pragma unroll 1
    for (int h = h0; h < h1; ++h, src += D * ES, dst += dst_step) {
        const RowPart<DT> now = next;
        if (h + 1 < h1) fetch<DT>(next, src + D * ES, d_lo, d_hi);
        float lo[8], hi[8];
        load8<DT>(lo, &now.u[0]);
        load8<DT>(hi, &now.u[N]);
        if constexpr (TURN == kTurnChunks) {
            if (turns) {
#pragma unroll
                for (int i = 0; i < 8; ++i) turn(lo[i], hi[i], cs[i], sn[i]);
            }
        } else if constexpr (TURN == kTurnPairs) {
            if (turns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (d_lo + 2 * i < rot) turn(lo[2 * i], lo[2 * i + 1], cs[i], sn[i]);
                    if (d_hi + 2 * i < rot) turn(hi[2 * i], hi[2 * i + 1], cs[4 + i], sn[4 + i]);
                }
            }
        } else if constexpr (TURN == kTurnAny) {
            if (turns) {
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int d = 16 * part + i, pair = d < half ? d : d - half;
                    if (d < rot) {
                        float x = load_as_float(src, pair, DT), y = load_as_float(src, pair + half, DT);
                        turn(x, y, row[pair], row[half + pair]);
                        (i < 8 ? lo[i] : hi[i - 8]) = d < half ? x : y;
                    }
                }
            }
            __syncwarp(mask);                              // q_out may be q: its row is read by now
        }
        if (FMT != MOA_KV_INT4 || kind == 0) {
            store8<DT>(dst + d_lo * ES, lo);
            store8<DT>(dst + d_hi * ES, hi);
        } else {
            uint32_t c_lo, c_hi, params;
            pack_row<D>(lo, hi, c_lo, c_hi, params, mask);
            *reinterpret_cast<uint32_t *>(dst + d_lo / 2) = c_lo;
            *reinterpret_cast<uint32_t *>(dst + d_hi / 2) = c_hi;
            if (part == 0) *par = params;
            par += a.page_size;
        }
    }
}

// Rows [row_start, seq_len) of every sequence into [batch, h_kv, n_out, D].  A block takes 64 rows of one
// slab, a thread eight features of K and of V in four of them.
constexpr int kGatherRows = 64;
template <int FMT, int D>
__global__ void __launch_bounds__(256) paged_gather_kernel(const __grid_constant__ PagedIoArgs a, int out_dtype)
{
    constexpr int TPR = D / 8, SLOTS = 256 / TPR, PASSES = kGatherRows / SLOTS;
    launch_dependents();
    grid_dependency_wait();
    const unsigned chunks = (a.n_out - 1) / kGatherRows + 1;
    const unsigned slab = blockIdx.x / chunks;
    const int i0 = (int)(blockIdx.x - slab * chunks) * kGatherRows;
    const int b = (int)(slab / a.h_kv), h = (int)(slab - (unsigned)b * a.h_kv);
    const int len = a.seq_lens[b], from = a.row_start != nullptr ? a.row_start[b] : 0;
    if (from < 0 || len < from || (long long)len - from > a.n_out || len > (long long)a.max_pages * a.page_size) {
        if (i0 == 0 && h == 0 && threadIdx.x == 0) raise_status(MOA_STATUS_SEQLEN_RANGE);
        return;
    }
    const int d = (threadIdx.x % TPR) * 8;
    constexpr int ES = FMT == MOA_KV_F32 ? 4 : 2;
    const unsigned char *kh = a.k_pool + h * a.k_sh + (FMT == MOA_KV_INT4 ? d / 2 : d * ES);
    const unsigned char *vh = a.v_pool + h * a.v_sh + (FMT == MOA_KV_INT4 ? d / 2 : d * ES);
#pragma unroll
    for (int p = 0; p < PASSES; ++p) {
        const int i = i0 + p * SLOTS + threadIdx.x / TPR, row = from + i;
        if (i >= len - from) return;                       // (and so are the rows of later passes)
        const int pi = a.page_shift >= 0 ? row >> a.page_shift : row / a.page_size;
        const int off = row - pi * a.page_size;
        const long long page = a.table[(long long)b * a.max_pages + pi];
        if (page < 0 || page >= a.num_pages) {
            if (d == 0) raise_status(MOA_STATUS_PAGE_RANGE);
            continue;
        }
        const unsigned char *ks = kh + page * a.k_sp + off * a.k_sr, *vs = vh + page * a.v_sp + off * a.v_sr;
        float x[8], y[8];
        if constexpr (FMT == MOA_KV_INT4) {
            const long long at = (page * a.h_kv + h) * a.page_size + off;
            const uint32_t kc = *reinterpret_cast<const uint32_t *>(ks), vc = *reinterpret_cast<const uint32_t *>(vs);
            const float2 kf = unpack16<false>(a.kp[at]), vf = unpack16<false>(a.vp[at]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {                  // a code as the low bits of 2^23 + code
                x[e] = fmaf(kf.x, __uint_as_float(((kc >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f, kf.y);
                y[e] = fmaf(vf.x, __uint_as_float(((vc >> (4 * e)) & 15u) | 0x4b000000u) - 8388608.0f, vf.y);
            }
        } else {
            load8<FMT>(x, ks);
            load8<FMT>(y, vs);
        }
        const long long to = ((long long)slab * a.n_out + i) * D + d;
        if (out_dtype == MOA_F32) {
            store8<MOA_F32>(static_cast<float *>(a.k_out) + to, x);
            store8<MOA_F32>(static_cast<float *>(a.v_out) + to, y);
        } else if (out_dtype == MOA_BF16) {
            store8<MOA_BF16>(static_cast<uint16_t *>(a.k_out) + to, x);
            store8<MOA_BF16>(static_cast<uint16_t *>(a.v_out) + to, y);
        } else {
            store8<MOA_F16>(static_cast<uint16_t *>(a.k_out) + to, x);
            store8<MOA_F16>(static_cast<uint16_t *>(a.v_out) + to, y);
        }
    }
}

}  // namespace moa
