// moa_prompt.cuh -- attention of many new tokens at once: whole prompts packed one behind the other, and chunks of
// new tokens over a paged cache (16-bit rows, or 4-bit rows with 16-bit queries).
//
// For query head h of token i of a sequence of n new tokens behind `past` rows (0 for a prompt), K/V head h / g:
//     s[l] = scale <q, K[l]>,  out = sum_l 2^(log2e (s[l] - m)) V[l] / sum_l 2^(log2e (s[l] - m)),  l <= past + i
// (all l of the sequence where a prompt is not causal), in one pass over the rows with a running reference m.
//
// Both products run on the tensor core (tcgen05, accumulators in tensor memory).  A UNIT is up to 256 rows of
// queries -- the g heads of consecutive tokens, which share K and V -- against the rows of one K/V head, 128 keys
// at a time:
//   warps 0-3, 4-7   softmax of slot 0 and slot 1, a thread to a query row (a tensor memory lane): scores out, weights in,
//                    the weighted sum rescaled where the reference moves (it moves when weights pass 2^AHEAD, which
//                    after the first tiles is rare), and the output at the end of the unit
//   warps 8, 9       copies of Q, K and V into swizzled tiles: tiled ones where the layout allows them, else row by row
//                    (a page may end anywhere); 4 bits are unpacked here
//   warps 10, 11     issue the products of slot 0 and slot 1
// The two slots hold rows 0..127 and 128..255 of the unit, both against every tile of keys; a unit of at most 128
// rows has the same rows in both, against the even and the odd tiles, and the slots are joined at its end.
//
// A slot's scores and weights share 128 columns of tensor memory, 64 for each half of a tile of keys; the weights of a half (32
// columns) overwrite its scores.  Products of one thread run in order, so the scores of a half of the next tile are issued
// behind the product that uses up the weights in their place, while the softmax is at the other half.
//
// Work is handed out unit by unit (one CTA per SM; the next one's number comes from a counter; what a unit gives does not depend
// on who takes it).  Where there are few units their keys are cut into pieces; the CTA that delivers a unit's last piece
// joins them in order.
//
// What bounds it: the softmax.  A tile of each slot takes its scheduler 2118 cycles when nothing else runs (1549
// without the exponentials; a spilled register is an L2 round trip, since shared memory leaves no L1), the tensor
// core 2048 in whole tiles and 3072 with the scores by halves, and beside MMA and copy warps a tile of both slots comes out at
// 2700..3100 cycles: 951 GFLOP of two causal prompts (7001 and 8192 tokens, 32/8 heads of 128) in 0.94..1.06 ms, by the power that
// is left, against 0.57 ms at the measured GEMM rate.  Rows of 64 halve the products, not the softmax.
#pragma once

#include "moa_grouped64.cuh"
#include "moa_paged.cuh"

namespace moa {

struct PromptArgs {
    const unsigned char *q;
    unsigned char *out;
    long long q_st, o_st;            // bytes between consecutive tokens
    const unsigned char *k, *v;      // tensors (heads of a token are dense), or pools
    const uint32_t *kp, *vp;         // 4-bit rows: (scale, least) pairs
    long long k_sp, k_sh, k_sr;      // bytes: page (pools), kv head, row
    long long v_sp, v_sh, v_sr;
    int num_pages, page_size;
    uint32_t page_mul;               // row / page_size = row * page_mul >> page_sh, for rows below 2^31
    int page_sh;
    int box;                         // rows of a tiled copy (16 or 32; a page is a multiple of them); 0: there are no tensor maps
    const int32_t *table;
    int max_pages, len_max;
    const int32_t *token_start;      // [batch + 1]; null: one token each (pools), one sequence (tensors)
    const int32_t *seq_lens;         // pools: lengths with the new rows
    int tokens, batch, h_q, h_kv, g;
    uint32_t g_mul;                  // row / g, as above
    int g_sh;
    int causal;
    float qscale;                    // |scale| * log2(e)
    int negate;                      // scale < 0
    float *slots;                    // partial results of pieces, slot_rows * (D + 2) floats each
    int slot_cap, slot_rows;
    unsigned long long *tickets;     // slot_cap counters of pieces, then the counter of items handed out
    unsigned long long ticket_tag;
    uint32_t wait_limit;             // polls after which a wait gives up (behind the first 64)
    int skip_tile;                   // test hook: this tile's K is announced and never copied (tiled copies); -1: none
};

template <int FMT_, bool BF_, int D_, bool PAGED_>
struct PromptCfg {
    static constexpr int FMT = FMT_, D = D_;               // FMT: MOA_KV_INT4, or the 16-bit type
    static constexpr bool BF = BF_, PAGED = PAGED_, Q4 = FMT == MOA_KV_INT4;
    static constexpr int THREADS = 384, TILE = 128;
    static constexpr int KV = TILE * D * 2;                // bytes of a tile of K or V in shared memory
    static constexpr int NST = D == 128 ? 2 : 4;           // stages of K and of V
    static constexpr int NPAR = 2 * NST;                   // parameters of 4-bit rows: twice as many tiles as stages
    static constexpr uint32_t OFF_Q = 0;
    static constexpr uint32_t OFF_K = OFF_Q + 2 * KV;
    static constexpr uint32_t OFF_V = OFF_K + NST * KV;
    static constexpr uint32_t OFF_PAR = OFF_V + NST * KV;  // [NPAR][4][128]: K scale, K least + 8 scale, V scale, V least + 8 scale
    static constexpr uint32_t OFF_PMAX = OFF_PAR + (Q4 ? NPAR * 2 * 128 * 8 : 0);      // [NPAR][4] largest scales of V
    static constexpr uint32_t OFF_NF = OFF_PMAX + (Q4 ? NPAR * 16 : 0);                // [2][D] first key with a V that is not finite
    static constexpr uint32_t OFF_ML = OFF_NF + 2 * D * 4; // [2][128] (m, l) of the slots
    static constexpr uint32_t OFF_ROWS = OFF_ML + 2 * 128 * 8;      // [128] places of a tile's rows, K and V
    static constexpr uint32_t OFF_PLAN = OFF_ROWS + (PAGED ? 128 * 16 : 0);
    static constexpr uint32_t SMEM = OFF_PLAN + THREADS * 28 + 1024;      // (1024: alignment of the base)
    // How far (log2) a score may pass the reference before it moves, and what the weights are taken larger by: those held
    // in fp16 reach 2^15, and 64 weights of 1 are no reason to move.
    static constexpr float AHEAD = BF ? 8.0f : 7.0f;
    static constexpr float SHIFT = BF ? 0.0f : 8.0f;
    static constexpr int DEG = BF ? 3 : 4;
    static constexpr unsigned POLY = 0x88;                 // of eight pairs of weights, those that go through the polynomial
};

struct PromptSeq { int first, n, past, len; };

// Sequence b; n = 0 where it has no new tokens or is refused (bad: its status).  `floor`: the largest entry of token_start before
// b's that lies inside the call, carried on to b + 1.  A sequence that starts below it is refused, so no token is two sequences'
// and the host's bound on the blocks of rows, which follows from the number of tokens, holds whatever the entries are.
template <bool PAGED>
__host__ __device__ __forceinline__ PromptSeq prompt_seq(const PromptArgs &a, int b, int &floor, int &bad)
{
    PromptSeq s;
    long long first, next;
    if (a.token_start != nullptr) { first = a.token_start[b]; next = a.token_start[b + 1]; }
    else if (PAGED) { first = b; next = b + 1; }
    else { first = 0; next = a.tokens; }
    bad = 0;
    const int before = floor;
    if (first <= a.tokens && first > floor) floor = (int)first;
    if (next <= a.tokens && next > floor) floor = (int)next;
    if (first < before || next < first || next > a.tokens) { bad = MOA_STATUS_SEQLEN_RANGE; first = next = 0; }
    s.first = (int)first; s.n = (int)(next - first);
    s.len = PAGED ? a.seq_lens[b] : s.n;
    s.past = s.len - s.n;
    if (PAGED && s.n > 0) {
        const bool none = a.token_start == nullptr && s.len == 0;      // a padded batch: a token that sees nothing
        if (!none && (s.len < s.n || s.len > a.len_max)) { bad = MOA_STATUS_SEQLEN_RANGE; s.n = 0; }
    }
    return s;
}

__host__ __device__ __forceinline__ int div_g(const PromptArgs &a, int r) { return (int)(((unsigned long long)(uint32_t)r * a.g_mul) >> a.g_sh); }

// Keys that row r (token r / g) of a sequence sees.
__host__ __device__ __forceinline__ int prompt_sees(const PromptArgs &a, const PromptSeq &s, int r)
{
    if (!a.causal) return s.len;
    return s.past + div_g(a, r) + 1;
}

struct PromptItem {
    int first, past, len;            // the sequence
    int head;                        // kv head
    int table_row;                   // sequence number
    int row0, rows;                  // query rows of the unit: first one, and how many (1..256); 0: there is no further item
    int t0, e0, e1;                  // tiles of keys: first one, and the ends for slot 0 and slot 1
    int pair;                        // the slots take the even and the odd tiles of the same rows
    int least;                       // keys that the unit's first row sees
    int slot, pieces, slot_step;     // piece 0's slot (-1: one piece), pieces, distance of the pieces' slots
    int piece;
};

// ---- how the work is cut ------------------------------------------------------------------
struct PromptPlan { int rows, step_max, items; };

template <bool PAGED>
__host__ __device__ __forceinline__ void prompt_counts(const PromptArgs &a, const PromptSeq &s, int R, int T, int &tiles, int &pieces)
{
    const long long rows = (long long)s.n * a.g;
    tiles = (int)((rows + R - 1) / R);
    pieces = 0;
    if (s.n == 0) return;
    const int keys = (prompt_sees(a, s, (int)rows - 1) + 127) >> 7;
    const int steps = rows <= 128 || R == 128 ? (keys + 1) >> 1 : keys;
    pieces = steps > T ? (steps + T - 1) / T : 1;
}

// Sums of two numbers over the block, the same for every thread; any: whether any thread's was set.
__device__ __forceinline__ longlong2 prompt_block_sum(long long x, long long y, int &any, longlong2 *scratch)
{
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        x += __shfl_xor_sync(0xffffffffu, x, off);
        y += __shfl_xor_sync(0xffffffffu, y, off);
    }
    any = __syncthreads_or(any);
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = make_longlong2(x, y);
    __syncthreads();
    longlong2 t = make_longlong2(0, 0);
    for (int i = 0; i < (int)blockDim.x / 32; ++i) { t.x += scratch[i].x; t.y += scratch[i].y; }
    return t;
}

// The largest entry of token_start inside the call before those of this thread's sequences b0 .. b1 - 1.  Whole blocks; needed only
// where some sequence is refused (entries that ascend have none).
__device__ __forceinline__ int prompt_floor(const PromptArgs &a, int b0, int b1, int *scratch)
{
    if (a.token_start == nullptr) return 0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = 0;
    for (int b = b0; b < b1; ++b) {
        const int at = a.token_start[b];
        if (at <= a.tokens) x = max(x, at);
    }
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x = max(x, y);
    }
    __syncthreads();
    if (lane == 31) scratch[warp] = x;
    __syncthreads();
    x = __shfl_up_sync(0xffffffffu, x, 1);
    if (lane == 0) x = 0;
    for (int w = 0; w < warp; ++w) x = max(x, scratch[w]);
    return x;
}

// What a thread keeps of its sequences: how many (items, slots) come before them, and the sequence where it is only one, else
// what the first one may not start below.
struct PromptGroup { int items, slots; PromptSeq s; int floor; };

// Every CTA finds the same plan: rows of a unit and the most steps (a tile of keys for 256 rows) that a piece has.
template <bool PAGED>
__device__ __forceinline__ PromptPlan prompt_plan(const PromptArgs &a, PromptGroup *groups, longlong2 *scratch, bool report)
{
    const int tid = threadIdx.x, nt = blockDim.x;
    const int gs = (a.batch + nt - 1) / nt;                // sequences of a group: one thread's
    const int b0 = min(tid * gs, a.batch), b1 = min(b0 + gs, a.batch);
    int bad, tiles, pieces, floor = 0;
    PromptSeq s = {0, 0, 0, 0};
    longlong2 sums;
    for (bool again = false;; again = true) {              // (again: what was refused may be a start that the ones behind it are to be held against)
        long long units = 0, work = 0;
        int wrong = 0, f = floor;
        for (int b = b0; b < b1; ++b) {
            s = prompt_seq<PAGED>(a, b, f, bad);
            if (bad != 0) { wrong = 1; if (report) raise_status(bad); }
            if (s.n == 0) continue;
            prompt_counts<PAGED>(a, s, 256, 0x7fffffff, tiles, pieces);
            const long long rows = (long long)s.n * a.g;
            const int last = (prompt_sees(a, s, (int)rows - 1) + 127) >> 7, front = (prompt_sees(a, s, 0) + 127) >> 7;
            units += (long long)tiles * a.h_kv;
            work += rows <= 128 ? (long long)a.h_kv * ((last + 1) >> 1) : (long long)a.h_kv * tiles * (last + front + 1) / 2;
        }
        sums = prompt_block_sum(units, work, wrong, scratch);
        if (!wrong || again) break;
        floor = prompt_floor(a, b0, b1, reinterpret_cast<int *>(scratch + 16));
    }
    const int grid = gridDim.x;
    PromptPlan p;
    // 256 rows read K and V half as often; 128 spread better where there are few short units (us, 256 rows against 128: 7 prompts of
    // 301..2047 tokens 172 and 215, one of 77 tokens 20.6 and 17.4, 13 pieces over pages of 20 rows 267 and 392, this rule 252).
    p.rows = sums.x >= 2 * grid || sums.y >= 32LL * grid ? 256 : 128;
    long long T = (sums.y + grid - 1) / grid;
    if (T < 6) T = 6;                                      // (joining pieces costs what four or five steps do)
    int items, slots;
    for (;;) {                                             // (ends: with T long enough nothing is cut)
        long long all = 0;
        items = slots = 0;
        int none = 0, f = floor;
        for (int b = b0; b < b1; ++b) {
            if (gs > 1) s = prompt_seq<PAGED>(a, b, f, bad);
            prompt_counts<PAGED>(a, s, p.rows, (int)min(T, 0x7fffffffLL), tiles, pieces);
            const long long c = (long long)tiles * pieces * a.h_kv;
            if (pieces > 1) { all += c; if (c <= a.slot_cap) slots += (int)c; }
            items += (int)min(c, 0x7fffffffLL);
        }
        const longlong2 t = prompt_block_sum(all, items, none, scratch);
        p.items = (int)t.y;
        if (t.x <= a.slot_cap) break;
        T += T / 2;
    }
    p.step_max = (int)min(T, 0x7fffffffLL);
    // exclusive prefix over the groups
    int2 inc = make_int2(items, slots);
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc.x, off), y = __shfl_up_sync(0xffffffffu, inc.y, off);
        if ((tid & 31) >= off) { inc.x += x; inc.y += y; }
    }
    int2 *const per_warp = reinterpret_cast<int2 *>(scratch + 16);
    if ((tid & 31) == 31) per_warp[tid >> 5] = inc;
    __syncthreads();
    int2 before = make_int2(0, 0);
    for (int i = 0; i < (tid >> 5); ++i) { before.x += per_warp[i].x; before.y += per_warp[i].y; }
    groups[tid].items = before.x + inc.x - items;
    groups[tid].slots = before.y + inc.y - slots;
    groups[tid].s = s;
    groups[tid].floor = floor;
    return p;                                              // (a block barrier follows)
}

// Item number `i`.  One thread.
template <bool PAGED>
__device__ __forceinline__ void prompt_item(const PromptArgs &a, const PromptPlan &p, const PromptGroup *groups, int nt, int i, PromptItem &it)
{
    it.rows = 0;
    if (i >= p.items) return;
    int lo = 0, hi = nt;                                   // last group with items <= i
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (groups[mid].items <= i) lo = mid; else hi = mid;
    }
    const int gs = (a.batch + nt - 1) / nt;
    int at = groups[lo].items, slot = groups[lo].slots, bad, tiles = 0, pieces = 0, b = lo * gs, floor = groups[lo].floor;
    PromptSeq s = groups[lo].s;
    for (;; ++b) {
        if (b >= a.batch) return;                          // (not reached: the plan counted the item)
        if (gs > 1) s = prompt_seq<PAGED>(a, b, floor, bad);
        prompt_counts<PAGED>(a, s, p.rows, p.step_max, tiles, pieces);
        const int c = tiles * pieces * a.h_kv;
        if (i < at + c) break;
        at += c;
        if (pieces > 1) slot += c;
    }
    // inside a sequence: the last tiles of rows, which see most keys, first; heads innermost
    const int j = i - at, head = j % a.h_kv, k = j / a.h_kv, piece = k % pieces, tile = tiles - 1 - k / pieces;
    const int all = s.n * a.g;
    it.first = s.first; it.past = s.past; it.len = s.len; it.head = head; it.table_row = b;
    it.row0 = tile * p.rows;
    it.rows = min(p.rows, all - it.row0);
    it.pair = it.rows <= 128;
    it.least = prompt_sees(a, s, it.row0);
    const int end1 = (prompt_sees(a, s, it.row0 + it.rows - 1) + 127) >> 7;
    const int end0 = it.pair ? end1 : (prompt_sees(a, s, it.row0 + 127) + 127) >> 7;
    it.t0 = (int)((long long)end1 * piece / pieces);
    it.e1 = (int)((long long)end1 * (piece + 1) / pieces);
    it.e0 = min(it.e1, end0);
    it.piece = piece; it.pieces = pieces;
    it.slot_step = a.h_kv;
    it.slot = pieces > 1 ? slot + (k - piece) * a.h_kv + head : -1;
}

// Steps of slot s of an item.
__device__ __forceinline__ int prompt_steps(const PromptItem &it, int s)
{
    const int n = it.e1 - it.t0;
    if (it.pair) return s == 0 ? (n + 1) >> 1 : n >> 1;
    return s == 0 ? max(0, it.e0 - it.t0) : n;
}

// ---- tensor core --------------------------------------------------------------------------
namespace tc {
// Instruction descriptor of kind::f16, fp32 accumulate: A and B bf16 or fp16; bit 13 negates A.
__host__ __device__ constexpr uint32_t idesc_16(bool bf16, int M, int N, bool b_mn_major)
{
    return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) |
           ((uint32_t)(M >> 4) << 24);
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void *tmap, int c0, int c1, int c2, int c3, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(tmap), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
        : "memory");
}
// One lane of a converged warp: the compiler knows the choice for uniform, and issues products from uniform registers.
__device__ __forceinline__ bool elect_one()
{
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void mma_16_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
}  // namespace tc

// Wait of a whole warp: all lanes leave it with the same answer.  The first polls are a loop of a few instructions (code
// that is fetched from far away costs as much as the wait) and may each be suspended for up to a millisecond: without
// the hint they take issue slots from the softmax (two prompts of 7001 and 8192 tokens 1280 us instead of 1003, at a step
// on the way).  `limit`: of the polls behind them, from the arguments: kept in shared memory beside the flag it cost 3 % of
// the long cases, a load for each wait that comes this far.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int *abort_flag, uint32_t limit)
{
    uint32_t ok;
    asm volatile(
            "{\n\t.reg .pred p, q;\n\t.reg .u32 n;\n\tmov.u32 n, 0;\n"
            "WAIT_%=:\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\t@p bra DONE_%=;\n\t"
            "add.u32 n, n, 1;\n\tsetp.lt.u32 q, n, 64;\n\t@q bra WAIT_%=;\n"
            "DONE_%=:\n\tselp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok) : "r"(bar), "r"(parity), "r"(1000000u) : "memory");
    if (__all_sync(0xffffffffu, ok)) return true;
#pragma unroll 1
    for (uint32_t it = 0; it < limit; ++it) {
        if (__all_sync(0xffffffffu, mbar_try_wait(bar, parity))) return true;
        if ((it & 15u) == 15u && __any_sync(0xffffffffu, *abort_flag)) return false;
    }
    *abort_flag = 1;
    raise_status(MOA_STATUS_WAIT_TIMEOUT);
    return false;
}
// Whether a phase is over, asked by one lane.
__device__ __forceinline__ bool test_warp(uint32_t bar, uint32_t parity)
{
    uint32_t ok = 1;
    if ((threadIdx.x & 31) == 0) ok = mbar_test_wait(bar, parity);
    return __all_sync(0xffffffffu, ok);
}

__device__ __forceinline__ float max_nan(float x, float y)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ float max_nan(float x, float y, float z)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t pack2f(float lo, float hi) { return pack2(__float_as_uint(lo), __float_as_uint(hi)); }
__device__ __forceinline__ float2 unpack2f(uint64_t v)
{
    uint32_t lo, hi;
    unpack2(v, lo, hi);
    return make_float2(__uint_as_float(lo), __uint_as_float(hi));
}

// 2^x for two x at once on the FMA units: x = n + f with |f| <= 1/2, a polynomial in f (least relative error over
// the interval, fitted for this file: 7.5e-5 of degree 3, 2.6e-6 of degree 4), times 2^n as a bit pattern.  x at or
// below -127 gives 0; the caller sees to it that x is no larger than 15.  The special function unit makes 16 results a cycle and
// SM; a tile of 128 x 128 scores would keep it busy exactly as long as the tensor core takes for the tile's two products, so a
// quarter of the weights goes this way (two slots on a scheduler, cycles for a tile of each: a quarter 2118, an eighth 2064, none
// 2266; beside the other warps, which share the issue slots, a quarter is the best: 2 x 8192 tokens 899 us, an eighth 926).
template <int DEG>
__device__ __forceinline__ float2 exp2_pair(uint64_t x)
{
    const float2 v = unpack2f(x);
    x = pack2f(fmaxf(v.x, -127.0f), fmaxf(v.y, -127.0f));
    const uint64_t magic = pack2f(12582912.0f + 127.0f, 12582912.0f + 127.0f);      // low bits: n + 127
    const uint64_t t = add2(x, magic);
    const uint64_t f = sub2(x, sub2(t, magic));
    uint64_t r;
    if (DEG == 3) {
        r = fma2(f, pack2f(0.0551716685f, 0.0551716685f), pack2f(0.2426111251f, 0.2426111251f));
        r = fma2(f, r, pack2f(0.6932609677f, 0.6932609677f));
        r = fma2(f, r, pack2f(0.9999280572f, 0.9999280572f));
    } else {
        r = fma2(f, pack2f(0.0095701022f, 0.0095701022f), pack2f(0.0559178591f, 0.0559178591f));
        r = fma2(f, r, pack2f(0.2402474433f, 0.2402474433f));
        r = fma2(f, r, pack2f(0.6931217909f, 0.6931217909f));
        r = fma2(f, r, pack2f(0.9999992847f, 0.9999992847f));
    }
    uint32_t a, b;
    unpack2(t, a, b);
    return unpack2f(mul2(r, pack2(a << 23, b << 23)));
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) prompt_attn_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v)
{
    constexpr int D = C::D, NST = C::NST;
    constexpr bool BF = C::BF, Q4 = C::Q4, PAGED = C::PAGED;
    extern __shared__ unsigned char smem_prompt[];
    __shared__ __align__(8) uint64_t bars[4 * NST + 25 + C::NPAR];
    __shared__ PromptItem s_item[2];
    __shared__ longlong2 s_scratch[16 + 8];
    __shared__ uint32_t s_tmem;
    __shared__ int s_abort, s_last, s_nf[2];
    __shared__ float2 s_more[Q4 ? 2 : 1][Q4 ? 128 : 1];      // 4 bits: what joins the slots beside (m, l)
    const uint32_t base = (smem_u32(smem_prompt) + 1023u) & ~1023u;
    unsigned char *const smem = smem_prompt + (base - smem_u32(smem_prompt));
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    volatile int *abort_flag = &s_abort;

    const uint32_t bar0 = smem_u32(bars);
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    auto k_full = [&](int i) { return bar(i); };
    auto k_empty = [&](int i) { return bar(NST + i); };
    auto v_full = [&](int i) { return bar(2 * NST + i); };
    auto v_empty = [&](int i) { return bar(3 * NST + i); };
    constexpr int B0 = 4 * NST;
    auto s_full = [&](int s, int h) { return bar(B0 + 2 * s + h); };         // scores of half a tile
    auto p_full = [&](int s, int h) { return bar(B0 + 4 + 2 * s + h); };     // its weights
    auto summed = [&](int s) { return bar(B0 + 8 + s); };                    // its part of the weighted sum
    auto o_full = [&](int s) { return bar(B0 + 10 + s); };                   // the weighted sum of a unit
    const uint32_t q_full = bar(B0 + 12), q_empty = bar(B0 + 13);
    auto item_full = [&](int i) { return bar(B0 + 14 + i); };
    auto item_empty = [&](int i) { return bar(B0 + 16 + i); };
    const uint32_t joined = bar(B0 + 18), parted = bar(B0 + 19), delivered = bar(B0 + 20), counted = bar(B0 + 21), drained = bar(B0 + 22);
    auto landed = [&](int w) { return bar(B0 + 23 + w); };                   // tiled copies of V that are looked at first
    auto par_full = [&](int i) { return bar(B0 + 25 + i); };

    if (tid == 0) {
        for (int i = 0; i < NST; ++i) { mbar_init(k_full(i), 2); mbar_init(k_empty(i), 2); mbar_init(v_full(i), 2); mbar_init(v_empty(i), 2); }
        for (int s = 0; s < 2; ++s) {
            mbar_init(s_full(s, 0), 1); mbar_init(s_full(s, 1), 1); mbar_init(p_full(s, 0), 4); mbar_init(p_full(s, 1), 4);
            mbar_init(summed(s), 1); mbar_init(o_full(s), 1); mbar_init(landed(s), 1);
            mbar_init(item_full(s), 1); mbar_init(item_empty(s), 11);
        }
        mbar_init(q_full, 2); mbar_init(q_empty, 2);
        mbar_init(joined, 8); mbar_init(parted, 8); mbar_init(delivered, 8); mbar_init(counted, 1); mbar_init(drained, 2);
        for (int i = 0; i < C::NPAR; ++i) mbar_init(par_full(i), 2);
        mbar_fence_init();
        s_abort = 0;
    }
    if (warp == 10) tc::tmem_alloc(smem_u32(&s_tmem), 512);
    if (tid == 32 * 8 && a.box > 0) { tc::prefetch_tmap(&map_k); tc::prefetch_tmap(&map_v); }
    launch_dependents();
    grid_dependency_wait();
    PromptGroup *const groups = reinterpret_cast<PromptGroup *>(smem + C::OFF_PLAN);
    const PromptPlan plan = prompt_plan<PAGED>(a, groups, s_scratch, blockIdx.x == 0);
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = s_tmem;
    auto t_s = [tmem](int s) -> uint32_t { return tmem + 128u * (uint32_t)s; };
    auto t_o = [tmem](int s) -> uint32_t { return tmem + 256u + (uint32_t)(s * D); };

    // 384 threads of 168 registers at launch: 256 x 200 + 128 x 104.
    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 104;");
        if (warp >= 10) {
            // ================= products: a warp for each slot =================
            // A thread that issues products is held until the tensor core has all but the last two of them, and whatever it does
            // between two batches (a look at a barrier: 80 to 220 cycles) the tensor core waits for, unless another warp has
            // products for it.
            const int s = warp - 10;
            const uint32_t sQ = base + C::OFF_Q, sK = base + C::OFF_K, sV = base + C::OFF_V, tS = t_s(s), tO = t_o(s);
            const uint32_t negate = a.negate ? 1u << 13 : 0u;
            constexpr uint32_t id_pv = tc::idesc_16(BF, 128, D, true);
            constexpr uint32_t hiword = 64u | (1u << 14) | (2u << 29);       // 1024 bytes between groups of 8 rows, 128-byte swizzle
            uint32_t nk = 0, nq = 0, np = 0;               // tiles of keys, items, own tiles so far
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                if (!wait_warp(item_full(n & 1), (n >> 1) & 1, abort_flag, a.wait_limit)) { ok = false; break; }
                const PromptItem &it = s_item[n & 1];
                if (it.rows == 0) break;
                const int cnt = prompt_steps(it, s), other = prompt_steps(it, s ^ 1);
                const bool pair = it.pair;
                if (max(cnt, other) > 0) {
                    ok = wait_warp(q_full, nq & 1, abort_flag, a.wait_limit);
                    const uint32_t qa = sQ + (pair ? 0u : (uint32_t)(s * C::KV));
                    if (cnt == 0 && lane == 0) tc::mbar_arrive(q_empty);
                    // step (i, h): half h of tile i into the weighted sum, then the scores of half h of tile i + 1 in their place
#pragma unroll 1
                    for (int u = -2; ok && u < 2 * cnt; ++u) {
                        const int i = u >> 1, h = u & 1;
                        const uint32_t vt = nk + (uint32_t)(pair ? 2 * i + s : i), vst = vt % NST;
                        const uint32_t kt = nk + (uint32_t)(pair ? 2 * (i + 1) + s : i + 1), kst = kt % NST;
                        const bool more = i + 1 < cnt;
                        if (i >= 0) {
                            // A unit's first V behind its first weights: in a unit of few rows this warp sees every second tile only, and a
                            // wait tells a phase that is over by its parity, so the one before, the other slot's, has to be over by then.
                            // The first weights come behind the join of the unit before, when all its tiles are used up.  (Tiles that slot 0
                            // of more rows does not see are looked through before the next unit's Q is there.)  From then on V
                            // first: a look at its barrier behind every tile's weights costs 1 % of the long cases.
                            const bool late = u == 0;
                            const uint32_t v_bar = v_full(vst), v_par = (vt / NST) & 1, p_bar = p_full(s, h), p_par = np & 1;
                            if (h == 0) ok = wait_warp(late ? p_bar : v_bar, late ? p_par : v_par, abort_flag, a.wait_limit);
                            ok = ok && wait_warp(late ? v_bar : p_bar, late ? v_par : p_par, abort_flag, a.wait_limit);
                            if (!ok) break;
                            np += h;
                            tc::fence_after_sync();
                            const uint32_t vb = sV + vst * C::KV + (uint32_t)h * 8192u, tP = tS + 64u * (uint32_t)h;
                            if (tc::elect_one()) {
#pragma unroll
                                for (uint32_t ks = 0; ks < 4; ++ks)
                                    tc::mma_16_ts(tO, tP + 8u * ks, tc::pack64(((vb + ks * 2048u) >> 4) | (1024u << 16), hiword), id_pv, (u != 0 || ks != 0));
                                tc::mma_commit(summed(s));
                                if (h == 1) {
                                    tc::mma_commit(v_empty(vst));
                                    if (pair || i >= other) tc::mma_commit(v_empty(vst));  // (for the other slot)
                                    if (!more) tc::mma_commit(o_full(s));
                                }
                            }
                            __syncwarp();
                        }
                        // The scores by halves, so that one is there while the softmax is at the other: 64 keys take the tensor core
                        // as long as 128 (the queries are read again), which is still the better (2 x 8192 tokens 0.90 ms;
                        // whole tiles 1.15, or 0.92..1.2 with the two warps in turns).  A unit of few rows waits for memory
                        // and takes whole tiles (64 x 4 draft tokens 296 us; by halves 450).
                        if (more && (h == 1 || !pair)) {
                            if (h == 0 || pair) {
                                ok = wait_warp(k_full(kst), (kt / NST) & 1, abort_flag, a.wait_limit);
                                if (!ok) break;
                                tc::fence_after_sync();
                            }
                            const uint32_t half = pair ? 0u : (uint32_t)h, kb = sK + kst * C::KV + half * 8192u, tH = tS + 64u * half;
                            const uint32_t id_qk = tc::idesc_16(BF, 128, pair ? 128 : 64, false) | negate;
                            if (tc::elect_one()) {
#pragma unroll
                                for (uint32_t ks = 0; ks < D / 16; ++ks) {
                                    const uint32_t off = (ks / 4) * 16384u + (ks % 4) * 32u;
                                    tc::mma_16_ss(tH, tc::pack64(((qa + off) >> 4) | (1u << 16), hiword), tc::pack64(((kb + off) >> 4) | (1u << 16), hiword), id_qk, ks != 0);
                                }
                                if (pair) tc::mma_commit(s_full(s, 0));
                                tc::mma_commit(s_full(s, h));
                                if (h == 1) {
                                    tc::mma_commit(k_empty(kst));
                                    if (pair || i + 1 >= other) tc::mma_commit(k_empty(kst));
                                    if (i + 2 == cnt) tc::mma_commit(q_empty);
                                }
                            }
                            __syncwarp();
                        }
                    }
                    nk += (uint32_t)(it.e1 - it.t0);
                    ++nq;
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(item_empty(n & 1));
            }
            if (!ok) {                                     // leave nothing in flight
                if (tc::elect_one()) tc::mma_commit(drained);
                __syncwarp();
                mbar_wait_bounded(drained, 0, 1u << 16);
            }
        } else {
        // ================= copies =================
        const int w = warp - 8;                            // of rows 64 w .. 64 w + 63 of a tile
        constexpr int CPR = D / 8, RPI = 32 / CPR;         // 16-byte chunks of a 16-bit row; rows of a warp's copy
        const int chunk = lane % CPR, rsub = lane / CPR;
        const uint32_t col = (uint32_t)(chunk >> 3) * 16384u;
        uint32_t nk = 0, nq = 0;
        bool ok = true;
        // The copies under way before the ones being made: the barrier that their arrival is told to, and for tiles of V that
        // not every row of the unit sees whole, what to look for: rows behind `pend_rows` (zeroed), and values that are not
        // finite (zeroed, and noted: the rows that see them become NaN at the unit's end).
        uint32_t pend_bar = 0, pend_at = 0, lands = 0;
        int pend_tile = -1, pend_rows = 0, pend_set = 0;   // pend_tile: of keys, -1: nothing to look for
        bool pending = false, pend_tma = false;
        auto dst_of = [&](int r) -> uint32_t { return col + (uint32_t)r * 128u + (uint32_t)(((chunk & 7) ^ (r & 7)) << 4); };
        auto look = [&]() {
            // a product with 0 is NaN where a value is not finite: one fused multiply-add for two values
            uint32_t sum = 0;
#pragma unroll 8
            for (int i = 0; i < 64 / RPI; ++i) {
                const int r = 64 * w + RPI * i + rsub;
                const uint32_t p = pend_at + dst_of(r);
                uint32_t u[4];
                if (r >= pend_rows) asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(p), "r"(0u) : "memory");
                asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(p) : "memory");
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (BF) asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u[e]), "r"(0u));
                    else asm("fma.rn.f16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u[e]), "r"(0u));
                }
            }
            if ((sum & 0x7fff7fffu) == 0u) return;
            for (int i = 0; i < 64 / RPI; ++i) {
                const int r = 64 * w + RPI * i + rsub;
                const uint32_t p = pend_at + dst_of(r);
                for (int e = 0; e < 8; ++e) {
                    uint16_t x;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(p + 2 * e) : "memory");
                    if ((x & (BF ? 0x7f80 : 0x7c00)) == (BF ? 0x7f80 : 0x7c00)) {
                        atomicMin(reinterpret_cast<int *>(smem + C::OFF_NF) + pend_set * D + chunk * 8 + e, pend_tile * 128 + r);
                        s_nf[pend_set] = 1;
                        asm volatile("st.shared.u16 [%0], %1;" ::"r"(p + 2 * e), "h"((uint16_t)0) : "memory");
                    }
                }
            }
        };
        auto retire = [&]() {                              // they have arrived
            if (pend_tma) { wait_warp(landed(w), lands & 1, abort_flag, a.wait_limit); ++lands; }
            if (pend_tile >= 0) look();
            tc::fence_async_smem();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(pend_bar);
            pending = false;
        };
        auto drain = [&]() { if (pending) { cp_wait<0>(); retire(); } };
        // What has been issued is what is under way from now on; what was before is waited for.
        auto push = [&](uint32_t b, uint32_t at, int tile, int rows, int set, bool tma) {
            cp_commit();
            if (pending) { cp_wait<1>(); retire(); }
            pend_bar = b; pend_at = at; pend_tile = tile; pend_rows = rows; pend_set = set; pend_tma = tma;
            pending = true;
        };
        auto wait_free = [&](uint32_t b, uint32_t parity) {
            if (test_warp(b, parity)) return true;
            drain();                  // what this waits for may need them
            return wait_warp(b, parity, abort_flag, a.wait_limit);
        };

        // Item n: drawn when the copies of the one before are issued (drawing it a tile earlier changed nothing).
        auto fetch = [&](uint32_t n) {
            const int set = n & 1;
            if (n >= 2) {
                ok = wait_free(item_empty(set), ((n >> 1) - 1) & 1);
                if (!ok) return;
            }
            if (lane == 0) {
                int i = blockIdx.x;
                if (n > 0) {
                    i = 0x7fffffff;
                    if (plan.items > (int)gridDim.x) {
                        unsigned long long *word = a.tickets + a.slot_cap;
                        const unsigned j = ticket_arrive(word, a.ticket_tag);
                        if (j + 1 == (unsigned)plan.items) *word = 0;          // every CTA has drawn its last number
                        i = (int)min((unsigned)gridDim.x + j, 0x7fffffffu);
                    }
                }
                prompt_item<PAGED>(a, plan, groups, C::THREADS, i, s_item[set]);
                s_nf[set] = 0;
            }
            for (int f = lane; f < D; f += 32) reinterpret_cast<int *>(smem + C::OFF_NF)[set * D + f] = 0x7fffffff;
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(item_full(set));
        };
        if (w == 0) fetch(0);

        for (uint32_t n = 0; ok; ++n) {
            const int set = n & 1;
            ok = wait_free(item_full(set), (n >> 1) & 1);
            if (!ok) break;
            const PromptItem &it = s_item[set];
            if (it.rows == 0) break;
            const int tiles = it.e1 - it.t0;
            if (prompt_steps(it, 0) + prompt_steps(it, 1) > 0) {
                PromptSeq sq;
                sq.first = it.first; sq.past = it.past; sq.len = it.len; sq.n = 0;
                const int sees = prompt_sees(a, sq, it.row0 + it.rows - 1);     // rows behind are not read
                // Where the rows of a tile are: a lane finds those of rows 64 w + lane and 32 further, and in pools tells them to the warp
                // through shared memory (an odd address: there is no such row).  The pages' numbers are read a tile ahead.
                uint2 *const places = reinterpret_cast<uint2 *>(smem + C::OFF_ROWS) + 128 * w;     // [64 rows][K, V]
                uint32_t k_pair[2] = {}, v_pair[2] = {};
                int page_next[2] = {-1, -1};
                bool row_ok[2] = {}, row_bad[2] = {};
                auto page_index = [&](long long row) { return (int)(((unsigned long long)(uint32_t)row * a.page_mul) >> a.page_sh); };
                auto look_up = [&](int t) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const long long row = (long long)t * 128 + 64 * w + 32 * g + lane;
                        if (PAGED && row < sees) page_next[g] = a.table[(long long)it.table_row * a.max_pages + page_index(row)];
                    }
                };
                auto locate = [&](int t, bool last) {
                    if (!PAGED) return;
                    const int pages[2] = {page_next[0], page_next[1]};
                    if (!last) look_up(t + 1);
                    __syncwarp();                          // (the tile before is through)
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const long long row = (long long)t * 128 + 64 * w + 32 * g + lane;
                        const int page = pages[g];
                        row_ok[g] = row < sees;
                        row_bad[g] = row_ok[g] && (page < 0 || page >= a.num_pages);
                        if (row_bad[g]) { row_ok[g] = false; raise_status(MOA_STATUS_PAGE_RANGE); }
                        const unsigned char *ka = a.k + 1, *va = a.v + 1;
                        if (row_ok[g]) {
                            const int off = (int)row - page_index(row) * a.page_size;
                            ka = a.k + (page * a.k_sp + it.head * a.k_sh + off * a.k_sr);
                            va = a.v + (page * a.v_sp + it.head * a.v_sh + off * a.v_sr);
                            if (Q4) {
                                const long long at = ((long long)page * a.h_kv + it.head) * a.page_size + off;
                                k_pair[g] = a.kp[at]; v_pair[g] = a.vp[at];
                            }
                        }
                        *reinterpret_cast<uint4 *>(places + 2 * (32 * g + lane)) =
                            make_uint4((uint32_t)(uintptr_t)ka, (uint32_t)((uintptr_t)ka >> 32), (uint32_t)(uintptr_t)va, (uint32_t)((uintptr_t)va >> 32));
                    }
                    __syncwarp();
                };
                auto place = [&](int r, bool is_k) {
                    const uint2 u = places[2 * r + (is_k ? 0 : 1)];
                    return ((unsigned long long)u.y << 32) | u.x;
                };
                auto copy_rows = [&](uint32_t at, int t, bool is_k) {
                    if (PAGED) {
#pragma unroll 8
                        for (int i = 0; i < 64 / RPI; ++i) {
                            const int from = RPI * i + rsub;
                            const unsigned long long p = place(from, is_k);
                            cp16(at + dst_of(64 * w + from), reinterpret_cast<const unsigned char *>(p & ~1ull) + 16 * chunk, (p & 1) == 0);
                        }
                        if (is_k && __any_sync(0xffffffffu, row_bad[0] || row_bad[1])) {      // a page that does not exist: its scores are NaN
                            cp_commit(); cp_wait<0>(); __syncwarp();
                            for (int i = 0; i < 64 / RPI; ++i) {
                                const int from = RPI * i + rsub;
                                const int b0 = __shfl_sync(0xffffffffu, (int)row_bad[0], from & 31), b1 = __shfl_sync(0xffffffffu, (int)row_bad[1], from & 31);
                                if (from < 32 ? b0 : b1)
                                    asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(at + dst_of(64 * w + from)), "r"(0x7fff7fffu) : "memory");
                            }
                        }
                    } else {
                        const long long first = (long long)t * 128 + 64 * w + rsub;
                        const long long sr = is_k ? a.k_sr : a.v_sr;
                        const unsigned char *p = (is_k ? a.k + it.head * a.k_sh : a.v + it.head * a.v_sh) + (it.first + first) * sr + 16 * chunk;
                        const int left = sees - (int)first;          // rows from this lane's first on
#pragma unroll 8
                        for (int i = 0; i < 64 / RPI; ++i, p += RPI * sr) {
                            const bool in = RPI * i < left;
                            cp16(at + dst_of(64 * w + RPI * i + rsub), in ? p : a.k, in);
                        }
                    }
                };
                // 4-bit rows: a code c becomes c - 8 (exact), two to a register; the row's scale and least value go to the softmax.
                constexpr int CP4 = D / 32;                // 16-byte chunks of a row of codes, 32 codes each
                auto fetch_rows = [&](uint4 (&x)[CP4], int g, bool is_k) {
#pragma unroll
                    for (int i = 0; i < CP4; ++i) {
                        const unsigned long long p = place(32 * g + i * (32 / CP4) + lane / CP4, is_k);
                        x[i] = (p & 1) == 0 ? *reinterpret_cast<const uint4 *>(p + 16 * (lane % CP4)) : make_uint4(0, 0, 0, 0);
                    }
                };
                auto unpack_rows = [&](uint32_t at, int g, const uint4 (&x)[CP4]) {
#pragma unroll
                    for (int i = 0; i < CP4; ++i) {
                        const int r = 64 * w + 32 * g + i * (32 / CP4) + lane / CP4;
                        const uint32_t c4[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint32_t o[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t two = (((c4[e] >> (8 * k)) & 0xffu) * 0x1001u) & 0x000f000fu;
                                if (BF) {                  // 128 + c, less 136
                                    const uint32_t y = two | 0x43004300u;
                                    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&y), __floats2bfloat162_rn(136.f, 136.f));
                                    o[k] = *reinterpret_cast<const uint32_t *>(&d);
                                } else {                   // 1024 + c, less 1032
                                    const uint32_t y = two | 0x64006400u;
                                    const __half2 d = __hsub2(*reinterpret_cast<const __half2 *>(&y), __floats2half2_rn(1032.f, 1032.f));
                                    o[k] = *reinterpret_cast<const uint32_t *>(&d);
                                }
                            }
                            const int ch = 4 * (lane % CP4) + e;              // 8 features of the row
                            const uint32_t p = at + (uint32_t)(ch >> 3) * 16384u + (uint32_t)r * 128u + (uint32_t)(((ch & 7) ^ (r & 7)) << 4);
                            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(p), "r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]) : "memory");
                        }
                    }
                };
                auto copy_q = [&]() {
                    ok = nq == 0 || wait_free(q_empty, (nq - 1) & 1);
                    if (!ok) return;
                    ++nq;
                    const int parts = it.pair ? 1 : 2;
                    for (int s = 0; s < parts; ++s) {
#pragma unroll 8
                        for (int i = 0; i < 64 / RPI; ++i) {
                            const int r = 64 * w + RPI * i + rsub, at = 128 * s + r;
                            const bool in = at < it.rows;
                            const int row = it.row0 + at, tok = div_g(a, row);
                            const unsigned char *p = a.q + (long long)(it.first + tok) * a.q_st + ((long long)it.head * a.g + (row - tok * a.g)) * (D * 2) + 16 * chunk;
                            cp16(base + C::OFF_Q + s * C::KV + dst_of(r), in ? p : a.q, in);
                        }
                    }
                    push(q_full, 0, -1, 0, 0, false);
                    drain();
                };
                look_up(it.t0);
                uint4 codes[2][CP4];
                for (int t = 0; ok && t < tiles; ++t) {
                    const uint32_t st = nk % NST;
                    // Tiled copies where there are tensor maps: this warp's 64 rows as 64 features x 16 or 32 rows each, as far as
                    // rows are seen.  (Rows of a tensor behind the sequence come along; their scores are masked, their V is zeroed.)
                    if (!Q4 && a.box > 0) {
                        const int pages[2] = {page_next[0], page_next[1]};
                        const int row = (it.t0 + t) * 128 + 64 * w, r0 = lane / (D / 64) * a.box, half = lane % (D / 64);      // the copy that this lane makes
                        const bool copies = r0 < 64 && row + r0 < sees;
                        const int p0 = __shfl_sync(0xffffffffu, pages[0], r0 & 31), p1 = __shfl_sync(0xffffffffu, pages[1], r0 & 31);
                        const int mine = r0 < 32 ? p0 : p1;
                        if (!PAGED || !__any_sync(0xffffffffu, copies && (mine < 0 || mine >= a.num_pages))) {
                            if (PAGED && t + 1 < tiles) look_up(it.t0 + t + 1);
                            const int c1 = PAGED ? row + r0 - page_index(row + r0) * a.page_size : it.first + row + r0, c3 = PAGED ? mine : 0;
                            const uint32_t to = (uint32_t)(half * 16384 + (64 * w + r0) * 128);
                            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xffffffffu, copies)) * (uint32_t)a.box * 128u;
                            ok = nk < NST || wait_free(k_empty(st), (nk / NST - 1) & 1);
                            if (!ok) break;
                            if (lane == 0) mbar_expect_tx(k_full(st), bytes);
                            __syncwarp();
                            if (copies && it.t0 + t != a.skip_tile) tc::tma_load_4d(base + C::OFF_K + st * C::KV + to, &map_k, 64 * half, c1, it.head, c3, k_full(st));
                            if (t == 0) { copy_q(); if (!ok) break; }
                            ok = nk < NST || wait_free(v_empty(st), (nk / NST - 1) & 1);
                            if (!ok) break;
                            const bool looks = (it.t0 + t + 1) * 128LL > it.least;
                            const uint32_t vd = base + C::OFF_V + st * C::KV, to_bar = looks ? landed(w) : v_full(st);
                            if (looks) drain();
                            if (lane == 0) mbar_expect_tx(to_bar, bytes);
                            __syncwarp();
                            if (copies) tc::tma_load_4d(vd + to, &map_v, 64 * half, c1, it.head, c3, to_bar);
                            if (looks) push(v_full(st), vd, it.t0 + t, sees - (it.t0 + t) * 128, set, true);
                            ++nk;
                            continue;
                        }
                    }                                      // (a page that does not exist: row by row)
                    locate(it.t0 + t, t + 1 == tiles);
                    if constexpr (Q4) { fetch_rows(codes[0], 0, true); fetch_rows(codes[1], 1, true); }
                    ok = nk < NST || wait_free(k_empty(st), (nk / NST - 1) & 1);
                    if (!ok) break;
                    const uint32_t kd = base + C::OFF_K + st * C::KV, vd = base + C::OFF_V + st * C::KV;
                    if constexpr (Q4) {
                        // parameters: the softmax of the tile that had this place is done (its V is used up, NPAR / 2 tiles ago at the least)
                        const uint32_t ps = nk % C::NPAR;
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const float2 kf = unpack16<false>(k_pair[g]), vf = unpack16<false>(v_pair[g]);
                            float *par = reinterpret_cast<float *>(smem + C::OFF_PAR) + ps * 512 + 64 * w + 32 * g + lane;
                            const float nan = __uint_as_float(0x7fffffffu);
                            par[0] = row_bad[g] ? nan : row_ok[g] ? kf.x : 0.f;
                            par[128] = row_bad[g] ? nan : row_ok[g] ? fmaf(8.f, kf.x, kf.y) : 0.f;
                            par[256] = row_ok[g] ? vf.x : 0.f;
                            par[384] = row_ok[g] ? fmaf(8.f, vf.x, vf.y) : 0.f;
                            float top = row_ok[g] && fabsf(vf.x) < INFINITY ? fabsf(vf.x) : 0.f;
#pragma unroll
                            for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                            if (lane == 0) reinterpret_cast<float *>(smem + C::OFF_PMAX)[ps * 4 + 2 * w + g] = top;
                        }
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(par_full(ps));
                        unpack_rows(kd, 0, codes[0]);
                        fetch_rows(codes[0], 0, false);
                        unpack_rows(kd, 1, codes[1]);
                        fetch_rows(codes[1], 1, false);
                        tc::fence_async_smem();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(k_full(st));
                    } else {
                        copy_rows(kd, it.t0 + t, true);
                        push(k_full(st), 0, -1, 0, 0, false);
                    }
                    if (t == 0) { copy_q(); if (!ok) break; }
                    ok = nk < NST || wait_free(v_empty(st), (nk / NST - 1) & 1);
                    if (!ok) break;
                    if constexpr (Q4) {
                        unpack_rows(vd, 0, codes[0]);
                        unpack_rows(vd, 1, codes[1]);
                        tc::fence_async_smem();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(v_full(st));
                    } else {
                        copy_rows(vd, it.t0 + t, false);
                        push(v_full(st), vd, (it.t0 + t + 1) * 128LL > it.least ? it.t0 + t : -1, 128, set, false);
                    }
                    ++nk;
                }
                drain();
            }
            if (ok && w == 0) fetch(n + 1);
            if (w != 0 && ok) { __syncwarp(); if (lane == 0) tc::mbar_arrive(item_empty(set)); }
        }
        drain();
        cp_wait<0>();
        if (!ok)                                           // a wait ran out: tiled copies may be under way
            for (uint32_t j = nk > (uint32_t)NST ? nk - NST : 0u; j <= nk; ++j) {
                mbar_wait_bounded(k_full(j % NST), (j / NST) & 1, 1u << 8);
                mbar_wait_bounded(v_full(j % NST), (j / NST) & 1, 1u << 8);
            }
        }
    } else {
        // ================= softmax =================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const int s = warp >> 2, wq = warp & 3, row = 32 * wq + lane;       // slot; row of the slot = tensor memory lane
        const uint32_t lane_at = (uint32_t)(32 * wq) << 16;
        const uint32_t tS = t_s(s) + lane_at, tO = t_o(s) + lane_at;
        float2 *const ml = reinterpret_cast<float2 *>(smem + C::OFF_ML);
        uint32_t ns = 0, no = 0, nj = 0, nc = 0, np = 0;   // uses of s_full, o_full, joins, pieces, tiles of keys before the item
        bool ok = true, unread = false;                    // unread: the other slot may still read this slot's sums
        for (uint32_t n = 0; ok; ++n) {
            ok = wait_warp(item_full(n & 1), (n >> 1) & 1, abort_flag, a.wait_limit);
            if (!ok) break;
            const PromptItem &it = s_item[n & 1];
            if (it.rows == 0) break;
            const int cnt = prompt_steps(it, s), other = prompt_steps(it, s ^ 1);
            const int r = row + (it.pair ? 0 : 128 * s);   // row of the unit
            const bool valid = r < it.rows;
            PromptSeq sq;
            sq.first = it.first; sq.past = it.past; sq.len = it.len; sq.n = 0;
            const int my = it.row0 + (valid ? r : 0), tok = div_g(a, my), qh = it.head * a.g + (my - tok * a.g);
            const int lim = valid ? prompt_sees(a, sq, my) : 0;
            float m = -INFINITY, l = 0.f;                  // reference (log2), sum of weights
            float lm = 0.f, sigma = 0.f, sumq = 0.f;       // 4 bits: sum of weight * (least + 8 scale); power of two of the scales; sum of q
            if (Q4 && cnt > 0 && valid) {
                const uint4 *p = reinterpret_cast<const uint4 *>(a.q + (long long)(it.first + tok) * a.q_st + (long long)qh * (D * 2));
                float s0 = 0.f, s1 = 0.f;
#pragma unroll 4
                for (int i = 0; i < D / 8; ++i) {
                    const uint4 u = p[i];
                    const float2 x0 = unpack16<BF>(u.x), x1 = unpack16<BF>(u.y), x2 = unpack16<BF>(u.z), x3 = unpack16<BF>(u.w);
                    s0 += (x0.x + x1.x) + (x2.x + x3.x);
                    s1 += (x0.y + x1.y) + (x2.y + x3.y);
                }
                sumq = a.negate ? -(s0 + s1) : s0 + s1;
            }
            const int dead = !__any_sync(0xffffffffu, valid);                // a warp without rows only keeps step
            for (int i = 0; ok && i < cnt; ++i, ++ns) {
                const int t = it.t0 + (it.pair ? 2 * i + s : i);
                if (i == 0 && unread) {                    // (the join before: the other slot's reads come before these weights)
                    ok = wait_warp(parted, (nj - 1) & 1, abort_flag, a.wait_limit);
                    unread = false;
                    if (!ok) break;
                }
                const uint32_t ps = (np + (uint32_t)(t - it.t0)) % C::NPAR;
                if (Q4) {
                    ok = wait_warp(par_full(ps), ((np + (uint32_t)(t - it.t0)) / C::NPAR) & 1, abort_flag, a.wait_limit);
                    if (!ok) break;
                }
                if (!dead) {
                    const float *const par = reinterpret_cast<const float *>(smem + C::OFF_PAR) + ps * 512;
                    const int vis = lim - t * 128;         // keys of this tile that the row sees
                    const bool masked = !__all_sync(0xffffffffu, vis >= 128);
                    const uint64_t qs2 = pack2f(a.qscale, a.qscale);
                    const bool scales = Q4 && !BF;
#pragma unroll 1
                    for (int h = 0; h < 2; ++h) {          // 64 keys at a time: the first half's product runs under the second's weights
                        ok = wait_warp(s_full(s, h), ns & 1, abort_flag, a.wait_limit);
                        if (!ok) break;
                        tc::fence_after_sync();
                        uint32_t x[64];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            uint32_t z[32];
                            tc::tmem_ld32(tS + 64 * h + 32 * c, z);
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[32 * c + e] = z[e];
                        }
                        tc::tmem_ld_wait();
                        const float *const kpar = par + 64 * h, *const vpar = kpar + 256;
                        const int left = vis - 64 * h;     // keys of this half that the row sees
                        if (Q4) {                          // scale * <q, c - 8> + (least + 8 scale) * sum(q)
                            const uint64_t sq2 = pack2f(sumq, sumq);
#pragma unroll
                            for (int e = 0; e < 64; e += 4) {
                                const float4 ks = *reinterpret_cast<const float4 *>(kpar + e), km = *reinterpret_cast<const float4 *>(kpar + 128 + e);
                                const uint64_t y0 = fma2(pack2f(ks.x, ks.y), pack2(x[e], x[e + 1]), mul2(pack2f(km.x, km.y), sq2));
                                const uint64_t y1 = fma2(pack2f(ks.z, ks.w), pack2(x[e + 2], x[e + 3]), mul2(pack2f(km.z, km.w), sq2));
                                unpack2(y0, x[e], x[e + 1]);
                                unpack2(y1, x[e + 2], x[e + 3]);
                            }
                        }
                        if (masked) {
                            const uint32_t see0 = left >= 32 ? 0xffffffffu : left <= 0 ? 0u : (1u << left) - 1u;
                            const uint32_t see1 = left >= 64 ? 0xffffffffu : left <= 32 ? 0u : (1u << (left - 32)) - 1u;
#pragma unroll
                            for (int e = 0; e < 64; ++e)
                                if (!((e < 32 ? see0 : see1) & (1u << (e & 31)))) x[e] = 0xff800000u;
                        }
                        float sig_new = sigma;
                        if (scales && h == 0) {            // the largest scale among the rows that this query sees
                            const float4 u = *reinterpret_cast<const float4 *>(smem + C::OFF_PMAX + ps * 16);
                            float st = fmaxf(fmaxf(u.x, u.y), fmaxf(u.z, u.w));
                            if (masked && vis < 128) {
                                st = 0.f;
#pragma unroll 1
                                for (int e = 0; e < 128; e += 4) {
                                    const float4 y = *reinterpret_cast<const float4 *>(par + 256 + e);
                                    const float z[4] = {fabsf(y.x), fabsf(y.y), fabsf(y.z), fabsf(y.w)};
#pragma unroll
                                    for (int k = 0; k < 4; ++k) if (e + k < vis && z[k] < INFINITY) st = fmaxf(st, z[k]);
                                }
                            }
                            if (st > sigma) sig_new = __uint_as_float((__float_as_uint(st) + 0x007fffffu) & 0x7f800000u);
                        }
                        // The weights by the reference as it is.  Where one may be above 2^AHEAD -- their sum is, or a score that goes
                        // through the polynomial, which takes no larger ones -- the reference moves to the largest score, and the
                        // warp makes its weights again.  (It moves by the sum too: where it had to be a score beyond AHEAD, scores 5 above
                        // the first ones had every half tile made twice, 4096 keys for 16 heads of 4096 tokens 297 us instead of 201.)
                        uint64_t sum[2], summ;
                        const bool none = masked && left <= 0;
                        for (bool again = false;; again = true) {
                            const float ref = m == -INFINITY ? 0.f : m;
                            const uint64_t nm2 = pack2f(C::SHIFT - ref, C::SHIFT - ref);
                            const float isig = scales ? 1.f / fmaxf(sigma, 1e-30f) : 1.f;
                            const uint64_t is2 = pack2f(isig, isig);
                            float mx = -INFINITY;
                            sum[0] = sum[1] = summ = 0;
                            float4 vs4 = make_float4(0.f, 0.f, 0.f, 0.f), vm4 = vs4;
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t pk[8];
#pragma unroll
                                for (int e = 0; e < 16; e += 2) {
                                    const uint32_t x0 = x[16 * c + e], x1 = x[16 * c + e + 1];
                                    const uint64_t y = fma2(pack2(x0, x1), qs2, nm2);
                                    float2 p;
                                    if (C::POLY >> (e >> 1) & 1) {
                                        mx = max_nan(mx, __uint_as_float(x0), __uint_as_float(x1));
                                        p = exp2_pair<C::DEG>(y);
                                    } else { const float2 v = unpack2f(y); p = make_float2(fast_exp2(v.x), fast_exp2(v.y)); }
                                    const uint64_t pp = pack2f(p.x, p.y);
                                    sum[(e >> 1) & 1] = add2(sum[(e >> 1) & 1], pp);
                                    if (Q4) {
                                        const int at = 16 * c + e;
                                        if (e % 4 == 0) {
                                            vs4 = *reinterpret_cast<const float4 *>(vpar + at);
                                            vm4 = *reinterpret_cast<const float4 *>(vpar + 128 + at);
                                        }
                                        float2 vs = e % 4 == 0 ? make_float2(vs4.x, vs4.y) : make_float2(vs4.z, vs4.w);
                                        float2 vm = e % 4 == 0 ? make_float2(vm4.x, vm4.y) : make_float2(vm4.z, vm4.w);
                                        if (masked) {      // a row that is not seen may hold anything
                                            if (at >= left) vs.x = vm.x = 0.f;
                                            if (at + 1 >= left) vs.y = vm.y = 0.f;
                                        }
                                        summ = fma2(pp, pack2f(vm.x, vm.y), summ);
                                        p = unpack2f(mul2(scales ? mul2(pp, is2) : pp, pack2f(vs.x, vs.y)));
                                    }
                                    pk[e >> 1] = pack16<BF>(p.x, p.y);
                                }
                                tc::tmem_st8(tS + 64 * h + 8 * c, pk);
                            }
                            const float2 both = unpack2f(add2(sum[0], sum[1]));
                            constexpr float kMost = BF ? 256.f : 32768.f;                          // 2^(AHEAD + SHIFT)
                            const float high = mx * a.qscale;
                            const bool far = !none && (m == -INFINITY || !(both.x + both.y <= kMost) || !(high <= ref + C::AHEAD || high == -INFINITY));
                            if (again || !__any_sync(0xffffffffu, far || sig_new != sigma)) break;
                            float top = -INFINITY;
#pragma unroll
                            for (int e = 0; e < 64; e += 2) top = max_nan(top, __uint_as_float(x[e]), __uint_as_float(x[e + 1]));
                            top = none ? -INFINITY : top * a.qscale;                // (nothing seen, whatever the scale)
                            // (each row by its own scores: what it gives does not depend on its neighbours)
                            float mn = far ? max_nan(m, top) : m;
                            if (mn == INFINITY) mn = __uint_as_float(0x7fffffffu);         // (infinity less itself: the row is NaN)
                            float f = mn == m ? 1.f : m == -INFINITY && mn == mn ? 0.f : fast_exp2(m - mn);
                            l *= f; lm *= f;
                            if (scales) { if (sigma > 0.f) f *= sigma / sig_new; sigma = sig_new; }
                            m = mn;
                            if (i > 0 || h == 1) {         // (the half before is on its way into the sum)
                                ok = wait_warp(summed(s), (h ^ 1) & 1, abort_flag, a.wait_limit);
                                if (!ok) break;
                                tc::fence_after_sync();
#pragma unroll 1
                                for (int c = 0; c < D; c += 16) {
                                    uint32_t o[16];
                                    tc::tmem_ld16(tO + c, o);
                                    tc::tmem_ld_wait();
#pragma unroll
                                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                                    tc::tmem_st16(tO + c, o);
                                }
                            }
                        }
                        if (!ok) break;
                        const float2 u = unpack2f(add2(sum[0], sum[1]));
                        l += u.x + u.y;
                        if (Q4) { const float2 v = unpack2f(summ); lm += v.x + v.y; }
                        tc::tmem_st_wait();
                        tc::fence_before_sync();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(p_full(s, h));
                    }
                    if (!ok) break;
                } else {
                    for (int h = 0; h < 2; ++h) {
                        ok = ok && wait_warp(s_full(s, h), ns & 1, abort_flag, a.wait_limit);
                        if (ok && lane == 0) tc::mbar_arrive(p_full(s, h));
                    }
                    if (!ok) break;
                }
            }
            if (!ok) break;
            np += (uint32_t)(it.e1 - it.t0);

            // ---- the unit's end ----
            if (cnt > 0) { ok = wait_warp(o_full(s), no & 1, abort_flag, a.wait_limit); ++no; if (!ok) break; }
            int c0 = 0, c1 = D;                            // this thread's columns
            float fa = 1.f, fb = 0.f;                      // factors of the slots' sums
            float M = m, L = l, add = lm;
            if (Q4 && !BF) fa = sigma;
            if (it.pair) {                                 // each thread joins half the columns of both slots
                if (unread) {                              // (a slot without a tile of this unit has not waited for that yet)
                    ok = wait_warp(parted, (nj - 1) & 1, abort_flag, a.wait_limit);
                    unread = false;
                    if (!ok) break;
                }
                ml[s * 128 + row] = make_float2(m, l);
                if (Q4) s_more[Q4 ? s : 0][Q4 ? row : 0] = make_float2(lm, sigma);
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(joined);
                ok = wait_warp(joined, nj & 1, abort_flag, a.wait_limit);
                if (!ok) break;
                tc::fence_after_sync();
                const float2 o = ml[(s ^ 1) * 128 + row];
                M = max_nan(m, o.x);
                const float f0 = m == -INFINITY ? 0.f : fast_exp2(m - M), f1 = o.x == -INFINITY ? 0.f : fast_exp2(o.x - M);
                L = l * f0 + o.y * f1;
                fa = f0; fb = f1;
                if (Q4) {
                    const float2 e = s_more[Q4 ? s ^ 1 : 0][Q4 ? row : 0];
                    add = lm * f0 + e.x * f1;
                    if (!BF) { fa *= sigma; fb *= e.y; }
                }
                c0 = s * (D / 2); c1 = c0 + D / 2;
            }
            // (behind the join: the other slot's tiles have been looked through by then)
            const bool nf = s_nf[n & 1] != 0;
            const int *const nf_key = reinterpret_cast<const int *>(smem + C::OFF_NF) + (n & 1) * D;
            const uint32_t tB = t_o(s ^ 1) + lane_at;
            float inv = 1.f;
            float *part = nullptr;
            if (it.slot < 0) inv = lim <= 0 ? 0.f : 1.f / L;
            else part = a.slots + (long long)(it.slot + it.piece * it.slot_step) * a.slot_rows * (D + 2);
            unsigned char *const dst = a.out + (long long)(it.first + tok) * a.o_st + (long long)qh * (D * 2);
#pragma unroll 1
            for (int c = c0; c < c1; c += 32) {
                uint32_t o[32];
                if (cnt > 0) { tc::tmem_ld32(tO + c, o); tc::tmem_ld_wait(); }
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = cnt > 0 && M != -INFINITY ? __float_as_uint(__uint_as_float(o[e]) * fa) : 0u;
                if (it.pair && other > 0) {
                    uint32_t o2[32];
                    tc::tmem_ld32(tB + c, o2);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) if (M != -INFINITY) o[e] = __float_as_uint(fmaf(__uint_as_float(o2[e]), fb, __uint_as_float(o[e])));
                }
                if (Q4) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) + add);
                }
                if (nf) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) if (nf_key[c + e] < lim) o[e] = 0x7fffffffu;
                }
                if (valid) {
                    if (part == nullptr) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t y[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                y[k] = pack16<BF>(__uint_as_float(o[e + 2 * k]) * inv, __uint_as_float(o[e + 2 * k + 1]) * inv);
                            *reinterpret_cast<uint4 *>(dst + (c + e) * 2) = make_uint4(y[0], y[1], y[2], y[3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            reinterpret_cast<uint4 *>(part)[(long long)((c + e) >> 2) * a.slot_rows + r] = make_uint4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
            }
            if (it.pair) {
                tc::fence_before_sync();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(parted);
                ++nj;
                unread = true;
            }
            if (part != nullptr) {
                if (valid && (!it.pair || s == 0)) reinterpret_cast<float2 *>(part + (long long)D * a.slot_rows)[r] = make_float2(M, L);
                __threadfence();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(delivered);
                ok = wait_warp(delivered, nc & 1, abort_flag, a.wait_limit);
                if (!ok) break;
                if (tid == 0) {
                    unsigned long long *word = a.tickets + it.slot;
                    const bool last = ticket_arrive(word, a.ticket_tag) + 1 == (unsigned)it.pieces;
                    if (last) *word = 0;
                    __threadfence();
                    s_last = last;
                    tc::mbar_arrive(counted);
                }
                ok = wait_warp(counted, nc & 1, abort_flag, a.wait_limit);
                ++nc;
                if (!ok) break;
                if (s_last && valid) {                     // join the pieces, in order
                    const float *const p0 = a.slots + (long long)it.slot * a.slot_rows * (D + 2);
                    const long long step = (long long)it.slot_step * a.slot_rows * (D + 2);
                    float top = -INFINITY, total = 0.f;
                    for (int p = 0; p < it.pieces; ++p) top = max_nan(top, __ldcg(reinterpret_cast<const float2 *>(p0 + p * step + (long long)D * a.slot_rows) + r).x);
                    for (int p = 0; p < it.pieces; ++p) {
                        const float2 e = __ldcg(reinterpret_cast<const float2 *>(p0 + p * step + (long long)D * a.slot_rows) + r);
                        total = fmaf(e.y, exp2_diff(e.x, top), total);
                    }
                    const float scale = lim <= 0 ? 0.f : 1.f / total;
#pragma unroll 1
                    for (int c = c0; c < c1; c += 16) {
                        float acc[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) acc[e] = 0.f;
                        for (int p = 0; p < it.pieces; ++p) {
                            const float *const pp = p0 + p * step;
                            const float f = exp2_diff(__ldcg(reinterpret_cast<const float2 *>(pp + (long long)D * a.slot_rows) + r).x, top);
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const float4 u = __ldcg(reinterpret_cast<const float4 *>(pp) + (long long)((c + e) >> 2) * a.slot_rows + r);
                                acc[e] = fmaf(u.x, f, acc[e]); acc[e + 1] = fmaf(u.y, f, acc[e + 1]);
                                acc[e + 2] = fmaf(u.z, f, acc[e + 2]); acc[e + 3] = fmaf(u.w, f, acc[e + 3]);
                            }
                        }
#pragma unroll
                        for (int e = 0; e < 16; e += 8)
                            *reinterpret_cast<uint4 *>(dst + (c + e) * 2) =
                                make_uint4(pack16<BF>(acc[e] * scale, acc[e + 1] * scale), pack16<BF>(acc[e + 2] * scale, acc[e + 3] * scale),
                                           pack16<BF>(acc[e + 4] * scale, acc[e + 5] * scale), pack16<BF>(acc[e + 6] * scale, acc[e + 7] * scale));
                    }
                }
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(item_empty(n & 1));
        }
    }
    __syncwarp();
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    if (warp == 10) tc::tmem_dealloc(tmem, 512);
}

}  // namespace moa
