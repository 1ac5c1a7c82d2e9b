// Attention of one or a few new rows per sequence over the paged KV cache (Voltron Section 2.1, decode
// phase).
//
//   o_c = sum_j softmax_j(scale q_c . k_j) v_j over the positions of column c, one pass over K and V with a
//   running maximum m (log2 units), sum l and o per column.  The columns of a sequence's KV head are its new
//   rows times the query heads of the group (column i group + h: row i, head h).
//
// What bounds it: every K and V byte is read once and meets a few columns (one FLOP a byte and column), so
// HBM.  The work of a unit (a sequence's KV head and up to 8 NT of its columns) is cut into steps of 16
// positions; the steps of all units form one line, and CTA c takes its c-th equal part, whatever the
// sequences' lengths are.  They are known on the device only, so that a captured launch serves any
// lengths.  A unit counts kUnitCost steps more than it has, as its queries and its result take that time.
// Inside a CTA step i goes to warp i % 4 (short units: whole units to a warp), each with its own ring of
// asynchronous 16-byte copies (K and V rows gathered through the page table), so no barrier stands in the
// stream; 128 KB or more a SM are in flight.  A unit that several CTAs share is joined by the last of them
// to finish: partial (m, l, o) in a workspace, added in CTA order, so a result does not depend on timing.
//
// Products run on mma.sync m16n8k16 (tcgen05 would need 64 or more rows where there are 1 to 16):
//   S [16 columns x 8 keys] = Q . K^T       A: Q from registers, B: K rows by ldmatrix
//   O^T [16 dims x 8 columns] += V^T . P^T  A: V by ldmatrix.trans, B: P as S leaves it in registers
// P is cut into two 16-bit terms, hi = round(p) and lo = round(p - hi), two products each: the weights
// then carry 16 (bf16) or 22 (fp16) bits and the output's own rounding is the only one that counts.  fp16 has
// no steps below 2^-24, so its p goes up to 2^15: a weight loses at most 2^-40 of the largest one, where at
// a largest p of 1 a history of 40,000 small weights beside a large one came out 98% short.
//
// Over a pool of codes (paged_mx.cuh) a step has 32 positions, about as many bytes, and both products are of fp16, whatever
// the rows' type: a code is an fp16 number, and the scales of 32 dimensions stay outside,
//   S = sum_b scale_K[key][b] (Q_b . codes_b)     a sum for each 32 dimensions b, multiplied and added in fp32
//   O_b += (P scale_V[.][b] / unit) . codes_b     weights for each b; unit: the largest scale of V that the column has
//                                                 attended to, by which O is rescaled when it grows
// Columns of one row share the unit.  Of several rows each has its own: what a column does not attend to, such as the new rows
// behind its own, may be any powers above the rest and would leave its weights no bits.
// bf16 queries become fp16 times a power of two of their row.  Weights have two terms, 22 bits (one, for bf16 rows, left outputs
// 9e-4 of their size off beside their own rounding, two 7e-5, for 1 us of 55 on the long history below).  m moves only when P would
// pass 2^15, down to 2^12, so that a weight loses at most 2^-37 of the largest one, times the largest value.  What it costs beside
// the 16-bit pool's kernel are the conversions: 390 instructions a 16 positions and warp, which fit beside the copies at the
// memory's rate.
//
// Measured: one history of 131,000 positions, 8 KV heads of 4, dh 128: 92 us, 5830 GB/s (86% of a copy's rate: the
// start, the last steps and the join of 38 parts a head are the rest); 64 sequences of up to 8191, some idle: 47 us, 5310
// GB/s; 16 of 500 to 4096 with 32 KV heads and a window of 1024: 46 us, 5290 GB/s; 128 positions of 8 heads: 5.6 us, all
// of it latency (lengths, table, first rows, merge).  Codes: 56 us (e4m3, bf16), 39 and 40 us on the same three; from 131,000 to
// 524,000 positions each further position comes at 6800 to 6900 GB/s, and 15 us are start, merge and join.
#pragma once

#include <cuda_runtime.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "paged_mx.cuh"
#include "tcgen05.cuh"

namespace vt {

constexpr int kPdWarps = 4, kPdThreads = kPdWarps * 32;
constexpr int kPdRing = 96 * 1024;           // bytes of the four warps' rings, at most
constexpr int kPdSoloUnits = 2;              // (see kSoloSteps)
// Codes: parts that are joined by several threads an item (fp16; 130,000 positions, 38 parts a head, 66.0 us by one, 63.1 by
// several; 9 parts 56.7 and 56.3, 57.6 and 57.0; 5 parts 59.4 and 59.7; 64 ragged sequences, 2 to 3 parts, 40.9 and 41.9: the longer
// code comes from far away).
constexpr int kPdManyParts = 8;
// Codes: units begin at the least scale that an entry may have.  Where columns have their own, V's scales are kept times 2^kPdShift and weights over the
// unit times 2^-kPdShift, so that neither a weight of 2^15 over the least unit nor a scale of 2^119 passes the largest fp32 number.
constexpr float kPdLeastScale = 0x1p-117f;
constexpr int kPdShift = 6;
// int8 codes of bf16 rows have scales up to 2^119, and a score's sum without its scales goes up to 2^25 (queries below 2^11, 128 codes
// up to 127): the scales of K are then kept times 2^-kPdKeyShift, and the factor of the scores times 2^kPdKeyShift; not where a query is
// past 2^kPdLargeQuery, whose factor is large itself.
constexpr int kPdKeyShift = 17, kPdLargeQuery = 90;

template <class Src, int DH, int NT>
struct PdGeom {
    static constexpr bool kMx = Src::kMx;
    static constexpr bool kWideKeys = Src::kWide;
    static constexpr int kCtas = 2;                                                // an SM
    static constexpr int kKeys = kMx ? 32 : 16;                                  // positions of a step
    static constexpr int kRow = DH * Src::kBytes;                                // bytes of a K or V row
    static constexpr int kSide = kKeys * kRow;                                   // of a step's K
    static constexpr int kScales = kMx ? kKeys * (DH / kMxBlock) : 0;            // of its scales
    static constexpr int kStage = 2 * (kSide + kScales);                         // K rows, V rows, K scales, V scales
    static constexpr int kStages = kMx ? (DH == 128 ? 3 : 6) : kPdRing / (kPdWarps * kStage);
    static constexpr int kRing = kPdWarps * kStages * kStage;
    static constexpr int kFloats = kMx ? 2 * kKeys * (DH / kMxBlock) : 8 * DH;   // of a warp: a step's scales; results to be merged
    static constexpr size_t kSmem = kRing + (size_t)kPdWarps * kFloats * 4;
    // A unit's queries, merge and result cost as much as this many steps (measured, 16 bits: 64 ragged sequences 75 us at 0,
    // 56 at 4, 47 at 8 to 24, 50 at 32).
    static constexpr int kUnitCost = 256 / kKeys;
    // What a CTA takes at least: where the largest unit costs no more than kWhole (16 bits: 12 steps), that much, so that few
    // are split and joined (8 heads of 128 positions: 5.4 us, split 6.7; at 48, units of 20 to 30 steps lost up to 2 us);
    // otherwise kMinSteps.  (Codes, steps of 32: 8 heads of 128 positions 6.2 both ways, of 400 9.7 and 9.5 split, 30 sequences of 800
    // 22.6 and 22.4: it does not count there.)
    static constexpr int kMinSteps = 256 / kKeys, kWhole = 448 / kKeys;
    // Where the largest unit has no more steps than kSoloSteps and there are kPdSoloUnits or more such units for every CTA,
    // each warp has units of its own: merging four warps would cost more than the steps.  Measured (16 bits), merged and alone:
    // 168 sequences of 1 to 3 positions, 32 heads, 38 and 15 us; 1024 sequences of 61 to 65 positions, 8 KV heads, 87 and 56;
    // 24 sequences of 201 to 251, 32 heads, 24 and 22.  At 32 steps 300 sequences of 21 to 501 positions lost (51 to 63).
    // Codes (e4m3, fp16), merged and alone: the first three 58 and 21, 110 and 54, 24 and 21; at 16 steps the last 51 and 54.
    static constexpr int kSoloSteps = 256 / kKeys;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool full) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(full ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(addr)
                 : "memory");
}
// Where 16-byte chunk x of row r of codes lies in its row of CPR chunks: 8 rows of one chunk (ldmatrix), and 4 rows of one
// pair of chunks (the 32 dimensions of a scale), fall into different banks.
template <int CPR>
__device__ __forceinline__ uint32_t pd_chunk(int r, int x) {
    return (uint32_t)((x ^ ((CPR == 8 ? (r & 3) << 1 : r & 2) | ((r >> 2) & 1))) << 4);
}
__device__ __forceinline__ void sts32(uint32_t addr, float v) { asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory"); }
// Two floats in a register pair, one or two such pairs.
__device__ __forceinline__ uint64_t lds1x64(uint32_t addr) {
    uint64_t v;
    asm volatile("ld.shared.b64 %0, [%1];" : "=l"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void lds2x64(uint32_t addr, uint64_t (&v)[2]) {
    asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(addr) : "memory");
}
// 1 / x of a power of two; 2^e.
__device__ __forceinline__ float pd_inverse(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }
__device__ __forceinline__ constexpr float pd_power(int e) { return e < 0 ? 1.f / (float)(1 << -e) : (float)(1 << e); }
// 2^x; over codes without the steps that keep results below 2^-126, which are nothing beside weights up to 2^12 and more.
template <class Src>
__device__ __forceinline__ float pd_exp2(float x) {
    if constexpr (Src::kMx) {
        float y;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
        return y;
    }
    return exp2f(x);
}
template <class T>
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (std::is_same<T, __half>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
            : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// The product alone, of fp16.
__device__ __forceinline__ void mma16816_new(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}

// A sequence's new rows, and the positions [beg, end) that they attend to (end 0: none), in steps of kKeys.
template <class G>
struct PdSeq {
    static constexpr int KEYS = G::kKeys;
    int row0, rows, len, beg, end, tiles, steps;
    bool over;
    // tiles: units of a KV head, of `cols` columns
    template <bool ROWS>
    __device__ __forceinline__ void open(const PagedAttnArgs& a, int b, int cols) {
        len = paged_len(a.c, b);
        row0 = b;
        rows = 1;
        over = false;
        if (ROWS) {
            row0 = paged_start(a.c, b, a.n_rows);
            rows = max(0, paged_start(a.c, b + 1, a.n_rows) - row0);
            over = rows > a.rows_most && len >= 0;  // the next launch's (idle slots' zeros are this one's)
            if (over) rows = 0;
        }
        end = len < 0 || rows == 0 ? 0 : min(len + rows, a.c.cap);
        beg = a.window > 0 ? max(0, len + 1 - a.window) : 0;
        if (beg >= end) beg = end = 0;  // a length past the table may leave the window nothing
        steps = (end + KEYS - 1) / KEYS - beg / KEYS;
        tiles = (rows * a.group + cols - 1) / cols;
    }
    // its share of the line, for one KV head
    __device__ __forceinline__ int64_t cost() const { return steps > 0 ? (int64_t)tiles * (steps + G::kUnitCost) : 0; }
};

// Where a walk over the steps of the units stands: unit u of sequence b (KV head u / tiles), step i - kUnitCost.
template <bool ROWS, int COLS, class G>
struct PdCursor {
    int b, u, i;
    PdSeq<G> s;
    __device__ __forceinline__ void open(const PagedAttnArgs& a, int seq) {
        b = seq;
        s.steps = 0;
        if (b < a.c.n_seqs) s.template open<ROWS>(a, b, COLS);
    }
    // on to the next unit that has steps
    __device__ __forceinline__ void next(const PagedAttnArgs& a) {
        i = 0;
        if (s.steps > 0 && ++u < a.c.n_kv_heads * s.tiles) return;
        u = 0;
        do open(a, b + 1);
        while (s.steps == 0 && b < a.c.n_seqs);
    }
};

template <class Src, int DH, int NT, bool ROWS>
__global__ void __launch_bounds__(kPdThreads, PdGeom<Src, DH, NT>::kCtas) k_paged_decode(const __grid_constant__ PagedAttnArgs a) {
    using T = typename Src::T;
    using E = Elem<T>;
    using G = PdGeom<Src, DH, NT>;
    constexpr uint32_t FULL = G::kKeys == 32 ? 0xffffffffu : 0xffffu;
    constexpr int KEYS = G::kKeys, NB = DH / kMxBlock;
    constexpr int S = G::kStages, CPR = G::kRow / 16, RPI = 32 / CPR;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t s_sum[kPdWarps], s_before[kPdWarps + 1];
    __shared__ int s_seq[kPdWarps + 1], s_last, s_max[kPdWarps];
    __shared__ float s_ml[2][kPdWarps][8 * NT];
    __shared__ uint32_t s_mask[kPdWarps][S];
    __shared__ int s_free[kPdWarps];
    const PagedView& c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    constexpr int COLS = 8 * NT;
    pdl_wait();
    pdl_launch_dependents();

    // ---- this CTA's part of the line: thread t sums the sequences [t ch, (t + 1) ch)
    const int ch = (c.n_seqs + kPdThreads - 1) / kPdThreads;
    int64_t mine = 0;
    int largest = 0;
    bool idle = false, over = false;
    for (int b = tid * ch; b < min(c.n_seqs, (tid + 1) * ch); ++b) {
        PdSeq<G> s;
        s.template open<ROWS>(a, b, COLS);
        if (blockIdx.x == 0 && s.rows > 0 && s.len >= 0 && s.len + s.rows > c.cap) set_status(c.status, VT_DEV_KV_OVERFLOW);
        idle |= s.steps == 0 && !s.over;
        over |= s.over;
        largest = max(largest, s.steps);
        mine += s.cost();
    }
    largest = __reduce_max_sync(0xffffffffu, largest);
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 31) {
        s_sum[warp] = upto;
        s_max[warp] = largest;
    }
    const bool any_idle = __syncthreads_or(idle);
    if (ROWS && blockIdx.x == 0 && a.over) {
        const bool any_over = __syncthreads_or(over);
        if (tid == 0) *a.over = any_over;
    }
    int64_t total = 0;
    for (int w = 0; w < kPdWarps; ++w) {
        if (w < warp) upto += s_sum[w];
        total += s_sum[w];
        largest = max(largest, s_max[w]);
    }
    if (any_idle)  // rows that attend to nothing get zeros
        for (int b = blockIdx.x; b < c.n_seqs; b += gridDim.x) {
            PdSeq<G> s;
            s.template open<ROWS>(a, b, COLS);
            if (s.steps == 0)
                for (int r = s.row0; r < s.row0 + s.rows; ++r)
                    for (int e = tid; e < a.n_heads * DH / 8; e += kPdThreads)
                        reinterpret_cast<uint4*>(a.out + r * a.out_ld)[e] = make_uint4(0u, 0u, 0u, 0u);
        }
    const int64_t line = total * c.n_kv_heads;
    const bool solo = largest <= G::kSoloSteps && line >= (int64_t)kPdSoloUnits * gridDim.x * (largest + G::kUnitCost);
    const int64_t per = max(paged_div(line + gridDim.x - 1, gridDim.x),
                            (int64_t)(largest + G::kUnitCost <= G::kWhole ? largest + G::kUnitCost : G::kMinSteps));
    int64_t t0 = blockIdx.x * per, t1 = min(line, t0 + per);
    if (t0 >= t1) return;
    // the sequences that hold t0 and, for warps with units of their own, the beginnings of their parts and the last one's end
    const int64_t per_warp = solo ? paged_div(t1 - t0 + kPdWarps - 1, kPdWarps) : 0;
    for (int k = 0; k <= (solo ? kPdWarps : 0); ++k) {
        const int64_t head = paged_div(min(t1, t0 + k * per_warp), c.n_kv_heads);
        if (upto - mine <= head && head < upto) {  // the thread whose sequences hold it
            int64_t before = upto - mine;
            int b = tid * ch;
            for (;; ++b) {
                PdSeq<G> s;
                s.template open<ROWS>(a, b, COLS);
                if (head < before + s.cost()) break;
                before += s.cost();
            }
            s_seq[k] = b;
            s_before[k] = before;
        }
    }
    __syncthreads();

    // ---- the copies.  Step k of the CTA's part (unit costs left out) is warp k % 4's, or each warp has its own part, from
    // the first unit that begins in it to the first that begins in the next.
    const int stride = solo ? 1 : kPdWarps;
    PdCursor<ROWS, COLS, G> at;  // of the whole CTA, or of the warp
    if (solo) {
        auto unit_start = [&](int64_t pos, int k) {  // of the first unit that begins at pos or after it
            if (pos >= line) return line;
            PdSeq<G> s;
            s.template open<ROWS>(a, s_seq[k], COLS);
            const int64_t r = pos - s_before[k] * c.n_kv_heads, cost = s.steps + G::kUnitCost;
            return pos + (cost - 1 - (r + cost - 1 - paged_div(r + cost - 1, cost) * cost));
        };
        const int64_t w0 = unit_start(min(t1, t0 + warp * per_warp), warp);
        const int64_t w1 = unit_start(min(t1, t0 + (warp + 1) * per_warp), warp + 1);
        if (w0 >= w1) return;  // (no barrier of the whole CTA follows)
        at.open(a, s_seq[warp]);
        const int64_t r = w0 - s_before[warp] * c.n_kv_heads, cost = at.s.steps + G::kUnitCost;
        at.u = (int)paged_div(r, cost) - 1;  // the unit before it, unless it is the sequence's first
        at.i = 0;
        if (at.u < 0) at.u = 0;
        else at.next(a);
        t0 = w0;
        t1 = w1;
    } else {
        at.open(a, s_seq[0]);
        const int64_t r = t0 - s_before[0] * c.n_kv_heads;
        at.u = (int)paged_div(r, at.s.steps + G::kUnitCost);
        at.i = (int)(r - (int64_t)at.u * (at.s.steps + G::kUnitCost));
    }
    PdCursor<ROWS, COLS, G> ld = at;               // of this warp's copies: the unit of its next step
    int64_t ld_now = t0;                        // where that unit's part begins in the line
    int ld_i, ld_n, ld_skip = solo ? 0 : warp;  // next step of the unit, steps of it here, steps until this warp's next
    int64_t ld_hoff = 0, ld_soff = 0;           // codes: its KV head's offsets
    auto ld_unit = [&]() {                      // the steps [first, n) of the unit that lie in this part
        const int first = max(0, ld.i - G::kUnitCost);
        ld_n = (int)min((int64_t)ld.s.steps, t1 - ld_now + ld.i - G::kUnitCost);
        ld_i = first;
        if constexpr (Src::kMx) {
            ld_hoff = (ld.u / ld.s.tiles) * c.head_stride;
            ld_soff = (ld.u / ld.s.tiles) * a.scale_head;
        }
    };
    // moves to this warp's next step; false: none
    auto ld_seek = [&]() -> bool {
        while (ld_i + ld_skip >= ld_n) {
            if (ld_n > ld_i) ld_skip -= ld_n - ld_i;
            ld_now += ld.s.steps + G::kUnitCost - ld.i;
            if (ld_now >= t1) return false;
            ld.next(a);
            ld_unit();
        }
        ld_i += ld_skip;
        ld_skip = 0;
        return true;
    };
    ld_unit();
    bool more = ld_seek();
    const uint32_t ring = smem_u32(smem) + (uint32_t)(warp * S * G::kStage);
    int page = 0;         // lane r < KEYS: the table's entry for row r of the next step to load, whatever it holds;
    bool needed = false;  // whether that row is attended to is known apart from it
    auto look_up = [&]() {
        const int p = more ? (ld.s.beg / KEYS + ld_i) * KEYS + lane : -1;
        needed = more && lane < KEYS && p >= ld.s.beg && p < ld.s.end;
        if (needed) page = c.tables[(int64_t)ld.b * c.per_seq + (p >> c.page_shift)];
    };
    look_up();
    int st_load = 0;
    // codes: a lane's 16 bytes of the first rows (RPI of them a copy), and of the scales, which hold those of PER positions
    constexpr int PER = Src::kMx ? 16 / NB : 1, CHUNKS = KEYS / PER;
    const int64_t mine_at = (lane / CPR) * c.pos_stride + (lane % CPR) * 16, hop = RPI * c.pos_stride;
    const uint8_t *k_at = reinterpret_cast<const uint8_t*>(a.kpool) + mine_at, *v_at = reinterpret_cast<const uint8_t*>(a.vpool) + mine_at;
    const uint8_t* s_at = lane % (2 * CHUNKS) < CHUNKS ? a.kscale : a.vscale;
    const uint32_t mine_to = (uint32_t)((lane / CPR) * G::kRow) + pd_chunk<CPR>(lane / CPR, lane % CPR);
    auto load_step = [&]() {
        if (more) {
            const bool on = needed && (unsigned)page < (unsigned)c.n_pages;
            if (needed && !on) set_status(c.status, VT_DEV_BAD_PAGE);
            const uint32_t mask = __ballot_sync(0xffffffffu, on);
            if (lane == 0) s_mask[warp][st_load] = mask;
            const uint32_t dst = ring + (uint32_t)(st_load * G::kStage);
            const int chunk = lane % CPR;
            if constexpr (!Src::kMx) {
                const int p = (ld.s.beg / KEYS + ld_i) * KEYS + lane;
                const int64_t off = on ? page * c.page_stride + (ld.u / ld.s.tiles) * c.head_stride + (p & (c.page_size - 1)) * c.pos_stride
                                       : -1;
#pragma unroll
                for (int r0 = 0; r0 < KEYS; r0 += RPI) {
                    const int r = r0 + lane / CPR;
                    const int64_t o = __shfl_sync(0xffffffffu, off, r);
                    const uint32_t d = dst + (uint32_t)(r * G::kRow + ((chunk ^ (r & 7)) << 4));
                    const int64_t src = (o < 0 ? 0 : o) + chunk * 8;  // rows without a position are filled with zeros
                    cp_async16(d, a.kpool + src, o >= 0);
                    cp_async16(d + KEYS * G::kRow, a.vpool + src, o >= 0);
                }
            } else {
                const int first = (ld.s.beg / KEYS + ld_i) * KEYS;
                if (mask == FULL && c.page_size >= 16) {  // 16 rows of one page
                    int pg = 0;
                    int64_t at = 0;
#pragma unroll
                    for (int h = 0; h < KEYS; h += 16) {
                        if (h == 0 || c.page_size == 16) {
                            pg = __shfl_sync(0xffffffffu, page, h);
                            at = pg * c.page_stride + ld_hoff + ((first + h) & (c.page_size - 1)) * c.pos_stride;
                        }
                        const uint8_t *ksrc = k_at + at, *vsrc = v_at + at;
#pragma unroll
                        for (int r = h; r < h + 16; r += RPI) {
                            const uint32_t d = dst + (uint32_t)(r * G::kRow) + (mine_to ^ (CPR == 8 && (r & 4) ? 16u : 0u));
                            cp_async16(d, ksrc);
                            cp_async16(d + G::kSide, vsrc);
                            ksrc += hop;
                            vsrc += hop;
                        }
                        at += 16 * c.pos_stride;
                    }
                    const int x = lane % CHUNKS * PER;  // the first position of this lane's scales
                    if (c.page_size == 16) pg = __shfl_sync(0xffffffffu, page, x);
                    if (lane < 2 * CHUNKS)
                        cp_async16(dst + (uint32_t)(2 * G::kSide + lane * 16),
                                   s_at + (pg * a.scale_page + ld_soff + ((first + x) & (c.page_size - 1)) * NB));
                } else {
#pragma unroll 1
                    for (int h = 0; h < KEYS; h += 8) {  // a page holds 8 positions or more
                        const uint32_t bits = (mask >> h) & 0xffu;
                        const int pg = __shfl_sync(0xffffffffu, page, h + max(0, __ffs(bits) - 1));
                        int64_t at = bits ? pg * c.page_stride + ld_hoff + ((first + h) & (c.page_size - 1)) * c.pos_stride : 0;
#pragma unroll
                        for (int k = 0; k < 8; k += RPI) {
                            const uint32_t d = dst + (uint32_t)((h + k) * G::kRow) + (mine_to ^ (CPR == 8 && (k & 4) ? 16u : 0u));
                            const bool full = (bits >> (k + lane / CPR)) & 1u;  // rows without a position are filled with zeros
                            cp_async16(d, full ? k_at + at : k_at - mine_at, full);
                            cp_async16(d + G::kSide, full ? v_at + at : v_at - mine_at, full);
                            at += hop;
                        }
                    }
                    const int x = lane % CHUNKS * PER, some = __ffs((mask >> x) & ((1u << PER) - 1u));
                    const int pg = __shfl_sync(0xffffffffu, page, x + max(0, some - 1));
                    const int64_t at = some ? pg * a.scale_page + ld_soff + ((first + x) & (c.page_size - 1)) * NB : 0;
                    if (lane < 2 * CHUNKS) cp_async16(dst + (uint32_t)(2 * G::kSide + lane * 16), s_at + at, some > 0);
                }
            }
            ld_skip = stride;
            more = ld_seek();
            look_up();
        }
        cp_async_commit();
        st_load = st_load + 1 == S ? 0 : st_load + 1;
    };
#pragma unroll
    for (int s = 0; s < S - 1; ++s) load_step();

    // ---- the steps, unit by unit
    int st = 0, skip = solo ? 0 : warp;  // skip: steps until this warp's next
    // where warp w leaves its results to be merged.  Codes: in the stage that it fills next
    auto merge_at = [&](int w) {
        return reinterpret_cast<float*>(smem + (Src::kMx ? (w * S + s_free[w]) * G::kStage : G::kRing + w * 8 * DH * 4));
    };
    const uint32_t fs = smem_u32(smem) + (uint32_t)(G::kRing + warp * G::kFloats * 4);  // codes: a step's scales
    auto dim_of = [&](int i, int e) { return 16 * i + (Src::kMx ? 2 * g + (e >> 1) : g + 8 * (e >> 1)); };  // of o[i][.][e]
    for (int64_t now = t0; now < t1;) {
        // steps [i0, i0 + n) of the unit are in this part
        const int i0 = max(0, at.i - G::kUnitCost), n = (int)min((int64_t)at.s.steps, t1 - now + at.i - G::kUnitCost) - i0;
        const int64_t u0 = now - at.i + G::kUnitCost;  // where its steps begin in the line
        now += at.s.steps + G::kUnitCost - at.i;
        if (n <= 0) {
            at.next(a);
            continue;
        }
        const int kvh = at.u / at.s.tiles, c0 = (at.u - kvh * at.s.tiles) * COLS, nc = min(COLS, at.s.rows * a.group - c0);
        // column c0 + c: its element offset in q and out
        auto col_at = [&](int c, int64_t ld) {
            const int row = ROWS ? (c0 + c) / a.group : 0;
            return (at.s.row0 + row) * ld + (int64_t)(kvh * a.group + c0 + c - row * a.group) * DH;
        };
        uint32_t q[DH / 16][4];
        float qs[NT];  // what a score is multiplied by
#pragma unroll
        for (int x = 0; x < NT; ++x) qs[x] = a.scale_log2;
        // codes: a column of o counts in the largest scale of V that it has attended to (single tokens: one for all columns);
        // least: of the warp's columns
        float unit[NT], least = kPdLeastScale;
#pragma unroll
        for (int x = 0; x < NT; ++x) unit[x] = kPdLeastScale;
        float k_by = 1.f;  // codes: what K's scales are multiplied by
        bool large = false;
        int last_key[NT];  // of this lane's columns, in the steps' keys
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool on = x < NT && g + 8 * x < nc;
            if constexpr (!Src::kMx) {
                const uint16_t* src = a.q + (on ? col_at(g + 8 * x, a.q_ld) : 0) + 2 * t;
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    q[k][x] = on ? *reinterpret_cast<const uint32_t*>(src + k * 16) : 0u;
                    q[k][2 + x] = on ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8) : 0u;
                }
            } else {  // product k is over the dimensions 32 (k / 2) + 8 t + 4 (k % 2) + 0 .. 3 of its four lanes
                const uint16_t* src = a.q + (on ? col_at(g + 8 * x, a.q_ld) : 0) + 8 * t;
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    const uint2 w = on ? *reinterpret_cast<const uint2*>(src + (k >> 1) * 32 + (k & 1) * 4) : make_uint2(0u, 0u);
                    q[k][x] = w.x;
                    q[k][2 + x] = w.y;
                }
                if constexpr (!std::is_same<T, __half>::value) {  // bf16 to fp16: the row's largest is brought to 2^10 .. 2^11
                    uint32_t most = 0u;
#pragma unroll
                    for (int k = 0; k < DH / 16; ++k) {
                        most = max(most, max(q[k][x] & 0x7fffu, (q[k][x] >> 16) & 0x7fffu));
                        most = max(most, max(q[k][2 + x] & 0x7fffu, (q[k][2 + x] >> 16) & 0x7fffu));
                    }
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
                    most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
                    const int up = 10 - max((int)(most >> 7) - 127, -116);
                    const float f = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
                    for (int k = 0; k < DH / 16; ++k)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const float2 v = E::unpack(q[k][e + x]);
                            q[k][e + x] = Elem<__half>::pack(v.x * f, v.y * f);
                        }
                    // (not infinite: its product with a score of 0 is 0)
                    if (x < NT) qs[x] = fminf(a.scale_log2 * __uint_as_float((uint32_t)(127 - up) << 23), 3.4028235e38f);
                    large |= -up >= kPdLargeQuery;
                }
            }
            if (x < NT) last_key[x] = ROWS ? at.s.len + (c0 + g + 8 * x) / a.group : 0;
        }
        if constexpr (G::kWideKeys)  // room for 2^25 times the largest scale, but not where a score's factor has none
            if (!__any_sync(0xffffffffu, large)) {
                k_by = pd_power(-kPdKeyShift);
#pragma unroll
                for (int x = 0; x < NT; ++x) qs[x] = fminf(qs[x] * pd_power(kPdKeyShift), 3.4028235e38f);
            }
        float m[NT], l[NT], o[DH / 16][NT][4];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            m[x] = -INFINITY;
            l[x] = 0.f;
#pragma unroll
            for (int i = 0; i < DH / 16; ++i) o[i][x][0] = o[i][x][1] = o[i][x][2] = o[i][x][3] = 0.f;
        }
        int k0 = skip;
        for (; k0 < n; k0 += stride) {
            const int p0 = ROWS ? (at.s.beg / KEYS + i0 + k0) * KEYS : 0;  // the step's first position
            load_step();
            cp_async_wait<S - 1>();
            __syncwarp();
            const uint32_t ks = ring + (uint32_t)(st * G::kStage), vs = ks + G::kSide;
            const uint32_t mask = s_mask[warp][st];
            const int lr = ((lane >> 4) << 3) + (lane & 7), lc = (lane >> 3) & 1;  // ldmatrix: row, chunk of a pair
            constexpr int NS = KEYS / 8;
            float s[NS][4] = {};
            float v_most = 0.f, grown = 1.f;  // codes: the step's largest scale of V, where some column's unit is less
            if constexpr (!Src::kMx) {
#pragma unroll
                for (int k = 0; k < DH / 16; ++k) {
                    uint32_t kb[4];
                    ldsm4(ks + (uint32_t)(lr * G::kRow + (((2 * k + lc) ^ (lr & 7)) << 4)), kb);
                    mma16816<T>(s[0], q[k], kb[0], kb[1]);
                    mma16816<T>(s[1], q[k], kb[2], kb[3]);
                }
            } else {
                // The step's scales as floats, [K, V][pair of positions][block][position], each worked out by one lane; those of V
                // over the unit or, where columns have units of their own, times 2^kPdShift.
                constexpr int WORDS = 2 * KEYS * NB / 4, PASSES = (WORDS + 31) / 32;  // of 4 bytes; half of them K's
                float f[PASSES][4];
                bool odd = false;
#pragma unroll
                for (int j = 0; j < PASSES; ++j) {
                    const int i = (32 * j + lane) % WORDS;
                    const bool of_v = i >= WORDS / 2;
                    uint32_t w = lds32(vs + G::kSide + (uint32_t)(i * 4));
                    if (of_v && mask != FULL) {  // what nothing attends to may be anything
                        const uint32_t bits = mask >> (i % (WORDS / 2) * (4 / NB));
                        if (NB == 4)
                            w = bits & 1u ? w : 0u;
                        else
                            w &= (bits & 1u ? 0xffffu : 0u) | (bits & 2u ? 0xffff0000u : 0u);
                    }
                    float most = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) most = fmaxf(most, f[j][e] = mx_scale(w, e));
                    odd |= of_v ? most > least : most == INFINITY;
                }
                if (__any_sync(0xffffffffu, odd)) {  // (an infinite scale is NaN's: it sets no unit)
                    float most = 0.f;
#pragma unroll
                    for (int j = 0; j < PASSES; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (f[j][e] == INFINITY) f[j][e] = __int_as_float(0x7fc00000);
                            if ((32 * j + lane) % WORDS >= WORDS / 2) most = fmaxf(most, f[j][e]);
                        }
                    v_most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
                    if (!ROWS && v_most > least) {
                        grown = least * pd_inverse(v_most);
                        unit[0] = least = v_most;
                    }
                }
#pragma unroll
                for (int j = 0; j < PASSES; ++j) {
                    const int i = (32 * j + lane) % WORDS, at = i % (WORDS / 2);
                    const bool of_v = i >= WORDS / 2;
                    const float by = !of_v ? k_by : ROWS ? pd_power(kPdShift) : pd_inverse(unit[0]);
                    const uint32_t to = fs + (uint32_t)(of_v ? KEYS * NB * 4 : 0);
                    if (NB == 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) sts32(to + (uint32_t)((at >> 1) * 32 + e * 8 + (at & 1) * 4), f[j][e] * by);
                    } else {
                        sts128_at(to + (uint32_t)(at * 16), __float_as_uint(f[j][0] * by), __float_as_uint(f[j][2] * by),
                                  __float_as_uint(f[j][1] * by), __float_as_uint(f[j][3] * by));
                    }
                }
                __syncwarp();
                using C = typename Src::H;
#pragma unroll
                for (int n = 0; n < NS; ++n) {  // keys 8 n + g; a scale's 32 dimensions into a sum of their own
                    const int r = 8 * n + g;
                    uint64_t sum2[NT] = {};
#pragma unroll
                    for (int b = 0; b < NB; b += 2) {
                        uint64_t f2[2];
                        lds2x64(fs + (uint32_t)((4 * n + t) * NB * 8 + b * 8), f2);
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const uint2 w = lds64(ks + (uint32_t)(r * G::kRow + ((t & 1) << 3)) + pd_chunk<CPR>(r, 2 * (b + e) + (t >> 1)));
                            float part[4];
                            mma16816_new(part, q[2 * (b + e)], C::lo(w.x), C::hi(w.x));
                            mma16816<__half>(part, q[2 * (b + e) + 1], C::lo(w.y), C::hi(w.y));
#pragma unroll
                            for (int x = 0; x < NT; ++x) sum2[x] = f2_fma(f2_pack(part[2 * x], part[2 * x + 1]), f2[e], sum2[x]);
                        }
                    }
#pragma unroll
                    for (int x = 0; x < NT; ++x) f2_unpack(sum2[x], s[n][2 * x], s[n][2 * x + 1]);
                }
            }
            // whether some column does not attend to all of the step
            const bool partial = !Src::kMx || mask != FULL ||
                                 (ROWS && (p0 + KEYS - 1 > at.s.len || (a.window > 0 && p0 <= at.s.len + at.s.rows - 1 - a.window)));
            // Weights.  m is a reference: the maximum less kUp where P is fp16, so that P goes up to 2^15 (it has no steps below
            // 2^-24); over codes it moves only when P would pass that, down to 2^12.  l, o and every later join agree on it.
            constexpr bool HALF_P = Src::kMx || std::is_same<T, __half>::value;
            constexpr float kUp = !HALF_P ? 0.f : Src::kMx ? 12.f : 15.f, kSlack = Src::kMx ? 3.f : 0.f;
            uint32_t hi[NT][NS], lo[NT][NS];  // of 16-bit values' weights
            float al[NT], pw[Src::kMx ? NT : 1][2 * NS];
            bool moved = false;
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                float v[2 * NS], mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 2 * NS; ++e) {  // keys 2t, 2t + 1, 2t + 8, 2t + 9, ... of column g + 8x
                    v[e] = s[e >> 1][2 * x + (e & 1)] * qs[x];
                    if (partial) {
                        const int key = 8 * (e >> 1) + 2 * t + (e & 1);
                        bool on = (mask >> key) & 1u;
                        if (ROWS) on = on && p0 + key <= last_key[x] && (a.window == 0 || p0 + key > last_key[x] - a.window);
                        v[e] = on ? v[e] : -INFINITY;
                    }
                    mx = fmaxf(mx, v[e]);
                }
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                const float mn = Src::kMx && !(mx > m[x] + (kUp + kSlack)) ? m[x] : fmaxf(m[x], mx - kUp);
                const float ref = mn == -INFINITY ? 0.f : mn;
                al[x] = pd_exp2<Src>(m[x] - ref);
                moved |= mn != m[x];
                m[x] = mn;
                float(&p)[2 * NS] = pw[Src::kMx ? x : 0];
#pragma unroll
                for (int e = 0; e < 2 * NS; ++e) p[e] = pd_exp2<Src>(v[e] - ref);
                float sum = (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                for (int e = 4; e < 2 * NS; e += 4) sum += (p[e] + p[e + 1]) + (p[e + 2] + p[e + 3]);
                l[x] = l[x] * al[x] + sum;
                if constexpr (!Src::kMx) {
#pragma unroll
                    for (int e = 0; e < NS; ++e) {
                        hi[x][e] = E::pack(p[2 * e], p[2 * e + 1]);
                        const float2 f = E::unpack(hi[x][e]);
                        lo[x][e] = E::pack(p[2 * e] - f.x, p[2 * e + 1] - f.y);
                    }
                }
            }
            if constexpr (Src::kMx && !ROWS) {
#pragma unroll
                for (int x = 0; x < NT; ++x) al[x] *= grown;
                moved |= grown != 1.f;
            }
            if constexpr (Src::kMx && ROWS) {
                if (v_most > least) {
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        float most = v_most;
                        if (partial) {  // of the positions that this lane's column attends to (weights of the others are 0)
                            most = 0.f;
#pragma unroll
                            for (int e = 0; e < NS; ++e)
#pragma unroll
                                for (int b = 0; b < NB; ++b) {
                                    float f0, f1;
                                    f2_unpack(lds1x64(fs + (uint32_t)(KEYS * NB * 4 + (4 * e + t) * NB * 8 + b * 8)), f0, f1);
                                    const int key = p0 + 8 * e + 2 * t, first = a.window == 0 ? INT_MIN : last_key[x] - a.window;
                                    if (key <= last_key[x] && key > first) most = fmaxf(most, f0);
                                    if (key + 1 <= last_key[x] && key + 1 > first) most = fmaxf(most, f1);
                                }
                            most *= pd_power(-kPdShift);
                            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
                            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
                        }
                        most = fmaxf(most, unit[x]);
                        al[x] *= unit[x] * pd_inverse(most);
                        moved |= most != unit[x];
                        unit[x] = most;
                    }
                    least = unit[0];
#pragma unroll
                    for (int x = 1; x < NT; ++x) least = fminf(least, unit[x]);
                    least = __uint_as_float(__reduce_min_sync(0xffffffffu, __float_as_uint(least)));
                }
#pragma unroll
                for (int x = 0; x < NT; ++x) {
                    const float by = pd_inverse(unit[x]) * pd_power(-kPdShift);
#pragma unroll
                    for (int e = 0; e < 2 * NS; ++e) pw[x][e] *= by;
                }
            }
            if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
                for (int x = 0; x < NT; ++x) {  // heads 2t and 2t + 1 of o's columns
                    const float a0 = __shfl_sync(0xffffffffu, al[x], 8 * t), a1 = __shfl_sync(0xffffffffu, al[x], 8 * t + 4);
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i) {
                        o[i][x][0] *= a0;
                        o[i][x][1] *= a1;
                        o[i][x][2] *= a0;
                        o[i][x][3] *= a1;
                    }
                }
            }
            if constexpr (!Src::kMx) {
#pragma unroll
                for (int i = 0; i < DH / 16; ++i) {
                    uint32_t va[4], vt[4];
                    ldsm4_t(vs + (uint32_t)(lr * G::kRow + (((2 * i + lc) ^ (lr & 7)) << 4)), va);
                    vt[0] = va[0], vt[1] = va[1], vt[2] = va[2], vt[3] = va[3];
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        mma16816<T>(o[i][x], vt, hi[x][0], hi[x][1]);
                        mma16816<T>(o[i][x], vt, lo[x][0], lo[x][1]);
                    }
                }
            } else {
                // Two codes of a row go through ldmatrix.trans as one element: a lane gets dimensions 2 g and 2 g + 1 of
                // positions 2 t and 2 t + 1.  Row g of A is made of the first, row g + 8 of the second.  The scales go to the
                // weights, which for 32 dimensions at a time are then those of the codes.
                using C = typename Src::H;
                using H = Elem<__half>;
                const int mr = (lane & 7) + (lane & 8), mc = lane >> 4;  // ldmatrix: row, chunk of a pair
#pragma unroll
                for (int n = 0; n < KEYS / 16; ++n)
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        uint64_t f2[2];
#pragma unroll
                        for (int e = 0; e < 2; ++e) f2[e] = lds1x64(fs + (uint32_t)(KEYS * NB * 4 + (8 * n + 4 * e + t) * NB * 8 + b * 8));
                        uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
                        for (int x = 0; x < NT; ++x)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const uint64_t w = f2_mul(f2_pack(pw[x][4 * n + 2 * e], pw[x][4 * n + 2 * e + 1]), f2[e]);
                                float w0, w1;
                                f2_unpack(w, w0, w1);
                                hi[x][e] = H::pack(w0, w1);
                                const float2 h = H::unpack(hi[x][e]);
                                f2_unpack(f2_fma(f2_pack(h.x, h.y), f2_pack(-1.f, -1.f), w), w0, w1);
                                lo[x][e] = H::pack(w0, w1);
                            }
                        const int r = 16 * n + mr;
                        uint32_t w[4];
                        ldsm4_t(vs + (uint32_t)(r * G::kRow) + pd_chunk<CPR>(r, 2 * b + mc), w);
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            uint32_t vt[4];
                            C::split(w[2 * y], vt[0], vt[1]);
                            C::split(w[2 * y + 1], vt[2], vt[3]);
#pragma unroll
                            for (int x = 0; x < NT; ++x) {
                                mma16816<__half>(o[2 * b + y][x], vt, hi[x][0], hi[x][1]);
                                mma16816<__half>(o[2 * b + y][x], vt, lo[x][0], lo[x][1]);
                            }
                        }
                    }
            }
            __syncwarp();
            st = st + 1 == S ? 0 : st + 1;
        }
        skip = k0 - n;
        if constexpr (Src::kMx) {  // in the values' units, of weights up to 1
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                l[x] *= 0x1p-15f;
                const float own = (ROWS ? unit[x] : unit[0]) * 0x1p-15f;
                const float u[2] = {ROWS ? __shfl_sync(0xffffffffu, own, 8 * t) : own,
                                    ROWS ? __shfl_sync(0xffffffffu, own, 8 * t + 4) : own};  // of o's columns
#pragma unroll
                for (int i = 0; i < DH / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][x][e] *= u[e & 1];
            }
        }

        if (solo) {  // ---- the unit's end: one warp's (m, l, o)
            if (Src::kMx && lane == 0) s_free[warp] = st_load;
            __syncwarp();
            float* ws = merge_at(warp);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
                l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
                const float inv = l[x] == 0.f ? 0.f : 1.f / l[x];  // of column g + 8x; o's columns are 2t and 2t + 1
                const float f[2] = {__shfl_sync(0xffffffffu, inv, 8 * t), __shfl_sync(0xffffffffu, inv, 8 * t + 4)};
#pragma unroll
                for (int i = 0; i < DH / 16; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        ws[(2 * t + (e & 1)) * DH + (dim_of(i, e) ^ (8 * t))] = o[i][x][e] * f[e & 1];
                __syncwarp();
                for (int e = lane; e < 8 * DH / 8; e += 32) {  // 8 dims of a column
                    const int h = e / (DH / 8), d = (e % (DH / 8)) * 8;
                    if (8 * x + h >= nc) continue;
                    const float4* v = reinterpret_cast<const float4*>(ws + h * DH + (d ^ (8 * (h >> 1))));
                    const float4 v0 = v[0], v1 = v[1];
                    *reinterpret_cast<uint4*>(a.out + col_at(8 * x + h, a.out_ld) + d) =
                        make_uint4(E::pack(v0.x, v0.y), E::pack(v0.z, v0.w), E::pack(v1.x, v1.y), E::pack(v1.z, v1.w));
                }
                __syncwarp();
            }
            at.next(a);
            continue;
        }

        // ---- the unit's end here: the four warps' (m, l, o) into one
        const bool whole = n == at.s.steps;
        const int64_t first = paged_div(u0, per), last = paged_div(u0 + at.s.steps - 1, per);  // the CTAs that share the unit
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            l[x] += __shfl_xor_sync(0xffffffffu, l[x], 1);
            l[x] += __shfl_xor_sync(0xffffffffu, l[x], 2);
            if (t == 0) {
                s_ml[0][warp][8 * x + g] = m[x];
                s_ml[1][warp][8 * x + g] = l[x];
            }
        }
        if (Src::kMx && lane == 0) s_free[warp] = st_load;
        __syncthreads();
        float* mine_so = merge_at(warp);
        const int slot = (int)(2 * blockIdx.x + (first == blockIdx.x ? 1 : 0));
        float* part = a.work + (int64_t)slot * kPagedDecodeSlot;
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            float f[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int h = 8 * x + 2 * t + e;
                float mm = s_ml[0][0][h];
                for (int w = 1; w < kPdWarps; ++w) mm = fmaxf(mm, s_ml[0][w][h]);
                f[e] = exp2f(s_ml[0][warp][h] - (mm == -INFINITY ? 0.f : mm));
            }
            if (x > 0) __syncthreads();  // the buffer holds 8 heads
#pragma unroll
            for (int i = 0; i < DH / 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int h = 2 * t + (e & 1), d = dim_of(i, e) ^ (8 * t);
                    mine_so[h * DH + d] = o[i][x][e] * f[e & 1];
                }
            __syncthreads();
            for (int e = tid; e < 8 * DH / 8; e += kPdThreads) {  // 8 dims of a head
                const int h = e / (DH / 8), d = (e % (DH / 8)) * 8, ds = d ^ (8 * (h >> 1));
                if (8 * x + h >= nc) continue;
                float sum[8] = {};
                float mm = s_ml[0][0][8 * x + h], ll = 0.f;
                for (int w = 1; w < kPdWarps; ++w) mm = fmaxf(mm, s_ml[0][w][8 * x + h]);
                const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
                for (int w = 0; w < kPdWarps; ++w) {
                    ll += s_ml[1][w][8 * x + h] * exp2f(s_ml[0][w][8 * x + h] - ref);
                    const float4* v = reinterpret_cast<const float4*>(merge_at(w) + h * DH + ds);
                    const float4 v0 = v[0], v1 = v[1];
                    sum[0] += v0.x, sum[1] += v0.y, sum[2] += v0.z, sum[3] += v0.w;
                    sum[4] += v1.x, sum[5] += v1.y, sum[6] += v1.z, sum[7] += v1.w;
                }
                if (whole) {
                    const float inv = ll == 0.f ? 0.f : 1.f / ll;
                    uint16_t* dst = a.out + col_at(8 * x + h, a.out_ld) + d;
                    *reinterpret_cast<uint4*>(dst) = make_uint4(E::pack(sum[0] * inv, sum[1] * inv), E::pack(sum[2] * inv, sum[3] * inv),
                                                                E::pack(sum[4] * inv, sum[5] * inv), E::pack(sum[6] * inv, sum[7] * inv));
                } else {
                    float* po = part + 16 * NT + (8 * x + h) * DH + d;
                    reinterpret_cast<float4*>(po)[0] = make_float4(sum[0], sum[1], sum[2], sum[3]);
                    reinterpret_cast<float4*>(po)[1] = make_float4(sum[4], sum[5], sum[6], sum[7]);
                    if (d == 0) {
                        part[8 * x + h] = mm;
                        part[8 * NT + 8 * x + h] = ll;
                    }
                }
            }
        }
        if (!whole) {
            // ---- the last CTA of the unit to get here joins the parts, in CTA order
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                const int parts = (int)(last - first) + 1;
                s_last = atomicAdd(&a.arrived[first], 1) == parts - 1;
                if (s_last) a.arrived[first] = 0;  // ready for the next call
            }
            __syncthreads();
            if (Src::kMx && s_last && last - first >= kPdManyParts) {
                // Several threads an item (8 dims of a column), each with every so many-th part, and eight of them on their way at
                // once.  One warp a scheduler is left here: what counts is the instructions of a thread.
                __threadfence();
                constexpr int UP = 8;
                const int items = nc * (DH / 8), tpi = items <= 16 ? 8 : items <= 32 ? 4 : items <= 64 ? 2 : 1, parts = (int)(last - first) + 1;
                const float* base = a.work + 2 * first * kPagedDecodeSlot;  // of part p: 2 p slots further (the first: one)
#pragma unroll 1
                for (int e0 = 0; e0 < items; e0 += kPdThreads / tpi) {
                    const int e = e0 + tid / tpi, sub = tid % tpi, h = min(e, items - 1) / (DH / 8), d = (e % (DH / 8)) * 8;
                    float sum[8] = {}, mm = -INFINITY, ll = 0.f;
#pragma unroll 1
                    for (int p0 = sub; p0 < parts; p0 += UP * tpi) {
                        float pm[UP], pl[UP];
                        float4 v[UP][2];
                        float mn = mm;
#pragma unroll
                        for (int k = 0; k < UP; ++k) {
                            const int p = min(p0 + k * tpi, parts - 1);
                            const float* src = base + (p == 0 ? 1 : 2 * p) * (int)kPagedDecodeSlot;
                            pm[k] = __ldcg(src + h);
                            pl[k] = __ldcg(src + 8 * NT + h);
                            v[k][0] = __ldcg(reinterpret_cast<const float4*>(src + 16 * NT + h * DH + d));
                            v[k][1] = __ldcg(reinterpret_cast<const float4*>(src + 16 * NT + h * DH + d) + 1);
                        }
#pragma unroll
                        for (int k = 0; k < UP; ++k) {
                            if (p0 + k * tpi >= parts) pm[k] = -INFINITY, pl[k] = 0.f;
                            mn = fmaxf(mn, pm[k]);
                        }
                        const float ref = mn == -INFINITY ? 0.f : mn, fa = pd_exp2<Src>(mm - ref);
                        mm = mn;
                        ll *= fa;
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[i] *= fa;
#pragma unroll
                        for (int k = 0; k < UP; ++k) {
                            const float fb = pd_exp2<Src>(pm[k] - ref);
                            ll = fmaf(pl[k], fb, ll);
                            sum[0] = fmaf(v[k][0].x, fb, sum[0]), sum[1] = fmaf(v[k][0].y, fb, sum[1]);
                            sum[2] = fmaf(v[k][0].z, fb, sum[2]), sum[3] = fmaf(v[k][0].w, fb, sum[3]);
                            sum[4] = fmaf(v[k][1].x, fb, sum[4]), sum[5] = fmaf(v[k][1].y, fb, sum[5]);
                            sum[6] = fmaf(v[k][1].z, fb, sum[6]), sum[7] = fmaf(v[k][1].w, fb, sum[7]);
                        }
                    }
#pragma unroll 1
                    for (int o = 1; o < tpi; o <<= 1) {  // the item's threads, side by side
                        const float om = __shfl_xor_sync(0xffffffffu, mm, o), mn = fmaxf(mm, om), ref = mn == -INFINITY ? 0.f : mn;
                        const float fa = pd_exp2<Src>(mm - ref), fb = pd_exp2<Src>(om - ref);
                        mm = mn;
                        ll = ll * fa + __shfl_xor_sync(0xffffffffu, ll, o) * fb;
#pragma unroll
                        for (int i = 0; i < 8; ++i) sum[i] = sum[i] * fa + __shfl_xor_sync(0xffffffffu, sum[i], o) * fb;
                    }
                    const float inv = ll == 0.f ? 0.f : 1.f / ll;
                    if (sub == 0 && e < items)
                        *reinterpret_cast<uint4*>(a.out + col_at(h, a.out_ld) + d) =
                            make_uint4(E::pack(sum[0] * inv, sum[1] * inv), E::pack(sum[2] * inv, sum[3] * inv),
                                       E::pack(sum[4] * inv, sum[5] * inv), E::pack(sum[6] * inv, sum[7] * inv));
                }
            } else if (s_last) {
                __threadfence();
                for (int e = tid; e < nc * (DH / 8); e += kPdThreads) {
                    const int h = e / (DH / 8), d = (e % (DH / 8)) * 8;
                    float sum[8] = {}, mm = -INFINITY, ll = 0.f;
#pragma unroll 4
                    for (int64_t p = first; p <= last; ++p) {
                        const float* src = a.work + (2 * p + (p == first ? 1 : 0)) * kPagedDecodeSlot;
                        const float pm = __ldcg(src + h), pl = __ldcg(src + 8 * NT + h);
                        const float4* v = reinterpret_cast<const float4*>(src + 16 * NT + h * DH + d);
                        const float4 v0 = __ldcg(v), v1 = __ldcg(v + 1);
                        const float mn = fmaxf(mm, pm), ref = mn == -INFINITY ? 0.f : mn;
                        const float fa = exp2f(mm - ref), fb = exp2f(pm - ref);
                        mm = mn;
                        ll = ll * fa + pl * fb;
                        sum[0] = sum[0] * fa + v0.x * fb, sum[1] = sum[1] * fa + v0.y * fb;
                        sum[2] = sum[2] * fa + v0.z * fb, sum[3] = sum[3] * fa + v0.w * fb;
                        sum[4] = sum[4] * fa + v1.x * fb, sum[5] = sum[5] * fa + v1.y * fb;
                        sum[6] = sum[6] * fa + v1.z * fb, sum[7] = sum[7] * fa + v1.w * fb;
                    }
                    const float inv = ll == 0.f ? 0.f : 1.f / ll;
                    uint16_t* dst = a.out + col_at(h, a.out_ld) + d;
                    *reinterpret_cast<uint4*>(dst) = make_uint4(E::pack(sum[0] * inv, sum[1] * inv), E::pack(sum[2] * inv, sum[3] * inv),
                                                                E::pack(sum[4] * inv, sum[5] * inv), E::pack(sum[6] * inv, sum[7] * inv));
                }
            }
        }
        __syncthreads();  // results and s_ml are free for the next unit
        at.next(a);
    }
    cp_async_wait<0>();
}

// Length of the line at the longest lengths, with units of `cols` columns.
template <class G>
int64_t paged_decode_line_of(const PagedAttnArgs& a, int cols) {
    const int64_t tiles = (int64_t)a.n_rows * a.group / cols + a.c.n_seqs;
    const int64_t span = a.window > 0 ? std::min<int64_t>((int64_t)a.window + a.n_rows, a.c.cap) : a.c.cap;
    return tiles * a.c.n_kv_heads * (span / G::kKeys + 2 + G::kUnitCost);
}

template <class Src, int DH, int NT, bool ROWS>
static cudaError_t decode_nt(const PagedAttnArgs& a, cudaStream_t st) {
    using G = PdGeom<Src, DH, NT>;
    const int64_t most = paged_decode_line_of<G>(a, 8 * NT);
    const int64_t grid = std::min<int64_t>(std::min(kPagedMaxGrid, G::kCtas * g_num_sms), (most + G::kMinSteps - 1) / G::kMinSteps);
    return launch_paged_k(k_paged_decode<Src, DH, NT, ROWS>, (unsigned)grid, kPdThreads, G::kSmem, st, a);
}
template <class Src, bool ROWS>
static cudaError_t decode_dh(const PagedAttnArgs& a, int dh, cudaStream_t st) {
    // columns that the sequences have on average; more than 8 share a pass over K and V in tiles of 16
    const bool wide = (int64_t)a.n_rows * a.group > (int64_t)8 * a.c.n_seqs;
    if (dh == 128) return wide ? decode_nt<Src, 128, 2, ROWS>(a, st) : decode_nt<Src, 128, 1, ROWS>(a, st);
    return wide ? decode_nt<Src, 64, 2, ROWS>(a, st) : decode_nt<Src, 64, 1, ROWS>(a, st);
}
template <class Src>
static cudaError_t decode_src(const PagedAttnArgs& a, int dh, cudaStream_t st) {
    return a.c.starts ? decode_dh<Src, true>(a, dh, st) : decode_dh<Src, false>(a, dh, st);
}

template <class Src, int DH, int NT>
static cudaError_t init_one() {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_decode<Src, DH, NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)PdGeom<Src, DH, NT>::kSmem);
    return e != cudaSuccess ? e
                            : cudaFuncSetAttribute(k_paged_decode<Src, DH, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)PdGeom<Src, DH, NT>::kSmem);
}
template <class Src>
static cudaError_t init_src() {
    for (cudaError_t x : {init_one<Src, 64, 1>(), init_one<Src, 64, 2>(), init_one<Src, 128, 1>(), init_one<Src, 128, 2>()})
        if (x != cudaSuccess) return x;
    return cudaSuccess;
}

}  // namespace vt
