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
// lengths.  A unit counts kPdUnitCost steps more than it has, as its queries and its result take that time.
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
// Measured: one history of 131,000 positions, 8 KV heads of 4, dh 128: 92 us, 5830 GB/s (86% of a copy's rate: the
// start, the last steps and the join of 38 parts a head are the rest); 64 sequences of up to 8191, some idle: 47 us, 5310
// GB/s; 16 of 500 to 4096 with 32 KV heads and a window of 1024: 46 us, 5290 GB/s; 128 positions of 8 heads: 5.6 us, all
// of it latency (lengths, table, first rows, merge).
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>

#include "paged.cuh"

namespace vt {

constexpr int kPdWarps = 4, kPdThreads = kPdWarps * 32;
constexpr int kPdKeys = 16;                  // positions of a step
constexpr int kPdRing = 96 * 1024;           // bytes of the four warps' rings
constexpr int kPdCtasPerSm = 2;
// A unit's queries, merge and result cost as much as this many steps (measured: 64 ragged sequences 75 us at 0, 56 at
// 4, 47 at 8 to 24, 50 at 32).
constexpr int kPdUnitCost = 16;
// What a CTA takes at least: where the largest unit costs no more than kPdWhole (12 steps), that much, so that few are
// split and joined (8 heads of 128 positions: 5.4 us, split 6.7; at 48, units of 20 to 30 steps lost up to 2 us);
// otherwise kPdMinSteps.
constexpr int kPdMinSteps = 16, kPdWhole = 28;

// Where the largest unit has no more steps than kPdSoloSteps and there are kPdSoloUnits or more such units for every CTA,
// each warp has units of its own: merging four warps would cost more than the steps.  Measured, merged and alone: 168
// sequences of 1 to 3 positions, 32 heads, 38 and 15 us; 1024 sequences of 61 to 65 positions, 8 KV heads, 87 and 56;
// 24 sequences of 201 to 251, 32 heads, 24 and 22.  At 32 steps 300 sequences of 21 to 501 positions lost (51 to 63).
constexpr int kPdSoloSteps = 16, kPdSoloUnits = 2;

template <int DH>
struct PdGeom {
    static constexpr int kRow = DH * 2;                            // bytes of a K or V row
    static constexpr int kStage = 2 * kPdKeys * kRow;              // K rows, then V rows
    static constexpr int kStages = kPdRing / (kPdWarps * kStage);  // 3 (dh 128) or 6 (dh 64)
    static constexpr size_t kSmem = kPdRing + (size_t)kPdWarps * 8 * DH * 4;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool full) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(full ? 16 : 0) : "memory");
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

// A sequence's new rows, and the positions [beg, end) that they attend to (end 0: none).
struct PdSeq {
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
        steps = (end + kPdKeys - 1) / kPdKeys - beg / kPdKeys;
        tiles = (rows * a.group + cols - 1) / cols;
    }
    // its share of the line, for one KV head
    __device__ __forceinline__ int64_t cost() const { return steps > 0 ? (int64_t)tiles * (steps + kPdUnitCost) : 0; }
};

// Where a walk over the steps of the units stands: unit u of sequence b (KV head u / tiles), step i - kPdUnitCost.
template <bool ROWS, int COLS>
struct PdCursor {
    int b, u, i;
    PdSeq s;
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

template <class T, int DH, int NT, bool ROWS>
__global__ void __launch_bounds__(kPdThreads, kPdCtasPerSm) k_paged_decode(const __grid_constant__ PagedAttnArgs a) {
    using E = Elem<T>;
    using G = PdGeom<DH>;
    constexpr int S = G::kStages, CPR = DH / 8, RPI = 32 / CPR;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int64_t s_sum[kPdWarps], s_before[kPdWarps + 1];
    __shared__ int s_seq[kPdWarps + 1], s_last, s_max[kPdWarps];
    __shared__ float s_ml[2][kPdWarps][8 * NT];
    __shared__ uint32_t s_mask[kPdWarps][S];
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
        PdSeq s;
        s.open<ROWS>(a, b, COLS);
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
            PdSeq s;
            s.open<ROWS>(a, b, COLS);
            if (s.steps == 0)
                for (int r = s.row0; r < s.row0 + s.rows; ++r)
                    for (int e = tid; e < a.n_heads * DH / 8; e += kPdThreads)
                        reinterpret_cast<uint4*>(a.out + r * a.out_ld)[e] = make_uint4(0u, 0u, 0u, 0u);
        }
    const int64_t line = total * c.n_kv_heads;
    const bool solo = largest <= kPdSoloSteps && line >= (int64_t)kPdSoloUnits * gridDim.x * (largest + kPdUnitCost);
    const int64_t per = max(paged_div(line + gridDim.x - 1, gridDim.x),
                            (int64_t)(largest + kPdUnitCost <= kPdWhole ? largest + kPdUnitCost : kPdMinSteps));
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
                PdSeq s;
                s.open<ROWS>(a, b, COLS);
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
    PdCursor<ROWS, COLS> at;  // of the whole CTA, or of the warp
    if (solo) {
        auto unit_start = [&](int64_t pos, int k) {  // of the first unit that begins at pos or after it
            if (pos >= line) return line;
            PdSeq s;
            s.open<ROWS>(a, s_seq[k], COLS);
            const int64_t r = pos - s_before[k] * c.n_kv_heads, cost = s.steps + kPdUnitCost;
            return pos + (cost - 1 - (r + cost - 1 - paged_div(r + cost - 1, cost) * cost));
        };
        const int64_t w0 = unit_start(min(t1, t0 + warp * per_warp), warp);
        const int64_t w1 = unit_start(min(t1, t0 + (warp + 1) * per_warp), warp + 1);
        if (w0 >= w1) return;  // (no barrier of the whole CTA follows)
        at.open(a, s_seq[warp]);
        const int64_t r = w0 - s_before[warp] * c.n_kv_heads, cost = at.s.steps + kPdUnitCost;
        at.u = (int)paged_div(r, cost) - 1;  // the unit before it, unless it is the sequence's first
        at.i = 0;
        if (at.u < 0) at.u = 0;
        else at.next(a);
        t0 = w0;
        t1 = w1;
    } else {
        at.open(a, s_seq[0]);
        const int64_t r = t0 - s_before[0] * c.n_kv_heads;
        at.u = (int)paged_div(r, at.s.steps + kPdUnitCost);
        at.i = (int)(r - (int64_t)at.u * (at.s.steps + kPdUnitCost));
    }
    PdCursor<ROWS, COLS> ld = at;               // of this warp's copies: the unit of its next step
    int64_t ld_now = t0;                        // where that unit's part begins in the line
    int ld_i, ld_n, ld_skip = solo ? 0 : warp;  // next step of the unit, steps of it here, steps until this warp's next
    auto ld_unit = [&]() {                      // the steps [first, n) of the unit that lie in this part
        const int first = max(0, ld.i - kPdUnitCost);
        ld_n = (int)min((int64_t)ld.s.steps, t1 - ld_now + ld.i - kPdUnitCost);
        ld_i = first;
    };
    // moves to this warp's next step; false: none
    auto ld_seek = [&]() -> bool {
        while (ld_i + ld_skip >= ld_n) {
            if (ld_n > ld_i) ld_skip -= ld_n - ld_i;
            ld_now += ld.s.steps + kPdUnitCost - ld.i;
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
    int page = 0;         // lane r < 16: the table's entry for row r of the next step to load, whatever it holds;
    bool needed = false;  // whether that row is attended to is known apart from it
    auto look_up = [&]() {
        const int p = more ? (ld.s.beg / kPdKeys + ld_i) * kPdKeys + lane : -1;
        needed = more && lane < kPdKeys && p >= ld.s.beg && p < ld.s.end;
        if (needed) page = c.tables[(int64_t)ld.b * c.per_seq + (p >> c.page_shift)];
    };
    look_up();
    int st_load = 0;
    auto load_step = [&]() {
        if (more) {
            const bool on = needed && (unsigned)page < (unsigned)c.n_pages;
            if (needed && !on) set_status(c.status, VT_DEV_BAD_PAGE);
            const int p = (ld.s.beg / kPdKeys + ld_i) * kPdKeys + lane;
            const int64_t off = on ? page * c.page_stride + (ld.u / ld.s.tiles) * c.head_stride + (p & (c.page_size - 1)) * c.pos_stride
                                   : -1;
            const uint32_t mask = __ballot_sync(0xffffffffu, on);
            if (lane == 0) s_mask[warp][st_load] = mask;
            const uint32_t dst = ring + (uint32_t)(st_load * G::kStage);
            const int chunk = lane % CPR;
#pragma unroll
            for (int r0 = 0; r0 < kPdKeys; r0 += RPI) {
                const int r = r0 + lane / CPR;
                const int64_t o = __shfl_sync(0xffffffffu, off, r);
                const uint32_t d = dst + (uint32_t)(r * G::kRow + ((chunk ^ (r & 7)) << 4));
                const int64_t src = (o < 0 ? 0 : o) + chunk * 8;  // rows without a position are filled with zeros
                cp_async16(d, a.kpool + src, o >= 0);
                cp_async16(d + kPdKeys * G::kRow, a.vpool + src, o >= 0);
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
    float* so = reinterpret_cast<float*>(smem + kPdRing);
    for (int64_t now = t0; now < t1;) {
        // steps [i0, i0 + n) of the unit are in this part
        const int i0 = max(0, at.i - kPdUnitCost), n = (int)min((int64_t)at.s.steps, t1 - now + at.i - kPdUnitCost) - i0;
        const int64_t u0 = now - at.i + kPdUnitCost;  // where its steps begin in the line
        now += at.s.steps + kPdUnitCost - at.i;
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
        int last_key[NT];  // of this lane's columns, in the steps' keys
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const bool on = x < NT && g + 8 * x < nc;
            const uint16_t* src = a.q + (on ? col_at(g + 8 * x, a.q_ld) : 0) + 2 * t;
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                q[k][x] = on ? *reinterpret_cast<const uint32_t*>(src + k * 16) : 0u;
                q[k][2 + x] = on ? *reinterpret_cast<const uint32_t*>(src + k * 16 + 8) : 0u;
            }
            if (x < NT) last_key[x] = ROWS ? at.s.len + (c0 + g + 8 * x) / a.group : 0;
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
            const int p0 = ROWS ? (at.s.beg / kPdKeys + i0 + k0) * kPdKeys : 0;  // the step's first position
            load_step();
            cp_async_wait<S - 1>();
            __syncwarp();
            const uint32_t ks = ring + (uint32_t)(st * G::kStage), vs = ks + kPdKeys * G::kRow;
            const uint32_t mask = s_mask[warp][st];
            const int lr = ((lane >> 4) << 3) + (lane & 7), lc = (lane >> 3) & 1;  // ldmatrix: row, chunk of a pair
            float s[2][4] = {};
#pragma unroll
            for (int k = 0; k < DH / 16; ++k) {
                uint32_t kb[4];
                ldsm4(ks + (uint32_t)(lr * G::kRow + (((2 * k + lc) ^ (lr & 7)) << 4)), kb);
                mma16816<T>(s[0], q[k], kb[0], kb[1]);
                mma16816<T>(s[1], q[k], kb[2], kb[3]);
            }
            uint32_t hi[NT][2], lo[NT][2];
            float al[NT];
            bool moved = false;
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                float v[4], mx = -INFINITY;
#pragma unroll
                for (int e = 0; e < 4; ++e) {  // keys 2t, 2t + 1, 2t + 8, 2t + 9 of column g + 8x
                    const int key = 8 * (e >> 1) + 2 * t + (e & 1);
                    bool on = (mask >> key) & 1u;
                    if (ROWS) on = on && p0 + key <= last_key[x] && (a.window == 0 || p0 + key > last_key[x] - a.window);
                    v[e] = on ? s[e >> 1][2 * x + (e & 1)] * a.scale_log2 : -INFINITY;
                    mx = fmaxf(mx, v[e]);
                }
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                // m is the maximum less kPdUp, so that P goes up to 2^kPdUp; l, o and every later join agree on it
                constexpr float kPdUp = std::is_same<T, __half>::value ? 15.f : 0.f;
                const float mn = fmaxf(m[x], mx - kPdUp), ref = mn == -INFINITY ? 0.f : mn;
                al[x] = exp2f(m[x] - ref);
                moved |= mn != m[x];
                m[x] = mn;
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) p[e] = exp2f(v[e] - ref);
                l[x] = l[x] * al[x] + ((p[0] + p[1]) + (p[2] + p[3]));
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    hi[x][e] = E::pack(p[2 * e], p[2 * e + 1]);
                    const float2 f = E::unpack(hi[x][e]);
                    lo[x][e] = E::pack(p[2 * e] - f.x, p[2 * e + 1] - f.y);
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
            __syncwarp();
            st = st + 1 == S ? 0 : st + 1;
        }
        skip = k0 - n;

        if (solo) {  // ---- the unit's end: one warp's (m, l, o)
            float* ws = so + warp * 8 * DH;
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
                        ws[(2 * t + (e & 1)) * DH + ((16 * i + g + 8 * (e >> 1)) ^ (8 * t))] = o[i][x][e] * f[e & 1];
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
        __syncthreads();
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
                    const int h = 2 * t + (e & 1), d = (16 * i + g + 8 * (e >> 1)) ^ (8 * t);
                    so[(warp * 8 + h) * DH + d] = o[i][x][e] * f[e & 1];
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
                    const float4* v = reinterpret_cast<const float4*>(so + (w * 8 + h) * DH + ds);
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
            if (s_last) {
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
        __syncthreads();  // so and s_ml are free for the next unit
        at.next(a);
    }
    cp_async_wait<0>();
}

// Length of the line at the longest lengths, with units of `cols` columns.
int64_t paged_decode_line(const PagedAttnArgs& a, int cols) {
    const int64_t tiles = (int64_t)a.n_rows * a.group / cols + a.c.n_seqs;
    const int64_t span = a.window > 0 ? std::min<int64_t>((int64_t)a.window + a.n_rows, a.c.cap) : a.c.cap;
    return tiles * a.c.n_kv_heads * (span / kPdKeys + 2 + kPdUnitCost);
}

template <class T, int DH, int NT, bool ROWS>
static cudaError_t decode_nt(const PagedAttnArgs& a, cudaStream_t st) {
    const int64_t most = paged_decode_line(a, 8 * NT);
    const int64_t grid = std::min<int64_t>(std::min(kPagedMaxGrid, kPdCtasPerSm * g_num_sms), (most + kPdMinSteps - 1) / kPdMinSteps);
    return launch_paged_k(k_paged_decode<T, DH, NT, ROWS>, (unsigned)grid, kPdThreads, PdGeom<DH>::kSmem, st, a);
}
template <class T, bool ROWS>
static cudaError_t decode_t(const PagedAttnArgs& a, int dh, cudaStream_t st) {
    // columns that the sequences have on average; more than 8 share a pass over K and V in tiles of 16
    const bool wide = (int64_t)a.n_rows * a.group > (int64_t)8 * a.c.n_seqs;
    if (dh == 128) return wide ? decode_nt<T, 128, 2, ROWS>(a, st) : decode_nt<T, 128, 1, ROWS>(a, st);
    return wide ? decode_nt<T, 64, 2, ROWS>(a, st) : decode_nt<T, 64, 1, ROWS>(a, st);
}
cudaError_t launch_paged_decode(const PagedAttnArgs& a, int dtype, int dh, cudaStream_t st) {
    if (a.c.starts) return dtype == VT_F16 ? decode_t<__half, true>(a, dh, st) : decode_t<__nv_bfloat16, true>(a, dh, st);
    return dtype == VT_F16 ? decode_t<__half, false>(a, dh, st) : decode_t<__nv_bfloat16, false>(a, dh, st);
}

template <class T, int DH, int NT>
static cudaError_t init_one() {
    const cudaError_t e = cudaFuncSetAttribute(k_paged_decode<T, DH, NT, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)PdGeom<DH>::kSmem);
    return e != cudaSuccess ? e
                            : cudaFuncSetAttribute(k_paged_decode<T, DH, NT, true>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)PdGeom<DH>::kSmem);
}
cudaError_t init_paged_decode() {
    cudaError_t e[8] = {init_one<__half, 64, 1>(),        init_one<__half, 64, 2>(),        init_one<__half, 128, 1>(),
                        init_one<__half, 128, 2>(),       init_one<__nv_bfloat16, 64, 1>(), init_one<__nv_bfloat16, 64, 2>(),
                        init_one<__nv_bfloat16, 128, 1>(), init_one<__nv_bfloat16, 128, 2>()};
    for (cudaError_t x : e)
        if (x != cudaSuccess) return x;
    return cudaSuccess;
}

}  // namespace vt
