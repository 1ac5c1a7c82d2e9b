// Causal attention of several new rows per sequence over the paged KV cache, on the 5th-generation tensor
// cores (Voltron Section 2.1, prefill phase, for several sequences).
//
// A unit of work is a sequence's KV head and two tiles of query rows: row r of a tile is query head
// r % group of the KV head and token r / group, so the group's heads share the K and V blocks and a few
// new tokens still fill a tile.  Both tiles walk the unit's positions in blocks of 128 keys:
//   S_x = Q_x . K_j^T       tcgen05, M 128, N 128, K dh, operands in shared memory, S in tensor memory
//   P_x = 2^(S_x scale log2(e) - m), masked, 16 bits, written over S_x in tensor memory
//   O_x += P_x . V_j        tcgen05, M 128, N dh, K 128, P from tensor memory, V as it lies in the pages
// While the softmax of one tile runs, the tensor core has the other tile's products, and K and V pass through
// shared memory once for both tiles.
//
// What bounds it: by operations the tensor cores (4 dh FLOPs a score), 2 x 2 x 520 cycles a block of both
// tiles; the 2 x 128 x 128 exponentials take as long on the SM's special-function units.  In fact one tile's
// chain, softmax (2200 cycles) and then P to V, S and its notice (2350), takes about 5000 cycles a block, of
// which the two tiles hide half from each other.  Measured: 4096 rows, 32 heads, dh 128: 170 us, 810 TFLOP/s
// (42% of what a matrix product reaches); 512 rows behind 16000, 8 KV heads of 4: 154 us, 885; 5 prompts of
// 150 to 900 rows: 42 us, of which a CTA's start takes 7.  One tile a CTA with two threads a row
// took 171 and 147 us on the first two, but 55 on the third; 64-key halves were slower throughout.
//
//   warps 0-3, 4-7  softmax of tile 0 and 1, one thread a row (its lane of the tensor memory): no exchange
//                   between threads.  m is a reference: the maximum when it was set, less 7 (fp16) or 0 (bf16).
//                   O and l are rescaled only when a block's maximum exceeds that by more than 8 (log2) more, so
//                   the largest P is between 2^7 and 2^15 in fp16, whose smallest step is 2^-24 (a weight then
//                   loses at most 2^-32 of the largest one), and between 1 and 2^8 in bf16.
//   warps 8, 9      copies: Q, and K and V through the page table, by tensor copies of a page's rows; blocks that
//                   hold positions outside the unit's range (whatever lies there must not reach V: they are
//                   filled with zeros), bad pages or pages of fewer than 16 positions by 16-byte asynchronous
//                   copies into the same swizzled layout
//   warps 10, 11    the MMAs of tile 0 and 1: the waits and the issue of one fall into the other's products (one warp
//                   for both took 4700 cycles for two blocks)
//
// Over a pool of codes (paged_mx.cuh) the blocks are converted on the way: K and V in the ring are the values that the
// entries stand for, in the type of Q, so that everything after it is the same, bit for bit.  Then there are 16 warps:
//   warps 8-11      conversions, one on each of the SM's schedulers
//   warps 12, 13    the MMAs of tile 0 and 1
//   warps 14, 15    copies of codes and scales as they are, into buffers of their own; the queries
// A CTA of 512 threads has 128 registers a thread, and all roles share the instruction cache: the softmax reads S twice, in
// halves, and what can be a loop is one.  (4096 rows of int8 codes, bf16: 462 us with the 12 warps and unrolled, 310 with the
// roles apart, 221 with the conversions a loop, 181 with the softmax's parts loops too; the 16-bit pool takes 168.)
// Measured: 512 rows behind 16000, e4m3 and fp16: 151 us (the 16-bit pool 154); 7 prompts of 300 to 2500 rows 165.
//
// The blocks of all units form one line, and CTA c (one an SM) takes its c-th equal part, so neither few
// long histories nor ragged prompts leave SMs idle; lengths are known on the device only.  A unit that
// several CTAs share is joined in CTA order, by the last of them to finish or (few long units) by
// k_paged_join, so a result does not depend on timing.  Every mbarrier wait is bounded; on a timeout a warp
// sets VT_DEV_WAIT_TIMEOUT, issues nothing more, stores no output (a part of nothing where others wait for
// one), and still passes every named barrier.
#include <cuda_runtime.h>
#include <math.h>

#include <algorithm>
#include <climits>

#include "paged_mx.cuh"
#include "tcgen05.cuh"

namespace vt {

constexpr int kPfRows = 128, kPfKeys = 128;  // rows of a tile, keys of a block
constexpr int kPfMaskRing = 8;   // validity words of the last blocks (the copies lead by fewer blocks)
// The start and end of a unit cost as much as this many blocks (5 prompts: 46 us at 1, 42 at 2, 44 at 3).
constexpr int kPfUnitCost = 2;
// What a CTA takes at least: where the largest unit costs no more than kPfWhole, that much, so that few are split and
// joined; otherwise kPfMinBlocks.  (3 prompts of 300 rows, 12 heads: 20 us; with 4 and 2 for them 27, as every unit is
// split then.)
constexpr int kPfMinBlocks = 4, kPfWhole = 8;
// Units of this many parts or more on average are joined by a kernel of its own.  Measured, by the last CTA and by a
// kernel: 38 parts 63 and 47 us (32 rows behind 30000, 2 sequences of 2 KV heads), 9 parts 37 and 29 (100 rows behind 3000,
// 8 KV heads of 4), 7 parts 37 and 32, 6 parts 38 and 36, 5 parts 40 and 38 (150 rows behind 3000; 7, 8 and 10 KV heads of
// 4), 2 parts 156 and 162 (a kernel adds its launch, and joins that would have been hidden behind other CTAs' work).
constexpr int kPfJoinParts = 5;
// Parts that the joining CTA reads at once; most units have two (with 4 at once: 45 us for 5 prompts instead of 42).
constexpr int kPfJoinChunk = 2;
constexpr int kPfLag = 2;        // copy groups in flight behind the one just issued

template <class Src, int DH>
struct PfGeom {
    // Warps: 8 of softmax, those of the copies, then one MMA warp a tile.  Codes: four warps convert them, so that each of the
    // SM's four schedulers has one (a warp's conversions of a block take it about 1000 instructions).
    static constexpr int kCopyWarps = Src::kMx ? 4 : 2, kMma = 8 + kCopyWarps;
    static constexpr int kThreads = Src::kMx ? 512 : 384;
    // Registers a thread: at launch 65536 / threads, rounded down to 8; then 2 x 128 threads of softmax, and 128 of copies and
    // MMAs, or (codes) 128 of conversions and 128 of MMAs and copies.
    static constexpr int kLaunchRegs = Src::kMx ? 128 : 168, kSoftmaxRegs = Src::kMx ? 176 : 208, kCopyRegs = Src::kMx ? 72 : 88;
    static constexpr int kMmaRegs = 88;
    static_assert(256 * kSoftmaxRegs + 128 * kCopyRegs + (kThreads - 384) * kMmaRegs <= kThreads * kLaunchRegs,
                  "the register split must fit in the registers the block is launched with");
    static constexpr int kTile = kPfRows * DH * 2;         // bytes of a Q tile, of a K or V block
    static constexpr int kAtom = kPfRows * 128;            // its 64-column box
    static constexpr int kSlots = (DH == 128 ? 1 : 2) * (Src::kMx ? 3 : 5);  // K and V blocks of the ring, in turn
    static constexpr int kRaw = Src::kMx ? kPfKeys * (DH + DH / kMxBlock) : 0;  // codes and scales of a block
    static constexpr int kRaws = 3;                        // of them on their way
    static constexpr size_t kSmem = 1024 + (size_t)(2 + kSlots) * kTile + kRaws * kRaw + 512 + (Src::kMx ? 128 : 0) + kThreads / 32 * 64;
};

// The units in order: sequence, KV head, tile pair.
struct PfCursor {
    int b, kvh, pt;        // unit
    int i, n, kb0;         // place in the unit (block i - kPfUnitCost), blocks of the unit, its first block's number
    int len, row0, rows;   // the sequence (rows 0: idle)
    int kbeg, kend;        // attended positions of the unit
    __device__ __forceinline__ void seq(const PagedAttnArgs& a, int at) {
        b = at;
        kvh = pt = 0;
        rows = 0;
        if (b < a.c.n_seqs) {
            len = paged_len(a.c, b);
            row0 = paged_start(a.c, b, a.n_rows);
            rows = len < 0 ? 0 : max(0, paged_start(a.c, b + 1, a.n_rows) - row0);
            if (rows <= a.rows_over) rows = 0;  // another launch's
        }
    }
    // attended positions of tokens [t0, t1) of the sequence
    __device__ __forceinline__ void range(const PagedAttnArgs& a, int t0, int t1, int& beg, int& end) const {
        end = min(len + t1, a.c.cap);
        beg = a.window > 0 ? max(0, len + t0 + 1 - a.window) : 0;
        if (beg >= end) beg = end = 0;
    }
    __device__ __forceinline__ static int blocks(int beg, int end) { return (end + kPfKeys - 1) / kPfKeys - beg / kPfKeys; }
    __device__ __forceinline__ void unit(const PagedAttnArgs& a, int tr) {
        const int t0 = pt * 2 * tr;
        range(a, t0, min(t0 + 2 * tr, rows), kbeg, kend);
        kb0 = kbeg / kPfKeys;
        n = blocks(kbeg, kend);
        i = 0;
    }
    // on to the next unit that has blocks
    __device__ __forceinline__ void next(const PagedAttnArgs& a, int tr) {
        do {
            if ((pt + 1) * 2 * tr < rows)
                ++pt;
            else if (rows > 0 && kvh + 1 < a.c.n_kv_heads)
                ++kvh, pt = 0;
            else {
                do seq(a, b + 1);
                while (rows == 0 && b < a.c.n_seqs);
                if (b >= a.c.n_seqs) return;
            }
            unit(a, tr);
        } while (n == 0);
    }
    // The unit's blocks [i0, i0 + n_here) of the `left` that the CTA still has; none: the unit's start lies here only.
    __device__ __forceinline__ int part(int64_t left, int& n_here) const {
        const int i0 = max(0, i - kPfUnitCost);
        n_here = (int)min((int64_t)n, left + i - kPfUnitCost) - i0;
        return i0;
    }
    __device__ __forceinline__ int rest() const { return n + kPfUnitCost - i; }  // of the unit, in the line
    // blocks [lo, hi) of those numbered j0 .. j1 - 1 that tile x attends to; false: the tile has no tokens
    __device__ __forceinline__ bool tile(const PagedAttnArgs& a, int tr, int x, int j0, int j1, int& lo, int& hi) const {
        const int t0 = (2 * pt + x) * tr, t1 = min(t0 + tr, rows);
        lo = hi = j0;
        if (t0 >= t1) return false;
        int beg, end;
        range(a, t0, t1, beg, end);
        if (end > beg) {
            lo = max(j0, beg / kPfKeys);
            hi = max(lo, min(j1, (end + kPfKeys - 1) / kPfKeys));
        }
        return true;
    }
};

__device__ __forceinline__ void pf_copy16(uint32_t dst, const void* src, bool full) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(full ? 16 : 0) : "memory");
}
// The wait of a whole warp.  A phase that is there or about to be is seen by plain tests (15 cycles each, where
// a bounded wait takes 150 to 240 although the phase is complete); after kPfTests of them one lane waits, so that
// a dozen waiting warps do not keep shared memory busy.
constexpr int kPfTests = 64;
__device__ __forceinline__ bool pf_wait(uint64_t* bar, uint32_t parity) {
#pragma unroll 1
    for (int i = 0; i < kPfTests; ++i)
        if (__all_sync(0xffffffffu, fa_test(bar, parity))) return true;
    int ok = 1;
    if ((threadIdx.x & 31) == 0) ok = mbar_wait(bar, parity) ? 1 : 0;
    ok = __shfl_sync(0xffffffffu, ok, 0);
    __syncwarp();  // what the one lane acquired holds for all of them (a shuffle orders no memory)
    return ok != 0;
}
// Two at once: their tests overlap.
__device__ __forceinline__ bool pf_wait2(uint64_t* bar0, uint32_t parity0, uint64_t* bar1, uint32_t parity1) {
#pragma unroll 1
    for (int i = 0; i < kPfTests; ++i) {
        const bool p = fa_test(bar0, parity0), q = fa_test(bar1, parity1);
        if (__all_sync(0xffffffffu, p && q)) return true;
    }
    return pf_wait(bar0, parity0) && pf_wait(bar1, parity1);
}
__device__ __forceinline__ void pf_zero_row(const PagedAttnArgs& a, int row, int words, int lane) {
    for (int e = lane; e < words; e += 32) reinterpret_cast<uint4*>(a.out + row * a.out_ld)[e] = make_uint4(0u, 0u, 0u, 0u);
}

// A unit that several CTAs share: the first of them leaves this, all of them their parts.
struct PfSplit {
    int parts, kvh, row0, tokens;  // parts 0: none begins in the CTA; of both tiles
};
__device__ __forceinline__ float* pf_slot(const PagedAttnArgs& a, int cta, int first, int x) {
    return a.work + (int64_t)(4 * cta + (cta == first ? 2 : 0) + x) * kPagedPrefillSlot;
}

struct PfParams {
    PagedAttnArgs a;
    PfSplit* split;       // [CTAs]
    int tma;              // blocks that are whole come by tensor copies
    CUtensorMap tq;       // [rows][heads][dh], boxes of a tile's rows by 64 columns
    CUtensorMap tk, tv;   // [pages][KV heads][positions][dh], boxes of a page's positions (128 at most) by 64 columns
};

// Over a pool of codes, three roles take the place of the copy warps:
//   copies        (one warp) codes and scales of a block of K or V as they are, into one of kRaws buffers: by tensor copies of
//                 a page's rows, or by asynchronous copies of 16 bytes where a block is not whole or pages are small
//   conversions   (four warps) from there to the type of Q, into the ring, as the tensor copies of a 16-bit pool would leave
//                 them there.  They know nothing of units: they follow the buffers until one says that it is the last
//   queries       (one warp)
// Positions outside the unit's range and bad pages get scale 0, whose product with any code (they are filled with zeros) is
// 0.  A page holds 8 positions or more, so a group of 8 rows lies in one.
struct PfRaw {
    uint8_t* data;         // [kRaws] codes [128][dh] with the swizzle of dh bytes, then [kRaws] scales [128][dh / 32]
    uint64_t *full, *empty;
    uint32_t* rows;        // [kRaws][4] which rows hold something
    int* last;             // [kRaws] nothing follows, and nothing is there
};
template <int DH>
__device__ __forceinline__ uint32_t pf_raw_at(int row, int chunk) {
    const uint32_t at = (uint32_t)(row * DH + chunk * 16);
    return at ^ ((at >> 3) & (DH == 128 ? 0x70u : 0x30u));
}

template <class Src, int DH>
__device__ __forceinline__ bool pf_copy_codes(const PfParams& P, const PfRaw& m, uint32_t* valid, PfCursor at, int64_t left) {
    using G = PfGeom<Src, DH>;
    constexpr int NB = DH / kMxBlock, CPR = DH / 16, RPI = 32 / CPR, PIECES = kPfKeys * NB / 16;  // 16-byte pieces of the scales
    const PagedAttnArgs& a = P.a;
    const PagedView& c = a.c;
    const int lane = threadIdx.x & 31, tr = kPfRows / a.group, chunk = lane % CPR, sub = lane / CPR;
    const int box_rows = min(c.page_size, kPfKeys);
    const uint32_t codes = smem_u32(m.data), scales = codes + G::kRaws * kPfKeys * DH;
    int buf = 0, round = 0, blk = 0;
    bool ok = true;
    // lane g < 16: the page of 8-row group g of block j, requested a block ahead
    auto request = [&](int j) {
        const int p = j * kPfKeys + 8 * (lane & 15);
        return p + 8 > at.kbeg && p < at.kend ? c.tables[(int64_t)at.b * c.per_seq + (p >> c.page_shift)] : 0;
    };
    while (ok && left > 0) {
        int n;
        const int j0 = at.kb0 + at.part(left, n);
        left -= at.rest();
        int next = n > 0 ? request(j0) : 0;
        for (int j = j0; ok && j < j0 + n; ++j, ++blk) {
            int page = next;
            if (j + 1 < j0 + n) next = request(j + 1);
            const int p0 = j * kPfKeys, g0 = p0 + 8 * (lane & 15);
            uint32_t rows = fa_range_bits(at.kbeg - g0, at.kend - g0) & 0xffu;
            if (rows && (unsigned)page >= (unsigned)c.n_pages) {
                rows = 0;
                set_status(c.status, VT_DEV_BAD_PAGE);
            }
            if (!rows) page = 0;
            const bool whole = P.tma && __all_sync(0xffffffffu, rows == 0xffu);
            if (lane < 16) reinterpret_cast<uint8_t*>(valid)[(blk % kPfMaskRing) * 16 + lane] = (uint8_t)rows;
#pragma unroll 1
            for (int kv = 0; kv < 2; ++kv) {
                if (round > 0) ok = pf_wait(&m.empty[buf], (round - 1) & 1);
                if (!ok) break;
                if (lane < 16) reinterpret_cast<uint8_t*>(m.rows)[buf * 16 + lane] = (uint8_t)rows;
                if (lane == 0) m.last[buf] = 0;
                const uint32_t dst = codes + (uint32_t)(buf * kPfKeys * DH), sdst = scales + (uint32_t)(buf * kPfKeys * NB);
                const uint8_t* scale = (kv ? a.vscale : a.kscale) + at.kvh * a.scale_head;
                __syncwarp();  // what the lanes stored, before any of them arrives
                if (whole) {
                    if (elect_one()) mbar_arrive_expect_tx(&m.full[buf], (uint32_t)(kPfKeys * (DH + NB)));
                    for (int r = 0; r < kPfKeys; r += box_rows) {
                        const int pg = __shfl_sync(0xffffffffu, page, r >> 3), first = (p0 + r) & (c.page_size - 1);
                        if (elect_one()) {
                            tc::tma_load_4d(dst + (uint32_t)(r * DH), kv ? &P.tv : &P.tk, 0, first, at.kvh, pg, &m.full[buf]);
                            bulk_g2s(m.data + (sdst - codes) + r * NB, scale + pg * a.scale_page + first * NB, (uint32_t)(box_rows * NB),
                                     &m.full[buf]);
                        }
                        __syncwarp();
                    }
                    mbar_arrive(&m.full[buf]);
                } else {
                    const uint8_t* pool = reinterpret_cast<const uint8_t*>(kv ? a.vpool : a.kpool) + at.kvh * c.head_stride + chunk * 16;
#pragma unroll 2
                    for (int g = 0; g < 16; ++g) {
                        const uint8_t* src = pool + __shfl_sync(0xffffffffu, page, g) * c.page_stride +
                                             (((p0 + 8 * g) & (c.page_size - 1)) + sub) * c.pos_stride;
                        const uint32_t bits = __shfl_sync(0xffffffffu, rows, g) >> sub;
#pragma unroll
                        for (int k = 0; k < 8; k += RPI, src += RPI * c.pos_stride)
                            pf_copy16(dst + pf_raw_at<DH>(8 * g + k + sub, chunk), src, (bits >> k) & 1u);
                    }
                    const int x = lane % PIECES, g = x * 16 / PIECES, pg = __shfl_sync(0xffffffffu, page, g);
                    const bool any = __shfl_sync(0xffffffffu, rows, g) != 0;
                    if (lane < PIECES)
                        pf_copy16(sdst + (uint32_t)(lane * 16), scale + pg * a.scale_page + ((p0 + x * (16 / NB)) & (c.page_size - 1)) * NB, any);
                    if (lane == 0) mbar_arrive(&m.full[buf]);
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(smem_u32(&m.full[buf])) : "memory");
                }
                if (++buf == G::kRaws) buf = 0, ++round;
            }
        }
        at.next(a, tr);
    }
    if (ok && round > 0) ok = pf_wait(&m.empty[buf], (round - 1) & 1);
    if (ok) {
        if (lane == 0) m.last[buf] = 1;
        __syncwarp();
        if (lane == 0) mbar_arrive(&m.full[buf]);
        mbar_arrive(&m.full[buf]);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (!ok)  // no tensor copy may still be in flight when the CTA ends
        for (int b = 0; b < G::kRaws; ++b) {
            const int fills = round + (b < buf ? 1 : 0);
            if (fills > 0) pf_wait(&m.full[b], (fills - 1) & 1);
        }
    return ok;
}

struct PfRing {
    uint8_t* data;  // [kSlots][kTile]
    uint64_t *full, *empty;
};
template <class Src, int DH>
__device__ __forceinline__ bool pf_convert(const PfRaw& m, const PfRing& ring, int w, volatile int* err) {
    using G = PfGeom<Src, DH>;
    using C = typename Src::C;
    constexpr int S = G::kSlots, NB = DH / kMxBlock, CPR = DH / 16, RPI = 32 / CPR, CHUNKS = 128 / (RPI * G::kCopyWarps);
    const int lane = threadIdx.x & 31;
    // A pass of the four warps covers 4 RPI rows.  8 lanes have 4 chunks of two rows whose numbers differ in bits 0 and 2
    // (dh 64: bit 0): then their loads and their stores fall into different banks
    const int chunk = CPR == 8 ? (lane & 3) | ((lane >> 1) & 4) : lane & 3;
    const int row0 = CPR == 8 ? 8 * (w >> 1) + ((2 * (w & 1) + (lane >> 4)) ^ (lane & 4 ? 5 : 0)) : 8 * w + (lane >> 2);
    const uint32_t from = smem_u32(m.data) + pf_raw_at<DH>(row0, chunk);
    const uint32_t scl = smem_u32(m.data) + (uint32_t)(G::kRaws * kPfKeys * DH + row0 * NB + (chunk >> 1));
    // chunks 2 chunk and 2 chunk + 1 of the row's 16-bit values (a pass is 16 or 32 rows further)
    const uint32_t to = smem_u32(ring.data) + (uint32_t)((chunk >> 2) * G::kAtom + row0 * 128);
    const int c2 = (2 * chunk) & 7;
    int buf = 0, bufs = 0, slot = 0, round = 0;
    bool ok = true;
    for (;;) {
        ok = pf_wait(&m.full[buf], bufs & 1);
        if (!ok || m.last[buf]) break;
        if (round > 0) ok = pf_wait(&ring.empty[slot], (round - 1) & 1);
        if (!ok || *err) break;
        const uint32_t dst = to + (uint32_t)(slot * G::kTile), src = from + (uint32_t)(buf * kPfKeys * DH), sc = scl + (uint32_t)(buf * kPfKeys * NB);
        const uint4 have = *reinterpret_cast<const uint4*>(m.rows + 4 * buf);
        const bool whole = (have.x & have.y & have.z & have.w) == 0xffffffffu;
        // Chunks whose loads are in flight together.  The loop stays one: unrolled, the code of all roles did not fit in the
        // instruction cache (4096 rows of int8 codes: 310 us, 215 as it is).
        constexpr int BATCH = 2;
#pragma unroll 1
        for (int x0 = 0; x0 < CHUNKS; x0 += BATCH) {
            uint4 w4[BATCH];
            uint32_t f[BATCH];
#pragma unroll
            for (int y = 0; y < BATCH; ++y) {
                const int r = (x0 + y) * RPI * G::kCopyWarps;
                w4[y] = lds128_at(src + (uint32_t)(r * DH));
                f[y] = lds8(sc + (uint32_t)(r * NB));
            }
            if (!whole)
#pragma unroll
                for (int y = 0; y < BATCH; ++y) {
                    const int r = row0 + (x0 + y) * RPI * G::kCopyWarps;
                    if (!((m.rows[4 * buf + (r >> 5)] >> (r & 31)) & 1u)) f[y] = 0u;
                }
#pragma unroll
            for (int y = 0; y < BATCH; ++y) {
                const uint32_t v[4] = {w4[y].x, w4[y].y, w4[y].z, w4[y].w}, k = C::scale(f[y]);
                uint32_t z[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    z[2 * e] = C::mul(C::lo(v[e]), k);
                    z[2 * e + 1] = C::mul(C::hi(v[e]), k);
                }
                const int r = (x0 + y) * RPI * G::kCopyWarps;
                const uint32_t at = dst + (uint32_t)(r * 128) + (uint32_t)((c2 ^ (row0 & 7)) << 4);
                sts128_at(at, z[0], z[1], z[2], z[3]);
                sts128_at(at ^ 16u, z[4], z[5], z[6], z[7]);
            }
        }
        fence_proxy_async_smem();  // written as threads do; the MMA reads as the copy engine does
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(&m.empty[buf]);
            mbar_arrive(&ring.full[slot]);
        }
        if (++buf == G::kRaws) buf = 0, ++bufs;
        if (++slot == S) slot = 0, ++round;
    }
    // the CTA may not end while a commit that releases a slot is on its way
    for (int s = 0; ok && s < S; ++s) {
        const int fills = round + (s < slot ? 1 : 0);
        if (fills > 0) ok = pf_wait(&ring.empty[s], (fills - 1) & 1);
    }
    return ok;
}

// Each unit's queries, once the last unit's products with its own are done.
template <class Src, int DH>
__device__ __forceinline__ bool pf_load_queries(const PfParams& P, uint8_t* Qs, uint64_t* q_full, uint64_t* q_empty, PfCursor at, int64_t left) {
    using G = PfGeom<Src, DH>;
    const PagedAttnArgs& a = P.a;
    const int tr = kPfRows / a.group;
    int nq = 0;
    bool ok = true;
    while (left > 0) {
        int n;
        at.part(left, n);
        left -= at.rest();
        if (n > 0) {
            if (nq > 0) ok = pf_wait(q_empty, (nq - 1) & 1);
            if (!ok) break;
            ++nq;
            const int tiles = (2 * at.pt + 1) * tr < at.rows ? 2 : 1;
            if (elect_one()) {
                mbar_arrive_expect_tx(q_full, (uint32_t)(tiles * (DH / 64) * tr * a.group * 128));
                for (int y = 0; y < tiles; ++y)
                    for (int h = 0; h < DH / 64; ++h)
                        tc::tma_load_3d(Qs + y * G::kTile + h * G::kAtom, &P.tq, 64 * h, at.kvh * a.group, at.row0 + (2 * at.pt + y) * tr,
                                        smem_u32(q_full));
            }
            __syncwarp();
        }
        at.next(a, tr);
    }
    if (nq > 0 && !pf_wait(q_full, (nq - 1) & 1)) ok = false;  // no tensor copy may be in flight when the CTA ends
    return ok;
}

// JOIN: the parts of units that several CTAs share are left to k_paged_join; otherwise the last of a unit's CTAs to finish
// joins them.
template <class Src, int DH, bool JOIN>
__global__ void __launch_bounds__(PfGeom<Src, DH>::kThreads, 1) k_paged_prefill(const __grid_constant__ PfParams P) {
    const PagedAttnArgs& a = P.a;
    using T = typename Src::T;
    using E = Elem<T>;
    using G = PfGeom<Src, DH>;
    constexpr int S = G::kSlots, kPfCopyWarps = G::kCopyWarps, kPfMma = G::kMma, kPfThreads = G::kThreads;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* Qs = smem;                      // [2][kTile]
    uint8_t* Rs = Qs + 2 * G::kTile;         // [S][kTile]
    uint8_t* raw = Rs + S * G::kTile;        // [kRaws][kRaw]
    uint32_t* valid = reinterpret_cast<uint32_t*>(raw + G::kRaws * G::kRaw);  // [kPfMaskRing][4]
    uint64_t* bars = reinterpret_cast<uint64_t*>(valid + kPfMaskRing * 4);
    // codes: the raw buffers' own barriers and words
    const PfRaw rw = {raw, bars, bars + G::kRaws, reinterpret_cast<uint32_t*>(bars + 2 * G::kRaws),
                      reinterpret_cast<int*>(bars + 4 * G::kRaws)};
    if (Src::kMx) bars += 4 * G::kRaws + 2;
    uint64_t* full = bars;                   // [S]
    uint64_t* empty = full + S;              // [S]
    uint64_t* q_full = empty + S;
    uint64_t* q_empty = q_full + 1;
    uint64_t* s_full = q_empty + 1;          // [2] S_x is there (and O_x holds every earlier block)
    uint64_t* p_full = s_full + 2;           // [2][2] halves of P_x, 64 keys each
    uint64_t* pv_done = p_full + 4;          // [2] one more block is in O_x, and P_x has been read
    uint64_t* o_full = pv_done + 2;          // [2] the unit's last block is in O_x
    uint64_t* o_free = o_full + 2;           // [2] O_x has been read
    uint64_t* done = o_free + 2;             // [2]
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 2);
    volatile int* s_err = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* s_last = s_err + 1;        // [2]
    int64_t* s_at = reinterpret_cast<int64_t*>(tmem_slot + 4);  // length of the line
    int* s_unit = reinterpret_cast<int*>(s_at + 2);             // [4]
    int* s_largest = reinterpret_cast<int*>(s_at + 1);          // blocks of the largest unit
    // where each warp stands between units: in shared memory, as the registers hold S meanwhile
    PfCursor* cursor = reinterpret_cast<PfCursor*>(s_unit + 4) + (threadIdx.x >> 5);

    const PagedView& c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int tr = kPfRows / a.group;  // tokens of a tile
    if (tid == 0) {
        for (int s = 0; s < S; ++s) {
            mbar_init(&full[s], kPfCopyWarps);
            mbar_init(&empty[s], 2);
        }
        mbar_init(q_full, 1);
        mbar_init(q_empty, 2);
        for (int x = 0; x < 2; ++x) {
            mbar_init(&s_full[x], 1);
            mbar_init(&p_full[2 * x], 4);
            mbar_init(&p_full[2 * x + 1], 4);
            mbar_init(&pv_done[x], 1);
            mbar_init(&o_full[x], 1);
            mbar_init(&o_free[x], 4);
        }
        if (Src::kMx)
            for (int s = 0; s < G::kRaws; ++s) {
                mbar_init(&rw.full[s], 33);  // the copying lanes, and one for what they stored
                mbar_init(&rw.empty[s], G::kCopyWarps);
            }
        mbar_init(&done[0], 1);
        mbar_init(&done[1], 1);
        *s_err = 0;
        *s_largest = 0;
        fence_mbar_init();
    }
    pdl_wait();  // a preceding kernel may hold tensor memory
    pdl_launch_dependents();
    if (JOIN && tid == 0) P.split[blockIdx.x].parts = 0;
    if (a.over && !__ldcg(a.over)) return;  // every sequence was the preceding launch's
    if (warp == kPfMma) {
        tc::tmem_alloc(tmem_slot, 512);
        tc::tmem_relinquish();
    }

    __syncthreads();
    // ---- blocks of each sequence for one KV head (a warp a sequence, a lane a tile pair); rows that
    // attend to nothing get zeros
    int64_t* tot = reinterpret_cast<int64_t*>(smem);
    PfCursor at;
    int largest = 0;
    for (int b = warp; b < c.n_seqs; b += kPfThreads / 32) {
        at.seq(a, b);
        int64_t sum = 0;
        if (at.len < 0) {
            const int end = paged_start(c, b + 1, a.n_rows);
            for (int r = at.row0; r < end; ++r)
                if (r % gridDim.x == blockIdx.x) pf_zero_row(a, r, a.n_heads * DH / 8, lane);
        } else {
            if (blockIdx.x == 0 && lane == 0 && at.rows > 0 && at.len + at.rows > c.cap) set_status(c.status, VT_DEV_KV_OVERFLOW);
            for (int p0 = 0; p0 * 2 * tr < at.rows; p0 += 32) {
                const int t0 = (p0 + lane) * 2 * tr;
                int n = 0;
                if (t0 < at.rows) {
                    int beg, end;
                    at.range(a, t0, min(t0 + 2 * tr, at.rows), beg, end);
                    n = PfCursor::blocks(beg, end);
                }
                largest = max(largest, n);
                for (unsigned none = __ballot_sync(0xffffffffu, t0 < at.rows && n == 0); none; none &= none - 1) {
                    const int z0 = (p0 + __ffs(none) - 1) * 2 * tr;
                    for (int r = z0; r < min(z0 + 2 * tr, at.rows); ++r)
                        if ((at.row0 + r) % gridDim.x == blockIdx.x) pf_zero_row(a, at.row0 + r, a.n_heads * DH / 8, lane);
                }
                sum += n > 0 ? n + kPfUnitCost : 0;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        }
        if (lane == 0) tot[b] = sum;
    }
    largest = __reduce_max_sync(0xffffffffu, largest);
    if (lane == 0 && largest > 0) atomicMax(s_largest, largest);
    __syncthreads();
    largest = *s_largest + kPfUnitCost;
    const int least = largest <= kPfWhole ? largest : kPfMinBlocks;
    // ---- where this CTA's part of the line begins
    if (warp == 0) {
        int64_t sum = 0;
        for (int b = lane; b < c.n_seqs; b += 32) sum += tot[b];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        const int64_t line = sum * c.n_kv_heads;
        const int64_t per = max(paged_div(line + gridDim.x - 1, gridDim.x), (int64_t)least);
        const int64_t t0 = blockIdx.x * per;
        if (lane == 0) s_at[0] = line;
        if (t0 < line) {
            int64_t before = 0;  // blocks of the sequences before b0, one KV head
            int b = 0;
            for (int b0 = 0;; b0 += 32) {
                const int64_t v = b0 + lane < c.n_seqs ? tot[b0 + lane] : 0;
                int64_t upto = v;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t w = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += w;
                }
                const unsigned m = __ballot_sync(0xffffffffu, (before + upto) * c.n_kv_heads > t0);
                if (m) {
                    const int k = __ffs(m) - 1;
                    b = b0 + k;
                    before += __shfl_sync(0xffffffffu, upto - v, k);
                    break;
                }
                before += __shfl_sync(0xffffffffu, upto, 31);
            }
            int64_t r = t0 - before * c.n_kv_heads;
            const int kvh = (int)paged_div(r, tot[b]);
            r -= (int64_t)kvh * tot[b];
            at.seq(a, b);
            for (int p0 = 0;; p0 += 32) {  // the tile pair
                const int q0 = (p0 + lane) * 2 * tr;
                int n = 0;
                if (q0 < at.rows) {
                    int beg, end;
                    at.range(a, q0, min(q0 + 2 * tr, at.rows), beg, end);
                    n = PfCursor::blocks(beg, end);
                    if (n > 0) n += kPfUnitCost;
                }
                int64_t upto = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int64_t w = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += w;
                }
                const unsigned m = __ballot_sync(0xffffffffu, upto > r);
                if (m) {
                    const int k = __ffs(m) - 1;
                    const int64_t skip = __shfl_sync(0xffffffffu, upto - n, k);
                    if (lane == 0) {
                        s_unit[0] = b;
                        s_unit[1] = kvh;
                        s_unit[2] = p0 + k;
                        s_unit[3] = (int)(r - skip);
                    }
                    break;
                }
                r -= __shfl_sync(0xffffffffu, upto, 31);
            }
        }
    }
    __syncthreads();
    const int64_t line = s_at[0];
    const int64_t per = max(paged_div(line + gridDim.x - 1, gridDim.x), (int64_t)least);
    const int64_t t0 = blockIdx.x * per, t1 = min(line, t0 + per);
    if (t0 >= t1) {
        if (warp == kPfMma) tc::tmem_dealloc(*tmem_slot, 512);
        return;
    }
    at.seq(a, s_unit[0]);
    at.kvh = s_unit[1];
    at.pt = s_unit[2];
    at.unit(a, tr);
    at.i = s_unit[3];
    if (lane == 0) *cursor = at;
    fence_proxy_async_smem();  // tot was written and read as threads do; the copy engine writes Q and the ring over it
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    const uint32_t tmem = *tmem_slot;  // S_0, S_1 (128 columns each, P over them), O_0, O_1
    constexpr uint32_t kOCol = 2 * kPfKeys;

    if (warp >= 8 && warp < 12)  // a whole warpgroup
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(G::kCopyRegs));
    if (G::kThreads > 384 && warp >= 12) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(G::kMmaRegs));
    if (Src::kMx && warp >= 8 && warp < kPfMma) {
        if constexpr (Src::kMx)
            if (!pf_convert<Src, DH>(rw, {Rs, full, empty}, warp - 8, s_err) && lane == 0) {
                *s_err = 1;
                set_status(c.status, VT_DEV_WAIT_TIMEOUT);
            }
    } else if (Src::kMx && warp >= kPfMma + 2) {
        if constexpr (Src::kMx) {
            const bool ok = warp == kPfMma + 2 ? pf_copy_codes<Src, DH>(P, rw, valid, *cursor, t1 - t0)
                                               : pf_load_queries<Src, DH>(P, Qs, q_full, q_empty, *cursor, t1 - t0);
            if (!ok && lane == 0) {
                *s_err = 1;
                set_status(c.status, VT_DEV_WAIT_TIMEOUT);
            }
        }
    } else if (!Src::kMx && warp >= 8 && warp < kPfMma) {
        // ================================================================ copies
        const int w = warp - 8;
        bool ok = true;
        PfCursor at = *cursor;
        const int box_rows = min(c.page_size, kPfKeys), pages = kPfKeys / box_rows;  // of a block
        constexpr int HALVES = DH / 64;
        auto page_of = [&](int p) { return c.tables[(int64_t)at.b * c.per_seq + (p >> c.page_shift)]; };
        // By tensor copies: lane i holds the page of rows i box_rows .. of block j, requested a block ahead.
        auto request = [&](int j) {
            const int p = j * kPfKeys + lane * box_rows;
            return P.tma && lane < pages && p >= at.kbeg && p < at.kend ? page_of(p) : -1;
        };
        // By asynchronous copies: a pass of a warp covers RPI rows, CPR 16-byte chunks each; lane (sub, chunk) copies its
        // chunk of rows sub, sub + RPI, ... of 8-row group g.  Groups go to the copy warps in turn.
        constexpr int CPR = DH / 8, RPI = 32 / CPR, GROUPS = (16 + kPfCopyWarps - 1) / kPfCopyWarps;
        const int chunk = lane % CPR, sub = lane / CPR;
        const uint32_t lane_dst = (uint32_t)((chunk >> 3) * G::kAtom + sub * 128);
        auto copy_row = [&](uint32_t dst, int g, int k, const uint16_t* src, bool on) {
            pf_copy16(dst + lane_dst + (uint32_t)((8 * g + k) * 128 + (((chunk & 7) ^ (sub + k)) << 4)), src, on);
        };
        uint64_t *sent1 = nullptr, *sent2 = nullptr;  // the last two groups of asynchronous copies, not yet announced
        auto announce = [&](uint64_t* bar) {
            fence_proxy_async_smem();  // the copies wrote as threads do; the MMA reads as the copy engine does
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
        };
        auto flush = [&]() {
            if (!sent1) return;
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            if (sent2) announce(sent2);
            announce(sent1);
            sent1 = sent2 = nullptr;
        };
        int slot = 0, round = 0, blk = 0, nq = 0;
        for (int64_t left = t1 - t0; ok && left > 0;) {
            int n;
            const int j0 = at.kb0 + at.part(left, n);
            left -= at.rest();
            int next_page = n > 0 ? request(j0) : 0;
            for (int j = j0; ok && j < j0 + n; ++j, ++blk) {
                const int p0 = j * kPfKeys, lo = at.kbeg - p0, hi = at.kend - p0;  // attended rows [lo, hi)
                const int page = next_page;
                if (j + 1 < j0 + n) next_page = request(j + 1);
                const bool clean = P.tma && __all_sync(0xffffffffu, lo <= 0 && hi >= kPfKeys &&
                                                                        (lane >= pages || (unsigned)page < (unsigned)c.n_pages));
                int64_t off[GROUPS];  // asynchronous copies: the lane's element in the first row of each group; -1: bad page
                if (clean) {
                    if (w == 0 && lane < 4) valid[(blk % kPfMaskRing) * 4 + lane] = 0xffffffffu;
                    __syncwarp();  // the words are stored before the elected lane arrives
                    flush();
                } else {
                    if (w == 0)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int r = 32 * q + lane;
                            bool on = r >= lo && r < hi;
                            if (on && (unsigned)page_of(p0 + r) >= (unsigned)c.n_pages) {
                                on = false;
                                set_status(c.status, VT_DEV_BAD_PAGE);
                            }
                            const uint32_t m = __ballot_sync(0xffffffffu, on);
                            if (lane == 0) valid[(blk % kPfMaskRing) * 4 + q] = m;
                        }
                    if (c.page_size >= 8)  // 8 rows that begin at a multiple of 8 lie in one page
#pragma unroll
                        for (int i = 0; i < GROUPS; ++i) {
                            const int r = 8 * (w + i * kPfCopyWarps), p = p0 + r;
                            const int pg = r < hi && r + 8 > lo && r < kPfKeys ? page_of(p) : 0;
                            off[i] = (unsigned)pg < (unsigned)c.n_pages
                                         ? pg * c.page_stride + at.kvh * c.head_stride +
                                               ((p & (c.page_size - 1)) + sub) * c.pos_stride + chunk * 8
                                         : -1;
                        }
                }
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (ok && round > 0) ok = pf_wait(&empty[slot], (round - 1) & 1);
                    if (!ok) break;
                    const uint32_t dst = smem_u32(Rs + slot * G::kTile);
                    if (clean) {
                        const CUtensorMap* map = kv == 0 ? &P.tk : &P.tv;
                        const int boxes = (pages * HALVES - w + kPfCopyWarps - 1) / kPfCopyWarps;  // of this warp
                        if (elect_one()) mbar_arrive_expect_tx(&full[slot], (uint32_t)(boxes * box_rows * 128));
                        for (int x = w; x < pages * HALVES; x += kPfCopyWarps) {
                            const int i = x / HALVES, h = x % HALVES;
                            const int pg = __shfl_sync(0xffffffffu, page, i);
                            if (elect_one())
                                tc::tma_load_4d(dst + (uint32_t)(h * G::kAtom + i * box_rows * 128), map, 64 * h,
                                                (p0 + i * box_rows) & (c.page_size - 1), at.kvh, pg, &full[slot]);
                            __syncwarp();
                        }
                    } else {
                        const uint16_t* pool = kv == 0 ? a.kpool : a.vpool;
                        if (c.page_size >= 8) {
#pragma unroll
                            for (int i = 0; i < GROUPS; ++i) {
                                const int g = w + i * kPfCopyWarps;
                                if (g >= 16) break;
                                const uint16_t* src = pool + (off[i] < 0 ? 0 : off[i]);
                                const int end = off[i] < 0 ? 0 : hi;
#pragma unroll
                                for (int k = 0; k < 8; k += RPI) {
                                    const int r = 8 * g + k + sub;
                                    copy_row(dst, g, k, src + k * c.pos_stride, r >= lo && r < end);
                                }
                            }
                        } else {
#pragma unroll 1
                            for (int g = w; g < 16; g += kPfCopyWarps)
#pragma unroll 1
                                for (int k = 0; k < 8; k += RPI) {
                                    const int r = 8 * g + k + sub, p = p0 + r;
                                    const int pg = r >= lo && r < hi ? page_of(p) : -1;
                                    const bool on = (unsigned)pg < (unsigned)c.n_pages;
                                    const int64_t o = on ? pg * c.page_stride + at.kvh * c.head_stride + (p & (c.page_size - 1)) * c.pos_stride : 0;
                                    copy_row(dst, g, k, pool + o + chunk * 8, on);
                                }
                        }
                        asm volatile("cp.async.commit_group;" ::: "memory");
                        if (sent2) {
                            asm volatile("cp.async.wait_group %0;" ::"n"(kPfLag) : "memory");
                            announce(sent2);
                        }
                        sent2 = sent1;
                        sent1 = &full[slot];
                    }
                    if (++slot == S) slot = 0, ++round;
                    if (kv == 0 && j == j0 && w == 0) {  // the unit's queries, once the last unit's products with its own are done
                        if (nq > 0) ok = pf_wait(q_empty, (nq - 1) & 1);
                        ++nq;
                        const int tiles = (2 * at.pt + 1) * tr < at.rows ? 2 : 1;
                        if (ok && elect_one()) {
                            mbar_arrive_expect_tx(q_full, (uint32_t)(tiles * HALVES * tr * a.group * 128));
                            for (int x = 0; x < tiles; ++x)
                                for (int h = 0; h < HALVES; ++h)
                                    tc::tma_load_3d(Qs + x * G::kTile + h * G::kAtom, &P.tq, 64 * h, at.kvh * a.group,
                                                    at.row0 + (2 * at.pt + x) * tr, smem_u32(q_full));
                        }
                        __syncwarp();
                    }
                }
            }
            at.next(a, tr);
        }
        if (ok) flush();
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        // nor may the CTA end while a commit that releases a slot is on its way
        for (int s = 0; ok && s < S; ++s) {
            const int fills = round + (s < slot ? 1 : 0);
            if (fills > 0) ok = pf_wait(&empty[s], (fills - 1) & 1);
        }
        if (!ok) {
            if (lane == 0) {
                *s_err = 1;
                set_status(c.status, VT_DEV_WAIT_TIMEOUT);
            }
            // no tensor copy may still be in flight when the CTA ends
            for (int s = 0; s < S; ++s) {
                const int fills = round + (s < slot ? 1 : 0);
                if (fills > 0) pf_wait(&full[s], (fills - 1) & 1);
            }
            if (w == 0 && nq > 0) pf_wait(q_full, (nq - 1) & 1);
        }
    } else if (warp >= kPfMma && warp < kPfMma + 2) {
        // ================================================================ MMAs of tile x
        constexpr uint32_t kType = std::is_same<T, __half>::value ? 0u : tc::kIdescBf16;
        constexpr uint32_t idesc_s = tc::idesc_f16(kPfRows, kPfKeys) | kType, idesc_o = tc::idesc_f16_bmn(kPfRows, DH) | kType;
        constexpr uint32_t kStep = G::kTile >> 4;
        const int x = warp - kPfMma;
        const uint32_t qd = tc::desc_sw128_lo(smem_u32(Qs + x * G::kTile)), kd = tc::desc_sw128_lo(smem_u32(Rs));
        const uint64_t vd = tc::desc_sw128_mn(smem_u32(Rs), G::kAtom);
        const uint32_t vd_hi = (uint32_t)(vd >> 32), vd_lo = (uint32_t)vd;
        const uint32_t s_tmem = tmem + (uint32_t)(x * kPfKeys), o_tmem = tmem + kOCol + (uint32_t)(x * DH);
        bool ok = true;
        int slot = 0, par = 0, nq = 0, npv = 0, seen = 0, no = 0;  // npv, seen: products with V issued, and known to be done
        for (int64_t left = t1 - t0; ok && left > 0;) {
            int n, j0, j1, lo, hi;
            {
                PfCursor at = *cursor;
                j0 = at.kb0 + at.part(left, n);
                j1 = j0 + n;
                at.tile(a, tr, x, j0, j1, lo, hi);
                left -= at.rest();
                at.next(a, tr);
                __syncwarp();  // every lane has read the cursor
                if (lane == 0) *cursor = at;
                __syncwarp();
            }
            if (n <= 0) continue;
            ok = pf_wait(q_full, nq & 1);
            ++nq;
            for (int j = j0 - 1; ok && j < j1; ++j) {
                if (j >= j0) {  // O_x += P_x . V_j
                    if (j >= lo && j < hi) {
                        if (j == lo) {
                            if (no > 0) ok = pf_wait(&o_free[x], (no - 1) & 1);
                            ++no;
                        }
#pragma unroll
                        for (int half = 0; half < 2; ++half) {
                            ok = ok && (half == 0 ? pf_wait2(&full[slot], par, &p_full[2 * x], npv & 1) : pf_wait(&p_full[2 * x + 1], npv & 1));
                            if (!ok) break;
                            tc::fence_after();
                            if (elect_one()) {
#pragma unroll
                                for (int kk = 4 * half; kk < 4 * half + 4; ++kk)
                                    tc::mma_f16_ts(o_tmem, s_tmem + (uint32_t)(kk * 8),
                                                   tc::desc_of(vd_hi, vd_lo + (uint32_t)slot * kStep + (uint32_t)kk * (2048 >> 4)), idesc_o,
                                                   (j > lo || kk > 0) ? 1u : 0u);
                                if (half == 1) {
                                    tc::mma_commit(&pv_done[x]);
                                    if (j == hi - 1) tc::mma_commit(&o_full[x]);
                                    tc::mma_commit(&empty[slot]);
                                }
                            }
                            __syncwarp();
                        }
                        ++npv;
                    } else {
                        ok = pf_wait(&full[slot], par);
                        if (ok && elect_one()) tc::mma_commit(&empty[slot]);
                        __syncwarp();
                    }
                    if (++slot == S) slot = 0, par ^= 1;
                }
                if (ok && j + 1 < j1) {  // S_x = Q_x . K_{j+1}^T, over P_x: nothing but this wait orders it behind the last product
                    const bool on = j + 1 >= lo && j + 1 < hi;
                    ok = on && seen < npv ? pf_wait2(&full[slot], par, &pv_done[x], seen & 1) : pf_wait(&full[slot], par);
                    if (on) seen = npv;
                    if (!ok) break;
                    tc::fence_after();
                    if (elect_one()) {
                        if (on) {
#pragma unroll
                            for (int kk = 0; kk < DH / 16; ++kk) {
                                const uint32_t off = (uint32_t)(kk >> 2) * (G::kAtom >> 4) + (uint32_t)(kk & 3) * 2;
                                tc::mma_f16(s_tmem, tc::desc_of(tc::kDescSw128Hi, qd + off),
                                            tc::desc_of(tc::kDescSw128Hi, kd + (uint32_t)slot * kStep + off), idesc_s, kk > 0);
                            }
                            tc::mma_commit(&s_full[x]);
                        }
                        tc::mma_commit(&empty[slot]);
                        if (j + 1 == j1 - 1) tc::mma_commit(q_empty);
                    }
                    __syncwarp();
                    if (++slot == S) slot = 0, par ^= 1;
                }
                if (*s_err) ok = false;
            }
        }
        if (!ok && lane == 0) {
            *s_err = 1;
            set_status(c.status, VT_DEV_WAIT_TIMEOUT);
        }
        // tensor memory is freed only after every MMA issued has completed
        if (elect_one()) tc::mma_commit(&done[x]);
        __syncwarp();
        if (!pf_wait(&done[x], 0) && lane == 0) set_status(c.status, VT_DEV_WAIT_TIMEOUT);
    } else if (warp < 8) {
        // ================================================================ softmax of tile x
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(G::kSoftmaxRegs));
        const int x = warp >> 2, row = tid & 127;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_at_col = tmem + lane_off + (uint32_t)(x * kPfKeys), o_at_col = tmem + lane_off + kOCol + (uint32_t)(x * DH);
        const float sl2 = a.scale_log2;
        bool ok = true;
        int ns = 0, no = 0, blk = 0;
        for (int64_t left = t1 - t0; left > 0;) {
            int n, j0, lo, hi, qp;
            bool has, live;
            {
                PfCursor at = *cursor;
                j0 = at.kb0 + at.part(left, n);
                if (n <= 0) {
                    left -= at.rest();
                    at.next(a, tr);
                    __syncwarp();  // every lane has read the cursor
                    if (lane == 0) *cursor = at;
                    __syncwarp();
                    continue;
                }
                has = at.tile(a, tr, x, j0, j0 + n, lo, hi);
                const int tok = (2 * at.pt + x) * tr + row / a.group;
                live = row < tr * a.group && tok < at.rows;
                qp = live ? at.len + tok : -1;  // position of this row (-1: it attends to nothing)
            }
            const int first_key = a.window > 0 ? qp - a.window + 1 : 0;
            float m_use = -INFINITY, l = 0.f;
            for (int j = lo; j < hi; ++j) {
                if (ok && *s_err) ok = false;
                if (ok) ok = pf_wait(&s_full[x], ns & 1);
                ++ns;
                if (!ok) continue;
                tc::fence_after();
                // S by 32 keys.  Codes: the block's threads have fewer registers and more code, so S is read in halves, once for
                // the maximum and once for the weights, both in loops.
                constexpr int KEPT = Src::kMx ? 2 : 4;
                uint32_t sv[KEPT][32];
                auto half_of_s = [&](int q) {
                    tc::tmem_ld32(s_at_col + 64 * q, sv[0]);
                    tc::tmem_ld32(s_at_col + 64 * q + 32, sv[1]);
                    tc::tmem_ld_wait_on(sv[0]);
                    tc::tmem_ld_wait_on(sv[1]);
                };
                if constexpr (!Src::kMx)
#pragma unroll
                    for (int q = 0; q < KEPT; ++q) tc::tmem_ld32(s_at_col + 32 * q, sv[q]);
                const uint32_t* vw = valid + ((blk + j - j0) % kPfMaskRing) * 4;
                const int kp0 = j * kPfKeys, cb = first_key - kp0, ce = qp + 1 - kp0;
                uint32_t mw[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) mw[q] = fa_range_bits(cb - 32 * q, ce - 32 * q) & vw[q];
                const bool plain = __all_sync(0xffffffffu, (mw[0] & mw[1] & mw[2] & mw[3]) == 0xffffffffu);
                if constexpr (Src::kMx) {
                    if (!plain) {  // hidden scores become -inf where they lie (a loop: less code, see pf_convert; its masks
                                   // worked out again, as a loop's index would put mw into memory)
#pragma unroll 1
                        for (int q = 0; q < 4; ++q) {
                            const uint32_t on = fa_range_bits(cb - 32 * q, ce - 32 * q) & vw[q];
                            tc::tmem_ld32(s_at_col + 32 * q, sv[0]);
                            tc::tmem_ld_wait_on(sv[0]);
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((on >> e) & 1u)) sv[0][e] = 0xff800000u;
                            tc::tmem_st32(s_at_col + 32 * q, sv[0]);
                        }
                        tc::tmem_st_wait();
                    }
                }
                float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                if constexpr (!Src::kMx) {
#pragma unroll
                    for (int q = 0; q < KEPT; ++q) {
                        tc::tmem_ld_wait_on(sv[q]);
                        if (!plain)
#pragma unroll
                            for (int e = 0; e < 32; ++e)
                                if (!((mw[q] >> e) & 1u)) sv[q][e] = 0xff800000u;  // -inf
                    }
#pragma unroll
                    for (int e = 0; e < 32; e += 2)
#pragma unroll
                        for (int q = 0; q < KEPT; ++q) mx[q] = fa_max3(mx[q], __uint_as_float(sv[q][e]), __uint_as_float(sv[q][e + 1]));
                } else {
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {
                        half_of_s(q);
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                mx[k] = fa_max3(mx[k], __uint_as_float(sv[k & 1][e + (k & 2)]), __uint_as_float(sv[k & 1][e + (k & 2) + 1]));
                    }
                }
                const float pm = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                const float bms = pm == -INFINITY ? pm : pm * sl2;
                float alpha = 1.f;
                bool resc = false;
                constexpr float kPfUp = std::is_same<T, __half>::value ? 7.f : 0.f;
                if (bms > m_use + (8.f + kPfUp)) {
                    const float mn = bms - kPfUp;
                    if (m_use != -INFINITY) {
                        alpha = fa_ex2(m_use - mn);
                        resc = true;
                    }
                    m_use = mn;
                }
                if (__any_sync(0xffffffffu, resc)) {  // O_x holds every earlier block (s_full)
#pragma unroll(Src::kMx ? 1 : DH / 32)
                    for (int q = 0; q < DH / 32; ++q) {
                        uint32_t o[32];
                        tc::tmem_ld32(o_at_col + 32 * q, o);
                        tc::tmem_ld_wait_on(o);
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tc::tmem_st32(o_at_col + 32 * q, o);
                    }
                    l *= alpha;
                }
                // P is rounded to the type of V, as the product needs it: half a unit in its last place, of the
                // same size as the output's own rounding.  Its first 64 keys are announced while the others are
                // worked out.
                const float nm = m_use == -INFINITY ? 0.f : -m_use;
                const uint64_t sl2x2 = f2_pack(sl2, sl2), nmx2 = f2_pack(nm, nm);
                uint64_t ls[2] = {0ull, 0ull};
#pragma unroll(Src::kMx ? 1 : 2)
                for (int q = 0; q < 2; ++q) {
                    if constexpr (Src::kMx) half_of_s(q);
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 32; ++e) {
                        const uint32_t* s2 = &sv[Src::kMx ? e >> 4 : 2 * q + (e >> 4)][2 * (e & 15)];
                        float p0, p1;
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(s2[0]), __uint_as_float(s2[1])), sl2x2, nmx2), p0, p1);
                        p0 = fa_ex2(p0);
                        p1 = fa_ex2(p1);
                        ls[e & 1] = f2_add(ls[e & 1], f2_pack(p0, p1));
                        w[e] = E::pack(p0, p1);
                    }
                    tc::tmem_st32(s_at_col + 32 * q, w);
                    tc::tmem_st_wait();
                    tc::fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[2 * x + q]);
                }
                float l0, l1;
                f2_unpack(f2_add(ls[0], ls[1]), l0, l1);
                l += l0 + l1;
            }
            blk += n;
            // ---- the tile's end here
            PfCursor at = *cursor;
            const int tok = (2 * at.pt + x) * tr + row / a.group;
            const bool any = hi > lo, whole = n == at.n;
            if (any) {
                if (ok) ok = pf_wait(&o_full[x], no & 1);
                ++no;
                if (ok) tc::fence_after();
            }
            if (!ok && lane == 0) {
                *s_err = 1;
                set_status(c.status, VT_DEV_WAIT_TIMEOUT);
            }
            uint16_t* dst = a.out + (at.row0 + tok) * a.out_ld + (int64_t)(at.kvh * a.group + row % a.group) * DH;
            if (Src::kMx && whole) {  // by 32 columns: less code (see pf_convert)
                const float inv = l == 0.f ? 0.f : 1.f / l;
                uint4* to = reinterpret_cast<uint4*>(dst);
#pragma unroll 1
                for (uint32_t q = 0; q < DH; q += 32, to += 4) {
                    uint32_t o[32];
                    if (any && ok) {
                        tc::tmem_ld32(o_at_col + q, o);
                        tc::tmem_ld_wait_on(o);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[e] = 0u;
                    }
                    if (live && ok)
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[e] = E::pack(__uint_as_float(o[8 * u + 2 * e]) * inv, __uint_as_float(o[8 * u + 2 * e + 1]) * inv);
                            to[u] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                }
            } else if (whole) {
                const float inv = l == 0.f ? 0.f : 1.f / l;
                uint32_t o[DH / 32][32];
                if (any && ok) {
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q) tc::tmem_ld32(o_at_col + 32 * q, o[q]);
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q) tc::tmem_ld_wait_on(o[q]);
                } else {
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q)
#pragma unroll
                        for (int e = 0; e < 32; ++e) o[q][e] = 0u;
                }
                if (live && ok)
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q)
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                w[e] = E::pack(__uint_as_float(o[q][8 * u + 2 * e]) * inv, __uint_as_float(o[q][8 * u + 2 * e + 1]) * inv);
                            reinterpret_cast<uint4*>(dst)[4 * q + u] = make_uint4(w[0], w[1], w[2], w[3]);
                        }
            } else if (has) {
                // a part: (m, l) and O by four columns, all rows side by side
                const int64_t u0 = t1 - left - at.i + kPfUnitCost;  // where the unit's blocks begin in the line
                const int first = (int)paged_div(u0, per), last = (int)paged_div(u0 + at.n - 1, per);
                float* part = pf_slot(a, (int)blockIdx.x, first, x);
                reinterpret_cast<float2*>(part)[row] = ok ? make_float2(m_use, l) : make_float2(-INFINITY, 0.f);
                if (Src::kMx && any && ok) {
#pragma unroll 1
                    for (int q = 0; q < DH / 32; ++q) {
                        uint32_t o[32];
                        tc::tmem_ld32(o_at_col + 32 * q, o);
                        tc::tmem_ld_wait_on(o);
                        if (live)
#pragma unroll
                            for (int u = 0; u < 8; ++u)
                                reinterpret_cast<uint4*>(part + 2 * kPfRows)[(8 * q + u) * kPfRows + row] =
                                    make_uint4(o[4 * u], o[4 * u + 1], o[4 * u + 2], o[4 * u + 3]);
                    }
                } else if (any && ok) {
                    uint32_t o[DH / 32][32];
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q) tc::tmem_ld32(o_at_col + 32 * q, o[q]);
#pragma unroll
                    for (int q = 0; q < DH / 32; ++q) tc::tmem_ld_wait_on(o[q]);
                    if (live)
#pragma unroll
                        for (int q = 0; q < DH / 32; ++q)
#pragma unroll
                            for (int u = 0; u < 8; ++u)
                                reinterpret_cast<uint4*>(part + 2 * kPfRows)[(8 * q + u) * kPfRows + row] =
                                    make_uint4(o[q][4 * u], o[q][4 * u + 1], o[q][4 * u + 2], o[q][4 * u + 3]);
                }
                if (JOIN) {
                    if (tid == 0 && first == (int)blockIdx.x)
                        P.split[first] = {last - first + 1, at.kvh, at.row0 + 2 * at.pt * tr, min(2 * tr, at.rows - 2 * at.pt * tr)};
                } else {
                    __threadfence();
                    consumer_bar(1 + x, 128);
                    if (row == 0) {
                        const int mine = atomicAdd(&a.arrived[2 * first + x], 1);
                        s_last[x] = mine == last - first;
                        if (mine == last - first) a.arrived[2 * first + x] = 0;  // ready for the next call
                    }
                    consumer_bar(1 + x, 128);
                    if (s_last[x] && live && ok) {  // the last to get here joins the parts, in CTA order
                        __threadfence();
                        float mm = -INFINITY, ll = 0.f, ref = 0.f;
                        for (int p0 = first; p0 <= last; p0 += 4) {
                            float2 ml[4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) ml[k] = __ldcg(reinterpret_cast<const float2*>(pf_slot(a, min(p0 + k, last), first, x)) + row);
                            float mn = mm;
#pragma unroll
                            for (int k = 0; k < 4; ++k) mn = fmaxf(mn, ml[k].x);
                            ref = mn == -INFINITY ? 0.f : mn;
                            ll *= fa_ex2(mm - ref);
                            mm = mn;
#pragma unroll
                            for (int k = 0; k < 4; ++k)
                                if (p0 + k <= last) ll += ml[k].y * fa_ex2(ml[k].x - ref);
                        }
                        const float inv = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll 1
                        for (int q = 0; q < DH / 32; ++q) {
                            float o[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = 0.f;
#pragma unroll 1
                            for (int p0 = first; p0 <= last; p0 += kPfJoinChunk) {
                                float4 v[kPfJoinChunk][8];
                                float f[kPfJoinChunk];
#pragma unroll
                                for (int k = 0; k < kPfJoinChunk; ++k) {
                                    const float* src = pf_slot(a, min(p0 + k, last), first, x);
                                    const float2 ml = __ldcg(reinterpret_cast<const float2*>(src) + row);
                                    f[k] = p0 + k <= last && ml.y != 0.f ? fa_ex2(ml.x - ref) * inv : 0.f;
#pragma unroll
                                    for (int u = 0; u < 8; ++u)
                                        v[k][u] = __ldcg(reinterpret_cast<const float4*>(src + 2 * kPfRows) + (8 * q + u) * kPfRows + row);
                                }
#pragma unroll
                                for (int k = 0; k < kPfJoinChunk; ++k)
                                    if (f[k] != 0.f)  // else nothing attended to there, and nothing stored
#pragma unroll
                                        for (int u = 0; u < 8; ++u) {
                                            o[4 * u] += f[k] * v[k][u].x;
                                            o[4 * u + 1] += f[k] * v[k][u].y;
                                            o[4 * u + 2] += f[k] * v[k][u].z;
                                            o[4 * u + 3] += f[k] * v[k][u].w;
                                        }
                            }
#pragma unroll
                            for (int u = 0; u < 4; ++u)
                                reinterpret_cast<uint4*>(dst)[4 * q + u] =
                                    make_uint4(E::pack(o[8 * u], o[8 * u + 1]), E::pack(o[8 * u + 2], o[8 * u + 3]),
                                               E::pack(o[8 * u + 4], o[8 * u + 5]), E::pack(o[8 * u + 6], o[8 * u + 7]));
                        }
                    }
                    consumer_bar(1 + x, 128);  // s_last is free
                }
            }
            if (any) {
                tc::fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&o_free[x]);
            }
            left -= at.rest();
            at.next(a, tr);
            __syncwarp();  // every lane has read the cursor
            if (lane == 0) *cursor = at;
            __syncwarp();
        }
    }
    tc::fence_before();
    __syncthreads();
    if (warp == kPfMma) {
        tc::fence_after();
        tc::tmem_dealloc(tmem, 512);
    }
}

// The units that several CTAs share: out = sum_p 2^(m_p - m) O_p / sum_p 2^(m_p - m) l_p over the parts in CTA order,
// so a result does not depend on timing.  All CTAs take the items (unit, tile, 16 dims) in turn; a thread has 8 dims of
// a row.  Bytes of the parts bound it, which lie in the L2.
struct PfJoin {
    PagedAttnArgs a;
    const PfSplit* split;
    int ctas;  // of the attention kernel
};
constexpr int kPfJoinThreads = 256;
template <class T, int DH>
__global__ void __launch_bounds__(kPfJoinThreads) k_paged_join(const __grid_constant__ PfJoin J) {
    using E = Elem<T>;
    const PagedAttnArgs& a = J.a;
    constexpr int ITEMS = 2 * (DH / 16);  // of a unit
    __shared__ int s_unit[kPagedMaxGrid / 2], s_n;
    const int tid = threadIdx.x, tr = kPfRows / a.group;
    pdl_wait();
    pdl_launch_dependents();
    if (tid < 32) {  // the units, in order
        int n = 0;
        for (int c0 = 0; c0 < J.ctas; c0 += 32) {
            const bool on = c0 + tid < J.ctas && __ldcg(&J.split[c0 + tid].parts) > 0;
            const unsigned m = __ballot_sync(0xffffffffu, on);
            if (on) s_unit[n + __popc(m & ((1u << tid) - 1u))] = c0 + tid;
            n += __popc(m);
        }
        if (tid == 0) s_n = n;
    }
    __syncthreads();
    const int row = tid & (kPfRows - 1);
    for (int e = blockIdx.x; e < s_n * ITEMS; e += gridDim.x) {
        const int first = s_unit[e / ITEMS], x = e % ITEMS / (ITEMS / 2), g = (e % (ITEMS / 2)) * 2 + tid / kPfRows;
        const int4 d = __ldcg(reinterpret_cast<const int4*>(J.split + first));
        const PfSplit u = {d.x, d.y, d.z, d.w};
        const int tok = x * tr + row / a.group;
        if (row >= tr * a.group || tok >= u.tokens) continue;
        auto ml_of = [&](int p) { return __ldcg(reinterpret_cast<const float2*>(pf_slot(a, first + p, first, x)) + row); };
        float mm = -INFINITY, ll = 0.f;
#pragma unroll 8
        for (int p = 0; p < u.parts; ++p) mm = fmaxf(mm, ml_of(p).x);
        const float ref = mm == -INFINITY ? 0.f : mm;
        float o[8] = {};
#pragma unroll 4
        for (int p = 0; p < u.parts; ++p) {
            const float2 ml = ml_of(p);
            const float4* src = reinterpret_cast<const float4*>(pf_slot(a, first + p, first, x) + 2 * kPfRows) + 2 * g * kPfRows + row;
            const float4 v0 = __ldcg(src), v1 = __ldcg(src + kPfRows);
            const float f = fa_ex2(ml.x - ref);
            ll += ml.y * f;
            if (ml.y != 0.f) {  // else nothing attended to there, and nothing stored
                o[0] += f * v0.x, o[1] += f * v0.y, o[2] += f * v0.z, o[3] += f * v0.w;
                o[4] += f * v1.x, o[5] += f * v1.y, o[6] += f * v1.z, o[7] += f * v1.w;
            }
        }
        const float inv = ll == 0.f ? 0.f : 1.f / ll;
        uint16_t* dst = a.out + (int64_t)(u.row0 + tok) * a.out_ld + (int64_t)(u.kvh * a.group + row % a.group) * DH + 8 * g;
        *reinterpret_cast<uint4*>(dst) = make_uint4(E::pack(o[0] * inv, o[1] * inv), E::pack(o[2] * inv, o[3] * inv),
                                                    E::pack(o[4] * inv, o[5] * inv), E::pack(o[6] * inv, o[7] * inv));
    }
}

// Workspace of both attention kernels.
static size_t part_floats() { return (size_t)(4 * g_num_sms * kPagedPrefillSlot); }
#ifndef VT_POOL_CODES
size_t paged_work_floats() {
    return std::max((size_t)(2 * kPagedMaxGrid * kPagedDecodeSlot), part_floats() + kPagedMaxGrid / 2 * sizeof(PfSplit) / sizeof(float));
}
#endif

template <class Src, int DH>
static cudaError_t prefill_dh(const PagedAttnArgs& a, cudaStream_t st) {
    // the line at the longest lengths
    const int64_t pairs = (int64_t)a.n_rows / (2 * (kPfRows / a.group)) + a.c.n_seqs;
    const int64_t span = a.window > 0 ? std::min<int64_t>((int64_t)a.window + 2 * kPfRows, a.c.cap) : a.c.cap;
    const int64_t most = pairs * a.c.n_kv_heads * (span / kPfKeys + 2 + kPfUnitCost);
    const int64_t grid = std::min<int64_t>(std::min(kPagedMaxGrid / 2, g_num_sms), (most + kPfMinBlocks - 1) / kPfMinBlocks);
    PfParams P{};
    P.a = a;
    // Where a long unit has many parts, joining them by one CTA takes longer than a second kernel, in which all SMs join.
    const bool join = pairs * a.c.n_kv_heads * kPfJoinParts <= grid && span / kPfKeys + 2 + kPfUnitCost > kPfWhole;
    P.split = reinterpret_cast<PfSplit*>(a.work + part_floats());
    const PagedView& c = a.c;
    using T = typename Src::T;
    constexpr size_t smem = PfGeom<Src, DH>::kSmem;
    const bool bf16 = !std::is_same<T, __half>::value;
    const uint64_t qd[3] = {DH, (uint64_t)a.n_heads, (uint64_t)a.n_rows};
    const uint64_t qs[2] = {DH * 2, (uint64_t)(a.q_ld ? a.q_ld : (int64_t)a.n_heads * DH) * 2};
    const uint32_t qb[3] = {64, (uint32_t)a.group, (uint32_t)(kPfRows / a.group)};
    if (!make_tensor_map(&P.tq, bf16, 3, a.q, qd, qs, qb)) return cudaErrorInvalidValue;
    // Boxes of fewer than 16 rows would cost more than the copies of 16 bytes (2 KB boxes: 1160 cycles a block of 32 KB,
    // 16 KB boxes 680, asynchronous copies 1210 to 1310, all of them measured with every SM copying from the L2).
    if (c.page_size >= 16) {  // (codes: two of them as an element of 16 bits, strides in bytes)
        constexpr uint64_t W = Src::kMx ? DH / 2 : DH, B = Src::kBytes;
        const uint64_t kd[4] = {W, (uint64_t)c.page_size, (uint64_t)c.n_kv_heads, (uint64_t)c.n_pages};
        const uint64_t ks[3] = {(uint64_t)c.pos_stride * B, (uint64_t)(c.head_stride ? c.head_stride : DH) * B,
                                (uint64_t)(c.page_stride ? c.page_stride : DH) * B};
        const uint32_t kb[4] = {(uint32_t)std::min<uint64_t>(W, 64), (uint32_t)std::min(c.page_size, kPfKeys), 1, 1};
        constexpr int span = W * 2 < 128 ? 64 : 128;
        P.tma = make_tensor_map(&P.tk, bf16, 4, a.kpool, kd, ks, kb, span) && make_tensor_map(&P.tv, bf16, 4, a.vpool, kd, ks, kb, span);
    }
    if (!join) return launch_paged_k(k_paged_prefill<Src, DH, false>, (unsigned)grid, PfGeom<Src, DH>::kThreads, smem, st, P);
    const cudaError_t e = launch_paged_k(k_paged_prefill<Src, DH, true>, (unsigned)grid, PfGeom<Src, DH>::kThreads, smem, st, P);
    if (e != cudaSuccess) return e;
    return launch_paged_k(k_paged_join<T, DH>, (unsigned)(2 * g_num_sms), kPfJoinThreads, 0, st, PfJoin{a, P.split, (int)grid});
}

template <class Src, int DH, bool JOIN>
static cudaError_t init_one() {
    cudaFuncAttributes f;
    cudaError_t e = cudaFuncGetAttributes(&f, k_paged_prefill<Src, DH, JOIN>);
    if (e != cudaSuccess) return e;
    if (f.numRegs != PfGeom<Src, DH>::kLaunchRegs) return cudaErrorInvalidConfiguration;  // (see paged_tiles_error)
    return cudaFuncSetAttribute(k_paged_prefill<Src, DH, JOIN>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)PfGeom<Src, DH>::kSmem);
}
template <class Src, int DH>
static cudaError_t init_both() {
    const cudaError_t e = init_one<Src, DH, false>();
    return e != cudaSuccess ? e : init_one<Src, DH, true>();
}

// The library's entry points to the kernel over one kind of pool: POOL<T> is what it holds, SUFFIX its name.
// The register split needs exactly the registers that it was planned with: a build that gives the kernel another number
// fails the calls that need the kernel, and no others.
#define VT_PAGED_TILES(POOL, SUFFIX)                                                                                               \
    cudaError_t launch_paged_prefill##SUFFIX(const PagedAttnArgs& a, int dtype, int dh, cudaStream_t st) {                         \
        if (dtype == VT_F16) return dh == 128 ? prefill_dh<POOL<__half>, 128>(a, st) : prefill_dh<POOL<__half>, 64>(a, st);        \
        return dh == 128 ? prefill_dh<POOL<__nv_bfloat16>, 128>(a, st) : prefill_dh<POOL<__nv_bfloat16>, 64>(a, st);               \
    }                                                                                                                              \
    static cudaError_t g_tiles_err = cudaErrorNotReady;                                                                            \
    void init_paged_prefill##SUFFIX() {                                                                                            \
        g_tiles_err = cudaSuccess;                                                                                                 \
        for (cudaError_t e : {init_both<POOL<__half>, 64>(), init_both<POOL<__half>, 128>(), init_both<POOL<__nv_bfloat16>, 64>(), \
                              init_both<POOL<__nv_bfloat16>, 128>()})                                                              \
            if (e != cudaSuccess) g_tiles_err = e;                                                                                 \
        if (g_tiles_err != cudaSuccess) cudaGetLastError(); /* not the next call's */                                              \
    }                                                                                                                              \
    const char* paged_tiles_error##SUFFIX() {                                                                                      \
        if (g_tiles_err == cudaSuccess) return nullptr;                                                                            \
        return g_tiles_err == cudaErrorInvalidConfiguration                                                                        \
                   ? "the prefill kernel on tensor-core tiles was built with another register count than its split needs"          \
                   : cudaGetErrorString(g_tiles_err);                                                                              \
    }

#ifndef VT_POOL_CODES  // (pools of codes: paged_prefill_e4m3.cu, paged_prefill_int8.cu, each a translation unit for itself)
VT_PAGED_TILES(PoolPlain, )
#endif

}  // namespace vt
