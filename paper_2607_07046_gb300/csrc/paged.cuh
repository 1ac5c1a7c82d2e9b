// Shared by the kernels of the paged KV cache: 16-bit element types, the view of a pool through the
// page tables of a batch, and the search for a row's sequence.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <stdint.h>

#include <type_traits>

#include "device.cuh"
#include "internal.h"

namespace vt {

// A launch that may set up while the preceding kernel of the stream finishes.
template <typename Args>
static cudaError_t launch_paged_k(void (*kern)(Args), unsigned grid, int threads, size_t smem, cudaStream_t st,
                                  const Args& a) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = g_use_pdl ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

// Two 16-bit elements of a word as floats, and back (round to nearest even).
template <class T>
struct Elem;
template <>
struct Elem<__half> {
    static __device__ __forceinline__ float2 unpack(uint32_t u) { return h2_to_f2(u); }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};
template <>
struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float2 unpack(uint32_t u) {
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
    static __device__ __forceinline__ uint32_t pack(float lo, float hi) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&h);
    }
};

// Length of sequence b, clamped so that adding rows cannot overflow.  A row's window ends at its true position, also past
// the table, so lengths are true up to the one that leaves a window nothing of the table: the capacity (at most 2^30) plus
// the window, and at most 2^31 - 2^25.
__device__ __forceinline__ int paged_len(const PagedView& c, int b) { return min(c.lens[b], c.len_most); }

// Element offset of the entry of position p of sequence b (K head h), or -1 when its page id is not
// one of the pool's (flagged).  p is inside [0, cap).
__device__ __forceinline__ int64_t paged_entry(const PagedView& c, int b, int h, int p) {
    const int page = c.tables[(int64_t)b * c.per_seq + (p >> c.page_shift)];
    if ((unsigned)page >= (unsigned)c.n_pages) {
        set_status(c.status, VT_DEV_BAD_PAGE);
        return -1;
    }
    return page * c.page_stride + h * c.head_stride + (p & (c.page_size - 1)) * c.pos_stride;
}

// a / b for a, b >= 0; the 64-bit division takes about four times as long as the 32-bit one.
__device__ __forceinline__ int64_t paged_div(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// First row of sequence b, and the row past its last, inside [0, n_rows].
__device__ __forceinline__ int paged_start(const PagedView& c, int b, int n_rows) {
    return c.starts ? max(0, min(n_rows, c.starts[b])) : b;
}

// The sequence that holds `row` (every lane of the warp takes part; -1: none): the last b with
// starts[b] <= row, 32 candidates a round, so that the chain of dependent loads is two for up to
// 1024 sequences.
__device__ __forceinline__ int paged_seq_of_row(const PagedView& c, int row, int lane) {
    if (!c.starts) return row < c.n_seqs ? row : -1;
    int lo = 0, n = c.n_seqs;  // candidates lo .. lo + n - 1
    while (n > 0) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool le = lane * step < n && c.starts[at] <= row;
        const unsigned m = __ballot_sync(0xffffffffu, le);
        if (m == 0) return -1;
        const int k = 31 - __clz(m);
        const int left = n - k * step;
        lo += k * step;
        n = min(step, left);
        if (step == 1) break;
    }
    return row < c.starts[lo + 1] ? lo : -1;
}

}  // namespace vt
