// Rotation and append of the paged KV cache (Voltron Section 2.1, the KV cache of prefill and decode, for
// several sequences in pages of one pool).
#include <cuda_runtime.h>

#include "paged.cuh"

namespace vt {

// ================================================================== append
//
// k'[i] = k[i] cos - k[i + dh/2] sin, k'[i + dh/2] = k[i + dh/2] cos + k[i] sin, in fp32 and rounded
// once; the same for q; v is copied.  dh / 16 lanes hold a head (8 dimensions of each half, two 16-byte
// loads), so a pass of a warp covers 32 / (dh / 16) heads of one row, and the rotation of a row is
// loaded once for a warp's PASSES passes.
//
// What bounds it: bytes (q, k and v read, q and the entries written) for prompts: 7 prompts of 300 to 2500 rows, 32 query
// and 8 KV heads of 128: 29.7 us, 6250 GB/s (92% of a copy's rate; with one pass a warp 34.5, as the rotation came from
// the L2 for every 4 heads).  For single tokens the chain starts, lengths, table: 2.0 us for one, 2.4 for 64.
constexpr int kAppendWarps = 8;

template <class T, int DH, int PASSES>
__global__ void __launch_bounds__(kAppendWarps * 32) k_paged_append(const __grid_constant__ PagedAppendArgs a) {
    constexpr int LPH = DH / 16, HPW = 32 / LPH;
    using E = Elem<T>;
    pdl_wait();
    pdl_launch_dependents();
    const PagedView& c = a.c;
    const int lane = threadIdx.x & 31, sub = lane % LPH;
    const int H = a.n_heads, K = c.n_kv_heads, heads = H + 2 * K;
    const int per_row = (heads + HPW * PASSES - 1) / (HPW * PASSES);  // warps of a row
    const int64_t gw = (int64_t)blockIdx.x * kAppendWarps + (threadIdx.x >> 5);
    const int row = (int)(gw / per_row), h0 = (int)(gw - (int64_t)row * per_row) * HPW * PASSES + lane / LPH;
    if (row >= a.n_rows) return;
    // the data does not depend on the position: its loads go out first
    uint4 x[PASSES][2];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int h = h0 + i * HPW;
        const uint16_t* src = h < H       ? a.q + row * a.q_ld + (int64_t)h * DH
                              : h < H + K ? a.k + row * a.k_ld + (int64_t)(h - H) * DH
                                          : a.v + row * a.v_ld + (int64_t)(h - H - K) * DH;
        if (h < heads) {
            x[i][0] = *reinterpret_cast<const uint4*>(src + sub * 8);
            x[i][1] = *reinterpret_cast<const uint4*>(src + DH / 2 + sub * 8);
        }
    }
    const int b = paged_seq_of_row(c, row, lane);
    if (b < 0) return;
    const int len = paged_len(c, b), pos = len + (row - paged_start(c, b, a.n_rows));
    bool fits = len >= 0;
    if (fits && (pos >= c.cap || pos >= a.rope_len)) {
        fits = false;
        if (lane == 0) set_status(c.status, VT_DEV_KV_OVERFLOW);
    }
    float2 cs[8];
    int64_t entry = -1;
    if (fits) {
        const float4* t = reinterpret_cast<const float4*>(a.rope + (int64_t)pos * (DH / 2) + sub * 8);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float4 f = t[e];
            cs[2 * e] = make_float2(f.x, f.y);
            cs[2 * e + 1] = make_float2(f.z, f.w);
        }
        entry = paged_entry(c, b, 0, pos);
    }
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int h = h0 + i * HPW;
        if (h >= heads) continue;
        if (h < H + K) {
            const uint32_t u[4] = {x[i][0].x, x[i][0].y, x[i][0].z, x[i][0].w},
                           w[4] = {x[i][1].x, x[i][1].y, x[i][1].z, x[i][1].w};
            uint32_t lo[4] = {0u, 0u, 0u, 0u}, hi[4] = {0u, 0u, 0u, 0u};
            if (fits) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 p = E::unpack(u[e]), r = E::unpack(w[e]);
                    const float2 c0 = cs[2 * e], c1 = cs[2 * e + 1];
                    lo[e] = E::pack(p.x * c0.x - r.x * c0.y, p.y * c1.x - r.y * c1.y);
                    hi[e] = E::pack(r.x * c0.x + p.x * c0.y, r.y * c1.x + p.y * c1.y);
                }
            }
            x[i][0] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            x[i][1] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        }
        uint16_t* dst;
        if (h < H)
            dst = a.q_out + row * a.q_out_ld + (int64_t)h * DH;
        else if (entry < 0)
            continue;
        else
            dst = (h < H + K ? a.kpool + (h - H) * c.head_stride : a.vpool + (h - H - K) * c.head_stride) + entry;
        *reinterpret_cast<uint4*>(dst + sub * 8) = x[i][0];
        *reinterpret_cast<uint4*>(dst + DH / 2 + sub * 8) = x[i][1];
    }
}

template <class T, int DH, int PASSES>
static cudaError_t append_passes(const PagedAppendArgs& a, cudaStream_t st) {
    constexpr int HPW = 32 / (DH / 16);
    const int heads = a.n_heads + 2 * a.c.n_kv_heads;
    const int64_t warps = (int64_t)a.n_rows * ((heads + HPW * PASSES - 1) / (HPW * PASSES));
    return launch_paged_k(k_paged_append<T, DH, PASSES>, (unsigned)((warps + kAppendWarps - 1) / kAppendWarps),
                          kAppendWarps * 32, 0, st, a);
}

// Few rows: a warp a pass, so that all loads are in flight at once (one row: 2.0 us a launch).  Many: three passes a warp
// share the rotation and the search for the sequence (7392 rows of 32 + 16 heads: 34.4 us at one pass, 30.7 at two, 29.7
// at three, 29.9 at four, 31.8 at eight; 185 MB at the copy rate take 27.3).
constexpr int kAppendPasses = 3, kAppendManyRows = 512;

template <class T, int DH>
static cudaError_t append_dh(const PagedAppendArgs& a, cudaStream_t st) {
    return a.n_rows >= kAppendManyRows ? append_passes<T, DH, kAppendPasses>(a, st) : append_passes<T, DH, 1>(a, st);
}

cudaError_t launch_paged_append(const PagedAppendArgs& a, int dtype, int dh, cudaStream_t st) {
    if (dtype == VT_F16) return dh == 128 ? append_dh<__half, 128>(a, st) : append_dh<__half, 64>(a, st);
    return dh == 128 ? append_dh<__nv_bfloat16, 128>(a, st) : append_dh<__nv_bfloat16, 64>(a, st);
}

}  // namespace vt
