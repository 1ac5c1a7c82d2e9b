// Norm, rotation and append of the paged KV cache in one pass (Voltron Section 2.1, the KV cache of prefill and
// decode), into pools of 16 bits and of 8.
#include <cuda_runtime.h>

#include "paged_mx.cuh"

namespace vt {

// Head by head, in fp32:
//   x = x / sqrt(mean(x^2) + eps) * gain            (queries and keys, where a gain is given)
//   (a, b) = (a cos - b sin, b cos + a sin)         for the pairs of the first `rotary` dimensions: (i, i + rotary / 2),
//                                                   or the neighbours (2i, 2i + 1)
// and rounded once: to the rows' type, or (F) to codes with the scale of their 32 dimensions.
//
// dh / 8 lanes hold a head, 8 dimensions each (one 16-byte load): the sum of squares takes a few shuffles, the other
// half of a pair comes from one other lane (neighbours lie in the lane), and four lanes share a scale.  A pass of a
// warp covers 32 / (dh / 8) heads of one row.
constexpr int kQkWarps = 8;

template <class T, int DH, int F, int PASSES>
__global__ void __launch_bounds__(kQkWarps * 32) k_paged_append_qk(const __grid_constant__ PagedQkArgs a) {
    constexpr int LPH = DH / 8, HPW = 32 / LPH, NB = DH / kMxBlock;
    constexpr bool MX = F >= 0;
    constexpr int FF = MX ? F : 0;
    using E = Elem<T>;
    pdl_wait();
    pdl_launch_dependents();
    const PagedView& c = a.c;
    const int lane = threadIdx.x & 31, sub = lane % LPH;
    const int H = a.n_heads, K = c.n_kv_heads, heads = H + 2 * K;
    const int per_row = (heads + HPW * PASSES - 1) / (HPW * PASSES);  // warps of a row
    const int64_t gw = (int64_t)blockIdx.x * kQkWarps + (threadIdx.x >> 5);
    const int row = (int)(gw / per_row), h0 = (int)(gw - (int64_t)row * per_row) * HPW * PASSES + lane / LPH;
    if (row >= a.n_rows) return;
    // the data does not depend on the position: its loads go out first
    uint4 x[PASSES];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int h = h0 + i * HPW;
        const uint16_t* src = h < H       ? a.q + row * a.q_ld + (int64_t)h * DH
                              : h < H + K ? a.k + row * a.k_ld + (int64_t)(h - H) * DH
                                          : a.v + row * a.v_ld + (int64_t)(h - H - K) * DH;
        x[i] = h < heads ? *reinterpret_cast<const uint4*>(src + sub * 8) : make_uint4(0u, 0u, 0u, 0u);
    }
    const int b = paged_seq_of_row(c, row, lane);
    if (b < 0) return;
    const int len = paged_len(c, b), pos = len + (row - paged_start(c, b, a.n_rows));
    bool fits = len >= 0;
    if (fits && (pos >= c.cap || (a.rotary > 0 && pos >= a.rope_len))) {
        fits = false;
        if (lane == 0) set_status(c.status, VT_DEV_KV_OVERFLOW);
    }
    // this lane's part of the rotation.  Halves: lanes 0 .. part - 1 have a, the next `part` b; neighbours: each has 4 pairs
    const int part = a.rotary / 16;
    const bool turns = sub < 2 * part, second = turns && !a.neighbours && sub >= part;
    const int other = a.neighbours || !turns ? lane : second ? lane - part : lane + part;
    float2 cs[8];
    int page = -1;
    if (fits) {
        if (turns) {
            const float4* t = reinterpret_cast<const float4*>(a.rope + (int64_t)pos * (a.rotary / 2) +
                                                              (a.neighbours ? sub * 4 : (second ? sub - part : sub) * 8));
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < 2 || !a.neighbours) {
                    const float4 f = t[e];
                    cs[2 * e] = make_float2(f.x, f.y);
                    cs[2 * e + 1] = make_float2(f.z, f.w);
                }
        }
        page = c.tables[(int64_t)b * c.per_seq + (pos >> c.page_shift)];
        if ((unsigned)page >= (unsigned)c.n_pages) {
            page = -1;
            if (lane == 0) set_status(c.status, VT_DEV_BAD_PAGE);
        }
    }
    const int in_page = pos & (c.page_size - 1);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {  // (every lane takes part in the shuffles)
        const int h = h0 + i * HPW;
        const uint32_t u[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        float y[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = E::unpack(u[e]);
            y[2 * e] = p.x;
            y[2 * e + 1] = p.y;
        }
        const bool formed = h < H + K;
        const uint16_t* gain = h < H ? a.q_gain : formed ? a.k_gain : nullptr;
        if (__any_sync(0xffffffffu, gain != nullptr)) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) ss += y[e] * y[e];
#pragma unroll
            for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            if (gain) {
                const float inv = rsqrtf(ss * (1.f / DH) + a.eps);
                const uint4 g = *reinterpret_cast<const uint4*>(gain + sub * 8);
                const uint32_t gu[4] = {g.x, g.y, g.z, g.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 f = E::unpack(gu[e]);
                    y[2 * e] *= inv * f.x;
                    y[2 * e + 1] *= inv * f.y;
                }
            }
        }
        if (part > 0 && __any_sync(0xffffffffu, formed)) {
            if (a.neighbours) {
                if (formed && turns && fits)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = y[2 * e], r = y[2 * e + 1];
                        y[2 * e] = p * cs[e].x - r * cs[e].y;
                        y[2 * e + 1] = r * cs[e].x + p * cs[e].y;
                    }
            } else {
                float w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = __shfl_sync(0xffffffffu, y[e], other);
                if (formed && turns && fits)
#pragma unroll
                    for (int e = 0; e < 8; ++e) y[e] = y[e] * cs[e].x + (second ? w[e] : -w[e]) * cs[e].y;
            }
        }
        const bool q_row = h < H, is_k = formed && !q_row, stored = !q_row && h < heads && page >= 0;
        const int kvh = is_k ? h - H : h - H - K;
        uint32_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) out[e] = fits ? E::pack(y[2 * e], y[2 * e + 1]) : 0u;
        if (q_row) {
            *reinterpret_cast<uint4*>(a.q_out + row * a.q_out_ld + (int64_t)h * DH + sub * 8) =
                make_uint4(out[0], out[1], out[2], out[3]);
        } else if (!MX && stored) {
            uint16_t* dst = static_cast<uint16_t*>(is_k ? a.kpool : a.vpool) + page * c.page_stride + kvh * c.head_stride +
                            in_page * c.pos_stride;
            // (a value goes as it came: a NaN keeps its bits)
            *reinterpret_cast<uint4*>(dst + sub * 8) = is_k ? make_uint4(out[0], out[1], out[2], out[3]) : x[i];
        }
        if constexpr (MX)
            if (__any_sync(0xffffffffu, stored)) {
            uint32_t most = 0u;  // compared as whole numbers, in which NaN is above infinity
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __float_as_uint(y[e]) & 0x7fffffffu);
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
            const bool finite = most < 0x7f800000u;
            const int p2 = mx_exponent<FF>(most, a.e_lo, a.e_hi);
            const float inv = finite ? __uint_as_float((uint32_t)(127 - p2) << 23) : 0.f;
            uint32_t lo = 0u, hi = 0u;
            if (finite) {
                lo = mx_codes<FF>(y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv);
                hi = mx_codes<FF>(y[4] * inv, y[5] * inv, y[6] * inv, y[7] * inv);
            }
            // the head's scales in one word
            uint32_t s = (finite ? (uint32_t)(p2 + 127) : 255u) << (8 * (sub >> 2));
            s |= __shfl_xor_sync(0xffffffffu, s, 4);
            if (NB == 4) s |= __shfl_xor_sync(0xffffffffu, s, 8);
            if (stored) {
                uint8_t* dst = static_cast<uint8_t*>(is_k ? a.kpool : a.vpool) + page * c.page_stride + kvh * c.head_stride +
                               in_page * c.pos_stride;
                *reinterpret_cast<uint2*>(dst + sub * 8) = make_uint2(lo, hi);
                uint8_t* sd = (is_k ? a.kscale : a.vscale) + page * a.scale_page + kvh * a.scale_head + in_page * NB;
                if (sub == 0) {
                    if (NB == 4)
                        *reinterpret_cast<uint32_t*>(sd) = s;
                    else
                        *reinterpret_cast<uint16_t*>(sd) = (uint16_t)s;
                }
            }
        }
    }
}

// Few rows: a warp a pass, so that all loads are in flight at once.  Many: several passes a warp share the rotation
// and the search for the sequence.
constexpr int kQkPasses = 3, kQkManyRows = 512;

template <class T, int DH, int F, int PASSES>
static cudaError_t qk_passes(const PagedQkArgs& a, cudaStream_t st) {
    constexpr int HPW = 32 / (DH / 8);
    const int heads = a.n_heads + 2 * a.c.n_kv_heads;
    const int64_t warps = (int64_t)a.n_rows * ((heads + HPW * PASSES - 1) / (HPW * PASSES));
    return launch_paged_k(k_paged_append_qk<T, DH, F, PASSES>, (unsigned)((warps + kQkWarps - 1) / kQkWarps), kQkWarps * 32, 0,
                          st, a);
}
template <class T, int F>
static cudaError_t qk_dh(const PagedQkArgs& a, int dh, cudaStream_t st) {
    const bool many = a.n_rows >= kQkManyRows;
    if (dh == 128) return many ? qk_passes<T, 128, F, kQkPasses>(a, st) : qk_passes<T, 128, F, 1>(a, st);
    return many ? qk_passes<T, 64, F, kQkPasses>(a, st) : qk_passes<T, 64, F, 1>(a, st);
}
template <class T>
static cudaError_t qk_format(const PagedQkArgs& a, int format, int dh, cudaStream_t st) {
    if (format == VT_MX_E4M3) return qk_dh<T, VT_MX_E4M3>(a, dh, st);
    if (format == VT_MX_INT8) return qk_dh<T, VT_MX_INT8>(a, dh, st);
    return qk_dh<T, -1>(a, dh, st);
}
cudaError_t launch_paged_append_qk(const PagedQkArgs& a, int dtype, int format, int dh, cudaStream_t st) {
    return dtype == VT_F16 ? qk_format<__half>(a, format, dh, st) : qk_format<__nv_bfloat16>(a, format, dh, st);
}

}  // namespace vt
