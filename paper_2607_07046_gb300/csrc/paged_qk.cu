// Norm, rotation and append of the paged KV cache in one pass (Voltron Section 2.1, the KV cache of prefill and
// decode), into pools of 16 bits and of 8.
#include <cuda_runtime.h>

#include "paged_mx.cuh"
#include "tcgen05.cuh"

namespace vt {

// Head by head, in fp32:
//   x = x / sqrt(mean(x^2) + eps) * gain            (queries and keys, where a gain is given)
//   (a, b) = (a cos - b sin, b cos + a sin)         for the pairs of the first `rotary` dimensions: (i, i + rotary / 2),
//                                                   or the neighbours (2i, 2i + 1)
// and rounded once: to the rows' type, or (F) to codes with the scale of their 32 dimensions.
//
// dh / 16 lanes hold a head, two chunks of 8 dimensions each (two 16-byte loads): for pairs of halves those that are paired,
// so that no value goes from lane to lane but the sum of squares, and the unrotated ones side by side; for neighbours, and
// for values, 16 dimensions side by side.  A pass of a warp covers 32 / (dh / 16) heads of one row.  A warp has queries or
// keys and values only: the gains times the rotation's cosines and sines, four numbers a pair, are worked out once, lie in
// shared memory and serve all its passes.
//
// What bounds it: for prompts bytes (as for the plain append), and behind them the registers, which leave 24 warps an SM.  7
// prompts of 300 to 2500 rows, 32 query and 8 KV heads of 128, with norms and full rotation: fp16 rows 34.8 us (16 bits, 5330 GB/s),
// 34.8 (e4m3) and 36.4 (int8), bf16 rows, whose far heads are looked for, 35.8, 37.4 and 38.8; without either 32.  With a lane for
// 8 dimensions and the pairs' other halves by shuffles it took 50 and 53, with the four numbers in registers and 16 warps 36.8
// and 37.1.  The 80 registers do not hold all of it: the forms for many rows spill 8 to 64 bytes a thread.  For single
// tokens the chain starts, lengths, table, rotation.
constexpr int kQkWarps = 8, kQkCtas = 3;

// Squares of bf16 values go past what 32 bits hold.  A head whose sum of squares is below kQkSquares, or above 1 over it, is far: its
// values are multiplied by a power of two first, and eps by its square, which the norm takes out again.  That is done for all far
// heads of a warp after its others (in line it cost the prompts 2.5 us more, by registers; as it is 1.2).
constexpr float kQkSquares = 0x1p-40f;
// The power that brings the larger of a far head's largest magnitude and eps's root to 1 .. 2 (or is 2^127, or 2^-126); 1 for what is
// not finite.
template <int LPH>
__device__ __forceinline__ float qk_power(const float (&y)[16], float eps) {
    uint32_t most = __float_as_uint(sqrtf(eps));
#pragma unroll
    for (int e = 0; e < 16; ++e) most = max(most, __float_as_uint(y[e]) & 0x7fffffffu);
#pragma unroll
    for (int o = LPH / 2; o > 0; o >>= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, o));
    return most < 0x7f800000u ? __uint_as_float((uint32_t)max(1, 254 - (int)(most >> 23)) << 23) : 1.f;
}

// One row's queries, or its keys and values, from head `at` (of this lane) on: `batches` times PASSES passes.  Those in which a
// lane's head is far are left out and set in its word `far`; FAR: those alone.
template <class T, int DH, int F, bool NEIGH, int PASSES, bool OF_Q, bool FAR>
__device__ __forceinline__ void qk_heads(const PagedQkArgs& a, ulonglong2 (*coef)[DH / 16], uint32_t* far, int row, int at, int batches) {
    constexpr int LPH = DH / 16, HPW = 32 / LPH, NB = DH / kMxBlock;
    constexpr bool MX = F >= 0 && !OF_Q;
    using E = Elem<T>;
    const PagedView& c = a.c;
    const int lane = threadIdx.x & 31, s = lane % LPH, K = c.n_kv_heads, heads = OF_Q ? a.n_heads : 2 * K;
    const int part = a.rotary / 16;  // lanes of a head that rotate
    const bool turns = s < part, split = !NEIGH && turns;
    const int side = split ? s : 2 * s, other = split ? s + part : 2 * s + 1;  // the lane's chunks of queries and keys
    const uint16_t *q = a.q + row * a.q_ld + (int64_t)at * DH, *k = a.k + row * a.k_ld, *v = a.v + row * a.v_ld;
    uint4 x[PASSES][2];
    auto load = [&](int h0) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int h = h0 + i * HPW;
            const bool is_v = !OF_Q && h >= K;
            const uint16_t* src = OF_Q ? q + i * HPW * DH : is_v ? v + (h - K) * DH : k + h * DH;
            if (h < heads) {
                x[i][0] = *reinterpret_cast<const uint4*>(src + (is_v ? 2 * s : side) * 8);
                x[i][1] = *reinterpret_cast<const uint4*>(src + (is_v ? 2 * s + 1 : other) * 8);
            } else {
                x[i][0] = x[i][1] = make_uint4(0u, 0u, 0u, 0u);
            }
        }
        q += PASSES * HPW * DH;
    };
    load(at);  // the data does not depend on the position: its loads go out first
    const int b = paged_seq_of_row(c, row, lane);
    if (b < 0) return;
    const int len = paged_len(c, b), pos = len + (row - paged_start(c, b, a.n_rows));
    bool fits = len >= 0;
    if (fits && (pos >= c.cap || (a.rotary > 0 && pos >= a.rope_len))) {
        fits = false;
        if (lane == 0) set_status(c.status, VT_DEV_KV_OVERFLOW);
    }
    if (!fits) {
        if (OF_Q)
            for (int h = at; h < min(heads, at + batches * PASSES * HPW); h += HPW) {
                uint4* dst = reinterpret_cast<uint4*>(a.q_out + row * a.q_out_ld + (int64_t)h * DH);
                dst[2 * s] = dst[2 * s + 1] = make_uint4(0u, 0u, 0u, 0u);
            }
        return;
    }
    uint16_t* out_at = a.q_out + row * a.q_out_ld + (int64_t)at * DH;
    int64_t entry = 0, scale = 0;
    if (!OF_Q) {
        const int page = c.tables[(int64_t)b * c.per_seq + (pos >> c.page_shift)], in_page = pos & (c.page_size - 1);
        if ((unsigned)page >= (unsigned)c.n_pages) {
            if (lane == 0) set_status(c.status, VT_DEV_BAD_PAGE);
            return;
        }
        entry = page * c.page_stride + in_page * c.pos_stride;
        scale = page * a.scale_page + in_page * NB;
    }
    auto unpack = [](const uint4& u, float* y) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 p = E::unpack(w[e]);
            y[2 * e] = p.x;
            y[2 * e + 1] = p.y;
        }
    };
    // pair e of the lane is values first(e) and second(e) of its 16; two pairs go through an instruction
    auto first = [](int e) { return NEIGH ? 2 * e : e; };
    auto second = [](int e) { return NEIGH ? 2 * e + 1 : 8 + e; };
    // a' = a ca - b sb, b' = b cb + a sa, with the gains: (ca, -sb) and (cb, sa) of two pairs, which the heads of the warp share
    if (lane < LPH) {
        const uint16_t* gain = OF_Q ? a.q_gain : a.k_gain;
        float g[16];
        if (gain) {
            unpack(*reinterpret_cast<const uint4*>(gain + side * 8), g);
            unpack(*reinterpret_cast<const uint4*>(gain + other * 8), g + 8);
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) g[e] = 1.f;
        }
        const float4* t = reinterpret_cast<const float4*>(a.rope + (int64_t)pos * (a.rotary / 2) + s * 8);
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            const float4 f = turns ? t[e / 2] : make_float4(1.f, 0.f, 1.f, 0.f);
            coef[e][s] = {f2_pack(g[first(e)] * f.x, g[first(e + 1)] * f.z), f2_pack(-g[second(e)] * f.y, -g[second(e + 1)] * f.w)};
            coef[e + 1][s] = {f2_pack(g[second(e)] * f.x, g[second(e + 1)] * f.z), f2_pack(g[first(e)] * f.y, g[first(e + 1)] * f.w)};
        }
    }
    __syncwarp();
    const bool norm = OF_Q ? a.q_gain != nullptr : a.k_gain != nullptr;
    for (int h0 = at;;) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {  // (every lane takes part in the shuffles)
            const int h = h0 + i * HPW;
            const bool formed = OF_Q || h < K;
            bool here = h < heads;
            const int c0 = formed ? side : 2 * s, c1 = formed ? other : 2 * s + 1;
            float y[16];
            unpack(x[i][0], y);
            unpack(x[i][1], y + 8);
            float inv = 1.f;
            if (norm) {
                auto squares = [&]() {
                    uint64_t sum = f2_mul(f2_pack(y[0], y[1]), f2_pack(y[0], y[1]));
#pragma unroll
                    for (int e = 2; e < 16; e += 2) sum = f2_fma(f2_pack(y[e], y[e + 1]), f2_pack(y[e], y[e + 1]), sum);
                    float ss, s1;
                    f2_unpack(sum, ss, s1);
                    ss += s1;
#pragma unroll
                    for (int o = LPH / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                    return ss;
                };
                float ss = squares(), eps = a.eps;
                if (!FAR && std::is_same<T, __nv_bfloat16>::value && formed && here && !(ss >= kQkSquares && ss <= 1.f / kQkSquares)) {
                    *far |= 1u << ((h - at) / HPW);
                    here = false;
                }
                if (FAR) {
                    here = (*far >> ((h - at) / HPW)) & 1u;
                    const float f = qk_power<LPH>(y, eps);
#pragma unroll
                    for (int e = 0; e < 16; ++e) y[e] *= f;
                    eps = eps * f * f;
                    ss = squares();
                }
                const float ms = fmaf(ss, 1.f / DH, eps), r = rsqrtf(ms);
                // one step of Newton's method: what the root is off by, all of the head's values are, next to borders of codes too
                inv = ms < INFINITY ? fmaf(0.5f * r, fmaf(-ms * r, r, 1.f), r) : r;
            }
            if (formed) {
                const uint64_t inv2 = f2_pack(inv, inv);
#pragma unroll
                for (int e = 0; e < 8; e += 2) {  // (the root's inverse last: of products of a 16-bit value fewer are rounded)
                    const uint64_t p = f2_pack(y[first(e)], y[first(e + 1)]), r = f2_pack(y[second(e)], y[second(e + 1)]);
                    const ulonglong2 of_a = coef[e][s], of_b = coef[e + 1][s];
                    uint64_t pp = f2_mul(p, of_a.x), rr = f2_mul(r, of_b.x);
                    if (turns) pp = f2_fma(r, of_a.y, pp), rr = f2_fma(p, of_b.y, rr);
                    f2_unpack(f2_mul(pp, inv2), y[first(e)], y[first(e + 1)]);
                    f2_unpack(f2_mul(rr, inv2), y[second(e)], y[second(e + 1)]);
                }
            }
            if constexpr (!MX) {
                uint4 out[2];
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    out[j] = make_uint4(E::pack(y[8 * j], y[8 * j + 1]), E::pack(y[8 * j + 2], y[8 * j + 3]), E::pack(y[8 * j + 4], y[8 * j + 5]),
                                        E::pack(y[8 * j + 6], y[8 * j + 7]));
                if (!formed) out[0] = x[i][0], out[1] = x[i][1];  // (a value goes as it came: a NaN keeps its bits)
                if (here) {
                    uint16_t* dst = OF_Q ? out_at + i * HPW * DH
                                         : static_cast<uint16_t*>(formed ? a.kpool : a.vpool) + entry + (formed ? h : h - K) * c.head_stride;
                    *reinterpret_cast<uint4*>(dst + c0 * 8) = out[0];
                    *reinterpret_cast<uint4*>(dst + c1 * 8) = out[1];
                }
            } else {
                // largest magnitudes of the chunks, then of their 32 dimensions; as whole numbers, in which NaN is above infinity
                uint32_t m[2] = {0u, 0u};
#pragma unroll
                for (int e = 0; e < 16; ++e) m[e / 8] = max(m[e / 8], __float_as_uint(y[e]) & 0x7fffffffu);
                if (NEIGH || part % 4 == 0) {
                    const bool whole = NEIGH || !turns || !formed;  // side by side: a scale's chunks are two lanes', else one of four lanes'
                    if (whole) m[0] = m[1] = max(m[0], m[1]);
                    m[0] = max(m[0], __shfl_xor_sync(0xffffffffu, m[0], 1));
                    m[1] = max(m[1], __shfl_xor_sync(0xffffffffu, m[1], 1));
                    const uint32_t n0 = __shfl_xor_sync(0xffffffffu, m[0], 2), n1 = __shfl_xor_sync(0xffffffffu, m[1], 2);
                    if (!whole) m[0] = max(m[0], n0), m[1] = max(m[1], n1);
                } else {
                    uint32_t most[NB];
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        most[n] = max((c0 >> 2) == n ? m[0] : 0u, (c1 >> 2) == n ? m[1] : 0u);
#pragma unroll
                        for (int o = LPH / 2; o > 0; o >>= 1) most[n] = max(most[n], __shfl_xor_sync(0xffffffffu, most[n], o));
                    }
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        if ((c0 >> 2) == n) m[0] = most[n];
                        if ((c1 >> 2) == n) m[1] = most[n];
                    }
                }
                if (here) {
                    const int kvh = formed ? h : h - K;
                    uint8_t* dst = static_cast<uint8_t*>(formed ? a.kpool : a.vpool) + entry + kvh * c.head_stride;
                    uint8_t* sd = (formed ? a.kscale : a.vscale) + scale + kvh * a.scale_head;
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const bool finite = m[j] < 0x7f800000u;
                        const int p2 = mx_exponent<F>(m[j], a.e_lo, a.e_hi), ch = j == 0 ? c0 : c1;
                        const float by = __uint_as_float((uint32_t)(127 - p2) << 23);
                        uint2 code = make_uint2(0u, 0u);
                        if (finite) {
                            const float* z = y + 8 * j;
                            code.x = mx_codes<F>(z[0] * by, z[1] * by, z[2] * by, z[3] * by);
                            code.y = mx_codes<F>(z[4] * by, z[5] * by, z[6] * by, z[7] * by);
                        }
                        *reinterpret_cast<uint2*>(dst + ch * 8) = code;
                        if ((ch & 3) == 0) sd[ch >> 2] = finite ? (uint8_t)(p2 + 127) : (uint8_t)255;
                    }
                }
            }
        }
        if (--batches == 0) return;
        h0 += PASSES * HPW;
        out_at += PASSES * HPW * DH;
        load(h0);
    }
}

template <class T, int DH, int F, bool NEIGH, bool OF_Q>
__device__ __noinline__ void qk_far(const PagedQkArgs& a, ulonglong2 (*coef)[DH / 16], uint32_t* far, int row, int at, int passes) {
    qk_heads<T, DH, F, NEIGH, 1, OF_Q, true>(a, coef, far, row, at, passes);
}
// All heads of a warp.
template <class T, int DH, int F, bool NEIGH, int PASSES, bool OF_Q>
__device__ __forceinline__ void qk_warp(const PagedQkArgs& a, ulonglong2 (*coef)[DH / 16], uint32_t* far, int row, int at, int batches) {
    qk_heads<T, DH, F, NEIGH, PASSES, OF_Q, false>(a, coef, far, row, at, batches);
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        if (__any_sync(0xffffffffu, *far != 0u)) qk_far<T, DH, F, NEIGH, OF_Q>(a, coef, far, row, at, batches * PASSES);
}

// A row's warps: its queries', then its keys' and values', of `batches` times PASSES passes each at most.
template <class T, int DH, int F, bool NEIGH, int PASSES>
__global__ void __launch_bounds__(kQkWarps * 32, kQkCtas) k_paged_append_qk(const __grid_constant__ PagedQkArgs a) {
    constexpr int HPW = 32 / (DH / 16), HPB = HPW * PASSES;  // heads of a batch
    __shared__ ulonglong2 coef[kQkWarps][8][DH / 16];
    __shared__ uint32_t far[kQkWarps * 32];
    far[threadIdx.x] = 0u;
    pdl_wait();
    pdl_launch_dependents();
    const int lane = threadIdx.x & 31;
    const int q_warps = (a.n_heads + HPB * a.batches - 1) / (HPB * a.batches), kv_warps = (2 * a.c.n_kv_heads + HPB * a.batches - 1) / (HPB * a.batches);
    const int64_t gw = (int64_t)blockIdx.x * kQkWarps + (threadIdx.x >> 5);
    const int row = (int)paged_div(gw, q_warps + kv_warps);
    if (row >= a.n_rows) return;
    const int w = (int)(gw - (int64_t)row * (q_warps + kv_warps)), sub = lane / (DH / 16);
    if (w < q_warps) {
        const int from = w * HPB * a.batches;
        qk_warp<T, DH, F, NEIGH, PASSES, true>(a, coef[threadIdx.x >> 5], &far[threadIdx.x], row, from + sub, min(a.batches, (a.n_heads - from + HPB - 1) / HPB));
    } else {
        const int from = (w - q_warps) * HPB * a.batches;
        qk_warp<T, DH, F, NEIGH, PASSES, false>(a, coef[threadIdx.x >> 5], &far[threadIdx.x], row, from + sub, min(a.batches, (2 * a.c.n_kv_heads - from + HPB - 1) / HPB));
    }
}

// Few rows: a warp a pass, so that all loads are in flight at once.  Many: several passes a warp share the rotation,
// the gains and the search for the sequence.  (32 query and 8 KV heads of 128, a pass a warp and several: 2048 rows 20 and 15 us, 1024
// 10.8 and 8.2; at 512 and below both take the call's own time, 8.  The prompts above, 16 bits and e4m3: 4 passes twice
// 35.3 and 35.3 us, 4 once 35.4 and 39.2, 3 three times 37.1 and 37.3; 2 passes and 4 CTAs an SM 34.1 and 36.4 twice, 37.6 and 36.5
// four times; 2 CTAs 38.)
constexpr int kQkPasses = 4, kQkBatches = 2, kQkManyRows = 512;

template <class T, int DH, int F, bool NEIGH, int PASSES>
static cudaError_t qk_passes(PagedQkArgs a, cudaStream_t st) {
    constexpr int HPB = 32 / (DH / 16) * PASSES;
    a.batches = PASSES == 1 ? 1 : kQkBatches;
    const int64_t warps = (int64_t)a.n_rows * ((a.n_heads + HPB * a.batches - 1) / (HPB * a.batches) + (2 * a.c.n_kv_heads + HPB * a.batches - 1) / (HPB * a.batches));
    return launch_paged_k(k_paged_append_qk<T, DH, F, NEIGH, PASSES>, (unsigned)((warps + kQkWarps - 1) / kQkWarps), kQkWarps * 32, 0,
                          st, a);
}
template <class T, int DH, int F>
static cudaError_t qk_pairs(const PagedQkArgs& a, cudaStream_t st) {
    const bool many = a.n_rows >= kQkManyRows;
    if (a.neighbours) return many ? qk_passes<T, DH, F, true, kQkPasses>(a, st) : qk_passes<T, DH, F, true, 1>(a, st);
    return many ? qk_passes<T, DH, F, false, kQkPasses>(a, st) : qk_passes<T, DH, F, false, 1>(a, st);
}
template <class T, int F>
static cudaError_t qk_dh(const PagedQkArgs& a, int dh, cudaStream_t st) {
    return dh == 128 ? qk_pairs<T, 128, F>(a, st) : qk_pairs<T, 64, F>(a, st);
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
