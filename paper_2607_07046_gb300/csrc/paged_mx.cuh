// Entries of a paged pool in 8 bits: a code for each dimension and a scale for each 32 of them, the power of two
// 2^(s - 127) of its byte s.  Codes are e4m3 or whole numbers (two's complement).
//
// A code times its scale is a value of the rows' type (exactly: a code has 8 significant bits at most, and the
// append keeps the scales where no step falls below the type's).  Byte 255 is NaN.  Scale 0 (which no entry has) hides
// whatever finite codes lie in entries that nothing attends to.
#pragma once

#include <cuda_fp8.h>

#include "paged.cuh"

namespace vt {

constexpr int kMxBlock = 32;  // dimensions that share a scale

// Codes of format F as pairs of values of type T, without their scale: the lower and upper two of w, or its bytes 0, 2 and
// 1, 3; and the scale of byte s as a pair to multiply them by (byte 0 gives 0, 255 NaN).
template <class T, int F>
struct MxCodes;

// e4m3: one conversion for two codes.  int8: 1024 + u, u the code + 128, is a sum of bits, less 1152.
template <int F>
struct MxCodes<__half, F> {
    static constexpr bool kFloat = F == VT_MX_E4M3;
    static __device__ __forceinline__ uint32_t convert(uint16_t two) {
        uint32_t r;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(two));
        return r;
    }
    template <int S>  // bytes S & 15 and S >> 4
    static __device__ __forceinline__ uint32_t whole(uint32_t w) {
        const uint32_t x = __byte_perm(w ^ 0x80808080u, 0x64646464u, (S & 15) | (4u << 4) | ((S >> 4) << 8) | (4u << 12));
        const uint32_t k = 0x64806480u;  // 1152
        const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&x), *reinterpret_cast<const __half2*>(&k));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ uint32_t lo(uint32_t w) {
        if constexpr (kFloat) return convert((uint16_t)w);
        return whole<0x10>(w);
    }
    static __device__ __forceinline__ uint32_t hi(uint32_t w) {
        if constexpr (kFloat) return convert((uint16_t)(w >> 16));
        return whole<0x32>(w);
    }
    static __device__ __forceinline__ void split(uint32_t w, uint32_t& even, uint32_t& odd) {
        if constexpr (kFloat) {
            const uint32_t x = __byte_perm(w, 0u, 0x3120);
            even = lo(x);
            odd = hi(x);
        } else {
            even = whole<0x20>(w);
            odd = whole<0x31>(w);
        }
    }
    static __device__ __forceinline__ uint32_t scale(uint32_t s) {
        const float f = __uint_as_float(s << 23);
        return s == 255u ? 0x7fff7fffu : Elem<__half>::pack(f, f);
    }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) {
        const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
};

// e4m3: the bits move to their places (no conversion: the value is then less by 2^120, the difference of the exponents'
// biases, which the scale makes up for; subnormal codes become subnormal numbers).  int8: 128 + the low 7 bits is a sum of
// bits, less 128, or 256 for a negative code.
template <int F>
struct MxCodes<__nv_bfloat16, F> {
    static constexpr bool kFloat = F == VT_MX_E4M3;
    template <int S>
    static __device__ __forceinline__ uint32_t two(uint32_t w) {
        if constexpr (kFloat) {
            const uint32_t x = __byte_perm(w, 0u, 4u | ((S & 15) << 4) | (4u << 8) | ((S >> 4) << 12));  // codes in the upper bytes
            const uint32_t y = (x >> 4) & 0x07f007f0u;
            return (x & 0x80008000u) | y;
        } else {
            const uint32_t x = __byte_perm(w, 0u, (S & 15) | (4u << 4) | ((S >> 4) << 8) | (4u << 12));
            const uint32_t a = (x & 0x007f007fu) | 0x43004300u, b = (x & 0x00800080u) | 0x43004300u;
            const __nv_bfloat162 r = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
            return *reinterpret_cast<const uint32_t*>(&r);
        }
    }
    static __device__ __forceinline__ uint32_t lo(uint32_t w) { return two<0x10>(w); }
    static __device__ __forceinline__ uint32_t hi(uint32_t w) { return two<0x32>(w); }
    static __device__ __forceinline__ uint32_t scale(uint32_t s) {
        const uint32_t p = s * 0x00800080u;
        return s == 255u ? 0x7fff7fffu : kFloat ? mul(p, 0x7b807b80u) : p;  // 2^120
    }
    static __device__ __forceinline__ uint32_t mul(uint32_t a, uint32_t b) {
        const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
};

// Scale b of a word of scales.
__device__ __forceinline__ float mx_scale(uint32_t w, int b) {
    return __uint_as_float((b == 3 ? w >> 1 : w << (23 - 8 * b)) & 0x7f800000u);
}

// What a pool holds: 16-bit values of type T, or 8-bit codes of format F that stand for values of type T.
template <class E>
struct PoolPlain {
    using T = E;
    static constexpr bool kMx = false, kWide = false;
    static constexpr int kBytes = 2;  // of a value
};
template <class E, int F>
struct PoolMx {
    using T = E;
    using C = MxCodes<E, F>;
    using H = MxCodes<__half, F>;
    static constexpr bool kMx = true;
    static constexpr bool kWide = F == VT_MX_INT8 && std::is_same<E, __nv_bfloat16>::value;  // scales up to 2^119
    static constexpr int kBytes = 1;
};

__device__ __forceinline__ uint4 lds128_at(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void sts128_at(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
    uint2 v;
    asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds16(uint32_t addr) {
    uint16_t v;
    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t lds8(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// The scale of a block whose largest magnitude has the bits `most` (of a float): the least E with 2^E times the
// largest code at least as large, kept in [lo, hi].
template <int F>
__device__ __forceinline__ int mx_exponent(uint32_t most, int lo, int hi) {
    const int e = (int)(most >> 23) - 127;
    const uint32_t part = most & 0x7fffffu;
    const int E = F == VT_MX_E4M3 ? e - 8 + (part > 0x600000u) : e - 6 + (part > 0x7e0000u);  // 448 = 1.75 2^8, 127 = 1.984375 2^6
    return max(lo, min(hi, E));
}
// Four codes of values already divided by the scale, ties to even; what is past the largest code becomes it.
template <int F>
__device__ __forceinline__ uint32_t mx_codes(float a, float b, float c, float d) {
    if constexpr (F == VT_MX_E4M3) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
        return lo | (hi << 16);
    } else {
        auto code = [](float x) { return (uint32_t)__float2int_rn(fminf(fmaxf(x, -127.f), 127.f)) & 0xffu; };
        return code(a) | (code(b) << 8) | (code(c) << 16) | (code(d) << 24);
    }
}

}  // namespace vt
