// Microscaled 4-bit floating point: what the quantiser, the products and the 4-bit cache share; barriers of the products and of the prompts' attention.
//
//   codes    uint8 [rows][K/2], two E2M1 values to a byte, the even column in the low half
//   scales   uint8 [rows][K/B]: MXFP4 B = 32, E8M0 (2^(byte - 127), 255 = NaN); NVFP4 B = 16, E4M3 (sign bit clear, 127 = NaN)
#pragma once

#include <cuda_bf16.h>

#include "common.cuh"

namespace elutq {

inline int mx4_block(int format) { return format == ELUTQ_MX4_MXFP4 ? 32 : 16; }

// The arguments of every entry that are the same: a format, and a K that fills whole blocks and 16-byte pieces of codes.
inline int mx4_check(int format, int rows, int K) {
    if (rows <= 0 || K <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (format != ELUTQ_MX4_MXFP4 && format != ELUTQ_MX4_NVFP4) return ELUTQ_ERR_INVALID_ARG;
    return K % 32 != 0 ? ELUTQ_ERR_SHAPE : ELUTQ_OK;
}
inline bool mx4_aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The status words of the 4-bit products, one a device (mx4_gemm.cu); a cudaError_t value each.  The current device's, copied in `stream` (which is waited for): no CUDA
// call but the device's number where no product has been launched on it.  Clearing: of every device that one has been launched on, which is waited for.
int mx4_status(unsigned* word, cudaStream_t stream);
int mx4_clear_status();

// ---- values, codes and scales on the device ---------------------------------------------

// 32 bytes at p, 32-byte aligned with WIDE and 16-byte aligned otherwise
template <bool WIDE>
__device__ __forceinline__ void load32(uint32_t (&v)[8], const void* p) {
    if constexpr (WIDE) {
        asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                     : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
    } else {
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(p)), b = __ldg(reinterpret_cast<const uint4*>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}

template <bool WIDE>
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {
    if constexpr (WIDE) {
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                     :: "l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// A word's values: one of fp32, two of 16 bits
template <int TYPE>
__device__ __forceinline__ void word_values(float* y, uint32_t v) {
    if constexpr (TYPE == ELUTQ_TYPE_F32) {
        y[0] = __uint_as_float(v);
    } else if constexpr (TYPE == ELUTQ_TYPE_F16) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
        y[0] = f.x;
        y[1] = f.y;
    } else {
        y[0] = __uint_as_float(v << 16);
        y[1] = __uint_as_float(v & 0xffff0000u);
    }
}
// Eight values (already divided by their scale) as a word of codes, the first in the lowest bits
__device__ __forceinline__ uint32_t codes_of(const float* v) {
    uint32_t d;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(d) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return d;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)byte));
    return __half2float(__ushort_as_half((uint16_t)h));
}
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float reciprocal(float x) {                // one unit in the last place off at most
    float r;
    asm("rcp.approx.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// FULL: values of up to 24 bits; otherwise of up to 11.  (The remainder is taken negative: so the sign of a zero survives.)
template <bool FULL>
__device__ __forceinline__ float quotient(float y, float s, float r) {
    float q = y * r;
    q = fmaf(fmaf(q, s, -y), -r, q);
    if constexpr (FULL) {
        const float over = fmaf(q, s, -y);
        const int above = (__float_as_int(over) ^ __float_as_int(q)) < 0 ? 0 : 1;      // |q| is above the exact quotient's magnitude
        if (over != 0.0f && q != 0.0f) q = __int_as_float((__float_as_int(q) - above) | 1);
    }
    return q;
}

// ---- barriers in shared memory ------------------------------------------------------------

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory"); }
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
// CLUSTER: what other CTAs of the cluster did in front of their arrivals is seen behind it
template <bool CLUSTER = false>
__device__ __forceinline__ bool try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    if constexpr (CLUSTER)
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
__device__ __forceinline__ unsigned long long now_ns() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __forceinline__ bool elect_one() {
    uint32_t e;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(e));
    return e != 0;
}

}  // namespace elutq
