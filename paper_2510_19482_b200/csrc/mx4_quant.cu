// Microscaled 4-bit floating point: dense values to codes and block scales, and back.
//
// A block is 32 (MXFP4) or 16 (NVFP4) consecutive columns of a row.  With amax its largest magnitude:
//
//   MXFP4   scale 2^e, e = floor(log2(amax)) - 2 (the exponent field of amax less that of 6), not below 2^-127.  Dividing by it
//           is exact, so a code is one rounding of the value.  Values above 6 scales (amax / 2^e is below 8) become 6.
//   NVFP4   scale E4M3(amax / 6), the quotient rounded to fp32 first; 448 at most, 0 where amax is below 6 * 2^-10 (all codes are 0 then)
//   code    the E2M1 value nearest to value / scale, ties to the even code, 6 at most, with the value's sign
//
// NVFP4's quotient: a code has to be that of the exact value / scale, and a value half-way between two codes is common (a scale has
// four significant bits, a half-way point three).  r = 1 / s within a unit in the last place, q = y r and one correction by the remainder
// y - q s (exact in a fused multiply-add) give the quotient rounded to nearest: what is left is 2^-21 of a unit, and a quotient by four bits
// is a 30th of a unit or more from where rounding changes, unless it is exact.  So a true tie is hit exactly, and
// for 16-bit inputs nothing else rounds onto a half-way point (y and the point times s have at most 11 bits between them).  For
// 24-bit values something can: by the remainder's sign the quotient is then rounded to odd (cut off, and the last bit set if anything
// was left), which no half-way point is.
//
// Bound: HBM.  A thread takes 32 columns (loads and stores of 32 bytes, whole sectors; one block of MXFP4 or two of NVFP4, so no amax is shared between
// threads) and moves 16 bytes of codes.  With 16 columns and stores of 16 bytes 14336 x 4096 values came back at 4.7 TB/s.
#include <cuda_bf16.h>

#include "mx4.cuh"

namespace elutq {

namespace {

constexpr int kChunk = 32;                 // columns of a thread

struct QuantArgs {
    const void* X;
    long long ld;              // elements between rows of X
    const float* prescale;     // null: 1
    const int* index;          // null: row r of X; otherwise row index[r] / div (none: zeros)
    const int* n_rows;         // null: all
    uint4* codes;
    uint8_t* scales;
    int row0, rows, K;         // this launch: rows [row0, row0 + rows)
    long long x_rows;          // rows of X, times div
    Div per_row, div;          // chunks of a row; the index's divisor
    int wide;                  // rows of X start on 32 bytes
    int pairs;                 // scales start on 2 bytes
};

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

// 32 bytes of X from element `at` on, and their values: 8 of fp32, 16 of 16 bits
template <int TYPE, bool WIDE>
__device__ __forceinline__ void load_raw(uint32_t (&v)[8], const void* X, long long at) {
    load32<WIDE>(v, reinterpret_cast<const uint8_t*>(X) + at * (TYPE == ELUTQ_TYPE_F32 ? 4 : 2));
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
template <int TYPE>
__device__ __forceinline__ void values_of(float* y, const uint32_t (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) word_values<TYPE>(y + (TYPE == ELUTQ_TYPE_F32 ? i : 2 * i), v[i]);
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
// g / (1 + exp(-g)) within a few units in the last place.  exp(-g) = 2^t 2^lo with t = -g log2(e) rounded and lo what that left, also of
// the constant (|lo| < 2^-17), 2^lo = 1 + lo ln 2.  Where exp(-g) is
// above kOpen (g below -63.7) or NaN (g above 10^38), gate_far_out has the result.
__device__ __forceinline__ float silu(float g, float& e) {
    float r;
    const float t = g * -1.44269502f;
    const float lo = fmaf(g, -1.92596303e-8f, fmaf(g, -1.44269502f, -t));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    e = fmaf(e, lo * 0.693147182f, e);
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return g * r;
}
// silu(g) u for |g| above 60.  Below zero exp(g) may have left the range of fp32 though its product with u has not: 1 + exp(-g) is exp(-g) there, so
// g exp(g) u, with exp(g) = 2^n h (h within 2^-22) and the powers of two last, in two steps that are both normal.  The first step only rounds what the second takes
// to 0, so a subnormal result is rounded once.  Below -200 nothing is left of the largest u; -inf counts as such (0 u).
constexpr float kOpen = 0x1p92f;
__device__ __forceinline__ float gate_far_out(float g, float u) {
    if (g > 0.0f) return g * u;
    g = fmaxf(g, -200.0f);
    const float n = rintf(g * 1.44269502f);
    float h;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(h) : "f"(fmaf(g, 1.92596303e-8f, fmaf(g, 1.44269502f, -n))));
    const int m = (int)n + 40, half = m >> 1;                          // -249 to -47
    return g * h * 0x1p-40f * u * __int_as_float((127 + half) << 23) * __int_as_float((127 + m - half) << 23);
}
// Of a word of gates, with that of u `apart` words on: the values given, those of gates far out replaced
template <int TYPE>
__device__ __noinline__ float2 far_out_word(const uint32_t* gates, int apart, float y0, float y1) {
    float gate[2], up[2];
    word_values<TYPE>(gate, __ldg(gates));
    word_values<TYPE>(up, __ldg(gates + apart));
    if (fabsf(gate[0]) > 60.0f) y0 = gate_far_out(gate[0], up[0]);
    if constexpr (TYPE == ELUTQ_TYPE_F32) return make_float2(y0, y0);
    if (fabsf(gate[1]) > 60.0f) y1 = gate_far_out(gate[1], up[1]);
    return make_float2(y0, y1);
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

template <int FMT, int TYPE, bool SWIGLU, bool WIDE>
__device__ __forceinline__ void quantise_chunk(const QuantArgs& a, int row, int chunk) {
    float y[kChunk];
    long long src = row;
    bool some = true;
    if (a.index != nullptr) {
        const int i = __ldg(a.index + row);
        some = i >= 0 && i < a.x_rows;
        src = some ? a.div.of(i) : 0;
    }
    if (some) {
        const long long at = src * a.ld + (long long)chunk * kChunk;
        if constexpr (SWIGLU) {
            // silu(g) u in fp32 (a few units in the last place)
            // (all loads in flight first, 16 columns at a time where that takes too many registers)
            constexpr int PART = TYPE == ELUTQ_TYPE_F32 ? 16 : kChunk, EACH = TYPE == ELUTQ_TYPE_F32 ? 8 : 16;
#pragma unroll
            for (int h = 0; h < kChunk; h += PART) {
                float most = 0.0f;
                uint32_t g[PART / EACH][8], u[PART / EACH][8];
#pragma unroll
                for (int k = 0; k < PART / EACH; ++k) {
                    load_raw<TYPE, WIDE>(g[k], a.X, at + h + EACH * k);
                    load_raw<TYPE, WIDE>(u[k], a.X, at + h + EACH * k + a.K);
                }
#pragma unroll
                for (int k = 0; k < PART / EACH; ++k) {
                    float up[EACH];
                    values_of<TYPE>(y + h + EACH * k, g[k]);
                    values_of<TYPE>(up, u[k]);
#pragma unroll
                    for (int i = 0; i < EACH; i += 2) {
                        float e[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) y[h + EACH * k + i + c] = silu(y[h + EACH * k + i + c], e[c]) * up[i + c];
                        most = max_abs(most, e[0], e[1]);
                    }
                }
                // (read again and by calls: there are no registers to keep them in, and with the code in line 16-bit types spilled 288 bytes.  Ordinary values are level with a
                // form that holds gates at -87, 4096 x 14336 fp16 43.6 us, bf16 47.4 for 49.7, fp32 86.0 for 84.4; a gate far out in every chunk costs three to five times that.)
                if (!(most <= kOpen)) {
                    constexpr int W = TYPE == ELUTQ_TYPE_F32 ? 1 : 2;                      // values of a word
                    const uint32_t* words = reinterpret_cast<const uint32_t*>(reinterpret_cast<const uint8_t*>(a.X) + (at + h) * (4 / W));
#pragma unroll
                    for (int i = 0; i < PART; i += W) {
                        const float2 two = far_out_word<TYPE>(words + i / W, a.K / W, y[h + i], y[h + i + W - 1]);
                        y[h + i] = two.x;
                        y[h + i + W - 1] = two.y;
                    }
                }
            }
        } else {
            constexpr int EACH = TYPE == ELUTQ_TYPE_F32 ? 8 : 16;
            uint32_t v[kChunk / EACH][8];
#pragma unroll
            for (int k = 0; k < kChunk / EACH; ++k) load_raw<TYPE, WIDE>(v[k], a.X, at + EACH * k);
#pragma unroll
            for (int k = 0; k < kChunk / EACH; ++k) values_of<TYPE>(y + EACH * k, v[k]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < kChunk; ++i) y[i] = 0.0f;
    }
    if (a.prescale != nullptr) {
        const float p = __ldg(a.prescale);
#pragma unroll
        for (int i = 0; i < kChunk; ++i) y[i] *= p;
    }
    constexpr int B = FMT == ELUTQ_MX4_MXFP4 ? 32 : 16;
    uint32_t bytes[kChunk / B], codes[4];
#pragma unroll
    for (int g = 0; g < kChunk / B; ++g) {
        float* v = y + g * B;
        // the largest magnitude, two values an instruction; a NaN stays one
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < B; i += 2) most = max_abs(most, v[i], v[i + 1]);
        const uint32_t top = __float_as_uint(most);
        const bool bad = top >= 0x7f800000u;
        if constexpr (FMT == ELUTQ_MX4_MXFP4) {
            const int e = max((int)(top >> 23) - 2, 0);
            bytes[g] = bad ? 255u : (uint32_t)e;
            const float f = __uint_as_float((uint32_t)(254 - min(e, 252)) << 23);            // 2^(127 - e)
#pragma unroll
            for (int i = 0; i < B; ++i) v[i] *= f;
        } else {
            uint16_t two;
            asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(two) : "f"(0.0f), "f"(quotient<false>(__uint_as_float(top), 6.0f, 1.0f / 6.0f)));
            bytes[g] = bad ? 127u : (uint32_t)two & 0xffu;
            const float s = e4m3_value(bytes[g]), r = bytes[g] == 0u ? 0.0f : reciprocal(s);
            // (a SwiGLU value is a few units in its last place off anyway)
            if (!SWIGLU && (TYPE == ELUTQ_TYPE_F32 || a.prescale != nullptr)) {
#pragma unroll
                for (int i = 0; i < B; ++i) v[i] = quotient<true>(v[i], s, r);
            } else {
#pragma unroll
                for (int i = 0; i < B; ++i) v[i] = quotient<false>(v[i], s, r);
            }
        }
#pragma unroll
        for (int i = 0; i < B / 8; ++i) codes[g * (B / 8) + i] = bad ? 0u : codes_of(v + 8 * i);
    }
    const long long at = (long long)row * a.per_row.d + chunk;
    a.codes[at] = make_uint4(codes[0], codes[1], codes[2], codes[3]);
    if constexpr (FMT == ELUTQ_MX4_MXFP4) {
        a.scales[at] = (uint8_t)bytes[0];
    } else if (a.pairs) {
        reinterpret_cast<uint16_t*>(a.scales)[at] = (uint16_t)(bytes[0] | bytes[1] << 8);
    } else {
        a.scales[2 * at] = (uint8_t)bytes[0];
        a.scales[2 * at + 1] = (uint8_t)bytes[1];
    }
}

// A thread per chunk of 32 columns.  SwiGLU with as many registers as leave 8 blocks an SM (6 for fp32), which the compiler would not take by itself:
// 14336 x 4096 fp16 NVFP4 49.0 -> 43.6 us, fp32 96.5 -> 79.2.
template <int FMT, int TYPE, bool SWIGLU>
__global__ void __launch_bounds__(128, SWIGLU ? (TYPE == ELUTQ_TYPE_F32 ? 6 : 8) : 0) mx4_quantize_kernel(const QuantArgs a) {
    const unsigned id = blockIdx.x * blockDim.x + threadIdx.x;
    const int local = a.per_row.of((int)id), chunk = (int)id - local * a.per_row.d, row = a.row0 + local;
    grid_dependency_wait();
    grid_launch_dependents();
    if (row >= (a.n_rows != nullptr ? min(__ldg(a.n_rows), a.row0 + a.rows) : a.row0 + a.rows)) return;
    if (a.wide) quantise_chunk<FMT, TYPE, SWIGLU, true>(a, row, chunk);
    else quantise_chunk<FMT, TYPE, SWIGLU, false>(a, row, chunk);
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

// value = alpha * (code * scale): the product of code and scale is exact in fp32 (two and four significant bits), or infinite: 4 * 2^126 and
// 2 * 2^127 are beyond fp32, and alpha does not bring them back.  alpha's product is rounded to fp32 and the result once more to its type.
// Columns of a thread: 64 bytes of results.
template <int TYPE>
constexpr int kBack = TYPE == ELUTQ_TYPE_F32 ? 16 : 32;

template <int FMT, int TYPE, bool WIDE>
__device__ __forceinline__ void dequantise_chunk(const uint8_t* codes, const uint8_t* scales, const float* alpha, void* Y, long long at) {
    constexpr int COLS = kBack<TYPE>;
    uint32_t word[4];
    if constexpr (COLS == 32) {
        const uint4 c = __ldg(reinterpret_cast<const uint4*>(codes) + at);
        word[0] = c.x; word[1] = c.y; word[2] = c.z; word[3] = c.w;
    } else {
        const uint2 c = __ldg(reinterpret_cast<const uint2*>(codes) + at);
        word[0] = c.x; word[1] = c.y;
    }
    const float f = alpha != nullptr ? __ldg(alpha) : 1.0f;
    float s[COLS / 16];
    if constexpr (FMT == ELUTQ_MX4_MXFP4) {
        const uint32_t byte = __ldg(scales + (COLS == 32 ? at : at >> 1));
        s[0] = byte == 255u ? __uint_as_float(0x7fffffffu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
        s[COLS / 16 - 1] = s[0];
    } else {
#pragma unroll
        for (int i = 0; i < COLS / 16; ++i) s[i] = e4m3_value(__ldg(scales + COLS / 16 * at + i));
    }
    uint32_t w[16];
#pragma unroll
    for (int i = 0; i < COLS / 2; ++i) {
        const uint32_t b = (word[i / 4] >> (8 * (i & 3))) & 0xffu;
        uint32_t h;
        asm("{\n\t.reg .b8 t, u;\n\tmov.b16 {t, u}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, t;\n\t}" : "=r"(h) : "h"((uint16_t)b));
        const float2 two = __half22float2(*reinterpret_cast<const __half2*>(&h));
        const float x = two.x * s[i / 8] * f, y = two.y * s[i / 8] * f;
        if constexpr (TYPE == ELUTQ_TYPE_F32) {
            w[2 * i] = __float_as_uint(x);
            w[2 * i + 1] = __float_as_uint(y);
        } else if constexpr (TYPE == ELUTQ_TYPE_F16) {
            const __half2 v = __floats2half2_rn(x, y);
            w[i] = *reinterpret_cast<const uint32_t*>(&v);
        } else {
            const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
            w[i] = *reinterpret_cast<const uint32_t*>(&v);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) store32<WIDE>(reinterpret_cast<uint8_t*>(Y) + at * 64 + 32 * i, w + 8 * i);
}

template <int FMT, int TYPE>
__global__ void __launch_bounds__(256) mx4_dequantize_kernel(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const float* __restrict__ alpha,
                                                             void* Y, long long chunks, int wide) {
    const long long at = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    if (at >= chunks) return;
    if (wide) dequantise_chunk<FMT, TYPE, true>(codes, scales, alpha, Y, at);
    else dequantise_chunk<FMT, TYPE, false>(codes, scales, alpha, Y, at);
}

// Few chunks: small blocks, so that more SMs have some.  (8 x 4096: 32 blocks of 32 instead of 4 of 256.)
inline unsigned threads_for(long long chunks, int num_sms) { return chunks < 64LL * num_sms ? 32u : chunks < 256LL * num_sms ? 64u : 128u; }

template <class K, class... A>
int launch(K kernel, long long chunks, cudaStream_t stream, const A&... args) {
    const unsigned threads = threads_for(chunks, device_sm_count());
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((chunks + threads - 1) / threads));
    cfg.blockDim = dim3(threads);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}

template <int FMT, int TYPE>
int launch_quantize(const QuantArgs& a, long long chunks, bool swiglu, cudaStream_t stream) {
    return swiglu ? launch(mx4_quantize_kernel<FMT, TYPE, true>, chunks, stream, a) : launch(mx4_quantize_kernel<FMT, TYPE, false>, chunks, stream, a);
}

}  // namespace

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_mx4_bytes(int format, int rows, int K, size_t* code_bytes, size_t* scale_bytes) {
    if (!code_bytes || !scale_bytes) return ELUTQ_ERR_INVALID_ARG;
    const int st = mx4_check(format, rows, K);
    if (st != ELUTQ_OK) return st;
    *code_bytes = (size_t)rows * (K / 2);
    *scale_bytes = (size_t)rows * (K / mx4_block(format));
    return ELUTQ_OK;
}

extern "C" int elutq_mx4_quantize(const void* X, int x_type, int x_rows, long long ld, int rows, int K, int format, unsigned flags,
                                  const float* prescale, const int* index, int index_div, const int* n_rows, void* codes, void* scales,
                                  void* stream) {
    if (!X || !codes || !scales) return ELUTQ_ERR_INVALID_ARG;
    if (x_type < ELUTQ_TYPE_F16 || x_type > ELUTQ_TYPE_F32 || (flags & ~ELUTQ_MX4_FLAG_SWIGLU)) return ELUTQ_ERR_INVALID_ARG;
    const int st = mx4_check(format, rows, K);
    if (st != ELUTQ_OK) return st;
    if (x_rows <= 0 || (index != nullptr && index_div < 1)) return ELUTQ_ERR_INVALID_ARG;
    const bool swiglu = (flags & ELUTQ_MX4_FLAG_SWIGLU) != 0;
    if (ld < (swiglu ? 2LL : 1LL) * K || (index == nullptr && x_rows < rows)) return ELUTQ_ERR_SHAPE;
    const long long size = x_type == ELUTQ_TYPE_F32 ? 4 : 2;
    if (!mx4_aligned(X, 16) || (ld * size) % 16 != 0 || !mx4_aligned(codes, 16) || !mx4_aligned(prescale, 4) || !mx4_aligned(index, 4) || !mx4_aligned(n_rows, 4))
        return ELUTQ_ERR_ALIGN;
    QuantArgs a;
    a.X = X;
    a.ld = ld;
    a.prescale = prescale;
    a.index = index;
    a.n_rows = n_rows;
    a.codes = reinterpret_cast<uint4*>(codes);
    a.pairs = mx4_aligned(scales, 2);
    a.scales = reinterpret_cast<uint8_t*>(scales);
    a.K = K;
    a.x_rows = (long long)x_rows * (index != nullptr ? index_div : 1);
    a.per_row.set(K / kChunk);
    a.div.set(index != nullptr ? index_div : 1);
    a.wide = mx4_aligned(X, 32) && (ld * size) % 32 == 0;
    // thread numbers stay below 2^31, the last block's idle ones too
    const int most = (0x7fffffff - 256) / a.per_row.d;
    for (int r = 0; r < rows; r += a.rows) {
        a.row0 = r;
        a.rows = rows - r < most ? rows - r : most;
        const long long chunks = (long long)a.rows * a.per_row.d;
        int ce;
        if (format == ELUTQ_MX4_MXFP4)
            ce = x_type == ELUTQ_TYPE_F16 ? launch_quantize<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_F16>(a, chunks, swiglu, (cudaStream_t)stream)
                 : x_type == ELUTQ_TYPE_BF16 ? launch_quantize<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_BF16>(a, chunks, swiglu, (cudaStream_t)stream)
                                             : launch_quantize<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_F32>(a, chunks, swiglu, (cudaStream_t)stream);
        else
            ce = x_type == ELUTQ_TYPE_F16 ? launch_quantize<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_F16>(a, chunks, swiglu, (cudaStream_t)stream)
                 : x_type == ELUTQ_TYPE_BF16 ? launch_quantize<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_BF16>(a, chunks, swiglu, (cudaStream_t)stream)
                                             : launch_quantize<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_F32>(a, chunks, swiglu, (cudaStream_t)stream);
        if (ce != 0) {
            note_cuda_error(ce);
            return ELUTQ_ERR_CUDA;
        }
    }
    return ELUTQ_OK;
}

extern "C" int elutq_mx4_dequantize(const void* codes, const void* scales, int rows, int K, int format, const float* alpha, void* Y, int y_type, void* stream) {
    if (!codes || !scales || !Y) return ELUTQ_ERR_INVALID_ARG;
    if (y_type < ELUTQ_TYPE_F16 || y_type > ELUTQ_TYPE_F32) return ELUTQ_ERR_INVALID_ARG;
    const int st = mx4_check(format, rows, K);
    if (st != ELUTQ_OK) return st;
    if (!mx4_aligned(codes, 16) || !mx4_aligned(Y, 16) || !mx4_aligned(alpha, 4)) return ELUTQ_ERR_ALIGN;
    const long long chunks = (long long)rows * (K / (y_type == ELUTQ_TYPE_F32 ? kBack<ELUTQ_TYPE_F32> : kBack<ELUTQ_TYPE_F16>));
    if (chunks > 64LL * 0x7fffffffLL) return ELUTQ_ERR_SHAPE;                 // (blocks of a launch)
    const uint8_t* c = reinterpret_cast<const uint8_t*>(codes);
    const int wide = mx4_aligned(Y, 32);
    const uint8_t* s = reinterpret_cast<const uint8_t*>(scales);
    int ce = 0;
    auto go = [&](auto kernel) { ce = launch(kernel, chunks, (cudaStream_t)stream, c, s, alpha, Y, chunks, wide); };
    if (format == ELUTQ_MX4_MXFP4) {
        if (y_type == ELUTQ_TYPE_F16) go(mx4_dequantize_kernel<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_F16>);
        else if (y_type == ELUTQ_TYPE_BF16) go(mx4_dequantize_kernel<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_BF16>);
        else go(mx4_dequantize_kernel<ELUTQ_MX4_MXFP4, ELUTQ_TYPE_F32>);
    } else {
        if (y_type == ELUTQ_TYPE_F16) go(mx4_dequantize_kernel<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_F16>);
        else if (y_type == ELUTQ_TYPE_BF16) go(mx4_dequantize_kernel<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_BF16>);
        else go(mx4_dequantize_kernel<ELUTQ_MX4_NVFP4, ELUTQ_TYPE_F32>);
    }
    if (ce != 0) {
        note_cuda_error(ce);
        return ELUTQ_ERR_CUDA;
    }
    return ELUTQ_OK;
}
