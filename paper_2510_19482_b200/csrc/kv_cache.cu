// Rotary positions and the paged cache: the table of angles, new tokens into the cache, and the cache back to dense rows.
//
//   rotation   pairs (x1, x2) of the first R values of a head, (x_i, x_{i + R/2}) or (x_2i, x_{2i+1}):  y1 = x1 c - x2 s, y2 = x2 c + x1 s, where c and s are
//              the table's entries of the token's position.  Products and sums are rounded to fp32 one by one (no fused multiply-add), so that what a code
//              is chosen from does not hang on how the compiler joins them.
//   16 bits    y rounded once.   E4M3: y * (1 / factor), nearest, 448 at most.   NVFP4: the same product in blocks of 16, as in mx4_quant.cu.
//
// A row (token, head) takes head_dim / 8 lanes, 16 bytes of input each; a pair's other half is in a lane of the same row, a block of 16 in two.  A warp keeps
// the cosines and sines of its token in registers for all of its heads.
//
// Bound: HBM, and for few tokens the latency of one load after another (position, angles, values); in writes of many tokens issue slots beside it.  Measured (us in a graph, and of the copy
// rate): writing 16384 tokens of 64 + 16 heads of 128 in 16 bits 124 (0.85), E4M3 123 (0.81), NVFP4 130 (0.75), with the rotated keys 2 more each; 4700 tokens of 24 + 12 heads of 64 in
// 16 bits 12.7 (0.54), E4M3 13.1 (0.48), NVFP4 15.6 (0.38); 8 tokens 2.4 to 2.8.  Reading 110 thousand tokens of 8 heads of 128 in 16 bits 135 (1.04), E4M3 115 (0.91), NVFP4 107 (0.84).
// The table of angles: 131072 positions of 128 in 66 (0.16), with scaled bands 93 (0.11): a power of two, a sine and a cosine in 64 bits for each pair; it is made once for a model.
#include "kv.cuh"

namespace elutq {

namespace {

struct WriteArgs {
    KvView c;
    const uint8_t *q, *k, *v;
    uint8_t *q_out, *k_out;
    long long ldq, ldk, ldv, ldqo, ldko;       // elements between tokens
    const int *positions, *slots;
    const float* rope;
    int n_pos, rot, interleaved;
    int n_q, heads_all;                        // query heads; all rows of a token: queries, keys, values
    long long warps;
    int turns, batches;                        // warps of a token; batches of rows that a warp handles
};

template <int TYPE>
__device__ __forceinline__ uint32_t to_pair(float lo, float hi) {
    if constexpr (TYPE == ELUTQ_TYPE_F16) {
        const __half2 v = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    } else {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
}
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}

// Eight values of a row into the cache: lane `part` of the row
template <int D, int FMT, int TYPE>
__device__ __forceinline__ void store_row(uint8_t* base, uint8_t* scales, const float* factors, long long row, int head, int part, float (&y)[8], bool on) {
    if constexpr (FMT == ELUTQ_KV_16) {
        if (on) *reinterpret_cast<uint4*>(base + row * (2 * D) + 16 * part) = make_uint4(to_pair<TYPE>(y[0], y[1]), to_pair<TYPE>(y[2], y[3]), to_pair<TYPE>(y[4], y[5]), to_pair<TYPE>(y[6], y[7]));
        return;
    }
    if (factors != nullptr) {
        const float r = __frcp_rn(__ldg(factors + head));
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = __fmul_rn(y[i], r);
    }
    if constexpr (FMT == ELUTQ_KV_E4M3) {
        if (on)
            *reinterpret_cast<uint2*>(base + row * D + 8 * part) = make_uint2(to_e4m3x2(y[0], y[1]) | to_e4m3x2(y[2], y[3]) << 16, to_e4m3x2(y[4], y[5]) | to_e4m3x2(y[6], y[7]) << 16);
    } else {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) most = max_abs(most, y[i], y[i + 1]);
        most = max_abs(most, __shfl_xor_sync(0xffffffffu, most, 1), 0.0f);       // the block's other half
        const bool bad = __float_as_uint(most) >= 0x7f800000u;
        uint32_t byte = to_e4m3x2(__fdiv_rn(most, 6.0f), 0.0f) & 0xffu;
        if (bad) byte = 127u;
        const float s = e4m3_value(byte), r = byte == 0u ? 0.0f : reciprocal(s);
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = quotient<true>(y[i], s, r);
        if (on) {
            *reinterpret_cast<uint32_t*>(base + row * (D / 2) + 4 * part) = bad ? 0u : codes_of(y);
            if ((part & 1) == 0) scales[row * (D / 16) + part / 2] = (uint8_t)byte;
        }
    }
}

// U: rows of a batch that a lane handles, their loads in flight together
template <int D, int FMT, int TYPE, int U>
__global__ void __launch_bounds__(128, 8) kv_write_kernel(const WriteArgs a) {
    constexpr int LANES = D / 8, ROWS = 32 / LANES;        // of a row; rows of a warp at a time
    const long long w = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
    grid_dependency_wait();
    grid_launch_dependents();
    if (w >= a.warps) return;
    const int lane = threadIdx.x & 31, part = lane % LANES, d0 = 8 * part;
    const long long token = w / a.turns;
    int first = (int)(w - token * a.turns) * a.batches * (ROWS * U) + lane / LANES;
    const int slot = __ldg(a.slots + token);
    const uint8_t *q = a.q + 2 * token * a.ldq, *k = a.k + 2 * token * a.ldk, *v = a.v + 2 * token * a.ldv;
    uint4 x[U];
    auto load = [&] {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = first + u * ROWS, kv = r - a.n_q;
            const uint8_t* src = kv < 0 ? q + r * (2 * D) : kv < a.c.heads ? k + kv * (2 * D) : v + (kv - a.c.heads) * (2 * D);
            x[u] = make_uint4(0u, 0u, 0u, 0u);
            if (r < a.heads_all) x[u] = *(reinterpret_cast<const uint4*>(src) + part);
        }
    };
    load();
    float c[8], s[8];
    const int half = a.rot / 2;
    const bool turned = d0 < a.rot;
    int other = lane;                                       // the lane with the pairs' other values
    if (a.rope != nullptr) {
        const int pos = __ldg(a.positions + token);
        if (pos < 0 || pos >= a.n_pos) return;              // (the same for the whole warp)
        const float* t = a.rope + (long long)pos * a.rot;
        if (turned && a.interleaved) {
            const float4 cc = __ldg(reinterpret_cast<const float4*>(t + d0 / 2)), ss = __ldg(reinterpret_cast<const float4*>(t + half + d0 / 2));
            c[0] = cc.x; c[1] = cc.y; c[2] = cc.z; c[3] = cc.w;
            s[0] = ss.x; s[1] = ss.y; s[2] = ss.z; s[3] = ss.w;
        } else if (turned) {
            const int at = d0 < half ? d0 : d0 - half;
            other = d0 < half ? lane + half / 8 : lane - half / 8;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 cc = __ldg(reinterpret_cast<const float4*>(t + at) + i), ss = __ldg(reinterpret_cast<const float4*>(t + half + at) + i);
                c[4 * i] = cc.x; c[4 * i + 1] = cc.y; c[4 * i + 2] = cc.z; c[4 * i + 3] = cc.w;
                s[4 * i] = ss.x; s[4 * i + 1] = ss.y; s[4 * i + 2] = ss.z; s[4 * i + 3] = ss.w;
            }
            if (d0 < half) {
#pragma unroll
                for (int i = 0; i < 8; ++i) s[i] = -s[i];
            }
        }
    }
    const bool held = slot >= 0 && slot < a.c.n_pages * a.c.page_size;
    const int page = held ? a.c.page.of(slot) : 0;
    const long long row0 = (long long)page * a.c.heads * a.c.page_size + (held ? slot - page * a.c.page_size : 0);
    for (int batch = 0;; ++batch) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = first + u * ROWS;
            if (U > 1 && __all_sync(0xffffffffu, r >= a.heads_all)) break;
            const int kv = r - a.n_q;
            const bool is_v = kv >= a.c.heads;
            float y[8];
            word_values<TYPE>(y, x[u].x);
            word_values<TYPE>(y + 2, x[u].y);
            word_values<TYPE>(y + 4, x[u].z);
            word_values<TYPE>(y + 6, x[u].w);
            if (a.rope != nullptr) {
                if (a.interleaved) {
                    if (turned && !is_v) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float y1 = __fsub_rn(__fmul_rn(y[2 * i], c[i]), __fmul_rn(y[2 * i + 1], s[i]));
                            y[2 * i + 1] = __fadd_rn(__fmul_rn(y[2 * i + 1], c[i]), __fmul_rn(y[2 * i], s[i]));
                            y[2 * i] = y1;
                        }
                    }
                } else {
                    float z[8];
                    word_values<TYPE>(z, __shfl_sync(0xffffffffu, x[u].x, other));
                    word_values<TYPE>(z + 2, __shfl_sync(0xffffffffu, x[u].y, other));
                    word_values<TYPE>(z + 4, __shfl_sync(0xffffffffu, x[u].z, other));
                    word_values<TYPE>(z + 6, __shfl_sync(0xffffffffu, x[u].w, other));
                    if (turned && !is_v) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) y[i] = __fadd_rn(__fmul_rn(y[i], c[i]), __fmul_rn(z[i], s[i]));
                    }
                }
            }
            const bool there = r < a.heads_all;
            if (there && !is_v) {
                uint8_t* out = kv < 0 ? a.q_out + 2 * (token * a.ldqo + (long long)r * D) : a.k_out == nullptr ? nullptr : a.k_out + 2 * (token * a.ldko + (long long)kv * D);
                if (out != nullptr)
                    reinterpret_cast<uint4*>(out)[part] = make_uint4(to_pair<TYPE>(y[0], y[1]), to_pair<TYPE>(y[2], y[3]), to_pair<TYPE>(y[4], y[5]), to_pair<TYPE>(y[6], y[7]));
            }
            if (__any_sync(0xffffffffu, there && kv >= 0)) {
                const int h = is_v ? kv - a.c.heads : kv < 0 ? 0 : kv;
                store_row<D, FMT, TYPE>(is_v ? a.c.v : a.c.k, is_v ? a.c.vs : a.c.ks, is_v ? a.c.vf : a.c.kf, row0 + (long long)h * a.c.page_size, there ? h : 0, part, y, there && kv >= 0 && held);
            }
        }
        first += U * ROWS;
        if (batch + 1 >= a.batches || first - lane / LANES >= a.heads_all) break;
        load();
    }
}

struct ReadArgs {
    KvView c;
    const int *table, *first, *cu;
    long long ld_table;
    int wide;                  // pages of a sequence in the table
    int B, rows;
    uint8_t *k_out, *v_out;
    long long ldk, ldv;
    long long work;            // threads
};

// 16 stored values as 16-bit results.  code * scale is exact in fp32 (6 significant bits), its product with the factor is rounded to fp32, and once more to the type.
template <int FMT, int TYPE>
struct Stored {
    uint4 w[FMT == ELUTQ_KV_16 ? 2 : 1];
    uint32_t scale;
    __device__ __forceinline__ void load(const uint8_t* base, const uint8_t* scales, long long row, int part, int D) {
        if constexpr (FMT == ELUTQ_KV_16) {
            w[0] = __ldg(reinterpret_cast<const uint4*>(base + row * (2 * D) + 32 * part));
            w[1] = __ldg(reinterpret_cast<const uint4*>(base + row * (2 * D) + 32 * part) + 1);
        } else if constexpr (FMT == ELUTQ_KV_E4M3) {
            w[0] = __ldg(reinterpret_cast<const uint4*>(base + row * D + 16 * part));
        } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(base + row * (D / 2) + 8 * part));
            w[0].x = v.x;
            w[0].y = v.y;
            scale = __ldg(scales + row * (D / 16) + part);
        }
    }
    __device__ __forceinline__ void store(uint8_t* out, int part, float f) const {
        uint32_t o[8];
        if constexpr (FMT == ELUTQ_KV_16) {
            o[0] = w[0].x; o[1] = w[0].y; o[2] = w[0].z; o[3] = w[0].w;
            o[4] = w[1].x; o[5] = w[1].y; o[6] = w[1].z; o[7] = w[1].w;
        } else {
            float s = 1.0f;
            if constexpr (FMT == ELUTQ_KV_NVFP4) s = e4m3_value(scale);
            const uint32_t words[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t h;
                if constexpr (FMT == ELUTQ_KV_E4M3) asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)(words[i / 2] >> (16 * (i & 1)))));
                else asm("{\n\t.reg .b8 b;\n\tcvt.u8.u32 b, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(h) : "r"(words[i / 4] >> (8 * (i & 3))));
                const float2 v = __half22float2(*reinterpret_cast<const __half2*>(&h));
                o[i] = to_pair<TYPE>(v.x * s * f, v.y * s * f);
            }
        }
        reinterpret_cast<uint4*>(out)[2 * part] = make_uint4(o[0], o[1], o[2], o[3]);
        reinterpret_cast<uint4*>(out)[2 * part + 1] = make_uint4(o[4], o[5], o[6], o[7]);
    }
};

constexpr int kReadTokens = 32;                // consecutive rows of one head for a block's neighbouring threads

template <int D, int FMT, int TYPE>
__global__ void __launch_bounds__(128) kv_read_kernel(const ReadArgs a) {
    constexpr int PARTS = D / 16;
    const long long id = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    if (id >= a.work) return;
    const int part = (int)(id % PARTS), in_tile = (int)(id / PARTS % kReadTokens);
    const long long tile = id / (PARTS * kReadTokens);
    const int head = (int)(tile % a.c.heads);
    const long long row_ = tile / a.c.heads * kReadTokens + in_tile;
    if (row_ >= a.rows) return;
    const int row = (int)row_;
    // the sequence: the last one that begins at or in front of the row
    int lo = 0, hi = a.B;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (__ldg(a.cu + mid) <= row) lo = mid;
        else hi = mid;
    }
    const int begin = __ldg(a.cu + lo);
    if (row < begin || row >= __ldg(a.cu + lo + 1)) return;
    const long long pos = (long long)(a.first == nullptr ? 0 : __ldg(a.first + lo)) + (row - (long long)begin);
    uint8_t* ko = a.k_out + 2 * (row * a.ldk + (long long)head * D);
    uint8_t* vo = a.v_out + 2 * (row * a.ldv + (long long)head * D);
    int page = -1, at = 0;
    if (pos >= 0 && pos <= 0x7fffffffLL) {
        const int n = a.c.page.of((int)pos);
        at = (int)pos - n * a.c.page_size;
        if (n < a.wide) page = __ldg(a.table + lo * a.ld_table + n);
    }
    if (page < 0 || page >= a.c.n_pages) {
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        reinterpret_cast<uint4*>(ko)[2 * part] = reinterpret_cast<uint4*>(ko)[2 * part + 1] = zero;
        reinterpret_cast<uint4*>(vo)[2 * part] = reinterpret_cast<uint4*>(vo)[2 * part + 1] = zero;
        return;
    }
    const long long src = ((long long)page * a.c.heads + head) * a.c.page_size + at;
    Stored<FMT, TYPE> k, v;
    k.load(a.c.k, a.c.ks, src, part, D);
    v.load(a.c.v, a.c.vs, src, part, D);
    k.store(ko, part, a.c.kf == nullptr ? 1.0f : __ldg(a.c.kf + head));
    v.store(vo, part, a.c.vf == nullptr ? 1.0f : __ldg(a.c.vf + head));
}

struct TableArgs {
    float* table;
    long long pairs;
    int half, scaling;
    double theta_log2, factor, low, high, original, magnitude;
    int rot;
};

// A thread per (position, pair): cos and sin of position * frequency, in 64 bits
__global__ void __launch_bounds__(256) rope_table_kernel(const TableArgs a) {
    const long long id = (long long)blockIdx.x * blockDim.x + threadIdx.x;
    grid_dependency_wait();
    grid_launch_dependents();
    if (id >= a.pairs) return;
    const long long pos = id / a.half;
    const int i = (int)(id - pos * a.half);
    double f = exp2(-2.0 * i / a.rot * a.theta_log2);
    if (a.scaling == ELUTQ_ROPE_LINEAR) {
        f /= a.factor;
    } else if (a.scaling == ELUTQ_ROPE_BANDS) {
        const double turns = a.original * f / 6.283185307179586476925286766559;      // over the original length
        double keep = (turns - a.low) / (a.high - a.low);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        f *= keep + (1.0 - keep) / a.factor;
    }
    double s, c;
    sincos((double)pos * f, &s, &c);
    float* row = a.table + pos * a.rot;
    row[i] = (float)(c * a.magnitude);
    row[a.half + i] = (float)(s * a.magnitude);
}

template <class K, class A>
int launch(K kernel, long long threads, int block, cudaStream_t stream, const A& args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((threads + block - 1) / block));
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}
int finish(int ce) {
    if (ce == 0) return ELUTQ_OK;
    note_cuda_error(ce);
    return ELUTQ_ERR_CUDA;
}

constexpr int kUnroll = 4;

template <int D, int FMT, int TYPE>
int launch_write(WriteArgs& a, long long tokens, cudaStream_t stream) {
    constexpr int ROWS = 32 / (D / 8);
    // few tokens: a row to a lane, so that the rows' latencies run side by side; otherwise the angles are loaded once for several
    const bool few = tokens * a.heads_all / ROWS < 16LL * device_sm_count();
    const int rows = ROWS * (few ? 1 : kUnroll), batches = (a.heads_all + rows - 1) / rows;
    // ... for all of a token where there are tokens enough
    a.turns = few ? batches : 1;
    while (a.turns < batches && tokens * a.turns < 300LL * device_sm_count()) ++a.turns;
    a.batches = (batches + a.turns - 1) / a.turns;
    a.warps = tokens * a.turns;
    return few ? launch(kv_write_kernel<D, FMT, TYPE, 1>, a.warps * 32, 128, stream, a) : launch(kv_write_kernel<D, FMT, TYPE, kUnroll>, a.warps * 32, 128, stream, a);
}
template <int D, int FMT>
int launch_write(WriteArgs& a, int type, long long tokens, cudaStream_t stream) {
    return type == ELUTQ_TYPE_F16 ? launch_write<D, FMT, ELUTQ_TYPE_F16>(a, tokens, stream) : launch_write<D, FMT, ELUTQ_TYPE_BF16>(a, tokens, stream);
}
template <int D>
int launch_write(WriteArgs& a, int format, int type, long long tokens, cudaStream_t stream) {
    return format == ELUTQ_KV_16 ? launch_write<D, ELUTQ_KV_16>(a, type, tokens, stream)
           : format == ELUTQ_KV_E4M3 ? launch_write<D, ELUTQ_KV_E4M3>(a, type, tokens, stream) : launch_write<D, ELUTQ_KV_NVFP4>(a, type, tokens, stream);
}
template <int D, int FMT>
int launch_read(const ReadArgs& a, int type, cudaStream_t stream) {
    return type == ELUTQ_TYPE_F16 ? launch(kv_read_kernel<D, FMT, ELUTQ_TYPE_F16>, a.work, 128, stream, a) : launch(kv_read_kernel<D, FMT, ELUTQ_TYPE_BF16>, a.work, 128, stream, a);
}
template <int D>
int launch_read(const ReadArgs& a, int format, int type, cudaStream_t stream) {
    return format == ELUTQ_KV_16 ? launch_read<D, ELUTQ_KV_16>(a, type, stream) : format == ELUTQ_KV_E4M3 ? launch_read<D, ELUTQ_KV_E4M3>(a, type, stream) : launch_read<D, ELUTQ_KV_NVFP4>(a, type, stream);
}

}  // namespace

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_rope_table(float* table, int n_pos, int rot_dim, double theta, int scaling, double factor, double low, double high, double original, double magnitude,
                                void* stream) {
    if (!table || n_pos <= 0 || rot_dim <= 0 || scaling < ELUTQ_ROPE_PLAIN || scaling > ELUTQ_ROPE_BANDS) return ELUTQ_ERR_INVALID_ARG;
    if (!(theta > 1.0) || !(theta < 1e300) || !(magnitude > 0.0) || !(magnitude < 1e30)) return ELUTQ_ERR_INVALID_ARG;
    if (scaling != ELUTQ_ROPE_PLAIN && (!(factor >= 1.0) || !(factor < 1e30))) return ELUTQ_ERR_INVALID_ARG;
    if (scaling == ELUTQ_ROPE_BANDS && (!(low >= 0.0) || !(high > low) || !(high < 1e30) || !(original >= 1.0) || !(original < 1e30))) return ELUTQ_ERR_INVALID_ARG;
    if (rot_dim % 16 != 0) return ELUTQ_ERR_SHAPE;
    if (!mx4_aligned(table, 16)) return ELUTQ_ERR_ALIGN;
    TableArgs a;
    a.table = table;
    a.half = rot_dim / 2;
    a.rot = rot_dim;
    a.pairs = (long long)n_pos * a.half;
    if (a.pairs > 256LL * 0x7fffffffLL) return ELUTQ_ERR_SHAPE;               // (blocks of a launch)
    a.scaling = scaling;
    a.theta_log2 = log2(theta);
    a.factor = factor; a.low = low; a.high = high; a.original = original; a.magnitude = magnitude;
    return finish(launch(rope_table_kernel, a.pairs, 256, (cudaStream_t)stream, a));
}

extern "C" int elutq_kv_bytes(int format, int n_pages, int heads, int page_size, int head_dim, size_t* data_bytes, size_t* scale_bytes) {
    if (!data_bytes || !scale_bytes || n_pages <= 0 || heads <= 0 || page_size <= 0 || format < ELUTQ_KV_16 || format > ELUTQ_KV_NVFP4) return ELUTQ_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return ELUTQ_ERR_UNSUPPORTED;
    if (page_size % 16 != 0 || (long long)n_pages * page_size > 0x7fffffffLL) return ELUTQ_ERR_SHAPE;
    const size_t rows = (size_t)n_pages * page_size * heads;
    *data_bytes = rows * kv_row_bytes(format, head_dim);
    *scale_bytes = format == ELUTQ_KV_NVFP4 ? rows * (head_dim / 16) : 0;
    return ELUTQ_OK;
}

extern "C" int elutq_kv_write(const elutq_kv_cache* cache, const void* q, long long ldq, void* q_out, long long ldqo, int n_q_heads, const void* k, long long ldk, void* k_out,
                              long long ldko, const void* v, long long ldv, int tokens, const int* slots, const int* positions, const float* rope, int n_pos, int rot_dim,
                              unsigned flags, void* stream) {
    int st = kv_check(cache);
    if (st != ELUTQ_OK) return st;
    if (!k || !v || !slots || tokens <= 0 || n_q_heads < 0 || (flags & ~ELUTQ_ROPE_INTERLEAVED)) return ELUTQ_ERR_INVALID_ARG;
    if (n_q_heads > 0 && (!q || !q_out)) return ELUTQ_ERR_INVALID_ARG;
    if (rope != nullptr && (!positions || n_pos <= 0 || rot_dim <= 0)) return ELUTQ_ERR_INVALID_ARG;
    const int D = cache->head_dim, H = cache->heads;
    if (rope != nullptr && (rot_dim > D || rot_dim % 16 != 0)) return ELUTQ_ERR_SHAPE;
    if (n_q_heads > 0 && ((st = kv_rows_check(q, ldq, n_q_heads, D)) != ELUTQ_OK || (st = kv_rows_check(q_out, ldqo, n_q_heads, D)) != ELUTQ_OK)) return st;
    if ((st = kv_rows_check(k, ldk, H, D)) != ELUTQ_OK || (st = kv_rows_check(v, ldv, H, D)) != ELUTQ_OK) return st;
    if (k_out != nullptr && (st = kv_rows_check(k_out, ldko, H, D)) != ELUTQ_OK) return st;
    if (!mx4_aligned(slots, 4) || !mx4_aligned(positions, 4) || !mx4_aligned(rope, 16)) return ELUTQ_ERR_ALIGN;
    if ((long long)n_q_heads + 2LL * H > (1 << 22) || (long long)tokens * (n_q_heads + 2LL * H) > (1LL << 34)) return ELUTQ_ERR_SHAPE;        // (blocks of a launch)
    // in place or apart: a warp reads the rows of its token only just before it writes them
    const Rows kr = {k, ldk, tokens, H}, vr = {v, ldv, tokens, H}, qr = {q, ldq, tokens, n_q_heads}, qo = {q_out, ldqo, tokens, n_q_heads}, ko = {k_out, ldko, tokens, H};
    if (n_q_heads > 0 && (rows_meet_apart(qo, qr, D) || rows_meet(qo, kr, D) || rows_meet(qo, vr, D))) return ELUTQ_ERR_INVALID_ARG;
    if (k_out != nullptr && (rows_meet_apart(ko, kr, D) || rows_meet(ko, vr, D) || (n_q_heads > 0 && (rows_meet(ko, qr, D) || rows_meet(ko, qo, D))))) return ELUTQ_ERR_INVALID_ARG;
    WriteArgs a;
    a.c = kv_view(cache);
    a.q = (const uint8_t*)q; a.k = (const uint8_t*)k; a.v = (const uint8_t*)v;
    a.q_out = (uint8_t*)q_out; a.k_out = (uint8_t*)k_out;
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldqo = ldqo; a.ldko = ldko;
    a.positions = positions; a.slots = slots; a.rope = rope;
    a.n_pos = n_pos;
    a.rot = rope != nullptr ? rot_dim : 0;
    a.interleaved = (flags & ELUTQ_ROPE_INTERLEAVED) != 0;
    a.n_q = n_q_heads;
    a.heads_all = n_q_heads + 2 * H;
    return finish(D == 128 ? launch_write<128>(a, cache->format, cache->type, tokens, (cudaStream_t)stream) : launch_write<64>(a, cache->format, cache->type, tokens, (cudaStream_t)stream));
}

extern "C" int elutq_kv_read(const elutq_kv_cache* cache, const int* table, long long ld_table, int pages, const int* first, const int* cu, int B, int rows, void* k_out,
                             long long ldk, void* v_out, long long ldv, void* stream) {
    int st = kv_check(cache);
    if (st != ELUTQ_OK) return st;
    if (!table || !cu || !k_out || !v_out || pages <= 0 || B <= 0 || rows <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (ld_table < pages) return ELUTQ_ERR_SHAPE;
    const int D = cache->head_dim, H = cache->heads;
    if ((st = kv_rows_check(k_out, ldk, H, D)) != ELUTQ_OK || (st = kv_rows_check(v_out, ldv, H, D)) != ELUTQ_OK) return st;
    if (!mx4_aligned(table, 4) || !mx4_aligned(first, 4) || !mx4_aligned(cu, 4)) return ELUTQ_ERR_ALIGN;
    if (rows_meet({k_out, ldk, rows, H}, {v_out, ldv, rows, H}, D)) return ELUTQ_ERR_INVALID_ARG;
    ReadArgs a;
    a.c = kv_view(cache);
    a.table = table; a.first = first; a.cu = cu;
    a.ld_table = ld_table;
    a.wide = pages;
    a.B = B;
    a.rows = rows;
    a.k_out = (uint8_t*)k_out; a.v_out = (uint8_t*)v_out;
    a.ldk = ldk; a.ldv = ldv;
    a.work = ((long long)rows + kReadTokens - 1) / kReadTokens * H * kReadTokens * (D / 16);
    if (a.work > 128LL * 0x7fffffffLL) return ELUTQ_ERR_SHAPE;                // (blocks of a launch)
    return finish(D == 128 ? launch_read<128>(a, cache->format, cache->type, (cudaStream_t)stream) : launch_read<64>(a, cache->format, cache->type, (cudaStream_t)stream));
}
