// Attention of the newest token(s) of every sequence over a paged cache in 16 bits, E4M3 or NVFP4, which is read once and never written out in 16 bits.
//
//   o = sum_j 2^(x_j - m) V_j / sum_j 2^(x_j - m),   x_j = log2(e) scale q . K_j,   j up to the query's own position
//
// work       Query rows of one key head (the heads that share it, times the new tokens) are the N of both products, 8 or 16 at a time, the cache's tokens the
//            M of the first and head dimensions the M of the second: with 4 or 8 heads to a key head no row of the tensor core's tiles is left empty.
//              S^T [tokens x rows] = K Q^T,   O^T [dims x rows] += V^T P^T
//            The order of an inner index is free, so a lane takes whole 16-byte pieces of K rows and of V rows from global memory straight into the
//            registers of the fragments: no shared memory, no transposition but that of P (movmatrix) and of pairs of V rows (byte permutes).
// split      All (sequence, key head, rows) segments laid behind one another, in tiles, are cut into equal shares, one for each CTA that the GPU holds: lengths may
//            be as ragged as they like.  The warps of a CTA take the tiles of a segment in turn and join through shared memory; a segment that lies within one share
//            is finished there, the parts of others go to the workspace and a second kernel joins them in their order.
// softmax    One running maximum for all lanes of a column, moved only when a tile rises more than 2^10 above it (then everything is scaled): P stays below
//            2^14, in 16 bits whatever the type.  Maximum, sum and result are fp32.
// codes      E4M3 and E2M1 values, also times an E4M3 block scale, are exact in fp16, so both products are fp16 ones, with q brought to fp16 by a power of two for each row.
//            The heads' factors are multiplied into the scale and into the result.
//
// Masked places never reach the result, whatever they hold: scores are selected, V rows behind the sequence are replaced by zeros, and in the last tiles, where
// the new tokens of a sequence see different lengths, every token's product is formed by itself.
//
// Bound: HBM (the cache), for few tokens the latency of table, keys, joining.
#include "kv.cuh"

namespace elutq {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr float kNone = 1e30f;               // offset of a column that has seen no token: any score rises above it
constexpr float kBase = 4.0f, kRise = 14.0f; // 2^(x - m + 4), m moved when that would pass 2^14

struct DecodeArgs {
    KvView c;
    const uint8_t* q;
    uint8_t* out;
    long long ldq, ldo;        // elements between tokens
    const int *table, *lens;
    long long ld_table;
    int wide;                  // pages of a sequence in the table
    int B, fresh, group;       // sequences, new tokens of each, query heads of a key head
    int rows, row_tiles;       // query rows of a key head; tiles of them
    int type;
    float scale;               // times log2(e)
    float* parts;
    long long cap;             // wide * page_size: tokens that the table has room for
};

__host__ __device__ constexpr int tile_tokens(int format, int D) {
    const int row = format == ELUTQ_KV_16 ? 2 * D : format == ELUTQ_KV_E4M3 ? D : D / 2;
    return 4096 / row > 64 ? 64 : 4096 / row;
}

__device__ __forceinline__ int length_of(const DecodeArgs& a, int b) {
    const long long n = __ldg(a.lens + b);
    return (int)(n < 0 ? 0 : n > a.cap ? a.cap : n);
}

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t d;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
    const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t bytes) {           // of the low 16 bits, as fp16
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)bytes));
    return h;
}
__device__ __forceinline__ uint32_t e2m1_pair(uint32_t byte) {            // of the low 8 bits, as fp16
    uint32_t h;
    asm("{\n\t.reg .b8 b, x, y, z;\n\tmov.b32 {b, x, y, z}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(h) : "r"(byte));
    return h;
}
template <int BYTES>
__device__ __forceinline__ void load_stream(uint32_t* w, const uint8_t* p) {
    if constexpr (BYTES == 16) asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    else if constexpr (BYTES == 8) asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
    else asm volatile("ld.global.nc.L1::no_allocate.u32 %0, [%1];" : "=r"(w[0]) : "l"(p));
}

// Where a share begins: its first segment's sequence and the units in front of that sequence.
struct Place {
    long long before, total;
    int b;
};
template <int TT>
__device__ __forceinline__ int tiles_of(int len) { return (len + TT - 1) / TT; }

// Units (tiles of segments) in front of sequence `upto` and of all sequences, by the whole block.
template <int TT>
__device__ __forceinline__ void count_units(const DecodeArgs& a, int upto, long long& before, long long& total, long long* scratch) {
    long long mine = 0, front = 0;
    const int each = a.c.heads * a.row_tiles;
    for (int b = threadIdx.x; b < a.B; b += blockDim.x) {
        const long long n = (long long)tiles_of<TT>(length_of(a, b)) * each;
        mine += n;
        if (b < upto) front += n;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        mine += __shfl_xor_sync(0xffffffffu, mine, o);
        front += __shfl_xor_sync(0xffffffffu, front, o);
    }
    const int warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    if ((threadIdx.x & 31) == 0) { scratch[2 * warp] = mine; scratch[2 * warp + 1] = front; }
    __syncthreads();
    total = before = 0;
    for (int w = 0; w < warps; ++w) { total += scratch[2 * w]; before += scratch[2 * w + 1]; }
    __syncthreads();
}
// Units of a share: all CTAs take the same, at least one tile for each warp.
__device__ __forceinline__ long long share_of(long long total, int ctas) {
    const long long n = (total + ctas - 1) / ctas;
    return n < kWarps ? kWarps : n;
}

template <int D, int FMT, bool BF16, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? 3 : 2) attn_decode_kernel(const DecodeArgs a) {
    constexpr int TT = tile_tokens(FMT, D), SUB = TT / 16, NC = 8 * NT;
    constexpr int ROW = FMT == ELUTQ_KV_16 ? 2 * D : FMT == ELUTQ_KV_E4M3 ? D : D / 2;
    constexpr int PER_WORD = FMT == ELUTQ_KV_16 ? 2 : FMT == ELUTQ_KV_E4M3 ? 4 : 8;      // values of a word
    constexpr int KW = ROW / 16, KC = KW < 4 ? KW : 4;       // words of a K row in a lane; of a piece
    constexpr int VW = ROW / 32, VC = VW < 4 ? VW : 4;
    constexpr int STEPS = D / 16;                            // of 16 head dimensions; also 16-dimension tiles of the result
    constexpr bool SCALED = FMT == ELUTQ_KV_NVFP4;
    constexpr int PAD = D + 4;
    __shared__ __align__(16) float s_o[kWarps][NC][PAD];
    __shared__ float s_off[kWarps][NC], s_sum[kWarps][NC];
    __shared__ long long s_scan[2 * kWarps];
    __shared__ long long s_before;
    __shared__ int s_b;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    grid_dependency_wait();
    grid_launch_dependents();

    // ---- this CTA's share -----------------------------------------------------------------------------------------------------------------------
    const int each = a.c.heads * a.row_tiles;
    long long share, f0, f1;
    {
        // (a run of sequences to a thread; the thread whose run holds the first unit walks it)
        const int run = (a.B + kThreads - 1) / kThreads, b0 = min(a.B, tid * run), b1 = min(a.B, b0 + run);
        long long mine = 0;
        for (int b = b0; b < b1; ++b) mine += (long long)tiles_of<TT>(length_of(a, b)) * each;
        long long incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const long long v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) s_scan[warp] = incl;
        __syncthreads();
        long long front = incl - mine, total = 0;
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) front += s_scan[w];
            total += s_scan[w];
        }
        share = share_of(total, gridDim.x);
        f0 = blockIdx.x * share;
        f1 = f0 + share < total ? f0 + share : total;
        if (f0 >= f1) return;                                 // (the whole CTA)
        if (f0 >= front && f0 < front + mine) {
            int b = b0;
            for (; b < b1; ++b) {
                const long long n = (long long)tiles_of<TT>(length_of(a, b)) * each;
                if (f0 < front + n) break;
                front += n;
            }
            s_before = front;
            s_b = b;
        }
        __syncthreads();
    }
    int b = s_b;
    long long before = s_before;

    for (long long f = f0; f < f1;) {
        const int len = length_of(a, b), tiles = tiles_of<TT>(len);
        if (tiles == 0) { ++b; continue; }
        const long long local = f - before;
        const int seg = (int)(local / tiles), tile0 = (int)(local - (long long)seg * tiles);
        const int h = seg / a.row_tiles, rt = seg - h * a.row_tiles;
        const int count = (int)(f1 - f < tiles - tile0 ? f1 - f : tiles - tile0);
        const int* pages = a.table + b * a.ld_table;
        const int least = len - a.fresh + 1;                  // tokens that the first of the new tokens sees
        const int mine = warp < count ? (count - warp + kWarps - 1) / kWarps : 0;        // this warp's tiles: tile0 + warp + n kWarps

        // ---- loads -----------------------------------------------------------------------------------------------------------------------------
        uint32_t kr[SUB][2][KW], vr[SUB][4][VW];
        uint32_t ksc[SUB][2], vsc[SUB];
        uint32_t there = 0;                                   // sub-tiles of the K in hand whose page exists
        int ids = -1;                                         // lane i: page of the i-th of 32 16-token pieces of this warp's tiles
        auto fetch_ids = [&](int n) {                         // for tiles n, n + 1, .. of this warp
            const int tile = tile0 + warp + (n + lane / SUB) * kWarps;
            const int tok = tile * TT + (lane % SUB) * 16;
            ids = -1;
            if (n + lane / SUB < mine && tok < len) ids = __ldg(pages + a.c.page.of(tok));
            if (ids >= a.c.n_pages) ids = -1;
        };
        auto row_of = [&](int n, int s) {                     // first row of a piece (whatever page: see `there`)
            const int tok = (tile0 + warp + n * kWarps) * TT + 16 * s;
            const int page = max(0, __shfl_sync(0xffffffffu, ids, (n * SUB + s) & 31));
            return ((long long)page * a.c.heads + h) * a.c.page_size + (tok - a.c.page.of(tok) * a.c.page_size);
        };
        auto load_k = [&](int n) {
            if (((n * SUB) & 31) == 0) fetch_ids(n);
            there = 0;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const long long row = row_of(n, s);
                const bool ok = __shfl_sync(0xffffffffu, ids, (n * SUB + s) & 31) >= 0;
                there |= (uint32_t)ok << s;
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const uint8_t* p = a.c.k + (row + g + 8 * r) * ROW + t * (4 * KC);
#pragma unroll
                    for (int i = 0; i < KW / KC; ++i) load_stream<4 * KC>(&kr[s][r][i * KC], p + i * (16 * KC));
                    if constexpr (SCALED) {
                        const uint8_t* q = a.c.ks + (row + g + 8 * r) * (D / 16);
                        ksc[s][r] = D == 128 ? (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(q) + t) : (uint32_t)__ldg(q + t);
                    }
                }
            }
        };
        auto load_v = [&](int n) {                            // (behind load_k of the same tile)
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                const long long row = row_of(n, s);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int tok = 2 * t + (r & 1) + 8 * (r >> 1);
                    const uint8_t* p = a.c.v + (row + tok) * ROW + g * (4 * VC);
#pragma unroll
                    for (int i = 0; i < VW / VC; ++i) load_stream<4 * VC>(&vr[s][r][i * VC], p + i * (32 * VC));
                }
                if constexpr (SCALED) {
                    uint32_t v = 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int tok = 2 * t + (r & 1) + 8 * (r >> 1);
                        v |= (uint32_t)__ldg(a.c.vs + (row + tok) * (D / 16) + (D == 128 ? g : g / 2)) << (8 * r);
                    }
                    vsc[s] = v;
                }
            }
        };
        if (mine > 0) {
            load_k(0);
            load_v(0);
        }

        // ---- query rows as fragments: column g of each eight; the columns of this lane's scores are 2 t and 2 t + 1 -------------------------------
        uint32_t qf[NT][STEPS][2];
        float cs[NT][2], off[NT][2], sum[NT][2];
        int limit[NT][2];
        const float kf = a.c.kf == nullptr ? 1.0f : __ldg(a.c.kf + h);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int r = rt * NC + nt * 8 + g;
            const int tok = r / a.group, head = h * a.group + (r - tok * a.group);
            const uint8_t* p = a.q + 2 * (((long long)b * a.fresh + tok) * a.ldq + (long long)head * D);
            constexpr int PIECE = KC * PER_WORD;              // head dimensions of a piece of K
#pragma unroll
            for (int i = 0; i < KW / KC; ++i)
#pragma unroll
                for (int j = 0; j < PIECE / 8; ++j) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if (r < a.rows) v = __ldg(reinterpret_cast<const uint4*>(p + 2 * (PIECE * (t + 4 * i) + 8 * j)));
                    const int step = (i * PIECE + 8 * j) / 4;
                    qf[nt][step][0] = v.x; qf[nt][step][1] = v.y;
                    qf[nt][step + 1][0] = v.z; qf[nt][step + 1][1] = v.w;
                }
            float up = 1.0f;                                  // what brings a row's scores back
            if (FMT != ELUTQ_KV_16 && a.type == ELUTQ_TYPE_BF16) {
                // bf16 to fp16: the row times a power of two, its largest magnitude in [1, 2).  What is less than 2^-24 of that is cut off, as it would be from the sum.
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < STEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) top = max(top, max(qf[nt][k][i] & 0x7fffu, qf[nt][k][i] >> 16 & 0x7fffu));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int e = min(max((int)(top >> 7), 1), 253);           // (subnormal rows and those with infinities: as near as a normal power gets)
                const float down = __uint_as_float((uint32_t)(254 - e) << 23);
                up = __uint_as_float((uint32_t)e << 23);
#pragma unroll
                for (int k = 0; k < STEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        qf[nt][k][i] = pack<false>(__uint_as_float(qf[nt][k][i] << 16) * down, __uint_as_float(qf[nt][k][i] & 0xffff0000u) * down);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // (lane 8 t + 4 j holds column 2 t + j)
                cs[nt][j] = a.scale * kf * __shfl_sync(0xffffffffu, up, 8 * t + 4 * j);
                const int rr = rt * NC + nt * 8 + 2 * t + j;
                limit[nt][j] = rr < a.rows ? least + rr / a.group : len;
                off[nt][j] = kNone;
                sum[nt][j] = 0.0f;
            }
        }
        float o[STEPS][NT][4];
#pragma unroll
        for (int m = 0; m < STEPS; ++m)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[m][nt][i] = 0.0f;

        for (int n = 0; n < mine; ++n) {
            const int tok0 = (tile0 + warp + n * kWarps) * TT;
            // ---- scores ----------------------------------------------------------------------------------------------------------------------
            float sc[SUB][NT][4];
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[s][nt][i] = 0.0f;
                [[maybe_unused]] uint32_t blk[2][2];          // [row][block of this lane]: scale, in both halves
                if constexpr (SCALED) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t two = e4m3_pair(ksc[s][r]);
                        blk[r][0] = prmt(two, two, 0x1010);
                        blk[r][1] = prmt(two, two, 0x3232);
                    }
                }
#pragma unroll
                for (int w = 0; w < KW; ++w) {                // a word of both rows: PER_WORD / 4 steps
                    uint32_t x[2][PER_WORD / 2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const uint32_t v = kr[s][r][w];
                        if constexpr (FMT == ELUTQ_KV_16) {
                            x[r][0] = v;
                        } else if constexpr (FMT == ELUTQ_KV_E4M3) {
                            x[r][0] = e4m3_pair(v);
                            x[r][1] = e4m3_pair(v >> 16);
                        } else {
#pragma unroll
                            for (int i = 0; i < 4; ++i) x[r][i] = hmul2(e2m1_pair(v >> (8 * i)), blk[r][w / 2]);
                        }
                    }
                    if constexpr (FMT == ELUTQ_KV_16) {
                        if (w % 2 == 1) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                mma<BF16>(sc[s][nt], kr[s][0][w - 1], kr[s][1][w - 1], kr[s][0][w], kr[s][1][w], qf[nt][w / 2][0], qf[nt][w / 2][1]);
                        }
                    } else {
#pragma unroll
                        for (int i = 0; i < PER_WORD / 4; ++i)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
                                mma<BF16>(sc[s][nt], x[0][2 * i], x[1][2 * i], x[0][2 * i + 1], x[1][2 * i + 1], qf[nt][w * (PER_WORD / 4) + i][0], qf[nt][w * (PER_WORD / 4) + i][1]);
                    }
                }
            }
            const uint32_t pages_there = there;
            const bool last = tok0 + TT > least;              // some column may not see all of the tile
            if (last || pages_there != (1u << SUB) - 1u) {
#pragma unroll
                for (int s = 0; s < SUB; ++s)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int tok = tok0 + 16 * s + g + 8 * (i >> 1);
                            if (tok >= limit[nt][i & 1] || !(pages_there >> s & 1u)) sc[s][nt][i] = -INFINITY;
                        }
            }
            // ---- softmax: P of this tile ---------------------------------------------------------------------------------------------------------
            float top[NT][2];
            bool rises = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    top[nt][j] = -INFINITY;
#pragma unroll
                    for (int s = 0; s < SUB; ++s) top[nt][j] = fmaxf(top[nt][j], fmaxf(sc[s][nt][j], sc[s][nt][j + 2]));
                    rises |= fmaf(top[nt][j], cs[nt][j], off[nt][j]) > kRise;
                }
            if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float x = top[nt][j];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                        const float to = x == -INFINITY ? off[nt][j] : fminf(off[nt][j], kBase - x * cs[nt][j]);
                        const float by = exp2_approx(to - off[nt][j]);
                        off[nt][j] = to;
                        sum[nt][j] *= by;
#pragma unroll
                        for (int m = 0; m < STEPS; ++m) {
                            o[m][nt][j] *= by;
                            o[m][nt][j + 2] *= by;
                        }
                    }
            }
            uint32_t pf[SUB][NT][2];
#pragma unroll
            for (int s = 0; s < SUB; ++s)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        p[i] = exp2_approx(fmaf(sc[s][nt][i], cs[nt][i & 1], off[nt][i & 1]));
                        sum[nt][i & 1] += p[i];
                    }
                    pf[s][nt][0] = transposed(pack<BF16>(p[0], p[1]));
                    pf[s][nt][1] = transposed(pack<BF16>(p[2], p[3]));
                }
            // ---- P V ---------------------------------------------------------------------------------------------------------------------------
            if (tok0 + TT > len || pages_there != (1u << SUB) - 1u) {        // rows that no column sees: zeros
#pragma unroll
                for (int s = 0; s < SUB; ++s)
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        if (tok0 + 16 * s + 2 * t + (r & 1) + 8 * (r >> 1) >= len || !(pages_there >> s & 1u)) {
#pragma unroll
                            for (int i = 0; i < VW; ++i) vr[s][r][i] = 0;
                            if constexpr (SCALED) vsc[s] &= ~(0xffu << (8 * r));
                        }
            }
            // V rows of a piece as fragments: word w of its four rows holds dimensions 2 w, 2 w + 1 of this lane's, tile w of the result
            auto v_word = [&](int s, int r, int w) {
                if constexpr (FMT == ELUTQ_KV_16) return vr[s][r][w];
                else if constexpr (FMT == ELUTQ_KV_E4M3) return e4m3_pair(vr[s][r][w / 2] >> (16 * (w & 1)));
                else return e2m1_pair(vr[s][r][w / 4] >> (8 * (w & 3)));
            };
            auto v_fragment = [&](int s, int w, uint32_t (&x)[4]) {
                const uint32_t r0 = v_word(s, 0, w), r1 = v_word(s, 1, w), r2 = v_word(s, 2, w), r3 = v_word(s, 3, w);
                x[0] = prmt(r0, r1, 0x5410);
                x[1] = prmt(r0, r1, 0x7632);
                x[2] = prmt(r2, r3, 0x5410);
                x[3] = prmt(r2, r3, 0x7632);
                if constexpr (SCALED) {
                    const uint32_t lo = e4m3_pair(vsc[s]), hi = e4m3_pair(vsc[s] >> 16);
                    x[0] = hmul2(x[0], lo);
                    x[1] = hmul2(x[1], lo);
                    x[2] = hmul2(x[2], hi);
                    x[3] = hmul2(x[3], hi);
                }
            };
            if (!last || a.fresh == 1) {
#pragma unroll
                for (int s = 0; s < SUB; ++s)
#pragma unroll
                    for (int m = 0; m < STEPS; ++m) {
                        uint32_t x[4];
                        v_fragment(s, m, x);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<BF16>(o[m][nt], x[0], x[1], x[2], x[3], pf[s][nt][0], pf[s][nt][1]);
                    }
            } else {
                // each new token's columns by themselves, with V rows that it does not see replaced by zeros
                const int first = rt * NC / a.group, end = min(a.fresh, (rt * NC + NC - 1) / a.group + 1);
                for (int nw = first; nw < end; ++nw) {
                    const int sees = least + nw;
#pragma unroll
                    for (int m = 0; m < STEPS; ++m) {
                        float part[NT][4];
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i) part[nt][i] = 0.0f;
#pragma unroll
                        for (int s = 0; s < SUB; ++s) {
                            uint32_t x[4];
                            v_fragment(s, m, x);
                            const int tok = tok0 + 16 * s + 2 * t;
                            const uint32_t lo = (tok < sees ? 0xffffu : 0u) | (tok + 1 < sees ? 0xffff0000u : 0u);
                            const uint32_t hi = (tok + 8 < sees ? 0xffffu : 0u) | (tok + 9 < sees ? 0xffff0000u : 0u);
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma<BF16>(part[nt], x[0] & lo, x[1] & lo, x[2] & hi, x[3] & hi, pf[s][nt][0], pf[s][nt][1]);
                        }
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (limit[nt][i & 1] == sees) o[m][nt][i] += part[nt][i];
                    }
                }
            }
            if (n + 1 < mine) {
                load_k(n + 1);
                load_v(n + 1);
            }
        }

        // ---- the warps' parts meet ----------------------------------------------------------------------------------------------------------------
        const int active = min(kWarps, count);
        if (mine > 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], d);
                    const int col = nt * 8 + 2 * t + j;
                    if (g == 0) {
                        s_off[warp][col] = off[nt][j];
                        s_sum[warp][col] = sum[nt][j];
                    }
#pragma unroll
                    for (int m = 0; m < STEPS; ++m) {
                        // dimension of word m of this lane's pieces of V rows
                        constexpr int PIECE = VC * PER_WORD;
                        const int d = PIECE * (g + 8 * (2 * m / PIECE)) + 2 * m % PIECE;
                        *reinterpret_cast<float2*>(&s_o[warp][col][d]) = make_float2(o[m][nt][j], o[m][nt][j + 2]);
                    }
                }
        }
        __syncthreads();
        const bool begins = tile0 == 0, whole = begins && count == tiles;
        const int used = min(NC, a.rows - rt * NC);
        const float vf = a.c.vf == nullptr ? 1.0f : __ldg(a.c.vf + h);
        float* part = a.parts + ((long long)blockIdx.x * 2 + (begins ? 1 : 0)) * (NC * (D + 2));
        for (int i = tid; i < used * (D / 2); i += kThreads) {
            const int col = i / (D / 2), d = 2 * (i - col * (D / 2));
            float low = kNone;
            for (int w = 0; w < active; ++w) low = fminf(low, s_off[w][col]);
            float total = 0.0f, x = 0.0f, y = 0.0f;
            for (int w = 0; w < active; ++w) {
                const float by = exp2_approx(low - s_off[w][col]);
                const float2 v = *reinterpret_cast<const float2*>(&s_o[w][col][d]);
                total = fmaf(s_sum[w][col], by, total);
                x = fmaf(v.x, by, x);
                y = fmaf(v.y, by, y);
            }
            if (whole) {
                const float r = total == 0.0f ? 0.0f : vf / total;
                const int rr = rt * NC + col, tok = rr / a.group, head = h * a.group + (rr - tok * a.group);
                uint8_t* p = a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D + d);
                *reinterpret_cast<uint32_t*>(p) = a.type == ELUTQ_TYPE_F16 ? pack<false>(x * r, y * r) : pack<true>(x * r, y * r);
            } else {
                if (d == 0) {
                    part[col] = low;
                    part[NC + col] = total;
                }
                *reinterpret_cast<float2*>(part + 2 * NC + col * D + d) = make_float2(x, y);
            }
        }
        __syncthreads();
        f += count;
        if (f - before == (long long)tiles * each) {
            before = f;
            ++b;
        }
    }
}

// Joins the parts of the segments that several shares hold, in their order; columns that see nothing get zeros.  A block per (segment, query row), a thread per dimension.
template <int D, int TT, int NT>
__global__ void __launch_bounds__(D) attn_join_kernel(const DecodeArgs a, int ctas) {
    constexpr int NC = 8 * NT;
    __shared__ long long s_scan[2 * (D / 32)];
    grid_dependency_wait();
    grid_launch_dependents();
    const int row = blockIdx.x % a.rows, seg_all = blockIdx.x / a.rows, h = seg_all % a.c.heads, b = seg_all / a.c.heads;
    const int rt = row / NC, col = row - rt * NC, d = threadIdx.x;
    long long before, total;
    count_units<TT>(a, b, before, total, s_scan);
    const int tiles = tiles_of<TT>(length_of(a, b));
    const int tok = row / a.group, head = h * a.group + (row - tok * a.group);
    uint8_t* out = a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D + d);
    if (tiles == 0) {
        *reinterpret_cast<uint16_t*>(out) = 0;
        return;
    }
    const long long share = share_of(total, ctas);
    const long long first = before + (long long)(h * a.row_tiles + rt) * tiles, last = first + tiles - 1;
    const int c0 = (int)(first / share), c1 = (int)(last / share);
    if (c0 == c1) return;
    constexpr int SIZE = NC * (D + 2);
    auto part_of = [&](int c) { return a.parts + ((long long)c * 2 + (c == c0 ? 1 : 0)) * SIZE; };
    float low = kNone;
    for (int c = c0; c <= c1; ++c) low = fminf(low, part_of(c)[col]);
    float sum = 0.0f, x = 0.0f;
    for (int c = c0; c <= c1; ++c) {
        const float* p = part_of(c);
        const float by = exp2_approx(low - p[col]);
        sum = fmaf(p[NC + col], by, sum);
        x = fmaf(p[2 * NC + col * D + d], by, x);
    }
    x *= sum == 0.0f ? 0.0f : (a.c.vf == nullptr ? 1.0f : __ldg(a.c.vf + h)) / sum;
    const uint32_t v = a.type == ELUTQ_TYPE_F16 ? pack<false>(x, 0.0f) : pack<true>(x, 0.0f);
    *reinterpret_cast<uint16_t*>(out) = (uint16_t)v;
}

// CTAs of a launch: as many as are resident at once
inline int ctas_of(int nt) { return device_sm_count() * (nt == 1 ? 3 : 2); }
inline int columns_of(int rows) { return rows <= 8 ? 1 : 2; }

int launch_one(const void* kernel, int grid, int block, void** args, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}

template <int D, int FMT, bool BF16, int NT>
int launch_decode(DecodeArgs a, cudaStream_t stream) {
    int ctas = ctas_of(NT);
    void* args[] = {&a, &ctas};
    const int e = launch_one((const void*)attn_decode_kernel<D, FMT, BF16, NT>, ctas, kThreads, args, stream);
    if (e != 0) return e;
    return launch_one((const void*)attn_join_kernel<D, tile_tokens(FMT, D), NT>, a.B * a.c.heads * a.rows, D, args, stream);
}
template <int D, int FMT, bool BF16>
int launch_decode(const DecodeArgs& a, cudaStream_t stream) {
    return columns_of(a.rows) == 1 ? launch_decode<D, FMT, BF16, 1>(a, stream) : launch_decode<D, FMT, BF16, 2>(a, stream);
}
template <int D>
int launch_decode(const DecodeArgs& a, int format, cudaStream_t stream) {
    if (format == ELUTQ_KV_16) return a.type == ELUTQ_TYPE_BF16 ? launch_decode<D, ELUTQ_KV_16, true>(a, stream) : launch_decode<D, ELUTQ_KV_16, false>(a, stream);
    return format == ELUTQ_KV_E4M3 ? launch_decode<D, ELUTQ_KV_E4M3, false>(a, stream) : launch_decode<D, ELUTQ_KV_NVFP4, false>(a, stream);
}

}  // namespace

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_attn_decode_workspace_bytes(int n_q_heads, int heads, int head_dim, int new_tokens, size_t* bytes) {
    if (!bytes || n_q_heads <= 0 || heads <= 0 || new_tokens <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (head_dim != 64 && head_dim != 128) return ELUTQ_ERR_UNSUPPORTED;
    if (n_q_heads % heads != 0 || (long long)n_q_heads / heads * new_tokens > 0xffff) return ELUTQ_ERR_SHAPE;
    const int nt = columns_of(n_q_heads / heads * new_tokens);
    *bytes = (size_t)ctas_of(nt) * 2 * (8 * nt) * (head_dim + 2) * sizeof(float);
    return ELUTQ_OK;
}

extern "C" int elutq_attn_decode(const elutq_kv_cache* cache, const void* q, long long ldq, void* out, long long ldo, const int* table, long long ld_table, int pages,
                                 const int* lens, int B, int new_tokens, int n_q_heads, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    int st = kv_check(cache);
    if (st != ELUTQ_OK) return st;
    if (!q || !out || !table || !lens || !workspace || pages <= 0 || B <= 0 || new_tokens <= 0 || n_q_heads <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !(scale < 1e30f)) return ELUTQ_ERR_INVALID_ARG;
    const int D = cache->head_dim, H = cache->heads;
    size_t need = 0;
    if ((st = elutq_attn_decode_workspace_bytes(n_q_heads, H, D, new_tokens, &need)) != ELUTQ_OK) return st;
    if (ld_table < pages) return ELUTQ_ERR_SHAPE;
    if ((st = kv_rows_check(q, ldq, n_q_heads, D)) != ELUTQ_OK || (st = kv_rows_check(out, ldo, n_q_heads, D)) != ELUTQ_OK) return st;
    if (!mx4_aligned(table, 4) || !mx4_aligned(lens, 4) || !mx4_aligned(workspace, 16)) return ELUTQ_ERR_ALIGN;
    if (workspace_bytes < need) return ELUTQ_ERR_BUFFER_TOO_SMALL;
    DecodeArgs a;
    a.c = kv_view(cache);
    a.q = (const uint8_t*)q;
    a.out = (uint8_t*)out;
    a.ldq = ldq; a.ldo = ldo;
    a.table = table; a.lens = lens;
    a.ld_table = ld_table;
    a.wide = pages;
    a.B = B;
    a.fresh = new_tokens;
    a.group = n_q_heads / H;
    a.rows = a.group * new_tokens;
    const int nc = 8 * columns_of(a.rows);
    a.row_tiles = (a.rows + nc - 1) / nc;
    a.type = cache->type;
    a.scale = scale * 1.44269504088896340736f;
    a.parts = (float*)workspace;
    a.cap = (long long)pages * cache->page_size;
    if (a.cap > 0x7fff0000LL) a.cap = 0x7fff0000LL;               // (token numbers a little behind the last one are formed)
    if ((long long)B * n_q_heads * new_tokens > 0x7fffffffLL) return ELUTQ_ERR_SHAPE;      // (blocks of a launch)
    const int ce = D == 128 ? launch_decode<128>(a, cache->format, (cudaStream_t)stream) : launch_decode<64>(a, cache->format, (cudaStream_t)stream);
    if (ce == 0) return ELUTQ_OK;
    note_cuda_error(ce);
    return ELUTQ_ERR_CUDA;
}
