// Attention of the newest token(s) of every sequence over a paged cache in 16 bits, E4M3 or NVFP4, which is read once and never written out in 16 bits.
//
//   o = sum_j 2^(x_j - m) V_j / sum_j 2^(x_j - m),   x_j = log2(e) scale q . K_j,   j up to the query's own position
//
// work       Query rows of one key head (the heads that share it, times the new tokens) are the N of both products, 8 or 16 at a time, the cache's tokens the
//            M of the first and head dimensions the M of the second: with 4 or 8 heads to a key head no row of the tensor core's tiles is left empty.
//              S^T [tokens x rows] = K Q^T,   O^T [dims x rows] += V^T P^T
//            The order of an inner index is free, so a lane takes whole 16-byte pieces of K rows and of V rows as fragments: no transposition but that of P
//            (movmatrix) and of pairs of V rows (byte permutes, on the codes).
// loads      Every warp has a ring of stages of its own in shared memory, filled by asynchronous copies of 16 bytes to a lane, so a warp never waits for another within a
//            segment.  Pieces are placed so that the fragments' reads meet no bank twice.  Rows behind a sequence and on pages that do not exist come as zeros.
// split      All (sequence, key head, rows) segments laid behind one another, in tiles, are cut into equal shares, one for each warp that the GPU holds: lengths may
//            be as ragged as they like.  A segment counts kLead tiles more, for what it costs to begin one.  A segment that lies within one share is finished there, the
//            parts of others go to the workspace and a second kernel joins them in their order.  Where all shares of a CTA are of one segment they are joined
//            in shared memory first.
// softmax    One running maximum for all lanes of a column, moved only when a tile rises more than 2^10 above it (then everything is scaled): P stays below
//            2^14, in fp16; in bf16, which has the range for it, below half of one over the number of tokens, so that sums of the largest values are finite.  Maximum, sum
//            and result are fp32.
//            (P goes to 16 bits because the tensor core takes it so: a weight is off by 2^-12 of itself in fp16, 2^-9 in bf16, next to a result of 16 bits.  The sum takes the weights as
//            they were.  Against the definition in 64 bits results are off 1.0 to 1.4 times as far as with weights of fp32, most where one weight outdoes all others.)
// codes      E4M3 and E2M1 values, also times an E4M3 block scale, are exact in fp16, so both products are fp16 ones, with q brought to fp16 by a power of two for each row.
//            The heads' factors are multiplied into the scale and into the result.
//
// Masked places never reach the result, whatever they hold: scores are selected, V rows behind the sequence are zeros, and in the last tiles, where
// the new tokens of a sequence see different lengths, every token's product is formed by itself.
//
// Bound: HBM (the cache), for few tokens the latency of table, keys, joining.  Measured (32 query heads, 8 key heads, dimension 128, us in a graph): 16 bits, 64 sequences of 2048 to
// 4096 tokens 128, 98 % of the copy rate; E4M3, 64 of 4096 to 8192 138, 91 %; NVFP4, 64 of 4096 to 16384 166, 72 %: two warps to a scheduler, each a chain of scores, softmax
// and products, no unit full (issue 54 %, of its stalls two thirds the wait for the instruction in front).  One sequence of 128K tokens in NVFP4 42, 55 %; one of 1000 in 16 bits 6.5.
#include <atomic>
#include <cmath>

#include "kv.cuh"

namespace elutq {

namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kLead = 4;
constexpr long long kMostTokens = 0x7fff0000LL;      // of a sequence (numbers a little behind the last one are formed)
constexpr int kShortTokens = 128;            // of a warp
constexpr float kRise = 14.0f, kLag = 10.0f; // 2^(x - m + 4) in fp16, m moved when that would pass 2^14

struct DecodeArgs {
    KvView c;
    const uint8_t* q;
    uint8_t* out;
    long long ldq, ldo;        // elements between tokens
    const int *table, *lens;
    long long ld_table;
    int B, fresh, group;       // sequences, new tokens of each, query heads of a key head
    int rows, row_tiles;       // query rows of a key head; tiles of them
    int type;
    float scale;               // times log2(e)
    float part;                // the same as part * 2^power, part in [0.5, 1)
    int power;
    float* parts;
    int4* begun;               // segments that begin in a share and go on in the next ones: sequence, key head and tile of rows, worker, where its parts are (0: none).  For each
                               // segment, or, where there are more of them than shares, for each share
    int by_segment;
    int split;                 // CTAs of a cluster that have a segment to themselves; 0: shares of the whole
    long long cap;             // wide * page_size: tokens that the table has room for
};

__host__ __device__ constexpr int row_bytes(int format, int D) { return format == ELUTQ_KV_16 ? 2 * D : format == ELUTQ_KV_E4M3 ? D : D / 2; }
// Tokens of a stage
__host__ __device__ constexpr int tile_tokens(int format, int D) { return row_bytes(format, D) >= 128 ? 16 : 32; }
__host__ __device__ constexpr int stage_bytes(int format, int D) { return tile_tokens(format, D) * 2 * (row_bytes(format, D) + (format == ELUTQ_KV_NVFP4 ? D / 16 : 0)); }
__host__ __device__ constexpr int stages_of(int format, int D) { return stage_bytes(format, D) > 4608 ? 2 : 13824 / stage_bytes(format, D); }
// CTAs that an SM holds: by shared memory, and by the registers that the results take.  NVFP4 has its 32 tokens a turn in registers, too: 234 of them for dimension 128, 223
// for 64 and two tiles of columns.  With three CTAs of 168 some are spilled; that is still ahead where a grid of short sequences runs in fewer rounds that way (plan_of).
__host__ __device__ constexpr bool either(int format, int D, int nt) { return format == ELUTQ_KV_NVFP4 && (D == 128) == (nt == 1); }
__host__ __device__ constexpr int resident(int format, int D, int nt) { return (nt == 2 && D == 128) || either(format, D, nt) ? 2 : 3; }

__device__ __forceinline__ int length_of(const DecodeArgs& a, int b) {
    const long long n = __ldg(a.lens + b);
    return (int)(n < 0 ? 0 : n > a.cap ? a.cap : n);
}

template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The same without a sum in front
template <bool BF16>
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (BF16)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
            : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
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
// All codes of a word as fp16, two at a time.  (Bytes unpacked in one piece: the conversion takes its byte from any place of a register, while a shift in front of it costs as
// much as the conversion itself.)
__device__ __forceinline__ void e4m3_pairs(uint32_t (&h)[2], uint32_t w) {
    asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\tcvt.rn.f16x2.e4m3x2 %1, hi;\n\t}" : "=r"(h[0]), "=r"(h[1]) : "r"(w));
}
__device__ __forceinline__ void e2m1_pairs(uint32_t (&h)[4], uint32_t w) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float((e + 127) << 23); }       // -126 <= e <= 127
// 16 bytes to shared memory
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(dst), "l"(src) : "memory");
}
// ... the first `bytes` of them and zeros
__device__ __forceinline__ void copy16(uint32_t dst, const uint8_t* src, int bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}
// (plain loads: the compiler may move them, but not over the wait for the copies)
template <int BYTES>
__device__ __forceinline__ void read_shared(uint32_t* w, const uint8_t* p) {
    if constexpr (BYTES == 16) {
        const uint4 v = *reinterpret_cast<const uint4*>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (BYTES == 8) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}

// Four 8 x 8 matrices of 16 bits, as they are or turned; a lane gives the address of a row
template <bool TURNED>
__device__ __forceinline__ void read_matrices(uint32_t (&x)[4], uint32_t addr) {
    if constexpr (TURNED) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}

template <int TT>
__device__ __forceinline__ int tiles_of(int len) { return (len + TT - 1) / TT; }

// Units of a segment: its tiles and kLead more; none without a token
template <int TT>
__device__ __forceinline__ int units_of(int len) { return len == 0 ? 0 : tiles_of<TT>(len) + kLead; }
// Units of all sequences, by a warp.
template <int TT>
__device__ __forceinline__ long long count_units(const DecodeArgs& a) {
    long long total = 0;
    for (int b = threadIdx.x & 31; b < a.B; b += 32) total += units_of<TT>(length_of(a, b));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
    return total * a.c.heads * a.row_tiles;
}
// a / b, a below 2^63: mostly a 32-bit division, a tenth of a 64-bit one's instructions
__device__ __forceinline__ long long quotient_of(long long a, int b) {
    return a >> 32 == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
template <int D, int FMT, bool BF16, int NT, int PER>
__global__ void __launch_bounds__(kThreads, PER) attn_decode_kernel(const DecodeArgs a) {
    constexpr int TT = tile_tokens(FMT, D), SUB = TT / 16, NC = 8 * NT, S = stages_of(FMT, D), STAGE = stage_bytes(FMT, D);
    constexpr int ROW = row_bytes(FMT, D), PIECES = ROW / 16;
    constexpr int PER_WORD = FMT == ELUTQ_KV_16 ? 2 : FMT == ELUTQ_KV_E4M3 ? 4 : 8;      // values of a word
    constexpr int KW = ROW / 16, KC = KW < 4 ? KW : 4;       // words of a K row in a lane; of a piece
    constexpr int VW = ROW / 32, VC = VW < 4 ? VW : 4;
    constexpr int STEPS = D / 16;                            // of 16 head dimensions; also 16-dimension tiles of the result
    constexpr bool SCALED = FMT == ELUTQ_KV_NVFP4;
    constexpr int PAD = D + 4;
    constexpr int V0 = TT * ROW, KS0 = 2 * TT * ROW, VS0 = KS0 + TT * (D / 16);          // in a stage: K, V, their scales
    extern __shared__ __align__(1024) uint8_t smem[];
    // (the warps' parts lie over their rings, which are empty by then)
    float (*s_o)[NC][PAD] = reinterpret_cast<float (*)[NC][PAD]>(smem);
    __shared__ float s_off[kWarps][NC], s_sum[kWarps][NC], s_all[2][NC];

    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), g = lane >> 2, t = lane & 3;
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * (S * STAGE);
    grid_dependency_wait();
    grid_launch_dependents();

    // ---- this warp's share: units [f0, f1) of [0, total), or a part of the segment that the cluster has ---------------------------------------------------
    const int each = a.c.heads * a.row_tiles, worker = blockIdx.x * kWarps + warp;
    int b = 0;
    long long total = 0, share = 0, cta0 = 0, cta1 = 0, f0 = 0, f1 = 0;
    long long before = 0;                                     // units in front of the sequence
    bool joint = true;                                        // all of the CTA's units are of one segment
    if (a.split != 0) {
        b = blockIdx.x / a.split / each;
    } else {
        total = count_units<TT>(a);
        share = quotient_of(total + gridDim.x * kWarps - 1, gridDim.x * kWarps);
        cta0 = blockIdx.x * kWarps * share;
        cta1 = cta0 + kWarps * share < total ? cta0 + kWarps * share : total;
        // sequences without a token: zeros
        for (int e = blockIdx.x; e < a.B; e += gridDim.x)
            if (length_of(a, e) == 0) {
                if (a.by_segment)
                    for (int i = tid; i < each; i += kThreads) a.begun[e * each + i] = make_int4(0, 0, 0, 0);
                for (long long i = tid; i < (long long)a.fresh * a.c.heads * a.group * (D / 8); i += kThreads) {
                    const long long tok = i / (a.c.heads * a.group * (D / 8));
                    reinterpret_cast<uint4*>(a.out + 2 * ((long long)e * a.fresh + tok) * a.ldo)[i - tok * (a.c.heads * a.group * (D / 8))] = make_uint4(0u, 0u, 0u, 0u);
                }
            }
        if (cta0 >= cta1) {                                   // (the whole CTA)
            if (lane == 0 && !a.by_segment) a.begun[worker] = make_int4(0, 0, 0, 0);
            return;
        }
        // the sequence that the CTA's first unit belongs to: 32 at a time
        for (; b < a.B; b += 32) {
            const long long mine = b + lane < a.B ? (long long)units_of<TT>(length_of(a, b + lane)) * each : 0;
            long long incl = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const uint32_t behind = __ballot_sync(0xffffffffu, before + incl > cta0);
            if (behind != 0) {
                const int l = __ffs(behind) - 1;
                before += __shfl_sync(0xffffffffu, incl - mine, l);
                b += l;
                break;
            }
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (b >= a.B) return;                                 // (only where lengths change during the call)
        const int units = units_of<TT>(length_of(a, b));
        joint = cta1 <= before + (quotient_of(cta0 - before, units) + 1) * units;
        f0 = cta0 + warp * share;
        f1 = f0 + share < cta1 ? f0 + share : cta1;
    }

    // where a lane copies to and reads from.  A piece's place in its row is its number with some bits of the row's number turned, so that the lanes that are served together
    // meet different banks: 16 bits, the same piece of eight rows (ldmatrix); codes, two K rows, or four V rows, of which every second.
    auto k_turn = [](int r) { return FMT == ELUTQ_KV_16 ? r & 7 : PIECES >= 8 ? (r & 1) << 2 : 0; };
    auto v_turn = [](int r) { return FMT == ELUTQ_KV_16 ? r & 7 : PIECES >= 8 ? (r >> 1 & 3) << 1 : PIECES == 4 ? r >> 1 & 3 : 0; };
    constexpr int ROWS = 32 / PIECES;                         // rows of a copy of the warp
    const int cr = lane / PIECES, cc = lane % PIECES;
    // (in the 512 bytes of one; after TURNS of them the rows' turns are the first one's again)
    constexpr int TURNS = PIECES >= 8 ? PIECES / 4 : 1;
    uint32_t k_to[TURNS], v_to[TURNS];
#pragma unroll
    for (int i = 0; i < TURNS; ++i) {
        k_to[i] = cr * ROW + 16 * (cc ^ k_turn(i * ROWS + cr));
        v_to[i] = cr * ROW + 16 * (cc ^ v_turn(i * ROWS + cr));
    }
    const uint8_t *k_lane = a.c.k + lane * 16, *v_lane = a.c.v + lane * 16;
    [[maybe_unused]] const uint8_t* s_lane = (lane < 16 ? a.c.ks : a.c.vs) + (lane & 15) % (D / 16) * 16;
    [[maybe_unused]] const uint32_t s_to = (lane < 16 ? KS0 : VS0) + (lane & 15) * 16;
    const uint8_t* own = smem + warp * (S * STAGE);
    const uint32_t k_read = FMT == ELUTQ_KV_16 ? (lane & 15) * ROW + 16 * (lane >> 4 ^ (lane & 7))
                                               : g * ROW + (KC == 4 ? 16 * (t ^ k_turn(g)) : 4 * KC * t);
    const uint32_t v_read = V0 + (FMT == ELUTQ_KV_16 ? ((lane & 7) + (lane >> 4) * 8) * ROW + 16 * ((lane >> 3 & 1) ^ (lane & 7))
                                                     : 2 * t * ROW + (VC == 4 ? 16 * (g ^ v_turn(2 * t)) : VC == 2 ? 16 * ((g >> 1) ^ v_turn(2 * t)) + 8 * (g & 1) : 4 * g));

    bool recorded = false;
    // (joint: every warp once, with or without tiles)
    for (long long f = f0; f < f1 || joint;) {
        const int len = length_of(a, b), tiles = tiles_of<TT>(len), units = units_of<TT>(len);
        if (!joint && f - before >= (long long)units * each) {
            before += (long long)units * each;
            if (++b >= a.B) break;
            continue;
        }
        int seg, tile0, mine, unit0 = 0, unit1 = 0;           // the segment of the sequence; this warp's tiles
        long long seg0 = 0;                                   // the segment's first unit
        if (a.split != 0) {
            const int rank = blockIdx.x % a.split, at = kWarps * rank + warp, of = kWarps * a.split;
            seg = blockIdx.x / a.split - b * each;
            tile0 = (int)((long long)tiles * at / of);
            mine = (int)((long long)tiles * (at + 1) / of) - tile0;
        } else {
            const long long at_most = f1 - f, local = (f < cta1 ? f : cta1 - 1) - before;
            seg = (int)quotient_of(local, units);
            seg0 = before + (long long)seg * units;
            unit0 = (int)(local - (long long)seg * units);
            unit1 = (int)(at_most < units - unit0 ? (at_most < 0 ? unit0 : unit0 + at_most) : units);
            tile0 = max(0, unit0 - kLead);
            mine = max(0, unit1 - kLead) - tile0;
        }
        const int h = seg / a.row_tiles, rt = seg - h * a.row_tiles;
        if (!joint && mine == 0) {
            f += unit1 - unit0;
            continue;
        }
        const int* pages = a.table + b * a.ld_table;
        // (bf16: len weights of less than half of 1 / len cannot bring the largest values beyond fp32.  It is values next to the smallest normal number that lose bits for it.)
        const float most = FMT == ELUTQ_KV_16 && BF16 ? (float)(__clz(len) - 33) : kRise;
        const int least = len - a.fresh + 1;                  // tokens that the first of the new tokens sees

        // ---- copies ----------------------------------------------------------------------------------------------------------------------------
        uint32_t gone = 0;                                    // a bit for each 16 tokens of the stages: their page does not exist
        long long from = -1;                                  // lane i: where the i-th of 32 pieces of 16 tokens of this warp's tiles begins in the cache, in bytes of K; below 0: nowhere
        int page = -1;                                        // the same of the next 32 pieces: their page
        auto look_up = [&](int n) {
            const int tok = (tile0 + n + lane / SUB) * TT + (lane % SUB) * 16;
            page = n + lane / SUB < mine && tok < len ? __ldg(pages + a.c.page.of(tok)) : -1;
        };
        look_up(0);
        auto copy = [&](int n, int slot) {
            const int piece = n * SUB & 31;
            if (piece == 0) {
                const int tok = (tile0 + n + lane / SUB) * TT + (lane % SUB) * 16;
                from = page < 0 || page >= a.c.n_pages ? -1 : (((long long)page * a.c.heads + h) * a.c.page_size + (tok - a.c.page.of(tok) * a.c.page_size)) * ROW;
                look_up(n + 32 / SUB);
            }
            const int left = len - (tile0 + n) * TT;          // tokens from the stage's first on
            const uint32_t at = ring + slot * STAGE;
            long long src[SUB];
            bool all = left >= TT;
#pragma unroll
            for (int s = 0; s < SUB; ++s) {
                src[s] = __shfl_sync(0xffffffffu, from, piece + s);
                all &= src[s] >= 0;
            }
            if (gone != 0) gone &= ~(((1u << SUB) - 1u) << (slot * SUB));
            if (all) {
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    const uint8_t *k = k_lane + src[s], *v = v_lane + src[s];
#pragma unroll
                    for (int i = 0; i < 16 / ROWS; ++i) copy16(at + k_to[i % TURNS] + (16 * s * ROW + i * 512), k + i * 512);
#pragma unroll
                    for (int i = 0; i < 16 / ROWS; ++i) copy16(at + v_to[i % TURNS] + (V0 + 16 * s * ROW + i * 512), v + i * 512);
                }
            } else {
#pragma unroll
                for (int s = 0; s < SUB; ++s) {
                    const long long start = src[s] < 0 ? 0 : src[s];
                    const int some = src[s] < 0 ? 0 : left - 16 * s;
                    gone |= (uint32_t)(src[s] < 0) << (slot * SUB + s);
#pragma unroll
                    for (int i = 0; i < 16 / ROWS; ++i) {
                        copy16(at + k_to[i % TURNS] + (16 * s * ROW + i * 512), k_lane + start + i * 512, i * ROWS + cr < some ? 16 : 0);
                        copy16(at + v_to[i % TURNS] + (V0 + 16 * s * ROW + i * 512), v_lane + start + i * 512, i * ROWS + cr < some ? 16 : 0);
                    }
                }
            }
            if constexpr (SCALED) {
                // 16 tokens' scales are D bytes, D / 16 lanes', an eighth of their codes; half of the lanes copy K's and half V's
                constexpr int LANES = D / 16;
                const int l = lane & 15, s = l / LANES;
                const long long start = __shfl_sync(0xffffffffu, from, piece + (s < SUB ? s : 0));
                if (s < SUB) {
                    if (all) copy16(at + s_to, s_lane + (start >> 3));
                    else copy16(at + s_to, s_lane + ((start < 0 ? 0 : start) >> 3), start < 0 ? 0 : min(max((left - 16 * s) * (D / 16) - l % LANES * 16, 0), 16));
                }
            }
        };
        auto commit = [] { asm volatile("cp.async.commit_group;" ::: "memory"); };
#pragma unroll
        for (int n = 0; n < S; ++n) {
            if (n < mine) copy(n, n);
            commit();
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
            if constexpr (FMT == ELUTQ_KV_16) {
#pragma unroll
                for (int k = 0; k < STEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) qf[nt][k][i] = r < a.rows ? __ldg(reinterpret_cast<const uint32_t*>(p) + 8 * k + 4 * i + t) : 0u;
            } else {
                constexpr int PIECE = KC * PER_WORD;          // head dimensions of a piece of K
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
            }
            int back = 0;                                     // the power of two that brings a row's scores back
            if (FMT != ELUTQ_KV_16 && a.type == ELUTQ_TYPE_BF16) {
                // bf16 to fp16: the row times a power of two, its largest magnitude in [2^15, 2^16) (65280 at most).  So values down to 2^-32 of the largest keep their bits; below, they are
                // rounded to multiples of 2^-24, 2^-39 of it.
                uint32_t top = 0;
#pragma unroll
                for (int k = 0; k < STEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i) top = max(top, max(qf[nt][k][i] & 0x7fffu, qf[nt][k][i] >> 16 & 0x7fffu));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                const int e = min(max((int)(top >> 7), 16), 254);          // (rows below 2^-111 and those with infinities: as near as a normal power gets)
                const float down = power_of_two(142 - e);
                back = e - 142;
#pragma unroll
                for (int k = 0; k < STEPS; ++k)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
                        qf[nt][k][i] = pack<false>(__uint_as_float(qf[nt][k][i] << 16) * down, __uint_as_float(qf[nt][k][i] & 0xffff0000u) * down);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                // (lane 8 t + 4 j holds column 2 t + j)
                [[maybe_unused]] const int power = max(a.power + __shfl_sync(0xffffffffu, back, 8 * t + 4 * j), -252), half = power >> 1;
                // Scale, factor and power of two, in an order that leaves the range only where their product does, and kept to normal numbers, as a masked place is -inf times it.
                // (Below them every score of the row vanishes, above them only the largest counts, with this product as with the true one.)
                if constexpr (FMT == ELUTQ_KV_16) cs[nt][j] = a.scale;
                else cs[nt][j] = fminf(fmaxf(a.part * kf * power_of_two(half) * power_of_two(power - half), 1.17549435e-38f), 3.40282347e38f);
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

        // 16 tokens at a time, NVFP4 a stage's 32 (the vote on the maximum and its like are then paid for once: 64 sequences of 4 to 16 K tokens 186 -> 169 us)
        constexpr int U = SCALED ? SUB : 1, TURN = SUB / U;
        int slot = 0;
        for (int n = 0; n < mine * TURN; ++n) {
            if (n % TURN == 0) {
                asm volatile("cp.async.wait_group %0;" :: "n"(S - 1) : "memory");
                __syncwarp();
            }
            const int tok0 = tile0 * TT + 16 * U * n;
            const uint32_t at = slot * STAGE + n % TURN * 16 * U * ROW;
            [[maybe_unused]] const uint8_t* scales = own + slot * STAGE;
            // ---- scores ----------------------------------------------------------------------------------------------------------------------
            float sc[U][NT][4];
            auto product = [&](int u, int step, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
                    if (step == 0) mma_first<BF16>(sc[u][nt], a0, a1, a2, a3, qf[nt][step][0], qf[nt][step][1]);
                    else mma<BF16>(sc[u][nt], a0, a1, a2, a3, qf[nt][step][0], qf[nt][step][1]);
            };
            if constexpr (FMT == ELUTQ_KV_16) {
#pragma unroll
                for (int k = 0; k < STEPS; ++k) {
                    uint32_t x[4];
                    read_matrices<false>(x, ring + at + (k_read ^ (k * 32)));
                    product(0, k, x[0], x[1], x[2], x[3]);
                }
            } else {
                uint32_t kr[U][2][KW];
                [[maybe_unused]] uint32_t blk[U][2];          // [row]: the scales of this lane's blocks
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
#pragma unroll
                        for (int i = 0; i < KW / KC; ++i) read_shared<4 * KC>(&kr[u][r][i * KC], own + ((k_read ^ (i * 64)) + at + (16 * u + 8 * r) * ROW));
                        if constexpr (SCALED) {
                            const uint8_t* p = scales + KS0 + (g + 16 * u + 8 * r) * (D / 16);
                            blk[u][r] = e4m3_pair(D == 128 ? (uint32_t)reinterpret_cast<const uint16_t*>(p)[t] : (uint32_t)p[t]);
                        }
                    }
#pragma unroll
                for (int w = 0; w < KW; ++w)                  // a word of both rows: PER_WORD / 4 steps
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        uint32_t x[2][PER_WORD / 2];
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            if constexpr (FMT == ELUTQ_KV_E4M3) {
                                e4m3_pairs(x[r], kr[u][r][w]);
                            } else {
                                const uint32_t scale = prmt(blk[u][r], blk[u][r], w < 2 ? 0x1010 : 0x3232);
                                e2m1_pairs(x[r], kr[u][r][w]);
#pragma unroll
                                for (int i = 0; i < 4; ++i) x[r][i] = hmul2(x[r][i], scale);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < PER_WORD / 4; ++i) product(u, w * (PER_WORD / 4) + i, x[0][2 * i], x[1][2 * i], x[0][2 * i + 1], x[1][2 * i + 1]);
                    }
            }
            const bool last = tok0 + 16 * U > least;              // some column may not see all of them
            if (last || gone != 0) {
                const uint32_t none = gone >> (slot * SUB + n % TURN * U);
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (tok0 + 16 * u + g + 8 * (i >> 1) >= limit[nt][i & 1] || (none >> u & 1u)) sc[u][nt][i] = -INFINITY;
            }
            // ---- softmax: P of these tokens --------------------------------------------------------------------------------------------------------
            float top[NT][2];
            bool rises = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    top[nt][j] = fmaxf(sc[0][nt][j], sc[0][nt][j + 2]);
#pragma unroll
                    for (int u = 1; u < U; ++u) top[nt][j] = fmaxf(top[nt][j], fmaxf(sc[u][nt][j], sc[u][nt][j + 2]));
                    rises |= __fmul_rn(top[nt][j], cs[nt][j]) + off[nt][j] > most;
                }
            if (__any_sync(0xffffffffu, rises)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float x = top[nt][j];
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, d));
                        const float to = x == -INFINITY ? off[nt][j] : fminf(off[nt][j], most - kLag - __fmul_rn(x, cs[nt][j]));
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
            uint32_t pf[U][NT][2];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float p[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        // (not fused: the offset comes from a rounded product, and where products are large the difference of the two would be anything)
                        p[i] = exp2_approx(__fmul_rn(sc[u][nt][i], cs[nt][i & 1]) + off[nt][i & 1]);
                        sum[nt][i & 1] += p[i];
                    }
                    pf[u][nt][0] = transposed(pack<BF16>(p[0], p[1]));
                    pf[u][nt][1] = transposed(pack<BF16>(p[2], p[3]));
                }
            // ---- P V: fragments of V rows, and what is done with each of them (a tile of 16 dimensions of the result) -----------------------------------------------
            // 16 bits: dimensions 16 m + g and 8 more.  Codes: V rows 2 t, 2 t + 1, 2 t + 8, 2 t + 9; tile m has dimensions 2 m and 2 m + 1 of this lane's, the two tokens of a pair side by
            // side.  They are brought there before they are converted.
            auto with_v = [&](int u, auto&& use) {
                if constexpr (FMT == ELUTQ_KV_16) {
#pragma unroll
                    for (int m = 0; m < STEPS; ++m) {
                        uint32_t x[4];
                        read_matrices<true>(x, ring + at + (v_read ^ (m * 32)));
                        use(m, x[0], x[1], x[2], x[3]);
                    }
                } else {
                    uint32_t vr[4][VW];
                    [[maybe_unused]] uint32_t vsc[2];
#pragma unroll
                    for (int r = 0; r < 4; ++r)
#pragma unroll
                        for (int i = 0; i < VW / VC; ++i) read_shared<4 * VC>(&vr[r][i * VC], own + (v_read + at + (16 * u + (r & 1) + 8 * (r >> 1)) * ROW + i * 128));
                    if constexpr (SCALED) {
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const uint8_t* q = scales + VS0 + (16 * u + 2 * t + 8 * p) * (D / 16) + (D == 128 ? g : g / 2);
                            vsc[p] = e4m3_pair((uint32_t)q[0] | (uint32_t)q[D / 16] << 8);
                        }
                    }
                    constexpr int MS = FMT == ELUTQ_KV_E4M3 ? 2 : 4;           // tiles of the result from a word of the four rows
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        uint32_t x[MS][4];
#pragma unroll
                        for (int p = 0; p < 2; ++p) {
                            const uint32_t v0 = vr[2 * p][w], v1 = vr[2 * p + 1][w];
                            if constexpr (FMT == ELUTQ_KV_E4M3) {
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    uint32_t h[2];
                                    e4m3_pairs(h, prmt(v0, v1, i == 0 ? 0x5140 : 0x7362));
                                    x[i][2 * p] = h[0];
                                    x[i][2 * p + 1] = h[1];
                                }
                            } else {
                                uint32_t lo[4], hi[4];
                                e2m1_pairs(lo, (v0 & 0x0f0f0f0fu) | (v1 << 4 & 0xf0f0f0f0u));
                                e2m1_pairs(hi, (v0 >> 4 & 0x0f0f0f0fu) | (v1 & 0xf0f0f0f0u));
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    x[i][2 * p] = hmul2(lo[i], vsc[p]);
                                    x[i][2 * p + 1] = hmul2(hi[i], vsc[p]);
                                }
                            }
                        }
#pragma unroll
                        for (int i = 0; i < MS; ++i) use(w * MS + i, x[i][0], x[i][1], x[i][2], x[i][3]);
                    }
                }
            };
            if (!last || a.fresh == 1) {
#pragma unroll
                for (int u = 0; u < U; ++u)
                    with_v(u, [&](int m, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma<BF16>(o[m][nt], x0, x1, x2, x3, pf[u][nt][0], pf[u][nt][1]);
                    });
            } else {
                // each new token's columns by themselves, with V rows that it does not see replaced by zeros
                const int first = rt * NC / a.group, end = min(a.fresh, (rt * NC + NC - 1) / a.group + 1);
                for (int nw = first; nw < end; ++nw)
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int sees = least + nw, tok = tok0 + 16 * u + 2 * t;
                        const uint32_t lo = (tok < sees ? 0xffffu : 0u) | (tok + 1 < sees ? 0xffff0000u : 0u);
                        const uint32_t hi = (tok + 8 < sees ? 0xffffu : 0u) | (tok + 9 < sees ? 0xffff0000u : 0u);
                        with_v(u, [&](int m, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                float part[4];
                                mma_first<BF16>(part, x0 & lo, x1 & lo, x2 & hi, x3 & hi, pf[u][nt][0], pf[u][nt][1]);
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    if (limit[nt][i & 1] == sees) o[m][nt][i] += part[i];
                            }
                        });
                    }
            }
            if (n % TURN == TURN - 1) {
                __syncwarp();
                if (n / TURN + S < mine) copy(n / TURN + S, slot);
                commit();
                slot = slot + 1 == S ? 0 : slot + 1;
            }
        }

        // ---- the end of a segment, or of the share ------------------------------------------------------------------------------------------------------
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum[nt][j] += __shfl_xor_sync(0xffffffffu, sum[nt][j], d);
        // this lane's two dimensions of tile m of the result: the first, and how far the other one is
        constexpr int APART = FMT == ELUTQ_KV_16 ? 8 : 1;
        auto dim_of = [&](int m) {
            constexpr int PIECE = VC * PER_WORD;
            return FMT == ELUTQ_KV_16 ? 16 * m + g : PIECE * (g + 8 * (2 * m / PIECE)) + 2 * m % PIECE;
        };
        auto put = [&](float* row, int m, float x, float y) {
            if constexpr (APART == 1) {
                *reinterpret_cast<float2*>(row + dim_of(m)) = make_float2(x, y);
            } else {
                row[dim_of(m)] = x;
                row[dim_of(m) + APART] = y;
            }
        };
        auto part_of = [&](int w, int place) { return a.parts + ((long long)w * 2 + place) * (NC * (D + 2)); };
        // The segment begins in worker w's share and ends in another's.  Its other parts: of `near` workers behind w in this CTA, one of each of `whole` CTAs that have units of no
        // other segment, and of the first `last` workers of the CTA behind those.
        auto record = [&](int w) {
            const int end = (int)quotient_of(seg0 + units - 1, share), cta = end / kWarps;
            const long long stop = (long long)(cta + 1) * kWarps * share;
            const bool all = (stop < total ? stop : total) <= seg0 + units;        // the last CTA has units of no other segment
            const int near = joint ? 0 : min(end, blockIdx.x * kWarps + kWarps - 1) - w;
            const int whole = cta > blockIdx.x ? cta - blockIdx.x - (all ? 0 : 1) : 0, last = cta > blockIdx.x && !all ? end - cta * kWarps + 1 : 0;
            a.begun[a.by_segment ? b * each + seg : w] = make_int4(b, seg, w, 1 + (near << 1) + (last << 3) + (whole << 6));
        };
        const float vf = a.c.vf == nullptr ? 1.0f : __ldg(a.c.vf + h);
        if (!joint) {
            const bool begins = tile0 == 0, whole = begins && mine == tiles;
            float* part = part_of(worker, begins ? 1 : 0);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = nt * 8 + 2 * t + j, rr = rt * NC + col;
                    if (rr >= a.rows) continue;
                    if (whole) {
                        const float r = sum[nt][j] == 0.0f ? 0.0f : vf / sum[nt][j];
                        const int tok = rr / a.group, head = h * a.group + (rr - tok * a.group);
                        uint8_t* p = a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D);
#pragma unroll
                        for (int m = 0; m < STEPS; ++m) {
                            const float x = o[m][nt][j] * r, y = o[m][nt][j + 2] * r;
                            const uint32_t two = a.type == ELUTQ_TYPE_F16 ? pack<false>(x, y) : pack<true>(x, y);
                            if constexpr (APART == 1) {
                                *reinterpret_cast<uint32_t*>(p + 2 * dim_of(m)) = two;
                            } else {
                                reinterpret_cast<uint16_t*>(p)[dim_of(m)] = (uint16_t)two;
                                reinterpret_cast<uint16_t*>(p)[dim_of(m) + APART] = (uint16_t)(two >> 16);
                            }
                        }
                    } else {
                        if (g == 0) {
                            part[col] = off[nt][j];
                            part[NC + col] = sum[nt][j];
                        }
#pragma unroll
                        for (int m = 0; m < STEPS; ++m) put(part + 2 * NC + col * D, m, o[m][nt][j], o[m][nt][j + 2]);
                    }
                }
            if (begins && !whole) {
                if (lane == 0) record(worker);
                recorded = true;
            }
            if (whole && a.by_segment && lane == 0) a.begun[b * each + seg] = make_int4(0, 0, 0, 0);
            f += unit1 - unit0;
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int col = nt * 8 + 2 * t + j;
                if (g == 0) {
                    s_off[warp][col] = off[nt][j];
                    s_sum[warp][col] = sum[nt][j];
                }
#pragma unroll
                for (int m = 0; m < STEPS; ++m) put(s_o[warp][col], m, o[m][nt][j], o[m][nt][j + 2]);
            }
        __syncthreads();
        const int used = min(NC, a.rows - rt * NC);
        if (a.split > 1) {
            // the CTAs' parts meet in distributed shared memory: each CTA sums up its warps', and then a share of the values over all CTAs
            for (int i = tid; i < used * (D / 2); i += kThreads) {
                const int col = i / (D / 2), d = 2 * (i - col * (D / 2));
                float low = kNone;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) low = fminf(low, s_off[w][col]);
                float all = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float by = exp2_approx(low - s_off[w][col]);
                    const float2 v = *reinterpret_cast<const float2*>(&s_o[w][col][d]);
                    all = fmaf(s_sum[w][col], by, all);
                    x = fmaf(v.x, by, x);
                    y = fmaf(v.y, by, y);
                }
                *reinterpret_cast<float2*>(&s_o[0][col][d]) = make_float2(x, y);
                if (d == 0) {
                    s_all[0][col] = low;
                    s_all[1][col] = all;
                }
            }
            cluster_barrier();
            const int rank = blockIdx.x % a.split;
            for (int i = tid * a.split + rank; i < used * (D / 2); i += kThreads * a.split) {
                const int col = i / (D / 2), d = 2 * (i - col * (D / 2));
                float lows[8], sums[8], xs[8], ys[8], low = kNone;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    lows[r] = kNone;
                    sums[r] = xs[r] = ys[r] = 0.0f;
                    if (r < a.split) {
                        lows[r] = ld_cluster_f32(&s_all[0][col], r);
                        sums[r] = ld_cluster_f32(&s_all[1][col], r);
                        xs[r] = ld_cluster_f32(&s_o[0][col][d], r);
                        ys[r] = ld_cluster_f32(&s_o[0][col][d + 1], r);
                    }
                }
#pragma unroll
                for (int r = 0; r < 8; ++r) low = fminf(low, lows[r]);
                float all = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const float by = exp2_approx(low - lows[r]);
                    all = fmaf(sums[r], by, all);
                    x = fmaf(xs[r], by, x);
                    y = fmaf(ys[r], by, y);
                }
                const float r = all == 0.0f ? 0.0f : vf / all;
                const int rr = rt * NC + col, tok = rr / a.group, head = h * a.group + (rr - tok * a.group);
                uint8_t* p = a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D + d);
                *reinterpret_cast<uint32_t*>(p) = a.type == ELUTQ_TYPE_F16 ? pack<false>(x * r, y * r) : pack<true>(x * r, y * r);
            }
            cluster_barrier();                                // (nobody leaves while its memory is read)
            return;
        }
        const bool begins = a.split != 0 || cta0 <= seg0 + kLead, whole = begins && (a.split != 0 || cta1 >= seg0 + units);
        if (whole || cta1 > seg0 + kLead) {                   // (there are tiles)
            const int first = !whole && begins ? (int)quotient_of(seg0 + kLead, share) : blockIdx.x * kWarps;      // the worker whose part it is
            float* part = part_of(first, begins ? 1 : 0);
            for (int i = tid; i < used * (D / 2); i += kThreads) {
                const int col = i / (D / 2), d = 2 * (i - col * (D / 2));
                float low = kNone;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) low = fminf(low, s_off[w][col]);
                float all = 0.0f, x = 0.0f, y = 0.0f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const float by = exp2_approx(low - s_off[w][col]);
                    const float2 v = *reinterpret_cast<const float2*>(&s_o[w][col][d]);
                    all = fmaf(s_sum[w][col], by, all);
                    x = fmaf(v.x, by, x);
                    y = fmaf(v.y, by, y);
                }
                if (whole) {
                    const float r = all == 0.0f ? 0.0f : vf / all;
                    const int rr = rt * NC + col, tok = rr / a.group, head = h * a.group + (rr - tok * a.group);
                    uint8_t* p = a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D + d);
                    *reinterpret_cast<uint32_t*>(p) = a.type == ELUTQ_TYPE_F16 ? pack<false>(x * r, y * r) : pack<true>(x * r, y * r);
                } else {
                    if (d == 0) {
                        part[col] = low;
                        part[NC + col] = all;
                    }
                    *reinterpret_cast<float2*>(part + 2 * NC + col * D + d) = make_float2(x, y);
                }
            }
            if (begins && !whole && worker == first) {
                if (lane == 0) record(worker);
                recorded = true;
            }
            if (whole && a.by_segment && a.split == 0 && tid == 0) a.begun[b * each + seg] = make_int4(0, 0, 0, 0);
        }
        break;
    }
    if (lane == 0 && !recorded && !a.by_segment && a.split == 0) a.begun[worker] = make_int4(0, 0, 0, 0);
}

// Joins the parts of the segments that several shares hold, in their order.  A block for each segment, or for each share in which one may begin, and for `cols` query rows: a warp to a
// row and to every `split`-th part, a lane to D / 32 dimensions; `split` warps join through shared memory.
template <int D, int NT>
__global__ void __launch_bounds__(256) attn_join_kernel(const DecodeArgs a, int split) {
    constexpr int NC = 8 * NT, SIZE = NC * (D + 2), W = D / 32;
    __shared__ float s_low[8], s_sum[8], s_x[8][D];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, cols = 8 / split;
    grid_dependency_wait();
    grid_launch_dependents();
    const int4 seg = a.begun[blockIdx.x];                     // sequence, key head and tile of rows, worker, where its parts are
    const int b = seg.x, h = seg.y / a.row_tiles, rt = seg.y - h * a.row_tiles, worker = seg.z, near = seg.w >> 1 & 3, whole = seg.w >> 6, parts = seg.w == 0 ? 0 : 1 + near + whole + (seg.w >> 3 & 7);
    const int col = blockIdx.y * cols + warp / split, row = rt * NC + col, first = warp % split;
    if (parts == 0) return;                                   // (the whole block)
    const bool some = col < NC && row < a.rows;
    // part 0 is the share's second place, the others are first places
    auto part_of = [&](int i) {
        const int cta = worker / kWarps, w = i <= near ? worker + i : i <= near + whole ? (cta + i - near) * kWarps : (cta + whole + 1) * kWarps + (i - near - whole - 1);
        return a.parts + ((long long)w * 2 + (i == 0 ? 1 : 0)) * SIZE;
    };
    float low = kNone, sum = 0.0f, x[W];
#pragma unroll
    for (int i = 0; i < W; ++i) x[i] = 0.0f;
    if (some) {
        for (int i0 = first; i0 < parts; i0 += 4 * split) {   // four parts on their way
            float off[4], s[4], v[4][W];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int i = i0 + k * split;
                off[k] = kNone;
                s[k] = 0.0f;
#pragma unroll
                for (int e = 0; e < W; ++e) v[k][e] = 0.0f;
                if (i < parts) {
                    const float* p = part_of(i);
                    off[k] = p[col];
                    s[k] = p[NC + col];
#pragma unroll
                    for (int e = 0; e < W / 2; ++e) {
                        const float2 two = *reinterpret_cast<const float2*>(p + 2 * NC + col * D + lane * W + 2 * e);
                        v[k][2 * e] = two.x;
                        v[k][2 * e + 1] = two.y;
                    }
                }
            }
            const float to = fminf(fminf(fminf(off[0], off[1]), fminf(off[2], off[3])), low), by = exp2_approx(to - low);
            low = to;
            sum *= by;
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] *= by;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float w = exp2_approx(to - off[k]);
                sum = fmaf(s[k], w, sum);
#pragma unroll
                for (int e = 0; e < W; ++e) x[e] = fmaf(v[k][e], w, x[e]);
            }
        }
    }
    if (split > 1) {
        if (lane == 0) {
            s_low[warp] = low;
            s_sum[warp] = sum;
        }
#pragma unroll
        for (int e = 0; e < W; ++e) s_x[warp][lane * W + e] = x[e];
        __syncthreads();
        if (first != 0) return;
        for (int w = warp + 1; w < warp + split; ++w) {
            const float to = fminf(low, s_low[w]), mine = exp2_approx(to - low), other = exp2_approx(to - s_low[w]);
            low = to;
            sum = fmaf(s_sum[w], other, sum * mine);
#pragma unroll
            for (int e = 0; e < W; ++e) x[e] = fmaf(s_x[w][lane * W + e], other, x[e] * mine);
        }
    }
    if (!some) return;
    const float r = sum == 0.0f ? 0.0f : (a.c.vf == nullptr ? 1.0f : __ldg(a.c.vf + h)) / sum;
    const int tok = row / a.group, head = h * a.group + (row - tok * a.group);
    uint32_t* out = reinterpret_cast<uint32_t*>(a.out + 2 * (((long long)b * a.fresh + tok) * a.ldo + (long long)head * D)) + lane * (W / 2);
#pragma unroll
    for (int e = 0; e < W / 2; ++e) out[e] = a.type == ELUTQ_TYPE_F16 ? pack<false>(x[2 * e] * r, x[2 * e + 1] * r) : pack<true>(x[2 * e] * r, x[2 * e + 1] * r);
}

// CTAs of a launch: as many as are resident at once
inline int ctas_of(int per_sm) { return device_sm_count() * per_sm; }
inline int columns_of(int rows) { return rows <= 8 ? 1 : 2; }

int launch_one(const void* kernel, dim3 grid, int block, int smem, void** args, cudaStream_t stream, int cluster = 1) {
    cudaLaunchConfig_t cfg = {};
    cfg.dynamicSmemBytes = smem;
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)block);
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelExC(&cfg, kernel, args);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}

// Short sequences: a cluster of CTAs for each segment, joined in distributed shared memory, one launch instead of two.  How long they are only the device knows; the table says how
// long they may be.  A warp takes up to 128 tokens that way, and 256 where the clusters take more than half of the CTAs that are resident at once, so that shares of
// the whole would not be much shorter.  Measured with 8 key heads (us, clusters : shares of the whole): 1 x 1000 NVFP4 6.9 : 9.3, 8 x 2000 NVFP4 11.3 : 13.7, 16 x 2000 NVFP4 16.1 :
// 19.2, 4 x 8000 16 bits 27.5 : 29.8, 64 x 500 16 bits 28.6 : 29.3, 128 x 700 16 bits 61 : 66, 100 x 1000 E4M3 41.0 : 44.9, at worst 64 x 1000 NVFP4 29.4 : 28.1; not
// taken: 1 x 8000 16 bits 14.9 : 12.7, and 64 clusters of 8, more than are resident at once, 19.5 : 13.2.
int split_of(long long segments, long long cap, int ctas) {
    if (segments > 0xffffff) return 0;
    int split = 1;
    while (split < 8 && 2 * split * segments <= ctas && split * kWarps * 16 < cap) split *= 2;
    const bool most = 2 * split * segments > ctas;
    return cap <= split * kWarps * kShortTokens * (most ? 2 : 1) ? split : 0;
}

// What a call of a shape is: columns of a tile of query rows (in eights), CTAs that are resident at once, CTAs of a cluster (0: shares of the whole), bytes of workspace
struct Plan {
    int nt, per, ctas, split;
    size_t bytes;
};
Plan plan_of(const elutq_kv_cache* c, int pages, int B, int new_tokens, int n_q_heads) {
    Plan p;
    const int rows = n_q_heads / c->heads * new_tokens;
    p.nt = columns_of(rows);
    p.per = resident(c->format, c->head_dim, p.nt);
    p.ctas = ctas_of(p.per);
    const long long cap = (long long)pages * c->page_size;
    const long long segments = (long long)B * c->heads * ((rows + 8 * p.nt - 1) / (8 * p.nt));
    p.split = split_of(segments, cap < kMostTokens ? cap : kMostTokens, p.ctas);
    // A round of three CTAs to an SM takes about 4/3 of one of two.  NVFP4, 8 key heads, dimension 128, us, two : three: 50 x 900 tokens (400 segments) 23.4 : 19.3, 64 x 1000 26.8 :
    // 30.2, 256 x 300 46.3 : 40.8, 300 x 700 71.5 : 63.4.  Fewer CTAs, or shares: two (30 x 1000 14.0 : 17.8, 4 x 30000 36.1 : 40.2, 128 x 4000 88.0 : 90.9).  Dimension 64 with 12 query
    // rows to a key head: 50 x 900 25.8 : 17.5, 64 x 1000 29.6 : 31.4, 256 x 300 58.5 : 48.3, 300 x 700 98.8 : 78.0, 30 x 1000 14.1 : 16.9; at worst, where the two are
    // even by this count, 120 x 500 38.3 : 33.0 (two).
    if (either(c->format, c->head_dim, p.nt) && p.split == 1) {
        const long long two = device_sm_count() * 2, three = device_sm_count() * 3;
        if (4 * ((segments + three - 1) / three) < 3 * ((segments + two - 1) / two)) p.per = 3;
    }
    p.bytes = p.split != 0 ? 0 : (size_t)p.ctas * kWarps * (2 * (8 * p.nt) * (c->head_dim + 2) * sizeof(float) + sizeof(int4));
    return p;
}

template <int D, int FMT, bool BF16, int NT, int PER>
int launch_decode(DecodeArgs a, const Plan& plan, cudaStream_t stream) {
    constexpr int kRings = kWarps * stages_of(FMT, D) * stage_bytes(FMT, D), kParts = kWarps * 8 * NT * (D + 4) * 4, kSmem = kRings > kParts ? kRings : kParts;
    // once for each device (a call would take half a microsecond of the host's time)
    static std::atomic<unsigned long long> ready{0};
    int dev = 0;
    cudaError_t ce = cudaGetDevice(&dev);
    if (ce != cudaSuccess) return (int)ce;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(ready.load(std::memory_order_acquire) & bit)) {
        ce = cudaFuncSetAttribute(attn_decode_kernel<D, FMT, BF16, NT, PER>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (ce != cudaSuccess) return (int)ce;
        ready.fetch_or(bit, std::memory_order_release);
    }
    const int ctas = plan.ctas;
    const long long segments = (long long)a.B * a.c.heads * a.row_tiles;
    a.by_segment = segments <= ctas * kWarps;
    a.split = plan.split;
    if (a.split != 0) {
        void* args[] = {&a};
        return launch_one((const void*)attn_decode_kernel<D, FMT, BF16, NT, PER>, dim3((unsigned)(segments * a.split)), kThreads, kSmem, args, stream, a.split);
    }
    void* args[] = {&a};
    const int e = launch_one((const void*)attn_decode_kernel<D, FMT, BF16, NT, PER>, dim3(ctas), kThreads, kSmem, args, stream);
    if (e != 0) return e;
    // few segments have many parts each: more warps to a row
    const long long parts = ctas / segments;
    int split = parts >= 32 ? 8 : parts >= 8 ? 4 : parts >= 4 ? 2 : 1;
    void* join[] = {&a, &split};
    const int cols = 8 / split, wide = a.rows < 8 * NT ? a.rows : 8 * NT;
    return launch_one((const void*)attn_join_kernel<D, NT>, dim3(a.by_segment ? (unsigned)segments : ctas * kWarps, (wide + cols - 1) / cols), 256, 0, join, stream);
}
template <int D, int FMT, bool BF16, int NT>
int launch_decode(const DecodeArgs& a, const Plan& plan, cudaStream_t stream) {
    constexpr int PER = resident(FMT, D, NT);
    if constexpr (either(FMT, D, NT)) {
        if (plan.per == 3) return launch_decode<D, FMT, BF16, NT, 3>(a, plan, stream);
    }
    return launch_decode<D, FMT, BF16, NT, PER>(a, plan, stream);
}
template <int D, int FMT, bool BF16>
int launch_decode(const DecodeArgs& a, const Plan& plan, cudaStream_t stream) {
    return plan.nt == 1 ? launch_decode<D, FMT, BF16, 1>(a, plan, stream) : launch_decode<D, FMT, BF16, 2>(a, plan, stream);
}
template <int D>
int launch_decode(const DecodeArgs& a, int format, const Plan& plan, cudaStream_t stream) {
    if (format == ELUTQ_KV_16) return a.type == ELUTQ_TYPE_BF16 ? launch_decode<D, ELUTQ_KV_16, true>(a, plan, stream) : launch_decode<D, ELUTQ_KV_16, false>(a, plan, stream);
    return format == ELUTQ_KV_E4M3 ? launch_decode<D, ELUTQ_KV_E4M3, false>(a, plan, stream) : launch_decode<D, ELUTQ_KV_NVFP4, false>(a, plan, stream);
}

// The arguments that the size of the workspace hangs on, too
int check_sizes(const elutq_kv_cache* c, int pages, int B, int new_tokens, int n_q_heads) {
    const int st = kv_check(c);
    if (st != ELUTQ_OK) return st;
    if (pages <= 0 || B <= 0 || new_tokens <= 0 || n_q_heads <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (n_q_heads % c->heads != 0 || (long long)n_q_heads / c->heads * new_tokens > 0xffff || (long long)B * n_q_heads * new_tokens > 0x7fffffffLL) return ELUTQ_ERR_SHAPE;
    return ELUTQ_OK;
}

}  // namespace

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_attn_decode_workspace_bytes(const elutq_kv_cache* cache, int pages, int B, int new_tokens, int n_q_heads, size_t* bytes) {
    if (!bytes) return ELUTQ_ERR_INVALID_ARG;
    const int st = check_sizes(cache, pages, B, new_tokens, n_q_heads);
    if (st == ELUTQ_OK) *bytes = plan_of(cache, pages, B, new_tokens, n_q_heads).bytes;
    return st;
}

extern "C" int elutq_attn_decode(const elutq_kv_cache* cache, const void* q, long long ldq, void* out, long long ldo, const int* table, long long ld_table, int pages,
                                 const int* lens, int B, int new_tokens, int n_q_heads, float scale, void* workspace, size_t workspace_bytes, void* stream) {
    int st = check_sizes(cache, pages, B, new_tokens, n_q_heads);
    if (st != ELUTQ_OK) return st;
    if (!q || !out || out == q || !table || !lens) return ELUTQ_ERR_INVALID_ARG;
    if (!(scale > 0.0f) || !(scale < 1e30f)) return ELUTQ_ERR_INVALID_ARG;
    const int D = cache->head_dim, H = cache->heads;
    const Plan plan = plan_of(cache, pages, B, new_tokens, n_q_heads);
    if (plan.bytes != 0 && !workspace) return ELUTQ_ERR_INVALID_ARG;
    if (ld_table < pages) return ELUTQ_ERR_SHAPE;
    if ((st = kv_rows_check(q, ldq, n_q_heads, D)) != ELUTQ_OK || (st = kv_rows_check(out, ldo, n_q_heads, D)) != ELUTQ_OK) return st;
    if (!mx4_aligned(table, 4) || !mx4_aligned(lens, 4) || !mx4_aligned(workspace, 16)) return ELUTQ_ERR_ALIGN;
    if (workspace_bytes < plan.bytes) return ELUTQ_ERR_BUFFER_TOO_SMALL;
    const long long rows = (long long)B * new_tokens;
    if (rows_meet({q, ldq, rows, n_q_heads}, {out, ldo, rows, n_q_heads}, D)) return ELUTQ_ERR_INVALID_ARG;
    DecodeArgs a;
    a.c = kv_view(cache);
    a.q = (const uint8_t*)q;
    a.out = (uint8_t*)out;
    a.ldq = ldq; a.ldo = ldo;
    a.table = table; a.lens = lens;
    a.ld_table = ld_table;
    a.B = B;
    a.fresh = new_tokens;
    a.group = n_q_heads / H;
    a.rows = a.group * new_tokens;
    const int nc = 8 * plan.nt;
    a.row_tiles = (a.rows + nc - 1) / nc;
    a.type = cache->type;
    a.scale = scale * 1.44269504088896340736f;
    a.part = frexpf(a.scale, &a.power);
    a.begun = (int4*)workspace;
    a.parts = (float*)(a.begun + plan.ctas * kWarps);
    a.cap = (long long)pages * cache->page_size;
    if (a.cap > kMostTokens) a.cap = kMostTokens;
    const int ce = D == 128 ? launch_decode<128>(a, cache->format, plan, (cudaStream_t)stream) : launch_decode<64>(a, cache->format, plan, (cudaStream_t)stream);
    if (ce == 0) return ELUTQ_OK;
    note_cuda_error(ce);
    return ELUTQ_ERR_CUDA;
}
