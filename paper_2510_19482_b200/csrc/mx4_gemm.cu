// Products of microscaled 4-bit matrices, dense and grouped by expert, on tcgen05.mma with block scales.
//
//   Y[t][n] = alpha_e * sum_k X[t][k] W_e[n][k],  rows t of group e (one group: a dense product)
//
// The tensor core takes both operands as codes and multiplies every product of two blocks by their two scales; sums are fp32.
//
//   tile       128 weight rows (256 by a pair of CTAs) x up to 256 tokens.  Weight rows are the MMA's M, lanes of tensor memory; tokens its
//              N, columns of tensor memory, 8 at least: a decoding batch wastes nothing but padding to 8, and a group's rest is as wide as it is.
//   K          in steps of 256: 128 bytes of codes a row, one 128-byte swizzle atom wide, brought by TMA into a ring of stages.
//   scales     are row-major, while the tensor core wants, per 128 rows and 4 scales, 512 bytes with row r's four at
//              16 (r mod 32) + 4 (r / 32): a warp per 128 rows loads and stores them so, four steps at a time.  The fence that makes
//              its stores visible to the tensor core also waits for its loads, so none of the next ones may be in flight: two warps
//              per 128 rows take turns, one loads while the other stores.  The MMA thread copies them to tensor memory
//              (tcgen05.cp) in front of a step's MMAs; copies and MMAs of one thread run in order.
//   sums       two accumulators; the epilogue warps empty one while the next tile fills the other.  256 tokens leave no room for
//              two beside the scales: they share 48 columns, which the epilogue empties first.
//   few tiles  a cluster of CTAs shares a tile's K; the parts meet in shared memory, each CTA adds up its share of the tokens in the
//              cluster's order and stores them.
//   tail       K: TMA fills codes with zeros, the scale warps scales.  Rows behind the last one of the matrix or the group: whatever is
//              there; a row of one operand only reaches its own row or column of the sums, and those are not stored.
//
// Every wait is bounded: the thread whose wait runs out raises the device's status word, and all roles leave their loops.
//
// Measured (one B200, us, weights from HBM): 1 x 6144 x 4096 MXFP4 7.0, 64 x 57344 x 8192 NVFP4 46 (5.9 TB/s; 54 in long runs at the
// power limit), 64 rows over 64 experts of 4096 x 2048 27 (DRAM reads 1.00 of the bytes there are), 4096 x 28672 x 4096 190 to 200 (4.8 to 5.1
// PFLOP/s; 227 in long runs).  Bound: latencies of a launch, HBM, or at many tokens power: a step of 256 k takes 675 to 710 cycles for 512 of
// MMAs, at a clock of 1.35 GHz in long runs (with all codes zero the same call takes 154 and 158 us; L2 is 46 % busy).
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "mx4.cuh"
#include "tensor_map.cuh"

namespace elutq {

namespace {

constexpr int kTileW = 128;                // weight rows of a CTA
constexpr int kMaxTokens = 256;            // tokens of a tile
constexpr int kStepBytes = 128;            // codes of a row in a step: 256 k
constexpr int kMaxStages = 10;
constexpr int kMaxSplit = 8;
// Tiles that a cluster may share.  Their sums take 512 bytes of shared memory a token, and the exchange grows with the tokens: 80 x 5120 x 13824 NVFP4 18.3 us
// up to 64 tokens, 16.1 up to 96; 128 x 4096 x 14336 MXFP4 15.0 up to 96, 18.2 up to 128.
constexpr int kMaxSplitTokens = 96;
constexpr int kMaxGroups = 1024;
// Scales come in turns of four steps into a ring of two, one fence and one arrival for a turn; the two warps of 128 rows take alternate turns.  (A warp waits
// for a use of the ring one turn ahead of the other's: within what a barrier's parity tells apart.)  A step at a time, three warps could not keep up with
// the MMAs, as the fence takes 400 to 1000 cycles (4096 x 28672 x 4096, MXFP4 203 us, NVFP4 246).
constexpr int kTurn = 4, kTurns = 2;
template <int NB>
constexpr int kThreads = 32 * (6 + (1 + NB) * 2);
// Columns of tensor memory: scales at the end (48 NVFP4, 24 MXFP4 for pairs), in front of them two accumulators.  Tiles of up to kApart tokens have both to themselves;
// higher ones share kShared columns of them.
template <int FMT>
constexpr int kScaleCols = FMT == ELUTQ_MX4_NVFP4 ? 464 : 488;
template <int FMT>
constexpr int kApart = kScaleCols<FMT> / 2 / 16 * 16;
constexpr int kShared = 48;
constexpr int kSmem = 232448;
constexpr int kChunk = kShared;            // columns that the epilogue takes at once
constexpr int kTurnBytes = 4 * kChunk * 64;      // 32 weight rows of them for each epilogue warp, 16 bits each
constexpr unsigned long long kWaitNs = 1000000000ull;
// A tile's results are waited for through all of its K: 2^20 steps of 0.24 to 0.3 us stay well below the limit of a wait.
constexpr int kMaxK = 1 << 28;

__device__ unsigned g_status;              // 0, or what a launch on this device gave up on

struct Mx4Args {
    const uint8_t *x_scales, *w_scales;
    const float* alpha;
    const int* offsets;        // null: one group of all rows
    void* Y;
    int y_type;
    int M, N, K, E;
    int sk;                    // scale bytes of a row
    int tokens;                // tokens of a tile at most
    int w_tiles;               // of a group
    int steps;                 // of the whole K
    int split;                 // CTAs that share a tile's K
    int stages;
    int x_box;                 // rows of one X load
    int once;                  // weights are read by one tile of tokens
    int turn;                  // the epilogue turns 16-bit results in shared memory
    int x_wide, w_wide;        // scales of a row start on 16 bytes
    int test;                  // 1: no load is issued
    uint32_t wait_limit;       // polls (tests); a wait of a second runs out whatever this is
};

enum { kBarFull = 0, kBarEmpty = kBarFull + kMaxStages, kBarScalesFull = kBarEmpty + kMaxStages, kBarScalesEmpty = kBarScalesFull + kTurns, kBarAccFull = kBarScalesEmpty + kTurns, kBarAccFree = kBarAccFull + 2,
       kBarPartsFull = kBarAccFree + 2, kBarPartsFree, kBarDrain, kNumBars };

__device__ __forceinline__ uint32_t at_rank(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// On a barrier of another CTA (a shared::cluster address).  arrive_cluster orders all accesses in front of it for the cluster, which waits for those to global
// memory too; arrive_remote only those to this CTA's shared memory, which is what a pair's scales need beside their proxy fence, and a pair's accumulators beside tcgen05's
// (with the former 4096 x 28672 x 4096 takes 276 us instead of 220; an arrival that orders nothing beyond the CTA would save less than 1 % more).
__device__ __forceinline__ void arrive_remote(uint32_t bar) {
    asm volatile("fence.release.sync_restrict::shared::cta.cluster;" ::: "memory");
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
// Polls until the phase is over (true), something in the CTA has given up, or the time or the polls are (false).  A poll may be suspended by
// the hardware for some tens of microseconds, so the time is what counts.
template <bool CLUSTER>
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity, volatile const uint32_t* gave_up, uint32_t limit) {
    if (try_wait<CLUSTER>(bar, parity)) return true;
    unsigned long long since = 0;
    for (uint32_t i = 1; i < limit; ++i) {
        if (try_wait<CLUSTER>(bar, parity)) return true;
        if ((i & 15u) == 0u) {
            if (gave_up != nullptr && *gave_up) return false;
            const unsigned long long t = now_ns();
            if (since == 0) since = t;
            else if (t - since > kWaitNs) return false;
        }
    }
    return false;
}
// The same by one thread, which says so when it gives up.  EARLY: it may have come here while the kernels in front still run, for as long as they like; the clock then
// starts again behind them.  (Waiting for them first costs 0.1 us a call.)
template <bool CLUSTER = false, bool EARLY = false>
__device__ __forceinline__ bool wait_alone(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t limit) {
    if (poll<CLUSTER>(bar, parity, gave_up, limit)) return true;
    if constexpr (EARLY) {
        grid_dependency_wait();
        if (poll<CLUSTER>(bar, parity, gave_up, limit)) return true;
    }
    *gave_up = 1;
    atomicExch(&g_status, kStatusWaitExpired);
    return false;
}
// By a whole warp, with one answer for it: false once anything in the CTA has given up.
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t limit) {
    const bool ok = poll<CLUSTER>(bar, parity, gave_up, limit);
    if (__all_sync(0xffffffffu, ok)) return true;
    if (!ok) {
        *gave_up = 1;
        atomicExch(&g_status, kStatusWaitExpired);
    }
    __syncwarp();
    return false;
}
// Whether `ok` holds in all epilogue warps (which pass their barrier).
__device__ __forceinline__ bool epilogue_agrees(bool ok) {
    uint32_t all;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.and.pred q, 1, 128, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(all) : "r"((uint32_t)ok) : "memory");
    return all != 0;
}

template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
template <int CG>
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar, uint64_t policy) {
    if constexpr (CG == 2)
        asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy) : "memory");
    else
        asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.L2::cache_hint [%0], [%1, {%2, %3}], [%4], %5;"
                     :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy) : "memory");
}
// K-major, 128-byte swizzle, 1024 bytes per 8 rows
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// 32 rows of 16 bytes, no swizzle: 128 bytes per 8 rows
__device__ __forceinline__ uint64_t scales_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(128u >> 4) << 32) | ((uint64_t)1 << 46);
}
template <int CG>
__device__ __forceinline__ void copy_scales(uint32_t taddr, uint64_t desc) {
    if constexpr (CG == 2) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" :: "r"(taddr), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" :: "r"(taddr), "l"(desc) : "memory");
}
template <int FMT, int CG>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    if constexpr (FMT == ELUTQ_MX4_MXFP4 && CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else if constexpr (FMT == ELUTQ_MX4_MXFP4)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::mxf4.block_scale.block32 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else if constexpr (CG == 1)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::mxf4nvf4.block_scale.block16 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::mxf4nvf4.block_scale.block16 [%0], %1, %2, %3, [%5], [%6], p;\n\t}"
                     :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
}
// One arrival on `bar` (of both CTAs of a pair) once all MMAs and copies issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" :: "r"(bar), "h"((uint16_t)3) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t (&r)[16], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
                   "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait(uint32_t (&r)[16]) {     // names the registers: nothing may use them earlier
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) :: "memory");
}

// 16 lanes of tensor memory x 16 columns, as fragments: a thread's registers 0 and 1 hold row lane / 4, columns 2 (lane mod 4) and one more, 2 and 3 the same of
// row lane / 4 + 8, 4 to 7 the same 8 columns on.
__device__ __forceinline__ void tmem_ld_fragments(uint32_t* r, uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void store_transposed(uint32_t saddr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" :: "r"(saddr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// A ring's stage and the parity of its use
struct Ring {
    int len, i = 0;
    uint32_t phase = 0;
    __device__ explicit Ring(int n) : len(n) {}
    __device__ void next() {
        if (++i == len) { i = 0; phase ^= 1u; }
    }
};

// The first and last scales of a matrix of any alignment are read as the aligned words around them; of the words that the matrix shares with its
// surroundings only the bytes that belong to it are.
struct Ends {
    const uint32_t *lo, *hi;       // whole words: [lo, hi)
    uint32_t head, tail;           // the words in front of lo and at hi
};
__device__ __forceinline__ Ends ends_of(const uint8_t* base, const uint8_t* end) {
    Ends e;
    e.lo = reinterpret_cast<const uint32_t*>((reinterpret_cast<uintptr_t>(base) + 3) & ~(uintptr_t)3);
    e.hi = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(end) & ~(uintptr_t)3);
    auto bytes_at = [&](const uint32_t* word) {
        uint32_t v = 0;
        for (int b = 0; b < 4; ++b) {
            const uint8_t* p = reinterpret_cast<const uint8_t*>(word) + b;
            if (p >= base && p < end) v |= (uint32_t)__ldg(p) << (8 * b);
        }
        return v;
    };
    e.head = bytes_at(e.lo - 1);
    e.tail = bytes_at(e.hi);
    return e;
}
// Four words of a row's scales from p on; bytes from `end` (of the row) on are 0.
__device__ __forceinline__ void load_words(uint32_t (&w)[4], const uint8_t* p, const uint8_t* end, const Ends& e) {
    const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(p) & 3);
    const uint32_t* q = reinterpret_cast<const uint32_t*>(p - off);
    uint32_t v[5];
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        v[i] = q + i == e.hi ? e.tail : q + i == e.lo - 1 ? e.head : 0u;
        if (q + i >= e.lo && q + i < e.hi) v[i] = __ldg(q + i);
    }
    const int left = (int)(end - p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = __funnelshift_r(v[i], v[i + 1], 8u * off);
        if (left < 4 * i + 4) w[i] &= left <= 4 * i ? 0u : (1u << (8 * (left - 4 * i))) - 1u;
    }
}

// The 16 bytes at q (aligned) if `some`, else 0.
__device__ __forceinline__ void load_piece(uint32_t (&w)[4], const uint8_t* q, bool some) {
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    if (some) v = __ldg(reinterpret_cast<const uint4*>(q));
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}

struct Tile {
    int e, n0, t0, count;      // group, first weight row in it, first token, tokens
};

// Where the groups' tiles begin in the list of all tiles: starts[E + 1], then the first row [E] and the number of rows [E] of each group.
// Borders out of order or out of range are cut to what is left of [0, M).
__device__ __forceinline__ void list_groups(const Mx4Args& a, int* table) {
    int* starts = table;
    int* first = table + a.E + 1;
    int* rows = first + a.E;
    const int lane = threadIdx.x & 31;
    int tiles = 0, border = 0;                  // of the groups before this turn
    for (int e0 = 0; e0 < a.E; e0 += 32) {
        const int e = e0 + lane;
        int lo = 0, hi = 0;
        if (e < a.E) {
            lo = min(max(__ldg(a.offsets + e), 0), a.M);
            hi = min(max(__ldg(a.offsets + e + 1), 0), a.M);
        }
        int most = hi;                          // the largest border so far
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, most, o);
            if (lane >= o) most = max(most, v);
        }
        most = max(most, border);
        int before = __shfl_up_sync(0xffffffffu, most, 1);
        if (lane == 0) before = border;
        lo = max(lo, before);
        const int n = max(hi - lo, 0);
        const int mine = (n + a.tokens - 1) / a.tokens * a.w_tiles;
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o *= 2) {
            const int v = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += v;
        }
        if (e < a.E) {
            starts[e] = tiles + sum - mine;
            first[e] = lo;
            rows[e] = n;
        }
        tiles += __shfl_sync(0xffffffffu, sum, 31);
        border = __shfl_sync(0xffffffffu, most, 31);
    }
    if (lane == 0) starts[a.E] = tiles;
}

// A group's rows are cut into as many tiles as they need, of nearly equal height (multiples of 8).  The token tiles of one block of
// weights are neighbours in the list: they run at the same time and read the weights from L2.
template <int CG>
__device__ __forceinline__ Tile tile_at(const Mx4Args& a, const int* table, int i) {
    Tile t;
    int rows = a.M, local = i;
    t.e = 0;
    t.t0 = 0;
    if (a.offsets != nullptr) {
        int lo = 0, hi = a.E;                   // starts[lo] <= i < starts[hi]
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (table[mid] <= i) lo = mid;
            else hi = mid;
        }
        t.e = lo;
        local = i - table[lo];
        t.t0 = table[a.E + 1 + lo];
        rows = table[2 * a.E + 1 + lo];
    }
    const int n = (rows + a.tokens - 1) / a.tokens;
    const int height = ((rows + n - 1) / n + 7) / 8 * 8;
    const int w = local / n, p = local - w * n;
    t.n0 = w * (CG * kTileW);
    t.t0 += p * height;
    t.count = min(height, rows - p * height);
    return t;
}

__device__ __forceinline__ void store_y(const Mx4Args& a, long long at, float v) {
    if (a.y_type == ELUTQ_TYPE_F16) reinterpret_cast<__half*>(a.Y)[at] = __float2half_rn(v);
    else if (a.y_type == ELUTQ_TYPE_BF16) reinterpret_cast<__nv_bfloat16*>(a.Y)[at] = __float2bfloat16_rn(v);
    else reinterpret_cast<float*>(a.Y)[at] = v;
}

// CG: CTAs of a pair; NB: blocks of 128 tokens in a tile at most (pairs: two).  Warps: 0 loads codes, 1 issues MMAs, 4 to 7 epilogue, 2, 3 and 8 on scales, kTurns for the weights, then
// for tokens 0 to 127, then for 128 to 255.
template <int FMT, int CG>
__global__ void __launch_bounds__(kThreads<CG>, 1) mx4_gemm_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const Mx4Args a) {
    constexpr int CH = FMT == ELUTQ_MX4_MXFP4 ? 2 : 4;            // groups of four scales in a step
    constexpr int NB = CG;
    const bool overlap = a.tokens > kApart<FMT>;
    const int acc1 = overlap ? kMaxTokens - kShared : kApart<FMT>;                      // the second accumulator
    constexpr int SUB = 4 / CH;                                   // MMAs (64 k) that share a group
    extern __shared__ __align__(1024) uint8_t smem[];
    const int x_bytes = (a.tokens / CG + 7) / 8 * 1024;           // of a stage
    const int w_bytes = kTileW * kStepBytes, s_bytes = (1 + NB) * CH * 512 + 32;      // (scales: of a step, and 32 bytes that move the next step's banks)
    uint8_t* sW = smem;
    uint8_t* sX = sW + a.stages * w_bytes;
    uint8_t* sS = sX + a.stages * x_bytes;
    float* parts = reinterpret_cast<float*>(sS + kTurns * kTurn * s_bytes);                 // [tokens][128], clusters only
    uint8_t* sT = reinterpret_cast<uint8_t*>(parts) + (a.split > 1 ? a.tokens * kTileW * 4 : 0);
    uint64_t* bars = reinterpret_cast<uint64_t*>(sT + (a.turn ? kTurnBytes : 0));
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    volatile uint32_t* gave_up = tmem_slot + 1;
    int* table = reinterpret_cast<int*>(tmem_slot + 2);
    const uint32_t bar0 = smem_u32(bars);
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    uint32_t rank = 0;                                            // in the cluster
    if (CG == 2 || a.split > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    const bool leader = CG == 1 || rank == 0;

    if (warp == 1) {
        if constexpr (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(tmem_slot)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(tmem_slot)) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
    }
    if (threadIdx.x == 0) {
        auto init = [&](int i, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar(i)), "r"(n) : "memory"); };
        for (int i = 0; i < a.stages; ++i) {
            init(kBarFull + i, 1);
            init(kBarEmpty + i, 1);
        }
        for (int i = 0; i < kTurns; ++i) {
            init(kBarScalesFull + i, CG * (1 + NB));
            init(kBarScalesEmpty + i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            init(kBarAccFull + i, 1);
            init(kBarAccFree + i, CG * 4);
        }
        init(kBarPartsFull, a.split);
        init(kBarPartsFree, a.split);
        init(kBarDrain, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        *gave_up = 0;
        asm volatile("prefetch.tensormap [%0];" :: "l"(&x_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&w_map) : "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2 || a.split > 1) cluster_barrier();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    // What reads or writes global memory waits for the kernels in front of this one: the groups' borders here, each role otherwise where it begins.  (The next
    // kernel may start once this one's loader has waited: kernels of this library that read weights ahead of their own wait rely on that.)
    if (a.offsets != nullptr) {
        if (warp == 0) {
            grid_dependency_wait();
            list_groups(a, table);
        }
        __syncthreads();
    }
    const uint32_t tmem = *tmem_slot;

    const int team = CG == 2 ? 2 : a.split;                       // CTAs that work on one tile
    const int first = blockIdx.x / team, stride = gridDim.x / team;
    const int tiles = a.offsets != nullptr ? table[a.E] : a.w_tiles * ((a.M + a.tokens - 1) / a.tokens);
    // this CTA's steps, in pairs
    const int pairs = (a.steps + 1) / 2;
    const int step0 = CG == 2 ? 0 : 2 * (int)((long long)pairs * rank / a.split);
    const int step1 = CG == 2 ? a.steps : min(a.steps, 2 * (int)((long long)pairs * (rank + 1) / a.split));
    const uint32_t limit = a.wait_limit;

    // One lane runs the whole loop of the loads and of the MMAs: with all of a warp in it and a choice at every step, the MMA
    // warp took 900 cycles a step of at least 512, half of them in waits that were over (4096 x 28672 x 4096, MXFP4: 224 us).
    if (warp == 0) {
        if (elect_one() && !a.test) {
            Ring r(a.stages);
            int issued = 0;
            bool ok = true;
            // Weights that one tile of tokens reads are not wanted again: their lines make room first (us without and with it: 64 x 57344 x 8192 NVFP4 51.2 and 46.4,
            // 64 experts of 4096 x 2048 with 64 rows 30.4 and 27.6, 1 x 28672 x 4096 14.8 and 14.1).  All other loads go without a policy: with one that says nothing
            // the experts took 31.9.
            uint64_t once;
            asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(once));
            grid_dependency_wait();
            grid_launch_dependents();
            for (int i = first; i < tiles && ok; i += stride) {
                const Tile t = tile_at<CG>(a, table, i);
                const int per_cta = CG == 2 ? (t.count + 15) / 16 * 8 : (t.count + 7) / 8 * 8;
                const int boxes = (per_cta + a.x_box - 1) / a.x_box;
                const int w_row = t.e * a.N + t.n0 + (CG == 2 ? (int)rank * kTileW : 0), x_row = t.t0 + (CG == 2 ? (int)rank * per_cta : 0);
                const uint32_t bytes = CG * (w_bytes + boxes * a.x_box * kStepBytes);
                for (int s = step0; s < step1; ++s) {
                    ok = wait_alone(bar(kBarEmpty + r.i), r.phase ^ 1u, gave_up, limit);
                    if (!ok) break;
                    const uint32_t full = CG == 2 ? at_rank(bar(kBarFull + r.i), 0) : bar(kBarFull + r.i);
                    if (leader) expect(bar(kBarFull + r.i), bytes);
                    if (a.once) tma_load<CG>(smem_u32(sW + r.i * w_bytes), &w_map, s * kStepBytes, w_row, full, once);
                    else tma_load<CG>(smem_u32(sW + r.i * w_bytes), &w_map, s * kStepBytes, w_row, full);
                    for (int b = 0; b < boxes; ++b)
                        tma_load<CG>(smem_u32(sX + r.i * x_bytes + b * a.x_box * kStepBytes), &x_map, s * kStepBytes, x_row + b * a.x_box, full);
                    ++issued;
                    r.next();
                }
            }
            // a wait ran out: copies in flight still land (each stage's last ones), in front of the CTA's end
            if (!ok && leader) {
                for (int j = 0; j < min(issued, a.stages); ++j) {
                    if (r.i == 0) r.phase ^= 1u;
                    r.i = r.i == 0 ? a.stages - 1 : r.i - 1;
                    poll<false>(bar(kBarFull + r.i), r.phase, nullptr, limit);
                }
            }
        }
    } else if (warp == 1 && leader) {
        if (elect_one()) {
            Ring r(a.stages), rs(kTurns);
            const uint32_t sa = tmem + kScaleCols<FMT>, sb = sa + 4 * CH;
            const uint64_t da0 = operand_desc(smem_u32(sW)), db0 = operand_desc(smem_u32(sX)), ds0 = scales_desc(smem_u32(sS));
            const int whole = a.K / 256;                          // steps of four MMAs
            int n = 0;
            bool ok = true;
            for (int i = first; i < tiles && ok; i += stride, ++n) {
                const Tile t = tile_at<CG>(a, table, i);
                const int b = n & 1, use = n >> 1;
                if (overlap) ok = n == 0 || wait_alone<CG == 2>(bar(kBarAccFree + b), (uint32_t)(b == 1 ? use : use - 1) & 1u, gave_up, limit);
                else ok = wait_alone<CG == 2>(bar(kBarAccFree + b), ((uint32_t)use & 1u) ^ 1u, gave_up, limit);
                if (!ok) break;
                const int cols = CG == 2 ? (t.count + 15) / 16 * 16 : (t.count + 7) / 8 * 8;
                const uint32_t idesc = 1u << 7 | 1u << 10 | (uint32_t)(cols >> 3) << 17 | (FMT == ELUTQ_MX4_MXFP4 ? 1u << 23 : 0u) | (uint32_t)(CG * kTileW >> 4) << 24;
                const uint32_t acc = tmem + (b ? acc1 : 0);
                for (int s = step0; s < step1; ++s) {
                    const int in_turn = (s - step0) % kTurn;
                    ok = wait_alone<CG == 2, true>(bar(kBarFull + r.i), r.phase, gave_up, limit);
                    if (in_turn == 0) ok = ok && wait_alone<CG == 2>(bar(kBarScalesFull + rs.i), rs.phase, gave_up, limit);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t da = da0 + (uint32_t)(r.i * w_bytes >> 4), db = db0 + (uint32_t)(r.i * x_bytes >> 4), ds = ds0 + (uint32_t)((rs.i * kTurn + in_turn) * s_bytes >> 4);
#pragma unroll
                    for (int c = 0; c < CH; ++c) {
                        copy_scales<CG>(sa + 4 * c, ds + c * 32);
#pragma unroll
                        for (int h = 0; h < NB; ++h) copy_scales<CG>(sb + 4 * (c * NB + h), ds + (CH + c * NB + h) * 32);
                    }
                    auto step_mma = [&](int j, uint32_t accumulate) {
                        const int c = j / SUB;
                        const uint32_t id = (uint32_t)(j % SUB) * 2u;             // which of the group's scales
                        mma<FMT, CG>(acc, da + 2 * j, db + 2 * j, idesc | id << 29 | id << 4, sa + 4 * c, sb + 4 * c * NB, accumulate);
                    };
                    step_mma(0, s > step0);
                    if (s < whole) {
                        step_mma(1, 1);
                        step_mma(2, 1);
                        step_mma(3, 1);
                    } else {
                        if (a.K - s * 256 > 64) step_mma(1, 1);
                        if (a.K - s * 256 > 128) step_mma(2, 1);
                        if (a.K - s * 256 > 192) step_mma(3, 1);
                    }
                    commit<CG>(bar(kBarEmpty + r.i));
                    r.next();
                    if (in_turn == kTurn - 1 || s == step1 - 1) {
                        commit<CG>(bar(kBarScalesEmpty + rs.i));
                        rs.next();
                    }
                }
                if (ok) commit<CG>(bar(kBarAccFull + b));
            }
            if (!ok) {                         // what has been issued ends in front of the tensor memory's release
                commit<CG>(bar(kBarDrain));
                poll<false>(bar(kBarDrain), 0u, nullptr, limit);
            }
        }
    } else if (warp >= 4 && warp < 8) {
        const int quarter = warp & 3;                             // lanes of tensor memory
        grid_dependency_wait();
        int n = 0;
        bool ok = true;
        for (int i = first; i < tiles && ok; i += stride, ++n) {
            const Tile t = tile_at<CG>(a, table, i);
            const int b = n & 1, use = n >> 1;
            ok = wait<CG == 2>(bar(kBarAccFull + b), (uint32_t)use & 1u, gave_up, limit);
            if (a.split > 1) ok = epilogue_agrees(ok && wait<true>(bar(kBarPartsFree), ((uint32_t)n & 1u) ^ 1u, gave_up, limit));
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const uint32_t acc = tmem + (b ? acc1 : 0) + ((uint32_t)(quarter * 32) << 16);
            const float alpha = a.alpha != nullptr ? __ldg(a.alpha + t.e) : 1.0f;
            const int row = quarter * 32 + lane, col = t.n0 + (CG == 2 ? (int)rank * kTileW : 0) + row;
            auto release = [&](int which) {
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 2) arrive_remote(at_rank(bar(kBarAccFree + which), 0));
                    else arrive(bar(kBarAccFree + which));
                }
                __syncwarp();
            };
            if (a.split > 1) {
                for (int c0 = 0; c0 < t.count; c0 += 16) {
                    uint32_t v[16];
                    tmem_ld16(v, acc + c0);
                    tmem_ld_wait(v);
#pragma unroll
                    for (int c = 0; c < 16; ++c)
                        if (c0 + c < t.count) parts[(c0 + c) * kTileW + row] = __uint_as_float(v[c]);
                }
                release(b);
                asm volatile("bar.sync 1, 128;" ::: "memory");
                if (threadIdx.x - 128u < (unsigned)a.split) arrive_cluster(at_rank(bar(kBarPartsFull), threadIdx.x - 128u));
                __syncwarp();
                ok = wait<true>(bar(kBarPartsFull), (uint32_t)n & 1u, gave_up, limit);
                if (ok) {
                    // eight of this CTA's columns at a time: as many loads in flight
                    for (int c0 = (int)rank; c0 < t.count; c0 += 8 * a.split) {
                        float sum[8] = {};
                        for (int s = 0; s < a.split; ++s) {
                            const uint32_t from = at_rank(smem_u32(parts + row), (uint32_t)s);
                            float v[8];
#pragma unroll
                            for (int c = 0; c < 8; ++c)
                                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[c]) : "r"(from + (uint32_t)(min(c0 + c * a.split, t.count - 1) * kTileW * 4)) : "memory");
#pragma unroll
                            for (int c = 0; c < 8; ++c) sum[c] += v[c];
                        }
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            if (c0 + c * a.split < t.count && col < a.N) store_y(a, (long long)(t.t0 + c0 + c * a.split) * a.N + col, sum[c] * alpha);
                    }
                }
                if (i + stride >= tiles) break;                   // nothing comes behind it
                ok = epilogue_agrees(ok);
                if (threadIdx.x - 128u < (unsigned)a.split) arrive_cluster(at_rank(bar(kBarPartsFree), threadIdx.x - 128u));
                __syncwarp();
                continue;
            }
            // (N is below 2^30: a step of two rows fits 32 bits, one of three or four fits without a sign, one of eight does not.)
            // 48 columns at a time, whose reads of tensor memory are all in flight together (16 at a time took 11000 cycles for 256 beside
            // MMAs that needed 8200).  Overlapping accumulators: the 48 that both have come first; once they are in registers the other
            // accumulator may be filled.
            constexpr int G = kChunk / 16;
            auto columns = [&](int c0, int end, auto&& then) {
                uint32_t v[G][16];
#pragma unroll
                for (int g = 0; g < G; ++g) tmem_ld16(v[g], acc + c0 + 16 * g);       // (columns behind the last one are not used)
#pragma unroll
                for (int g = 0; g < G; ++g) tmem_ld_wait(v[g]);
                then();
                if (col < a.N) {
                    const long long at = (long long)(t.t0 + c0) * a.N + col;
                    auto put = [&](auto* y, auto&& cast) {            // four pointers: a short chain of additions
                        decltype(y) to[4] = {y, y + a.N, y + 2 * a.N, y + 3u * (unsigned)a.N};
                        const bool all = c0 + kChunk <= end;
#pragma unroll
                        for (int c = 0; c < kChunk; ++c) {
                            if (all || c0 + c < end) *to[c % 4] = cast(__uint_as_float(v[c / 16][c % 16]) * alpha);
                            to[c % 4] += 4u * (unsigned)a.N;
                        }
                    };
                    if (CG == 1 && a.y_type == ELUTQ_TYPE_F16) put(reinterpret_cast<__half*>(a.Y) + at, [](float f) { return __float2half_rn(f); });
                    else if (CG == 1 && a.y_type == ELUTQ_TYPE_BF16) put(reinterpret_cast<__nv_bfloat16*>(a.Y) + at, [](float f) { return __float2bfloat16_rn(f); });
                    else put(reinterpret_cast<float*>(a.Y) + at, [](float f) { return f; });
                }
                __syncwarp();
            };
            // The same for 16-bit results whose rows start on 4, 8 or 16 bytes: fragments are stored transposed, a block of 16 tokens x 32 weight rows at a time, read
            // back as so many bytes of a token's row and stored so: with 16 bytes 2 stores of 8 x 64 instead of 16 of 64.  The 16-byte pieces of two tokens'
            // rows share a line of 128 bytes, in an order by the line's number: no conflicts either way.  With an odd N every second row starts in the middle of 4
            // bytes: its words are made of two, and its first and last value go by themselves (857 x 41529 x 1472 MXFP4 58 -> 49 us); with few tokens a value at a
            // time is 5 to 9 % faster.
            auto columns_turned = [&](int c0, int end, auto&& then, auto half, auto width) {
                constexpr bool odd_n = decltype(width)::value == 2;          // every second row starts in the middle of 4 bytes
                constexpr int W = odd_n ? 4 : decltype(width)::value, LANES = 64 / W, AT_ONCE = 32 / LANES;      // bytes of a store; lanes of a row; rows
                uint32_t v[G][16];
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    tmem_ld_fragments(v[g], acc + c0 + 16 * g);
                    tmem_ld_fragments(v[g] + 8, acc + (16u << 16) + c0 + 16 * g);
                }
#pragma unroll
                for (int g = 0; g < G; ++g) tmem_ld_wait(v[g]);
                then();
                auto two = [&](uint32_t x, uint32_t y) -> uint32_t {
                    const float fx = __uint_as_float(x) * alpha, fy = __uint_as_float(y) * alpha;
                    if constexpr (decltype(half)::value) {
                        const __half2 h = __floats2half2_rn(fx, fy);
                        return *reinterpret_cast<const uint32_t*>(&h);
                    } else {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(fx, fy);
                        return *reinterpret_cast<const uint32_t*>(&h);
                    }
                };
                uint8_t* mine = sT + quarter * (kChunk * 64);
                const int token = 8 * (lane >> 4) + (lane & 7), piece = (lane >> 3) & 1;      // where this lane's row of a matrix goes
                const uint32_t to = smem_u32(mine + token * 64 + ((piece ^ ((token >> 1) & 3)) * 16));
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        store_transposed((to + g * 1024) ^ (32u * h), two(v[g][8 * h], v[g][8 * h + 1]), two(v[g][8 * h + 2], v[g][8 * h + 3]),
                                         two(v[g][8 * h + 4], v[g][8 * h + 5]), two(v[g][8 * h + 6], v[g][8 * h + 7]));
                __syncwarp();
                if constexpr (odd_n) {
                    const int n0 = t.n0 + (CG == 2 ? (int)rank * kTileW : 0) + quarter * 32;
                    auto at = [&](int tok, int value) { return mine + tok * 64 + (((value >> 3) ^ ((tok >> 1) & 3)) * 16) + (value & 7) * 2; };
                    uint16_t* out = reinterpret_cast<uint16_t*>(a.Y) + (long long)(t.t0 + c0) * a.N + n0;
                    if (n0 + 32 <= a.N) {
                        const int part = lane & 15, tok0 = lane >> 4;
                        const bool odd = (t.t0 + c0 + tok0) & 1;             // of all this lane's tokens
                        const int rest = odd && part == 15 ? 0 : end - c0 - tok0;
                        uint16_t* to2 = out + (long long)tok0 * a.N + 2 * part + odd;
#pragma unroll
                        for (int k0 = 0; k0 < kChunk / 2; k0 += 6) {
                            uint32_t y[6];
#pragma unroll
                            for (int k = 0; k < 6; ++k) {
                                const int tok = 2 * (k0 + k) + tok0;
                                const uint32_t x = *reinterpret_cast<const uint32_t*>(at(tok, 2 * part)), z = *reinterpret_cast<const uint32_t*>(at(tok, min(2 * part + 2, 30)));
                                y[k] = odd ? __funnelshift_r(x, z, 16) : x;
                            }
#pragma unroll
                            for (int k = 0; k < 6; ++k) {
                                if (2 * (k0 + k) < rest) *reinterpret_cast<uint32_t*>(to2) = y[k];
                                to2 += 2 * a.N;
                            }
                        }
                        const int first_odd = (t.t0 + c0 + 1) & 1, value = lane & 1 ? 31 : 0;      // the ends of those rows
#pragma unroll
                        for (int k = 0; k < (kChunk + 31) / 32; ++k) {
                            const int tok = 32 * k + 2 * (lane >> 1) + first_odd;
                            if (tok < kChunk && c0 + tok < end) out[(long long)tok * a.N + value] = *reinterpret_cast<const uint16_t*>(at(tok, value));
                        }
                    } else if (n0 + lane < a.N) {                            // the matrix's last columns
                        for (int tok = 0; tok < min(kChunk, end - c0); ++tok) out[(long long)tok * a.N + lane] = *reinterpret_cast<const uint16_t*>(at(tok, lane));
                    }
                } else {
                    const int part = lane % LANES, tok0 = lane / LANES, col0 = t.n0 + (CG == 2 ? (int)rank * kTileW : 0) + quarter * 32 + part * (W / 2);
                    uint16_t* out = reinterpret_cast<uint16_t*>(a.Y) + (long long)(t.t0 + c0 + tok0) * a.N + col0;
                    const int rest = col0 < a.N ? end - c0 - tok0 : 0;
                    using V = typename std::conditional<W == 16, uint4, typename std::conditional<W == 8, uint2, uint32_t>::type>::type;
                    constexpr int N_ST = kChunk / AT_ONCE, BATCH = N_ST < 6 ? N_ST : 6;
#pragma unroll
                    for (int k0 = 0; k0 < N_ST; k0 += BATCH) {
                        V y[BATCH];
#pragma unroll
                        for (int k = 0; k < BATCH; ++k) {
                            const int tok = AT_ONCE * (k0 + k) + tok0;
                            y[k] = *reinterpret_cast<const V*>(mine + tok * 64 + (((part * W / 16) ^ ((tok >> 1) & 3)) * 16) + part * W % 16);
                        }
#pragma unroll
                        for (int k = 0; k < BATCH; ++k) {
                            if (AT_ONCE * (k0 + k) < rest) *reinterpret_cast<V*>(out) = y[k];
                            if constexpr (AT_ONCE == 8) out += 4u * (unsigned)a.N;
                            out += (AT_ONCE < 4 ? AT_ONCE : 4u) * (unsigned)a.N;
                        }
                    }
                }
                __syncwarp();
            };
            auto all_columns = [&](auto&& some) {
                if (overlap) {
                    const int c0 = b == 0 ? acc1 : 0, c1 = b == 0 ? 0 : kShared, end = min(t.count, c1 + acc1);
                    some(c0, min(t.count, c0 + kChunk), [&] { release(b ^ 1); });
                    for (int c = c1; c < end; c += kChunk) some(c, end, [] {});
                } else {
                    for (int c = 0; c < t.count; c += kChunk) some(c, t.count, [] {});
                    release(b);
                }
            };
            // (a row's alignment decides the width of its stores)
            auto turned = [&](auto half) {
                if (a.N % 8 == 0) all_columns([&](int c0, int end, auto&& then) { columns_turned(c0, end, then, half, IntC<16>{}); });
                else if (a.N % 4 == 0) all_columns([&](int c0, int end, auto&& then) { columns_turned(c0, end, then, half, IntC<8>{}); });
                else if (CG == 1 || a.N % 2 == 0) all_columns([&](int c0, int end, auto&& then) { columns_turned(c0, end, then, half, IntC<4>{}); });
                else all_columns([&](int c0, int end, auto&& then) { columns_turned(c0, end, then, half, IntC<2>{}); });
            };
            if (!a.turn) all_columns(columns);
            else if (a.y_type == ELUTQ_TYPE_F16) turned(IntC<1>{});
            else turned(IntC<0>{});
        }
    } else {
        const int helper = warp < 4 ? warp - 2 : warp - 6, block = helper >> 1;      // weights, tokens 0 to 127, 128 to 255
        if (helper >= 0 && block <= NB) {
            Ring r(kTurns);
            const uint8_t* base = block == 0 ? a.w_scales : a.x_scales;
            const bool wide = block == 0 ? a.w_wide : a.x_wide;
            const long long all = block == 0 ? (long long)a.E * a.N : a.M;
            // A lane's pieces: 16 bytes of a row's turn (64 bytes NVFP4, 32 MXFP4), in rows r + 32 q with neighbours in q and r; the four words of a
            // piece go to as many groups of 512 bytes, without conflicts.  (A lane per row, 4 or 2 pieces of it, touched 32 lines a load
            // instead of 8 or 16, and NVFP4 was bound by that: 4096 x 28672 x 4096 245 us.)
            constexpr int PIECES = CH, LOADS = 4 * PIECES, ROWS = 8 / PIECES;             // pieces of a row; loads; rows r of a load
            const int piece = lane % PIECES, q = lane / PIECES % 4, r0 = lane / (4 * PIECES);
            // Of scales whose rows start elsewhere, a lane has pieces of rows c + 8 k (NVFP4, whose rows are an even number of bytes) or c + 16 k: all of these start at
            // the same place in 16 bytes, and where a lane's words go is the same for every k.  Lines touched by a load bound this too: its four lanes of a row meet in a
            // bank when they store, and pieces of different rows, whose words do not, took 1536 x 32056 x 2080 NVFP4 from 81 to 100 us when that was tried.  Words of 4 bytes loaded by
            // every lane for its own piece, 5 for 16 bytes: 8 x 6577 x 5952 NVFP4 11.4 us instead of 10.3, 34 rows of 11 experts of 5690 x 4160 33 instead of 29,
            // with pairs 2 to 4 % less.
            constexpr int EVERY = 32 / PIECES;
            const int row_c = lane / PIECES;
            const int first_word = block == 0 ? 0 : CH + block - 1, pitch = block == 0 ? 1 : NB;
            uint8_t* to = sS + first_word * 512;
            int turn = 0;
            bool ok = true;
            grid_dependency_wait();
            const uint8_t *first16 = base, *last16 = base;                        // the matrix's whole pieces of 16 bytes
            if (!wide) {
                first16 = base + (16u - (uint32_t)reinterpret_cast<uintptr_t>(base)) % 16u;
                last16 = base + all * a.sk - (reinterpret_cast<uintptr_t>(base + all * a.sk) & 15);
            }
            // of a row's words in a turn, where number d goes
            auto place = [&](int d) { return d / CH * s_bytes + d % CH * pitch * 512; };
            for (int i = first; i < tiles && ok; i += stride) {
                const Tile t = tile_at<CG>(a, table, i);
                const long long top = block == 0 ? (long long)t.e * a.N + t.n0 + (CG == 2 ? (int)rank * kTileW : 0) : t.t0 + 128 * (block - 1);
                for (int s = step0; s < step1 && ok; s += kTurn, turn ^= 1, r.next()) {
                    if (turn != (helper & 1)) continue;
                    uint32_t w[LOADS][4];
                    const int at = s * 4 * CH + 16 * piece;
                    if (wide) {
                        const long long row0 = top + r0 + 32 * q;
#pragma unroll
                        for (int k = 0; k < LOADS; ++k) {
                            uint4 v = make_uint4(0u, 0u, 0u, 0u);
                            if (at < a.sk) v = __ldg(reinterpret_cast<const uint4*>(base + min(row0 + ROWS * k, all - 1) * a.sk + at));
                            w[k][0] = v.x; w[k][1] = v.y; w[k][2] = v.z; w[k][3] = v.w;
                        }
                        ok = wait(bar(kBarScalesEmpty + r.i), r.phase ^ 1u, gave_up, limit);
                        if (!ok) break;
                        uint8_t* slot = to + r.i * kTurn * s_bytes + place(4 * piece) + r0 * 16 + q * 4;
#pragma unroll
                        for (int k = 0; k < LOADS; ++k)
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                *reinterpret_cast<uint32_t*>(slot + (c / CH) * s_bytes + (c % CH) * pitch * 512 + ROWS * k * 16) = w[k][c];
                    } else {
                        // The aligned piece that a lane's 16 bytes of a row begin in; the one behind the row's last by its lane k % PIECES.  Bytes are
                        // moved within words, with the next lane's first; words need not move, as each goes to where it belongs (the first ones of a
                        // row may belong to the turn before).  Pieces that are not wholly the matrix's come last, row by row.
                        const uint8_t* p = base + (top + row_c) * a.sk + at;
                        const unsigned pace = EVERY * (unsigned)a.sk;                  // (K is 2^28 at most)
                        const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 15u, shift = 8u * (off & 3u);
                        const int lead = (int)(off >> 2);                      // words in front of a row's
                        // how far behind q0 whole pieces begin (128 rows are less than 2^31 bytes); only the first one can lie in front of the matrix
                        const uint8_t* q0 = p - off;
                        const int room = (int)max(min((long long)(last16 - q0) - 16, 0x7fffffffLL), -1LL);
                        uint32_t behind[4][4];
#pragma unroll
                        for (int k = 0; k < LOADS; ++k) load_piece(w[k], q0 + k * pace, (k > 0 || q0 >= first16) && (int)(k * pace) <= room);
#pragma unroll
                        for (int m = 0; m < 4; ++m) {
                            const unsigned by = (m * PIECES + piece) * pace + 16 * (PIECES - piece);
                            load_piece(behind[m], q0 + by, (int)by <= room);
                        }
#pragma unroll
                        for (int k = 0; k < LOADS; ++k) {
                            const uint32_t beside = __shfl_down_sync(0xffffffffu, w[k][0], 1), last = __shfl_sync(0xffffffffu, behind[k / PIECES][0], k % PIECES, PIECES);
                            const uint32_t next = piece == PIECES - 1 ? last : beside;
#pragma unroll
                            for (int c = 0; c < 4; ++c) w[k][c] = __funnelshift_r(w[k][c], c < 3 ? w[k][c + 1] : next, shift);
                        }
#pragma unroll
                        for (int m = 0; m < 4; ++m)
#pragma unroll
                            for (int c = 0; c < 3; ++c) behind[m][c] = __funnelshift_r(behind[m][c], behind[m][c + 1], shift);
                        uint32_t keep[7] = {~0u, ~0u, ~0u, ~0u, ~0u, ~0u, ~0u};
                        if (s * 4 * CH + 16 * PIECES > a.sk) {                 // bytes behind the rows' end
                            auto mask = [&](int d) {
                                const int left = a.sk - s * 4 * CH - 4 * d;
                                return left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << (8 * left)) - 1u;
                            };
#pragma unroll
                            for (int c = 0; c < 4; ++c) keep[c] = mask(4 * piece + c - lead);
#pragma unroll
                            for (int c = 0; c < 3; ++c) keep[4 + c] = mask(4 * PIECES + c - lead);
                        }
                        ok = wait(bar(kBarScalesEmpty + r.i), r.phase ^ 1u, gave_up, limit);
                        if (!ok) break;
                        uint8_t* slot = to + r.i * kTurn * s_bytes;
                        // row c + EVERY k of 128 is number c + EVERY (k % PIECES) of 32s number k / PIECES
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            const int d = 4 * piece + c - lead;
                            if (d >= 0) {
                                uint8_t* dst = slot + place(d) + row_c * 16;
#pragma unroll
                                for (int k = 0; k < LOADS; ++k) *reinterpret_cast<uint32_t*>(dst + k % PIECES * EVERY * 16 + k / PIECES * 4) = w[k][c] & keep[c];
                            }
                        }
#pragma unroll
                        for (int c = 0; c < 3; ++c)
                            if (c < lead) {
                                uint8_t* dst = slot + place(4 * PIECES + c - lead) + (row_c + EVERY * piece) * 16;
#pragma unroll
                                for (int m = 0; m < 4; ++m) *reinterpret_cast<uint32_t*>(dst + m * 4) = behind[m][c] & keep[4 + c];
                            }
                        const long long below = min(top + 128, all);            // rows of the matrix end here
                        if (top * a.sk + s * 4 * CH < first16 - base || (below - 1) * a.sk + min(s * 4 * CH + 16 * PIECES, a.sk) > last16 - base) {
                            __syncwarp();
                            const Ends ends = ends_of(base, base + all * a.sk);
#pragma unroll 1
                            for (int k = 0; k < LOADS; ++k) {
                                const uint8_t* b = p + k * pace;
                                const bool edge = top + row_c + EVERY * k < all && at < a.sk && (b < first16 || b + min(16, a.sk - at) > last16);
                                if (!__any_sync(0xffffffffu, edge)) continue;
                                const uint8_t* row = base + min(top + row_c + EVERY * k, all - 1) * a.sk;
                                uint32_t f[4];
                                load_words(f, row + at, row + a.sk, ends);
#pragma unroll
                                for (int c = 0; c < 4; ++c)
                                    if (edge) *reinterpret_cast<uint32_t*>(slot + place(4 * piece + c) + (row_c + k % PIECES * EVERY) * 16 + k / PIECES * 4) = f[c];
                            }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (CG == 2) arrive_remote(at_rank(bar(kBarScalesFull + r.i), 0));
                        else arrive(bar(kBarScalesFull + r.i));
                    }
                    __syncwarp();
                }
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (CG == 2 || a.split > 1) cluster_barrier();                // no CTA leaves while another reads its memory or arrives on its barriers
    if (warp == 1) {
        if constexpr (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

struct Plan { int cg, tokens, x_box, split, stages, grid, turn; size_t smem; bool ok; };

constexpr int kFixed = kNumBars * 8 + 16;

// Ring length and shared memory of a plan whose other fields are set; false if the ring is too short.
bool fill_plan(Plan& p, int format, int E, bool grouped) {
    const int ch = format == ELUTQ_MX4_MXFP4 ? 2 : 4, nb = p.cg;
    const int stage = kTileW * kStepBytes + (p.tokens / p.cg + 7) / 8 * 1024;
    const int fixed = kFixed + kTurns * kTurn * ((1 + nb) * ch * 512 + 32) + (p.turn ? kTurnBytes : 0) + (p.split > 1 ? p.tokens * kTileW * 4 : 0) + (grouped ? (3 * E + 1) * 4 : 0);
    p.stages = (kSmem - fixed) / stage;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    p.smem = (size_t)p.stages * stage + fixed;
    return p.stages >= 2;
}

// Time in us of `tiles` tiles (weights of `groups` matrices in all): a launch's fixed part, which grows with the tokens that a tile's epilogue stores, and the
// longest of three: steps of the busiest SMs, weights from HBM, all tiles' operands (a rate that stands for L2 and, at many tokens, for power).  A
// further tile's steps overlap with the last one's epilogue.  Parts of a cluster cost their exchange.  Fitted to 4400 calls (1000 to 57344 weight rows,
// K 1024 to 14336, 1 to 512 tokens; used for more as well), 10 % off in the mean; a choice by it costs 1 % against the best plan measured, 15 % at
// most (10240 x 8192, 512 tokens).
double estimate_us(long long tiles, double groups, int N, int K, int format, int cg, int tokens, int split, int num_sms) {
    const int steps = (K + 255) / 256, units = (steps + 1) / 2;
    const long long teams = cg == 2 ? num_sms / 2 : split > 1 ? resident_clusters(split) : num_sms;
    if (teams <= 0) return 1e30;
    const long long rounds = (tiles + teams - 1) / teams;
    const int own = split > 1 ? 2 * ((units + split - 1) / split) : steps;
    const double row = 128.0 + 256.0 / mx4_block(format), step_us = (cg == 2 ? 0.25 : 0.24) + 0.0001 * tokens + (format == ELUTQ_MX4_NVFP4 ? 0.028 : 0.0);
    const double sm = rounds * own * step_us - 0.086 * (rounds - 1), hbm = groups * N * steps * row / 5.54e6;
    const double l2 = (double)tiles * steps * (cg * kTileW + tokens) * row / 10.6e6;
    const double longest = sm > hbm ? (sm > l2 ? sm : l2) : (hbm > l2 ? hbm : l2);
    const double exchange = split > 1 ? 1.26 + 0.256 * split + 0.0057 * tokens * split * rounds : 0.0;
    return 3.36 + 0.009 * tokens + (cg == 2 ? 0.63 : 0.0) + longest + exchange;
}

int round_up(int v, int m) { return (v + m - 1) / m * m; }

// Tile and cluster of a call.  Dense: the least estimate over tiles that share the rows evenly (as few as possible, one or two more, twice as many) and clusters of up to
// 8.  Groups: how many rows each has is known on the device only, and a tile's height on the host follows the mean; too much of it costs little (a
// tile is as wide as its rows; the ring gets shorter), too little reads weights again: us with 8, 16, 32, 64, 96, 128 rows and with pairs of 256,
// 128 experts of 1536 x 2048, MXFP4, 1024 rows (8 each) -, 39.7, 40.9, 40.8, 40.7, 42.4, -; 4096 rows (32 each) -, -, 49, 42.6, 42.4, 44.0, 46.2;
// 64 of 4096 x 2048, 8192 rows (128 each) -, -, -, 102.7, 78.1, 74.6, 63.4.
Plan plan_for(int M, int N, int K, int E, int format, bool grouped, int y_type, int num_sms) {
    Plan p = {};
    double best = 0.0;
    auto consider = [&](int cg, int tokens, int split, long long tiles, double groups) {
        const double us = estimate_us(tiles, groups, N, K, format, cg, tokens, split, num_sms);
        if (best == 0.0 || us < best) {
            best = us;
            p.cg = cg;
            p.tokens = tokens;
            p.split = split;
        }
    };
    const int units = (K + 511) / 512;
    if (grouped) {
        const int mean = (M + E - 1) / E;
        const int cg = mean > 96 ? 2 : 1;
        int tokens = mean <= 8 ? 32 : mean <= 16 ? 64 : mean <= 48 ? 96 : mean <= 96 ? 128 : 256;
        if (tokens > round_up(M, 8)) tokens = round_up(M, 8);
        const int busy = E < M ? E : M;
        for (int split = 1; split <= (tokens <= kMaxSplitTokens ? kMaxSplit : 1); split *= 2)
            if (split <= units) consider(cg, tokens, split, (long long)((N + cg * kTileW - 1) / (cg * kTileW)) * (busy + (M - busy) / tokens), busy);
    } else {
        for (int cg = 1; cg <= 2; ++cg) {
            const int least = (M + 128 * cg - 1) / (128 * cg);
            for (int k = 0; k < 4; ++k) {
                const int n = k < 3 ? least + k : 2 * least;
                if (n > least && M <= 32) continue;
                int tokens = round_up((M + n - 1) / n, 8);
                if (tokens > 32) tokens = round_up(tokens, 32);
                if (tokens > 128 * cg || (cg == 2 && tokens < 64)) continue;
                const long long tiles = (long long)((N + cg * kTileW - 1) / (cg * kTileW)) * ((M + tokens - 1) / tokens);
                for (int split = 1; split <= (cg == 1 && tokens <= kMaxSplitTokens ? kMaxSplit : 1); split *= 2)
                    if (split <= units) consider(cg, tokens, split, tiles, 1.0);
            }
        }
    }
    if (p.cg == 2) p.tokens = round_up(p.tokens, 16);
    // rows of one load: dense, all of a tile's; of groups, whose tiles are of any height, up to 32
    const int rows = p.tokens / p.cg;
    p.x_box = !grouped ? rows : rows % 32 == 0 ? 32 : rows % 16 == 0 ? 16 : 8;
    const long long w_tiles = (N + p.cg * kTileW - 1) / (p.cg * kTileW);
    const long long most = w_tiles * ((M + p.tokens - 1) / p.tokens + (grouped ? (E < M ? E : M) : 0));
    p.turn = p.split == 1 && y_type != ELUTQ_TYPE_F32 && (p.cg == 2 || N % 2 == 0);
    p.ok = fill_plan(p, format, E, grouped);
    const int team = p.cg == 2 ? 2 : p.split;
    const long long teams = p.cg == 2 ? num_sms / 2 : p.split > 1 ? resident_clusters(p.split) : num_sms;
    p.grid = (int)(most < teams ? most : teams) * team;
    return p;
}

int tensor_map(CUtensorMap* map, const void* base, long long rows, int K, int box) {
    const EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return (int)cudaErrorNotSupported;
    const cuuint64_t dims[2] = {(cuuint64_t)K / 2, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)K / 2};
    const cuuint32_t sizes[2] = {kStepBytes, (cuuint32_t)box}, elem[2] = {1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, sizes, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? 0 : (int)cudaErrorInvalidValue;
}

// Devices that products have been launched on, a bit for each number modulo 64
std::atomic<unsigned long long> g_devices{0};
inline unsigned long long device_bit(int dev) { return 1ull << (dev & 63); }

template <int FMT, int CG>
int launch_mx4(const Plan& p, const CUtensorMap& xm, const CUtensorMap& wm, const Mx4Args& a, cudaStream_t stream) {
    // once for each device (a call would take half a microsecond of the host's time)
    static std::atomic<unsigned long long> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return (int)e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(ready.load(std::memory_order_acquire) & bit)) {
        e = cudaFuncSetAttribute(mx4_gemm_kernel<FMT, CG>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        if (e != cudaSuccess) return (int)e;
        ready.fetch_or(bit, std::memory_order_release);
    }
    if (!(g_devices.load(std::memory_order_relaxed) & device_bit(dev))) g_devices.fetch_or(device_bit(dev));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.grid);
    cfg.blockDim = dim3((unsigned)kThreads<CG>);
    cfg.dynamicSmemBytes = p.smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)(CG == 2 ? 2 : p.split);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CG == 2 || p.split > 1 ? 2 : 1;
    e = cudaLaunchKernelEx(&cfg, mx4_gemm_kernel<FMT, CG>, xm, wm, a);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}

template <int FMT>
int launch_format(const Plan& p, const CUtensorMap& xm, const CUtensorMap& wm, const Mx4Args& a, cudaStream_t stream) {
    return p.cg == 2 ? launch_mx4<FMT, 2>(p, xm, wm, a, stream) : launch_mx4<FMT, 1>(p, xm, wm, a, stream);
}

int run_mx4(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, const int* offsets, void* Y, int y_type,
            int M, int N, int K, int E, int format, const float* alpha, uint32_t test_limit, void* stream) {
    if (!x_codes || !x_scales || !w_codes || !w_scales || !Y) return ELUTQ_ERR_INVALID_ARG;
    if (N <= 0 || E <= 0 || y_type < ELUTQ_TYPE_F16 || y_type > ELUTQ_TYPE_F32) return ELUTQ_ERR_INVALID_ARG;
    const int st = mx4_check(format, M, K);
    if (st != ELUTQ_OK) return st;
    if (E > kMaxGroups) return ELUTQ_ERR_UNSUPPORTED;
    if (K > kMaxK) return ELUTQ_ERR_SHAPE;
    if (M > 0x3fffffff || (long long)E * N > 0x3fffffffLL) return ELUTQ_ERR_SHAPE;           // rows are 32-bit coordinates
    if (!mx4_aligned(x_codes, 16) || !mx4_aligned(w_codes, 16) || !mx4_aligned(Y, 16) || !mx4_aligned(offsets, 4) || !mx4_aligned(alpha, 4)) return ELUTQ_ERR_ALIGN;
    const bool grouped = offsets != nullptr;
    const Plan p = plan_for(M, N, K, E, format, grouped, y_type, device_sm_count());
    if (!p.ok) return ELUTQ_ERR_UNSUPPORTED;
    const int w_tiles = (N + p.cg * kTileW - 1) / (p.cg * kTileW);
    if ((long long)w_tiles * ((M + p.tokens - 1) / p.tokens + (grouped ? E : 0)) > 0x3fffffffLL) return ELUTQ_ERR_SHAPE;
    Mx4Args a;
    a.x_scales = reinterpret_cast<const uint8_t*>(x_scales);
    a.w_scales = reinterpret_cast<const uint8_t*>(w_scales);
    a.alpha = alpha;
    a.offsets = offsets;
    a.Y = Y;
    a.y_type = y_type;
    a.M = M; a.N = N; a.K = K; a.E = E;
    a.sk = K / mx4_block(format);
    a.tokens = p.tokens;
    a.w_tiles = w_tiles;
    a.steps = (K + 255) / 256;
    a.split = p.split;
    a.stages = p.stages;
    a.x_box = p.x_box;
    a.once = (grouped ? (M + E - 1) / E : M) <= p.tokens;
    a.turn = p.turn;
    a.x_wide = mx4_aligned(x_scales, 16) && a.sk % 16 == 0;
    a.w_wide = mx4_aligned(w_scales, 16) && a.sk % 16 == 0;
    a.test = test_limit != 0;
    a.wait_limit = test_limit != 0 ? test_limit : 0xffffffffu;
    CUtensorMap xm, wm;
    int ce = tensor_map(&xm, x_codes, M, K, p.x_box);
    if (ce == 0) ce = tensor_map(&wm, w_codes, (long long)E * N, K, kTileW);
    if (ce == 0)
        ce = format == ELUTQ_MX4_MXFP4 ? launch_format<ELUTQ_MX4_MXFP4>(p, xm, wm, a, (cudaStream_t)stream) : launch_format<ELUTQ_MX4_NVFP4>(p, xm, wm, a, (cudaStream_t)stream);
    if (ce == 0) return ELUTQ_OK;
    note_cuda_error(ce);
    return ELUTQ_ERR_CUDA;
}

}  // namespace

int mx4_status(unsigned* word, cudaStream_t stream) {
    *word = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || !(g_devices.load() & device_bit(dev))) return (int)e;
    // (not in the default stream, which would wait for all others and end a capture of one)
    e = cudaMemcpyFromSymbolAsync(word, g_status, sizeof(*word), 0, cudaMemcpyDeviceToHost, stream);
    return (int)(e != cudaSuccess ? e : cudaStreamSynchronize(stream));
}
int mx4_clear_status() {
    const unsigned long long devices = g_devices.load();
    if (devices == 0) return 0;
    int count = 0, current = 0;
    cudaError_t first = cudaGetDeviceCount(&count);
    if (first == cudaSuccess) first = cudaGetDevice(&current);
    if (first != cudaSuccess) return (int)first;
    for (int dev = 0; dev < count; ++dev) {
        if (!(devices & device_bit(dev))) continue;
        const unsigned zero = 0;
        cudaError_t e = cudaSetDevice(dev);
        if (e == cudaSuccess) e = cudaDeviceSynchronize();
        if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_status, &zero, sizeof(zero));
        if (e != cudaSuccess && first == cudaSuccess) first = e;
    }
    const cudaError_t e = cudaSetDevice(current);
    return (int)(first != cudaSuccess ? first : e);
}

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_mx4_gemm(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, void* Y, int y_type,
                              int M, int N, int K, int format, const float* alpha, void* stream) {
    return run_mx4(x_codes, x_scales, w_codes, w_scales, nullptr, Y, y_type, M, N, K, 1, format, alpha, 0, stream);
}

extern "C" int elutq_mx4_gemm_grouped(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, const int* offsets,
                                      void* Y, int y_type, int M, int N, int K, int E, int format, const float* alpha, void* stream) {
    if (!offsets) return ELUTQ_ERR_INVALID_ARG;
    return run_mx4(x_codes, x_scales, w_codes, w_scales, offsets, Y, y_type, M, N, K, E, format, alpha, 0, stream);
}

extern "C" int elutq_mx4_test_wait_expiry(const void* x_codes, const void* x_scales, const void* w_codes, const void* w_scales, void* Y, int y_type,
                                          int M, int N, int K, int format, unsigned wait_limit, void* stream) {
    if (wait_limit == 0) return ELUTQ_ERR_INVALID_ARG;
    return run_mx4(x_codes, x_scales, w_codes, w_scales, nullptr, Y, y_type, M, N, K, 1, format, nullptr, wait_limit, stream);
}
