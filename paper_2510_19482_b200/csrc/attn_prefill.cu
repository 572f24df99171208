// Attention over whole prompts that lie one behind the other, causal or not, with grouped heads, on tcgen05.
//
//   o_i = sum_j 2^(x_ij - m_i) V_j / sum_j 2^(x_ij - m_i),   x_ij = log2(e) scale q_i . K_j,   j < n_k - n_q + 1 + i (causal) or j < n_k
//
// work       A CTA takes two tiles of 128 query rows that share keys: neighbouring (row block, query head) pairs of one key head, so the heads of a group on the same rows
//            where a group is even.  Keys and values come in tiles of 128 by TMA (128-byte swizzle) into one ring; the two query tiles use each of them once.
//            One CTA to an SM goes through every n-th of such pairs of tiles, those with the longest rows first, each other round backwards.
// roles      A warpgroup for each query tile: a thread owns a row, reads its 128 scores from tensor memory, forms the weights and writes them back as 16-bit values
//            over the scores, where the tensor core takes them as the first operand of P V, in two parts.  One thread issues all MMAs: while one tile's scores are with
//            its warpgroup, the other tile's products run.  One warp finds the next pair of tiles and loads, while the last one is still being worked on; one replaces what lies
//            behind a sequence by zeros.
// memory     Tensor memory: scores / weights and results of both tiles, 4 x 128 columns.
// softmax    A row's maximum moves only when a part of a tile rises more than 2^10 above it; the warp then scales its results in tensor memory.  Weights stay below 2^14.
//            Maximum, sum and results are fp32.  Weights go to 16 bits because the tensor core takes them so, off by 2^-12 of themselves in fp16 and 2^-9 in bf16, next to
//            results of 16 bits; their sum takes them as they were.  (Against 64 bits results are off 1.2 to 1.4 times as far as with weights of fp32, most where one outdoes all
//            others.)  (The unit for exponentials takes 8 cycles a warp, 2048 for a tile of both warpgroups, as long as the tensor core's products of
//            it.  A quarter of them formed by a polynomial instead brought nothing: 8192 tokens 439 -> 461 us; long runs are at the power limit.)
// masked     Scores are selected, and V rows behind a sequence (the next one's, or whatever lies behind the last) are replaced by zeros in shared memory.  A weight of zero
//            times a V that is not finite would still be NaN, for a row in front of such a token in the same tile: rows whose result is not finite are formed again,
//            one by one, from what they see.  So are rows whose scores pass 2^22.  Other inputs never come there.
//
// Bound: a tile's softmax and its hand-overs, and the power limit in long runs.  8192 tokens of 32 heads over 8 of 128 in bf16 432 to 450 us in a graph, 1.12 to 1.16 of the operations at the
// sustained rate; all keys seen 973, 1.26.  Few and even items run in rounds: 1024 and 867 tokens over 3500 more are 240 items of 29 to 36 tiles for 148 SMs, so the busiest has 63 tiles and
// the mean is 52 (121 us, 1.39; 1.16 of what the busiest SM's tiles come to).
//
// Every wait is bounded: the thread whose wait runs out raises the device's status word, and all roles leave their loops.
#include <atomic>

#include "kv.cuh"
#include "tensor_map.cuh"

namespace elutq {

namespace {

constexpr int kTile = 128;                 // query rows of a tile, keys of a tile
constexpr int kRing = 4;                   // tiles of keys and values on their way
constexpr int kMmaWarp = 8, kLoadWarp = 9, kTailWarp = 10;
constexpr int kStage = 8 * 32 * 128;        // where results become rows: 32 rows of 128 bytes for each warp
constexpr int kItems = 2;                  // pairs of tiles that the roles know of at once
constexpr int kThreads = 384;
// Registers of a thread: of the launch's 168 the two warpgroups of the softmax get more, the third less (2 x 208 + 80 is below 3 x 168).
constexpr int kRowRegs = 208, kOtherRegs = 80;
constexpr float kBase = 4.0f, kRise = 14.0f; // 2^(x - m + 4), m moved when that would pass 2^14
constexpr float kLarge = 4194304.0f;         // 2^22: scores beyond it leave less than half a bit behind the point in an offset
constexpr unsigned long long kWaitNs = 1000000000ull;
constexpr int kFirstPart = 96;               // keys of a tile whose weights are handed over first
constexpr int kScores = 0, kResults = 256;   // columns of tensor memory, 128 for each tile

__device__ unsigned g_attn_status;         // 0, or what a launch on this device gave up on

struct PrefillArgs {
    const int *cu_q, *cu_k;
    const uint8_t *q, *k, *v;
    uint8_t* out;
    long long ldq, ldk, ldv, ldo;          // elements between tokens
    int B, max_q, total_q, total_k;
    int heads, group;                      // key heads; query heads of each
    int causal;
    float scale;                           // times log2(e)
    int test;                              // 1: no load is issued; 2: no product is
    uint32_t wait_limit;                   // polls (tests); a wait of a second runs out whatever this is
};

enum { kBarQ = 0, kBarQFree = 2, kBarFull = 4, kBarEmpty = kBarFull + kRing, kBarScores = kBarEmpty + kRing, kBarWeights = kBarScores + 2, kBarPart = kBarWeights + 4, kBarDone = kBarPart + 2,
       kBarResults = kBarDone + 2, kBarTail = kBarResults + 2, kBarItem = kBarTail + kRing, kBarItemFree = kBarItem + kItems, kBarDrain = kBarItemFree + kItems, kNumBars };

struct Tile {
    int head, row0, tiles;                 // query head, first row in the sequence, tiles of keys
};
// A pair of query tiles
struct Item {
    int q0, nq, k0, nk;                    // the sequence's queries and keys; nq < 0: there are no more
    int h, kv0;                            // key head; how many tiles of keys and values were loaded before
    Tile t[2];
    __device__ __forceinline__ int most() const { return max(t[0].tiles, t[1].tiles); }
    __device__ __forceinline__ bool tail() const { return most() > 0 && most() * kTile > nk; }       // the last tile of keys reaches behind the sequence
};

template <int D>
constexpr int kTileBytes = kTile * D * 2;
template <int D>
constexpr int kSmem = (2 + kRing) * kTileBytes<D> + kStage + kNumBars * 8 + 16 + kItems * (int)sizeof(Item);

// Polls until the phase is over (true), something in the CTA has given up, or the time or the polls are (false).  gave_up[1] counts what rows formed one by one have seen: the
// time begins again while it moves.
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity, volatile const uint32_t* gave_up, uint32_t limit) {
    if (try_wait(bar, parity)) return true;
    unsigned long long since = 0;
    uint32_t seen = 0;
    for (uint32_t i = 1; i < limit; ++i) {
        if (try_wait(bar, parity)) return true;
        if ((i & 15u) == 0u) {
            if (gave_up != nullptr && *gave_up) return false;
            const unsigned long long t = now_ns();
            const uint32_t now = gave_up != nullptr ? gave_up[1] : 0u;
            if (since == 0 || now != seen) {
                since = t;
                seen = now;
            } else if (t - since > kWaitNs) {
                return false;
            }
        }
    }
    return false;
}
__device__ __forceinline__ bool wait_alone(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t limit) {
    if (poll(bar, parity, gave_up, limit)) return true;
    *gave_up = 1;
    atomicExch(&g_attn_status, kStatusWaitExpired);
    return false;
}
// By a whole warp, with one answer for it.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile uint32_t* gave_up, uint32_t limit) {
    const bool ok = poll(bar, parity, gave_up, limit);
    if (__all_sync(0xffffffffu, ok)) return true;
    if (!ok) {
        *gave_up = 1;
        atomicExch(&g_attn_status, kStatusWaitExpired);
    }
    __syncwarp();
    return false;
}
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// K-major, 128-byte swizzle, 1024 bytes per 8 rows
__device__ __forceinline__ uint64_t rows_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)1 << 16) | ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// The same tile with the rows as the inner index of the product: 64 columns (128 bytes) to a swizzled block, 1024 bytes per 8 rows, the next 64 columns a whole block on
__device__ __forceinline__ uint64_t columns_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | ((uint64_t)((kTile * 128) >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
#define ELUTQ_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define ELUTQ_B8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define ELUTQ_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
__device__ __forceinline__ void tmem_ld32(uint32_t* r, uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
                 "%26, %27, %28, %29, %30, %31}, [%32];"
                 : ELUTQ_R8(r, 0), ELUTQ_R8(r, 8), ELUTQ_R8(r, 16), ELUTQ_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait32(uint32_t* r) {         // names the registers: nothing may use them earlier
    asm volatile("tcgen05.wait::ld.sync.aligned;" : ELUTQ_B8(r, 0), ELUTQ_B8(r, 8), ELUTQ_B8(r, 16), ELUTQ_B8(r, 24) :: "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, "
                 "%26, %27, %28, %29, %30, %31, %32};"
                 :: "r"(addr), ELUTQ_I8(r, 0), ELUTQ_I8(r, 8), ELUTQ_I8(r, 16), ELUTQ_I8(r, 24) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 :: "r"(addr), ELUTQ_I8(r, 0), ELUTQ_I8(r, 8) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
template <bool BF16>
__device__ __forceinline__ float2 unpack(uint32_t v) {
    float y[2];
    word_values<BF16 ? ELUTQ_TYPE_BF16 : ELUTQ_TYPE_F16>(y, v);
    return make_float2(y[0], y[1]);
}

// One row by a warp, from the first `sees` keys: a lane takes D / 32 dimensions, four keys on their way.  Weights are at most half of one over the number of keys, so that sums of the
// largest values are finite.
template <int D, bool BF16>
__device__ __noinline__ void row_alone(const uint8_t* q, const uint8_t* k, const uint8_t* v, long long ldk, long long ldv, int sees, float scale, uint8_t* out, volatile uint32_t* seen) {
    constexpr int W = D / 64, AT_ONCE = 4;             // words of a lane
    const int lane = threadIdx.x & 31;
    float x[2 * W], o[2 * W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 t = unpack<BF16>(reinterpret_cast<const uint32_t*>(q)[lane * W + i]);
        x[2 * i] = t.x; x[2 * i + 1] = t.y;
        o[2 * i] = o[2 * i + 1] = 0.0f;
    }
    const float unit = __uint_as_float((uint32_t)(94 + __clz(sees)) << 23);     // 2^-(bits of sees + 1)
    float top = -INFINITY, sum = 0.0f;
    for (int j0 = 0; j0 < sees; j0 += AT_ONCE) {
        float s[AT_ONCE];
        uint32_t vw[AT_ONCE][W];
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            const long long j = min(j0 + n, sees - 1);
            s[n] = 0.0f;
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 t = unpack<BF16>(__ldg(reinterpret_cast<const uint32_t*>(k + 2 * j * ldk) + lane * W + i));
                vw[n][i] = __ldg(reinterpret_cast<const uint32_t*>(v + 2 * j * ldv) + lane * W + i);
                s[n] = fmaf(x[2 * i], t.x, fmaf(x[2 * i + 1], t.y, s[n]));
            }
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1)
#pragma unroll
            for (int n = 0; n < AT_ONCE; ++n) s[n] += __shfl_xor_sync(0xffffffffu, s[n], d);
#pragma unroll
        for (int n = 0; n < AT_ONCE; ++n) {
            if (j0 + n >= sees) break;
            s[n] *= scale;
            const float m = fmaxf(top, s[n]);  // (a NaN does not move it, and reaches the sum below)
            const float by = top == m ? 1.0f : exp2f(top - m), p = s[n] == -INFINITY ? 0.0f : exp2f(s[n] - m) * unit;
            top = m;
            sum = fmaf(sum, by, p);
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float2 t = unpack<BF16>(vw[n][i]);
                o[2 * i] = fmaf(o[2 * i], by, p * t.x);
                o[2 * i + 1] = fmaf(o[2 * i + 1], by, p * t.y);
            }
        }
        if ((j0 & 0xfff) == 0 && lane == 0) *seen = *seen + 1;
    }
    const float r = 1.0f / sum;
#pragma unroll
    for (int i = 0; i < W; ++i) reinterpret_cast<uint32_t*>(out)[lane * W + i] = sum == 0.0f ? 0u : pack<BF16>(o[2 * i] * r, o[2 * i + 1] * r);
}

// The n-th pair of tiles of all, level by level: level l holds the pairs l of all sequences that have so many, the highest level first.
struct Walk {
    int level, before, here;               // the level, pairs above it, pairs of it
    int mine;                              // pairs of sequence `lane` (the first 32 are asked for again and again)
    int at, passed;                        // where the last pair was found (32 sequences from there on), those of the level in front of it: n only rises
    __device__ __forceinline__ uint32_t have(const PrefillArgs& a, int b0) const {          // of 32 sequences, those that have this level
        const int b = b0 + (threadIdx.x & 31);
        return __ballot_sync(0xffffffffu, (b0 == 0 ? mine : b < a.B ? pairs_of(a, b) : 0) > level);
    }
    __device__ __forceinline__ int pairs_of(const PrefillArgs& a, int b) const {
        const int q0 = min(max(__ldg(a.cu_q + b), 0), a.total_q), nq = min(max(__ldg(a.cu_q + b + 1), q0), a.total_q) - q0;
        return ((min(nq, a.max_q) + kTile - 1) / kTile * a.group + 1) / 2;
    }
    // A long search is seen by those that wait for its result.
    __device__ __forceinline__ void moves(int b0, volatile uint32_t* seen) const {
        if ((b0 & 0x7fff) == 0x7fe0 && (threadIdx.x & 31) == 0) *seen = *seen + 1;
    }
    // by a whole warp, as the next ones
    __device__ void begin(const PrefillArgs& a, volatile uint32_t* seen) {
        before = here = at = passed = 0;
        const int b = threadIdx.x & 31;
        int most = mine = b < a.B ? pairs_of(a, b) : 0;
        for (int b0 = 32; b0 < a.B; b0 += 32) {
            if (b0 + b < a.B) most = max(most, pairs_of(a, b0 + b));
            moves(b0, seen);
        }
        level = __reduce_max_sync(0xffffffffu, most);
    }
    // false: there are no more
    __device__ bool find(const PrefillArgs& a, int n, int& b, int& h, volatile uint32_t* seen) {
        while (n >= before + here) {
            if (level == 0) return false;
            before += here;
            --level;
            at = passed = 0;
            int count = 0;
            for (int b0 = 0; b0 < a.B; b0 += 32) {
                count += __popc(have(a, b0));
                moves(b0, seen);
            }
            here = count * a.heads;
        }
        const int left = n - before, which = left / a.heads;       // of the sequences that have this level
        h = left - which * a.heads;
        for (; at < a.B; at += 32) {
            const uint32_t some = have(a, at);
            if (which - passed < __popc(some)) {
                b = at + __fns(some, 0, which - passed + 1);
                return true;
            }
            passed += __popc(some);
            moves(at, seen);
        }
        return false;
    }
};
// A role's way through the items: its slot in the queue and the parity of its use
struct Queue {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() {
        if (++slot == kItems) { slot = 0; phase ^= 1u; }
    }
};
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Two fp32 values in a register pair
__device__ __forceinline__ unsigned long long pair_of(float x, float y) {
    unsigned long long d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ void halves(unsigned long long v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ unsigned long long fma2(unsigned long long a, unsigned long long b, unsigned long long c) {
    unsigned long long d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ unsigned long long add2(unsigned long long a, unsigned long long b) {
    unsigned long long d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 1) attn_prefill_kernel(const __grid_constant__ CUtensorMap qm, const __grid_constant__ CUtensorMap km, const __grid_constant__ CUtensorMap vm,
                                                                   const PrefillArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    constexpr int BYTES = kTileBytes<D>, HALVES = D / 64;
    uint8_t* stage = smem + (2 + kRing) * BYTES;
    uint64_t* bars = reinterpret_cast<uint64_t*>(stage + kStage);
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + kNumBars);
    volatile uint32_t* gave_up = tmem_slot + 1;
    volatile Item* items = reinterpret_cast<volatile Item*>(tmem_slot + 4);
    const uint32_t bar0 = smem_u32(bars), smem0 = smem_u32(smem);
    auto bar = [&](int i) { return bar0 + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

    if (tid == 0) {
        auto init = [&](int i, int n) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar(i)), "r"(n) : "memory"); };
        // (weights and results: a warpgroup's four warps; items: the MMA thread, the tail's warp and both warpgroups)
        for (int i = 0; i < kNumBars; ++i) init(i, (i >= kBarWeights && i < kBarPart) || (i >= kBarResults && i < kBarTail) ? 4 : i >= kBarItemFree && i < kBarDrain ? 10 : 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        gave_up[0] = gave_up[1] = 0;
    }
    grid_dependency_wait();
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(tmem_slot)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    grid_launch_dependents();              // (with tensor memory in hand: a kernel that waits for this one may want some too)
    const uint32_t tmem = *tmem_slot;
    const uint32_t limit = a.wait_limit;
    auto item_at = [&](int slot) {
        Item it;
        const volatile int* from = reinterpret_cast<const volatile int*>(items + slot);
        int* to = reinterpret_cast<int*>(&it);
#pragma unroll
        for (int i = 0; i < (int)(sizeof(Item) / 4); ++i) to[i] = from[i];
        return it;
    };

    // of the warp that loads: tiles of keys and values; items that had the query tile; a bit for each slot: its last load was announced to the tail's warp, the parity of such uses
    int kv = 0, loaded[2] = {0, 0};
    uint32_t tails = 0, tail_parity = 0;
    if (warp >= kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(kOtherRegs));
        if (warp == kLoadWarp) {
            // ---- items and loads: keys 0, the query tiles, values 0, keys 1, .. ----------------------------------------------------------------------------
            Queue queue;
            Walk walk;
            walk.begin(a, gave_up + 1);
            bool ok = true;
            for (int round = 0; ok; ++round) {
                const int n = round * gridDim.x + (round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
                Item it;
                int b = 0, h = 0;
                const bool some = walk.find(a, n, b, h, gave_up + 1);
                if (some) {
                    it.q0 = min(max(__ldg(a.cu_q + b), 0), a.total_q);
                    it.nq = min(max(__ldg(a.cu_q + b + 1), it.q0), a.total_q) - it.q0;
                    it.k0 = min(max(__ldg(a.cu_k + b), 0), a.total_k);
                    it.nk = min(max(__ldg(a.cu_k + b + 1), it.k0), a.total_k) - it.k0;
                    it.h = h;
                    it.kv0 = kv;
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int count = (min(it.nq, a.max_q) + kTile - 1) / kTile * a.group, at = 2 * walk.level + i, blk = at / a.group;
                        it.t[i].head = at < count ? h * a.group + (at - blk * a.group) : -1;
                        it.t[i].row0 = blk * kTile;
                        const int sees = a.causal ? min(it.nk, min(it.t[i].row0 + kTile, it.nq) + it.nk - it.nq) : it.nk;
                        it.t[i].tiles = at < count ? (max(sees, 0) + kTile - 1) / kTile : 0;
                    }
                } else {
                    it.q0 = it.k0 = it.nk = it.h = it.kv0 = 0;
                    it.nq = -1;
                    it.t[0].head = it.t[0].row0 = it.t[0].tiles = it.t[1].head = it.t[1].row0 = it.t[1].tiles = 0;
                }
                ok = wait_warp(bar(kBarItemFree + queue.slot), queue.phase ^ 1u, gave_up, limit);
                if (!ok) break;
                if (lane == 0) {
                    volatile int* to = reinterpret_cast<volatile int*>(items + queue.slot);
                    const int* from = reinterpret_cast<const int*>(&it);
#pragma unroll
                    for (int i = 0; i < (int)(sizeof(Item) / 4); ++i) to[i] = from[i];
                    arrive(bar(kBarItem + queue.slot));
                }
                queue.next();
                if (!some) break;
                const int most = it.most();
                if (lane == 0 && a.test != 1) {
                    auto load_q = [&](int i) {
                        if (it.t[i].tiles == 0) return true;
                        if (!wait_alone(bar(kBarQFree + i), (uint32_t)(loaded[i] & 1) ^ 1u, gave_up, limit)) return false;
                        ++loaded[i];
                        expect(bar(kBarQ + i), BYTES);
                        for (int s = 0; s < HALVES; ++s) tma_load(smem0 + i * BYTES + s * (kTile * 128), &qm, 64 * s, it.t[i].head, it.q0 + it.t[i].row0, bar(kBarQ + i));
                        return true;
                    };
                    for (int m = 0; m < 2 * most && ok; ++m) {
                        if (m == 1) ok = load_q(0) && load_q(1);
                        const int slot = kv % kRing;
                        if (ok) ok = wait_alone(bar(kBarEmpty + slot), (uint32_t)(kv / kRing & 1) ^ 1u, gave_up, limit);
                        if (!ok) break;
                        const bool tail = m == 2 * most - 1 && it.tail();
                        const int to = tail ? kBarTail + slot : kBarFull + slot;
                        expect(bar(to), BYTES);
                        for (int s = 0; s < HALVES; ++s) tma_load(smem0 + (2 + slot) * BYTES + s * (kTile * 128), m & 1 ? &vm : &km, 64 * s, it.h, it.k0 + (m >> 1) * kTile, bar(to));
                        tails = tail ? tails | 1u << slot : tails & ~(1u << slot);
                        tail_parity ^= (uint32_t)tail << slot;
                        ++kv;
                    }
                }
                kv = __shfl_sync(0xffffffffu, kv, 0);
                ok = __all_sync(0xffffffffu, ok);
            }
        } else if (warp == kTailWarp) {
            // ---- V rows behind a sequence: zeros.  Such a tile is announced to this warp, which then announces it to the MMAs --------------------------------------
            uint32_t parity = 0;                              // a bit for each slot
            for (Queue queue;; queue.next()) {
                if (!wait_warp(bar(kBarItem + queue.slot), queue.phase, gave_up, limit)) break;
                const Item it = item_at(queue.slot);
                __syncwarp();
                if (lane == 0) arrive(bar(kBarItemFree + queue.slot));
                if (it.nq < 0) break;
                if (!it.tail()) continue;
                const int n = it.kv0 + 2 * it.most() - 1, slot = n % kRing;
                if (!wait_warp(bar(kBarTail + slot), parity >> slot & 1u, gave_up, limit)) break;
                parity ^= 1u << slot;
                for (int i = (it.nk - (it.most() - 1) * kTile) * 8 + lane; i < kTile * 8; i += 32)
                    for (int s = 0; s < HALVES; ++s) *reinterpret_cast<uint4*>(smem + (2 + slot) * BYTES + s * (kTile * 128) + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) arrive(bar(kBarFull + slot));
            }
        } else if (warp == kMmaWarp) {
            // ---- MMAs ------------------------------------------------------------------------------------------------------------------------------
            if (elect_one()) {
                constexpr uint32_t kTypes = (1u << 4) | (BF16 ? (1u << 7) | (1u << 10) : 0u);
                constexpr uint32_t kQK = kTypes | (uint32_t)(kTile >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
                constexpr uint32_t kPV = kTypes | (1u << 16) | (uint32_t)(D >> 3) << 17 | (uint32_t)(kTile >> 4) << 24;
                auto scores = [&](int i, int slot) {          // query tile i times the keys of a slot
                    const uint64_t q = rows_desc(smem0 + i * BYTES), k = rows_desc(smem0 + (2 + slot) * BYTES);
#pragma unroll
                    for (int s = 0; s < D / 16; ++s) {
                        const uint64_t at = (uint64_t)((s & 3) * 2 + (s >> 2) * (kTile * 128 >> 4));
                        mma_ss(tmem + kScores + i * kTile, q + at, k + at, kQK, s != 0);
                    }
                    commit(bar(kBarScores + i));
                };
                auto products = [&](int i, int slot, auto part, bool first) {
                    const uint64_t v = columns_desc(smem0 + (2 + slot) * BYTES);
#pragma unroll
                    for (int s = part == 0 ? 0 : kFirstPart / 16; s < (part == 0 ? kFirstPart / 16 : kTile / 16); ++s)
                        mma_ts(tmem + kResults + i * kTile, tmem + kScores + i * kTile + 8 * s, v + (uint64_t)(s * (2048 >> 4)), kPV, !first || s != 0);
                };
                auto full = [&](int n) { return wait_alone(bar(kBarFull + n % kRing), (uint32_t)(n / kRing) & 1u, gave_up, limit); };
                int used[2] = {0, 0}, done[2] = {0, 0};       // items that had the query tile, tiles of weights taken
                bool ok = a.test != 2;
                for (Queue queue; ok; queue.next()) {
                    ok = wait_alone(bar(kBarItem + queue.slot), queue.phase, gave_up, limit);
                    if (!ok) break;
                    const Item it = item_at(queue.slot);
                    arrive(bar(kBarItemFree + queue.slot));
                    if (it.nq < 0) break;
                    const int most = it.most();
                    if (most == 0) continue;
                    ok = full(it.kv0);
                    for (int i = 0; i < 2 && ok; ++i) {
                        if (it.t[i].tiles == 0) continue;
                        ok = wait_alone(bar(kBarQ + i), (uint32_t)used[i] & 1u, gave_up, limit);
                        fence_after();
                        if (ok) scores(i, it.kv0 % kRing);
                        if (it.t[i].tiles == 1) commit(bar(kBarQFree + i));
                    }
                    if (ok) commit(bar(kBarEmpty + it.kv0 % kRing));
                    for (int j = 0; j < most && ok; ++j) {
                        const int v = it.kv0 + 2 * j + 1;
                        for (int i = 0; i < 2 && ok; ++i) {
                            const int tiles = it.t[i].tiles;
                            if (j >= tiles) continue;
                            ok = full(v);
                            // (the results of the item before have been read)
                            if (ok && j == 0) ok = wait_alone(bar(kBarResults + i), (uint32_t)(used[i] & 1) ^ 1u, gave_up, limit);
                            if (ok) ok = wait_alone(bar(kBarWeights + 2 * i), (uint32_t)done[i] & 1u, gave_up, limit);
                            if (!ok) break;
                            fence_after();
                            products(i, v % kRing, IntC<0>{}, j == 0);
                            commit(bar(kBarPart + i));
                            ok = wait_alone(bar(kBarWeights + 2 * i + 1), (uint32_t)done[i] & 1u, gave_up, limit);
                            if (!ok) break;
                            fence_after();
                            products(i, v % kRing, IntC<1>{}, false);
                            ++done[i];
                            if (j + 1 == tiles) {
                                commit(bar(kBarDone + i));
                            } else {
                                ok = full(v + 1);
                                if (ok) scores(i, (v + 1) % kRing);
                                if (j + 2 == tiles) commit(bar(kBarQFree + i));
                            }
                        }
                        if (!ok) break;
                        commit(bar(kBarEmpty + v % kRing));
                        if (j + 1 < most) commit(bar(kBarEmpty + (v + 1) % kRing));
                    }
                    for (int i = 0; i < 2; ++i) used[i] += it.t[i].tiles != 0;
                }
                // (MMAs in flight read shared memory, and their commits arrive there)
                commit(bar(kBarDrain));
                poll(bar(kBarDrain), 0, nullptr, 0xffffffffu);
            }
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(kRowRegs));
        // ---- softmax: a thread to a row -------------------------------------------------------------------------------------------------------------
        const int i = warp >> 2;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, sc = tmem + lanes + kScores + i * kTile, res = tmem + lanes + kResults + i * kTile;
        const unsigned long long scale2 = pair_of(a.scale, a.scale);
        int done = 0, used = 0;                               // tiles of scores, items
        for (Queue queue;; queue.next()) {
            if (!wait_warp(bar(kBarItem + queue.slot), queue.phase, gave_up, limit)) break;
            const int q0 = items[queue.slot].q0, nq = items[queue.slot].nq, k0 = items[queue.slot].k0, nk = items[queue.slot].nk, h = items[queue.slot].h;
            const int head = items[queue.slot].t[i].head, row0 = items[queue.slot].t[i].row0, tiles = items[queue.slot].t[i].tiles;
            __syncwarp();
            if (lane == 0) arrive(bar(kBarItemFree + queue.slot));
            if (nq < 0) break;
            if (head < 0) continue;
            const int row = row0 + (tid & 127), shift = nk - nq;
            const int sees = a.causal ? max(min(nk, row + 1 + shift), 0) : nk;
            float off = kNone;
            unsigned long long sums[2] = {0ull, 0ull};
            bool ok = true;
            for (int j = 0; j < tiles; ++j, ++done) {
                ok = wait_warp(bar(kBarScores + i), (uint32_t)done & 1u, gave_up, limit);
                if (!ok) break;
                fence_after();
                uint32_t s[kTile];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(s + 32 * c, sc + 32 * c);
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld_wait32(s + 32 * c);
                const int left = sees - j * kTile;
                if (__any_sync(0xffffffffu, left < kTile)) {
#pragma unroll
                    for (int c = 0; c < kTile; ++c)
                        if (c >= left) s[c] = 0xff800000u;
                }
                auto part = [&](auto second) {
                    constexpr int FROM = decltype(second)::value ? kFirstPart : 0, TO = decltype(second)::value ? kTile : kFirstPart;
                    float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = FROM; c < TO; c += 2) tops[c / 2 % 4] = max3(tops[c / 2 % 4], __uint_as_float(s[c]), __uint_as_float(s[c + 1]));
                    const float top = max3(fmaxf(tops[0], tops[1]), tops[2], tops[3]);
                    if (__any_sync(0xffffffffu, fmaf(top, a.scale, off) > kRise)) {
                        const float to = top == -INFINITY ? off : fminf(off, kBase - top * a.scale);
                        const float by = exp2_approx(to - off);
                        off = to;
                        const unsigned long long by2 = pair_of(by, by);
#pragma unroll
                        for (int k = 0; k < 2; ++k) sums[k] = fma2(sums[k], by2, 0ull);
                        // (the products of the tiles before are done: the scores came behind them)
                        if (second) {
                            if (!wait_warp(bar(kBarPart + i), (uint32_t)done & 1u, gave_up, limit)) return false;
                            fence_after();
                        }
                        if (second || j > 0) {
#pragma unroll
                            for (int c = 0; c < D / 32; ++c) {
                                uint32_t o[32];
                                tmem_ld32(o, res + 32 * c);
                                tmem_ld_wait32(o);
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
                                tmem_st32(res + 32 * c, o);
                            }
                        }
                    }
                    const unsigned long long off2 = pair_of(off, off);
#pragma unroll
                    for (int c = FROM; c < TO; c += 32) {
                        uint32_t w[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const unsigned long long x2 = fma2(pair_of(__uint_as_float(s[c + 2 * e]), __uint_as_float(s[c + 2 * e + 1])), scale2, off2);
                            float lo, hi;
                            halves(x2, lo, hi);
                            lo = exp2_approx(lo);
                            hi = exp2_approx(hi);
                            sums[e & 1] = add2(sums[e & 1], pair_of(lo, hi));
                            w[e] = pack<BF16>(lo, hi);
                        }
                        tmem_st16(sc + c / 2, w);
                    }
                    tmem_st_wait();
                    fence_before();
                    __syncwarp();
                    if (lane == 0) arrive(bar(kBarWeights + 2 * i + (second ? 1 : 0)));
                    return true;
                };
                ok = part(IntC<0>{}) && part(IntC<1>{});
                if (!ok) break;
            }
            if (!ok) break;
            float x, y;
            halves(add2(sums[0], sums[1]), x, y);
            const float sum = x + y, r = sum == 0.0f ? 0.0f : 1.0f / sum;
            float check = 0.0f;
            if (tiles > 0) {
                if (!wait_warp(bar(kBarDone + i), (uint32_t)used & 1u, gave_up, limit)) break;
                ++used;
                fence_after();
            }
            // 64 columns at a time through shared memory, so that eight lanes write 128 bytes of a row.  (A lane's own row, 16 bytes at a time: 4 us an item, now 1.)
            uint8_t* turned = stage + warp * (32 * 128);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
                uint32_t o[64];
                if (tiles > 0) {
                    tmem_ld32(o, res + 64 * c);
                    tmem_ld32(o + 32, res + 64 * c + 32);
                    tmem_ld_wait32(o);
                    tmem_ld_wait32(o + 32);
                    if (c == D / 64 - 1) {                    // the next item's products may come
                        fence_before();
                        __syncwarp();
                        if (lane == 0) arrive(bar(kBarResults + i));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 64; ++e) o[e] = 0u;
                }
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const float lo = __uint_as_float(o[2 * e]) * r, hi = __uint_as_float(o[2 * e + 1]) * r;
                    check = fmaf(0.0f, lo, fmaf(0.0f, hi, check));
                    o[e] = pack<BF16>(lo, hi);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(turned + lane * 128 + 16 * (e ^ (lane & 7))) = make_uint4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
                __syncwarp();
                const int first = row0 + 32 * (warp & 3) + (lane >> 3);
                uint8_t* to = a.out + 2 * ((long long)(q0 + first) * a.ldo + (long long)head * D) + 128 * c + 16 * (lane & 7);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint4 v = *reinterpret_cast<const uint4*>(turned + (4 * e + (lane >> 3)) * 128 + 16 * ((lane & 7) ^ (4 * e + (lane >> 3) & 7)));
                    if (first + 4 * e < nq) *reinterpret_cast<uint4*>(to + 8 * e * a.ldo) = v;
                }
                __syncwarp();
            }
            // (NaN: something was not finite.  A large offset: fmaf(x, scale, offset) has its rounding in it, which may be anything)
            uint32_t again = __ballot_sync(0xffffffffu, (check != 0.0f || (tiles > 0 && fabsf(off) > kLarge && sees > 0)) && row < nq);
            while (again != 0) {
                const int l = __ffs(again) - 1;
                again &= again - 1;
                const int rr = row0 + 32 * (warp & 3) + l;
                __syncwarp();                                 // (the row's own stores come first)
                row_alone<D, BF16>(a.q + 2 * ((long long)(q0 + rr) * a.ldq + (long long)head * D), a.k + 2 * ((long long)k0 * a.ldk + (long long)h * D),
                                   a.v + 2 * ((long long)k0 * a.ldv + (long long)h * D), a.ldk, a.ldv, a.causal ? max(min(nk, rr + 1 + shift), 0) : nk, a.scale,
                                   a.out + 2 * ((long long)(q0 + rr) * a.ldo + (long long)head * D), gave_up + 1);
            }
        }
    }
    fence_before();
    __syncthreads();
    if (warp == kLoadWarp && lane == 0 && *gave_up) {
        // what is on its way lands before the CTA leaves (here, as another role may give up when the loads are all issued)
        for (int i = 0; i < 2; ++i)
            if (loaded[i] > 0) poll(bar(kBarQ + i), (uint32_t)(loaded[i] - 1) & 1u, nullptr, 0xffffffffu);
        for (int n = max(0, kv - kRing); n < kv; ++n) {
            const int slot = n % kRing;
            if (tails >> slot & 1u) poll(bar(kBarTail + slot), (tail_parity >> slot & 1u) ^ 1u, nullptr, 0xffffffffu);
            else poll(bar(kBarFull + slot), (uint32_t)(n / kRing) & 1u, nullptr, 0xffffffffu);
        }
    }
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(512) : "memory");
}

// [tokens][heads][D] of 16-bit values, boxes of 64 values x 128 tokens of one head
int rows_map(CUtensorMap* map, const void* base, int tokens, int heads, int D, long long ld, bool bf16) {
    const EncodeTiledFn enc = encode_tiled_fn();
    if (!enc) return (int)cudaErrorNotSupported;
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)tokens}, strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)ld * 2};
    const cuuint32_t box[3] = {64, 1, kTile}, elem[3] = {1, 1, 1};
    return enc(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
               ? 0 : (int)cudaErrorInvalidValue;
}

std::atomic<unsigned long long> g_devices{0};      // devices that this was launched on, a bit for each number modulo 64
inline unsigned long long device_bit(int dev) { return 1ull << (dev & 63); }

template <int D, bool BF16>
int launch_prefill(const CUtensorMap& qm, const CUtensorMap& km, const CUtensorMap& vm, const PrefillArgs& a, dim3 grid, cudaStream_t stream) {
    // once for each device (a call would take half a microsecond of the host's time)
    static std::atomic<unsigned long long> ready{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return (int)e;
    const unsigned long long bit = dev < 64 ? 1ull << dev : 0ull;
    if (!(ready.load(std::memory_order_acquire) & bit)) {
        e = cudaFuncSetAttribute(attn_prefill_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem<D>);
        if (e != cudaSuccess) return (int)e;
        ready.fetch_or(bit, std::memory_order_release);
    }
    if (!(g_devices.load(std::memory_order_relaxed) & device_bit(dev))) g_devices.fetch_or(device_bit(dev));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem<D>;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, attn_prefill_kernel<D, BF16>, qm, km, vm, a);
    if (e == cudaSuccess) count_launch(1);
    return (int)e;
}

int run_prefill(const void* q, long long ldq, const void* k, long long ldk, const void* v, long long ldv, void* out, long long ldo, int type, const int* cu_q, const int* cu_k, int B,
                int max_q, int total_q, int total_k, int n_q_heads, int heads, int D, float scale, unsigned flags, uint32_t test_limit, void* stream) {
    if (!q || !k || !v || !out || out == q || out == k || out == v || !cu_q || !cu_k || B <= 0 || max_q <= 0 || total_q <= 0 || total_k <= 0 || n_q_heads <= 0 || heads <= 0) return ELUTQ_ERR_INVALID_ARG;
    if ((type != ELUTQ_TYPE_F16 && type != ELUTQ_TYPE_BF16) || (flags & ~ELUTQ_ATTN_ALL_KEYS) || !(scale > 0.0f) || !(scale < 1e30f)) return ELUTQ_ERR_INVALID_ARG;
    if (D != 64 && D != 128) return ELUTQ_ERR_UNSUPPORTED;
    if (n_q_heads % heads != 0) return ELUTQ_ERR_SHAPE;
    int st;
    if ((st = kv_rows_check(q, ldq, n_q_heads, D)) != ELUTQ_OK || (st = kv_rows_check(k, ldk, heads, D)) != ELUTQ_OK || (st = kv_rows_check(v, ldv, heads, D)) != ELUTQ_OK ||
        (st = kv_rows_check(out, ldo, n_q_heads, D)) != ELUTQ_OK)
        return st;
    if (!mx4_aligned(cu_q, 4) || !mx4_aligned(cu_k, 4)) return ELUTQ_ERR_ALIGN;
    // strides of a tensor map are below 2^40 bytes; coordinates and row numbers 32 bits; blocks of a launch
    const long long most_ld = 1LL << 38;
    const int group = n_q_heads / heads;
    // (items are counted in 32 bits: at most one more for each sequence than the queries' tiles have pairs)
    const long long blocks = ((long long)(max_q < total_q ? max_q : total_q) + kTile - 1) / kTile, pairs = (blocks * group + 1) / 2;
    const long long total_items = (((long long)total_q / kTile + B) * group / 2 + B) * heads;
    if (ldq > most_ld || ldk > most_ld || ldv > most_ld || total_q > 0x3fffffff || total_k > 0x3fffffff || total_items > 0x3fffffffLL || total_items < 0) return ELUTQ_ERR_SHAPE;
    const Rows results = {out, ldo, total_q, n_q_heads};
    if (rows_meet(results, {q, ldq, total_q, n_q_heads}, D) || rows_meet(results, {k, ldk, total_k, heads}, D) || rows_meet(results, {v, ldv, total_k, heads}, D)) return ELUTQ_ERR_INVALID_ARG;
    PrefillArgs a;
    a.cu_q = cu_q; a.cu_k = cu_k;
    a.q = (const uint8_t*)q; a.k = (const uint8_t*)k; a.v = (const uint8_t*)v;
    a.out = (uint8_t*)out;
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
    a.B = B;
    a.max_q = (int)((((long long)max_q + kTile - 1) / kTile * kTile < 0x7fffff00LL) ? ((long long)max_q + kTile - 1) / kTile * kTile : 0x7fffff00LL);
    a.total_q = total_q; a.total_k = total_k;
    a.heads = heads;
    a.group = group;
    a.causal = (flags & ELUTQ_ATTN_ALL_KEYS) == 0;
    a.scale = scale * 1.44269504088896340736f;
    a.test = test_limit == 0 ? 0 : test_limit & ELUTQ_ATTN_TEST_LOADS ? 2 : 1;
    a.wait_limit = test_limit != 0 ? test_limit & ~ELUTQ_ATTN_TEST_LOADS : 0xffffffffu;
    const bool bf16 = type == ELUTQ_TYPE_BF16;
    CUtensorMap qm, km, vm;
    int ce = rows_map(&qm, q, total_q, n_q_heads, D, ldq, bf16);
    if (ce == 0) ce = rows_map(&km, k, total_k, heads, D, ldk, bf16);
    if (ce == 0) ce = rows_map(&vm, v, total_k, heads, D, ldv, bf16);
    const long long items = pairs * B * heads;
    const dim3 grid((unsigned)(items < device_sm_count() ? items : device_sm_count()));
    if (ce == 0)
        ce = D == 128 ? (bf16 ? launch_prefill<128, true>(qm, km, vm, a, grid, (cudaStream_t)stream) : launch_prefill<128, false>(qm, km, vm, a, grid, (cudaStream_t)stream))
                      : (bf16 ? launch_prefill<64, true>(qm, km, vm, a, grid, (cudaStream_t)stream) : launch_prefill<64, false>(qm, km, vm, a, grid, (cudaStream_t)stream));
    if (ce == 0) return ELUTQ_OK;
    note_cuda_error(ce);
    return ELUTQ_ERR_CUDA;
}

}  // namespace

int attn_status(unsigned* word, cudaStream_t stream) {
    *word = 0;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || !(g_devices.load() & device_bit(dev))) return (int)e;
    e = cudaMemcpyFromSymbolAsync(word, g_attn_status, sizeof(*word), 0, cudaMemcpyDeviceToHost, stream);
    return (int)(e != cudaSuccess ? e : cudaStreamSynchronize(stream));
}
int attn_clear_status() {
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
        if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_attn_status, &zero, sizeof(zero));
        if (e != cudaSuccess && first == cudaSuccess) first = e;
    }
    const cudaError_t e = cudaSetDevice(current);
    return (int)(first != cudaSuccess ? first : e);
}

}  // namespace elutq

using namespace elutq;

extern "C" int elutq_attn_prefill(const void* q, long long ldq, const void* k, long long ldk, const void* v, long long ldv, void* out, long long ldo, int type, const int* cu_q,
                                  const int* cu_k, int B, int max_q, int total_q, int total_k, int n_q_heads, int heads, int head_dim, float scale, unsigned flags, void* stream) {
    return run_prefill(q, ldq, k, ldk, v, ldv, out, ldo, type, cu_q, cu_k, B, max_q, total_q, total_k, n_q_heads, heads, head_dim, scale, flags, 0, stream);
}

extern "C" int elutq_attn_test_wait_expiry(const void* q, long long ldq, const void* k, long long ldk, const void* v, long long ldv, void* out, long long ldo, int type, const int* cu_q,
                                           const int* cu_k, int B, int max_q, int total_q, int total_k, int n_q_heads, int heads, int head_dim, float scale, unsigned flags,
                                           unsigned wait_limit, void* stream) {
    if ((wait_limit & ~ELUTQ_ATTN_TEST_LOADS) == 0) return ELUTQ_ERR_INVALID_ARG;
    return run_prefill(q, ldq, k, ldk, v, ldv, out, ldo, type, cu_q, cu_k, B, max_q, total_q, total_k, n_q_heads, heads, head_dim, scale, flags, wait_limit, stream);
}
