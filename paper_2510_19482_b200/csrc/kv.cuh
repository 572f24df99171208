// The paged cache of keys and values: what the entries that write it, read it and attend over it share.
//
//   k, v      [n_pages][heads][page_size] rows of head_dim values: 16 bits, E4M3 (a byte each) or NVFP4 codes (half a byte, the even column in the low half)
//   scales    NVFP4: [n_pages][heads][page_size] rows of head_dim / 16 bytes, E4M3 (sign bit clear, 127 = NaN)
//   factors   float [heads]: a stored value times it is the value that it stands for
// A token's slot is page * page_size + place in the page; page p's rows of head h start at row (p * heads + h) * page_size.
#pragma once

#include "mx4.cuh"

namespace elutq {

struct KvView {
    uint8_t *k, *v, *ks, *vs;
    const float *kf, *vf;
    int n_pages, heads, page_size;
    Div page;
};

inline int kv_row_bytes(int format, int head_dim) { return format == ELUTQ_KV_16 ? 2 * head_dim : format == ELUTQ_KV_E4M3 ? head_dim : head_dim / 2; }

// What every entry asks of a cache.
inline int kv_check(const elutq_kv_cache* c) {
    if (!c || !c->k || !c->v || c->n_pages <= 0 || c->heads <= 0 || c->page_size <= 0) return ELUTQ_ERR_INVALID_ARG;
    if (c->format < ELUTQ_KV_16 || c->format > ELUTQ_KV_NVFP4 || (c->type != ELUTQ_TYPE_F16 && c->type != ELUTQ_TYPE_BF16)) return ELUTQ_ERR_INVALID_ARG;
    if (c->format == ELUTQ_KV_NVFP4 && (!c->k_scales || !c->v_scales)) return ELUTQ_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return ELUTQ_ERR_UNSUPPORTED;
    if (c->page_size % 16 != 0 || (long long)c->n_pages * c->page_size > 0x7fffffffLL) return ELUTQ_ERR_SHAPE;
    if (!mx4_aligned(c->k, 32) || !mx4_aligned(c->v, 32)) return ELUTQ_ERR_ALIGN;
    if (c->format == ELUTQ_KV_NVFP4 && (!mx4_aligned(c->k_scales, 16) || !mx4_aligned(c->v_scales, 16))) return ELUTQ_ERR_ALIGN;
    if (!mx4_aligned(c->k_factor, 4) || !mx4_aligned(c->v_factor, 4)) return ELUTQ_ERR_ALIGN;
    return ELUTQ_OK;
}
inline KvView kv_view(const elutq_kv_cache* c) {
    KvView w;
    w.k = (uint8_t*)c->k;
    w.v = (uint8_t*)c->v;
    w.ks = (uint8_t*)c->k_scales;
    w.vs = (uint8_t*)c->v_scales;
    // (16-bit values stand for themselves)
    w.kf = c->format == ELUTQ_KV_16 ? nullptr : c->k_factor;
    w.vf = c->format == ELUTQ_KV_16 ? nullptr : c->v_factor;
    w.n_pages = c->n_pages;
    w.heads = c->heads;
    w.page_size = c->page_size;
    w.page.set(c->page_size);
    return w;
}
// Rows of tokens, heads of head_dim values side by side: the distance between tokens holds them, and 16-byte pieces start on 16 bytes.
inline int kv_rows_check(const void* p, long long ld, int heads, int head_dim) {
    if (ld < (long long)heads * head_dim) return ELUTQ_ERR_SHAPE;
    return !mx4_aligned(p, 16) || ld % 8 != 0 ? ELUTQ_ERR_ALIGN : ELUTQ_OK;
}
// Some row of a meets some row of b: rows of `heads` heads of D values of 16 bits, ld apart.  Exact where rows are the same distance apart (parts of one buffer); otherwise the first row of each
// is looked at with the other's rows.
struct Rows {
    const void* p;
    long long ld, n;
    int heads;
};
inline bool rows_meet(const Rows& a, const Rows& b, int D) {
    auto down = [](long long x, long long by) { return x / by - (x % by < 0 ? 1 : 0); };
    // [0, wa) meets [d + k L, d + k L + wb) for a k in [first, last]
    auto meet = [&](long long wa, long long wb, long long d, long long L, long long first, long long last) {
        const long long most = down(wa - d - 1, L), k = most < last ? most : last;       // the last one that begins in front of the end
        return k >= first && d + k * L + wb > 0;
    };
    const long long wa = 2LL * a.heads * D, wb = 2LL * b.heads * D, d = (long long)reinterpret_cast<uintptr_t>(b.p) - (long long)reinterpret_cast<uintptr_t>(a.p);
    auto bytes = [](long long ld) { return 2 * (ld < 1LL << 60 ? ld : 1LL << 60); };
    const long long la = bytes(a.n > 1 ? a.ld : b.ld), lb = bytes(b.n > 1 ? b.ld : a.ld);
    if (la == lb) return meet(wa, wb, d, la, 1 - a.n, b.n - 1);
    return meet(wa, wb, d, lb, 0, b.n - 1) || meet(wb, wa, -d, la, 0, a.n - 1);
}
// ... other than by being the same rows
inline bool rows_meet_apart(const Rows& a, const Rows& b, int D) {
    return !(a.p == b.p && a.heads == b.heads && a.n == b.n && (a.ld == b.ld || a.n == 1)) && rows_meet(a, b, D);
}

// ---- softmax, for both kernels of attention -----------------------------------------------
constexpr float kNone = 3e38f;               // offset of a row that has seen no key: any score rises above it

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Two values in 16 bits, the first in the low half
template <bool BF16>
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    uint32_t d;
    if constexpr (BF16) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
    return d;
}

// The status words of the prompts' attention, one a device (attn_prefill.cu): as mx4_status and mx4_clear_status.
int attn_status(unsigned* word, cudaStream_t stream);
int attn_clear_status();

}  // namespace elutq
