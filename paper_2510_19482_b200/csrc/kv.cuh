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

// The status words of the prompts' attention, one a device (attn_prefill.cu): as mx4_status and mx4_clear_status.
int attn_status(unsigned* word, cudaStream_t stream);
int attn_clear_status();

}  // namespace elutq
