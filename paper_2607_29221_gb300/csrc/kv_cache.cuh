// What the kernels of the key/value cache share: slot addressing with the
// checks that keep every access inside the pool, and the element types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mosaic_internal.cuh"

namespace mosaic {
namespace {

// n / d for 0 <= n < 2^31 by a multiply and a shift (Granlund and Montgomery,
// "Division by invariant integers using multiplication", 1994).
struct FastDiv {
    uint32_t d, mul, shift;
    explicit FastDiv(uint32_t d_) : d(d_), mul(0), shift(0) {
        while ((1ull << shift) < d) ++shift;
        mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (__umulhi(n, mul) + n) >> shift; }
};

// A cache as the kernels see it.
struct KvView {
    mosaic_kv_cache c;
    FastDiv page;
    explicit KvView(const mosaic_kv_cache &cache) : c(cache), page((uint32_t)cache.page_size) {}

    __device__ __forceinline__ int64_t slots() const { return c.table_cols * c.page_size; }
    // Length i, clamped to [0, max_len] and the table.
    __device__ __forceinline__ int length(const int32_t *lens, int64_t i, int64_t max_len) const {
        int64_t n = lens[i];
        n = n < max_len ? n : max_len;
        n = n < slots() ? n : slots();
        return n > 0 ? (int)n : 0;
    }
    // Page of slot s of sequence i and the offset in it; -1 without one.
    // 0 <= s < slots() and 0 <= i < seqs are the caller's.
    __device__ __forceinline__ int page_of(int64_t i, uint32_t s, uint32_t &off) const {
        const uint32_t col = page.div(s);
        off = s - col * page.d;
        const int id = c.table[i * c.ld_table + col];
        return (uint32_t)id < (uint64_t)c.pages ? id : -1;
    }
    __device__ __forceinline__ int64_t element(int id, int h, uint32_t off) const {
        return id * c.page_stride + h * c.head_stride + off * c.slot_stride;
    }
    // Index into position and weight.
    __device__ __forceinline__ int64_t mark(int id, int h, uint32_t off) const {
        return ((int64_t)id * c.kv_heads + h) * c.page_size + off;
    }
};

inline int64_t kv_element_bytes(int type) { return type == MOSAIC_KV_F32 ? 4 : 2; }

// What every call asks of a cache.
inline mosaic_status kv_check(const mosaic_kv_cache *c) {
    if (!c) return MOSAIC_ERR_ARG;
    if (c->type < MOSAIC_KV_F32 || c->type > MOSAIC_KV_F16) return MOSAIC_ERR_ARG;
    if (c->kv_heads < 1 || c->kv_heads > 65535 || c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 ||
        c->page_size < 1 || c->page_size > 65536 || c->pages < 1 || c->pages > 0x7fffffff || c->seqs < 0 ||
        c->seqs > (1 << 24) || c->table_cols < 1 || c->table_cols > 0x7fffffff || c->ld_table < c->table_cols)
        return MOSAIC_ERR_SHAPE;
    // Slots are counted in 31 bits, also at the end of a unit or group of look-ups (512 slots at
    // most) that begins inside a sequence.
    if (c->table_cols * c->page_size > ((int64_t)1 << 31) - 1024) return MOSAIC_ERR_SHAPE;
    if (c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0) return MOSAIC_ERR_SHAPE;
    if (!c->k || !c->v || (!c->table && c->seqs > 0)) return MOSAIC_ERR_ARG;
    const int64_t unit = 16 / kv_element_bytes(c->type);
    if (!aligned16(c->k) || !aligned16(c->v) || c->page_stride % unit || c->head_stride % unit || c->slot_stride % unit)
        return MOSAIC_ERR_ALIGN;
    return MOSAIC_OK;
}

template <class T> struct Elem;
template <> struct Elem<float> {
    static __device__ __forceinline__ float to(float x) { return x; }
    static __device__ __forceinline__ float from(float x) { return x; }
};
template <> struct Elem<__nv_bfloat16> {
    static __device__ __forceinline__ float to(__nv_bfloat16 x) { return __bfloat162float(x); }
    static __device__ __forceinline__ __nv_bfloat16 from(float x) { return __float2bfloat16_rn(x); }
};
template <> struct Elem<__half> {
    static __device__ __forceinline__ float to(__half x) { return __half2float(x); }
    static __device__ __forceinline__ __half from(float x) { return __float2half_rn(x); }
};

}  // namespace
}  // namespace mosaic
