// What the kernels of the key/value cache share: slot addressing with the
// checks that keep every access inside the pool, and the element types.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "mosaic_internal.cuh"

namespace mosaic {

struct Q4 {};   // the element type of 4-bit caches

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

inline int64_t kv_element_bytes(int type) { return type == MOSAIC_KV_F32 ? 4 : type == MOSAIC_KV_Q4 ? 1 : 2; }
// Bytes of a cached row: 4-bit rows are codes, then step and base of every
// kQ4Group channels, padded to 16 bytes.
constexpr int kQ4Group = 32;
inline int64_t kv_row_bytes(int type, int64_t head_dim) {
    return type == MOSAIC_KV_Q4 ? (5 * head_dim / 8 + 15) / 16 * 16 : head_dim * kv_element_bytes(type);
}

// A cache as the kernels see it.
struct KvView {
    mosaic_kv_cache c;
    FastDiv page;
    int row16;   // 16-byte chunks of a row
    explicit KvView(const mosaic_kv_cache &cache)
        : c(cache), page((uint32_t)cache.page_size), row16((int)(kv_row_bytes(cache.type, cache.head_dim) + 15) / 16) {}

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

// What every call asks of a cache.
inline mosaic_status kv_check(const mosaic_kv_cache *c) {
    if (!c) return MOSAIC_ERR_ARG;
    if (c->type < MOSAIC_KV_F32 || (c->type > MOSAIC_KV_F16 && c->type != MOSAIC_KV_Q4)) return MOSAIC_ERR_ARG;
    if (c->kv_heads < 1 || c->kv_heads > 65535 || c->head_dim < 8 || c->head_dim > 256 || c->head_dim % 8 ||
        c->page_size < 1 || c->page_size > 65536 || c->pages < 1 || c->pages > 0x7fffffff || c->seqs < 0 ||
        c->seqs > (1 << 24) || c->table_cols < 1 || c->table_cols > 0x7fffffff || c->ld_table < c->table_cols)
        return MOSAIC_ERR_SHAPE;
    if (c->type == MOSAIC_KV_Q4 && c->head_dim % kQ4Group) return MOSAIC_ERR_SHAPE;
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

// (x & mask) | bits as one instruction (the compiler makes two of it where both are constants).
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t mask, uint32_t bits) {
    uint32_t y;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(y) : "r"(x), "r"(mask), "r"(bits));
    return y;
}
__device__ __forceinline__ __half2 as_half2(uint32_t x) { return *reinterpret_cast<const __half2 *>(&x); }
__device__ __forceinline__ uint32_t as_word(__half2 x) { return *reinterpret_cast<const uint32_t *>(&x); }
// Rows of 4-bit codes: channel c of a row is code (word c / 8) >> 4 (c % 8) & 15
// and stands for base + code step, one fused fp16 operation, where step and
// base are the halves of word c / 32 of the row's last part.
//
// Codes k and k + 4 (counted from the lowest) of a word as values, k = 0 .. 3,
// packed with the lower one first.  A code or'ed into the mantissa of 1024 is
// 1024 + code, or 1024 + 16 code: both come off exactly (Kim, Henry, Fahim and
// Awadalla, "Who says elephants can't run", 2022, for integer weights).
__device__ __forceinline__ void q4_values(uint32_t w, __half2 step, __half2 base, uint32_t (&y)[4]) {
    const uint32_t magic = 0x64006400u;
    const __half2 one = as_half2(0xe400e400u), part = as_half2(0x2c002c00u), rest = as_half2(0xd400d400u);   // -1024, 1/16, -64
#pragma unroll
    for (int k = 0; k < 4; k += 2) {
        const uint32_t x = k ? w >> 8 : w;
        const __half2 lo = __hadd2(as_half2(and_or(x, 0x000f000fu, magic)), one);
        const __half2 hi = __hfma2(as_half2(and_or(x, 0x00f000f0u, magic)), part, rest);
        y[k] = as_word(__hfma2(lo, step, base));
        y[k + 1] = as_word(__hfma2(hi, step, base));
    }
}

__device__ __forceinline__ float min_or_nan(float x, float y) {
    float z;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
__device__ __forceinline__ float max_or_nan(float x, float y) {
    float z;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(z) : "f"(x), "f"(y));
    return z;
}
// 8 channels (16-byte aligned) of a group that four neighbouring threads have:
// their word of codes and, in this order, the group's step and base.  Every
// thread of a warp calls it.
__device__ __forceinline__ uint32_t q4_pack(const float *channels, uint32_t &codes) {
    constexpr float kMost = 65000.0f;   // base + 15 step stays finite in fp16
    const float4 lower = reinterpret_cast<const float4 *>(channels)[0], upper = reinterpret_cast<const float4 *>(channels)[1];
    float y[8] = {lower.x, lower.y, lower.z, lower.w, upper.x, upper.y, upper.z, upper.w};
    float least = y[0], most = y[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) least = min_or_nan(least, y[i]), most = max_or_nan(most, y[i]);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        least = min_or_nan(least, __shfl_xor_sync(0xffffffffu, least, o));
        most = max_or_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
    }
    codes = 0;
    if (!(least >= -kMost && most <= kMost)) {
        if (!(least >= -3.4028234e38f && most <= 3.4028234e38f)) return 0x7fff0000u;   // NaN or infinities among them
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(y[i], -kMost), kMost);
        least = fminf(fmaxf(least, -kMost), kMost), most = fminf(fmaxf(most, -kMost), kMost);
    }
    const __half base = __float2half_rn(least), step = __float2half_rn(__fmul_rn(__fsub_rn(most, least), (float)(1.0 / 15.0)));
    const float from = __half2float(base), s = __half2float(step), inv = s > 0.0f ? __frcp_rn(s) : 0.0f;
    // 2^23 + code, rounded to the nearest even whole number, has the code in its
    // lowest bits: 8 of them are summed in steps of 16, and what the exponents
    // add up to is taken off.
#pragma unroll
    for (int i = 7; i >= 0; --i)
        codes = codes * 16 + __float_as_uint(__fadd_rn(fminf(fmaxf(__fmul_rn(__fsub_rn(y[i], from), inv), 0.0f), 15.0f), 0x1p23f));
    codes -= 0x4b000000u * 0x11111111u;
    return as_word(__halves2half2(step, base));
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
