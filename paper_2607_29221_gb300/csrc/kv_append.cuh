// What the two kernels that append to the key/value cache share.
#pragma once

#include "kv_cache.cuh"

namespace mosaic {

struct AppendArgs {
    const float *qkv;
    int64_t ldx, l;
    int heads, vec;
    const int32_t *seq, *slot, *index;
    mosaic_rope rope;
    float *q;
    int64_t ldq;
    int share;   // heads of a block
};

// The kernel with norms (norm may be null) and for 4-bit caches.
mosaic_status append_norm_launch(const mosaic_kv_cache &c, AppendArgs a, const mosaic_head_norm *norm, cudaStream_t st);

namespace {

struct Load4 {
    float x[4];
};
__device__ __forceinline__ Load4 load4(const float *p, bool vec) {
    Load4 r;
    if (vec) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        r.x[0] = v.x; r.x[1] = v.y; r.x[2] = v.z; r.x[3] = v.w;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) r.x[i] = p[i];
    }
    return r;
}
__device__ __forceinline__ void store4(float *p, const Load4 &v, bool vec) {
    if (vec) *reinterpret_cast<float4 *>(p) = make_float4(v.x[0], v.x[1], v.x[2], v.x[3]);
    else {
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = v.x[i];
    }
}
// Four channels into the cache (rounded to nearest once); 8- or 16-byte
// aligned by the cache's strides and the multiples of 4 channels.
__device__ __forceinline__ void put4(float *p, const Load4 &v) { store4(p, v, true); }
template <class T>
__device__ __forceinline__ void put4(T *p, const Load4 &v) {
    T e[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) e[i] = Elem<T>::from(v.x[i]);
    *reinterpret_cast<uint2 *>(p) = *reinterpret_cast<const uint2 *>(e);
}

// Heads of a block (a.share): all of a token's, unless that leaves SMs without
// work (at most four blocks an SM, a head a thread at least; `lanes` heads at a
// time).  The grid: x share, y and z token.
inline dim3 append_grid(const mosaic_kv_cache &c, AppendArgs &a, int lanes) {
    const int64_t all = a.heads + 2 * (int64_t)c.kv_heads, most = (all + lanes - 1) / lanes;
    int64_t cut = 152 * 4 / a.l;
    cut = cut < 1 ? 1 : cut > most ? most : cut;
    a.share = (int)((most + cut - 1) / cut * lanes);
    return dim3((unsigned)((all + a.share - 1) / a.share), (unsigned)(a.l < 65535 ? a.l : 65535),
                (unsigned)((a.l + 65534) / 65535));
}

}  // namespace
}  // namespace mosaic
