// Attention of one new token per sequence over the paged cache, split over
// the cache's length and joined.
//
//   s_j = scale q . k_j,  p = softmax(s) over the live slots,  out = sum p_j v_j
#include <math.h>

#include "kv_cache.cuh"

namespace mosaic {
namespace {

constexpr int kChunk = 128, kThreads = 256;
constexpr int kMaxGroup = 64;

struct AttendArgs {
    const float *q;
    int64_t ldq;
    const int32_t *lens, *first;
    int64_t max_len;
    int heads, group, chunks;
    float scale, decay;
    float *out;
    int64_t ldo;
    float *m, *l, *o, *s;   // partial maxima, sums, outputs, and scores
};

__device__ __forceinline__ float minus_inf() { return __int_as_float(0xff800000); }

// Partial softmax of one (sequence, head, chunk) for the group's queries.
template <class T>
__global__ void __launch_bounds__(kThreads) attend_kernel(KvView kv, AttendArgs a) {
    extern __shared__ float sh[];
    const int D = kv.c.head_dim, G = a.group;
    float *qs = sh, *sc = sh + G * D;   // G x D, G x kChunk
    __shared__ int ids[kChunk];
    __shared__ uint32_t offs[kChunk];
    const int chunk = blockIdx.x % a.chunks;
    const int64_t job = blockIdx.x / a.chunks;
    const int h = (int)(job % kv.c.kv_heads);
    const int64_t i = job / kv.c.kv_heads;
    const int len = kv.length(a.lens, i, a.max_len), s0 = chunk * kChunk, n = min(kChunk, len - s0);
    if (n <= 0) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int x = threadIdx.x; x < G * D; x += kThreads)
        qs[x] = a.q[i * a.ldq + (int64_t)(h * G) * D + x] * a.scale;
    for (int j = threadIdx.x; j < n; j += kThreads) {
        uint32_t off;
        int id = kv.page_of(i, (uint32_t)(s0 + j), off);
        if (id >= 0 && a.first && kv.c.position[kv.mark(id, h, off)] < a.first[i]) id = -1;
        ids[j] = id, offs[j] = off;
    }
    __syncthreads();
    for (int j = warp; j < n; j += kThreads / 32) {
        const T *k = static_cast<const T *>(kv.c.k) + kv.element(max(ids[j], 0), h, offs[j]);
        for (int g = 0; g < G; ++g) {
            float x = 0.0f;
            for (int d = lane; d < D; d += 32) x = fmaf(qs[g * D + d], Elem<T>::to(k[d]), x);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
            if (lane == 0) sc[g * kChunk + j] = ids[j] >= 0 ? x : minus_inf();
        }
    }
    __syncthreads();
    for (int g = warp; g < G; g += kThreads / 32) {
        const int64_t at = (i * a.heads + h * G + g);
        float top = minus_inf(), bad = 0.0f;
        for (int j = lane; j < n; j += 32) {
            const float x = sc[g * kChunk + j];
            if (x != x) bad = x;
            top = fmaxf(top, x);
            if (a.s) a.s[at * a.chunks * kChunk + s0 + j] = x;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            bad += __shfl_xor_sync(0xffffffffu, bad, o);
        }
        top += bad;
        const float base = top == minus_inf() ? 0.0f : top;
        float sum = 0.0f;
        for (int j = lane; j < n; j += 32) {
            const float e = expf(sc[g * kChunk + j] - base);
            sc[g * kChunk + j] = e;
            sum += e;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) a.m[at * a.chunks + chunk] = top, a.l[at * a.chunks + chunk] = sum;
    }
    __syncthreads();
    for (int x = threadIdx.x; x < G * D; x += kThreads) {
        const int g = x / D, d = x % D;
        float o = 0.0f;
        for (int j = 0; j < n; ++j)
            if (ids[j] >= 0)
                o = fmaf(sc[g * kChunk + j],
                         Elem<T>::to(static_cast<const T *>(kv.c.v)[kv.element(ids[j], h, offs[j]) + d]), o);
        a.o[((i * a.heads + h * G + g) * a.chunks + chunk) * D + d] = o;
    }
}

// One block a (sequence, query head): the join of its chunks.
__global__ void __launch_bounds__(256) attend_join_kernel(KvView kv, AttendArgs a) {
    const int64_t at = blockIdx.x, i = at / a.heads;
    const int D = kv.c.head_dim, len = kv.length(a.lens, i, a.max_len), n = (len + kChunk - 1) / kChunk;
    float top = minus_inf();
    for (int c = 0; c < n; ++c) {
        const float m = a.m[at * a.chunks + c];
        top = m != m || top != top ? m + top : fmaxf(top, m);
    }
    const float base = top == minus_inf() ? 0.0f : top;
    float sum = 0.0f;
    for (int c = 0; c < n; ++c) {
        const float m = a.m[at * a.chunks + c];
        if (m != minus_inf()) sum += expf(m - base) * a.l[at * a.chunks + c];
    }
    const int d = threadIdx.x;
    if (d < D) {
        float o = 0.0f;
        for (int c = 0; c < n; ++c) {
            const float m = a.m[at * a.chunks + c];
            if (m != minus_inf()) o += expf(m - base) * a.o[(at * a.chunks + c) * D + d];
        }
        a.out[i * a.ldo + (at % a.heads) * D + d] = sum == 0.0f ? 0.0f : o / sum;
    }
    __syncthreads();
    if (a.s && d == 0) {   // kept for the weights
        a.m[at * a.chunks] = base, a.l[at * a.chunks] = sum;
    }
}

// One thread a (sequence, head, slot): the weight that it gathers.
__global__ void __launch_bounds__(256) attend_weight_kernel(KvView kv, AttendArgs a, int64_t total) {
    const int64_t row = (int64_t)a.chunks * kChunk;
    for (int64_t x = blockIdx.x * 256ll + threadIdx.x; x < total; x += gridDim.x * 256ll) {
        const int64_t job = x / row, i = job / kv.c.kv_heads;
        const int h = (int)(job % kv.c.kv_heads), s = (int)(x % row);
        if (s >= kv.length(a.lens, i, a.max_len)) continue;
        uint32_t off;
        const int id = kv.page_of(i, (uint32_t)s, off);
        if (id < 0) continue;
        float w = 0.0f;
        for (int g = 0; g < a.group; ++g) {
            const int64_t at = i * a.heads + h * a.group + g;
            const float sum = a.l[at * a.chunks];
            if (sum != 0.0f) w += expf(a.s[at * row + s] - a.m[at * a.chunks]) / sum;
        }
        float *p = kv.c.weight + kv.mark(id, h, off);
        *p = *p * a.decay + w;
    }
}

template <class T>
bool attend_launch(const KvView &kv, const AttendArgs &a, int64_t blocks, size_t smem, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    if (!ensure_smem_limit(done, attend_kernel<T>, 4 * kMaxGroup * (256 + kChunk))) return false;
    attend_kernel<T><<<(unsigned)blocks, kThreads, smem, st>>>(kv, a);
    return true;
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_kv_attention_workspace(const mosaic_kv_cache *cache, int64_t heads, int64_t max_len) {
    if (kv_check(cache) != MOSAIC_OK || max_len < 0 || max_len > 0x7fffffff || heads < 1 || heads % cache->kv_heads)
        return 0;
    const int64_t chunks = max_len ? (max_len + kChunk - 1) / kChunk : 1;
    const size_t rows = (size_t)(cache->seqs * heads * chunks);
    return 2 * up256(4 * rows) + up256(4 * rows * cache->head_dim) + (cache->weight ? up256(4 * rows * kChunk) : 0);
}

mosaic_status mosaic_kv_attention(const mosaic_kv_cache *cache, const float *q, int64_t ldq, int64_t heads,
                                  const int32_t *lens, int64_t max_len, const int32_t *first, float scale,
                                  float decay, float *out, int64_t ldo, void *ws, size_t ws_bytes, void *stream) {
    RoleScope role("kv_attention");
    MOSAIC_TRY(kv_check(cache));
    const int64_t D = cache->head_dim;
    if (heads < 1 || heads > 65535 || heads % cache->kv_heads || ldq < heads * D || ldo < heads * D || max_len < 0 ||
        max_len > 0x7fffffff)
        return MOSAIC_ERR_SHAPE;
    if (heads / cache->kv_heads > kMaxGroup) return MOSAIC_ERR_UNSUPPORTED;
    if (!isfinite(scale) || !isfinite(decay)) return MOSAIC_ERR_ARG;
    if (cache->seqs == 0) return MOSAIC_OK;
    if (!q || !out || !lens || (first && !cache->position)) return MOSAIC_ERR_ARG;
    if (ws_bytes < mosaic_kv_attention_workspace(cache, heads, max_len)) return MOSAIC_ERR_WORKSPACE;
    if (!ws) return MOSAIC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ws) % 16) return MOSAIC_ERR_ALIGN;
    AttendArgs a = {};
    a.q = q, a.ldq = ldq, a.lens = lens, a.first = first, a.max_len = max_len, a.heads = (int)heads;
    a.group = (int)(heads / cache->kv_heads), a.chunks = max_len ? (int)((max_len + kChunk - 1) / kChunk) : 1;
    a.scale = scale, a.decay = decay, a.out = out, a.ldo = ldo;
    const size_t rows = (size_t)(cache->seqs * heads * a.chunks);
    a.m = static_cast<float *>(ws);
    a.l = a.m + up256(4 * rows) / 4;
    a.o = a.l + up256(4 * rows) / 4;
    a.s = cache->weight ? a.o + up256(4 * rows * D) / 4 : nullptr;
    const int64_t blocks = cache->seqs * cache->kv_heads * a.chunks;
    if (blocks > 0x7fffffff) return MOSAIC_ERR_SHAPE;
    cudaStream_t st = as_stream(stream);
    const KvView kv(*cache);
    const size_t smem = 4 * (size_t)a.group * (D + kChunk);
    {
        KernelSpan span("attend", st);
        const bool ok = cache->type == MOSAIC_KV_F32    ? attend_launch<float>(kv, a, blocks, smem, st)
                        : cache->type == MOSAIC_KV_BF16 ? attend_launch<__nv_bfloat16>(kv, a, blocks, smem, st)
                                                        : attend_launch<__half>(kv, a, blocks, smem, st);
        if (!ok) return MOSAIC_ERR_CUDA;
    }
    MOSAIC_TRY(launch_status());
    {
        KernelSpan span("attend_join", st);
        attend_join_kernel<<<(unsigned)(cache->seqs * heads), 256, 0, st>>>(kv, a);
    }
    MOSAIC_TRY(launch_status());
    if (!a.s) return MOSAIC_OK;
    const int64_t total = blocks * kChunk;
    {
        KernelSpan span("attend_weight", st);
        attend_weight_kernel<<<grid_for(total, 256), 256, 0, st>>>(kv, a, total);
    }
    return launch_status();
}

}  // extern "C"
