// Rows of a list of cached tokens, copied out; those of 4-bit caches as the
// fp16 values that their codes stand for.
//
// Bound by HBM (a 4-bit row of 128 channels is 80 bytes in and 256 out).  A
// thread takes 16 bytes of a key row of the output and the same of the value
// row: a word of 8 codes with its step and base, or a copy.
#include "kv_cache.cuh"

namespace mosaic {
namespace {

// Threads, and tokens of a thread.  32768 tokens of 8 heads of 128 in 4 bits / 61 tokens, us: 128 x 1 41.9 / 7.1, 128 x 2
// 35.4 / 7.0, 128 x 4 36.9 / 7.9, 128 x 8 39.3 / 8.6, 256 x 2 36.4 / 7.3.
constexpr int kRowThreads = 128, kRowTokens = 2;

struct RowsArgs {
    const int32_t *seq, *slot;
    int64_t l, ld_token, ld_head;   // the strides in 16-byte units
    uint4 *k, *v;
    int units;                      // 16-byte units of an output row
    int together;                   // tokens that the threads of a block have side by side
};

template <bool Q>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(KvView kv, RowsArgs a) {
    constexpr int N = kRowTokens;
    // The thread's head and unit, the same of every token; all tokens are looked
    // up and read before the first is written.
    const uint32_t per = kv.c.kv_heads * a.units, x = blockIdx.y * kRowThreads + threadIdx.x;
    const uint32_t side = a.together > 1 ? x / per : 0, in = x - side * per;
    if (in >= per || side >= (uint32_t)a.together) return;
    const int h = in / (uint32_t)a.units, u = in - h * a.units;
    const int64_t t0 = (int64_t)blockIdx.x * (N * a.together) + side, head = h * kv.c.head_stride, out = h * a.ld_head + u;
    int64_t from[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int64_t t = t0 + k * a.together;
        from[k] = -1;
        if (t >= a.l) continue;
        const int64_t sq = a.seq[t], sl = a.slot[t];
        uint32_t off = 0;
        if (sq < 0 || sq >= kv.c.seqs || sl < 0 || sl >= kv.slots()) continue;
        const int id = kv.page_of(sq, (uint32_t)sl, off);
        if (id >= 0) from[k] = id * kv.c.page_stride + off * kv.c.slot_stride + head;
    }
    const char *const pools[2] = {static_cast<const char *>(kv.c.k), static_cast<const char *>(kv.c.v)};
    if constexpr (Q) {
        uint32_t codes[N][2], scales[N][2];
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                codes[k][i] = scales[k][i] = 0;   // zeros
                if (from[k] < 0) continue;
                codes[k][i] = *reinterpret_cast<const uint32_t *>(pools[i] + from[k] + 4 * u);
                scales[k][i] = *reinterpret_cast<const uint32_t *>(pools[i] + from[k] + kv.c.head_dim / 2 + u / 4 * 4);
            }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t w[4];
                q4_values(codes[k][i], __low2half2(as_half2(scales[k][i])), __high2half2(as_half2(scales[k][i])), w);
                // Words of channels k and k + 4 to words of neighbours.
                const uint4 y = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410),
                                           __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
                if (t0 + k * a.together < a.l) (i ? a.v : a.k)[(t0 + k * a.together) * a.ld_token + out] = y;
            }
    } else {
        const int64_t es = kv.c.type == MOSAIC_KV_F32 ? 4 : 2;
        uint4 y[N][2];
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                y[k][i] = make_uint4(0, 0, 0, 0);
                if (from[k] >= 0) y[k][i] = reinterpret_cast<const uint4 *>(pools[i] + from[k] * es)[u];
            }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (t0 + k * a.together < a.l) (i ? a.v : a.k)[(t0 + k * a.together) * a.ld_token + out] = y[k][i];
    }
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_kv_row_bytes(int type, int64_t head_dim) {
    if (type < MOSAIC_KV_F32 || (type > MOSAIC_KV_F16 && type != MOSAIC_KV_Q4)) return 0;
    if (head_dim < 8 || head_dim > 256 || head_dim % (type == MOSAIC_KV_Q4 ? kQ4Group : 8)) return 0;
    return (size_t)kv_row_bytes(type, head_dim);
}

mosaic_status mosaic_kv_rows(const mosaic_kv_cache *cache, const int32_t *seq, const int32_t *slot, int64_t l,
                             void *k, void *v, int64_t ld_token, int64_t ld_head, void *stream) {
    RoleScope role("kv_rows");
    MOSAIC_TRY(kv_check(cache));
    const int64_t D = cache->head_dim, KV = cache->kv_heads;
    if (l < 0 || (l > 1 && ld_token < D) || (l > 0 && KV > 1 && ld_head < D)) return MOSAIC_ERR_SHAPE;
    const int64_t unit = cache->type == MOSAIC_KV_F32 ? 4 : 8, units = D / unit;
    if (l > (int64_t)0x7fffffff) return MOSAIC_ERR_SHAPE;
    if (l == 0) return MOSAIC_OK;
    if (!seq || !slot || !k || !v) return MOSAIC_ERR_ARG;
    if (!aligned16(k) || !aligned16(v) || (l > 1 && ld_token % unit) || (KV > 1 && ld_head % unit)) return MOSAIC_ERR_ALIGN;
    const KvView kv(*cache);
    const int64_t per = KV * units, together = per < kRowThreads ? kRowThreads / per : 1;
    const RowsArgs a = {seq, slot, l, ld_token / unit, ld_head / unit, static_cast<uint4 *>(k), static_cast<uint4 *>(v), (int)units, (int)together};
    const dim3 grid((unsigned)((l + kRowTokens * together - 1) / (kRowTokens * together)), (unsigned)((per + kRowThreads - 1) / kRowThreads));
    cudaStream_t st = as_stream(stream);
    {
        KernelSpan span("rows", st);
        if (cache->type == MOSAIC_KV_Q4) rows_kernel<true><<<grid, kRowThreads, 0, st>>>(kv, a);
        else rows_kernel<false><<<grid, kRowThreads, 0, st>>>(kv, a);
    }
    return launch_status();
}

}  // extern "C"
