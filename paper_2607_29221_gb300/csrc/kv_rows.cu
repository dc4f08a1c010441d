// Rows of a list of cached tokens, copied out; those of 4-bit caches as the
// fp16 values that their codes stand for.
//
// Bound by HBM (a 4-bit row of 128 channels is 80 bytes in and 256 out).  A
// thread takes 16 bytes of a key row of the output and the same of the value
// row: a word of 8 codes with its step and base, or a copy.
#include "kv_cache.cuh"

namespace mosaic {
namespace {

// 32768 tokens of 8 heads of 128 in 4 bits, 61 tokens, us (threads, units a thread): 256 x 1 44.8 / 7.2, 256 x 2 38.0 / 7.5,
// 256 x 4 36.9 / 8.5, 128 x 2 37.1 / 7.1, 128 x 4 36.7 / 8.2.
constexpr int kRowThreads = 128, kRowUnits = 2;

struct RowsArgs {
    const int32_t *seq, *slot;
    int64_t l, ld_token, ld_head;   // the strides in 16-byte units
    uint4 *k, *v;
    int units;                      // 16-byte units of an output row
};

template <bool Q>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(KvView kv, RowsArgs a) {
    constexpr int N = kRowUnits;
    const uint32_t per = kv.c.kv_heads * a.units;   // of a token
    // Units of a block in a row; a thread's are kRowThreads apart, all looked up
    // and read before the first is written.
    const int64_t x0 = (int64_t)blockIdx.x * (N * kRowThreads);
    const int64_t t0 = x0 / per;                     // the block's
    const uint32_t in0 = (uint32_t)(x0 - t0 * per) + threadIdx.x;
    int64_t to[N], from[N];
    int u[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const uint32_t in = in0 + k * kRowThreads, more = in / per, r = in - more * per;
        const int64_t t = t0 + more;
        const int h = r / (uint32_t)a.units;
        u[k] = r - h * a.units;
        to[k] = from[k] = -1;
        if (t >= a.l) continue;
        to[k] = t * a.ld_token + h * a.ld_head + u[k];
        const int64_t sq = a.seq[t], sl = a.slot[t];
        uint32_t off = 0;
        if (sq < 0 || sq >= kv.c.seqs || sl < 0 || sl >= kv.slots()) continue;
        const int id = kv.page_of(sq, (uint32_t)sl, off);
        if (id >= 0) from[k] = kv.element(id, h, off);
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
                codes[k][i] = *reinterpret_cast<const uint32_t *>(pools[i] + from[k] + 4 * u[k]);
                scales[k][i] = *reinterpret_cast<const uint32_t *>(pools[i] + from[k] + kv.c.head_dim / 2 + u[k] / 4 * 4);
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
                if (to[k] >= 0) (i ? a.v : a.k)[to[k]] = y;
            }
    } else {
        const int64_t es = kv.c.type == MOSAIC_KV_F32 ? 4 : 2;
        uint4 y[N][2];
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                y[k][i] = make_uint4(0, 0, 0, 0);
                if (from[k] >= 0) y[k][i] = reinterpret_cast<const uint4 *>(pools[i] + from[k] * es)[u[k]];
            }
#pragma unroll
        for (int k = 0; k < N; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (to[k] >= 0) (i ? a.v : a.k)[to[k]] = y[k][i];
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
    if (l > ((int64_t)0x7fffffff * kRowThreads) / (KV * units)) return MOSAIC_ERR_SHAPE;
    if (l == 0) return MOSAIC_OK;
    if (!seq || !slot || !k || !v) return MOSAIC_ERR_ARG;
    if (!aligned16(k) || !aligned16(v) || (l > 1 && ld_token % unit) || (KV > 1 && ld_head % unit)) return MOSAIC_ERR_ALIGN;
    const KvView kv(*cache);
    const RowsArgs a = {seq, slot, l, ld_token / unit, ld_head / unit, static_cast<uint4 *>(k), static_cast<uint4 *>(v), (int)units};
    const unsigned grid = (unsigned)((l * KV * units + kRowThreads * kRowUnits - 1) / (kRowThreads * kRowUnits));
    cudaStream_t st = as_stream(stream);
    {
        KernelSpan span("rows", st);
        if (cache->type == MOSAIC_KV_Q4) rows_kernel<true><<<grid, kRowThreads, 0, st>>>(kv, a);
        else rows_kernel<false><<<grid, kRowThreads, 0, st>>>(kv, a);
    }
    return launch_status();
}

}  // extern "C"
