// Rows of a list of cached tokens, copied out; those of 4-bit caches as the
// fp16 values that their codes stand for.
//
// Bound by HBM (a 4-bit row of 128 channels is 80 bytes in and 256 out).  A
// thread takes 16 bytes of a key row of the output and the same of the value
// row: a word of 8 codes with its step and base, or a copy.
#include "kv_cache.cuh"

namespace mosaic {
namespace {

constexpr int kRowThreads = 256;

struct RowsArgs {
    const int32_t *seq, *slot;
    int64_t l, ld_token, ld_head;   // the strides in 16-byte units
    uint4 *k, *v;
    int units;                      // 16-byte units of an output row
};

template <bool Q>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(KvView kv, RowsArgs a) {
    const int per = kv.c.kv_heads * a.units;   // of a token
    const int64_t x = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    const int64_t t = x / per;
    if (t >= a.l) return;
    const int in = (int)(x - t * per), h = in / a.units, u = in - h * a.units;
    const int64_t sq = a.seq[t], sl = a.slot[t];
    uint4 y[2];
    y[0] = y[1] = make_uint4(0, 0, 0, 0);
    uint32_t off = 0;
    const int id = sq >= 0 && sq < kv.c.seqs && sl >= 0 && sl < kv.slots() ? kv.page_of(sq, (uint32_t)sl, off) : -1;
    if (id >= 0) {
        const int64_t at = kv.element(id, h, off);
        if constexpr (Q) {
            const char *p[2] = {static_cast<const char *>(kv.c.k) + at, static_cast<const char *>(kv.c.v) + at};
            uint32_t codes[2], scales[2], w[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                codes[i] = *reinterpret_cast<const uint32_t *>(p[i] + 4 * u);
                scales[i] = *reinterpret_cast<const uint32_t *>(p[i] + kv.c.head_dim / 2 + u / 4 * 4);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                q4_values(codes[i], __low2half2(as_half2(scales[i])), __high2half2(as_half2(scales[i])), w);
                // Words of channels k and k + 4 to words of neighbours.
                y[i] = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410),
                                  __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
            }
        } else {
            const int64_t es = kv.c.type == MOSAIC_KV_F32 ? 4 : 2;
            y[0] = reinterpret_cast<const uint4 *>(static_cast<const char *>(kv.c.k) + at * es)[u];
            y[1] = reinterpret_cast<const uint4 *>(static_cast<const char *>(kv.c.v) + at * es)[u];
        }
    }
    const int64_t to = t * a.ld_token + h * a.ld_head + u;
    a.k[to] = y[0];
    a.v[to] = y[1];
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
    const unsigned grid = (unsigned)((l * KV * units + kRowThreads - 1) / kRowThreads);
    cudaStream_t st = as_stream(stream);
    {
        KernelSpan span("rows", st);
        if (cache->type == MOSAIC_KV_Q4) rows_kernel<true><<<grid, kRowThreads, 0, st>>>(kv, a);
        else rows_kernel<false><<<grid, kRowThreads, 0, st>>>(kv, a);
    }
    return launch_status();
}

}  // extern "C"
