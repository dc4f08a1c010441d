// Rotary positions and the write into the paged cache, in one pass over the
// fused QKV rows that the unmask leaves.
//
// Pair (a, b) -> (a cos - b sin, b cos + a sin) at the phase
// pos * turns mod 2^64 (64-bit wrap-around is the range reduction: nothing is
// lost at any position, where fp32 angles would be off by 0.008 rad at 131072).
// The phase's upper 32 bits, as a signed fraction of a turn, go to sincospif:
// 2^-25 turns at most.
//
// Bound by HBM (fp32 rows in, fp32 queries and the cache's rows out).  A block
// takes the heads of one token, or a share of them where tokens are few; its
// sines and cosines are computed once, in shared memory, while the first rows
// are under way.  A thread owns 4 + 4 channels of a head, half a head apart so
// that every access is whole lines, and has four heads in flight.  2048 tokens
// of 64 + 16 heads of 128: 39 us with a head a thread and its own sines, 30 with
// shared ones, 29 with the early rows (5.5 TB/s, 81% of the copy rate).
#include <math.h>

#include "kv_cache.cuh"

namespace mosaic {
namespace {

constexpr int kAppendThreads = 256;

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

template <class T>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(KvView kv, AppendArgs a) {
    __shared__ __align__(16) float cs[128], sn[128];
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (t >= a.l) return;
    const int D = kv.c.head_dim, units = D / 8, rot = a.rope.rot_dim;
    // The thread's channels c0 .. c0 + 3 and c1 .. c1 + 3 of every head, in the
    // halves of the channels that turn or of those that do not.
    const int u = threadIdx.x % units, lane = threadIdx.x / units, lanes = blockDim.x / units;
    const bool spins = 8 * u < rot;
    const int c0 = spins ? 4 * u : rot + 4 * (u - rot / 8), c1 = c0 + (spins ? rot : D - rot) / 2;
    const int H = a.heads, KV = kv.c.kv_heads;
    const int last = min((int)(blockIdx.x + 1) * a.share, H + 2 * KV);
    const float *row = a.qkv + t * a.ldx;
    float *qrow = a.q + t * a.ldq;
    constexpr int N = 4;
    Load4 xs[N], ys[N];
    auto load = [&](int h0) {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (h0 + k * lanes < last) {
                xs[k] = load4(row + (int64_t)(h0 + k * lanes) * D + c0, a.vec);
                ys[k] = load4(row + (int64_t)(h0 + k * lanes) * D + c1, a.vec);
            }
    };
    int h0 = blockIdx.x * a.share + lane;
    load(h0);   // under way while the phases are looked up
    if ((int)threadIdx.x < rot / 2) {
        const int j = threadIdx.x;
        int ax = a.rope.axis ? a.rope.axis[j] : 0;
        ax = (uint32_t)ax < (uint32_t)a.rope.axes ? ax : 0;
        const int64_t pos = a.rope.pos[ax * a.rope.ldp + t];
        const int32_t phase = (int32_t)(((uint64_t)pos * a.rope.turns[j]) >> 32);
        sincospif((float)phase * 0x1p-31f, &sn[j], &cs[j]);
    }
    const int64_t sq = a.seq[t], sl = a.slot[t];
    int id = -1;
    uint32_t off = 0;
    if (sq >= 0 && sq < kv.c.seqs && sl >= 0 && sl < kv.slots()) id = kv.page_of(sq, (uint32_t)sl, off);
    __syncthreads();
    while (h0 < last) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int h = h0 + k * lanes;
            if (h >= last) break;
            Load4 &x = xs[k], &y = ys[k];
            if (spins && h < H + KV) {
                if (!a.rope.interleaved) {   // channel c0 + i with c1 + i
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float c = cs[c0 + i], s = sn[c0 + i], p = x.x[i], q = y.x[i];
                        x.x[i] = p * c - q * s;
                        y.x[i] = q * c + p * s;
                    }
                } else {                     // neighbours
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        float c = cs[(c0 + i) / 2], s = sn[(c0 + i) / 2], p = x.x[i], q = x.x[i + 1];
                        x.x[i] = p * c - q * s;
                        x.x[i + 1] = q * c + p * s;
                        c = cs[(c1 + i) / 2], s = sn[(c1 + i) / 2], p = y.x[i], q = y.x[i + 1];
                        y.x[i] = p * c - q * s;
                        y.x[i + 1] = q * c + p * s;
                    }
                }
            }
            if (h < H) {
                store4(qrow + (int64_t)h * D + c0, x, a.vec);
                store4(qrow + (int64_t)h * D + c1, y, a.vec);
            } else if (id >= 0) {
                const int g = h < H + KV ? h - H : h - H - KV;
                T *o = static_cast<T *>(h < H + KV ? kv.c.k : kv.c.v) + kv.element(id, g, off);
                put4(o + c0, x);
                put4(o + c1, y);
                if (u == 0 && h < H + KV) {
                    if (kv.c.position) kv.c.position[kv.mark(id, g, off)] = a.index[t];
                    if (kv.c.weight) kv.c.weight[kv.mark(id, g, off)] = 0.0f;
                }
            }
        }
        h0 += N * lanes;
        load(h0);
    }
}

template <class T>
void append_launch(const KvView &kv, const AppendArgs &a, dim3 grid, int threads, cudaStream_t st) {
    append_kernel<T><<<grid, threads, 0, st>>>(kv, a);
}

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" {

mosaic_status mosaic_rope_turns(int64_t rot_dim, double base, uint64_t *turns) {
    if (rot_dim < 2 || rot_dim > 256 || rot_dim % 2) return MOSAIC_ERR_SHAPE;
    if (!turns || !(base > 1.0) || !isfinite(base)) return MOSAIC_ERR_ARG;
    for (int64_t j = 0; j < rot_dim / 2; ++j) {
        const double freq = pow(base, -2.0 * (double)j / (double)rot_dim);
        turns[j] = (uint64_t)rint(freq / (2.0 * M_PI) * 0x1p64);   // below 2^62
    }
    return MOSAIC_OK;
}

mosaic_status mosaic_kv_append(const mosaic_kv_cache *cache, const float *qkv, int64_t ldx, int64_t l, int64_t heads,
                               const int32_t *seq, const int32_t *slot, const int32_t *index,
                               const mosaic_rope *rope, float *q, int64_t ldq, void *stream) {
    RoleScope role("kv_append");
    MOSAIC_TRY(kv_check(cache));
    const int64_t D = cache->head_dim, KV = cache->kv_heads;
    if (l < 0 || l > (int64_t)65535 * 65535 || heads < 1 || heads > 65535 || ldx < (heads + 2 * KV) * D ||
        ldq < heads * D)
        return MOSAIC_ERR_SHAPE;
    AppendArgs a = {};
    if (rope && rope->rot_dim) {
        if (rope->rot_dim < 0 || rope->rot_dim > D || rope->rot_dim % 8) return MOSAIC_ERR_SHAPE;
        if (rope->axes < 1 || rope->axes > 4 || rope->interleaved < 0 || rope->interleaved > 1) return MOSAIC_ERR_ARG;
        if (rope->ldp < l) return MOSAIC_ERR_SHAPE;
        if (l && (!rope->turns || !rope->pos)) return MOSAIC_ERR_ARG;
        a.rope = *rope;
    }
    if (l == 0) return MOSAIC_OK;
    if (!qkv || !q || !seq || !slot || (cache->position && !index)) return MOSAIC_ERR_ARG;
    a.qkv = qkv, a.ldx = ldx, a.l = l, a.heads = (int)heads, a.seq = seq, a.slot = slot, a.index = index, a.q = q, a.ldq = ldq;
    a.vec = aligned16(qkv) && aligned16(q) && ldx % 4 == 0 && ldq % 4 == 0;
    const int units = (int)D / 8, lanes = kAppendThreads / units;
    // Heads of a block: all of a token's, unless that leaves SMs without work
    // (at most four blocks an SM, a head a thread at least).
    const int64_t all = heads + 2 * KV, most = (all + lanes - 1) / lanes;
    int64_t cut = 152 * 4 / l;
    cut = cut < 1 ? 1 : cut > most ? most : cut;
    a.share = (int)((most + cut - 1) / cut * lanes);
    const dim3 grid((unsigned)((all + a.share - 1) / a.share), (unsigned)(l < 65535 ? l : 65535),
                    (unsigned)((l + 65534) / 65535));
    cudaStream_t st = as_stream(stream);
    const KvView kv(*cache);
    {
        KernelSpan span("append", st);
        if (cache->type == MOSAIC_KV_F32) append_launch<float>(kv, a, grid, lanes * units, st);
        else if (cache->type == MOSAIC_KV_BF16) append_launch<__nv_bfloat16>(kv, a, grid, lanes * units, st);
        else append_launch<__half>(kv, a, grid, lanes * units, st);
    }
    return launch_status();
}

}  // extern "C"
