// Eviction from the paged cache by gathered attention weight.
//
// Per (sequence, head): the rank of a slot is its weight as an ordered 32-bit
// key; the E = len - keep least (key, slot) leave.  A radix selection finds
// the E-th least key, one ordered pass the holes below keep and the stayers
// from keep on, and the k-th hole takes the k-th stayer's row.  Only rows
// that have to move do, and no row is both read and written.
#include "kv_cache.cuh"

namespace mosaic {
namespace {

constexpr int kSelectThreads = 1024;

// Weights as unsigned keys in ascending order; NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (w != w) w = -__int_as_float(0x7f800000);
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kKeyInf = 0xff800000u;   // order_key(+inf)

struct EvictArgs {
    const int32_t *lens, *recent_from;
    int32_t *new_lens;
    int64_t max_len, keep, cap;   // cap: most moves of a (sequence, head)
    int32_t *count, *from, *to;
};

__device__ __forceinline__ uint32_t slot_key(const KvView &kv, const EvictArgs &a, int64_t i, int h, int s, int from) {
    uint32_t off;
    const int id = kv.page_of(i, (uint32_t)s, off);
    if (id < 0) return kKeyInf;
    const int64_t at = kv.mark(id, h, off);
    if (a.recent_from && kv.c.position[at] >= from) return kKeyInf;
    return order_key(kv.c.weight[at]);
}

// Exclusive sum of `v` over the block and its total (all threads call it).
__device__ __forceinline__ int block_scan(int v, int *part, int &total) {
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    if (lane == 31) part[w] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int k = 0; k < kSelectThreads / 32; ++k) {
        if (k < w) before += part[k];
        all += part[k];
    }
    __syncthreads();
    total = all;
    return before + x - v;
}

__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(KvView kv, EvictArgs a) {
    __shared__ int hist[256], part[kSelectThreads / 32];
    __shared__ uint32_t prefix;
    __shared__ int left;
    const int h = blockIdx.x % kv.c.kv_heads;
    const int64_t i = blockIdx.x / kv.c.kv_heads;
    const int len = kv.length(a.lens, i, a.max_len), keep = (int)a.keep;
    if (len <= keep) {
        if (threadIdx.x == 0) a.count[blockIdx.x] = 0;
        return;
    }
    const int from = a.recent_from ? a.recent_from[i] : 0;
    if (threadIdx.x == 0) prefix = 0, left = len - keep;
    // The E-th least key, 8 bits a pass; `left`: its rank among the keys with this prefix.
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (threadIdx.x < 256) hist[threadIdx.x] = 0;
        __syncthreads();
        const uint32_t pre = prefix;
        for (int s = threadIdx.x; s < len; s += kSelectThreads) {
            const uint32_t k = slot_key(kv, a, i, h, s, from);
            if (shift == 24 || (k >> (shift + 8)) == (pre >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            int r = left, b = 0;
            while (hist[b] < r) r -= hist[b++];
            prefix = pre | ((uint32_t)b << shift);
            left = r;
        }
        __syncthreads();
    }
    const uint32_t least = prefix;
    const int ties = left;   // of the slots with that key, so many leave
    int32_t *to = a.to + (int64_t)blockIdx.x * a.cap, *src = a.from + (int64_t)blockIdx.x * a.cap;
    int seen = 0, holes = 0, stays = 0, total;
    for (int s0 = 0; s0 < len; s0 += kSelectThreads) {
        const int s = s0 + threadIdx.x;
        const bool in = s < len;
        const uint32_t k = in ? slot_key(kv, a, i, h, s, from) : 0xffffffffu;
        const bool tie = in && k == least;
        const int rank = seen + block_scan(tie, part, total);
        seen += total;
        const bool out = in && (k < least || (tie && rank < ties));
        const bool hole = out && s < keep, stay = in && !out && s >= keep;
        int at = holes + block_scan(hole, part, total);
        holes += total;
        if (hole && at < a.cap) to[at] = s;
        at = stays + block_scan(stay, part, total);
        stays += total;
        if (stay && at < a.cap) src[at] = s;
    }
    if (threadIdx.x == 0) a.count[blockIdx.x] = holes < a.cap ? holes : (int)a.cap;
}

// A warp a move: key and value row, position and weight.
__global__ void __launch_bounds__(256) evict_move_kernel(KvView kv, EvictArgs a, int chunks) {
    const int64_t job = blockIdx.x / chunks;
    const int part = blockIdx.x % chunks;
    const int h = (int)(job % kv.c.kv_heads), lane = threadIdx.x & 31;
    const int64_t i = job / kv.c.kv_heads;
    if (part == 0 && h == 0 && threadIdx.x == 0) {
        const int n = kv.length(a.lens, i, a.max_len);
        a.new_lens[i] = n < a.keep ? n : (int)a.keep;
    }
    const int count = a.count[job];
    const int es = kv.c.type == MOSAIC_KV_F32 ? 4 : 2, quads = kv.c.head_dim * es / 16;
    for (int m = part * 8 + (threadIdx.x >> 5); m < count; m += chunks * 8) {
        uint32_t so, to;
        const int sid = kv.page_of(i, (uint32_t)a.from[job * a.cap + m], so);
        const int tid = kv.page_of(i, (uint32_t)a.to[job * a.cap + m], to);
        if (sid < 0 || tid < 0) continue;
        const int64_t se = kv.element(sid, h, so) * es, te = kv.element(tid, h, to) * es;
        for (int b = lane; b < 2 * quads; b += 32) {
            char *pool = static_cast<char *>(b < quads ? kv.c.k : kv.c.v);
            const int o = 16 * (b < quads ? b : b - quads);
            *reinterpret_cast<uint4 *>(pool + te + o) = *reinterpret_cast<const uint4 *>(pool + se + o);
        }
        const int64_t sm = kv.mark(sid, h, so), tm = kv.mark(tid, h, to);
        if (lane == 0) kv.c.weight[tm] = kv.c.weight[sm];
        if (lane == 1 && kv.c.position) kv.c.position[tm] = kv.c.position[sm];
    }
}

int64_t most_moves(int64_t max_len, int64_t keep) {
    const int64_t over = max_len - keep;
    return over <= 0 ? 0 : over < keep ? over : keep;
}
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_kv_evict_workspace(const mosaic_kv_cache *cache, int64_t max_len, int64_t keep) {
    if (kv_check(cache) != MOSAIC_OK || max_len < 0 || max_len > 0x7fffffff || keep < 1) return 0;
    const int64_t jobs = cache->seqs * cache->kv_heads;
    return up256(4 * (size_t)jobs) + 2 * up256(4 * (size_t)(jobs * most_moves(max_len, keep)));
}

mosaic_status mosaic_kv_evict(const mosaic_kv_cache *cache, const int32_t *lens, int64_t max_len, int64_t keep,
                              const int32_t *recent_from, int32_t *new_lens, void *ws, size_t ws_bytes,
                              void *stream) {
    RoleScope role("kv_evict");
    MOSAIC_TRY(kv_check(cache));
    if (max_len < 0 || max_len > 0x7fffffff || keep < 1) return MOSAIC_ERR_SHAPE;
    if (cache->seqs == 0) return MOSAIC_OK;
    if (!lens || !new_lens || !cache->weight || (recent_from && !cache->position)) return MOSAIC_ERR_ARG;
    const int64_t jobs = cache->seqs * cache->kv_heads;
    if (jobs > 0x7fffffff) return MOSAIC_ERR_SHAPE;
    if (ws_bytes < mosaic_kv_evict_workspace(cache, max_len, keep)) return MOSAIC_ERR_WORKSPACE;
    if (!ws) return MOSAIC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ws) % 4) return MOSAIC_ERR_ALIGN;
    EvictArgs a = {lens, recent_from, new_lens, max_len, keep, most_moves(max_len, keep), nullptr, nullptr, nullptr};
    char *w = static_cast<char *>(ws);
    a.count = reinterpret_cast<int32_t *>(w);
    a.from = reinterpret_cast<int32_t *>(w + up256(4 * (size_t)jobs));
    a.to = a.from + up256(4 * (size_t)(jobs * a.cap)) / 4;
    cudaStream_t st = as_stream(stream);
    const KvView kv(*cache);
    {
        KernelSpan span("evict_select", st);
        evict_select_kernel<<<(unsigned)jobs, kSelectThreads, 0, st>>>(kv, a);
    }
    MOSAIC_TRY(launch_status());
    int64_t chunks = (a.cap + 63) / 64;
    if (chunks < 1) chunks = 1;
    while (chunks > 1 && chunks * jobs > 16384) chunks = (chunks + 1) / 2;
    {
        KernelSpan span("evict_move", st);
        evict_move_kernel<<<(unsigned)(chunks * jobs), 256, 0, st>>>(kv, a, (int)chunks);
    }
    return launch_status();
}

}  // extern "C"
