// Eviction from the paged cache by gathered attention weight.
//
// Per (sequence, head): the rank of a slot is its weight as an ordered 32-bit
// key; the E = len - keep least (key, slot) leave.  The E-th least key is
// found by narrowing [least, greatest] 2048-fold a pass with a histogram
// (three passes at most: the keys of positive weights are their logarithms,
// piecewise, so they spread over the bins).  The k-th hole below keep then
// takes the k-th stayer from keep on: only rows that have to move do, and no
// row is both read and written.
//
// Selection: bound by its trips to memory (length, page, weight) and barriers,
// not by bytes: of 37000 cycles for 16384 slots on one block about 12000 load the
// keys, 16000 are three histograms and 9000 the rest (23000 while every warp
// walked its slots 32 at a time, instead of every thread its neighbouring ones
// as bits of a word).  A cluster of blocks takes a (sequence, head), each block
// a stretch of slots whose keys it keeps in shared memory, with histograms and
// counts summed through the cluster's shared memory (all remote loads issued
// at once: 131072 slots on 8 blocks 33 -> 29 us a call, on a state evicted
// before).  Moves: bound by HBM (183935 rows of 8 heads of 128 in bf16 37 us, 5.2
// TB/s), a warp takes 32 and copies four rows at a time.
#include <cooperative_groups.h>

#include "kv_cache.cuh"

namespace mosaic {
namespace {

namespace cg = cooperative_groups;

constexpr int kBins = 2048;
constexpr int kOwnMoves = 512;
constexpr int kMaxKeys = 48 * 1024;   // keys in shared memory; those beyond are looked up again each pass

// Weights as unsigned keys in ascending order; NaN as -inf, -0 as 0.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (w != w) w = -__int_as_float(0x7f800000);
    const uint32_t u = __float_as_uint(w + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
constexpr uint32_t kKeyInf = 0xff800000u;   // order_key(+inf), the greatest

struct EvictArgs {
    const int32_t *lens, *recent_from;
    int32_t *new_lens;
    int64_t max_len, keep, cap;   // cap: most moves of a (sequence, head)
    int32_t *count, *from, *to;
    int keys;                     // keys a block has room for
    int quads;                    // four slots from a multiple of 4 on share a page and aligned words
    int moves;                    // the selection moves the rows itself and writes new_lens (which is not lens)
};

__device__ __forceinline__ uint32_t slot_key(const KvView &kv, const EvictArgs &a, int64_t i, int h, int s, int from) {
    uint32_t off;
    const int id = kv.page_of(i, (uint32_t)s, off);
    if (id < 0) return kKeyInf;
    const int64_t at = kv.mark(id, h, off);
    const float w = kv.c.weight[at];
    if (a.recent_from && kv.c.position[at] >= from) return kKeyInf;
    return order_key(w);
}

// Moves m0 .. m0 + 31 of a job, by one warp: key and value rows, positions and
// weights.
__device__ __forceinline__ void move32(const KvView &kv, const EvictArgs &a, int64_t job, int64_t i, int h, int m0,
                                       int count) {
    const int lane = threadIdx.x & 31;
    const int es = kv.c.type == MOSAIC_KV_F32 ? 4 : 2, quads = kv.c.head_dim * es / 16;
    char *const kp = static_cast<char *>(kv.c.k), *const vp = static_cast<char *>(kv.c.v);
    int64_t se = -1, te = 0;
    if (m0 + lane < count) {
        uint32_t so, to;
        const int sid = kv.page_of(i, (uint32_t)a.from[job * a.cap + m0 + lane], so);
        const int tid = kv.page_of(i, (uint32_t)a.to[job * a.cap + m0 + lane], to);
        if (sid >= 0 && tid >= 0) {
            se = kv.element(sid, h, so) * es, te = kv.element(tid, h, to) * es;
            const int64_t sm = kv.mark(sid, h, so), tm = kv.mark(tid, h, to);
            kv.c.weight[tm] = kv.c.weight[sm];
            if (kv.c.position) kv.c.position[tm] = kv.c.position[sm];
        }
    }
    for (int j0 = 0; j0 < 32 && m0 + j0 < count; j0 += 4) {
        int64_t s[4], t[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)
            s[j] = __shfl_sync(0xffffffffu, se, j0 + j), t[j] = __shfl_sync(0xffffffffu, te, j0 + j);
        for (int b = lane; b < 2 * quads; b += 32) {
            char *pool = b < quads ? kp : vp;
            const int o = 16 * (b < quads ? b : b - quads);
            uint4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (s[j] >= 0) x[j] = *reinterpret_cast<const uint4 *>(pool + s[j] + o);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (s[j] >= 0) *reinterpret_cast<uint4 *>(pool + t[j] + o) = x[j];
        }
    }
}

template <int THREADS>
struct SelectShared {
    int hist[2][kBins];
    int warp[3][THREADS / 32];
    uint32_t low, high;   // this block's least and greatest key below kKeyInf
    int finite, total[3];
    uint32_t pick_low, pick_high;
    int pick_rank, pick_count;
};

// Exclusive sum over the block's warps of a warp-uniform value (one lane a
// warp passes it); `total` gets the block's.
template <int THREADS>
__device__ __forceinline__ int warp_base(int v, int *part, int &total) {
    const int w = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) part[w] = v;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) {
        const int x = part[k];
        before += k < w ? x : 0;
        total += x;
    }
    return before;
}

template <int THREADS>
__global__ void __launch_bounds__(THREADS) evict_select_kernel(KvView kv, EvictArgs a) {
    extern __shared__ __align__(16) uint32_t keys[];
    __shared__ SelectShared<THREADS> sh;
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
    const int64_t job = blockIdx.x / C, i = job / kv.c.kv_heads;
    const int h = (int)(job % kv.c.kv_heads);
    auto sync = [&] {
        if (C > 1) cluster.sync();
        else __syncthreads();
    };
    pdl_enter();
    const int len = kv.length(a.lens, i, a.max_len), keep = (int)(a.keep < 0x7fffffff ? a.keep : 0x7fffffff);
    if (a.moves && h == 0 && rank == 0 && tid == 0) a.new_lens[i] = min(len, keep);
    if (len <= keep) {   // the whole cluster's
        if (rank == 0 && tid == 0) a.count[job] = 0;
        return;
    }
    const int from = a.recent_from ? a.recent_from[i] : 0;
    const int per = ((len + C - 1) / C + 3) / 4 * 4, s0 = min(len, rank * per), n = min(len, s0 + per) - s0;
    if (tid == 0) sh.low = 0xffffffffu, sh.high = 0, sh.finite = 0;
    for (int b = tid; b < kBins; b += THREADS) sh.hist[0][b] = 0;
    __syncthreads();
    {
        uint32_t low = 0xffffffffu, high = 0;
        int finite = 0;
        auto take = [&](int x, uint32_t k) {
            if (x < a.keys) keys[x] = k;
            if (k < kKeyInf) low = min(low, k), high = max(high, k), ++finite;
        };
        if (a.quads) {   // four slots share a page and a 16-byte word
#pragma unroll 2
            for (int x = 4 * tid; x < n; x += 4 * THREADS) {
                uint32_t off;
                const int id = kv.page_of(i, (uint32_t)(s0 + x), off);
                const int64_t at = kv.mark(max(id, 0), h, off);
                const float4 v = *reinterpret_cast<const float4 *>(kv.c.weight + at);
                int4 p = make_int4(0, 0, 0, 0);
                if (a.recent_from) p = *reinterpret_cast<const int4 *>(kv.c.position + at);
                const float w4[4] = {v.x, v.y, v.z, v.w};
                const int p4[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (x + j < n) take(x + j, id < 0 || (a.recent_from && p4[j] >= from) ? kKeyInf : order_key(w4[j]));
            }
        } else {
#pragma unroll 4
            for (int x = tid; x < n; x += THREADS) take(x, slot_key(kv, a, i, h, s0 + x, from));
        }
        low = __reduce_min_sync(0xffffffffu, low);
        high = __reduce_max_sync(0xffffffffu, high);
        finite = __reduce_add_sync(0xffffffffu, finite);
        if (lane == 0) atomicMin(&sh.low, low), atomicMax(&sh.high, high), atomicAdd(&sh.finite, finite);
    }
    auto key = [&](int x) { return x < a.keys ? keys[x] : slot_key(kv, a, i, h, s0 + x, from); };
    sync();
    uint32_t low = 0xffffffffu, high = 0;
    int finite = 0;
    for (int q = 0; q < C; ++q) {
        const SelectShared<THREADS> *o = C > 1 ? cluster.map_shared_rank(&sh, q) : &sh;
        low = min(low, o->low), high = max(high, o->high), finite += o->finite;
    }
    int left = len - keep;   // of the keys in [low, high], so many least ones leave
    int same = 0;            // slots with the last key that leaves, where known
    if (left > finite) low = high = kKeyInf, left -= finite;
    else if (left == 1) high = low;   // one slot over the budget: the least key is known
    for (int pass = 0; low < high; ++pass) {
        int *hist = sh.hist[pass & 1];
        const int shift = max(0, 21 - __clz((int)(high - low)));
        for (int x = tid; x < n; x += THREADS) {
            const uint32_t k = key(x);
            if (k >= low && k <= high) atomicAdd(&hist[(k - low) >> shift], 1);
        }
        sync();
        // The other histogram has been read by everyone (they passed this barrier).
        for (int b = tid; b < kBins; b += THREADS) sh.hist[~pass & 1][b] = 0;
        constexpr int kOwn = kBins / THREADS;
        int own[kOwn], sum = 0;
#pragma unroll
        for (int b = 0; b < kOwn; ++b) own[b] = 0;
        if (C == 1) {
#pragma unroll
            for (int b = 0; b < kOwn; ++b) own[b] = hist[tid * kOwn + b];
        } else {   // all remote loads at once
            int far[8][kOwn];
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int b = 0; b < kOwn; ++b)
                    far[q][b] = q < C ? cluster.map_shared_rank(hist, q)[tid * kOwn + b] : 0;
#pragma unroll
            for (int q = 0; q < 8; ++q)
#pragma unroll
                for (int b = 0; b < kOwn; ++b) own[b] += far[q][b];
        }
#pragma unroll
        for (int b = 0; b < kOwn; ++b) sum += own[b];
        int incl = sum, all;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        const int of_warp = __shfl_sync(0xffffffffu, incl, 31);
        int before = warp_base<THREADS>(of_warp, sh.warp[0], all) + incl - sum;
        if (before < left && left <= before + sum) {
#pragma unroll
            for (int b = 0; b < kOwn; ++b) {
                if (before < left && left <= before + own[b]) {
                    const uint32_t to = low + ((uint32_t)(tid * kOwn + b) << shift);
                    sh.pick_low = to;
                    sh.pick_high = min(high, to + ((1u << shift) - 1));
                    sh.pick_rank = left - before, sh.pick_count = own[b];
                }
                before += own[b];
            }
        }
        __syncthreads();
        low = sh.pick_low, high = sh.pick_high, left = sh.pick_rank, same = sh.pick_count;
        __syncthreads();
    }
    const uint32_t least = low;
    const int ties = left;   // of the slots with that key, the first so many leave

    // A thread up to 32 neighbouring slots a round: ties (unless all of them
    // leave), then holes and stayers, before each.
    auto before_block = [&](int which) {
        int v = 0;
        if (C > 1) {
#pragma unroll
            for (int q = 0; q < 8; ++q) v += q < rank ? cluster.map_shared_rank(&sh, q)->total[which] : 0;
        }
        return v;
    };
    const int own = min(32, ((n + THREADS - 1) / THREADS + 3) / 4 * 4), round = own * THREADS;
    // The thread's slots whose key passes the test.
    auto which = [&](int x0, auto test) {
        uint32_t m = 0;
        if (x0 + own <= min(n, a.keys)) {   // multiples of four
            for (int x = 0; x < own; x += 4) {
                const uint4 k = *reinterpret_cast<const uint4 *>(keys + x0 + x);
                m |= ((uint32_t)test(k.x) | (uint32_t)test(k.y) << 1 | (uint32_t)test(k.z) << 2 | (uint32_t)test(k.w) << 3) << x;
            }
        } else {
            for (int x = 0; x < own && x0 + x < n; ++x) m |= (uint32_t)test(key(x0 + x)) << x;
        }
        return m;
    };
    // Sum of the threads' values before this one, and of all.
    auto scan = [&](int v, int *part, int &all) {
        int incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += y;
        }
        return warp_base<THREADS>(__shfl_sync(0xffffffffu, incl, 31), part, all) + incl - v;
    };
    const bool ranked = same != ties;   // the cluster's
    int seen = 0;                       // ties in the blocks and rounds before
    if (ranked) {
        int count = 0, all;
        for (int r = 0; r < n; r += round) count += __popc(which(r + own * tid, [&](uint32_t k) { return k == least; }));
        scan(count, sh.warp[0], all);
        if (tid == 0) sh.total[0] = all;
        sync();
        seen = before_block(0);
    }
    // The thread's slots of a round that leave and lie below keep, or stay and lie above.
    auto marked = [&](int r, uint32_t &below) {
        const int x0 = r + own * tid, k0 = keep - (s0 + x0), in = n - x0;
        below = k0 >= 32 ? 0xffffffffu : k0 <= 0 ? 0u : (1u << k0) - 1;
        const uint32_t real = min(in, own) >= 32 ? 0xffffffffu : in <= 0 ? 0u : (1u << min(in, own)) - 1;
        uint32_t out;
        if (ranked) {
            const uint32_t eq = which(x0, [&](uint32_t k) { return k == least; });
            int all;
            const int before = seen + scan(__popc(eq), sh.warp[0], all);
            seen += all;
            out = which(x0, [&](uint32_t k) { return k < least; });
            uint32_t rest = eq;
            for (int t = before; t < ties && rest; ++t) out |= rest & -rest, rest &= rest - 1;
            __syncthreads();
        } else {
            out = which(x0, [&](uint32_t k) { return k <= least; });
        }
        return ((out & below) | (~out & ~below)) & real;
    };
    int hole = 0, stay = 0, all;
    uint32_t below, mark = 0;
    const int before = seen;
    for (int r = 0; r < n; r += round) {
        mark = marked(r, below);
        hole += __popc(mark & below), stay += __popc(mark & ~below);
    }
    hole = scan(hole, sh.warp[1], all);
    if (tid == 0) sh.total[1] = all;
    stay = scan(stay, sh.warp[2], all);
    if (tid == 0) sh.total[2] = all;
    sync();
    int hole_base = before_block(1), stay_base = before_block(2);
    if (rank == C - 1 && tid == 0) a.count[job] = hole_base + sh.total[1];   // at most a.cap
    int32_t *to = a.to + job * a.cap, *src = a.from + job * a.cap;
    if (n > round) seen = before;
    for (int r = 0; r < n; r += round) {
        if (n > round) {   // several rounds: the places of each, one after the other
            mark = marked(r, below);
            __syncthreads();
            hole = scan(__popc(mark & below), sh.warp[1], all);
            const int holes = all;
            __syncthreads();
            stay = scan(__popc(mark & ~below), sh.warp[2], all);
            const int stays = all;
            hole += hole_base, stay += stay_base;
            hole_base += holes, stay_base += stays;
        } else {
            hole += hole_base, stay += stay_base;
        }
        for (uint32_t m = mark; m; m &= m - 1) {
            const int x = __ffs(m) - 1, s = s0 + r + own * tid + x;
            if (below >> x & 1u) to[hole++] = s;
            else src[stay++] = s;
        }
    }
    if (C > 1) cluster.sync();   // the others have read this block's counts
    if (a.moves) {
        __syncthreads();         // one block a job: both lists are whole
        const int n = sh.total[1];
        for (int m0 = 32 * w; m0 < n; m0 += THREADS) move32(kv, a, job, i, h, m0, n);
    }
}

__global__ void __launch_bounds__(256) evict_move_kernel(KvView kv, EvictArgs a, int chunks) {
    pdl_enter();
    const int64_t job = blockIdx.x / chunks;
    const int part = (int)(blockIdx.x % chunks);
    const int h = (int)(job % kv.c.kv_heads);
    const int64_t i = job / kv.c.kv_heads;
    if (part == 0 && h == 0 && threadIdx.x == 0) {
        const int n = kv.length(a.lens, i, a.max_len);
        a.new_lens[i] = n < a.keep ? n : (int)a.keep;
    }
    const int count = a.count[job];
    for (int m0 = 32 * (part * 8 + (threadIdx.x >> 5)); m0 < count; m0 += chunks * 256)
        move32(kv, a, job, i, h, m0, count);
}

int64_t most_moves(int64_t max_len, int64_t keep) {
    const int64_t over = max_len - keep;
    return over <= 0 ? 0 : over < keep ? over : keep;
}
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

template <int THREADS>
mosaic_status select_launch(const KvView &kv, const EvictArgs &a, int64_t blocks, int cluster, cudaStream_t st) {
    static std::atomic<unsigned long long> done{0};
    if (!ensure_smem_limit(done, evict_select_kernel<THREADS>, 4 * kMaxKeys)) return MOSAIC_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = 4 * (size_t)a.keys;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    KernelSpan span("evict_select", st);
    cudaLaunchKernelEx(&cfg, evict_select_kernel<THREADS>, kv, a);   // a failure is read by launch_status
    return launch_status();
}

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
    if (jobs > 0x7fffffff / 8) return MOSAIC_ERR_SHAPE;
    if (ws_bytes < mosaic_kv_evict_workspace(cache, max_len, keep)) return MOSAIC_ERR_WORKSPACE;
    if (!ws) return MOSAIC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ws) % 4) return MOSAIC_ERR_ALIGN;
    EvictArgs a = {lens, recent_from, new_lens, max_len, keep, most_moves(max_len, keep), nullptr, nullptr, nullptr, 0, 0, 0};
    char *w = static_cast<char *>(ws);
    a.count = reinterpret_cast<int32_t *>(w);
    a.from = reinterpret_cast<int32_t *>(w + up256(4 * (size_t)jobs));
    a.to = a.from + up256(4 * (size_t)(jobs * a.cap)) / 4;
    cudaStream_t st = as_stream(stream);
    const KvView kv(*cache);
    // As many blocks a job as there are SMs for, of 2048 slots at least.
    int cluster = 1;
    while (cluster < 8 && jobs * cluster * 2 <= 152 && max_len / (cluster * 2) >= 2048) cluster *= 2;
    while (cluster < 8 && (max_len + cluster - 1) / cluster > kMaxKeys) cluster *= 2;
    const int64_t per = ((max_len + cluster - 1) / cluster + 3) / 4 * 4;
    a.quads = cache->page_size % 4 == 0 && aligned16(cache->weight) && (!recent_from || aligned16(cache->position));
    a.keys = (int)(per < kMaxKeys ? per : kMaxKeys);
    // Few moves a job are the selecting block's own: a launch less (4097 slots to
    // 4096, 32 sequences of 8 heads: 18.4 us with two, 16.4 with one).
    a.moves = a.cap <= kOwnMoves && cluster == 1 && new_lens != lens;
    if (per > 8192) MOSAIC_TRY(select_launch<1024>(kv, a, jobs * cluster, cluster, st));
    else MOSAIC_TRY(select_launch<512>(kv, a, jobs * cluster, cluster, st));
    if (a.moves) return MOSAIC_OK;
    // One wave of blocks for the moves (32 a warp, 256 a block).
    constexpr int64_t kWave = 152 * 8;
    int64_t chunks = (a.cap + 255) / 256;
    if (chunks * jobs > kWave) chunks = kWave / jobs;
    if (chunks < 1) chunks = 1;
    {
        KernelSpan span("evict_move", st);
        const dim3 grid((unsigned)(chunks * jobs));
        if (chunks * jobs <= kWave) pdl_launch(evict_move_kernel, grid, dim3(256), 0, st, kv, a, (int)chunks);
        else evict_move_kernel<<<grid, 256, 0, st>>>(kv, a, (int)chunks);
    }
    return launch_status();
}

}  // extern "C"
