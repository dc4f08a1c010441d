// Attention of one new token per sequence over the paged cache: the entry
// point, the join of jobs that blocks share, and the gathered weights.  The
// kernel that reads the cache is in kv_attention_impl.cuh.
#include <math.h>

#include "kv_attention.cuh"

namespace mosaic {
namespace {

constexpr int kMaxGroup = 64;
// Up to these lengths every job is one block's: nothing to join, and blocks
// beyond a wave follow as others end.  Microseconds, whole jobs / shared, 8
// key/value heads of 128, bf16 (one sequence, then 16, 32, 64 of equal and 64
// of spread lengths): 256 slots 8 / 12, 9 / 15, 11 / 19, 17 / 25, 14 / 21; 512:
// 12 / 13, 13 / 18, 17 / 24, 27 / 36, 23 / 26; 1024: 20 / 15, 22 / 24, 27 / 35,
// 47 / 56, 40 / 36; 2048: 35 / 19, 38 / 34, 47 / 55, 85 / 95, 67 / 57.  Long rows
// earlier: fp32, one sequence 256 slots 11 / 14, 512: 17 / 15; 64 of spread
// lengths 512: 47 / 47, 1024: 75 / 68.  The rule is that of instances of two or
// three blocks an SM.  Those of one (full lengths, one sequence / 16 / 64): bf16
// heads of 256, 256 slots 10 / 14, 14 / 24, 54 / 61, 512: 15 / 14, 20 / 32, 76 / 80,
// 1024: 25 / 14, 29 / 44, 117 / 121; 16 query heads of 128, 512: 18 / 21, 19 / 26, 44
// / 60, 1024: 25 / 22, 28 / 31, 56 / 79; fp32 heads of 128, 512: 16 / 13, 18 / 26, 46 /
// 60, 1024: 27 / 14, 29 / 36, 83 / 96: it shares some that are faster whole.
constexpr int64_t kWholeFew = 512, kWholeMany = 1024, kManyJobs = 128, kWholeBytes = 128 * 1024;
// Heads share a unit (the blocks' warps then have a head each and nothing to
// merge) while so many jobs remain to be shared out; whole jobs while there is
// more than a wave of them.  Shared jobs with 1 / 2 / 4 heads a unit, up to 1024
// slots: one sequence 14 / 19 / 27, 16: 20 / 20 / 22, 32: 29 / 26 / 25, 64: 42 /
// 38 / 36, 256: 117 / 106 / 102.
constexpr int64_t kFewestJobs = 64;
// What a job costs beside its slots, as bytes of cache read in that time.  48
// sequences of 41 to 2000 slots on 32 heads of 128: 266 us at 0, 231 at 32 KB,
// 140 at 128 KB, 135 at 192 KB, 139 at 256 KB, 153 at 512 KB; 400 of 3 to 1500
// on 8 heads of 64, windowed: 147, 122, 95, 93, 90 (256 KB).  With four heads a
// unit 64 KB to 384 KB are within 4 and 12 per cent.
constexpr int64_t kJobBytes = 256 * 1024;

// Block (c, y): the job that block c's end cuts.  Where jobs have many parts
// (`shared`), query head y of it, its parts taken in turn by eight warps; else
// key/value head y, a warp a query head.  A lane has four channels (two rounds
// beyond 128).
__global__ void __launch_bounds__(256) attend_join_kernel(AttendArgs a, AttendShape s, int dim, bool shared) {
    __shared__ float4 rest[7][2][32];
    __shared__ float rest_sum[7];
    pdl_enter();
    const int c = blockIdx.x, n = a.blocks, lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    const int64_t job = a.split[3 * c], last = a.split[3 * c + 1], total = a.split[3 * c + 2];
    if (job < 0) return;
    const int hi = shared ? blockIdx.y / s.heads : blockIdx.y, from = shared ? w : 0, each = shared ? 8 : 1;
    const uint32_t per_seq = a.heads / a.group / a.hpu * a.hb, at = (uint32_t)job / per_seq;   // jobs: below 2^31
    const int r = (int)((uint32_t)job - at * per_seq), h = r / a.hb * a.hpu + hi, hb = r % a.hb;
    const int64_t i = at;
    // Part k of the job: the cut block's second slot, then the first slots of
    // the blocks after it (some without a unit where units are fewer than blocks).
    const int parts = (int)(last - c) + 1;
    auto has = [&](int k) { return total >= n || total * (c + k) / n < total * (c + k + 1) / n; };
    for (int head = shared ? blockIdx.y % s.heads : w; head < s.heads && hb * s.heads + head < a.group; head += shared ? s.heads : 8) {
        const int64_t qh = (int64_t)h * a.group + hb * s.heads + head;
        auto slot = [&](int k) { return ((2 * (int64_t)(c + k) + (k == 0)) * a.hpu + hi) * s.heads + head; };
        float top = minus_inf();
        for (int k = lane; k < parts; k += 32)
            if (has(k)) top = fmaxf(top, a.part_ml[2 * slot(k)]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ref = top == minus_inf() ? 0.0f : top;
        float sum = 0.0f;
        float4 out[2];
        out[0] = out[1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int k0 = from; k0 < parts; k0 += 4 * each) {   // four parts' loads, then their sums
            float m[4], l[4];
            float4 x[4][2];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = k0 + j * each;
                m[j] = minus_inf(), l[j] = 0.0f;
                x[j][0] = x[j][1] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                if (k >= parts || !has(k)) continue;
                const float *p = a.part_o + slot(k) * s.dim + 4 * lane;
                m[j] = a.part_ml[2 * slot(k)], l[j] = a.part_ml[2 * slot(k) + 1];
                if (4 * lane < s.dim) x[j][0] = *reinterpret_cast<const float4 *>(p);
                if (128 + 4 * lane < s.dim) x[j][1] = *reinterpret_cast<const float4 *>(p + 128);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float f = power2(m[j] - ref);
                sum = fmaf(f, l[j], sum);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    float4 &o = out[half];
                    o.x = fmaf(f, x[j][half].x, o.x), o.y = fmaf(f, x[j][half].y, o.y);
                    o.z = fmaf(f, x[j][half].z, o.z), o.w = fmaf(f, x[j][half].w, o.w);
                }
            }
        }
        if (shared) {
            if (w) rest[w - 1][0][lane] = out[0], rest[w - 1][1][lane] = out[1];
            if (w && lane == 0) rest_sum[w - 1] = sum;
            __syncthreads();
            if (w) return;
            for (int k = 0; k < 7; ++k) {
                sum += rest_sum[k];
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const float4 y = rest[k][half][lane];
                    out[half].x += y.x, out[half].y += y.y, out[half].z += y.z, out[half].w += y.w;
                }
            }
        }
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int d = 128 * half + 4 * lane;
            const float o[4] = {out[half].x, out[half].y, out[half].z, out[half].w};
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (d + x < dim) a.out[i * a.ldo + qh * dim + d + x] = finite_or_nan(o[x] * inv);
        }
        if (a.scores && lane == 0) a.stats[2 * (i * a.heads + qh)] = ref, a.stats[2 * (i * a.heads + qh) + 1] = inv;
    }
}

// A thread four slots of a (sequence, key/value head): the weight that they
// gather.  Bound by reading the scores (4 bytes a slot and query head); every
// load of a thread is issued before its use.
constexpr int kWeightSlots = 4 * 128;
struct WeightWalk {
    int64_t chunks, jobs_step, chunk_step;   // the grid's stride over (job, chunk of slots)
};
__global__ void __launch_bounds__(128, 6) attend_weight_kernel(KvView kv, AttendArgs a, WeightWalk walk) {
    pdl_enter();
    const int64_t jobs = kv.c.seqs * kv.c.kv_heads;
    int64_t job = blockIdx.x / walk.chunks, chunk = blockIdx.x % walk.chunks;
    for (; job < jobs; job += walk.jobs_step, chunk += walk.chunk_step) {
        if (chunk >= walk.chunks && (chunk -= walk.chunks, ++job) >= jobs) break;
        const int64_t i = job / kv.c.kv_heads;
        const int h = (int)(job - i * kv.c.kv_heads), s = (int)chunk * kWeightSlots + 4 * threadIdx.x;
        const int len = kv.length(a.lens, i, a.max_len);
        if (s >= len) continue;
        float *at[4];
        __align__(16) float old[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        uint32_t off;
        const int id = kv.page_of(i, (uint32_t)s, off);
        at[0] = id < 0 ? nullptr : kv.c.weight + kv.mark(id, h, off);
        const bool quad = a.quads && s + 4 <= len;
        if (!quad) {
#pragma unroll
            for (int j = 1; j < 4; ++j) {
                const int jd = s + j < len ? kv.page_of(i, (uint32_t)(s + j), off) : -1;
                at[j] = jd < 0 ? nullptr : kv.c.weight + kv.mark(jd, h, off);
            }
        }
        const int64_t head = i * a.heads + (int64_t)h * a.group;
        const float *sc = a.scores + head * a.score_rows + s;
        const float2 *st = reinterpret_cast<const float2 *>(a.stats) + head;
        float w[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int g0 = 0; g0 < a.group; g0 += 8) {
            float4 x[8];
#pragma unroll
            for (int g = 0; g < 8; ++g)
                if (g0 + g < a.group) x[g] = *reinterpret_cast<const float4 *>(sc + (g0 + g) * a.score_rows);
            if (g0 == 0) {
                if (quad) {
                    if (at[0]) *reinterpret_cast<float4 *>(old) = *reinterpret_cast<const float4 *>(at[0]);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (at[j]) old[j] = *at[j];
                }
            }
#pragma unroll
            for (int g = 0; g < 8; ++g)
                if (g0 + g < a.group) {
                    const float2 y = st[g0 + g];
                    w[0] = fmaf(power2(x[g].x - y.x), y.y, w[0]);
                    w[1] = fmaf(power2(x[g].y - y.x), y.y, w[1]);
                    w[2] = fmaf(power2(x[g].z - y.x), y.y, w[2]);
                    w[3] = fmaf(power2(x[g].w - y.x), y.y, w[3]);
                }
        }
        if (a.first) {   // slots below the bound gather nothing (and may have no score)
            const int low = a.first[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float *p = quad ? at[0] ? at[0] + j : nullptr : at[j];
                if (p && kv.c.position[p - kv.c.weight] < low) w[j] = 0.0f;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) old[j] = fmaf(old[j], a.decay, w[j]);
        if (quad) {
            if (at[0]) *reinterpret_cast<float4 *>(at[0]) = *reinterpret_cast<const float4 *>(old);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (at[j]) *at[j] = old[j];
        }
    }
}

size_t up256(size_t v) { return (v + 255) / 256 * 256; }

template <class F>
auto by_type(int type, F f) {
    return type == MOSAIC_KV_F32 ? f(float()) : type == MOSAIC_KV_BF16 ? f(__nv_bfloat16()) : f(__half());
}

// The parts of the workspace, in order; `base` may be null (sizes only).
struct Parts {
    size_t ml, o, split, stats, scores;
    size_t total() const { return ml + o + split + stats + scores; }
};
// blocks: those that share the work (0: every job is one block's).
Parts parts(const mosaic_kv_cache &c, const AttendShape &s, int64_t heads, int64_t blocks, int64_t rows) {
    Parts p = {};
    p.ml = up256(16 * (size_t)(blocks * s.most_heads * s.heads));
    p.o = up256(8 * (size_t)(blocks * s.most_heads * s.heads) * s.dim);
    p.split = up256(24 * (size_t)blocks);
    if (c.weight) {
        p.stats = up256(8 * (size_t)(c.seqs * heads));
        p.scores = up256(4 * (size_t)(c.seqs * heads) * rows);
    }
    return p;
}
AttendShape shape_of(const mosaic_kv_cache &c, int64_t heads) {
    const int group = (int)(heads / c.kv_heads);
    return by_type(c.type, [&](auto t) { return attend_shape<decltype(t)>(c.head_dim, group); });
}
// How many blocks may share the units that the lengths may add up to.
int64_t most_blocks(const mosaic_kv_cache &c, const AttendShape &s, int64_t heads, int64_t max_len) {
    const int64_t group = heads / c.kv_heads, hb = (group + s.heads - 1) / s.heads;
    const int64_t units = c.seqs * c.kv_heads * hb * ((max_len + s.unit - 1) / s.unit);
    const bool many = c.seqs * c.kv_heads * hb >= kManyJobs;
    const int64_t row = c.head_dim * kv_element_bytes(c.type);
    const bool whole = max_len <= (many ? kWholeMany : kWholeFew) && max_len * row <= (many ? 2 : 1) * kWholeBytes;
    return whole ? 0 : units < kAttendWave ? units : kAttendWave;
}
mosaic_status check(const mosaic_kv_cache *c, int64_t heads, int64_t max_len) {
    MOSAIC_TRY(kv_check(c));
    if (heads < 1 || heads > 65535 || heads % c->kv_heads || max_len < 0 || max_len > 0x7fffffff)
        return MOSAIC_ERR_SHAPE;
    if (heads / c->kv_heads > kMaxGroup) return MOSAIC_ERR_UNSUPPORTED;
    if (c->seqs * heads > 0x7fffffff || c->seqs * heads * (max_len + 1) > (int64_t)1 << 46) return MOSAIC_ERR_SHAPE;
    // Units of a sequence (16 slots or more of a head, and a job's cost) are counted in 31 bits.
    if ((max_len / 16 + 4096) * heads > 0x7fffffff) return MOSAIC_ERR_SHAPE;
    return MOSAIC_OK;
}
int64_t rows_of(int64_t max_len) { return (max_len + 15) / 16 * 16; }

}  // namespace

// Reads and clears the timeout words of the attention kernels (after a stream sync).
mosaic_status kv_status() {
    const mosaic_status a = attend_status<float>(), b = attend_status<__nv_bfloat16>(), c = attend_status<__half>();
    return a != MOSAIC_OK ? a : b != MOSAIC_OK ? b : c;
}

}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_kv_attention_workspace(const mosaic_kv_cache *cache, int64_t heads, int64_t max_len) {
    if (check(cache, heads, max_len) != MOSAIC_OK) return 0;
    const AttendShape s = shape_of(*cache, heads);
    return parts(*cache, s, heads, most_blocks(*cache, s, heads, max_len), rows_of(max_len)).total();
}

mosaic_status mosaic_kv_attention(const mosaic_kv_cache *cache, const float *q, int64_t ldq, int64_t heads,
                                  const int32_t *lens, int64_t max_len, const int32_t *first, float scale,
                                  float decay, float *out, int64_t ldo, void *ws, size_t ws_bytes, void *stream) {
    RoleScope role("kv_attention");
    MOSAIC_TRY(check(cache, heads, max_len));
    const int64_t D = cache->head_dim;
    if (ldq < heads * D || ldo < heads * D) return MOSAIC_ERR_SHAPE;
    if (!isfinite(scale) || !isfinite(decay)) return MOSAIC_ERR_ARG;
    if (cache->seqs == 0) return MOSAIC_OK;
    if (!q || !out || !lens || (first && !cache->position)) return MOSAIC_ERR_ARG;
    const AttendShape s = shape_of(*cache, heads);
    const int64_t cap = most_blocks(*cache, s, heads, max_len);
    const Parts p = parts(*cache, s, heads, cap, rows_of(max_len));
    if (ws_bytes < p.total()) return MOSAIC_ERR_WORKSPACE;
    if (!ws && p.total()) return MOSAIC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ws) % 16) return MOSAIC_ERR_ALIGN;
    AttendArgs a = {};
    a.q = q, a.ldq = ldq, a.lens = lens, a.first = first, a.max_len = max_len, a.heads = (int)heads;
    a.group = (int)(heads / cache->kv_heads), a.hb = (a.group + s.heads - 1) / s.heads;
    a.hpu = 1;
    const int64_t one = cache->seqs * cache->kv_heads * a.hb;   // jobs with a key/value head each
    a.whole = cap == 0;
    for (int x = 2; x <= s.most_heads; ++x) {
        if (s.most_heads % x || cache->kv_heads % x || (x > s.buffers && x != s.most_heads)) continue;
        if (a.whole ? one / a.hpu > 152 * s.resident : one / x >= kFewestJobs) a.hpu = x;
    }
    a.scale2 = scale * 1.44269504088896341f, a.decay = decay, a.out = out, a.ldo = ldo;
    char *w = static_cast<char *>(ws);
    a.part_ml = reinterpret_cast<float *>(w), w += p.ml;
    a.part_o = reinterpret_cast<float *>(w), w += p.o;
    a.split = reinterpret_cast<int64_t *>(w), w += p.split;
    if (cache->weight) {
        a.stats = reinterpret_cast<float *>(w), w += p.stats;
        a.scores = reinterpret_cast<float *>(w);
        a.score_rows = rows_of(max_len);
        a.quads = cache->page_size % 4 == 0 && aligned16(cache->weight);
    }
    const int64_t jobs = cache->seqs * (cache->kv_heads / a.hpu) * a.hb;
    a.blocks = (int)(a.whole ? jobs : cap);
    const int64_t unit_bytes = 2 * s.unit * D * kv_element_bytes(cache->type);
    a.job_cost = (int)((kJobBytes + unit_bytes / 2) / unit_bytes);
    cudaStream_t st = as_stream(stream);
    MOSAIC_TRY(by_type(cache->type, [&](auto t) { return attend_launch<decltype(t)>(*cache, a, a.blocks, st); }));
    if (!a.whole) {
        {
            KernelSpan span("attend_join", st);
            const bool shared = jobs * 4 <= a.blocks;
            const dim3 grid((unsigned)a.blocks, (unsigned)(a.hpu * (shared ? s.heads : 1)));
            pdl_launch(attend_join_kernel, grid, dim3(256), 0, st, a, s, (int)D, shared);
        }
        MOSAIC_TRY(launch_status());
    }
    if (!a.scores || max_len == 0 || (a.whole && a.hb == 1)) return MOSAIC_OK;
    const int64_t chunks = (max_len + kWeightSlots - 1) / kWeightSlots, all = cache->seqs * cache->kv_heads * chunks;
    const KvView kv(*cache);
    {
        KernelSpan span("attend_weight", st);
        const int64_t grid = all < 152 * 6 ? all : 152 * 6;
        const WeightWalk walk = {chunks, grid / chunks, grid % chunks};
        pdl_launch(attend_weight_kernel, dim3((unsigned)grid), dim3(128), 0, st, kv, a, walk);
    }
    return launch_status();
}

}  // extern "C"
