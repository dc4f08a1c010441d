// Attention of one new token per sequence over the paged cache: the entry
// point, the join of jobs that blocks share, and the gathered weights.  The
// kernel that reads the cache is in kv_attention_impl.cuh.
#include <math.h>

#include "kv_attention.cuh"

namespace mosaic {
namespace {

constexpr int kMaxGroup = 64;
// Up to here every job is one block's: nothing to join, one launch fewer.
constexpr int64_t kWholeLen = 512;

// Block (c, head): the job that block c's end cuts, one query head of it.
__global__ void __launch_bounds__(128) attend_join_kernel(AttendArgs a, AttendShape s, int dim) {
    pdl_enter();
    const int c = blockIdx.x, head = blockIdx.y;
    const int64_t job = a.split[3 * c], last = a.split[3 * c + 1], total = a.split[3 * c + 2];
    if (job < 0) return;
    const int per_seq = a.heads / a.group * a.hb, r = (int)(job % per_seq), h = r / a.hb, hb = r % a.hb;
    if (hb * s.heads + head >= a.group) return;
    const int64_t i = job / per_seq, qh = (int64_t)h * a.group + hb * s.heads + head;
    const int n = a.blocks;
    // Part k of the job: the cut block's second slot, then the first slots of the blocks after it.
    auto slot = [&](int64_t k) { return (2 * k + (k == c)) * s.heads + head; };
    auto has = [&](int64_t k) { return total * k / n < total * (k + 1) / n; };
    float top = minus_inf();
    for (int64_t k = c; k <= last; ++k)
        if (has(k)) top = fmaxf(top, a.part_ml[2 * slot(k)]);
    const float ref = top == minus_inf() ? 0.0f : top;
    for (int d = threadIdx.x; d < dim; d += 128) {
        float sum = 0.0f, out = 0.0f;
        for (int64_t k = c; k <= last; ++k) {
            if (!has(k)) continue;
            const float f = exp2f(a.part_ml[2 * slot(k)] - ref);
            sum = fmaf(f, a.part_ml[2 * slot(k) + 1], sum);
            out = fmaf(f, a.part_o[slot(k) * s.dim + d], out);
        }
        a.out[i * a.ldo + qh * dim + d] = sum == 0.0f ? 0.0f : out / sum;
        if (a.scores && d == 0) a.stats[2 * (i * a.heads + qh)] = ref, a.stats[2 * (i * a.heads + qh) + 1] = sum;
    }
}

// A thread a slot of a (sequence, key/value head): the weight that it gathers.
__global__ void __launch_bounds__(256) attend_weight_kernel(KvView kv, AttendArgs a, int64_t chunks) {
    pdl_enter();
    const int64_t jobs = kv.c.seqs * kv.c.kv_heads * chunks;
    for (int64_t b = blockIdx.x; b < jobs; b += gridDim.x) {
        const int64_t job = b / chunks, i = job / kv.c.kv_heads;
        const int h = (int)(job % kv.c.kv_heads), s = (int)(b % chunks) * 256 + threadIdx.x;
        if (s >= kv.length(a.lens, i, a.max_len)) continue;
        uint32_t off;
        const int id = kv.page_of(i, (uint32_t)s, off);
        if (id < 0) continue;
        const float *sc = a.scores + (job * a.score_rows + s) * a.group;
        const float *st = a.stats + 2 * (i * a.heads + (int64_t)h * a.group);
        float w = 0.0f;
        for (int g = 0; g < a.group; ++g)
            if (st[2 * g + 1] != 0.0f) w += exp2f(sc[g] - st[2 * g]) / st[2 * g + 1];
        float *p = kv.c.weight + kv.mark(id, h, off);
        *p = *p * a.decay + w;
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
Parts parts(const mosaic_kv_cache &c, const AttendShape &s, int64_t heads, int64_t blocks, int64_t rows) {
    Parts p = {};
    p.ml = up256(16 * (size_t)(blocks * s.heads));
    p.o = up256(8 * (size_t)(blocks * s.heads) * s.dim);
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
// Units that the lengths may add up to, and how many blocks may share them.
int64_t most_units(const mosaic_kv_cache &c, const AttendShape &s, int64_t heads, int64_t max_len) {
    const int64_t group = heads / c.kv_heads, hb = (group + s.heads - 1) / s.heads;
    return c.seqs * c.kv_heads * hb * ((max_len + s.unit - 1) / s.unit);
}
mosaic_status check(const mosaic_kv_cache *c, int64_t heads, int64_t max_len) {
    MOSAIC_TRY(kv_check(c));
    if (heads < 1 || heads > 65535 || heads % c->kv_heads || max_len < 0 || max_len > 0x7fffffff)
        return MOSAIC_ERR_SHAPE;
    if (heads / c->kv_heads > kMaxGroup) return MOSAIC_ERR_UNSUPPORTED;
    if (c->seqs * heads > 0x7fffffff || c->seqs * heads * (max_len + 1) > (int64_t)1 << 46) return MOSAIC_ERR_SHAPE;
    return MOSAIC_OK;
}
int64_t rows_of(int64_t max_len) { return (max_len + 15) / 16 * 16; }

}  // namespace
}  // namespace mosaic

using namespace mosaic;

extern "C" {

size_t mosaic_kv_attention_workspace(const mosaic_kv_cache *cache, int64_t heads, int64_t max_len) {
    if (check(cache, heads, max_len) != MOSAIC_OK) return 0;
    const AttendShape s = shape_of(*cache, heads);
    const int64_t units = most_units(*cache, s, heads, max_len);
    return parts(*cache, s, heads, units < kAttendWave ? units : kAttendWave, rows_of(max_len)).total() + 256;
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
    const int64_t units = most_units(*cache, s, heads, max_len), cap = units < kAttendWave ? units : kAttendWave;
    const Parts p = parts(*cache, s, heads, cap, rows_of(max_len));
    if (ws_bytes < p.total() + 256) return MOSAIC_ERR_WORKSPACE;
    if (!ws) return MOSAIC_ERR_ARG;
    if (reinterpret_cast<uintptr_t>(ws) % 16) return MOSAIC_ERR_ALIGN;
    AttendArgs a = {};
    a.q = q, a.ldq = ldq, a.lens = lens, a.first = first, a.max_len = max_len, a.heads = (int)heads;
    a.group = (int)(heads / cache->kv_heads), a.hb = (a.group + s.heads - 1) / s.heads;
    a.scale2 = scale * 1.44269504088896341f, a.decay = decay, a.out = out, a.ldo = ldo;
    char *w = static_cast<char *>(ws);
    a.part_ml = reinterpret_cast<float *>(w), w += p.ml;
    a.part_o = reinterpret_cast<float *>(w), w += p.o;
    a.split = reinterpret_cast<int64_t *>(w), w += p.split;
    if (cache->weight) {
        a.stats = reinterpret_cast<float *>(w), w += p.stats;
        a.scores = reinterpret_cast<float *>(w);
        a.score_rows = rows_of(max_len);
    }
    const int64_t jobs = cache->seqs * cache->kv_heads * a.hb;
    a.whole = max_len <= kWholeLen;
    if (a.whole) a.blocks = (int)jobs;
    else {
        const int wave = by_type(cache->type, [&](auto t) { return attend_wave<decltype(t)>((int)D, a.group); });
        if (wave <= 0) return MOSAIC_ERR_CUDA;
        a.blocks = (int)(cap < wave ? cap : wave);
    }
    cudaStream_t st = as_stream(stream);
    MOSAIC_TRY(by_type(cache->type, [&](auto t) { return attend_launch<decltype(t)>(*cache, a, st); }));
    if (!a.whole) {
        {
            KernelSpan span("attend_join", st);
            pdl_launch(attend_join_kernel, dim3((unsigned)a.blocks, (unsigned)s.heads), dim3(128), 0, st, a, s, (int)D);
        }
        MOSAIC_TRY(launch_status());
    }
    if (!a.scores || max_len == 0) return MOSAIC_OK;
    const int64_t chunks = (max_len + 255) / 256, all = cache->seqs * cache->kv_heads * chunks;
    const KvView kv(*cache);
    {
        KernelSpan span("attend_weight", st);
        pdl_launch(attend_weight_kernel, dim3((unsigned)(all < 152 * 8 ? all : 152 * 8)), dim3(256), 0, st, kv, a,
                   chunks);
    }
    return launch_status();
}

}  // extern "C"
