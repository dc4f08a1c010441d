// The append of kv_append.cu with norms of the query and key heads, into any
// cache, and with or without them into a 4-bit one.
//
//   y = rotate((x r) gain),  r = 1 / sqrt(mean x^2 + eps) over a head
//
// Bound by HBM as kv_append.cu is (fp32 rows in, fp32 queries and the cache's
// rows out: 5003 tokens into an fp32 cache 80 us, 91% of the copy rate); the same
// split: a block the heads of one token, a thread 4 + 4 channels of a head, half a
// head apart, two heads in flight.  The threads of a head lie in one warp (their
// number rounded up to a power of two), which sums the squares.
//
// 4-bit rows: 32 neighbouring channels share a step and a base, and the halves
// of a head that a thread rotates do not lie in one group, so rotated keys and
// values of a round go through shared memory; there a thread takes the 8
// channels of a word of codes, four threads a group.  A code is the nearest of
// 16 levels, and a key next to the border between two must not fall to either
// side by the way it was computed: sines, cosines and r come from
// two-float arithmetic (Dekker, "A floating-point technique for extending the
// available precision", 1971; Taylor's series and one Newton step) rounded once,
// and the rest is IEEE operations without contraction.  Doubles would do the
// same at a sixty-fourth of the rate.  Keys and values go first and are packed by
// all warps while the queries come (a thread a group of 32: 42 us on 2048 tokens
// of 64 + 16 heads, two of eight warps at work; now 35 with 71% of the issue
// slots taken).
//
// Squares of channels past 2^-50 or 2^50 need not be fp32 numbers: a warp with a
// head whose mean is not an ordinary one scales it by a power of two and sums
// again (the test costs 1%: 36.9 -> 37.3 us with reading back, fp32 78.9 -> 79.9; the
// second sum written out instead of a loop: 38.9, 80.0).
#include "kv_append.cuh"

namespace mosaic {
namespace {

// Threads, blocks an SM and heads in flight of a thread.  2048 tokens of 64 + 16 heads of 128 with norms / 9001 of 28 +
// 8 without, 4 bits: 42 / 72 us (4 blocks, 4 heads), 37 / 67 (4, 2), 35 / 64 (5, 2), 36 / 62 (6, 1); 5003 of 32 + 64 with
// norms, fp32: 84, 86, 82, 84.
constexpr int kThreads = 256, kResident = 5, kRound = 2;

// A sum h + l of two floats, |l| at most half an ulp of h.
struct Two {
    float h, l;
};
__device__ __forceinline__ Two fast_two(float a, float b) {   // |a| >= |b|
    const float s = __fadd_rn(a, b);
    return {s, __fsub_rn(b, __fsub_rn(s, a))};
}
__device__ __forceinline__ Two two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), t = __fsub_rn(s, a);
    return {s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, t)), __fsub_rn(b, t))};
}
__device__ __forceinline__ Two add(Two a, Two b) {
    const Two t = two_sum(a.h, b.h);
    return fast_two(t.h, __fadd_rn(t.l, __fadd_rn(a.l, b.l)));
}
__device__ __forceinline__ Two mul(Two a, Two b) {
    const float p = __fmul_rn(a.h, b.h);
    return fast_two(p, __fmaf_rn(a.h, b.l, __fmaf_rn(a.l, b.h, __fmaf_rn(a.h, b.h, -p))));
}
__host__ __device__ constexpr Two two(double x) { return {(float)x, (float)(x - (double)(float)x)}; }

// Cosine and sine of phase / 2^32 turns, rounded once (2^-36 relative before
// that): Taylor's series on an eighth of a turn either side of 0.
__device__ __forceinline__ void spin(int32_t phase, float &cosine, float &sine) {
    const uint32_t quarter = ((uint32_t)phase + 0x20000000u) >> 30;
    const int32_t rest = (int32_t)((uint32_t)phase - (quarter << 30));   // -2^29 .. 2^29 - 1
    constexpr Two pi31 = two(3.14159265358979323846 * 0x1p-31);
    const Two x = mul(two_sum((float)(rest & ~0xff), (float)(rest & 0xff)), pi31);
    const Two z = mul(x, x);
    constexpr Two s3 = two(-1.0 / 6), s5 = two(1.0 / 120), c2 = two(-0.5), c4 = two(1.0 / 24), c6 = two(-1.0 / 720);
    const float a = fmaf(z.h, fmaf(z.h, fmaf(z.h, (float)(1.0 / 6227020800.0), (float)(-1.0 / 39916800.0)),
                                   (float)(1.0 / 362880.0)), (float)(-1.0 / 5040.0));
    const float b = fmaf(z.h, fmaf(z.h, (float)(1.0 / 479001600.0), (float)(-1.0 / 3628800.0)), (float)(1.0 / 40320.0));
    const Two s = add(x, mul(x, mul(z, add(s3, mul(z, add(s5, {__fmul_rn(z.h, a), 0.0f}))))));
    const Two c = add({1.0f, 0.0f}, mul(z, add(c2, mul(z, add(c4, mul(z, add(c6, {__fmul_rn(z.h, b), 0.0f})))))));
    cosine = quarter & 1 ? s.h : c.h;
    sine = quarter & 1 ? c.h : s.h;
    if (quarter == 1 || quarter == 2) cosine = -cosine;
    if (quarter & 2) sine = -sine;
}
// Means of squares between these lose nothing that counts below 2^-149 and have no sum past 2^108.
__device__ __forceinline__ bool ordinary(float mean) { return mean > 0x1p-100f && mean < 0x1p100f; }
// 1 / sqrt(a), rounded once (ordinary a; others are zeros, infinities and NaN).
__device__ __forceinline__ float root(Two a) {
    const float y = rsqrtf(a.h);
    if (!ordinary(a.h)) return y;
    const float t = __fmul_rn(y, y), tl = __fmaf_rn(y, y, -t);
    const float p = __fmul_rn(a.h, t);   // near 1
    const float pl = __fmaf_rn(a.l, t, __fmaf_rn(a.h, tl, __fmaf_rn(a.h, t, -p)));
    const float d = __fsub_rn(__fsub_rn(1.0f, p), pl);
    return __fmaf_rn(__fmul_rn(0.5f, y), d, y);
}

struct NormArgs {
    float eps;
    const float *q_gain, *k_gain;
    Two over_dim;      // 1 / head_dim
    int log_threads;   // of a head: head_dim / 8, rounded up to a power of two
};

// Channel c of a staged row: 32 and 4 floats of padding (threads read 32 neighbours each).
__device__ __forceinline__ int staged(int c) { return c + c / 32 * 4; }

// Sum over the threads of a head (a power of two of neighbours).
__device__ __forceinline__ float head_sum(float x, int threads) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < threads) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}
// mean of the head's squares + eps, to 2^-40.
__device__ __forceinline__ Two exact_mean(const Load4 &x, const Load4 &y, bool live, int threads, float eps, Two over_dim) {
    Two z = {0.0f, 0.0f};
    if (live) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = i < 4 ? x.x[i & 3] : y.x[i & 3], p = __fmul_rn(v, v);
            const Two w = two_sum(z.h, p);
            z = {w.h, __fadd_rn(z.l, __fadd_rn(w.l, __fmaf_rn(v, v, -p)))};
        }
    }
    z = fast_two(z.h, z.l);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < threads) z = add(z, {__shfl_xor_sync(0xffffffffu, z.h, o), __shfl_xor_sync(0xffffffffu, z.l, o)});
    return add(mul(z, over_dim), {eps, 0.0f});
}
// A head with other than ordinary means (`far`) is scaled by the power of two that brings the larger of its channels
// and sqrt(eps) to [1, 4): x r is the same, but for channels that then are below 2^-126.  Returns eps to that scale.
__device__ __forceinline__ float rescale(Load4 &x, Load4 &y, bool live, bool far, int threads, float eps) {
    float top = 0.0f;
    if (live) {
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, fmaxf(fabsf(x.x[i]), fabsf(y.x[i])));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        if (o < threads) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    top = fmaxf(top, sqrtf(eps));
    const int e = min(max((int)(__float_as_uint(top) >> 23) - 127, -126), 126);
    const float up = far && top < __int_as_float(0x7f800000) ? __uint_as_float((uint32_t)(127 - e) << 23) : 1.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) x.x[i] *= up, y.x[i] *= up;
    return eps * up * up;
}
template <bool kExact>
__device__ __forceinline__ void turn(float &p, float &q, float c, float s) {
    const float p0 = p, q0 = q;
    if constexpr (kExact) {
        p = __fsub_rn(__fmul_rn(p0, c), __fmul_rn(q0, s));
        q = __fadd_rn(__fmul_rn(q0, c), __fmul_rn(p0, s));
    } else {
        p = p0 * c - q0 * s;
        q = q0 * c + p0 * s;
    }
}

template <class T, bool kNorm, bool kVec>
__global__ void __launch_bounds__(kThreads, kResident) append_norm_kernel(KvView kv, AppendArgs a, NormArgs nm) {
    constexpr bool kPacked = std::is_same<T, Q4>::value;
    __shared__ __align__(16) float cs[128], sn[128], gain[kNorm ? 512 : 4];   // gains: the queries', then the keys'
    __shared__ __align__(16) float stage[kPacked ? kRound * kThreads * 9 : 4];
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (t >= a.l) return;
    const int D = kv.c.head_dim, rot = a.rope.rot_dim, threads = 1 << nm.log_threads;
    const int u = threadIdx.x & (threads - 1), lane = threadIdx.x >> nm.log_threads, lanes = kThreads >> nm.log_threads;
    const bool in = 8 * u < D, spins = 8 * u < rot;
    // The thread's channels c0 .. c0 + 3 and c1 .. c1 + 3 of every head, in the
    // halves of the channels that turn or of those that do not.
    const int c0 = spins ? 4 * u : rot + 4 * (u - rot / 8), c1 = c0 + (spins ? rot : D - rot) / 2;
    const int H = a.heads, KV = kv.c.kv_heads;
    const int first = blockIdx.x * a.share, last = min(first + a.share, H + 2 * KV), queries = min(last, H);
    const float *row = a.qkv + t * a.ldx;
    Load4 xs[kRound], ys[kRound];
    auto load = [&](int h, int end) {   // heads h + lane, + lanes and so on, below end
        const float *p = row + (h + lane) * D;
#pragma unroll
        for (int k = 0; k < kRound; ++k, p += lanes * D)
            if (in && h + lane + k * lanes < end) xs[k] = load4(p + c0, kVec), ys[k] = load4(p + c1, kVec);
    };
    int base = max(first, H);   // keys and values first: they are packed while the queries come
    if (base < last) load(base, last);
    else load(first, queries);
    if constexpr (kNorm)
        for (int j = threadIdx.x; j < 2 * D; j += kThreads) {
            const float *g = j < D ? nm.q_gain : nm.k_gain;
            gain[j] = g ? g[j < D ? j : j - D] : 1.0f;
        }
    if ((int)threadIdx.x < rot / 2) {
        const int j = threadIdx.x;
        int ax = a.rope.axis ? a.rope.axis[j] : 0;
        ax = (uint32_t)ax < (uint32_t)a.rope.axes ? ax : 0;
        const int64_t pos = a.rope.pos[ax * a.rope.ldp + t];
        const int32_t phase = (int32_t)(((uint64_t)pos * a.rope.turns[j]) >> 32);
        if constexpr (kPacked) spin(phase, cs[j], sn[j]);
        else sincospif((float)phase * 0x1p-31f, &sn[j], &cs[j]);
    }
    int id = -1;
    int64_t at = 0, mark = 0;   // of head 0
    if (base < last) {
        const int64_t sq = a.seq[t], sl = a.slot[t];
        uint32_t off = 0;
        if (sq >= 0 && sq < kv.c.seqs && sl >= 0 && sl < kv.slots()) id = kv.page_of(sq, (uint32_t)sl, off);
        if (id >= 0) at = kv.element(id, 0, off), mark = kv.mark(id, 0, off);
    }
    __syncthreads();
    float c[4], s[4];   // of c0 + i with c1 + i, or of neighbours
    if (spins) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = !a.rope.interleaved ? c0 + i : i < 2 ? c0 / 2 + i : c1 / 2 + i - 2;
            c[i] = cs[j], s[i] = sn[j];
        }
    }
    auto scale = [&](Load4 &x, Load4 &y, float r, const float *g) {
        const Load4 g0 = load4(g + c0, true), g1 = load4(g + c1, true);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x.x[i] = __fmul_rn(__fmul_rn(x.x[i], r), g0.x[i]);
            y.x[i] = __fmul_rn(__fmul_rn(y.x[i], r), g1.x[i]);
        }
    };
    auto rotate = [&](Load4 &x, Load4 &y, auto exact) {
        constexpr bool kExact = decltype(exact)::value;
        if (!a.rope.interleaved) {
#pragma unroll
            for (int i = 0; i < 4; ++i) turn<kExact>(x.x[i], y.x[i], c[i], s[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; i += 2)
                turn<kExact>(x.x[i], x.x[i + 1], c[i / 2], s[i / 2]), turn<kExact>(y.x[i], y.x[i + 1], c[2 + i / 2], s[2 + i / 2]);
        }
    };
    // 1 / rms of a head (`head`: one that counts; `live`: the thread has channels of it); rounded once if `exact`.
    auto head_root = [&](Load4 &x, Load4 &y, bool head, bool live, auto exact) {
        float eps = nm.eps;
#pragma unroll 1
        for (bool again = false;; again = true) {
            Two mean;
            if constexpr (decltype(exact)::value) {
                mean = exact_mean(x, y, live, threads, eps, nm.over_dim);
            } else {
                float ss = 0.0f;
                if (live) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss = fmaf(x.x[i], x.x[i], fmaf(y.x[i], y.x[i], ss));
                }
                mean.h = fmaf(head_sum(ss, threads), nm.over_dim.h, eps);
            }
            const bool far = head && !ordinary(mean.h);
            if (again || !__any_sync(0xffffffffu, far)) {
                if constexpr (decltype(exact)::value) return root(mean);
                else return rsqrtf(mean.h);
            }
            eps = rescale(x, y, live, far, threads, eps);
        }
    };

    for (; base < last; base += kRound * lanes) {   // the block's: shuffles and barriers inside
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            if (base + k * lanes >= last) break;   // the block's
            const int h = base + k * lanes + lane, g = h - H < KV ? h - H : h - H - KV;
            const bool live = in && h < last, key = h < H + KV;
            Load4 &x = xs[k], &y = ys[k];
            if (kNorm && __any_sync(0xffffffffu, key)) {   // not a warp of values alone
                const float r = head_root(x, y, key && h < last, live, std::integral_constant<bool, kPacked>());
                if (live && key) scale(x, y, r, gain + D);
            }
            if (!live || id < 0) continue;
            if (spins && key) rotate(x, y, std::integral_constant<bool, kPacked>());
            if constexpr (kPacked) {
                float *o = stage + (k * lanes + lane) * (D + D / 8);
                store4(o + staged(c0), x, true);
                store4(o + staged(c1), y, true);
            } else {
                T *o = static_cast<T *>(key ? kv.c.k : kv.c.v) + at + g * kv.c.head_stride;
                put4(o + c0, x);
                put4(o + c1, y);
            }
            if (u == 0 && key) {
                if (kv.c.position) kv.c.position[mark + g * kv.c.page_size] = a.index[t];
                if (kv.c.weight) kv.c.weight[mark + g * kv.c.page_size] = 0.0f;
            }
        }
        const int next = base + kRound * lanes;
        if (next < last) load(next, last);
        else load(first, queries);
        if (!kPacked || id < 0) continue;   // the block's
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRound; ++k) {   // a thread 8 channels
            if (base + k * lanes >= last) break;   // the block's
            const int r = k * lanes + lane, h = base + r - H;
            const bool mine = in && base + r < last;
            uint32_t codes;
            const uint32_t scales = q4_pack(stage + (mine ? r * (D + D / 8) + staged(8 * u) : 0), codes);
            if (mine) {
                char *o = (h < KV ? static_cast<char *>(kv.c.k) : static_cast<char *>(kv.c.v)) + at + (h < KV ? h : h - KV) * kv.c.head_stride;
                *reinterpret_cast<uint32_t *>(o + 4 * u) = codes;
                if (u % 4 == 0) *reinterpret_cast<uint32_t *>(o + D / 2 + u) = scales;
            }
        }
        if (next < last) __syncthreads();
    }
    float *q = a.q + t * a.ldq + (first + lane) * D;
    for (base = first; base < queries; base += kRound * lanes) {
#pragma unroll
        for (int k = 0; k < kRound; ++k, q += lanes * D) {
            if (base + k * lanes >= queries) break;   // the block's
            const bool live = in && base + k * lanes + lane < queries;
            Load4 &x = xs[k], &y = ys[k];
            if constexpr (kNorm) {
                const float r = head_root(x, y, base + k * lanes + lane < queries, live, std::false_type());
                if (live) scale(x, y, r, gain);
            }
            if (!live) continue;
            if (spins) rotate(x, y, std::false_type());
            store4(q + c0, x, kVec);
            store4(q + c1, y, kVec);
        }
        load(base + kRound * lanes, queries);
    }
}

}  // namespace

mosaic_status append_norm_launch(const mosaic_kv_cache &c, AppendArgs a, const mosaic_head_norm *norm, cudaStream_t st) {
    const KvView kv(c);
    NormArgs nm = {};
    if (norm) nm.eps = norm->eps, nm.q_gain = norm->q_gain, nm.k_gain = norm->k_gain;
    nm.over_dim = two(1.0 / kv.c.head_dim);
    while (8 << nm.log_threads < c.head_dim) ++nm.log_threads;
    const dim3 grid = append_grid(c, a, kThreads >> nm.log_threads);
    {
        KernelSpan span("append_norm", st);
        auto go = [&](auto t, auto on) {
            if (a.vec) append_norm_kernel<decltype(t), decltype(on)::value, true><<<grid, kThreads, 0, st>>>(kv, a, nm);
            else append_norm_kernel<decltype(t), decltype(on)::value, false><<<grid, kThreads, 0, st>>>(kv, a, nm);
        };
        if (c.type == MOSAIC_KV_F32) go(float(), std::true_type());
        else if (c.type == MOSAIC_KV_BF16) go(__nv_bfloat16(), std::true_type());
        else if (c.type == MOSAIC_KV_F16) go(__half(), std::true_type());
        else if (norm) go(Q4(), std::true_type());
        else go(Q4(), std::false_type());
    }
    return launch_status();
}

}  // namespace mosaic
