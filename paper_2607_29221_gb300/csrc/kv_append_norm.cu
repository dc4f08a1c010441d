// The append of kv_append.cu with norms of the query and key heads, into any
// cache, and with or without them into a 4-bit one.
//
//   y = rotate((x r) gain),  r = 1 / sqrt(mean x^2 + eps) over a head
//
// Bound by HBM as kv_append.cu is (fp32 rows in, fp32 queries and the cache's
// rows out); the same split: a block the heads of one token, a thread 4 + 4
// channels of a head, half a head apart, four heads in flight.  The threads of
// a head lie in one warp (their number rounded up to a power of two), which
// sums the squares.
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
// same at a sixty-fourth of the rate.
#include "kv_append.cuh"

namespace mosaic {
namespace {

constexpr int kThreads = 256, kRound = 4;   // heads in flight of a thread

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
// 1 / sqrt(a), rounded once but where a is not a normal number.
__device__ __forceinline__ float root(Two a) {
    const float y = rsqrtf(a.h);
    if (!(a.h > 0x1p-100f && a.h < 0x1p100f)) return y;
    const float t = __fmul_rn(y, y), tl = __fmaf_rn(y, y, -t);
    const float p = __fmul_rn(a.h, t);   // near 1
    const float pl = __fmaf_rn(a.l, t, __fmaf_rn(a.h, tl, __fmaf_rn(a.h, t, -p)));
    const float d = __fsub_rn(__fsub_rn(1.0f, p), pl);
    return __fmaf_rn(__fmul_rn(0.5f, y), d, y);
}

struct NormArgs {
    float eps;
    int on;
    const float *q_gain, *k_gain;
    Two over_dim;   // 1 / head_dim
};

template <class T>
__global__ void __launch_bounds__(kThreads) append_norm_kernel(KvView kv, AppendArgs a, NormArgs nm) {
    constexpr bool kExact = std::is_same<T, Q4>::value;
    __shared__ __align__(16) float cs[128], sn[128];
    __shared__ __align__(16) float stage[kExact ? kRound * kThreads * 8 : 4];
    const int64_t t = blockIdx.y + (int64_t)blockIdx.z * 65535;
    if (t >= a.l) return;
    const int D = kv.c.head_dim, units = D / 8, rot = a.rope.rot_dim;
    int pu = 1;   // threads of a head
    while (pu < units) pu *= 2;
    const int u = threadIdx.x % pu, lane = threadIdx.x / pu, lanes = kThreads / pu;
    const bool in = u < units, spins = 8 * u < rot;
    const int c0 = spins ? 4 * u : rot + 4 * (u - rot / 8), c1 = c0 + (spins ? rot : D - rot) / 2;
    const int H = a.heads, KV = kv.c.kv_heads;
    const int first = blockIdx.x * a.share, last = min(first + a.share, H + 2 * KV);
    const float *row = a.qkv + t * a.ldx;
    float *qrow = a.q + t * a.ldq;
    Load4 xs[kRound], ys[kRound];
    auto load = [&](int h0) {
#pragma unroll
        for (int k = 0; k < kRound; ++k)
            if (in && h0 + k * lanes < last) {
                xs[k] = load4(row + (int64_t)(h0 + k * lanes) * D + c0, a.vec);
                ys[k] = load4(row + (int64_t)(h0 + k * lanes) * D + c1, a.vec);
            }
    };
    int base = first;
    load(base + lane);   // under way while the phases are looked up
    for (int j = threadIdx.x; j < rot / 2; j += kThreads) {
        int ax = a.rope.axis ? a.rope.axis[j] : 0;
        ax = (uint32_t)ax < (uint32_t)a.rope.axes ? ax : 0;
        const int64_t pos = a.rope.pos[ax * a.rope.ldp + t];
        const int32_t phase = (int32_t)(((uint64_t)pos * a.rope.turns[j]) >> 32);
        if constexpr (kExact) spin(phase, cs[j], sn[j]);
        else sincospif((float)phase * 0x1p-31f, &sn[j], &cs[j]);
    }
    const int64_t sq = a.seq[t], sl = a.slot[t];
    int id = -1;
    uint32_t off = 0;
    if (sq >= 0 && sq < kv.c.seqs && sl >= 0 && sl < kv.slots()) id = kv.page_of(sq, (uint32_t)sl, off);
    auto gains = [&](const float *g, Load4 &x, Load4 &y) {
        for (int i = 0; i < 4; ++i) x.x[i] = g && in ? g[c0 + i] : 1.0f, y.x[i] = g && in ? g[c1 + i] : 1.0f;
    };
    Load4 gq[2], gk[2];
    if (nm.on) gains(nm.q_gain, gq[0], gq[1]), gains(nm.k_gain, gk[0], gk[1]);
    __syncthreads();
    for (; base < last; base += kRound * lanes) {   // the block's: shuffles and barriers inside
#pragma unroll
        for (int k = 0; k < kRound; ++k) {
            const int h = base + k * lanes + lane;
            const bool live = in && h < last;
            Load4 &x = xs[k], &y = ys[k];
            if (nm.on && base + k * lanes < min(last, H + KV)) {
                float r, ss = 0.0f;
                if (live) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) ss = fmaf(x.x[i], x.x[i], fmaf(y.x[i], y.x[i], ss));
                }
                for (int o = pu / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
                r = rsqrtf(fmaf(ss, nm.over_dim.h, nm.eps));
                if constexpr (kExact) {
                    if (__any_sync(0xffffffffu, h >= H && h < H + KV)) {
                        Two s = {0.0f, 0.0f};
                        if (live) {
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                const float v = i < 4 ? x.x[i & 3] : y.x[i & 3], p = __fmul_rn(v, v);
                                s = add(s, {p, __fmaf_rn(v, v, -p)});
                            }
                        }
                        for (int o = pu / 2; o > 0; o >>= 1)
                            s = add(s, {__shfl_xor_sync(0xffffffffu, s.h, o), __shfl_xor_sync(0xffffffffu, s.l, o)});
                        const float rk = root(add(mul(s, nm.over_dim), {nm.eps, 0.0f}));
                        r = h >= H ? rk : r;
                    }
                }
                if (h < H + KV) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x.x[i] = __fmul_rn(__fmul_rn(x.x[i], r), h < H ? gq[0].x[i] : gk[0].x[i]);
                        y.x[i] = __fmul_rn(__fmul_rn(y.x[i], r), h < H ? gq[1].x[i] : gk[1].x[i]);
                    }
                }
            }
            if (!live) continue;
            if (spins && h < H + KV) {
                auto turn = [&](float &p, float &q, int j) {
                    const float c = cs[j], s = sn[j], p0 = p, q0 = q;
                    if constexpr (kExact) {
                        p = __fsub_rn(__fmul_rn(p0, c), __fmul_rn(q0, s));
                        q = __fadd_rn(__fmul_rn(q0, c), __fmul_rn(p0, s));
                    } else {
                        p = p0 * c - q0 * s;
                        q = q0 * c + p0 * s;
                    }
                };
                if (!a.rope.interleaved) {   // channel c0 + i with c1 + i
#pragma unroll
                    for (int i = 0; i < 4; ++i) turn(x.x[i], y.x[i], c0 + i);
                } else {                     // neighbours
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        turn(x.x[i], x.x[i + 1], (c0 + i) / 2);
                        turn(y.x[i], y.x[i + 1], (c1 + i) / 2);
                    }
                }
            }
            if (h < H) {
                store4(qrow + (int64_t)h * D + c0, x, a.vec);
                store4(qrow + (int64_t)h * D + c1, y, a.vec);
            } else if (id >= 0) {
                const int g = h < H + KV ? h - H : h - H - KV;
                if constexpr (kExact) {
                    float *o = stage + (k * lanes + lane) * D;
                    store4(o + c0, x, true);
                    store4(o + c1, y, true);
                } else {
                    T *o = static_cast<T *>(h < H + KV ? kv.c.k : kv.c.v) + kv.element(id, g, off);
                    put4(o + c0, x);
                    put4(o + c1, y);
                }
                if (u == 0 && h < H + KV) {
                    if (kv.c.position) kv.c.position[kv.mark(id, g, off)] = a.index[t];
                    if (kv.c.weight) kv.c.weight[kv.mark(id, g, off)] = 0.0f;
                }
            }
        }
        const int round = base;
        load(base + kRound * lanes + lane);
        if constexpr (kExact) {
            if (id < 0 || min(last, round + kRound * lanes) <= H) continue;   // the block's
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kRound; ++k) {
                const int r = k * lanes + lane, h = round + r;
                const bool row = in && h >= H && h < last;
                float y[8];
                if (row) {
                    const Load4 p = load4(stage + r * D + 8 * u, true), q = load4(stage + r * D + 8 * u + 4, true);
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = p.x[i], y[4 + i] = q.x[i];
                }
                uint32_t codes;
                const uint32_t scales = q4_pack(y, codes);
                if (row) {
                    const int g = h < H + KV ? h - H : h - H - KV;
                    char *o = static_cast<char *>(h < H + KV ? kv.c.k : kv.c.v) + kv.element(id, g, off);
                    *reinterpret_cast<uint32_t *>(o + 4 * u) = codes;
                    if (u % 4 == 0) *reinterpret_cast<uint32_t *>(o + D / 2 + u) = scales;
                }
            }
            __syncthreads();
        }
    }
}

}  // namespace

mosaic_status append_norm_launch(const mosaic_kv_cache &c, AppendArgs a, const mosaic_head_norm *norm, cudaStream_t st) {
    const KvView kv(c);
    NormArgs nm = {};
    if (norm) nm.on = 1, nm.eps = norm->eps, nm.q_gain = norm->q_gain, nm.k_gain = norm->k_gain;
    nm.over_dim = two(1.0 / kv.c.head_dim);
    int pu = 1;
    while (pu < kv.c.head_dim / 8) pu *= 2;
    const dim3 grid = append_grid(kv.c, a, kThreads / pu);
    {
        KernelSpan span("append_norm", st);
        if (kv.c.type == MOSAIC_KV_F32) append_norm_kernel<float><<<grid, kThreads, 0, st>>>(kv, a, nm);
        else if (kv.c.type == MOSAIC_KV_BF16) append_norm_kernel<__nv_bfloat16><<<grid, kThreads, 0, st>>>(kv, a, nm);
        else if (kv.c.type == MOSAIC_KV_F16) append_norm_kernel<__half><<<grid, kThreads, 0, st>>>(kv, a, nm);
        else append_norm_kernel<Q4><<<grid, kThreads, 0, st>>>(kv, a, nm);
    }
    return launch_status();
}

}  // namespace mosaic
